// Host side of the forms that the row sorts take by their sizes, for test_operator_forms.py.
#include "rows_rule.hpp"

extern "C" int sort_form(int64_t T, int k, int E, int64_t row16) {
  return (int)ff8::sort_form(T * k, (T + ff8::kRouteChunk - 1) / ff8::kRouteChunk * E, row16);
}
extern "C" int sort_narrow(int64_t row16) { return ff8::narrow_rows(row16); }
