// Host side of the forms that the row sorts and the 4-bit products take by their sizes, for test_operator_forms.py.
#include "mxfp4_rule.hpp"
#include "rows_rule.hpp"

extern "C" int sort_form(int64_t T, int k, int E, int64_t row16) {
  return (int)ff8::sort_form(T * k, (T + ff8::kRouteChunk - 1) / ff8::kRouteChunk * E, row16);
}
extern "C" int sort_narrow(int64_t row16) { return ff8::narrow_rows(row16); }
// 1: blocks of up to 96 rows; otherwise the waves of a 16-row workgroup, negative where its weights are kept.
extern "C" int mxfp4_form(int64_t x_rows, int top_k, int64_t M_cap, int E, int64_t N, int64_t K, int swiglu, int64_t cus) {
  const ff8::Mxfp4Form f = ff8::mxfp4_form(x_rows, top_k, M_cap, E, N, K, swiglu != 0, cus);
  return f.many ? 1 : f.keep ? -f.waves : f.waves;
}
