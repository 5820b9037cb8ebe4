"""The kernels' forms that no other size reaches, each against the oracle (GPU).  test_operator_forms.py checks on
the host that the sizes here and beside it do reach them."""

import numpy as np
import pytest
import torch

from oracle import moe
from paper_2511_02302_amd import ff8

import test_gpu_rows as rows
from test_gpu_kernels import f64, host, poisoned

pytestmark = pytest.mark.gpu

# T, H, E, k, align, fraction of dropped slots
SORTS = [(700, 1152, 40, 7, 16, 0.1), (1031, 2048, 24, 5, 128, 0.05), (601, 4096, 600, 9, 16, 0.2),  # wide, counted
         (257, 7168, 32, 17, 32, 0.0),
         (3101, 1152, 1024, 5, 16, 0.1), (12289, 2048, 8, 4, 128, 0.02),  # wide, with the routing in front
         (3101, 256, 1024, 5, 16, 0.0)]                                   # narrow, the same


@pytest.mark.parametrize("T,H,E,k,align,dropped", SORTS)
def test_sort_bf16(T, H, E, k, align, dropped):
    rows.test_permute_bf16(T, H, E, k, align, dropped)


@pytest.mark.parametrize("fmt", ["f32", "e8m0"])
@pytest.mark.parametrize("T,H,E,k,align,dropped", SORTS)
def test_sort_fp8(T, H, E, k, align, dropped, fmt):
    rows.test_permute_fp8_is_permute_quant_of_the_same_rows(T, H, E, k, align, dropped, fmt)


@pytest.mark.parametrize("fmt", ["f32", "e8m0"])
@pytest.mark.parametrize("H", [128, 1024, 1152, 4096])
def test_sort_fp8_by_maps_that_are_there(H, fmt):
    T, E, k, align = 301, 12, 3, 32
    idx, x = rows._idx(T, E, k, 0.2), rows._bf16((T, H), 3).cuda()
    sdt = torch.float32 if fmt == "f32" else torch.uint8
    xq, xs = poisoned((T, H), torch.uint8), poisoned((T, H // 128), sdt)
    ff8.ff8_quant_rowwise(x, xq, xs)
    M_cap, row_map, offsets, src_row, ws = rows._buffers(T, k, E, align)
    ff8.ff8_route(torch.from_numpy(idx).cuda(), E, row_map, offsets, src_row, ws, align=align)
    q, s = poisoned((M_cap, H), torch.uint8), poisoned((M_cap, H // 128), sdt)
    ff8.ff8_permute_fp8(xq, xs, k, E, None, True, row_map, offsets, src_row, q, s, align=align)
    torch.cuda.synchronize()
    want = moe.route(idx, E, align)
    rows._same_maps((row_map, offsets, src_row), want, M_cap)
    m, src = int(want[1][-1]), want[3]
    zero = 1 if fmt == "e8m0" else 2.0 ** -126  # the scale of a row of zeros
    take = np.maximum(src, 0) // k
    assert np.array_equal(host(q[:m]), np.where(src[:, None] >= 0, host(xq)[take], 0)) and rows.untouched(q[m:])
    assert np.array_equal(host(s[:m]), np.where(src[:, None] >= 0, host(xs)[take], np.asarray(zero, host(xs).dtype)))
    assert rows.untouched(s[m:])


@pytest.mark.parametrize("H", [128, 256, 512, 640, 1024, 4096, 7168])
def test_return_dot_products(H):
    """The routing weights' gradient within what its sums can round.  Products are exact in float32.  A lane adds
    8 of them for every 512 columns (the first to zero), then at most 6 sums meet across the lanes, each addition
    off by half a step: 8 ceil(H / 512) + 5, and one more for the products of those errors."""
    (_, off, row_map, src), dy, w, yp, dyp, dp = rows._return_bwd(517, H, 20, 3, 16, 0.1, True)
    kept = row_map >= 0
    d, y = f64(dy)[:, None, :], np.where(kept[..., None], f64(yp)[np.maximum(row_map, 0)], 0.0)
    exact, size = (d * y).sum(2), (np.abs(d) * np.abs(y)).sum(2)
    assert np.all(np.abs(f64(dp) - exact) <= (8 * -(-H // 512) + 6) * 2.0 ** -24 * size)
    assert (f64(dp)[~kept] == 0).all()
