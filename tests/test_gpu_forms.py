"""The kernels' forms that no other size reaches, each against the oracle (GPU).  test_operator_forms.py checks on
the host that the sizes here and beside it do reach them."""

import numpy as np
import pytest
import torch

from oracle import moe
from paper_2511_02302_amd import ff8

import test_gpu_mxfp4 as products
import test_gpu_router as gate
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


# SwiGLU, columns of out, K, align, real rows of the experts, form (as test_operator_forms.py numbers them)
_FEW = [1, 0, 4, 5, 0, 16, 0, 2, 0, 0, 3, 0] * 3
GROUPED = [(False, 640, 128, 16, products.MANY * 8, 1), (False, 1408, 384, 128, products.MANY * 4, 1),
           (True, 384, 256, 16, products.MANY * 5, 1), (True, 640, 1664, 32, products.MANY * 3, 1),
           (False, 384, 1536, 16, _FEW, 2), (True, 128, 1408, 16, _FEW, 2),
           (False, 256, 1664, 16, _FEW, 4), (True, 384, 2048, 16, _FEW, 4),
           (False, 128, 512, 16, [33, 17, 130], -2), (True, 256, 640, 128, [33, 0, 130], -2),
           (False, 128, 4096, 64, [20, 40, 100], -4), (True, 128, 1792, 16, [20, 41, 97], -4)]


@pytest.mark.parametrize("swiglu,n_out,K,align,counts,form", GROUPED)
def test_grouped_rows_with_and_without_their_sources(swiglu, n_out, K, align, counts, form):
    """Each form on grouped rows: padding skipped by src_row, or rows of zeros that are computed like any other."""
    N, E = (2 * n_out if swiglu else n_out), len(counts)
    w, tq, ts = products._weights(E, N, K, N + K)
    offsets, src, M_cap = products._groups(counts, align, seed=1, extra=200)
    pad = torch.from_numpy((src < 0) | (np.arange(M_cap) >= offsets[-1]))
    x = products._bf16((M_cap, K), 4)
    call = ff8.ff8_grouped_gemv_mxfp4_swiglu if swiglu else ff8.ff8_grouped_gemv_mxfp4
    outs = []
    for fill, sources in ((float("nan"), torch.from_numpy(src).cuda()), (0.0, None)):
        x[pad] = fill  # padding rows are not read with src_row; behind the last group nothing is
        x[int(offsets[-1]):] = float("nan")
        outs.append(poisoned((M_cap, n_out), torch.bfloat16))
        call(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), outs[-1], src_row=sources)
    torch.cuda.synchronize()
    xs = np.nan_to_num(f64(x))
    if swiglu:
        products._swiglu_check(outs[0], xs, w, offsets, src, n_out)
    else:
        products._check_rows(outs[0], products.moe_product(xs, w, offsets), products._bound(xs, w, offsets), offsets, src)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


# T, E, k, I, K, form: a decoding step's up projection
GATHERED = [(1, 32, 8, 128, 2048, 4), (1, 8, 2, 256, 7168, 4), (5, 40, 3, 256, 1664, 4), (9, 12, 6, 128, 4096, 4),
            (40, 32, 8, 128, 1792, 4), (4, 24, 5, 128, 1536, 2), (64, 4, 2, 128, 2048, -4), (33, 3, 3, 384, 896, -2),
            (100, 16, 4, 1408, 384, 1)]


@pytest.mark.parametrize("T,E,k,I,K,form", GATHERED)
def test_swiglu_of_a_decoding_step(T, E, k, I, K, form):
    idx = rows._idx(T, E, k, 0.0, seed=T)
    _, offsets, _, s = moe.route(idx, E, 16)
    M_cap = ff8.ff8_rows_bound_aligned(T, k, E, 16)
    src = np.full(M_cap, 0x6BCDEF, dtype=np.int32)  # behind the last group anything may stand
    src[:len(s)] = s
    w, tq, ts = products._weights(E, 2 * I, K, I + K)
    x = products._bf16((T, K), 6)
    out = poisoned((M_cap, I), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4_swiglu(x.cuda(), tq, ts, torch.from_numpy(np.asarray(offsets, np.int32)).cuda(), out,
                                      src_row=torch.from_numpy(src).cuda(), top_k=k)
    torch.cuda.synchronize()
    m = int(offsets[-1])
    xs = np.where(src[:m, None] >= 0, f64(x)[np.maximum(src[:m], 0) // k], 0.0)
    products._swiglu_check(out, xs, w, offsets, src, I)


# Tokens, experts and k of the router's forms that its own tests leave out: 33 to 64 experts by k <= 16 and 65 to
# 256 experts by k > 16, each with a bias and without; in bf16 also batches above 2048 tokens
ROUTERS = [(70, 24, 5), (65, 31, 7), (40, 50, 16), (41, 64, 8), (31, 65, 17), (20, 100, 40), (9, 128, 33), (30, 127, 64),
           (25, 129, 20), (12, 200, 64), (14, 255, 17), (17, 256, 32), (2060, 100, 6), (2050, 72, 4), (2049, 256, 3),
           (3, 96, 2), (5, 192, 5)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,normalize", gate.MODES)
def test_router(dtype, score, normalize, monkeypatch):
    for with_bias in (False, True):
        for n, (T, E, k) in enumerate(ROUTERS):
            bias = torch.randn(E, generator=torch.Generator().manual_seed(n)) * 0.3 if with_bias else None
            gate._check(gate._logits(T, E, dtype, 10 + n), bias, k, score, normalize)
    monkeypatch.setattr(gate, "SHAPES", ROUTERS)
    gate.test_backward(dtype, score, normalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,normalize", gate.MODES)
def test_router_of_infinite_logits(dtype, score, normalize):
    """+inf is the largest logit.  Softmax scores of its token are NaN, as inf - inf is: with a bias it chooses nothing.
    Sigmoid scores are 1.  A NaN logit leaves normalized weights of the others as they are."""
    for E, k in ((12, 3), (60, 8), (200, 8), (100, 20), (600, 4)):
        z = gate._logits(8, E, dtype, E)
        z[0, E - 2] = float("inf")
        z[1, [1, 5, E - 1]] = float("inf")
        z[2] = float("inf")
        z[3, 2], z[3, 3] = float("inf"), float("nan")
        z[4, 7] = float("nan")
        z[5, 0], z[5, 1] = float("inf"), -float("inf")
        for bias in (None, torch.linspace(-0.3, 0.3, E)):
            gate._check(z, bias, k, score, normalize)
