"""Rows sorted by expert without a cast and the gradient of the weighted return, against the oracle (GPU)."""

import numpy as np
import pytest
import torch

from oracle import moe
from paper_2511_02302_amd import ff8

from test_gpu_kernels import f64, host, poisoned, untouched

pytestmark = pytest.mark.gpu

# T, H, E, k, align, fraction of dropped slots
CASES = [(1, 128, 1, 1, 128, 0.0), (1, 256, 8, 8, 16, 0.0), (7, 2048, 64, 6, 16, 0.1), (300, 384, 6, 2, 32, 0.5),
         (517, 1408, 64, 6, 16, 0.05), (1024, 256, 8, 2, 128, 0.0), (257, 128, 1024, 3, 64, 0.0),
         (64, 16384, 2, 2, 128, 0.0), (60, 8320, 5, 5, 16, 0.3), (130, 256, 64, 64, 16, 0.1), (5, 128, 4, 2, 16, 1.0),
         # routing by chunks of 256 tokens, in the rows' launch and in launches of its own
         (700, 256, 40, 7, 16, 0.1), (3000, 128, 24, 13, 128, 0.05), (600, 128, 1000, 10, 16, 0.0),
         (257, 128, 513, 33, 64, 0.3), (9000, 128, 16, 8, 32, 0.1), (1800, 128, 1024, 9, 16, 0.2)]


def _idx(T, E, k, dropped, seed=0):
    rng = np.random.default_rng(seed)
    p = rng.random(E) ** 3 + 1e-6
    idx = np.stack([rng.choice(E, size=k, replace=False, p=p / p.sum()) for _ in range(T)]).astype(np.int32)
    idx[rng.random((T, k)) < dropped] = -1
    return idx


def _buffers(T, k, E, align):
    M_cap = ff8.ff8_rows_bound_aligned(T, k, E, align)
    ws = torch.empty(max(1, ff8.ff8_permute_workspace_bytes(T, k, E)), dtype=torch.uint8, device="cuda")
    return M_cap, poisoned((T, k), torch.int32), poisoned((E + 1,), torch.int32), poisoned((M_cap,), torch.int32), ws


def _bf16(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _same_maps(maps, want, M_cap):
    row_map, offsets, src_row = maps
    _, w_off, w_map, w_src = want
    m = int(w_off[-1])
    assert np.array_equal(host(offsets), w_off) and np.array_equal(host(row_map), w_map)
    assert np.array_equal(host(src_row[:m]), w_src) and untouched(src_row[m:])


@pytest.mark.parametrize("T,H,E,k,align,dropped", CASES)
def test_permute_bf16(T, H, E, k, align, dropped):
    idx, x = _idx(T, E, k, dropped), _bf16((T, H), 1)
    x.view(-1)[:3] = torch.tensor([float("nan"), float("inf"), -0.0], dtype=torch.bfloat16)  # moved as they are
    want = moe.route(idx, E, align)
    m, src = int(want[1][-1]), want[3]
    rows = np.where(src[:, None] >= 0, x.view(torch.int16).numpy()[np.maximum(src, 0) // k], 0)
    M_cap, row_map, offsets, src_row, ws = _buffers(T, k, E, align)
    out = poisoned((M_cap, H), torch.bfloat16)
    xd, di = x.cuda(), torch.from_numpy(idx).cuda()
    ff8.ff8_permute_bf16(xd, k, E, di, False, row_map, offsets, src_row, out, ws, align=align)
    torch.cuda.synchronize()
    _same_maps((row_map, offsets, src_row), want, M_cap)
    assert np.array_equal(host(out[:m].view(torch.int16)), rows) and untouched(out[m:])
    # with the maps of an earlier call, and the maps alone
    again = poisoned((M_cap, H), torch.bfloat16)
    ff8.ff8_permute_bf16(xd, k, E, None, True, row_map, offsets, src_row, again, align=align)
    _, rm, off, src2, ws = _buffers(T, k, E, align)
    ff8.ff8_route(di, E, rm, off, src2, ws, align=align)
    torch.cuda.synchronize()
    _same_maps((rm, off, src2), want, M_cap)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("fmt", ["f32", "e8m0"])
@pytest.mark.parametrize("T,H,E,k,align,dropped", CASES)
def test_permute_fp8_is_permute_quant_of_the_same_rows(T, H, E, k, align, dropped, fmt):
    idx, x = torch.from_numpy(_idx(T, E, k, dropped)).cuda(), _bf16((T, H), 2).cuda()
    sdt = torch.float32 if fmt == "f32" else torch.uint8
    xq, xs = poisoned((T, H), torch.uint8), poisoned((T, H // 128), sdt)
    ff8.ff8_quant_rowwise(x, xq, xs)
    got, want = [], []
    for out in (got, want):
        M_cap, row_map, offsets, src_row, ws = _buffers(T, k, E, align)
        q, s = poisoned((M_cap, H), torch.uint8), poisoned((M_cap, H // 128), sdt)
        if out is got:
            ff8.ff8_permute_fp8(xq, xs, k, E, idx, False, row_map, offsets, src_row, q, s, ws, align=align)
        else:
            ff8.ff8_permute_quant(x, None, k, E, idx, False, row_map, offsets, src_row, q, s, ws, align=align)
        out += [row_map, offsets, src_row, q, s]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _return_bwd(T, H, E, k, align, dropped, with_dprobs):
    idx = _idx(T, E, k, dropped)
    want = moe.route(idx, E, align)
    M_cap, row_map, offsets, src_row, ws = _buffers(T, k, E, align)
    ff8.ff8_route(torch.from_numpy(idx).cuda(), E, row_map, offsets, src_row, ws, align=align)
    dy, w = _bf16((T, H), 3), torch.rand((T, k), generator=torch.Generator().manual_seed(4))
    w[torch.from_numpy(idx) < 0] = float("nan")  # what stands beside a dropped slot is not read
    yp = _bf16((M_cap, H), 5)
    yp[int(want[1][-1]):] = float("nan")
    yp[:len(want[3])][torch.from_numpy(want[3]) < 0] = float("nan")
    dyp = poisoned((M_cap, H), torch.bfloat16)
    dp = poisoned((T, k), torch.float32) if with_dprobs else None
    ff8.ff8_unpermute_bwd(dy.cuda(), w.cuda(), k, E, row_map, offsets, src_row, dyp, yp.cuda() if with_dprobs else None,
                          dp)
    torch.cuda.synchronize()
    return want, dy, w, yp, dyp, dp


@pytest.mark.parametrize("with_dprobs", [True, False])
@pytest.mark.parametrize("T,H,E,k,align,dropped", CASES)
def test_unpermute_bwd(T, H, E, k, align, dropped, with_dprobs):
    (_, off, row_map, src), dy, w, yp, dyp, dp = _return_bwd(T, H, E, k, align, dropped, with_dprobs)
    m = int(off[-1])
    # one float32 product, rounded to bf16: the same as torch's
    rows = torch.zeros((m, H), dtype=torch.bfloat16)
    real = torch.from_numpy(src >= 0)
    s = torch.from_numpy(src)[real]
    rows[real] = (w.reshape(-1)[s][:, None] * dy[s // k].float()).to(torch.bfloat16)
    assert np.array_equal(host(dyp[:m].view(torch.int16)), rows.view(torch.int16).numpy()) and untouched(dyp[m:])
    if not with_dprobs:
        return
    kept = row_map >= 0
    d, y = f64(dy)[:, None, :], np.where(kept[..., None], f64(yp)[np.maximum(row_map, 0)], 0.0)
    exact, size = (d * y).sum(2), (np.abs(d) * np.abs(y)).sum(2)
    # products are exact in float32; a lane adds at most H / 64 of them, then 6 steps and 8 waves
    assert np.all(np.abs(f64(dp) - exact) <= (H / 64 + 14) * 2.0 ** -24 * size)
    assert (f64(dp)[~kept] == 0).all()


def test_gradient_of_the_return_against_differences():
    """<unpermute(y_perm; w + h v) - unpermute(.; w - h v), dy> / 2h in float64 is <dprobs, v>."""
    T, H, E, k = 40, 256, 4, 2
    (_, off, row_map, src), dy, w, yp, dyp, dp = _return_bwd(T, H, E, k, 16, 0.1, True)
    v = np.random.default_rng(0).normal(size=(T, k))
    kept = row_map >= 0
    y = np.where(kept[..., None], f64(yp)[np.maximum(row_map, 0)], 0.0)
    f = lambda ww: (np.where(kept, ww, 0.0)[..., None] * y).sum(1)  # noqa: E731
    w64 = np.nan_to_num(w.double().numpy())
    num = ((f(w64 + 0.5 * v) - f(w64 - 0.5 * v)) * f64(dy)).sum()  # linear in w: any step is exact
    assert abs(num - (f64(dp) * v)[kept].sum()) <= 20 * 2.0 ** -24 * (np.abs(y) * np.abs(f64(dy))[:, None]).sum() * np.abs(v).max()
    # and in y_perm: <dy_perm, u> = <dy, unpermute(u; w)>, each element of dy_perm rounded by half a step
    u = np.random.default_rng(1).normal(size=y.shape)
    m = int(off[-1])
    got = (np.where(kept[..., None], f64(dyp[:m])[np.maximum(row_map, 0)], 0.0) * u).sum()
    terms = np.where(kept, w64, 0.0)[..., None] * f64(dy)[:, None] * u
    assert abs(got - terms.sum()) <= (2.0 ** -8 + 2.0 ** -24) * np.abs(terms).sum()


def test_empty_batch():
    E, k, H = 4, 2, 256
    M_cap = ff8.ff8_rows_bound_aligned(0, k, E, 16)
    i32 = lambda *s: poisoned(s, torch.int32)  # noqa: E731
    x = torch.empty((0, H), dtype=torch.bfloat16, device="cuda")
    row_map, offsets, src_row, out = i32(0, k), i32(E + 1), i32(M_cap), poisoned((M_cap, H), torch.bfloat16)
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    ff8.ff8_permute_bf16(x, k, E, i32(0, k), False, row_map, offsets, src_row, out, ws, align=16)
    ff8.ff8_unpermute_bwd(x, torch.empty((0, k), device="cuda"), k, E, row_map, offsets, src_row, out)
    torch.cuda.synchronize()
    assert host(offsets).tolist() == [0] * (E + 1) and untouched(out) and untouched(src_row)


def test_large_offsets():
    """Rows whose byte offset passes 32 bits: 300 000 rows of 8192 columns (4.9 GB)."""
    T, H, E, k = 300000, 8192, 2, 1
    idx = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    idx[::3] = 1
    x = torch.randn((T, 1), device="cuda").to(torch.bfloat16).expand(T, H).contiguous()
    M_cap, row_map, offsets, src_row, ws = _buffers(T, k, E, 16)
    out = torch.empty((M_cap, H), dtype=torch.bfloat16, device="cuda")
    ff8.ff8_permute_bf16(x, k, E, idx, False, row_map, offsets, src_row, out, ws, align=16)
    w = torch.full((T, k), 2.0, device="cuda")
    back = torch.empty((M_cap, H), dtype=torch.bfloat16, device="cuda")
    dp = torch.empty((T, k), device="cuda")
    ff8.ff8_unpermute_bwd(x, w, k, E, row_map, offsets, src_row, back, out, dp)
    torch.cuda.synchronize()
    rows = row_map.reshape(-1).long()
    for col in (0, H - 1):
        assert torch.equal(out[rows, col], x[:, col]) and torch.equal(back[rows, col], 2 * x[:, col])
    # 8192 equal squares: sums of powers of two of them are exact
    assert torch.equal(dp[:, 0], x[:, 0].float().square() * H)
