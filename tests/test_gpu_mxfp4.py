"""MXFP4 weights: quantization, tile order and the grouped products, against the oracle (GPU)."""

import numpy as np
import pytest
import torch

from oracle import moe, mxfp4
from paper_2511_02302_amd import ff8

from test_gpu_kernels import f64, host, poisoned, untouched

pytestmark = pytest.mark.gpu


def _bf16(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(torch.bfloat16)


@pytest.mark.parametrize("rows,cols", [(1, 128), (3, 256), (128, 1408), (257, 7168)])
def test_quant(rows, cols):
    w = _bf16((rows, cols), rows, 0.02)
    w.view(-1)[:32] = 0.0
    w.view(-1)[5] = -0.0
    w.view(-1)[32:64] = torch.tensor([6.0 * 2.0 ** -126] + [2.0 ** -133] * 31, dtype=torch.bfloat16)
    w.view(-1)[64:96] = torch.tensor([3.0e38] * 16 + [-1.0] * 16, dtype=torch.bfloat16)
    if cols > 128:  # every tie of the grid, both signs, at a scale of 1 and at its border
        ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.26, 0.74, 1.26, 1.74, 2.52, 3.48, 5.03, 4.97])
        w.view(-1)[96:128] = torch.cat([ties, -ties]).to(torch.bfloat16)
        w.view(-1)[128:160] = torch.cat([ties * 2.0 ** -20, torch.full((16,), 6.03125 * 2.0 ** -20)]).to(torch.bfloat16)
    q, s = poisoned((rows, cols // 2), torch.uint8), poisoned((rows, cols // 32), torch.uint8)
    ff8.ff8_quant_mxfp4(w.cuda(), q, s)
    torch.cuda.synchronize()
    wq, ws = mxfp4.quant(f64(w))
    assert np.array_equal(host(s), ws) and np.array_equal(host(q), wq)


@pytest.mark.parametrize("E,N,K", [(1, 128, 128), (3, 256, 384), (2, 1408, 2048)])
def test_pack(E, N, K):
    g = torch.Generator().manual_seed(N)
    q = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8)
    s = torch.randint(0, 256, (E, N, K // 32), generator=g, dtype=torch.uint8)
    tq, ts = poisoned((E, N // 16, K // 128, 64, 16), torch.uint8), poisoned((E, N // 32, K // 128, 64, 2), torch.uint8)
    ff8.ff8_pack_mxfp4(q.cuda(), s.cuda(), tq, ts)
    torch.cuda.synchronize()
    for e in range(E):
        wq, ws = mxfp4.pack(q[e].numpy(), s[e].numpy())
        assert np.array_equal(host(tq[e]), wq) and np.array_equal(host(ts[e]), ws)


def _weights(E, N, K, seed, lo=119, hi=122):
    """Row-major codes and scales, their values, and the packed device tensors."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8)
    s = torch.randint(lo, hi, (E, N, K // 32), generator=g, dtype=torch.uint8)
    tq = torch.empty((E, N // 16, K // 128, 64, 16), dtype=torch.uint8, device="cuda")
    ts = torch.empty((E, N // 32, K // 128, 64, 2), dtype=torch.uint8, device="cuda")
    ff8.ff8_pack_mxfp4(q.cuda(), s.cuda(), tq, ts)
    return [mxfp4.dequant(q[e].numpy(), s[e].numpy()) for e in range(E)], tq, ts


def _groups(counts, align, T=None, k=1, seed=0, extra=0):
    """offsets, src_row and M_cap of groups with so many real rows each; tokens drawn at random."""
    rng = np.random.default_rng(seed)
    sizes = [-(-c // align) * align for c in counts]
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    M_cap = max(128, -(-(int(offsets[-1]) + extra) // 128) * 128)
    src = np.full(M_cap, -1, dtype=np.int32)
    for e, c in enumerate(counts):
        pairs = np.arange(c) if T is None else np.sort(rng.choice(T * k, size=c, replace=False))
        src[offsets[e]:offsets[e] + c] = pairs
    src[offsets[-1]:] = 0x6BCDEF  # behind the last group anything may stand
    return offsets, src, M_cap


def _bound(x, w, offsets):
    """Bound on the float32 sums' errors.  Products are exact; a product goes through the additions of its matrix
    instruction (at most 8 in a row) and of at most K / 32 instructions and 8 waves, each of one unit (2^-23) at
    most of the sum of magnitudes."""
    K = x.shape[1]
    return (K / 32 + 16) * 2.0 ** -23 * moe_product(np.abs(x), [np.abs(v) for v in w], offsets)


def moe_product(x, w, offsets):
    return mxfp4.grouped_product(x, w, offsets)


def _check_rows(out, want, tol, offsets, src):
    m = int(offsets[-1])
    got = f64(out[:m])
    real = src[:m] >= 0
    assert np.all(np.abs(got - want)[real] <= (2.0 ** -8 * np.abs(want) + tol)[real])
    assert (got[~real] == 0).all() and untouched(out[m:])


COUNTS = [([1], 16), ([0, 1, 0], 16), ([5, 0, 17, 16, 1], 16), ([33, 2, 64, 65, 0, 15], 16), ([130, 1, 200], 128),
          ([300, 48, 31], 32), ([0, 0], 16)]
SIZES = [(128, 128), (256, 256), (384, 1408), (1408, 2048), (128, 7168)]


@pytest.mark.parametrize("counts,align", COUNTS)
@pytest.mark.parametrize("N,K", SIZES)
def test_product_of_grouped_rows(counts, align, N, K):
    E = len(counts)
    w, tq, ts = _weights(E, N, K, N + K)
    offsets, src, M_cap = _groups(counts, align)
    x = _bf16((M_cap, K), 1)
    x[torch.from_numpy(src < 0)] = float("nan")  # padding rows are not read
    x[int(offsets[-1]):] = float("nan")
    out = poisoned((M_cap, N), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                               src_row=torch.from_numpy(src).cuda())
    torch.cuda.synchronize()
    xs = np.nan_to_num(f64(x))
    _check_rows(out, moe_product(xs, w, offsets), _bound(xs, w, offsets), offsets, src)
    # without src_row every row below offsets[E] holds data
    y = torch.nan_to_num(x)
    out2 = poisoned((M_cap, N), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(y.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out2)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), out2.view(torch.int16))


def _swiglu_check(out, x, w, offsets, src, I):
    a, t = moe_product(x, w, offsets), _bound(x, w, offsets)
    g, u, tg, tu = a[:, :I], a[:, I:], t[:, :I], t[:, I:]
    sig = 1.0 / (1.0 + np.exp(-g))
    h = g * sig * u
    # |d silu| <= 1.1 |dg|; expf, the division and two products: at most 8 half-units
    tol = 1.1 * tg * (np.abs(u) + tu) + np.abs(g * sig) * tu + 8 * 2.0 ** -24 * np.abs(h)
    _check_rows(out, h, (1 + 2.0 ** -8) * tol, offsets, src)


@pytest.mark.parametrize("counts,align", COUNTS)
@pytest.mark.parametrize("I,K,T,k", [(128, 256, 400, 3), (256, 2048, 301, 2), (704 // 128 * 128, 1408, 300, 1)])
def test_swiglu_of_gathered_tokens(counts, align, I, K, T, k):
    E = len(counts)
    w, tq, ts = _weights(E, 2 * I, K, I + K)
    offsets, src, M_cap = _groups(counts, align, T, k, seed=2, extra=200)
    x = _bf16((T, K), 3)
    out = poisoned((M_cap, I), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4_swiglu(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                                      src_row=torch.from_numpy(src).cuda(), top_k=k)
    torch.cuda.synchronize()
    m = int(offsets[-1])
    xs = np.where(src[:m, None] >= 0, f64(x)[np.maximum(src[:m], 0) // k], 0.0)
    _swiglu_check(out, xs, w, offsets, src, I)


# experts with many rows beside some with few and none: enough of them for the form with 96-row blocks
MANY = [0, 1, 5, 16, 17, 40, 64, 79, 80, 96, 97, 130, 200, 33, 0, 12]


@pytest.mark.parametrize("N,K,align,copies", [(640, 128, 16, 8), (1408, 384, 16, 4), (256, 1408, 128, 14), (2048, 640, 32, 3)])
def test_many_rows_product(N, K, align, copies):
    counts = MANY * copies
    E = len(counts)
    w, tq, ts = _weights(E, N, K, N + K)
    offsets, src, M_cap = _groups(counts, align, seed=1, extra=300)
    x = _bf16((M_cap, K), 1)
    x[torch.from_numpy((src < 0) | (np.arange(M_cap) >= offsets[-1]))] = float("nan")  # not read
    out = poisoned((M_cap, N), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                               src_row=torch.from_numpy(src).cuda())
    torch.cuda.synchronize()
    xs = np.nan_to_num(f64(x))
    _check_rows(out, moe_product(xs, w, offsets), _bound(xs, w, offsets), offsets, src)


@pytest.mark.parametrize("I,K,T,k,align,copies", [(384, 256, 250, 3, 16, 4), (128, 896, 400, 2, 16, 12), (1408, 128, 201, 1, 64, 2)])
def test_many_rows_swiglu_of_gathered_tokens(I, K, T, k, align, copies):
    counts = MANY * copies
    E = len(counts)
    w, tq, ts = _weights(E, 2 * I, K, I + K)
    offsets, src, M_cap = _groups(counts, align, T, k, seed=2, extra=200)
    T_all = max(T, 12 * E // k + 1)  # more tokens in x than any row takes: what counts for the form is their number
    x = _bf16((T_all, K), 3)
    out = poisoned((M_cap, I), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4_swiglu(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                                      src_row=torch.from_numpy(src).cuda(), top_k=k)
    torch.cuda.synchronize()
    m = int(offsets[-1])
    xs = np.where(src[:m, None] >= 0, f64(x)[np.maximum(src[:m], 0) // k], 0.0)
    _swiglu_check(out, xs, w, offsets, src, I)


def test_source_rows_out_of_range_give_zeros():
    w, tq, ts = _weights(1, 128, 256, 0)
    offsets, src, M_cap = _groups([16], 16)
    src[:16] = [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10 ** 9, 2 ** 31 - 1, 10, -1, -7, 9]
    x = _bf16((10, 256), 0)
    out = poisoned((M_cap, 128), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                               src_row=torch.from_numpy(src).cuda(), top_k=1)
    torch.cuda.synchronize()
    got = f64(out[:16])
    assert (got[10:15] == 0).all() and np.array_equal(got[15], got[9]) and (np.abs(got[:10]).sum(1) > 0).all()


def test_extreme_scales_and_values():
    """UE8M0 bytes 0 (2^-127: subnormal weights) to 253 at codes that stay finite, x at bf16's ends."""
    N = K = 128
    for byte, code, xv in ((0, 1, 1.0), (0, 7, 2.0 ** 100), (1, 1, 2.0 ** 120), (253, 1, 2.0 ** -100), (252, 7, 2.0 ** -126),
                           (127, 7, 2.0 ** -133)):
        q = torch.full((1, N, K // 2), code * 17, dtype=torch.uint8)
        s = torch.full((1, N, K // 32), byte, dtype=torch.uint8)
        tq, ts = torch.empty((1, N // 16, 1, 64, 16), dtype=torch.uint8, device="cuda"), torch.empty((1, N // 32, 1, 64, 2), dtype=torch.uint8, device="cuda")
        ff8.ff8_pack_mxfp4(q.cuda(), s.cuda(), tq, ts)
        offsets, src, M_cap = _groups([3], 16)
        x = torch.full((M_cap, K), xv, dtype=torch.bfloat16)
        out = poisoned((M_cap, N), torch.bfloat16)
        ff8.ff8_grouped_gemv_mxfp4(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out, src_row=torch.from_numpy(src).cuda())
        torch.cuda.synchronize()
        want = K * float(mxfp4.E2M1[code]) * 2.0 ** (byte - 127) * xv  # powers of two times 0.5 or 6: exact
        assert (f64(out[:3]) == float(torch.tensor(want, dtype=torch.bfloat16))).all(), (byte, code, xv)


def test_scale_of_nan_reaches_its_rows_alone():
    E, N, K = 1, 128, 256
    g = torch.Generator().manual_seed(0)
    q = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8)
    s = torch.full((E, N, K // 32), 120, dtype=torch.uint8)
    s[0, 37, 3] = 255
    tq, ts = torch.empty((E, N // 16, K // 128, 64, 16), dtype=torch.uint8, device="cuda"), torch.empty((E, N // 32, K // 128, 64, 2), dtype=torch.uint8, device="cuda")
    ff8.ff8_pack_mxfp4(q.cuda(), s.cuda(), tq, ts)
    offsets, src, M_cap = _groups([20], 16)
    out = poisoned((M_cap, N), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(_bf16((M_cap, K), 1).cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                               src_row=torch.from_numpy(src).cuda())
    torch.cuda.synchronize()
    nan = np.isnan(f64(out[:20]))
    assert nan[:, 37].all() and nan.sum() == 20


def test_infinite_and_nan_tokens_stay_in_their_rows():
    w, tq, ts = _weights(1, 128, 512, 3)
    offsets, src, M_cap = _groups([40], 16)
    x = _bf16((M_cap, 512), 1)
    clean = poisoned((M_cap, 128), torch.bfloat16)
    args = (tq, ts, torch.from_numpy(offsets).cuda())
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), *args, clean, src_row=torch.from_numpy(src).cuda())
    x[7, 3], x[20, 100] = float("nan"), float("inf")
    out = poisoned((M_cap, 128), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), *args, out, src_row=torch.from_numpy(src).cuda())
    torch.cuda.synchronize()
    keep = np.ones(40, dtype=bool)
    keep[[7, 20]] = False
    assert np.isnan(f64(out[7])).all() and not np.isfinite(f64(out[20])).all()
    assert np.array_equal(f64(out[:40])[keep], f64(clean[:40])[keep])


def test_many_experts_few_rows():
    """1024 experts, one token each but for some that have none."""
    E, N, K, T = 1024, 128, 128, 700
    w, tq, ts = _weights(E, N, K, 9)
    counts = [1 if e % 3 else 0 for e in range(E)]
    offsets, src, M_cap = _groups(counts, 16, T, 1, seed=4)
    x = _bf16((T, K), 5)
    out = poisoned((M_cap, N), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), tq, ts, torch.from_numpy(offsets).cuda(), out,
                               src_row=torch.from_numpy(src).cuda(), top_k=1)
    torch.cuda.synchronize()
    m = int(offsets[-1])
    xs = np.where(src[:m, None] >= 0, f64(x)[np.maximum(src[:m], 0)], 0.0)
    _check_rows(out, moe_product(xs, w, offsets), _bound(xs, w, offsets), offsets, src)


def test_weights_past_four_gigabytes():
    """Tile offsets past 32 bits: 18 experts of 4096 x 131072 codes (4.8 GB); the last expert's rows."""
    E, N, K = 18, 4096, 131072
    tq = torch.zeros((E, N // 16, K // 128, 64, 16), dtype=torch.uint8, device="cuda")
    ts = torch.full((E, N // 32, K // 128, 64, 2), 127, dtype=torch.uint8, device="cuda")
    tq[E - 1, :, -1] = 0x22  # ones in the last 128 columns
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[E] = 16
    x = torch.zeros((128, K), dtype=torch.bfloat16, device="cuda")
    x[:16, -128:] = torch.arange(16, device="cuda")[:, None].to(torch.bfloat16)
    out = poisoned((128, N), torch.bfloat16)
    ff8.ff8_grouped_gemv_mxfp4(x, tq, ts, offsets, out)
    torch.cuda.synchronize()
    assert torch.equal(out[:16].float(), (128.0 * torch.arange(16, device="cuda"))[:, None].expand(16, N))


def test_repeatable_and_on_another_stream():
    w, tq, ts = _weights(4, 256, 1408, 1)
    offsets, src, M_cap = _groups([30, 0, 7, 100], 16, 200, 2, seed=1)
    x, off, sr = _bf16((200, 1408), 2).cuda(), torch.from_numpy(offsets).cuda(), torch.from_numpy(src).cuda()
    outs = [poisoned((M_cap, 128), torch.bfloat16) for _ in range(3)]
    torch.cuda.synchronize()
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream()]
    for o, st in zip(outs, streams):  # side by side: calls share nothing but their inputs
        ff8.ff8_grouped_gemv_mxfp4_swiglu(x, tq, ts, off, o, src_row=sr, top_k=2, stream=st)
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o.view(torch.int16), outs[0].view(torch.int16))
