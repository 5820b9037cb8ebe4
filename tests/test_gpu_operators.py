"""The router, the row sorts, the weighted return's gradient and the 4-bit products together: captured and
replayed, on two streams at once, with padded batches, odd views and what the binding refuses (GPU)."""

import numpy as np
import pytest
import torch

from oracle import moe, mxfp4, router
from paper_2511_02302_amd import ff8
from paper_2511_02302_amd.layer import ExpertLayerFP4

from test_gpu_kernels import f64, host, poisoned, untouched

pytestmark = pytest.mark.gpu

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Chain:
    """Every operator once, from tokens and logits of T tokens to the logits' gradient, on buffers of its own (but
    for a workspace that may be shared)."""

    def __init__(self, T, H, E, k, I, dtype, bias, ws=None, align=16):
        self.dims = T, H, E, k, align
        M = ff8.ff8_rows_bound_aligned(T, k, E, align)
        n = lambda *s, dt=BF16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
        self.x, self.dy, self.z = n(T, H), n(T, H), n(T, E, dt=dtype)
        self.bias = n(E, dt=F32) if bias else None
        self.w = n(E, 2 * I, H)
        self.idx, self.p, self.rm = n(T, k, dt=I32), n(T, k, dt=F32), n(T, k, dt=I32)
        self.off, self.src = n(E + 1, dt=I32), n(M, dt=I32)
        self.rm2, self.off2, self.src2 = n(T, k, dt=I32), n(E + 1, dt=I32), n(M, dt=I32)
        self.ws = n(max(1, ff8.ff8_permute_workspace_bytes(T, k, E)), dt=U8) if ws is None else ws
        self.xq, self.xs = n(T, H, dt=U8), n(T, H // 128, dt=U8)
        self.q, self.s = n(M, H, dt=U8), n(M, H // 128, dt=U8)
        self.xp, self.dyp, self.dp, self.dz = n(M, H), n(M, H), n(T, k, dt=F32), n(T, E, dt=dtype)
        self.wq, self.wsc = n(E, 2 * I, H // 2, dt=U8), n(E, 2 * I, H // 32, dt=U8)
        self.tq, self.ts = n(E, 2 * I // 16, H // 128, 64, 16, dt=U8), n(E, 2 * I // 32, H // 128, 64, 2, dt=U8)
        self.h, self.a = n(M, I), n(M, 2 * I)

    def fill(self, seed):
        g = torch.Generator().manual_seed(seed)
        for t, std in ((self.x, 1.0), (self.dy, 1.0), (self.z, 2.0), (self.w, 0.05)):
            t.copy_((torch.randn(t.shape, generator=g) * std).to(t.dtype))
        if self.bias is not None:
            self.bias.copy_(torch.randn(self.bias.shape, generator=g) * 0.2)
        return self

    def run(self, stream=None):
        _, _, E, k, al = self.dims
        st = {"stream": stream}
        mode = {"score": "sigmoid", "normalize": True, "scale": 2.5, **st}
        ff8.ff8_router_topk(self.z, self.idx, self.p, bias=self.bias, **mode)
        ff8.ff8_permute_bf16(self.x, k, E, self.idx, False, self.rm, self.off, self.src, self.xp, self.ws, align=al, **st)
        ff8.ff8_quant_rowwise(self.x, self.xq, self.xs, **st)
        ff8.ff8_permute_fp8(self.xq, self.xs, k, E, None, True, self.rm, self.off, self.src, self.q, self.s, align=al, **st)
        ff8.ff8_route(self.idx, E, self.rm2, self.off2, self.src2, self.ws, align=al, **st)
        ff8.ff8_quant_mxfp4(self.w, self.wq, self.wsc, **st)
        ff8.ff8_pack_mxfp4(self.wq, self.wsc, self.tq, self.ts, **st)
        ff8.ff8_grouped_gemv_mxfp4_swiglu(self.x, self.tq, self.ts, self.off2, self.h, src_row=self.src2, top_k=k, **st)
        ff8.ff8_grouped_gemv_mxfp4(self.xp, self.tq, self.ts, self.off, self.a, src_row=self.src, **st)
        ff8.ff8_unpermute_bwd(self.dy, self.p, k, E, self.rm, self.off, self.src, self.dyp, self.xp, self.dp, **st)
        ff8.ff8_router_topk_bwd(self.z, self.idx, self.dp, self.dz, **mode)

    def results(self):
        m = int(self.off[-1])
        rows = [t[:m] for t in (self.src, self.src2, self.xp, self.dyp, self.q, self.s, self.h, self.a)]
        return [t.clone() for t in (self.idx, self.p, self.rm, self.off, self.rm2, self.off2, self.dp, self.dz, *rows)]


def _same(a, b):
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x, y), i


# a few rows of each expert (routing and rows in one launch, the 16-row products) and many (routing launches of its
# own, the 96-row products)
SMALL = (37, 256, 16, 4, 128, BF16, False)
LARGE = (1100, 384, 8, 4, 1408, F32, True)


def test_two_captured_chains_that_share_a_workspace():
    ws = torch.zeros(1 << 20, dtype=U8, device="cuda")
    chains, graphs = [Chain(*SMALL, ws=ws), Chain(*LARGE, ws=ws)], []
    assert ws.numel() >= max(ff8.ff8_permute_workspace_bytes(c.dims[0], c.dims[3], c.dims[2]) for c in chains)
    for c in chains:
        c.fill(0).run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    eager = [Chain(*SMALL), Chain(*LARGE)]
    for rep in range(4):
        for c, e in zip(chains, eager):
            c.fill(10 + rep)
            e.fill(10 + rep).run()
        torch.cuda.synchronize()
        for g in graphs if rep % 2 else graphs[::-1]:
            g.replay()  # one behind the other on one stream
        for e in eager:
            e.run()  # the program's own work beside the replays
        torch.cuda.synchronize()
        for c, e in zip(chains, eager):
            _same(c.results(), e.results())


def test_two_streams_at_once():
    want = []
    for i, c in enumerate((SMALL, LARGE)):
        c = Chain(*c).fill(i)
        c.run()
        torch.cuda.synchronize()
        want.append(c.results())
    both = [Chain(*SMALL).fill(0), Chain(*LARGE).fill(1)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(both, streams):
            c.run(s)
    torch.cuda.synchronize()
    for c, w in zip(both, want):
        _same(c.results(), w)


@pytest.mark.parametrize("T", [40, 1500])
def test_padded_batch(T):
    """Tokens behind the batch's end have no expert: their rows are nowhere, their outputs zero."""
    H, E, k, N = 256, 8, 2, 1024
    real = T - T // 4
    g = torch.Generator().manual_seed(T)
    x = torch.randn((T, H), generator=g).to(BF16)
    x[real:] = float("nan")
    z = torch.randn((T, E), generator=g)
    z[real:] = -float("inf")
    idx, p = poisoned((T, k), I32), poisoned((T, k), F32)
    ff8.ff8_router_topk(z.cuda(), idx, p, normalize=True)
    M = ff8.ff8_rows_bound_aligned(T, k, E, 128)
    rm, off, src, xp = poisoned((T, k), I32), poisoned((E + 1,), I32), poisoned((M,), I32), poisoned((M, H), BF16)
    ws = torch.empty(max(1, ff8.ff8_permute_workspace_bytes(T, k, E)), dtype=U8, device="cuda")
    ff8.ff8_permute_bf16(x.cuda(), k, E, idx, False, rm, off, src, xp, ws, align=128)
    q = torch.randint(0, 256, (E, N, H // 2), generator=g, dtype=U8)
    s = torch.randint(119, 122, (E, N, H // 32), generator=g, dtype=U8)
    tq = torch.empty((E, N // 16, H // 128, 64, 16), dtype=U8, device="cuda")
    ts = torch.empty((E, N // 32, H // 128, 64, 2), dtype=U8, device="cuda")
    ff8.ff8_pack_mxfp4(q.cuda(), s.cuda(), tq, ts)
    out = [poisoned((M, N), BF16) for _ in range(2)]
    ff8.ff8_grouped_gemv_mxfp4(xp, tq, ts, off, out[0], src_row=src)
    ff8.ff8_grouped_gemv_mxfp4(x.cuda(), tq, ts, off, out[1], src_row=src, top_k=k)
    y, dyp, dp = poisoned((T, N), BF16), poisoned((M, N), BF16), poisoned((T, k), F32)
    ff8.ff8_unpermute(out[0], rm, p, y)
    dy = torch.randn((T, N), generator=g).to(BF16)
    ff8.ff8_unpermute_bwd(dy.cuda(), p, k, E, rm, off, src, dyp, out[0], dp)
    dz = poisoned((T, E), F32)
    ff8.ff8_router_topk_bwd(z.cuda(), idx, dp, dz, normalize=True)
    torch.cuda.synchronize()
    m = int(off[-1])
    _, w_off, w_map, w_src = moe.route(host(idx), E, 128)
    assert np.array_equal(host(off), w_off) and np.array_equal(host(rm), w_map) and np.array_equal(host(src[:m]), w_src)
    assert (host(idx)[real:] == -1).all() and (host(p)[real:] == 0).all() and (host(idx)[:real] >= 0).all()
    xs = np.where(w_src[:, None] >= 0, np.nan_to_num(f64(x))[np.maximum(w_src, 0) // k], 0.0)
    w = [mxfp4.dequant(q[e].numpy(), s[e].numpy()) for e in range(E)]
    a = mxfp4.grouped_product(xs, w, w_off)
    # half a bf16 step, and sums of 256 exact products: 24 additions of one unit of the sum of magnitudes
    tol = 2.0 ** -8 * np.abs(a) + 24 * 2.0 ** -23 * mxfp4.grouped_product(np.abs(xs), [np.abs(v) for v in w], w_off)
    for o in out:  # (the two may take row blocks of different heights, and then add in different orders)
        assert (np.abs(f64(o[:m]) - a) <= tol).all() and untouched(o[m:])
    assert (f64(y)[real:] == 0).all() and (f64(dz)[real:] == 0).all() and (host(dp)[real:] == 0).all()
    assert np.isfinite(f64(y)).all() and np.isfinite(f64(dyp[:m])).all() and np.isfinite(f64(dz)).all()
    assert (f64(dyp[:m])[w_src < 0] == 0).all() and untouched(dyp[m:])


def test_a_token_that_names_one_expert_twice():
    T, H, E, k = 70, 256, 4, 3
    g = torch.Generator().manual_seed(0)
    idx = torch.randint(0, E, (T, k), generator=g, dtype=I32)
    idx[:, 2] = idx[:, 0]
    x, dy = (torch.randn((T, H), generator=g).to(BF16) for _ in range(2))
    w = torch.rand((T, k), generator=g)
    M = ff8.ff8_rows_bound_aligned(T, k, E, 16)
    rm, off, src, xp = poisoned((T, k), I32), poisoned((E + 1,), I32), poisoned((M,), I32), poisoned((M, H), BF16)
    ws = torch.empty(max(1, ff8.ff8_permute_workspace_bytes(T, k, E)), dtype=U8, device="cuda")
    ff8.ff8_permute_bf16(x.cuda(), k, E, idx.cuda(), False, rm, off, src, xp, ws, align=16)
    dyp, dp = poisoned((M, H), BF16), poisoned((T, k), F32)
    ff8.ff8_unpermute_bwd(dy.cuda(), w.cuda(), k, E, rm, off, src, dyp, xp, dp)
    torch.cuda.synchronize()
    r = host(rm).astype(np.int64)
    _, w_off, w_map, _ = moe.route(idx.numpy(), E, 16)
    assert np.array_equal(host(off), w_off) and np.array_equal(r, w_map) and len(set(r.reshape(-1))) == T * k
    for j in range(k):
        assert torch.equal(xp.cpu()[r[:, j]], x)
        assert torch.equal(dyp.cpu()[r[:, j]], (w[:, j:j + 1] * dy.float()).to(BF16))
    want = (f64(dy) * f64(x)).sum(1)
    tol = (H / 64 + 6) * 2.0 ** -24 * (np.abs(f64(dy)) * np.abs(f64(x))).sum(1)
    assert (np.abs(f64(dp) - want[:, None]) <= tol[:, None]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,k", [(66, 6), (128, 8), (255, 9), (256, 16)])
def test_router_of_a_training_batch(dtype, E, k):
    """Above 64 experts and 2048 tokens, forward and backward, at an aligned and an odd address."""
    T = 2051
    g = torch.Generator().manual_seed(E)
    z = (torch.randn((T, E), generator=g) * 2).to(dtype)
    z[::7, ::2] = -float("inf")
    z[5] = -float("inf")
    dp = torch.randn((T, k), generator=g)
    want = router.choose(z.double().numpy(), None, k, "softmax")
    w = router.weights(z.double().numpy(), want, "softmax", False, 1.0)
    dw = router.weights_bwd(z.double().numpy(), want, dp.double().numpy(), "softmax", False, 1.0)
    outs = []
    for shift in (0, 1):
        zd = torch.empty(T * E + 8, dtype=dtype, device="cuda")[shift:shift + T * E].view(T, E)
        zd.copy_(z)
        dz = torch.empty(T * E + 8, dtype=dtype, device="cuda")[shift:shift + T * E].view(T, E)
        idx, p = poisoned((T, k), I32), poisoned((T, k), F32)
        ff8.ff8_router_topk(zd, idx, p)
        ff8.ff8_router_topk_bwd(zd, idx, dp.cuda(), dz)
        torch.cuda.synchronize()
        assert np.array_equal(host(idx), want)
        # an exponent's argument: at most |l - m| < 20 half-units; sums of 256 terms: 22 half-units
        assert (np.abs(f64(p) - w) <= (3 * 20 + 40) * 2.0 ** -24 * w).all()
        s = router.scores(z.double().numpy(), "softmax")
        dot = (w * np.abs(dp.double().numpy())).sum(1, keepdims=True)
        own = np.zeros_like(s)
        for j in range(k):
            rows = np.nonzero(want[:, j] >= 0)[0]
            own[rows, want[rows, j]] = np.abs(dp.double().numpy())[rows, j]
        tol = (100 + 2 * k) * 2.0 ** -24 * s * (own + dot) + torch.finfo(dtype).eps / 2 * np.abs(dw) + 2.0 ** -126
        assert (np.abs(f64(dz) - dw) <= tol).all()
        outs.append((idx, p, dz.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_empty_batches():
    L = ExpertLayerFP4(4, 256, 8, 2, 128)
    L.quantize_weights(torch.zeros((8, 256, 256), dtype=BF16, device="cuda"), torch.zeros((8, 256, 128), dtype=BF16, device="cuda"))
    y = L.forward(torch.empty((0, 256), dtype=BF16, device="cuda"), torch.empty((0, 8), device="cuda"))
    torch.cuda.synchronize()
    assert y.shape == (0, 256) and host(L.buf["offsets"]).tolist() == [0] * 9


def test_refuses_other_memory():
    z = torch.zeros((4, 8), device="cuda")
    idx, p = torch.zeros((4, 2), dtype=I32, device="cuda"), torch.zeros((4, 2), device="cuda")
    for bad in (lambda: ff8.ff8_router_topk(z.cpu(), idx, p), lambda: ff8.ff8_router_topk(z, idx.cpu(), p),
                lambda: ff8.ff8_router_topk(torch.zeros((4, 16), device="cuda")[:, ::2], idx, p),
                lambda: ff8.ff8_router_topk(z, idx, p, bias=torch.zeros(8)),
                lambda: ff8.ff8_router_topk_bwd(z, idx, p, z.t().contiguous().t())):
        with pytest.raises(ValueError):
            bad()
    x = torch.zeros(4 * 256 + 4, dtype=BF16, device="cuda")[4:].view(4, 256)  # 8 bytes off
    rm, off, src = torch.zeros_like(idx), torch.zeros(9, dtype=I32, device="cuda"), torch.zeros(256, dtype=I32, device="cuda")
    out = torch.zeros((256, 256), dtype=BF16, device="cuda")
    ws = torch.zeros(1 << 16, dtype=U8, device="cuda")
    with pytest.raises(RuntimeError, match="aligned"):
        ff8.ff8_permute_bf16(x, 2, 8, idx, False, rm, off, src, out, ws, align=16)
    with pytest.raises(RuntimeError, match="aligned"):
        ff8.ff8_quant_mxfp4(x, torch.zeros((4, 128), dtype=U8, device="cuda"), torch.zeros((4, 8), dtype=U8, device="cuda"))
    with pytest.raises(ValueError, match="workspace"):
        ff8.ff8_permute_bf16(x, 2, 8, idx, False, rm, off, src, out, ws.cpu(), align=16)
