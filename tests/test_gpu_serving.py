"""The serving layer (router, routing, 4-bit products, weighted return) against the oracle, captured and
replayed, and the bf16 training path around experts of another library (GPU)."""

import numpy as np
import pytest
import torch

from oracle import codec, moe, mxfp4, router
from paper_2511_02302_amd import ff8
from paper_2511_02302_amd.layer import ExpertLayerFP4

from test_gpu_kernels import f64, host, rel_frob

pytestmark = pytest.mark.gpu

# T, H, E, k, I, score, normalize, with a bias
CASES = [(1, 256, 8, 2, 128, "softmax", False, False), (33, 384, 6, 3, 256, "sigmoid", True, True),
         (64, 640, 24, 6, 384, "softmax", True, True), (300, 256, 4, 4, 256, "sigmoid", False, False)]


def _inputs(T, H, E, I, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda shape, std=1.0: (torch.randn(shape, generator=g) * std).to(torch.bfloat16)  # noqa: E731
    return r((T, H)), r((T, E)), r((E, 2 * I, H), 0.05), r((E, H, I), 0.05), torch.randn(E, generator=g) * 0.2


def _oracle(x, logits, bias, w1, w2, E, k, I, score, normalize, scale):
    z = f64(logits)
    idx = router.choose(z, None if bias is None else f64(bias), k, score)
    p = router.weights(z, idx, score, normalize, scale)
    _, off, row_map, src = moe.route(idx, E, 16)
    xs = np.where(src[:, None] >= 0, f64(x)[np.maximum(src, 0) // k], 0.0)
    a = mxfp4.grouped_product(xs, [mxfp4.dequant(*mxfp4.quant(f64(w))) for w in w1], off)
    h = codec.bf16_round(a[:, :I] / (1.0 + np.exp(-a[:, :I])) * a[:, I:])
    y_perm = codec.bf16_round(mxfp4.grouped_product(h, [mxfp4.dequant(*mxfp4.quant(f64(w))) for w in w2], off))
    return idx, p, moe.unpermute(y_perm, row_map, p)


@pytest.mark.parametrize("T,H,E,k,I,score,normalize,with_bias", CASES)
def test_layer_against_oracle(T, H, E, k, I, score, normalize, with_bias):
    x, logits, w1, w2, bias = _inputs(T, H, E, I)
    bias = bias if with_bias else None
    L = ExpertLayerFP4(max(T, 40), H, E, k, I, score=score, normalize=normalize, scale=2.5)
    L.quantize_weights(w1.cuda(), w2.cuda())
    y = L.forward(x.cuda(), logits.cuda(), None if bias is None else bias.cuda())
    torch.cuda.synchronize()
    idx, p, want = _oracle(x, logits, bias, w1, w2, E, k, I, score, normalize, 2.5)
    assert np.array_equal(host(L.buf["topk_idx"][:T]), idx)
    assert rel_frob(f64(L.buf["probs"][:T]), p) < 1e-6
    # bf16 roundings of h, y_perm and y, each off by at most 2^-8 of its value and by their root mean square of
    # about 2^-9 / sqrt(3) in norm: three of them, with room for one that falls to the other side
    assert rel_frob(f64(y), want) < 3 * 2.0 ** -9


def test_loaded_weights_equal_quantized_ones():
    T, H, E, k, I = 20, 256, 4, 2, 128
    x, logits, w1, w2, _ = _inputs(T, H, E, I, 1)
    a, b = ExpertLayerFP4(T, H, E, k, I), ExpertLayerFP4(T, H, E, k, I)
    a.quantize_weights(w1.cuda(), w2.cuda())
    ready = []
    for w in (w1, w2):
        qs = [mxfp4.quant(f64(v)) for v in w]
        ready += [torch.from_numpy(np.stack([q for q, _ in qs])).cuda(), torch.from_numpy(np.stack([s for _, s in qs])).cuda()]
    b.load_weights(*ready)
    assert torch.equal(a.forward(x.cuda(), logits.cuda()), b.forward(x.cuda(), logits.cuda()))


def test_captured_steps_replay_with_new_inputs():
    """Two batch sizes of one layer, captured, then replayed in turn with eager steps between."""
    T, H, E, k, I = 48, 512, 16, 4, 256
    _, _, w1, w2, _ = _inputs(1, H, E, I, 2)
    L, ref = (ExpertLayerFP4(T, H, E, k, I, score="sigmoid", normalize=True) for _ in range(2))
    for layer in (L, ref):
        layer.quantize_weights(w1.cuda(), w2.cuda())
    bias = torch.zeros(E, device="cuda")
    graphs = []
    for n in (T, 5):
        x, z = torch.zeros((n, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, E), dtype=torch.bfloat16, device="cuda")
        L.forward(x, z, bias)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.forward(x, z, bias)
        graphs.append((n, x, z, g))
    for rep in range(4):
        for n, x, z, g in graphs:
            xi, zi, _, _, _ = _inputs(n, H, E, I, 10 + rep)
            x.copy_(xi); z.copy_(zi)
            want = ref.forward(x, z, bias).clone()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(L.buf["y"][:n], want), (rep, n)


def test_a_tokens_output_does_not_depend_on_the_batch():
    T, H, E, k, I = 200, 512, 8, 2, 256
    x, logits, w1, w2, _ = _inputs(T, H, E, I, 3)
    L = ExpertLayerFP4(T, H, E, k, I)
    L.quantize_weights(w1.cuda(), w2.cuda())
    whole = L.forward(x.cuda(), logits.cuda()).clone()
    for t in (0, 77, 199):
        one = L.forward(x[t:t + 1].cuda(), logits[t:t + 1].cuda())
        # float32 sums in another order may fall to the other side of a bf16 step, in h, y_perm and y
        assert rel_frob(f64(one), f64(whole[t:t + 1])) < 3 * 2.0 ** -9


def test_layer_refuses():
    with pytest.raises(ValueError):
        ExpertLayerFP4(4, 200, 8, 2, 128)
    with pytest.raises(ValueError):
        ExpertLayerFP4(4, 256, 8, 9, 128)
    with pytest.raises(ValueError):
        ExpertLayerFP4(4, 256, 8, 2, 128, score="relu")
    L = ExpertLayerFP4(4, 256, 8, 2, 128)
    x, z, w1, w2, _ = _inputs(5, 256, 8, 128)
    with pytest.raises(ValueError):
        L.forward(x.cuda(), z.cuda())
    with pytest.raises(ValueError):
        L.quantize_weights(w2.cuda(), w1.cuda())


def test_training_path_around_other_experts():
    """Router, sort, experts that torch computes (one bf16 matrix each), weighted return, and all of it back:
    gradients of the tokens and the logits against autograd in float64."""
    T, H, E, k, align = 150, 256, 6, 2, 16
    g = torch.Generator().manual_seed(0)
    x = torch.randn((T, H), generator=g).to(torch.bfloat16)
    z = torch.randn((T, E), generator=g)
    w = (torch.randn((E, H, H), generator=g) * 0.06).to(torch.bfloat16)
    dy = torch.randn((T, H), generator=g).to(torch.bfloat16)
    M = ff8.ff8_rows_bound_aligned(T, k, E, align)
    new = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    idx, p = new(T, k, dt=torch.int32), new(T, k, dt=torch.float32)
    row_map, off, src = new(T, k, dt=torch.int32), new(E + 1, dt=torch.int32), new(M, dt=torch.int32)
    ws = new(ff8.ff8_permute_workspace_bytes(T, k, E), dt=torch.uint8)
    xd, zd, wd, dyd = x.cuda(), z.cuda(), w.cuda(), dy.cuda()
    ff8.ff8_router_topk(zd, idx, p, normalize=True)
    xp, yp, y = new(M, H), new(M, H), new(T, H)
    ff8.ff8_permute_bf16(xd, k, E, idx, False, row_map, off, src, xp, ws, align=align)
    o = off.tolist()
    for e in range(E):
        yp[o[e]:o[e + 1]] = (xp[o[e]:o[e + 1]].float() @ wd[e].float()).to(torch.bfloat16)
    ff8.ff8_unpermute(yp, row_map, p, y)
    dyp, dp, dz = new(M, H), new(T, k, dt=torch.float32), new(T, E, dt=torch.float32)
    ff8.ff8_unpermute_bwd(dyd, p, k, E, row_map, off, src, dyp, yp, dp)
    dxp, dx = new(M, H), new(T, H)
    for e in range(E):
        dxp[o[e]:o[e + 1]] = (dyp[o[e]:o[e + 1]].float() @ wd[e].float().t().contiguous()).to(torch.bfloat16)
    ff8.ff8_unpermute(dxp, row_map, None, dx)
    ff8.ff8_router_topk_bwd(zd, idx, dp, dz, normalize=True)
    torch.cuda.synchronize()
    x64, z64 = x.double().requires_grad_(), z.double().requires_grad_()
    top = torch.topk(z64, k, dim=1)
    assert torch.equal(top.indices.int(), idx.cpu())
    probs = torch.softmax(top.values, dim=1)
    full = torch.stack([x64 @ w[e].double() for e in range(E)], 1)
    want = (torch.gather(full, 1, top.indices[..., None].expand(T, k, H)) * probs[..., None]).sum(1)
    want.backward(dy.double())
    # y: two bf16 roundings; dx: three; dz: one of y_perm inside a dot product, whose random errors average
    assert rel_frob(f64(y), want.detach().numpy()) < 2 * 2.0 ** -9
    assert rel_frob(f64(dx), x64.grad.numpy()) < 3 * 2.0 ** -9
    assert rel_frob(f64(dz), z64.grad.numpy()) < 2.0 ** -8
