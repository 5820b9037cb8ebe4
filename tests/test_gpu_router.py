"""The router's top-k choice, weights and gradient against the float64 oracle (GPU)."""

import numpy as np
import pytest
import torch

from oracle import router
from paper_2511_02302_amd import ff8

from test_gpu_kernels import f64, host, poisoned

pytestmark = pytest.mark.gpu

MODES = [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)]
SHAPES = [(1, 1, 1), (3, 2, 2), (257, 5, 3), (64, 8, 2), (33, 16, 16), (70, 17, 17), (129, 32, 8), (65, 33, 1),
          (40, 64, 64), (31, 65, 64), (66, 100, 6), (9, 128, 8), (130, 160, 6), (12, 255, 9), (50, 256, 8),
          (21, 257, 33), (7, 384, 8), (18, 512, 8), (6, 513, 12), (11, 1000, 64), (10, 1024, 8),
          (37, 129, 8), (40, 130, 7), (50, 144, 8), (2100, 201, 3), (33, 160, 16), (70, 80, 5), (71, 66, 4)]


def _logits(T, E, dtype, seed, std=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, E), generator=g) * std).to(dtype)


def _run(logits, bias, k, score, normalize, scale):
    T = logits.shape[0]
    idx, probs = poisoned((T, k), torch.int32), poisoned((T, k), torch.float32)
    ff8.ff8_router_topk(logits.cuda(), idx, probs, bias=None if bias is None else bias.cuda(), score=score,
                        normalize=normalize, scale=scale)
    torch.cuda.synchronize()
    return host(idx), f64(probs)


def _rel(z):
    """Bound on the relative error of a weight.  An exponential's argument l - m has one rounding, of
    at most R * 2^-24 with R the largest |l - m| (both of log sigmoid's parts within it), expf at most
    2^-23; a sum of up to 16 a lane and six steps over lanes adds 22 half-units, sigmoid, division and
    scale a few more: (3 R + 40) * 2^-24, numerator and denominator together."""
    finite = z[np.isfinite(z)]
    R = 2 * np.abs(finite).max() if finite.size else 0.0
    return (3 * R + 40) * 2.0 ** -24


def _check(logits, bias, k, score, normalize, scale=2.5):
    z = logits.double().numpy()
    idx, p = _run(logits, bias, k, score, normalize, scale)
    want = router.choose(z, None if bias is None else bias.double().numpy(), k, score)
    assert np.array_equal(idx, want)
    w = router.weights(z, want, score, normalize, scale)
    assert np.array_equal(np.isnan(p), np.isnan(w))
    ok = ~np.isnan(w)
    assert np.all(np.abs(p - w)[ok] <= _rel(z) * np.abs(w)[ok] + 2.0 ** -126)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,normalize", MODES)
def test_forward_sizes(dtype, score, normalize):
    for n, (T, E, k) in enumerate(SHAPES):
        bias = torch.randn(E, generator=torch.Generator().manual_seed(n)) * 0.3 if n % 2 else None
        _check(_logits(T, E, dtype, 10 + n), bias, k, score, normalize)


@pytest.mark.parametrize("score,normalize", MODES)
@pytest.mark.parametrize("with_bias", [False, True])
def test_forward_masks_and_empty_rows(score, normalize, with_bias):
    for E, k in ((6, 4), (32, 8), (200, 16), (600, 8)):
        z = _logits(90, E, torch.float32, E)
        z[torch.rand((90, E), generator=torch.Generator().manual_seed(5)) < 0.8] = -float("inf")
        z[0] = -float("inf")                                # nothing to choose
        z[1] = -float("inf"); z[1, E - 1] = -3.0            # the last expert alone
        z[2] = torch.finfo(torch.float32).min               # all equal, at the type's lowest value
        z[3] = -float("inf"); z[3, 1] = torch.finfo(torch.float32).min
        bias = torch.linspace(-0.5, 0.5, E) if with_bias else None
        z_fin = z.clamp(min=-100.0)  # the bound of _rel is of the rows that have a sum; rows 2 and 3 are exact cases
        idx, p = _run(z, bias, k, score, normalize, 1.0)
        want = router.choose(z.double().numpy(), None if bias is None else bias.double().numpy(), k, score)
        assert np.array_equal(idx, want)
        w = router.weights(z.double().numpy(), want, score, normalize, 1.0)
        assert np.all(np.abs(p - w) <= _rel(z_fin.double().numpy()) * np.abs(w) + 2.0 ** -126)
        assert (idx[0] == -1).all() and (p[0] == 0).all()


@pytest.mark.parametrize("score,normalize", MODES)
def test_forward_nan_and_infinity(score, normalize):
    z = _logits(6, 40, torch.float32, 3)
    z[0, 7] = float("nan")
    z[1, :] = float("nan")
    z[2, 5] = float("nan"); z[2, 6] = -float("inf")
    bias = torch.zeros(40); bias[3] = float("nan"); bias[4] = -float("inf")
    _check(z, None, 8, score, normalize)
    idx, _ = _run(z, bias, 40, score, normalize, 1.0)
    assert not np.isin(idx, [3, 4]).any()
    if score == "sigmoid":  # one NaN logit leaves the others as they are
        z2 = z.clone(); z2[0, 7] = -float("inf")
        i1, p1 = _run(z[:1], None, 8, score, normalize, 1.0)
        i2, p2 = _run(z2[:1], None, 8, score, normalize, 1.0)
        assert np.array_equal(i1, i2) and np.array_equal(p1, p2)


def test_ties_and_near_ties():
    for E in (8, 64, 256, 1024):
        z = torch.zeros((4, E))
        z[1, ::2] = -0.0                                   # equal as numbers
        z[2] = torch.arange(E).remainder(3).float()
        _check(z, None, min(E, 8), "softmax", True)
        _check(z, torch.zeros(E), min(E, 8), "sigmoid", True)
        # score + bias whose float32 sums are equal and whose float64 sums are not
        b = torch.zeros(E)
        b[E - 1] = 2.0 ** -26
        _check(z[:1].contiguous(), b, 2, "sigmoid", False)
        _check(z[:1].contiguous(), b, 2, "softmax", False)
        # neighbours one float32 step apart, largest last: the scores' float32 values would tie
        step = torch.full((1, E), 1.0)
        step[0, E - 1] = float(np.nextafter(np.float32(1.0), np.float32(2.0)))
        _check(step, torch.zeros(E), 2, "sigmoid", True)
        _check(step, torch.full((E,), 8.0), 2, "softmax", False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T", [3, 2500])
def test_order_that_float32_does_not_tell(score, T):
    """Clusters of experts with equal logits and biases a few 2^-27 apart (one float32 step of the sums is 2^-24 and
    more), some exactly equal: the order of every cluster, and where it ends the choice, is the float64 one."""
    for E, n, k in ((16, 12, 8), (16, 16, 16), (48, 20, 8), (64, 30, 16), (256, 9, 8), (256, 24, 8), (256, 200, 8),
                    (256, 40, 12), (600, 30, 20)):
        rng = np.random.default_rng(E + n + k)
        z = rng.normal(size=(T, E)).astype(np.float32) - 6.0
        b = np.zeros(E, dtype=np.float32)
        at = rng.permutation(E)[:n]
        z[:, at] = 1.0
        b[at] = rng.integers(0, n, size=n) * 2.0 ** -27  # duplicates among them
        z[::3, at[: n // 3]] = 1.5                       # a second cluster in some rows
        idx, _ = _run(torch.from_numpy(z), torch.from_numpy(b), k, score, True, 1.0)
        assert np.array_equal(idx, router.choose(z, b, k, score)), (E, n, k)


def test_scores_that_underflow():
    z = torch.full((2, 64), -200.0)
    z[0, 3], z[0, 9] = -150.0, -151.0
    idx, p = _run(z, None, 2, "sigmoid", True, 1.0)
    assert idx[0].tolist() == [3, 9]
    want = router.weights(z.double().numpy(), idx, "sigmoid", True, 1.0)
    assert np.all(np.abs(p - want) <= _rel(z.double().numpy()) * want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,normalize", MODES)
def test_backward(dtype, score, normalize):
    for n, (T, E, k) in enumerate(SHAPES):
        z = _logits(T, E, dtype, 40 + n)
        if E > 4:
            z[0] = -float("inf")
            z[T // 2, ::3] = -float("inf")
        idx = torch.from_numpy(router.choose(z.double().numpy(), None, k, score)).int()
        if T > 2:
            idx[T - 1, k - 1] = -1
            idx[T - 2, :] = idx[T - 2, 0]  # one expert in every slot
        dp = torch.randn((T, k), generator=torch.Generator().manual_seed(n))
        dp[idx < 0] = float("nan")  # what stands beside a dropped slot is not read
        out = poisoned((T, E), dtype)
        ff8.ff8_router_topk_bwd(z.cuda(), idx.cuda(), dp.cuda(), out, score=score, normalize=normalize, scale=2.5)
        torch.cuda.synchronize()
        zd, i, d = z.double().numpy(), idx.numpy(), np.nan_to_num(dp.double().numpy())
        want = router.weights_bwd(zd, i, d, score, normalize, 2.5)
        # each of the two terms of a difference has a weight's error and k more roundings of the dot product;
        # terms of a slot's own gradient add up over slots of one expert
        bound = router.weights_bwd(zd, i, np.abs(d), score, False, 2.5) if score == "sigmoid" and not normalize else None
        if bound is None:
            if normalize:
                r = router.weights(zd, i, score, True, 2.5)
                per = r * (np.abs(d) + (r / 2.5 * np.abs(d)).sum(1, keepdims=True))
            else:
                s = router.scores(zd, score)
                per = np.where(i >= 0, np.take_along_axis(s, np.maximum(i, 0), 1), 0.0) * np.abs(d) * 2.5
                bound = s * per.sum(1, keepdims=True)
            bound = np.zeros_like(want) if bound is None else bound
            for j in range(k):
                rows = np.nonzero(i[:, j] >= 0)[0]
                np.add.at(bound, (rows, i[rows, j]), per[rows, j])
        tol = (_rel(zd) + 2 * k * 2.0 ** -24) * np.abs(bound) + torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -126
        assert np.all(np.abs(f64(out) - want) <= tol), (T, E, k)


def test_backward_against_differences_of_the_forward():
    """Central differences of the kernel's own float32 weights along random directions."""
    for score, normalize in MODES:
        z = _logits(16, 24, torch.float32, 7, std=1.0)
        k = 4
        idx, _ = _run(z, None, k, score, normalize, 1.0)
        dp = torch.randn((16, k), generator=torch.Generator().manual_seed(1))
        out = poisoned((16, 24), torch.float32)
        ff8.ff8_router_topk_bwd(z.cuda(), torch.from_numpy(idx).int().cuda(), dp.cuda(), out, score=score,
                                normalize=normalize)
        h = 2.0 ** -8
        v = torch.randn((16, 24), generator=torch.Generator().manual_seed(2))
        f = []
        for sign in (1, -1):
            p = router.weights((z.double() + sign * h * v.double()).numpy(), idx, score, normalize, 1.0)
            f.append((p * dp.double().numpy()).sum(1))
        num = (f[0] - f[1]) / (2 * h)
        got = (f64(out) * v.double().numpy()).sum(1)
        # truncation: h^2 / 6 * third derivative (products of at most 24 N(0, 1) directions: below 100)
        assert np.all(np.abs(num - got) <= h * h / 6 * 100 + 1e-5)


def test_empty_batch_and_other_stream():
    for dt in (torch.float32, torch.bfloat16):
        z = torch.empty((0, 8), dtype=dt, device="cuda")
        i, p = torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda")
        ff8.ff8_router_topk(z, i, p)
        ff8.ff8_router_topk_bwd(z, i, p, torch.empty_like(z))
    z = _logits(300, 64, torch.float32, 1).cuda()
    i, p = poisoned((300, 8), torch.int32), poisoned((300, 8), torch.float32)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ff8.ff8_router_topk(z, i, p, stream=s)
    s.synchronize()
    want = router.choose(z.cpu().double().numpy(), None, 8, "softmax")
    assert np.array_equal(host(i), want)


def test_bitwise_repeatable():
    z = _logits(500, 256, torch.bfloat16, 2)
    b = torch.randn(256, generator=torch.Generator().manual_seed(3)) * 0.1
    first = _run(z, b, 8, "sigmoid", True, 2.5)
    second = _run(z, b, 8, "sigmoid", True, 2.5)
    assert np.array_equal(first[0], second[0]) and np.array_equal(first[1], second[1])
