"""What the router, the uncast row sorts and the 4-bit products refuse, on the host (CPU only)."""

import ctypes

import pytest

from paper_2511_02302_amd import ff8

NULL, SHAPE, ARG = 1, 2, 3
P = ctypes.c_void_p(0x1000)    # never dereferenced: every call below is refused before a launch
ODD = ctypes.c_void_p(0x1008)  # not 16-byte aligned
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return ff8.load()


@pytest.mark.parametrize("name", ["ff8_router_topk", "ff8_router_topk_bf16"])
def test_router(lib, name):
    f = getattr(lib, name)
    ok = dict(logits=P, bias=None, T=4, E=8, k=2, score=0, norm=0, scale=1.0, idx=P, probs=P)
    call = lambda **o: f(*{**ok, **o}.values(), None)  # noqa: E731
    for bad in (dict(k=0), dict(k=9), dict(E=0, k=0), dict(E=1025), dict(E=100, k=65), dict(score=2), dict(score=-1),
                dict(norm=2), dict(scale=NAN), dict(scale=INF)):
        assert call(**bad) == ARG, bad
    for bad in (dict(T=-1), dict(T=1 << 31), dict(T=1 << 30, k=2)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(logits=None), dict(idx=None), dict(probs=None)):
        assert call(**bad) == NULL, bad
        assert b"NULL" in lib.ff8_last_error()
    assert call(T=0, logits=None, idx=None, probs=None) == 0  # an empty batch: nothing to launch


@pytest.mark.parametrize("name", ["ff8_router_topk_bwd", "ff8_router_topk_bwd_bf16"])
def test_router_bwd(lib, name):
    f = getattr(lib, name)
    ok = dict(logits=P, idx=P, dprobs=P, T=4, E=8, k=2, score=0, norm=0, scale=1.0, out=P)
    call = lambda **o: f(*{**ok, **o}.values(), None)  # noqa: E731
    assert call(k=9) == ARG and call(E=2000) == ARG and call(score=7) == ARG and call(norm=-1) == ARG
    assert call(scale=NAN) == ARG and call(T=-5) == SHAPE
    for n in ("logits", "idx", "dprobs", "out"):
        assert call(**{n: None}) == NULL


def test_route(lib):
    ok = dict(idx=P, T=16, k=2, E=4, row_map=P, offsets=P, src=P, M=640, ws=P, n=1 << 20, align=128)
    call = lambda **o: lib.ff8_route(*{**ok, **o}.values(), None)  # noqa: E731
    assert call(k=5) == ARG and call(E=1025) == ARG and call(align=24) == ARG and call(n=0) == ARG
    assert call(M=128) == SHAPE and call(M=641) == SHAPE and call(T=-1) == SHAPE
    for n in ("idx", "row_map", "offsets", "src", "ws"):
        assert call(**{n: None}) == NULL, n


@pytest.mark.parametrize("name", ["ff8_permute_bf16", "ff8_permute_fp8", "ff8_permute_fp8_e8m0"])
def test_permutes(lib, name):
    fp8 = "fp8" in name
    ok = dict(x=P, **({"xs": P} if fp8 else {}), T=16, H=128, k=2, E=4, idx=P, reuse=0, row_map=P, offsets=P, src=P,
              M=640, out=P, **({"s": P} if fp8 else {}), ws=P, n=1 << 20, align=128)
    call = lambda **o: getattr(lib, name)(*{**ok, **o}.values(), None)  # noqa: E731
    assert call(H=64) == SHAPE and call(H=0) == SHAPE and call(M=512) == SHAPE and call(T=-1) == SHAPE
    assert call(k=5) == ARG and call(reuse=2) == ARG and call(align=8) == ARG and call(n=4) == ARG
    assert call(x=ODD) == ARG and call(out=ODD) == ARG
    assert b"aligned" in lib.ff8_last_error()
    for n in ("x", "idx", "row_map", "offsets", "src", "out", "ws") + (("xs", "s") if fp8 else ()):
        assert call(**{n: None}) == NULL, n


def test_unpermute_bwd(lib):
    ok = dict(dy=P, w=P, T=16, H=128, k=2, E=4, row_map=P, offsets=P, src=P, M=640, dyp=P, yp=P, dp=P)
    call = lambda **o: lib.ff8_unpermute_bwd(*{**ok, **o}.values(), None)  # noqa: E731
    assert call(E=100, k=65, M=1 << 20) == ARG and call(k=5) == ARG and call(H=100) == SHAPE and call(M=0) == SHAPE
    for n in ("dy", "w", "row_map", "offsets", "src", "dyp", "yp", "dp"):
        assert call(**{n: None}) == NULL, n
    for n in ("dy", "dyp", "yp"):
        assert call(**{n: ODD}) == ARG, n


def test_mxfp4_formats(lib):
    q = lambda *a: lib.ff8_quant_mxfp4(*a, None)  # noqa: E731
    assert q(None, 4, 128, P, P) == NULL and q(P, 4, 128, None, P) == NULL and q(P, 4, 128, P, None) == NULL
    assert q(P, 0, 128, P, P) == SHAPE and q(P, 4, 96, P, P) == SHAPE and q(P, 1 << 28, 128, P, P) == SHAPE
    assert q(ODD, 4, 128, P, P) == ARG and q(P, 4, 128, ODD, P) == ARG
    p = lambda *a: lib.ff8_pack_mxfp4(*a, None)  # noqa: E731
    for i in range(6):
        args = [P, P, 128, 128, P, P]
        if i in (2, 3):
            args[i] = 64
            assert p(*args) == SHAPE
        else:
            args[i] = None
            assert p(*args) == NULL
    assert p(ODD, P, 128, 128, P, P) == ARG and p(P, P, 128, 128, ODD, P) == ARG and p(P, P, 128, 128, P, ODD) == ARG


@pytest.mark.parametrize("name", ["ff8_grouped_gemv_mxfp4", "ff8_grouped_gemv_mxfp4_swiglu"])
def test_mxfp4_products(lib, name):
    ok = dict(x=P, x_rows=256, tq=P, ts=P, offsets=P, E=4, src=P, top_k=0, M=256, N=128, K=128, out=P)
    call = lambda **o: getattr(lib, name)(*{**ok, **o}.values(), None)  # noqa: E731
    for bad in (dict(E=0), dict(E=1025), dict(top_k=-1), dict(x=ODD), dict(tq=ODD), dict(ts=ODD), dict(out=ODD)):
        assert call(**bad) == ARG, bad
    for bad in (dict(M=200), dict(M=0), dict(N=64), dict(N=192), dict(K=96), dict(K=0), dict(x_rows=100),
                dict(top_k=2, x_rows=-1), dict(top_k=2, x_rows=1 << 31), dict(M=1 << 31, x_rows=1 << 31),
                dict(top_k=2, x_rows=1 << 28, K=1 << 7), dict(M=1 << 28, x_rows=1 << 28, N=1 << 13)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(x=None), dict(tq=None), dict(ts=None), dict(offsets=None), dict(out=None),
                dict(src=None, top_k=1)):
        assert call(**bad) == NULL, bad


def test_binding_checks_shapes_and_types():
    torch = pytest.importorskip("torch")
    u8, f32, bf16, i32 = torch.uint8, torch.float32, torch.bfloat16, torch.int32
    e = lambda *shape, dtype=bf16: torch.empty(shape, dtype=dtype)  # noqa: E731
    T, E, k, H, M, N, K = 16, 8, 2, 256, 256, 384, 256
    idx, w, off, src = e(T, k, dtype=i32), e(T, k, dtype=f32), e(E + 1, dtype=i32), e(M, dtype=i32)
    tq, ts = e(E, N // 16, K // 128, 64, 16, dtype=u8), e(E, N // 32, K // 128, 64, 2, dtype=u8)
    wrong = [
        lambda: ff8.ff8_router_topk(e(T, E), e(T - 1, k, dtype=i32), w),
        lambda: ff8.ff8_router_topk(e(T, E), idx, e(T, k + 1, dtype=f32)),
        lambda: ff8.ff8_router_topk(e(T, E), idx, w, bias=e(E - 1, dtype=f32)),
        lambda: ff8.ff8_router_topk_bwd(e(T, E), idx, w, e(T, E + 1)),
        lambda: ff8.ff8_route(idx, E, e(T, k - 1, dtype=i32), off, src, None),
        lambda: ff8.ff8_permute_bf16(e(T, H), k, E, idx, False, idx, off, src, e(M, H + 128)),
        lambda: ff8.ff8_permute_bf16(e(T, H), k, E, idx, False, idx, off, e(M - 1, dtype=i32), e(M, H)),
        lambda: ff8.ff8_permute_fp8(e(T, H, dtype=u8), e(T, 1, dtype=f32), k, E, idx, False, idx, off, src,
                                    e(M, H, dtype=u8), e(M, 2, dtype=f32)),
        lambda: ff8.ff8_unpermute_bwd(e(T, H), w, k, E, idx, off, src, e(M, H), e(M - 128, H), w),
        lambda: ff8.ff8_unpermute_bwd(e(T, H), w, k, E, idx, off, src, e(M, H), e(M, H), e(T, k + 1, dtype=f32)),
        lambda: ff8.ff8_quant_mxfp4(e(N, K), e(N, K, dtype=u8), e(N, K // 32, dtype=u8)),
        lambda: ff8.ff8_pack_mxfp4(e(E, N, K // 2, dtype=u8), e(E, N, K // 16, dtype=u8), tq, ts),
        lambda: ff8.ff8_pack_mxfp4(e(E, N, K // 2, dtype=u8), e(E, N, K // 32, dtype=u8), tq[:, :1], ts),
        lambda: ff8.ff8_grouped_gemv_mxfp4(e(M, K + 128), tq, ts, off, e(M, N)),
        lambda: ff8.ff8_grouped_gemv_mxfp4(e(M, K), tq, ts, off, e(M, N // 2)),
        lambda: ff8.ff8_grouped_gemv_mxfp4_swiglu(e(M, K), tq, ts, off, e(M, N)),
        lambda: ff8.ff8_grouped_gemv_mxfp4(e(M, K), tq, ts, off, e(M, N), src_row=e(M + 1, dtype=i32)),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError, match="must (have shape|hold)"):
            call()
            pytest.fail(str(i))
    with pytest.raises(ValueError, match="score"):
        ff8.ff8_router_topk(e(T, E), idx, w, score="relu")
    for call in (lambda: ff8.ff8_router_topk(e(T, E, dtype=torch.float16), idx, w),
                 lambda: ff8.ff8_router_topk(e(T, E), idx.long(), w),
                 lambda: ff8.ff8_permute_fp8(e(T, H, dtype=u8), e(T, 2, dtype=f32), k, E, idx, False, idx, off, src,
                                             e(M, H, dtype=u8), e(M, 2, dtype=u8))):
        with pytest.raises((TypeError, ValueError)):
            call()
    # consistent calls stop at the device check here
    with pytest.raises(ValueError, match="device tensor"):
        ff8.ff8_grouped_gemv_mxfp4(e(M, K), tq, ts, off, e(M, N))


def test_sizes_of_one_launch(lib):
    """Beyond these a launch would have 2^32 threads or more."""
    big = 1 << 25
    assert lib.ff8_router_topk_bf16(P, None, big + 1, 8, 1, 0, 0, 1.0, P, P, None) == SHAPE
    assert lib.ff8_router_topk_bwd(P, P, P, big + 1, 8, 1, 0, 0, 1.0, P, None) == SHAPE
    M = 1 << 27
    assert lib.ff8_permute_bf16(P, big, 128, 2, 4, P, 0, P, P, P, M, P, P, 1 << 40, 16, None) == SHAPE
    assert lib.ff8_permute_fp8(P, P, big, 128, 2, 4, P, 0, P, P, P, M, P, P, P, 1 << 40, 16, None) == SHAPE
    assert lib.ff8_unpermute_bwd(P, P, big, 128, 2, 4, P, P, P, M, P, P, P, None) == SHAPE
    assert b"2^25" in lib.ff8_last_error()
    assert lib.ff8_quant_mxfp4(P, 1 << 27, 128, P, P, None) == SHAPE
    assert lib.ff8_grouped_gemv_mxfp4(P, 4, P, P, P, 4, P, 1, 1 << 21, 1 << 13, 128, P, None) == SHAPE


@pytest.mark.parametrize("rows,experts", [(4, 16), (4, 9), (4, 7), (3, 8), (5, 8)])
def test_serving_layer_checks_its_logits(rows, experts):
    """The router takes the number of experts from the logits, the routing from the layer: of wider logits the
    choices behind the layer's experts would be dropped without a word."""
    torch = pytest.importorskip("torch")
    from paper_2511_02302_amd.layer import ExpertLayerFP4
    layer = ExpertLayerFP4(4, 256, 8, 2, 128, device="cpu")
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="logits must have shape"):
        layer.forward(x, torch.zeros((rows, experts)))
    with pytest.raises(ValueError, match="device tensor"):  # the right shape stops at the device check here
        layer.forward(x, torch.zeros((4, 8)))
