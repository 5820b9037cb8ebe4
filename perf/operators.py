"""Operator cases around the experts of a routed MoE layer: what turns router logits into experts
and weights, what sorts token rows by expert and brings gradients back through the weighted return,
and the experts' products with 4-bit weights for serving.

A case is a dict of plain values.  Kinds:
  gate      top-k experts and routing weights from router logits (`ff8_router_topk`), or with
            bwd the gradient of the logits (`ff8_router_topk_bwd`)
  sort      token rows sorted by expert without a cast, with their routing maps
            (`ff8_permute_bf16`, `ff8_permute_fp8`)
  return    the gradient of the weighted return: the experts' rows of dY and the routing weights'
            gradient (`ff8_unpermute_bwd`)
  w4        grouped products of a few rows per expert with MXFP4 weights: "up" gathers the tokens
            and ends in SwiGLU (`ff8_grouped_gemv_mxfp4_swiglu`), "down" reads grouped rows
            (`ff8_grouped_gemv_mxfp4`)

With `own` false, `run` computes the same from elementary torch operations.
"""

import math

import torch

own = False

_TMIN = -126  # exponent of the scale of an all-zero tile


def _gate(T, E, k, **opts):
    return {"kind": "gate", "T": T, "E": E, "k": k, "dtype": "bf16", "score": "softmax", "normalize": False,
            "scale": 1.0, "bias": False, "masked": False, "bwd": False, **opts}


def _sort(T, H, E, k, **opts):
    return {"kind": "sort", "T": T, "H": H, "E": E, "k": k, "align": 128, "payload": "bf16", "routing": "iid",
            "dropped": False, **opts}


def _return(T, H, E, k, **opts):
    return {"kind": "return", "T": T, "H": H, "E": E, "k": k, "align": 128, "routing": "iid", "dropped": False,
            "dprobs": True, **opts}


def _w4(part, T, H, E, k, I, **opts):
    return {"kind": "w4", "part": part, "T": T, "H": H, "E": E, "k": k, "I": I, "routing": "iid", **opts}


def listed():
    return [
        # one token of a decoding step over all 256 experts of a model that selects by sigmoid
        # scores plus a balancing bias and scales the renormalized weights: latency alone
        {"name": "gate_one", **_gate(1, 256, 8, score="sigmoid", normalize=True, scale=2.5, bias=True)},
        # the same router over a training batch
        {"name": "gate_bias", **_gate(16384, 256, 8, score="sigmoid", normalize=True, scale=2.5, bias=True)},
        # the routing recipe of the layer's own benchmark (softmax over the experts, not renormalized)
        # with float32 logits, some experts masked out
        {"name": "gate_share", **_gate(16384, 32, 8, dtype="f32", masked=True)},
        # the gradient of a training batch's logits, every expert's through the softmax
        {"name": "gate_grad", **_gate(16384, 256, 8, bwd=True)},
        # the layer of the parity tests
        {"name": "sort_tiny", **_sort(1024, 256, 8, 2)},
        # one expert-parallel rank's tokens for experts that another library computes in bf16
        {"name": "sort_share", **_sort(16384, 7168, 32, 8)},
        # tokens that arrive already cast (FP8 dispatch), ragged, some routed to other ranks
        {"name": "sort_fp8", **_sort(5001, 7168, 32, 8, align=16, payload="fp8_e8m0", dropped=True)},
        # the weighted return's gradient at the same share
        {"name": "return_share", **_return(16384, 7168, 32, 8)},
        # and of a small ragged micro-batch on narrow experts with skewed routing
        {"name": "return_fine", **_return(517, 2048, 64, 6, align=16, routing="zipf", dropped=True)},
        # one token through the up projection and SwiGLU: eight experts' weights are the traffic
        {"name": "w4_one", **_w4("up", 1, 7168, 32, 8, 2048)},
        # a handful of sequences on many narrow experts, down projection
        {"name": "w4_fine", **_w4("down", 7, 2048, 64, 6, 1408)},
        # a decoding batch of 256 sequences: every expert, up to dozens of rows each
        {"name": "w4_batch", **_w4("up", 256, 7168, 32, 8, 2048)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gate", "gate", "sort", "return", "w4", "w4"])
    routing = rng.choice(["iid", "iid", "zipf"])
    align = rng.choice([16, 128])
    if kind == "gate":
        E = _log(rng, 4, 256)
        return _gate(_log(rng, 1, 16384), E, rng.randint(1, min(8, E)), dtype=rng.choice(["bf16", "f32"]),
                     score=rng.choice(["softmax", "sigmoid"]), normalize=rng.random() < 0.5,
                     scale=rng.choice([1.0, 2.5]), bias=rng.random() < 0.5, masked=rng.random() < 0.3,
                     bwd=rng.random() < 0.5)
    E = _log(rng, 4, 64)
    k = rng.randint(1, min(8, E))
    H = 128 * _log(rng, 1, 56)
    if kind == "sort":
        return _sort(_log(rng, 1, 16384), H, E, k, align=align, payload=rng.choice(["bf16", "fp8", "fp8_e8m0"]),
                     routing=routing, dropped=rng.random() < 0.3)
    if kind == "return":
        return _return(_log(rng, 1, 16384), H, E, k, align=align, routing=routing, dropped=rng.random() < 0.3,
                       dprobs=rng.random() < 0.7)
    I = 128 * _log(rng, 1, 16)
    E = min(E, 32) if H * I > 7168 * 1024 else E  # no more weights than the largest listed layer holds
    return _w4(rng.choice(["up", "down"]), _log(rng, 1, 256), H, E, min(k, E), I, routing=routing)


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, std, seed, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_gen(seed), device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _rows_bound(T, k, E, align):
    """Rows of the grouped buffers: every group is padded to a multiple of align, the whole to 128."""
    return -(-(T * k + (align - 1) * E) // 128) * 128


def _routing(c, seed):
    """Top-k experts of random logits (skewed: expert popularity ~ rank^-1.2), their softmax weights;
    dropped: one slot in twenty is an expert of another rank (-1)."""
    g = _gen(seed)
    T, E, k = c["T"], c["E"], c["k"]
    logits = torch.randn((T, E), generator=g, device="cuda")
    if c["routing"] == "zipf":
        p = (torch.randperm(E, generator=g, device="cuda").float() + 1.0) ** -1.2
        logits = torch.log(p / p.sum()) + 0.4 * logits
    idx = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    probs = torch.gather(torch.softmax(logits, dim=1), 1, idx)
    idx = idx.to(torch.int32)
    if c.get("dropped"):
        idx = torch.where(torch.rand((T, k), generator=g, device="cuda") < 0.05, -1, idx)
    return idx.contiguous(), probs.contiguous()


def _maps(idx, E, align, M_cap):
    """(row_map [T, k], offsets [E + 1], src_row [M_cap]): groups in expert order, padded to align,
    token order inside; -1 for dropped slots and for rows that hold no token."""
    T, k = idx.shape
    flat = idx.reshape(-1).long()
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True).indices
    counts = (flat[:, None] == torch.arange(E, device="cuda")).sum(0)
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    offsets = torch.cat([zero, torch.cumsum((counts + align - 1) // align * align, 0)])
    starts = torch.cat([zero, torch.cumsum(counts, 0)])
    e = flat[order]
    pos = torch.arange(T * k, device="cuda") - starts[e.clamp(min=0)] + offsets[e.clamp(min=0)]
    kept = e >= 0
    row_map = torch.full((T * k,), -1, dtype=torch.long, device="cuda")
    row_map[order] = torch.where(kept, pos, -1)
    # one entry past the end takes what is dropped
    src = torch.full((M_cap + 1,), -1, dtype=torch.long, device="cuda")
    src[torch.where(kept, pos, M_cap)] = torch.where(kept, order, -1)
    return row_map.view(T, k).int(), offsets.int(), src[:M_cap].int()


def _int_buffers(c, M_cap):
    full = lambda *shape: torch.full(shape, -1, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"row_map": full(c["T"], c["k"]), "offsets": full(c["E"] + 1), "src_row": full(M_cap)}


def prepare(case, seed):
    c, s = case, 16 * seed
    state = {"case": c}
    T, E, k = c["T"], c["E"], c["k"]
    if c["kind"] == "gate":
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        logits = _randn((T, E), 1.0, s + 1, torch.float32)
        if c["masked"]:  # experts that a row may not choose, now and then more than leave k
            hidden = torch.rand((T, E), generator=_gen(s + 2), device="cuda") < 0.25
            hidden[0] = True
            logits = logits.masked_fill(hidden, -math.inf)
        state["logits"] = logits.to(dt)
        state["bias"] = _randn((E,), 0.1, s + 3, torch.float32) if c["bias"] else None
        if c["bwd"]:
            state["topk_idx"] = _choose(state["logits"], state["bias"], c, torch.float64)
            state["dprobs"] = _randn((T, k), 1.0, s + 4, torch.float32)
            state["dlogits"] = torch.zeros((T, E), dtype=dt, device="cuda")
        else:
            state["topk_idx"] = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
            state["probs"] = torch.zeros((T, k), dtype=torch.float32, device="cuda")
        return state
    align = c.get("align", 16)
    M_cap = _rows_bound(T, k, E, align)
    idx, probs = _routing(c, s + 1)
    state.update(topk_idx=idx, probs=probs)
    if c["kind"] == "sort":
        H = c["H"]
        state.update(_int_buffers(c, M_cap))
        if c["payload"] == "bf16":
            state["x"] = _randn((T, H), 1.0, s + 2)
            state["out"] = torch.zeros((M_cap, H), dtype=torch.bfloat16, device="cuda")
        else:  # e4m3 bytes (no NaN codes) and power-of-two scales of 1x128 tiles
            b = torch.randint(0, 254, (T, H), generator=_gen(s + 2), device="cuda", dtype=torch.int32)
            state["xq"] = torch.where(b >= 127, b + 1, b).to(torch.uint8)
            t = torch.randint(-9, -5, (T, H // 128), generator=_gen(s + 3), device="cuda", dtype=torch.int32)
            e8m0 = c["payload"] == "fp8_e8m0"
            state["xs"] = (t + 127).to(torch.uint8) if e8m0 else torch.exp2(t.float())
            state["q"] = torch.zeros((M_cap, H), dtype=torch.uint8, device="cuda")
            state["s"] = torch.zeros((M_cap, H // 128), dtype=state["xs"].dtype, device="cuda")
        if own:
            from paper_2511_02302_amd import ff8
            n = max(4, ff8.ff8_permute_workspace_bytes(T, k, E))
            state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        return state
    state["row_map"], state["offsets"], state["src_row"] = _maps(idx, E, align, M_cap)
    if c["kind"] == "return":
        H = c["H"]
        state["dy"] = _randn((T, H), 1.0, s + 2)
        state["dy_perm"] = torch.zeros((M_cap, H), dtype=torch.bfloat16, device="cuda")
        state["y_perm"] = _randn((M_cap, H), 1.0, s + 3) if c["dprobs"] else None
        state["dprobs"] = torch.zeros((T, k), dtype=torch.float32, device="cuda") if c["dprobs"] else None
        return state
    H, I, up = c["H"], c["I"], c["part"] == "up"
    N, K = (2 * I, H) if up else (H, I)
    # MXFP4 as checkpoints hold it: two e2m1 codes a byte, the lower column in the low nibble, and one
    # UE8M0 byte for 32 columns; scales as weights of standard deviation 0.02 have them
    state["wq"] = torch.randint(0, 256, (E, N, K // 2), generator=_gen(s + 2), device="cuda", dtype=torch.uint8)
    state["ws"] = torch.randint(119, 122, (E, N, K // 32), generator=_gen(s + 3), device="cuda", dtype=torch.uint8)
    if up:
        state["x"] = _randn((T, K), 1.0, s + 4)
    else:  # the up projection's output: padding rows are zero
        state["x"] = _randn((M_cap, K), 1.0, s + 4).masked_fill_((state["src_row"] < 0)[:, None], 0.0)
    state["out"] = torch.zeros((M_cap, I if up else N), dtype=torch.bfloat16, device="cuda")
    if own:  # the kernel's tile order, laid out once when weights are loaded
        from paper_2511_02302_amd import ff8
        wq, ws = state.pop("wq"), state.pop("ws")
        state["tq"] = torch.empty((E, N // 16, K // 128, 64, 16), dtype=torch.uint8, device="cuda")
        state["ts"] = torch.empty((E, N // 16, K // 128, 64), dtype=torch.uint8, device="cuda")
        ff8.ff8_pack_mxfp4(wq, ws, state["tq"], state["ts"])
    return state


# ---- one pass ----

def run(state):
    c = state["case"]
    return (_own if own else _plain)[c["kind"]](c, state)


def _own_gate(c, s):
    from paper_2511_02302_amd import ff8
    opts = dict(score=c["score"], normalize=c["normalize"], scale=c["scale"])
    if c["bwd"]:
        ff8.ff8_router_topk_bwd(s["logits"], s["topk_idx"], s["dprobs"], s["dlogits"], **opts)
        return {"dlogits": s["dlogits"]}
    ff8.ff8_router_topk(s["logits"], s["topk_idx"], s["probs"], bias=s["bias"], **opts)
    return {"idx": s["topk_idx"], "probs": s["probs"]}


def _own_sort(c, s):
    from paper_2511_02302_amd import ff8
    maps = (c["k"], c["E"], s["topk_idx"], False, s["row_map"], s["offsets"], s["src_row"])
    if c["payload"] == "bf16":
        ff8.ff8_permute_bf16(s["x"], *maps, s["out"], s["workspace"], align=c["align"])
        out = {"x": s["out"]}
    else:
        ff8.ff8_permute_fp8(s["xq"], s["xs"], *maps, s["q"], s["s"], s["workspace"], align=c["align"])
        out = _fp8_values(s["q"], s["s"])
    return {**out, "row_map": s["row_map"], "offsets": s["offsets"], "src_row": s["src_row"]}


def _own_return(c, s):
    from paper_2511_02302_amd import ff8
    ff8.ff8_unpermute_bwd(s["dy"], s["probs"], c["k"], c["E"], s["row_map"], s["offsets"], s["src_row"],
                          s["dy_perm"], s["y_perm"], s["dprobs"])
    return {"dy_perm": s["dy_perm"], "dprobs": s["dprobs"]}


def _own_w4(c, s):
    from paper_2511_02302_amd import ff8
    if c["part"] == "up":
        ff8.ff8_grouped_gemv_mxfp4_swiglu(s["x"], s["tq"], s["ts"], s["offsets"], s["out"], src_row=s["src_row"],
                                          top_k=c["k"])
    else:
        ff8.ff8_grouped_gemv_mxfp4(s["x"], s["tq"], s["ts"], s["offsets"], s["out"], src_row=s["src_row"])
    return {"out": s["out"]}


def _fp8_values(q, s):
    """Bytes as the numbers they stand for (views): e4m3, and UE8M0 or float32 scales."""
    return {"q": q.view(torch.float8_e4m3fn), "s": s.view(torch.float8_e8m0fnu) if s.dtype is torch.uint8 else s}


def _scores(logits, c, dtype):
    """Each expert's score; a row without a selectable expert has scores of zero."""
    z = logits.to(dtype)
    if c["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(1, keepdim=True)
    return e / torch.where(total == 0.0, 1.0, total)


def _choose(logits, bias, c, dtype):
    """The k experts of the largest logits, or of the largest score + bias (in 64 bits: a rounding there
    would change an expert), ties to the lowest index; -1 where only masked experts are left."""
    key = logits.to(dtype) if bias is None else _scores(logits, c, dtype) + bias.to(dtype)
    key = torch.where(logits == -math.inf, -math.inf, key)
    top = torch.sort(key, dim=1, descending=True, stable=True)
    return torch.where(top.values[:, :c["k"]] == -math.inf, -1, top.indices[:, :c["k"]]).int()


def _weights(logits, idx, c, dtype):
    """Routing weights of the chosen experts, zero for -1."""
    kept = idx >= 0
    at = idx.long().clamp(min=0)
    if not c["normalize"]:
        p = torch.gather(_scores(logits, c, dtype), 1, at)
    else:  # over the chosen alone; through the logarithm, so that small scores do not divide zero by zero
        v = torch.gather(logits.to(dtype), 1, at)
        if c["score"] == "sigmoid":
            v = torch.clamp(v, max=0.0) - torch.log1p(torch.exp(-v.abs()))
        v = torch.where(kept, v, -math.inf)
        m = v.amax(1, keepdim=True)
        e = torch.exp(v - torch.where(m == -math.inf, 0.0, m))
        total = e.sum(1, keepdim=True)
        p = e / torch.where(total == 0.0, 1.0, total)
    return torch.where(kept, p * c["scale"], 0.0)


def _plain_gate(c, s):
    logits = s["logits"]
    if not c["bwd"]:
        idx = _choose(logits, s["bias"], c, torch.float32 if s["bias"] is None else torch.float64)
        return {"idx": idx, "probs": _weights(logits, idx, c, torch.float32)}
    idx, dp = s["topk_idx"], s["dprobs"]
    kept = idx >= 0
    at = idx.long().clamp(min=0)
    z = logits.float()
    dp = torch.where(kept, dp, 0.0)
    spread = lambda v: torch.zeros_like(z).scatter_add_(1, at, torch.where(kept, v, 0.0))  # noqa: E731
    if c["normalize"]:
        r = _weights(logits, idx, c, torch.float32)
        dv = r * (dp - (r * dp).sum(1, keepdim=True) / c["scale"])
        if c["score"] == "sigmoid":
            dv = dv / (1.0 + torch.exp(torch.gather(z, 1, at)))
        d = spread(dv)
    else:
        p = _scores(logits, c, torch.float32)
        chosen = torch.gather(p, 1, at) * dp
        if c["score"] == "sigmoid":
            d = spread(chosen * c["scale"] / (1.0 + torch.exp(torch.gather(z, 1, at))))
        else:
            d = c["scale"] * (spread(chosen) - p * torch.where(kept, chosen, 0.0).sum(1, keepdim=True))
    return {"dlogits": d.to(logits.dtype)}


def _plain_sort(c, s):
    row_map, offsets, src = _maps(s["topk_idx"], c["E"], c["align"], s["src_row"].numel())
    real = (src >= 0)[:, None]
    token = src.clamp(min=0).long() // c["k"]
    if c["payload"] == "bf16":
        out = {"x": torch.where(real, s["x"][token], 0.0)}
    else:
        q = torch.where(real, s["xq"][token], 0)
        low = 127 + _TMIN if s["xs"].dtype is torch.uint8 else 2.0 ** _TMIN
        used = (torch.arange(src.numel(), device="cuda") < offsets[-1])[:, None]
        out = _fp8_values(q, torch.where(real, s["xs"][token], torch.where(used, low, 0).to(s["xs"].dtype)))
    return {**out, "row_map": row_map, "offsets": offsets, "src_row": src}


def _plain_return(c, s):
    src = s["src_row"]
    at = src.clamp(min=0).long()
    w = torch.where(src >= 0, s["probs"].reshape(-1)[at], 0.0)
    dy_perm = (w[:, None] * s["dy"][at // c["k"]].float()).to(torch.bfloat16)
    if not c["dprobs"]:
        return {"dy_perm": dy_perm, "dprobs": None}
    rows = s["row_map"]
    dots = (s["y_perm"][rows.clamp(min=0).long()].float() * s["dy"][:, None, :].float()).sum(2)
    return {"dy_perm": dy_perm, "dprobs": torch.where(rows >= 0, dots, 0.0)}


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _dequant(wq, ws):
    """[E, N, K] float32 weights of the codes and scales (exact)."""
    E, N, half = wq.shape
    both = torch.tensor([[_E2M1[b & 15], _E2M1[b >> 4]] for b in range(256)], dtype=torch.float32, device="cuda")
    w = both[wq.int()].view(E, N, half // 16, 32)
    return w.mul_(torch.exp2(ws.float() - 127.0)[..., None]).view(E, N, 2 * half)


def _plain_w4(c, s):
    E, T, src, offsets = c["E"], c["T"], s["src_row"], s["offsets"].long()
    M_cap = src.numel()
    row = torch.arange(M_cap, device="cuda")
    e = torch.searchsorted(offsets, row, right=True) - 1  # E for the rows behind the last group
    real = (src >= 0) & (e < E)
    x = s["x"][src.clamp(min=0).long() // c["k"]] if c["part"] == "up" else s["x"]
    # an expert has at most T rows: [E, T + 1, K], the last row of each takes what holds no token
    slot = torch.where(real, row - offsets[e.clamp(max=E - 1)], T)
    a = torch.zeros((E, T + 1, x.shape[1]), dtype=torch.float32, device="cuda")
    a[e.clamp(max=E - 1), slot] = x.float()
    y = torch.bmm(a, _dequant(s["wq"], s["ws"]).transpose(1, 2).contiguous())[e.clamp(max=E - 1), slot]
    if c["part"] == "up":
        gate, up = y[:, :c["I"]], y[:, c["I"]:]
        y = gate / (1.0 + torch.exp(-gate)) * up
    return {"out": torch.where(real[:, None], y, 0.0).to(torch.bfloat16)}


_own = {"gate": _own_gate, "sort": _own_sort, "return": _own_return, "w4": _own_w4}
_plain = {"gate": _plain_gate, "sort": _plain_sort, "return": _plain_return, "w4": _plain_w4}


# ---- the definition in 64 bits ----

def exact(case, seed):
    c = case
    if c["kind"] == "sort":
        return None  # rows are moved, nothing is computed
    with _without_own():
        s = prepare(case, seed)
    if c["kind"] == "gate":
        return _exact_gate(c, s)
    if c["kind"] == "return":
        dy, w = s["dy"].double(), s["probs"].double()
        out = torch.zeros(s["dy_perm"].shape, dtype=torch.float64, device="cuda")
        dprobs = torch.zeros(w.shape, dtype=torch.float64, device="cuda")
        for j in range(c["k"]):
            t = (s["row_map"][:, j] >= 0).nonzero()[:, 0]
            rows = s["row_map"][t, j].long()
            out[rows] = dy[t] * w[t, j, None]
            if c["dprobs"]:
                dprobs[t, j] = (dy[t] * s["y_perm"][rows].double()).sum(1)
        return {"dy_perm": out, "dprobs": dprobs if c["dprobs"] else None}
    values = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    starts = s["offsets"].tolist()
    for e in range(c["E"]):
        rows = torch.arange(starts[e], starts[e + 1], device="cuda")
        rows = rows[s["src_row"][rows] >= 0]
        if rows.numel() == 0:
            continue
        codes = s["wq"][e].long()
        w = torch.stack([values[codes % 16], values[codes // 16]], 2).reshape(codes.shape[0], -1)
        w = w * torch.pow(2.0, s["ws"][e].double() - 127.0).repeat_interleave(32, 1)
        x = s["x"][s["src_row"][rows].long() // c["k"]] if c["part"] == "up" else s["x"][rows]
        y = x.double() @ w.t().contiguous()
        if c["part"] == "up":
            y = y[:, :c["I"]] * torch.sigmoid(y[:, :c["I"]]) * y[:, c["I"]:]
        out[rows] = y
    return {"out": out}


class _without_own:
    """The inputs as the plain form takes them, whichever side asks."""

    def __enter__(self):
        global own
        self.kept, own = own, False

    def __exit__(self, *_):
        global own
        own = self.kept


def _exact_gate(c, s):
    z = s["logits"].double()
    idx = s["topk_idx"] if c["bwd"] else _choose(s["logits"], s["bias"], c, torch.float64)
    z = z.requires_grad_(c["bwd"])
    kept = idx >= 0
    picked = torch.gather(z, 1, idx.long().clamp(min=0))
    if c["normalize"]:
        v = torch.nn.functional.logsigmoid(picked) if c["score"] == "sigmoid" else picked
        v = v.masked_fill(~kept, -math.inf)
        some = kept.any(1, keepdim=True)
        p = torch.softmax(v.masked_fill(~some, 0.0), 1)
    elif c["score"] == "sigmoid":
        p = torch.sigmoid(picked)
    else:
        none = (z == -math.inf).all(1, keepdim=True)
        p = torch.gather(torch.softmax(z.masked_fill(none, 0.0), 1), 1, idx.long().clamp(min=0))
    p = (p * c["scale"]).masked_fill(~kept, 0.0)
    if not c["bwd"]:
        return {"idx": None, "probs": p}
    (g,) = torch.autograd.grad(p, z, s["dprobs"].double().masked_fill(~kept, 0.0))
    return {"dlogits": torch.nan_to_num(g, nan=0.0)}


# ---- what a pass cannot do without ----

def work(case):
    c = case
    T, E, k = c["T"], c["E"], c["k"]
    if c["kind"] == "gate":
        size = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": T * E * size * (2 if c["bwd"] else 1) + 8 * T * k, "flops": 4.0 * T * E}
    rows = T * k * (0.95 if c.get("dropped") else 1.0)
    if c["kind"] == "sort":
        per_row = 2 * c["H"] if c["payload"] == "bf16" else c["H"] + c["H"] // 128 * (4 if c["payload"] == "fp8" else 1)
        return {"bytes": (T + rows) * per_row + 12 * T * k, "flops": 0.0}
    if c["kind"] == "return":
        H = c["H"]
        return {"bytes": 2 * H * (T + rows * (2 if c["dprobs"] else 1)) + 12 * T * k,
                "flops": rows * H * (3 if c["dprobs"] else 1)}
    H, I = c["H"], c["I"]
    N, K, n_out = (2 * I, H, I) if c["part"] == "up" else (H, I, H)
    experts = E * (1.0 - (1.0 - k / E) ** T)  # that some token chooses, by evenly spread routing
    n_in = T if c["part"] == "up" else rows
    return {"bytes": experts * N * K * 17 / 32 + 2 * (n_in * K + rows * n_out), "flops": 2.0 * rows * N * K}
