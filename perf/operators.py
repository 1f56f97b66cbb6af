"""The operators of a decode step with 4-bit microscaled weights and routed experts, as cases.

op              what one pass calls
  pack          a projection's bf16 weights to microscaled 4-bit numbers, and back to bf16 values
  project       1 to 4 matrices of such weights on one hidden state, y_k = s_{t_k}(x) W_k^T
  down          W_down of such weights on h = fp16(SiLU(gate) * up), formed in the call
  route         top-k experts and their weights from the router's logits
  experts       gate and up of the experts that the router chose for each token of a small batch
  experts_down  W_down of those experts on h, summed over a token's experts with the router's weights

Microscaled weights: blocks of 32 neighbouring outputs of one input channel share a power of two X, a value
is X times one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign.  Codes are [m][n/2] bytes (low nibble = even
output), scales one byte per block, 127 + log2 X, in tiles of 8 channels by 16 blocks (_scale_rows).
fmt is the weight format of the experts (bf16 or mx4); p is the share of input channels that are dropped.
"""
import math

import numpy as np
import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32                       # outputs of a channel that share a scale
TILE_ROWS, TILE_BLOCKS = 8, 16   # a tile of scales: 128 bytes


def _case(name, op, **kw):
    return {"name": name, "op": op, **kw}


def listed():
    return [
        # laying out one key projection with grouped-query heads when a model is loaded: the smallest matrix
        _case("pack_kv", "pack", m=4096, n=1024),
        # the largest matrix: the gate projection of a 70B-shaped block
        _case("pack_gate_70b", "pack", m=8192, n=28672),
        # the smallest product of a decode step: a square projection of a small model
        _case("project_2048", "project", m=2048, n="2048", p=0.5),
        # sizes that divide into nothing, most channels dropped
        _case("project_ragged", "project", m=5001, n="3424 416", p=0.8),
        # gate and up of a 70B-shaped block: the most bytes of a decode step
        _case("gate_up_70b", "project", m=8192, n="28672 28672", p=0.5),
        # W_down of an 8B-shaped block on its gated intermediate
        _case("down_8b", "down", m=14336, n=4096, p=0.5),
        # one token of a decode step: softmax over a few experts
        _case("route_token", "route", tokens=1, experts=64, groups=1, top_groups=1, group_top=1, top_k=6,
              score="softmax", bias=False, renormalise=False),
        # a long prompt: sigmoid scores, a bias for balance, groups of experts
        _case("route_prompt", "route", tokens=16384, experts=256, groups=8, top_groups=4, group_top=2, top_k=8,
              score="sigmoid", bias=True, renormalise=True),
        # one token, two of eight large experts
        _case("experts_large", "experts", fmt="bf16", tokens=1, padded=0, experts=8, top_k=2, m=4096, n=14336, p=0.5),
        _case("experts_large_down", "experts_down", fmt="bf16", tokens=1, padded=0, experts=8, top_k=2, m=14336,
              n=4096, p=0.5),
        # a small batch, one of its rows padding, and many small experts
        _case("experts_small_batch", "experts", fmt="mx4", tokens=8, padded=1, experts=128, top_k=8, m=2048, n=768,
              p=0.5),
        _case("experts_small_batch_down", "experts_down", fmt="mx4", tokens=8, padded=1, experts=128, top_k=8, m=768,
              n=2048, p=0.5),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _step(v, k):
    return max(k, int(v) // k * k)


def draw(rng):
    op = rng.choice(["pack", "project", "project", "down", "route", "route", "experts", "experts_down"])
    unit = rng.choice([BLOCK, BLOCK, 128])
    p = rng.choice([0.0, 0.25, 0.4, 0.5, 0.5, 0.65, 0.8, 0.95])
    if op == "pack":
        return {"op": op, "m": int(_log(rng, 200, 8192)), "n": _step(_log(rng, 64, 16384), unit)}
    if op == "project":
        n = [_step(_log(rng, 64, 16384), unit) for _ in range(rng.choice([1, 1, 2, 3, 4]))]
        return {"op": op, "m": int(_log(rng, 200, 8192)), "n": " ".join(map(str, n)), "p": p}
    if op == "down":
        return {"op": op, "m": int(_log(rng, 500, 28672)), "n": _step(_log(rng, 256, 8192), unit), "p": p}
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        size = rng.choice([4, 8, 11, 16, 32])
        top_groups = rng.randint(1, groups)
        return {"op": op, "tokens": int(_log(rng, 1, 8192)), "experts": groups * size, "groups": groups,
                "top_groups": top_groups, "group_top": rng.choice([1, 2]),
                "top_k": min(top_groups * size, rng.choice([1, 2, 4, 6, 8])),
                "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5,
                "renormalise": rng.random() < 0.5}
    fmt = rng.choice(["bf16", "mx4"])
    tokens = rng.randint(1, 8)
    experts = rng.choice([8, 16, 60, 128])
    top_k = rng.choice([1, 2, 4, 6, 8])
    wide, narrow = int(_log(rng, 512, 2048)), _step(_log(rng, 256, 1536), unit)
    if op == "experts_down":
        wide, narrow = narrow, _step(wide, unit)
    return {"op": op, "fmt": fmt, "tokens": tokens, "padded": rng.randint(0, tokens - 1), "experts": experts,
            "top_k": top_k, "m": wide, "n": narrow, "p": p}


# ---- inputs ----------------------------------------------------------------------------------------


def _scale_rows(scale, m, n):
    """One scale byte per channel and block, [..., m, n / 32], from their tiles."""
    tiles = scale.reshape(*scale.shape[:-1], -1, -(-n // (BLOCK * TILE_BLOCKS)), TILE_ROWS, TILE_BLOCKS)
    rows = tiles.transpose(-3, -2).flatten(-2).flatten(-3, -2)
    return rows[..., :m, :n // BLOCK]


def _scale_tiles(rows):
    """The tiles of [..., m, n / 32] scale bytes, zeros past the last channel and block."""
    m, blocks = rows.shape[-2:]
    rows = torch.nn.functional.pad(rows, (0, -blocks % TILE_BLOCKS, 0, -m % TILE_ROWS))
    tiles = rows.unflatten(-1, (-1, TILE_BLOCKS)).unflatten(-3, (-1, TILE_ROWS)).transpose(-3, -2)
    return tiles.flatten(-4).contiguous()


def _weights_mx4(gen, *shape):
    """Random microscaled weights, [..., m, n] of about 0.02 each: (codes, scales)."""
    *lead, m, n = shape
    # the magnitudes of normal numbers in blocks of 32 scaled by their largest, as a table of 64 likely codes
    table = torch.tensor([0] * 9 + [1] * 15 + [2] * 12 + [3] * 9 + [4] * 9 + [5] * 6 + [6] * 3 + [7],
                         dtype=torch.uint8, device="cuda")
    pick = torch.randint(0, 256, (*lead, m, n // 2), generator=gen, device="cuda", dtype=torch.uint8)
    codes = table[(pick & 63).int()] | (pick & 64) >> 3
    pick = torch.randint(0, 256, pick.shape, generator=gen, device="cuda", dtype=torch.uint8)
    codes |= (table[(pick & 63).int()] | (pick & 64) >> 3) << 4
    rows = 119 + torch.randint(0, 3, (*lead, m, n // BLOCK), generator=gen, device="cuda", dtype=torch.uint8)
    return codes, _scale_tiles(rows)


def _widths(case):
    """The output widths of a case of products, one per matrix."""
    return [int(n) for n in str(case["n"]).split()]


def _threshold(x, p):
    """A threshold that drops about the share p of the entries of x."""
    a = x.float().abs().flatten()
    return float(a.kthvalue(max(1, round(p * a.numel()))).values) if p > 0 else 0.0


def _swiglu_f16(gate, up):
    """fp16(SiLU(gate) * up) in the binary32 operations that the library states for it: the value decides
    which channels are dropped, so it is formed with exactly these.  (A product and a sum in binary64, rounded
    to binary32, are the fused multiply-add.)"""
    def fma(a, b, c):
        return (a.double() * float(np.float32(b)) + c).float()

    def horner(p, r, c):
        return (p.double() * r.double() + float(np.float32(1) / np.float32(c))).float()

    z = (-gate).clamp(-80.0, 80.0)
    k = (z * float(np.float32(1.44269502))).round()
    r = fma(k, -1.42860677e-06, fma(k, -0.693145752, z.double()).double())
    p = torch.full_like(r, float(np.float32(1) / np.float32(5040)))
    p = horner(horner(horner(p, r, 720), r, 120), r, 24)
    p = horner(horner(horner(horner(p, r, 6), r, 2), r, 1), r, 1)
    e = (p.double() * torch.exp2(k.double())).float()
    sigma = (1.0 / (1.0 + e).double()).float()
    return (gate * sigma * up).half()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c = case

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    st = dict(case)
    if c["op"] == "pack":
        m, n = c["m"], c["n"]
        # channels of different sizes, as in weights that follow a normalisation
        st["W"] = (normal(n, m) * (0.02 * torch.exp2(2 * uniform(m)))).bfloat16()
        st["codes"] = torch.empty(m, n // 2, dtype=torch.uint8, device="cuda")
        st["scale"] = torch.empty(-(-m // TILE_ROWS) * -(-n // (BLOCK * TILE_BLOCKS)) * TILE_ROWS * TILE_BLOCKS,
                                  dtype=torch.uint8, device="cuda")
        st["out"] = torch.empty_like(st["W"])
        return st
    if c["op"] == "route":
        tokens, experts = c["tokens"], c["experts"]
        st["logits"] = normal(tokens, experts) * 1.5
        st["bias_values"] = normal(experts) * 0.05 if c["bias"] else None
        st["idx"] = torch.empty(tokens, c["top_k"], dtype=torch.int32, device="cuda")
        st["weight"] = torch.empty(tokens, c["top_k"], device="cuda")
        return st

    # a decode program's scratch, zero before its first use
    st["workspace"] = torch.zeros(96 << 20, dtype=torch.uint8, device="cuda")
    m = c["m"]
    if c["op"] in ("project", "down"):
        st["n"] = widths = _widths(c)
        st["weights"] = [_weights_mx4(gen, m, n) for n in widths]
        st["y"] = [torch.empty(n, device="cuda") for n in widths]
        if c["op"] == "project":
            st["x"] = normal(m).half()
            st["t"] = [_threshold(st["x"], c["p"]) * (1 + 0.1 * k) for k in range(len(widths))]
        else:
            st["gate"], st["up"] = 1.5 * normal(m), normal(m)
            st["t"] = _threshold(_swiglu_f16(st["gate"], st["up"]), c["p"])
        return st

    tokens, experts, top_k, n = c["tokens"], c["experts"], c["top_k"], c["n"]
    count = 2 if c["op"] == "experts" else 1
    if c["fmt"] == "mx4":
        st["weights"] = [_weights_mx4(gen, experts, m, n) for _ in range(count)]
    else:
        st["weights"] = [0.02 * normal(experts, m, n, dtype=torch.bfloat16) for _ in range(count)]
    idx = uniform(tokens, experts).argsort(-1)[:, :top_k].int()
    idx[tokens - c["padded"]:] = -1                       # rows of padding have no experts
    st["idx"] = idx.contiguous()
    if c["op"] == "experts":
        st["x"] = normal(tokens, m).half()
        base = _threshold(st["x"], c["p"])
        st["y"] = [torch.empty(tokens, top_k, n, device="cuda") for _ in range(count)]
    else:
        st["gate"], st["up"] = 1.5 * normal(tokens, top_k, m), normal(tokens, top_k, m)
        base = _threshold(_swiglu_f16(st["gate"], st["up"]), c["p"])
        weight = uniform(tokens, top_k) + 0.1
        st["weight"] = (weight / weight.sum(-1, keepdim=True)).contiguous()
        st["y"] = [torch.empty(tokens, n, device="cuda")]
    st["t"] = [base * (0.9 + 0.2 * uniform(experts)) for _ in range(count)]     # every expert its own
    return st


# ---- one pass --------------------------------------------------------------------------------------


def run(st):
    if own:
        return _own(st)
    op = st["op"]
    if op == "pack":
        return _plain_pack(st["W"])
    if op == "project":
        return [_plain_product(st["x"], t, _values_mx4(*w, st["m"])) for t, w in zip(st["t"], st["weights"])]
    if op == "down":
        return _plain_product(_swiglu_f16(st["gate"], st["up"]), st["t"], _values_mx4(*st["weights"][0], st["m"]))
    if op == "route":
        return _plain_route(st)
    if op == "experts":
        x = st["x"][:, None].expand(-1, st["top_k"], -1)
        return [_plain_experts(st, x, t, w) for t, w in zip(st["t"], st["weights"])]
    y = _plain_experts(st, _swiglu_f16(st["gate"], st["up"]), st["t"][0], st["weights"][0])
    return (y * st["weight"][..., None]).sum(1)


def _own(st):
    import paper_2408_14690_amd as T

    op, m, n = st["op"], st.get("m"), st.get("n")
    if op == "pack":
        T.check(T.teal_pack_mx4(st["W"], st["codes"], st["scale"], m, n))
        T.check(T.teal_unpack_mx4(st["codes"], st["scale"], st["out"], m, n))
        return st["out"]
    if op == "project":
        codes, scales = zip(*st["weights"])
        if len(n) == 1:
            T.check(T.teal_sparse_gemv_mx4(codes[0], scales[0], st["x"], st["t"][0], st["y"][0], m, n[0],
                                           st["workspace"]))
        else:
            T.check(T.teal_sparse_gemv_mx4_multi(codes, scales, st["t"], st["y"], n, st["x"], m, st["workspace"]))
        return st["y"]
    if op == "down":
        codes, scale = st["weights"][0]
        T.check(T.teal_sparse_gemv_mx4_swiglu(codes, scale, st["gate"], st["up"], st["t"], st["y"][0], m,
                                              n[0], st["workspace"]))
        return st["y"][0]
    if op == "route":
        T.check(T.teal_route_experts(
            st["logits"], st["bias_values"], T.TEAL_SCORE_SIGMOID if st["score"] == "sigmoid" else T.TEAL_SCORE_SOFTMAX,
            st["tokens"], st["experts"], st["groups"], st["top_groups"], st["group_top"], st["top_k"],
            st["renormalise"], 2.5, st["idx"], st["weight"]))
        return st["idx"], st["weight"]
    tokens, experts, top_k = st["tokens"], st["experts"], st["top_k"]
    if op == "experts":
        if st["fmt"] == "mx4":
            codes, scales = zip(*st["weights"])
            T.check(T.teal_sparse_experts_mx4(codes, scales, st["t"], st["y"], [n, n], experts, st["idx"], tokens,
                                              top_k, st["x"], m, st["workspace"]))
        else:
            T.check(T.teal_sparse_experts_bf16(st["weights"], st["t"], st["y"], [n, n], experts, st["idx"], tokens,
                                               top_k, st["x"], m, st["workspace"]))
        return st["y"]
    if st["fmt"] == "mx4":
        codes, scale = st["weights"][0]
        T.check(T.teal_sparse_experts_mx4_swiglu(codes, scale, st["t"][0], st["y"][0], experts, st["idx"],
                                                 st["weight"], tokens, top_k, st["gate"], st["up"], m, n,
                                                 st["workspace"]))
    else:
        T.check(T.teal_sparse_experts_bf16_swiglu(st["weights"][0], st["t"][0], st["y"][0], experts, st["idx"],
                                                  st["weight"], tokens, top_k, st["gate"], st["up"], m, n,
                                                  st["workspace"]))
    return st["y"][0]


def _plain_pack(W):
    w = W.float().unflatten(0, (-1, BLOCK))
    largest = w.abs().amax(1, keepdim=True)
    exponent = (torch.frexp(largest).exponent - 3).clamp(min=-127)          # floor(log2 largest) - 2
    x = torch.exp2(torch.where(largest > 0, exponent, -127).float())
    a = w.abs() / x
    # to the nearest of LEVELS, ties to the one with an even code
    q = (0.5 * ((a > 0.25).float() + (a >= 0.75) + (a > 1.25) + (a >= 1.75)) + ((a > 2.5).float() + (a >= 3.5))
         + 2 * (a > 5).float())
    return (torch.copysign(q, w) * x).flatten(0, 1).bfloat16()


def _values_mx4(codes, scale, m):
    """[..., m, n] weights in 32 bits."""
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    n = 2 * codes.shape[-1]
    values = levels[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    x = torch.exp2(_scale_rows(scale, m, n).float() - 127)
    return (values.unflatten(-1, (-1, BLOCK)) * x[..., None]).flatten(-2)


def _plain_product(x, t, W):
    x = x.float()
    return torch.where(x.abs() > t, x, 0.0) @ W


def _plain_experts(st, x, t, weights):
    """s_t(x) W^T of every token's experts, [tokens][top_k][n]; zeros where there is none."""
    idx = st["idx"].flatten().long()
    chosen = idx.clamp(min=0)
    W = _values_mx4(*(w[chosen] for w in weights), st["m"]) if st["fmt"] == "mx4" else weights[chosen].float()
    x = x.float().flatten(0, 1)
    x = torch.where((x.abs() > t[chosen][:, None]) & (idx >= 0)[:, None], x, 0.0)
    return torch.bmm(x[:, None], W).reshape(st["tokens"], st["top_k"], -1)


def _plain_route(st):
    # in 64 bits: scores next to each other decide which expert is chosen
    z = st["logits"].double()
    if st["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-z))
    else:
        score = torch.exp(z - z.amax(-1, keepdim=True))
        score = score / score.sum(-1, keepdim=True)
    biased = score if st["bias_values"] is None else score + st["bias_values"].double()
    order = z if st["bias_values"] is None else biased
    if st["groups"] > 1:
        size = st["experts"] // st["groups"]
        ranked = (order if st["group_top"] == 1 else biased).unflatten(-1, (-1, size)).sort(-1, descending=True).values
        value = ranked[..., :st["group_top"]].sum(-1)
        best = value.sort(dim=-1, descending=True, stable=True).indices[:, :st["top_groups"]]
        taken = torch.zeros_like(value).scatter(-1, best, 1.0) > 0
        order = torch.where(taken.repeat_interleave(size, -1), order, -math.inf)
    idx = order.sort(dim=-1, descending=True, stable=True).indices[:, :st["top_k"]]
    weight = score.gather(-1, idx)
    if st["renormalise"]:
        weight = weight / weight.sum(-1, keepdim=True)
    return idx.int(), (weight * 2.5).float()


# ---- what a pass cannot do without -------------------------------------------------------------------


def work(case):
    c, op = case, case["op"]
    if op == "pack":
        weights = c["m"] * c["n"]
        # the codes and scales of the one call are the input of the other
        return {"bytes": round(weights * (2 + 2 + 2 * (0.5 + 1 / BLOCK))), "flops": 4 * weights}
    if op == "route":
        scores = c["tokens"] * c["experts"]
        return {"bytes": 4 * scores + 8 * c["tokens"] * c["top_k"] + 4 * c["experts"] * c["bias"], "flops": 8 * scores}
    keep = 1 - c["p"]
    per_weight = 2 if c.get("fmt") == "bf16" else 0.5 + 1 / BLOCK
    if op in ("project", "down"):
        outputs = sum(_widths(c))
        inputs = 2 * c["m"] if op == "project" else 8 * c["m"]
        weights = keep * c["m"] * outputs
        return {"bytes": round(weights * per_weight + inputs + 4 * outputs), "flops": round(2 * weights)}
    rows = c["tokens"] - c["padded"]
    pairs = rows * c["top_k"]
    weights = keep * c["m"] * c["n"] * (2 if op == "experts" else 1)
    # an expert's rows are read once for the tokens that share it: the union of what they keep
    shared = weights / keep * c["experts"] * (1 - (1 - keep * c["top_k"] / c["experts"]) ** rows)
    if op == "experts":
        other = 2 * rows * c["m"] + 8 * c["tokens"] * c["top_k"] * c["n"]
    else:
        other = 8 * pairs * c["m"] + 4 * c["tokens"] * c["n"]
    return {"bytes": round(shared * per_weight + other), "flops": round(2 * weights * pairs)}


# ---- in 64 bits, from the definitions ------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    op = st["op"]
    if op == "pack":
        return _exact_pack(st["W"])
    if op == "route":
        return _exact_route(st)
    if op == "project":
        return [_exact_product(st["x"], t, *w) for t, w in zip(st["t"], st["weights"])]
    if op == "down":
        h = _exact_swiglu(st["gate"], st["up"])
        return _exact_product(h, st["t"], *st["weights"][0])
    outs = []
    state = st["x"] if op == "experts" else _exact_swiglu(st["gate"], st["up"])
    for t, w in zip(st["t"], st["weights"]):
        y = torch.zeros(st["tokens"], st["top_k"], st["n"], dtype=torch.float64, device="cuda")
        for b, row in enumerate(st["idx"].tolist()):
            for k, e in enumerate(row):
                if e >= 0:
                    x = state[b] if op == "experts" else state[b, k]
                    y[b, k] = _exact_product(x, float(t[e]), *((w[e],) if st["fmt"] == "bf16" else (w[0][e], w[1][e])))
        outs.append(y)
    if op == "experts":
        return outs
    return torch.einsum("bkn,bk->bn", outs[0].cpu(), st["weight"].double().cpu())


def _power64(e):
    return (e + 1023 << 52).view(torch.float64)           # a power function may be off in the last place


def _exact_pack(W):
    out = torch.empty(W.shape, dtype=torch.float64, device=W.device)
    step = max(BLOCK, (1 << 25) // W.shape[1] // BLOCK * BLOCK)
    for j in range(0, W.shape[0], step):
        w = W[j:j + step].double().unflatten(0, (-1, BLOCK))
        # the exponents as they are stored: of normal numbers, which the inputs of the cases are
        top = (W[j:j + step].view(torch.int16) >> 7 & 255).unflatten(0, (-1, BLOCK)).amax(1, keepdim=True)
        x = _power64(top.long() - 127 - 2)
        ratio, best, off = w.abs() / x, torch.zeros_like(w), torch.full_like(w, math.inf)
        for level in (0, 1, 2, 4, 0.5, 1.5, 3, 6):
            even = level in (0, 1, 2, 4)                  # its code is: a tie goes there
            d = (ratio - level).abs()
            better = (d < off) | (d == off) & even
            best, off = torch.where(better, torch.full_like(w, level), best), torch.where(better, d, off)
        out[j:j + step] = (w.sign() * best * x).flatten(0, 1)
    return out


def _exact_product(x, t, weights, scale=None):
    kept = torch.nonzero(x.double().abs() > t).flatten()
    if scale is None:
        return x[kept].double() @ weights[kept].double()
    m, n = x.numel(), 2 * weights.shape[-1]
    nibbles = torch.empty(kept.numel(), n, dtype=torch.uint8, device=x.device)
    nibbles[:, 0::2], nibbles[:, 1::2] = weights[kept] & 15, weights[kept] >> 4
    e, f = (nibbles >> 1 & 3).double(), (nibbles & 1).double()
    value = torch.where(e > 0, (1 + f / 2) * _power64(e.long() - 1), f / 2) * (1 - 2.0 * (nibbles >> 3))
    block = torch.arange(n, device=x.device) // BLOCK
    at = ((kept // TILE_ROWS)[:, None] * -(-n // 512) + block // TILE_BLOCKS) * (TILE_ROWS * TILE_BLOCKS)
    at = at + (kept % TILE_ROWS)[:, None] * TILE_BLOCKS + block % TILE_BLOCKS
    return x[kept].double() @ (value * _power64(scale[at].long() - 127))


def _exact_swiglu(gate, up):
    """The stated binary32 operations, in numpy: fused multiply-adds as products and sums in binary64."""
    f, d = np.float32, np.float64
    g, u = gate.cpu().numpy(), up.cpu().numpy()
    z = np.clip(-g, f(-80), f(80))
    k = np.rint(z * f(1.44269502))
    r = (d(f(-0.693145752)) * k + z).astype(f)
    r = (d(f(-1.42860677e-06)) * k + r).astype(f)
    p = np.full_like(r, f(1) / f(5040))
    for c in (720, 120, 24, 6, 2, 1, 1):
        p = (p.astype(d) * r + d(f(1) / f(c))).astype(f)
    e = np.ldexp(p, k.astype(np.int32))
    h = g * (f(1) / (f(1) + e)) * u
    return torch.from_numpy(h.astype(np.float16)).to(gate.device)


def _exact_route(st):
    z = st["logits"].cpu().numpy().astype(np.float64)
    score = 1 / (1 + np.exp(-z)) if st["score"] == "sigmoid" else np.exp(z - z.max(-1, keepdims=True))
    if st["score"] == "softmax":
        score /= score.sum(-1, keepdims=True)
    biased = score if st["bias_values"] is None else score + st["bias_values"].cpu().numpy().astype(np.float64)
    order = (z if st["bias_values"] is None else biased).copy()
    tokens, size = z.shape[0], st["experts"] // st["groups"]
    value = np.sort((order if st["group_top"] == 1 else biased).reshape(tokens, -1, size), -1)
    rank = np.argsort(-value[..., -st["group_top"]:].sum(-1), -1, kind="stable").argsort(-1)
    order[np.repeat(rank >= st["top_groups"], size, -1)] = -np.inf
    idx = np.argsort(-order, -1, kind="stable")[:, :st["top_k"]]
    weight = np.take_along_axis(score, idx, -1)
    if st["renormalise"]:
        weight = weight / weight.sum(-1, keepdims=True)
    return idx.astype(np.int32), weight * 2.5
