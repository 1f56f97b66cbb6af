"""Microscaled weights, routing and experts' products without a GPU: the quantiser's recipe, the sizes, and every
refusal (all are decided on the host before any GPU work)."""
import math

import numpy as np
import pytest

import paper_2408_14690_amd as T
import teal_inputs as ti
from test_abi import BIG, SC, W, WS, X, Y, _built  # noqa: F401

G, U, I = 0x60000, 0x70000, 0x80000       # further fake device addresses


def bits(values):
    return ti.f32_to_bf16_bits(np.array(values, np.float32))


def test_quantiser_rounds_to_the_nearest_level_with_ties_to_the_even_code():
    # the largest weight is 4 X with X = 1, so ratios are the weights themselves
    w = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 7.9375, -6.0, 0.26, 0.74, 1.26, 0.0] + 15 * [0.0]
    want = [4, 0, 1, 1, 2, 2, 4, 4, 0, -1, -4, 6, -6, 0.5, 0.5, 1.5, 0] + 15 * [0]
    codes, scales = ti.quantize_mx4(bits(w)[:, None])
    assert scales[0] == 127 and ti.mx4_values(codes, scales)[0].tolist() == want


def test_quantiser_scales():
    for value, byte in [(4.0, 127), (7.96875, 127), (8.0, 128), (0.02, 127 - 6 - 2), (2.0 ** -125, 0), (2.0 ** -130, 0),
                        (0.0, 0), (2.0 ** 127, 252), (math.inf, 255), (math.nan, 255)]:
        w = np.zeros((32, 1), np.uint16)
        w[5] = np.frombuffer(np.float32(value).tobytes(), np.uint16)[1]
        codes, scales = ti.quantize_mx4(w)
        assert scales[0] == byte, value


@pytest.mark.parametrize("m,n", [(1, 32), (8, 512), (9, 544), (4096, 14336)])
def test_sizes_of_the_scales(m, n):
    assert T.teal_mx4_scale_bytes(m, n) == ti.mx4_scale_bytes(m, n)
    if m < 100:
        places = ti.mx4_scale_places(m, n)
        assert len(np.unique(places)) == places.size and places.max() < T.teal_mx4_scale_bytes(m, n)


def test_sizes_out_of_range():
    for m, n in [(0, 32), (-1, 32), (1, 0), (1, 16), (1, 48), ((1 << 24) + 1, 32), (1, (1 << 24) + 32)]:
        assert T.teal_mx4_scale_bytes(m, n) == 0
    assert T.teal_workspace_bytes_experts(0, 64, 1) == 0
    assert T.teal_workspace_bytes_experts(64, 0, 1) == 0
    assert T.teal_workspace_bytes_experts(64, 64, 0) == 0
    assert T.teal_workspace_bytes_experts(64, 64, 8 * 32 + 1) == 0
    assert T.teal_workspace_bytes_experts(64, 1 << 22, 8) == 0
    assert T.teal_workspace_bytes_experts(4096, 28672, 2) > 0


@pytest.mark.parametrize("call", ["pack", "unpack"])
def test_layout_refusals(call):
    def run(w=W, q=X, s=SC, m=64, n=64):
        if call == "pack":
            return T.teal_pack_mx4(w, q, s, m, n, stream=0)
        return T.teal_unpack_mx4(q, s, w, m, n, stream=0)

    for name in ("w", "q", "s"):
        assert run(**{name: None}) == T.TEAL_ERR_NULL
    for kw in (dict(m=0), dict(n=0), dict(n=40), dict(n=16), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 32)):
        assert run(**kw) == T.TEAL_ERR_SHAPE
    for kw in (dict(w=W + 1), dict(q=X + 8), dict(s=SC + 8)):
        assert run(**kw) == T.TEAL_ERR_ALIGN


@pytest.mark.parametrize("call", ["plain", "swiglu", "multi", "rmsnorm_multi"])
def test_product_refusals(call):
    ok = dict(q=W, s=SC, t=0.5, y=Y, m=64, n=64, x=X, g=G, ws=WS, wb=BIG, eps=1e-5)

    def run(**kw):
        a = {**ok, **kw}
        if call == "plain":
            return T.teal_sparse_gemv_mx4(a["q"], a["s"], a["x"], a["t"], a["y"], a["m"], a["n"], a["ws"], a["wb"], stream=0)
        if call == "swiglu":
            return T.teal_sparse_gemv_mx4_swiglu(a["q"], a["s"], a["x"], a["g"], a["t"], a["y"], a["m"], a["n"], a["ws"],
                                                 a["wb"], stream=0)
        lists = [[W, a["q"]], [SC, a["s"]], [0.1, a["t"]], [Y, a["y"]], [32, a["n"]]]
        if call == "multi":
            return T.teal_sparse_gemv_mx4_multi(*lists, a["x"], a["m"], a["ws"], a["wb"], stream=0)
        return T.teal_sparse_gemv_mx4_rmsnorm_multi(*lists, a["x"], a["g"], a["eps"], a["m"], a["ws"], a["wb"], stream=0)

    for name in ("q", "s", "y", "x", "ws") + (() if call in ("plain", "multi") else ("g",)):
        assert run(**{name: None}) == T.TEAL_ERR_NULL, name
    for kw in (dict(m=0), dict(n=0), dict(n=48), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 32)):
        assert run(**kw) == T.TEAL_ERR_SHAPE, kw
    for kw in (dict(q=W + 8), dict(s=SC + 4), dict(y=Y + 2), dict(x=X + 1), dict(ws=WS + 128)):
        assert run(**kw) == T.TEAL_ERR_ALIGN, kw
    for t in (-0.5, math.nan, math.inf):
        assert run(t=t) == T.TEAL_ERR_THRESHOLD
    n = 64 if call in ("plain", "swiglu") else 96
    assert run(wb=T.teal_workspace_bytes(64, n) - 1) == T.TEAL_ERR_WORKSPACE
    if call == "rmsnorm_multi":
        assert run(m=12) == run(m=16392) == T.TEAL_ERR_SHAPE
        assert run(eps=-1.0) == T.TEAL_ERR_THRESHOLD
        assert run(x=X + 8) == T.TEAL_ERR_ALIGN
    if call == "multi":
        for count in (0, 5):
            assert T.teal_sparse_gemv_mx4_multi(count * [W], count * [SC], count * [0.5], count * [Y], count * [32], X, 64,
                                                WS, BIG, stream=0) == T.TEAL_ERR_UNSUPPORTED


def test_route_refusals():
    ok = dict(logits=X, bias=G, score=T.TEAL_SCORE_SOFTMAX, tokens=4, experts=64, groups=8, top_groups=2, group_top=2,
              top_k=6, renormalise=True, scaling=1.0, idx=I, weight=Y, stream=0)

    def run(**kw):
        return T.teal_route_experts(**{**ok, **kw})

    for name in ("logits", "idx", "weight"):
        assert run(**{name: None}) == T.TEAL_ERR_NULL
    for kw in (dict(tokens=-1), dict(tokens=(1 << 24) + 1), dict(experts=0), dict(experts=1025)):
        assert run(**kw) == T.TEAL_ERR_SHAPE
    for name in ("logits", "bias", "idx", "weight"):
        assert run(**{name: ok[name] + 2}) == T.TEAL_ERR_ALIGN
    for kw in (dict(score=2), dict(score=-1), dict(groups=0), dict(groups=7), dict(groups=65, experts=65), dict(top_groups=0),
               dict(top_groups=9), dict(group_top=0), dict(group_top=3), dict(top_k=0), dict(top_k=17),
               dict(top_k=33, top_groups=8)):
        assert run(**kw) == T.TEAL_ERR_UNSUPPORTED, kw
    for scaling in (math.nan, math.inf):
        assert run(scaling=scaling) == T.TEAL_ERR_THRESHOLD
    assert run(tokens=0, logits=None, idx=None, weight=None) == T.TEAL_OK


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("down", [False, True])
def test_experts_refusals(fmt, down):
    ok = dict(q=W, s=SC, t=U, y=Y, n=64, experts=8, idx=I, weight=G, tokens=2, top_k=2, x=X, up=U, m=64, ws=WS, wb=BIG)

    def run(**kw):
        a = {**ok, **kw}
        if down:
            weights = (a["q"], a["s"]) if fmt == "mx4" else (a["q"],)
            call = T.teal_sparse_experts_mx4_swiglu if fmt == "mx4" else T.teal_sparse_experts_bf16_swiglu
            return call(*weights, a["t"], a["y"], a["experts"], a["idx"], a["weight"], a["tokens"], a["top_k"], a["x"],
                        a["up"], a["m"], a["n"], a["ws"], a["wb"], stream=0)
        weights = ([W, a["q"]], [SC, a["s"]]) if fmt == "mx4" else ([W, a["q"]],)
        call = T.teal_sparse_experts_mx4 if fmt == "mx4" else T.teal_sparse_experts_bf16
        return call(*weights, [U, a["t"]], [Y, a["y"]], [32, a["n"]], a["experts"], a["idx"], a["tokens"], a["top_k"],
                    a["x"], a["m"], a["ws"], a["wb"], stream=0)

    for name in ["q", "t", "y", "idx", "x", "ws"] + ["s"] * (fmt == "mx4") + ["weight", "up"] * down:
        assert run(**{name: None}) == T.TEAL_ERR_NULL, name
    for kw in (dict(m=0), dict(n=0), dict(n=60), dict(tokens=0), dict(tokens=9), dict(top_k=0), dict(top_k=33),
               dict(experts=0), dict(experts=1025), dict(n=1 << 23), dict(m=(1 << 24) + 1)):
        assert run(**kw) == T.TEAL_ERR_SHAPE, kw
    for name, off in [("q", 8), ("t", 2), ("y", 2), ("idx", 2), ("x", 1), ("ws", 128)] + [("s", 8)] * (fmt == "mx4") \
            + [("weight", 2), ("up", 2), ("x", 2)] * down:
        assert run(**{name: ok[name] + off}) == T.TEAL_ERR_ALIGN, name
    need = T.teal_workspace_bytes_experts(64, 64 if down else 96, 4)
    assert run(wb=need - 1) == T.TEAL_ERR_WORKSPACE
    if not down:
        for count in (0, 5):
            weights = (count * [W], count * [SC]) if fmt == "mx4" else (count * [W],)
            call = T.teal_sparse_experts_mx4 if fmt == "mx4" else T.teal_sparse_experts_bf16
            assert call(*weights, count * [U], count * [Y], count * [32], 8, I, 2, 2, X, 64, WS, BIG,
                        stream=0) == T.TEAL_ERR_UNSUPPORTED


def test_tensors_that_are_too_small_or_not_contiguous_are_refused():
    torch = pytest.importorskip("torch")
    q, s = torch.zeros(64, 32, dtype=torch.uint8), torch.zeros(1024, dtype=torch.uint8)
    x, y = torch.zeros(64, dtype=torch.float16), torch.zeros(64)
    assert s.numel() == T.teal_mx4_scale_bytes(64, 64)
    for bad in (dict(q=q[:63]), dict(s=s[:1023]), dict(x=x[:63]), dict(y=y[:63]), dict(q=torch.zeros(32, 64).t())):
        a = {**dict(q=q, s=s, x=x, y=y), **bad}
        with pytest.raises(ValueError):
            T.teal_sparse_gemv_mx4(a["q"], a["s"], a["x"], 0.5, a["y"], 64, 64, WS, BIG, stream=0)
    logits, idx, weight = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for bad in (dict(logits=logits[:3]), dict(idx=idx[:3]), dict(weight=weight[:3]), dict(logits=torch.zeros(8, 4).t())):
        a = {**dict(logits=logits, idx=idx, weight=weight), **bad}
        with pytest.raises(ValueError):
            T.teal_route_experts(a["logits"], None, 0, 4, 8, 1, 1, 1, 2, True, 1.0, a["idx"], a["weight"], stream=0)
    with pytest.raises(ValueError):
        T.teal_sparse_experts_mx4([q], [s], [torch.zeros(2)], [torch.zeros(2, 64)], [64], 2, idx[:1, :2].contiguous(), 1, 2,
                                  x, 64, WS, BIG, stream=0)        # one expert's weights for two
    with pytest.raises(ValueError):                                # 64-bit numbers of experts, as torch.topk gives them
        T.teal_sparse_experts_mx4([q], [s], [torch.zeros(1)], [torch.zeros(64)], [64], 1, torch.zeros(1, 1, dtype=torch.int64),
                                  1, 1, x, 64, WS, BIG, stream=0)
    with pytest.raises(ValueError):
        T.teal_route_experts(logits, None, 0, 4, 8, 1, 1, 1, 2, True, 1.0, idx.long(), weight, stream=0)
    with pytest.raises(ValueError):
        T.teal_sparse_gemv_mx4_multi([q, q], [s], [0.5, 0.5], [y, y], [64, 64], x, 64, WS, BIG, stream=0)


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_experts_down_refuses_64_bit_numbers(fmt):
    torch = pytest.importorskip("torch")
    weights, call = ((W, SC), T.teal_sparse_experts_mx4_swiglu) if fmt == "mx4" else ((W,), T.teal_sparse_experts_bf16_swiglu)
    with pytest.raises(ValueError):
        call(*weights, U, Y, 8, torch.zeros(2, 2, dtype=torch.int64), G, 2, 2, U, U, 64, 64, WS, BIG, stream=0)


def test_a_threshold_beyond_32_bits_is_refused_by_the_call():
    assert T.teal_sparse_gemv_mx4(W, SC, X, 1e39, Y, 64, 32, WS, BIG, stream=0) == T.TEAL_ERR_THRESHOLD
    assert T.teal_sparse_gemv_mx4_multi([W, W], [SC, SC], [0.5, 1e39], [Y, Y], [32, 32], X, 64, WS, BIG,
                                        stream=0) == T.TEAL_ERR_THRESHOLD
