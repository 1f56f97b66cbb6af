"""What the calls of many rows refuse and how large their workspaces are, without a GPU."""
import math

import pytest

import paper_2408_14690_amd as T
from test_abi import BIG, SC, W, WS, X, Y, _built  # noqa: F401

G, U, I = 0x60000, 0x70000, 0x80000         # further fake device addresses
HUGE = 1 << 40


def test_quantized_pitch():
    assert [T.teal_quantized_pitch(m) for m in (1, 127, 128, 129, 5001, 131072)] == [128, 128, 128, 256, 5120, 131072]
    assert T.teal_quantized_pitch(0) == T.teal_quantized_pitch(-1) == T.teal_quantized_pitch(131073) == 0


@pytest.mark.parametrize("swiglu", [False, True])
def test_quantize_refusals(swiglu):
    ok = dict(x=X, up=U, type=T.TEAL_BF16, rows=3, m=40, t=0.5, q=W, s=SC)

    def run(**kw):
        a = {**ok, **kw}
        if swiglu:
            return T.teal_quantize_rows_swiglu(a["x"], a["up"], a["rows"], a["m"], a["t"], a["q"], a["s"], stream=0)
        return T.teal_quantize_rows(a["x"], a["type"], a["rows"], a["m"], a["t"], a["q"], a["s"], stream=0)

    for name in ["x", "q", "s"] + ["up"] * swiglu:
        assert run(**{name: None}) == T.TEAL_ERR_NULL, name
    for kw in (dict(rows=-1), dict(rows=T.TEAL_MAX_ROWS + 1), dict(m=0), dict(m=T.TEAL_MAX_ROW_SUM + 1)):
        assert run(**kw) == T.TEAL_ERR_SHAPE, kw
    for name, off in [("x", 2 if swiglu else 1), ("q", 8), ("s", 2)] + [("up", 2)] * swiglu:
        assert run(**{name: ok[name] + off}) == T.TEAL_ERR_ALIGN, name
    for t in (-0.5, math.nan, math.inf):
        assert run(t=t) == T.TEAL_ERR_THRESHOLD
    if not swiglu:
        assert run(type=2) == run(type=-1) == T.TEAL_ERR_UNSUPPORTED
    assert run(rows=0, x=None, up=None, q=None, s=None) == T.TEAL_OK


@pytest.mark.parametrize("multi", [False, True])
def test_gemm_w8_refusals(multi):
    ok = dict(w=W, s=SC, y=Y, n=64, q=X, rs=G, rows=5, m=40, ws=WS, wb=BIG)

    def run(**kw):
        a = {**ok, **kw}
        if multi:
            return T.teal_gemm_w8_multi([W, a["w"]], [SC, a["s"]], [Y, a["y"]], [32, a["n"]], a["q"], a["rs"], a["rows"],
                                        a["m"], a["ws"], a["wb"], stream=0)
        return T.teal_gemm_w8(a["w"], a["s"], a["q"], a["rs"], a["rows"], a["y"], a["m"], a["n"], a["ws"], a["wb"], stream=0)

    for name in ("w", "s", "y", "q", "rs", "ws"):
        assert run(**{name: None}) == T.TEAL_ERR_NULL, name
    for kw in (dict(rows=-1), dict(rows=T.TEAL_MAX_ROWS + 1), dict(m=0), dict(m=T.TEAL_MAX_ROW_SUM + 1), dict(n=0), dict(n=24),
               dict(n=-16), dict(n=(1 << 24) + 16), dict(rows=1 << 20, n=1 << 15)):
        assert run(**kw) == T.TEAL_ERR_SHAPE, kw
    for name, off in [("w", 8), ("s", 1), ("y", 2), ("q", 8), ("rs", 2), ("ws", 128)]:
        assert run(**{name: ok[name] + off}) == T.TEAL_ERR_ALIGN, name
    need = T.teal_workspace_bytes_gemm_w8(5, 40, 96 if multi else 64)
    assert need > 0 and run(wb=need - 1) == T.TEAL_ERR_WORKSPACE
    if multi:
        for count in (0, 5):
            assert T.teal_gemm_w8_multi(count * [W], count * [SC], count * [Y], count * [32], X, G, 5, 40, WS, BIG,
                                        stream=0) == T.TEAL_ERR_UNSUPPORTED
    assert run(rows=0, q=None, rs=None, y=None) == T.TEAL_OK
    for kw in (dict(rows=-1), dict(m=0), dict(n=8), dict(rows=T.TEAL_MAX_ROWS + 1)):
        a = {**dict(rows=5, m=40, n=64), **kw}
        assert T.teal_workspace_bytes_gemm_w8(a["rows"], a["m"], a["n"]) == 0, kw


def test_gemm_w8_ex_refuses_shapes_that_there_are_not():
    def run(tile_rows, tile_cols, splits, rows=5, n=64, wb=BIG):
        return T.teal_gemm_w8_ex([W], [SC], [Y], [n], X, G, rows, 4096, WS, wb, stream=0, tile_rows=tile_rows,
                                 tile_cols=tile_cols, splits=splits)

    for shape in [(8, 128, 1), (16, 256, 1), (128, 256, 1), (64, 64, 1), (0, 128, 1), (64, 0, 1), (0, 0, 2), (512, 128, 1), (64, 128, -1),
                  (64, 128, 17), (256, 128, 2), (256, 256, 2), (-16, 128, 1)]:
        assert run(*shape) == T.TEAL_ERR_UNSUPPORTED, shape
    assert run(16, 128, 2, rows=16 * 300) == T.TEAL_ERR_UNSUPPORTED                # more blocks than sliced sums have room for
    # 2^16 tiles of 16 rows by 128 of 128 columns are 2^23 blocks, more than the 2^22 of a launch; of 32 rows they would fit.
    assert run(16, 128, 1, rows=1 << 20, n=16384) == T.TEAL_ERR_UNSUPPORTED
    small = T.teal_workspace_bytes_gemm_w8(5, 4096, 64)
    assert small < T.teal_workspace_bytes_gemm_w8(128, 4096, 64)
    assert run(128, 128, 2, wb=small) == T.TEAL_ERR_WORKSPACE


def test_arrange_refusals():
    ok = dict(idx=I, tokens=5, top_k=2, experts=8, order=X, start=Y, ws=WS, wb=BIG)

    def run(**kw):
        a = {**ok, **kw}
        return T.teal_arrange_experts(a["idx"], a["tokens"], a["top_k"], a["experts"], a["order"], a["start"], a["ws"], a["wb"],
                                      stream=0)

    for name in ("idx", "order", "start", "ws"):
        assert run(**{name: None}) == T.TEAL_ERR_NULL, name
    for kw in (dict(tokens=-1), dict(top_k=0), dict(top_k=T.TEAL_MAX_TOP_K + 1), dict(tokens=(1 << 23) + 1), dict(experts=0),
               dict(experts=T.TEAL_MAX_EXPERTS + 1)):
        assert run(**kw) == T.TEAL_ERR_SHAPE, kw
    for name, off in [("idx", 2), ("order", 2), ("start", 1), ("ws", 128)]:
        assert run(**{name: ok[name] + off}) == T.TEAL_ERR_ALIGN, name
    need = T.teal_workspace_bytes_arrange_experts(8, 10)
    assert need > 0 and run(wb=need - 1) == T.TEAL_ERR_WORKSPACE
    assert T.teal_workspace_bytes_arrange_experts(0, 10) == T.teal_workspace_bytes_arrange_experts(8, (1 << 24) + 1) == 0


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("down", [False, True])
def test_grouped_refusals(fmt, down):
    ok = dict(w=W, s=SC, experts=8, order=I, start=G, tokens=5, top_k=2, idx=I, weight=U, x=X, out=Y, m=64, n=96, ws=WS, wb=HUGE)

    def run(**kw):
        a = {**ok, **kw}
        group = (a["experts"], a["order"], a["start"], a["tokens"], a["top_k"])
        own = (a["w"], a["s"]) if fmt == "mx4" else (a["w"],)
        if down:
            call = T.teal_grouped_experts_mx4_down if fmt == "mx4" else T.teal_grouped_experts_bf16_down
            return call(*own, *group, a["idx"], a["weight"], a["x"], a["out"], a["m"], a["n"], a["ws"], a["wb"], stream=0)
        other = (W, SC) if fmt == "mx4" else (W,)
        call = T.teal_grouped_experts_mx4_gate_up if fmt == "mx4" else T.teal_grouped_experts_bf16_gate_up
        assert call(*own, *other, *group, a["x"], a["out"], a["m"], a["n"], stream=0) == \
            call(*other, *own, *group, a["x"], a["out"], a["m"], a["n"], stream=0)
        return call(*other, *own, *group, a["x"], a["out"], a["m"], a["n"], stream=0)

    for name in ["w", "order", "start", "x", "out"] + ["s"] * (fmt == "mx4") + ["idx", "weight", "ws"] * down:
        assert run(**{name: None}) == T.TEAL_ERR_NULL, name
    for kw in (dict(experts=0), dict(experts=T.TEAL_MAX_EXPERTS + 1), dict(tokens=-1), dict(top_k=0), dict(top_k=33),
               dict(tokens=(1 << 23) + 1), dict(m=0), dict(m=60), dict(m=(1 << 20) + 8), dict(n=0), dict(n=100), dict(n=(1 << 20) + 32),
               dict(tokens=1 << 23, n=1 << 12), *([dict(n=40)] if fmt == "mx4" else [])):
        assert run(**kw) == T.TEAL_ERR_SHAPE, kw
    for name, off in [("w", 8), ("order", 2), ("start", 2), ("x", 8)] + [("s", 8)] * (fmt == "mx4") + \
            ([("idx", 2), ("weight", 2), ("ws", 128), ("out", 2)] if down else [("out", 8)]):
        assert run(**{name: ok[name] + off}) == T.TEAL_ERR_ALIGN, name
    if down:
        need = T.teal_workspace_bytes_grouped_experts(10, 96)
        assert need > 0 and run(wb=need - 1) == T.TEAL_ERR_WORKSPACE
    assert T.teal_workspace_bytes_grouped_experts(-1, 96) == T.teal_workspace_bytes_grouped_experts(10, 0) == 0


def test_workspace_of_the_grouped_products_is_bounded():
    """A row of sums per pair, of all columns while that is not much, of a part of them at a time beyond."""
    assert T.teal_workspace_bytes_grouped_experts(100, 4096) >= 100 * 4096 * 4
    assert T.teal_workspace_bytes_grouped_experts(1 << 20, 1 << 15) <= 1 << 31


def test_tensors_that_do_not_fit_are_refused():
    torch = pytest.importorskip("torch")
    x16, q, s = torch.zeros(3, 40).half(), torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3)
    ok = dict(x=x16, type=T.TEAL_F16, q=q, s=s)
    for bad in (dict(x=x16[:2]), dict(x=x16.float()), dict(x=x16.bfloat16()), dict(type=T.TEAL_BF16), dict(q=q[:, :40].contiguous()),
                dict(s=s[:2]), dict(s=s.double()), dict(x=torch.zeros(40, 3).half().t())):
        a = {**ok, **bad}
        with pytest.raises(ValueError):
            T.teal_quantize_rows(a["x"], a["type"], 3, 40, 0.0, a["q"], a["s"], stream=0)
    with pytest.raises(ValueError):
        T.teal_quantize_rows_swiglu(s.double(), s, 1, 3, 0.0, q, s, stream=0)
    w, sc, y = torch.zeros(40, 16, dtype=torch.int8), torch.zeros(16).half(), torch.zeros(3, 16)
    for bad in (dict(w=w[:39]), dict(sc=sc[:8]), dict(y=y[:2]), dict(y=y.double()), dict(q=q[:2]), dict(s=s[:2])):
        a = {**dict(w=w, sc=sc, y=y, q=q, s=s), **bad}
        with pytest.raises(ValueError):
            T.teal_gemm_w8(a["w"], a["sc"], a["q"], a["s"], 3, a["y"], 40, 16, WS, BIG, stream=0)
        with pytest.raises(ValueError):
            T.teal_gemm_w8_multi([a["w"]], [a["sc"]], [a["y"]], [16], a["q"], a["s"], 3, 40, WS, BIG, stream=0)
    with pytest.raises(ValueError):
        T.teal_gemm_w8_multi([w, w], [sc], [y, y], [16, 16], q, s, 3, 40, WS, BIG, stream=0)
    idx = torch.zeros(4, 2, dtype=torch.int32)
    order, start = torch.zeros(8, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    for bad in (dict(idx=idx.long()), dict(idx=idx[:3]), dict(order=order[:7]), dict(order=order.long()), dict(start=start[:4])):
        a = {**dict(idx=idx, order=order, start=start), **bad}
        with pytest.raises(ValueError):
            T.teal_arrange_experts(a["idx"], 4, 2, 4, a["order"], a["start"], WS, BIG, stream=0)
    wg, x, h = torch.zeros(4, 64, 32).bfloat16(), torch.zeros(4, 64).bfloat16(), torch.zeros(8, 32).bfloat16()
    for bad in (dict(wg=wg[:3]), dict(x=x[:3]), dict(x=x.half()), dict(x=x.float()), dict(h=h[:7]), dict(h=h.half()),
                dict(order=order.long())):
        a = {**dict(wg=wg, x=x, h=h, order=order), **bad}
        with pytest.raises(ValueError):
            T.teal_grouped_experts_bf16_gate_up(a["wg"], wg, 4, a["order"], start, 4, 2, a["x"], a["h"], 64, 32, stream=0)
    wd, y = torch.zeros(4, 32, 64).bfloat16(), torch.zeros(4, 64)
    for bad in (dict(wd=wd[:3]), dict(h=h[:7]), dict(y=y[:3]), dict(y=y.double()), dict(idx=idx.long()),
                dict(weight=torch.zeros(4, 2).double())):
        a = {**dict(wd=wd, h=h, y=y, idx=idx, weight=torch.zeros(4, 2)), **bad}
        with pytest.raises(ValueError):
            T.teal_grouped_experts_bf16_down(a["wd"], 4, order, start, 4, 2, a["idx"], a["weight"], a["h"], a["y"], 32, 64, WS, BIG,
                                             stream=0)
