"""What the binding keeps between calls and what it refuses, without a GPU."""
import os

import pytest

import paper_2408_14690_amd as T
from paper_2408_14690_amd import binding
from test_abi import BIG, SC, W, WS, X, Y, _built  # noqa: F401

U, I = 0x70000, 0x80000                     # further fake device addresses


@pytest.mark.skipif(not hasattr(os, "fork"), reason="no fork")
def test_a_forked_process_looks_for_the_stream_again(monkeypatch):
    """Not by the function its parent found: torch says there that HIP cannot be used after a fork."""
    monkeypatch.setattr(binding, "_find_current_stream", lambda: lambda: 7)
    monkeypatch.setattr(binding, "_current_stream", lambda: 5)             # as after the parent's first call
    pid = os.fork()
    if pid == 0:
        code = 1
        try:
            code = 0 if binding._stream(None) == 7 else 2
        finally:
            os._exit(code)
    assert os.waitstatus_to_exitcode(os.waitpid(pid, 0)[1]) == 0
    assert binding._stream(None) == 5                                       # the parent keeps it


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("down,name", [(False, "t"), (True, "t"), (True, "weight")])
def test_experts_refuse_64_bit_floats(fmt, down, name):
    """Thresholds and weights that were computed by numpy are as large as these calls need and more."""
    torch = pytest.importorskip("torch")
    a = {"t": U, "weight": U, name: torch.zeros(4, 4, dtype=torch.float64)}
    weights = (W, SC) if fmt == "mx4" else (W,)
    with pytest.raises(ValueError, match=name):
        if down:
            call = T.teal_sparse_experts_mx4_swiglu if fmt == "mx4" else T.teal_sparse_experts_bf16_swiglu
            call(*weights, a["t"], Y, 8, I, a["weight"], 2, 2, U, U, 64, 64, WS, BIG, stream=0)
        else:
            call = T.teal_sparse_experts_mx4 if fmt == "mx4" else T.teal_sparse_experts_bf16
            call(*[[w] for w in weights], [a["t"]], [Y], [64], 8, I, 2, 2, X, 64, WS, BIG, stream=0)


def test_weights_and_integers_of_many_rows_have_their_own_types():
    """Tensors that are large enough, and whose numbers are not those that the call reads."""
    torch = pytest.importorskip("torch")
    q, w, sc = torch.zeros(3, 128, dtype=torch.int8), torch.zeros(40, 16, dtype=torch.int8), torch.zeros(16).half()
    for bad in (dict(q=q.int()), dict(q=q.half()), dict(w=w.int()), dict(w=w.bfloat16()), dict(sc=sc.bfloat16()), dict(sc=sc.float())):
        a = {**dict(q=q, w=w, sc=sc), **bad}
        with pytest.raises(ValueError):
            T.teal_gemm_w8(a["w"], a["sc"], a["q"], U, 3, Y, 40, 16, WS, BIG, stream=0)
        with pytest.raises(ValueError):
            T.teal_gemm_w8_multi([a["w"]], [a["sc"]], [Y], [16], a["q"], U, 3, 40, WS, BIG, stream=0)
        with pytest.raises(ValueError):
            T.teal_gemm_w8_ex([a["w"]], [a["sc"]], [Y], [16], a["q"], U, 3, 40, WS, BIG, stream=0, tile_rows=16, tile_cols=128)
    with pytest.raises(ValueError):
        T.teal_quantize_rows(X, T.TEAL_F16, 3, 40, 0.0, q.int(), U, stream=0)
    with pytest.raises(ValueError):
        T.teal_quantize_rows_swiglu(U, U, 3, 40, 0.0, q.half(), U, stream=0)
    group = (4, I, I, 4, 2)
    wide, codes = torch.zeros(4, 64, 64).bfloat16(), torch.zeros(4, 64, 32, dtype=torch.uint8)
    scales = torch.zeros(4, T.teal_mx4_scale_bytes(64, 64), dtype=torch.uint8)
    for bad in (wide.half(), wide.float()):
        for pair in ((bad, wide), (wide, bad)):
            with pytest.raises(ValueError):
                T.teal_grouped_experts_bf16_gate_up(*pair, *group, X, Y, 64, 64, stream=0)
        with pytest.raises(ValueError):
            T.teal_grouped_experts_bf16_down(bad, *group, I, U, X, Y, 64, 64, WS, BIG, stream=0)
    for bad in ((codes.int(), scales), (codes, scales.int()), (codes.half(), scales)):
        for four in ((*bad, codes, scales), (codes, scales, *bad)):
            with pytest.raises(ValueError):
                T.teal_grouped_experts_mx4_gate_up(*four, *group, X, Y, 64, 64, stream=0)
        with pytest.raises(ValueError):
            T.teal_grouped_experts_mx4_down(*bad, *group, I, U, X, Y, 64, 64, WS, BIG, stream=0)
