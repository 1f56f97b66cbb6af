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
