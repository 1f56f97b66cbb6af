"""What the binding keeps between calls, without a GPU."""
import os

import pytest

from paper_2408_14690_amd import binding


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
