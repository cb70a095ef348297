"""A forked process looks for its current stream anew: torch refuses there what the parent's GPU state cannot serve, and only
the first look goes through that check."""
import os

import pytest

from paper_2607_22614_amd import dr


@pytest.mark.skipif(not hasattr(os, "fork"), reason="needs fork")
def test_a_forked_process_asks_torch_again(monkeypatch):
    monkeypatch.setattr(dr, "_current", lambda: 1234)  # as after the parent's first call
    assert dr._stream(None) == 1234

    def refuse():
        raise RuntimeError("re-initialised in a forked process")

    monkeypatch.setattr(dr, "_find_current", refuse)  # what torch does in a fork of a process that used the GPU
    assert dr._stream(None) == 1234
    pid = os.fork()
    if pid == 0:
        status = 1
        try:
            dr._stream(None)
        except RuntimeError:
            status = 0
        finally:
            os._exit(status)
    assert os.waitstatus_to_exitcode(os.waitpid(pid, 0)[1]) == 0
    assert dr._stream(None) == 1234
