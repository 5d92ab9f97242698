import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU")
    config.addinivalue_line("markers", "slow: long-running CPU test")


@pytest.fixture(scope="session")
def O():
    """The CPU oracle module (built on first use if missing)."""
    from oracle import oracle
    oracle.lib()
    return oracle


@pytest.fixture(autouse=True)
def _ones_are_there(request, monkeypatch):
    """What torch.ones_like makes beside a call that is given another stream is filled on the
    current one, and nothing orders the call behind that: it may read what the memory held
    before.  On the GPU the fill is waited for, so that such a call has the input that it
    names (in a capture the two are on one stream)."""
    if request.node.get_closest_marker("gpu"):
        torch = pytest.importorskip("torch")
        ones_like = torch.ones_like

        def filled(*args, **kw):
            t = ones_like(*args, **kw)
            if t.is_cuda and not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream().synchronize()
            return t

        monkeypatch.setattr(torch, "ones_like", filled)
    yield
