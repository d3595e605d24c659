import contextlib
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session")
def oracle():
    """The CPU oracle binding (builds oracle/libzvc_ref.so on first use)."""
    from oracle import zvc_ref
    zvc_ref.load()
    return zvc_ref


@contextlib.contextmanager
def repeatable_inputs(module):
    """tests.test_gpu_ffn seeds its inputs by hash(), which Python salts per process: a failure there could not be run
    again.  Its generator is one with a seed from the same key that every process computes alike."""
    if getattr(module, "__name__", "") != "tests.test_gpu_ffn":
        yield
        return
    from tests import ffn_inputs
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(module, "generator", lambda *key: ffn_inputs.generator(*key, device=module.DEV))
        yield


@pytest.fixture(autouse=True, scope="module")
def _repeatable_inputs(request):
    with repeatable_inputs(request.module):
        yield
