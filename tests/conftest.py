import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (sm_100a)")


@pytest.fixture(scope="session")
def orc():
    """The CPU oracle's ctypes front end (compiled on first use)."""
    from oracle import oracle as o
    o.lib()
    return o


@pytest.fixture(scope="module", autouse=True)
def profiler_off_behind_a_module():
    """The profiler is the process's, and steps under it do not run as graphs: a module of tests that leaves it on would take the graphs from all that follow."""
    yield
    binding = sys.modules.get("paper_2509_05679_b200.binding")
    torch = sys.modules.get("torch")
    if binding is None or torch is None or not torch.cuda.is_available() or not torch.cuda.is_initialized():
        return
    from paper_2509_05679_b200 import synth as sy
    ctx = binding.Context([(sy.LINEAR, 8, 4, 1, 1)], [], 1, 2, 0.1, dtype="fp32", in_shape=(1, 1, 8), num_classes=4)
    ctx.profile(False)
    ctx.close()
