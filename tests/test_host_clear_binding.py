"""The binding of the clear side's calls without a GPU."""
import os
import subprocess
import sys

import pytest

import paper_1906_00148_amd as she
from paper_1906_00148_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Library:
    """Takes every call; a context is on the GPU `device`."""

    def __init__(self, device=0):
        self.device, self.calls = device, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return self.device if name == "she_clear_device" else 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    return lib


def test_the_package_is_imported_without_torch():
    code = "import sys; sys.modules['torch'] = None; import paper_1906_00148_amd as she; she.Context, she.SheError, she.TOY"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, timeout=120)


def test_a_context_with_a_pool_of_its_own_leaves_torch_s_device_alone(library):
    import torch
    before = torch.cuda.is_initialized()
    with she.Context(she.TOY, 1, 16, use_torch_pool=False) as ctx:
        ctx.set_option(0, 1)
    assert torch.cuda.is_initialized() == before
    assert [name for name, _ in library.calls if name in ("she_keygen", "she_set_option")] == ["she_keygen", "she_set_option"]
