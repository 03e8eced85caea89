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


class On:
    """A tensor that says it is on a GPU."""

    def __init__(self, t, gpu):
        self._t, self._gpu = t, gpu
        self.is_cuda, self.device = True, f"cuda:{gpu}"

    def get_device(self):
        return self._gpu

    def __getattr__(self, name):
        return getattr(self._t, name)


def arguments():
    """Each call's tensors, all as they should be, and its other arguments."""
    import torch
    i32 = torch.int32

    def half(*size):
        return torch.zeros(*size, dtype=torch.bfloat16)
    rotation = dict(wq=torch.ones(8), wk=torch.ones(8), cos=torch.ones(5, 4), sin=torch.ones(5, 4), positions=torch.zeros(3, dtype=i32))
    adapters = dict(x=half(3, 16), down=half(2, 4, 16), up=half(2, 4, 24), starts=torch.zeros(3, dtype=i32), which=torch.zeros(2, dtype=i32),
                    scale=torch.ones(2), ranks=torch.zeros(2, dtype=i32))
    heads = dict(q=half(3, 2, 8), k=half(3, 1, 8))
    pages = dict(k_pages=half(4, 16, 1, 8), v_pages=half(4, 16, 1, 8))
    return {"adapters": dict(adapters, base=torch.zeros(3, 24, dtype=i32), step=torch.ones(24), out=half(3, 24)),
            "adapters_grad": dict(adapters, dy=half(3, 24), base=half(3, 16)),
            "qk_rotate": dict(heads, **rotation),
            "qk_rotate_append": dict(heads, v=half(3, 1, 8), **rotation, **pages, slots=torch.zeros(3, dtype=torch.int64), out=half(3, 2, 8)),
            "qk_rotate_grad": dict(heads, **rotation, dq_out=half(3, 2, 8), dk_out=half(3, 1, 8)),
            "attend_pages": dict(pages, q=half(3, 2, 8), table=torch.zeros(2, 4, dtype=i32), starts=torch.zeros(3, dtype=i32),
                                 lengths=torch.zeros(2, dtype=i32), out=half(3, 2, 8))}


@pytest.mark.parametrize("call", sorted(arguments()))
def test_tensors_of_another_gpu_are_refused(library, call):
    """Every argument in turn, with the context on cuda:2 and the others there."""
    library.device = 2
    tensors = arguments()[call]
    with she.Context(she.TOY, 1, 16, use_torch_pool=False) as ctx:
        for wrong in tensors:
            with pytest.raises(she.SheError) as e:
                getattr(ctx, call)(**{name: On(t, 0 if name == wrong else 2) for name, t in tensors.items()})
            assert e.value.code == -1 and "cuda:2" in str(e.value) and (wrong in str(e.value)), (wrong, e.value)
    assert not [name for name, _ in library.calls if name == "she_" + call]
