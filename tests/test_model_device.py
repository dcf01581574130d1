"""What the binding of ``toktier_model.h`` refuses before a launch, without a GPU: other devices, sizes past 32 bits."""

import pytest

import paper_2607_29678_amd as tt
from paper_2607_29678_amd import _lib, model

torch = pytest.importorskip("torch")


class OnDevice:
    """A host tensor that says it lies on a device."""

    def __init__(self, t, device):
        self._t, self._d = t, device

    def get_device(self):
        return self._d

    def __getattr__(self, name):
        return getattr(self._t, name)


class Library:
    """Records calls; workspace sizes are 0."""

    def __init__(self, current):
        self.calls, self._current = [], current

    def tt_current_device(self):
        return self._current

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *a: 0
        return lambda *a: self.calls.append(name) or 0


def _lib_error():
    """What ``tt_current_device`` returns where there is no device."""
    return next(k for k, v in _lib.STATUS.items() if v == "TT_ERR_HIP")


def calls(device):
    f = lambda *s, t=torch.float32: OnDevice(torch.zeros(s, dtype=t), device)  # noqa: E731
    i32, i64, bf = torch.int32, torch.int64, torch.bfloat16
    return {
        "tt_step_plan": lambda: tt.step_plan(f(3, t=i32), f(3, t=i32), f(3, 5, t=i32), f(9, t=i32), f(1, t=i64), 16, f(4, t=i32),
                                             f(3, t=i32), f(3, t=i32), f(8, t=i64), f(8, t=i32), f(8, t=i32), f(2, t=i64)),
        "tt_token_scores": lambda: tt.token_scores(f(4, 50), f(4, t=i32), f(4)),
        "tt_token_scores_grad": lambda: tt.token_scores_grad(f(4, 50), f(4, t=i32), f(4, 2), f(4), f(4), f(4), f(4, 50)),
        "tt_head_scores": lambda: tt.head_scores(f(4, 64, t=bf), f(90, 64, t=bf), f(4, t=i32), f(4)),
        "tt_head_scores_grad": lambda: tt.head_scores_grad(f(4, 64, t=bf), f(90, 64, t=bf), f(4, t=i32), f(4, 2), f(4), f(4), f(4),
                                                           f(4, 64, t=bf), f(90, 64, t=bf)),
    }


@pytest.fixture
def library(monkeypatch):
    def use(current):
        lib = Library(current)
        monkeypatch.setattr(_lib, "load", lambda: lib)
        model._need.cache_clear()
        return lib

    yield use
    model._need.cache_clear()


@pytest.mark.parametrize("name", sorted(calls(0)))
def test_the_device_has_to_be_the_current_one(library, name):
    for current, device in ((0, 1), (1, 0), (_lib_error(), 0)):
        lib = library(current)
        with pytest.raises(ValueError):
            calls(device)[name]()
        assert lib.calls == []
    for device in (0, 1):
        lib = library(device)
        calls(device)[name]()
        assert lib.calls == [name]


def test_tensors_on_several_devices(library):
    lib = library(0)
    with pytest.raises(ValueError):
        tt.token_scores(OnDevice(torch.zeros(4, 50), 0), OnDevice(torch.zeros(4, dtype=torch.int32), 1),
                        OnDevice(torch.zeros(4), 0))
    assert lib.calls == []


def test_the_library_knows_its_device():
    want = torch.cuda.current_device() if torch.cuda.is_available() else _lib_error()
    assert _lib.load().tt_current_device() == want


@pytest.mark.parametrize("page_size", [1 << 31, -(1 << 31) - 1, 1 << 40])
def test_page_sizes_past_32_bits(library, page_size):
    lib = library(0)
    f = lambda *s, t=torch.int32: OnDevice(torch.zeros(s, dtype=t), 0)  # noqa: E731
    args = [f(3), f(3), f(3, 5), f(9), f(1, t=torch.int64), page_size, f(4), f(3), f(3), f(8, t=torch.int64), f(8), f(8),
            f(2, t=torch.int64)]
    with pytest.raises(ValueError):
        tt.step_plan(*args)
    assert lib.calls == []
    args[5] = (1 << 31) - 1
    tt.step_plan(*args)
    assert lib.calls == ["tt_step_plan"]
