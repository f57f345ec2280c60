"""Host side of the routed-expert calls and of the layer on them: what is refused before any device is touched."""
import contextlib
import types

import pytest

from paper_2502_07021_b200 import binding as fs
from paper_2502_07021_b200 import build as fs_build

P = 0x1000  # never dereferenced: every case is refused on the host


@pytest.mark.parametrize("eps", [1e-39, 1e-46, 4e38, 1e300])
def test_balance_refuses_an_eps_beyond_fp32(eps):
    """eps and log2(e)/eps are fp32 numbers in the kernel; where one of them is 0 or infinite every dual would be NaN."""
    fs_build.build()
    need = fs.fs_router_workspace(10, 4, 1)
    assert fs.lib().fs_router_duals(P, fs.FS_F32, 4, 10, 4, None, None, eps, 1, None, None, P, None, P, need, None) == fs.FS_ERR_BAD_EPS


def test_rounding_no_rows_to_slots():
    """An empty array of slots has no address."""
    lib = fs.lib()
    assert lib.fs_mx4_quantize(None, fs.FS_BF16, 64, 0, 64, None, 3, 0, None, 32, None, 4, None) == fs.FS_OK
    assert lib.fs_mx4_quantize(P, fs.FS_BF16, 64, 1, 64, None, 3, 3, P, 32, P, 4, None) == fs.FS_ERR_BAD_N


class OnDevice:
    """A CPU tensor that says it lies on another device."""

    def __init__(self, t, device):
        self._t, self.device, self.is_cuda = t, device, True

    def __getattr__(self, name):
        return getattr(self._t, name)

    def view(self, *a):
        return OnDevice(self._t.view(*a), self.device)

    def reshape(self, *a):
        return OnDevice(self._t.reshape(*a), self.device)

    def contiguous(self):
        return self


@pytest.fixture
def second_device(monkeypatch):
    """experts with a torch whose current device is recorded, and library calls that note under which one they were made."""
    import torch
    from paper_2502_07021_b200 import experts
    one = torch.device("cuda", 1)
    current, calls = [torch.device("cuda", 0)], []

    @contextlib.contextmanager
    def select(d):
        current.append(d)
        yield
        current.pop()

    fake = types.SimpleNamespace(**{n: getattr(torch, n) for n in ("float32", "int32", "uint8", "bool", "autograd", "nn", "Tensor")})
    fake.cuda = types.SimpleNamespace(device=select, current_device=lambda: current[-1].index, current_stream=lambda d: 0)
    fake.empty = lambda *a, device=None, **kw: OnDevice(torch.empty(*a, **kw), device)
    monkeypatch.setattr(experts, "torch", fake)
    for name in ("fs_router_duals", "fs_router_forward", "fs_router_backward", "fs_router_dispatch", "fs_mx4_quantize", "fs_mx4_product"):
        monkeypatch.setattr(fs, name, lambda *a, _n=name: calls.append((_n, current[-1])))
    monkeypatch.setattr(fs, "fs_router_workspace", lambda *a: 64)
    monkeypatch.setattr(fs, "mx4_empty", lambda r, c, device: (OnDevice(torch.empty(r, 64, dtype=torch.uint8), device),
                                                              OnDevice(torch.empty(r, 4, dtype=torch.uint8), device)))
    return experts, one, calls


def test_calls_run_on_the_tensors_device(second_device):
    """With tensors on a device that is not the current one, every launch is made with theirs selected."""
    import torch
    experts, one, calls = second_device
    l = OnDevice(torch.zeros(20, 8), one)
    experts.balance(l, 0.1, 2)
    experts.choose(l, 2)
    q, s = experts.quantize(OnDevice(torch.zeros(20, 96), one))
    w = experts.quantize(OnDevice(torch.zeros(3, 20, 96), one))
    experts.product(q, s, w, OnDevice(torch.zeros(4, dtype=torch.int32), one), 96, torch.float32)
    ctx = types.SimpleNamespace(save_for_backward=lambda *a: setattr(ctx, "saved_tensors", a), mark_non_differentiable=lambda *a: None,
                                set_materialize_grads=lambda v: None)
    experts._Route.forward(ctx, l, 2, None, None, True)
    assert [n for n, _ in calls] == ["fs_router_duals", "fs_router_forward", "fs_mx4_quantize", "fs_mx4_quantize", "fs_mx4_product",
                                     "fs_router_forward"]
    assert all(d == one for _, d in calls), calls


def test_tensors_of_two_devices_are_refused(second_device):
    import torch
    experts, one, calls = second_device
    zero = torch.device("cuda", 0)
    l = OnDevice(torch.zeros(20, 8), one)
    other = OnDevice(torch.zeros(8), zero)
    for call in (lambda: experts.balance(l, 0.1, 2, share=other), lambda: experts.choose(l, 2, other),
                 lambda: experts.choose(l, 2, mask=OnDevice(torch.ones(20, dtype=torch.bool), zero))):
        with pytest.raises(ValueError):
            call()
    assert not calls
