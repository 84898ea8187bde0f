"""What the wrappers of the operators around the decomposed layers refuse before anything is launched (the library in them is a stand-in)."""
import pytest
import torch

from paper_2309_03824_amd import binding as lrd


class Library:
    """Takes every call."""
    calls = 0

    def __getattr__(self, name):
        def call(*args):
            Library.calls += 1
            return lrd.OK
        return call


@pytest.fixture
def on_host(monkeypatch):
    """The wrappers take host tensors, on `device` -1, for those of the current device."""
    monkeypatch.setattr(lrd, "_device", lambda t: t.get_device())
    monkeypatch.setattr(lrd, "_stream", lambda stream: None)
    monkeypatch.setattr(lrd, "_lib", Library())


T, D, OUT, R = 4, 8, 8, 8
X, V, U, H, A = torch.zeros(T, D), torch.zeros(2 * R, D), torch.zeros(2, OUT, R), torch.zeros(T, 2 * R), torch.zeros(T, OUT)
W = torch.ones(D)
CALLS = {
    "linear_gated_fwd": lambda ws: lrd.linear_gated_fwd(X, V, U, None, A, H, lrd.ACT_SILU, ws),
    "linear_gated_bwd": lambda ws: lrd.linear_gated_bwd(A, X, H, V, U, None, X, V, U, None, 0, lrd.ACT_SILU, ws),
    "linear_gated_bwd_data": lambda ws: lrd.linear_gated_bwd_data(A, H, V, U, None, X, torch.zeros(2, T, OUT), H, lrd.ACT_SILU, ws),
    "block_norm_bwd": lambda ws: lrd.block_norm_bwd(X, X, X, X, W, None, None, W, None, X, A, W, None, None, W, None, lrd.BlockNorm(), ws),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_workspace_of_another_device_or_with_strides_is_refused(on_host, name):
    Library.calls = 0
    CALLS[name](None)
    CALLS[name](torch.empty(4096, dtype=torch.uint8))
    assert Library.calls == 2
    for bad in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(8192, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            CALLS[name](bad)
    assert Library.calls == 2


def test_a_workspace_on_the_host_is_refused():
    with pytest.raises(ValueError):
        lrd._room(torch.empty(4096, dtype=torch.uint8), 0)
    assert lrd._room(None, 0) == (None, 0)


def test_a_backward_pass_without_a_gradient_is_refused(on_host):
    with pytest.raises(ValueError):
        lrd.block_norm_bwd(None, None, X, X, W, None, None, W, None, X, A, None, None, None, None, None, lrd.BlockNorm())
