"""The zeroth-order calls on another stream than the current one, on the host: which stream their own losses and
workspaces are allocated for."""
import ctypes as C

import pytest
import torch

import layers_fake as fake

CFG = dict(n_layers=1, vocab=32, embed=32, hidden=32, wdtype=0, probe=0)


@pytest.fixture
def device(monkeypatch):
    from paper_2505_17852_amd import layers, zo
    dev = fake.Device(layers, monkeypatch)
    dev.zo = zo
    monkeypatch.setattr(zo, "lib", lambda: dev.library)
    monkeypatch.setattr(zo, "_dev", lambda t, dtype, name: C.c_void_p(t.data_ptr()))
    monkeypatch.setattr(zo, "param_count", lambda cfg: 64)
    monkeypatch.setattr(zo, "workspace_bytes", lambda *a: 4096)
    return dev


def _call(dev, name, **kw):
    theta, tokens = torch.zeros(64), torch.zeros(2, 9, dtype=torch.int32)
    if name == "debug_probe":
        return dev.zo.debug_probe(0, 1, 0, 0, 64, device="cpu", **kw)
    if name == "debug_gauss_pairs":
        return dev.zo.debug_gauss_pairs(torch.zeros(8, dtype=torch.int32), **kw)
    return getattr(dev.zo, name)(CFG, theta, 1, 1e-3, 4, tokens, **kw)


NAMES = ["perturbed_losses", "fd_losses", "debug_probe", "debug_gauss_pairs"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_allocates_for_its_own_stream(device, name):
    """Not for the current one, whose queued work may still use a block just freed, and which may take the
    workspace's block while the call runs."""
    side = fake.Stream(22)
    out = _call(device, name, stream=side)
    (launch,) = [args for n, args in device.library.calls if not n.endswith("bytes")]
    assert launch[-1].value == side.cuda_stream and device.current is device.main
    assert device.allocated and all(s is side for s in device.allocated.values())
    for t in out if isinstance(out, tuple) else (out,):
        assert (t.data_ptr(), device.main) in device.recorded


@pytest.mark.parametrize("name", NAMES)
def test_a_call_without_a_stream_stays_on_the_current_one(device, name):
    _call(device, name)
    (launch,) = [args for n, args in device.library.calls if not n.endswith("bytes")]
    assert launch[-1].value == device.main.cuda_stream
    assert not device.recorded and all(s is device.main for s in device.allocated.values())


@pytest.mark.parametrize("name,given", [("perturbed_losses", ("Lplus", "Lminus")), ("fd_losses", ("L", "L0"))])
def test_a_call_with_all_its_buffers_allocates_nothing(device, name, given):
    side = fake.Stream(22)
    buffers = {n: torch.zeros(4) for n in given}
    ws = torch.zeros(4096, dtype=torch.uint8)
    _call(device, name, stream=side, workspace=ws, **buffers)
    assert not device.allocated and not device.recorded


@pytest.mark.parametrize("estimator", ["cd", "fd"])
def test_training_allocates_for_its_stream(device, estimator):
    from paper_2505_17852_amd import train
    side = fake.Stream(22)
    train.train(CFG, torch.zeros(64), torch.zeros(2, 9, dtype=torch.int32), None, N=4, eps=1e-3, lr=1e-2, steps=2, seed0=0,
                stream=side, estimator=estimator)
    assert device.allocated and all(s is side for s in device.allocated.values())
