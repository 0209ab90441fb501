"""Calls of the layers on another stream than the current one, on the host: which stream every buffer of
theirs is allocated for, which launches, and whose uses are recorded."""
import pytest
import torch

import layers_fake as fake


@pytest.fixture
def device(monkeypatch):
    from paper_2505_17852_amd import layers
    dev = fake.Device(layers, monkeypatch)
    dev.layers = layers
    return dev


def attention_inputs(B=2, T=70, H=2, D=8):
    return [torch.ones(B, T, H, D) for _ in range(3)] + [torch.zeros(H)]


def _adamw(device, what, stream):
    opt = device.layers.AdamW([torch.ones(300)], state_bits=8)
    device.allocated.clear()
    if what == "moments":
        return opt.moments(stream=stream), [opt.m]
    grads = [torch.ones(300)]
    return opt.step(grads, stream=stream), grads + opt.params + [opt.m, opt.v, opt.m_scale, opt.v_scale]


def _call(device, name, stream):
    """(what the call returned, the tensors that it was given)."""
    m = device.layers
    q, k, v, decay = given = attention_inputs()
    state = torch.zeros(2, 2, 8, 8)
    if name == "forward":
        return m.linear_attention(*given, initial_state=state, return_state=True, stream=stream), given + [state]
    if name == "forward in place":
        return m.linear_attention(*given, initial_state=state, final_state=state, stream=stream), given + [state]
    if name == "backward":
        return m.linear_attention_backward(torch.ones_like(q), *given, initial_state=state, stream=stream), given + [state]
    if name == "token":
        return m.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state, stream=stream), [decay, state]
    x, w = torch.ones(6, 8), torch.ones(8)
    if name == "norm":
        return m.layer_norm(x, w, stream=stream), [x, w]
    if name == "norm backward":
        mean, rstd, dy = torch.ones(6), torch.ones(6), torch.ones(6, 8)
        return m.layer_norm_backward(dy, x, w, mean, rstd, stream=stream), [dy, x, w, mean, rstd]
    return _adamw(device, name, stream)


NAMES = ["forward", "forward in place", "backward", "token", "norm", "norm backward", "adamw", "moments"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_allocates_for_its_own_stream(device, name):
    """Not for the current one, where a block just freed may still be in use by queued work."""
    side = fake.Stream(22)
    out, given = _call(device, name, side)
    launches = [args for n, args in device.library.calls if not n.endswith("workspace_bytes")]
    assert len(launches) == 1 and launches[0][-1] == side.cuda_stream
    ours = {p: s for p, s in device.allocated.items() if p not in {t.data_ptr() for t in given}}
    assert (ours or name == "adamw") and all(s is side for s in ours.values())
    assert device.current is device.main
    out = [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]
    for t in out:  # used by the caller's stream
        assert (t.data_ptr(), device.main) in device.recorded
    if name != "moments":
        for t in given:  # held until the side stream has done with them
            assert (t.data_ptr(), side) in device.recorded


@pytest.mark.parametrize("name", NAMES)
def test_a_call_without_a_stream_stays_on_the_current_one(device, name):
    _call(device, name, None)
    launches = [args for n, args in device.library.calls if not n.endswith("workspace_bytes")]
    assert len(launches) == 1 and launches[0][-1] == device.main.cuda_stream
    assert not device.recorded and all(s is device.main for s in device.allocated.values())
