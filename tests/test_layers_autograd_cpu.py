"""The layers and torch's autograd, on the host: nothing is silently cut off from a gradient."""
import pytest
import torch

import layers_fake as fake


@pytest.fixture
def device(monkeypatch):
    from paper_2505_17852_amd import layers
    dev = fake.Device(layers, monkeypatch)
    dev.layers = layers
    return dev


def calls(m):
    q = lambda: torch.ones(2, 5, 2, 8)  # noqa: E731
    row = lambda: torch.ones(2, 2, 8)  # noqa: E731
    decay = torch.zeros(2)
    return {
        "linear_attention": (lambda a: m.linear_attention(a[0], a[1], a[2], decay, initial_state=a[3]),
                             [q(), q(), q(), torch.zeros(2, 2, 8, 8)]),
        "linear_attention_step": (lambda a: m.linear_attention_step(a[0], a[1], a[2], decay, a[3]),
                                  [row(), row(), row(), torch.zeros(2, 2, 8, 8)]),
        "layer_norm": (lambda a: m.layer_norm(*a), [torch.ones(3, 8), torch.ones(8), torch.ones(8)]),
    }


@pytest.mark.parametrize("name", ["linear_attention", "linear_attention_step", "layer_norm"])
def test_inputs_that_require_gradients_are_refused_where_they_would_be_recorded(device, name):
    f, args = calls(device.layers)[name]
    f(args)
    before = len(device.library.calls)
    for i in range(len(args)):
        args[i].requires_grad_(True)
        with pytest.raises(ValueError, match="no_grad"):
            f(args)
        assert len(device.library.calls) == before
        with torch.no_grad():
            f(args)
        with torch.inference_mode():
            f(args)
        args[i].requires_grad_(False)
        before = len(device.library.calls)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_counts_as_a_change_of_its_parameters(device, bits):
    """A gradient whose backward pass needs the values from before the step fails in torch, as after torch's own optimizers."""
    w = torch.ones(4, requires_grad=True)
    opt = device.layers.AdamW([w], state_bits=bits)
    loss = (w * w).sum()
    opt.step([torch.ones(4)])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    (w * w).sum().backward()
    assert torch.equal(w.grad, torch.full((4,), 2.0))
