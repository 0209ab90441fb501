"""AdamW's own checks on the host: nothing reaches the library that would make the kernels write past a buffer, or
write one value twice."""
import pytest
import torch

import layers_fake as fake


@pytest.fixture
def device(monkeypatch):
    from paper_2505_17852_amd import layers
    dev = fake.Device(layers, monkeypatch)
    dev.layers = layers
    return dev


@pytest.mark.parametrize("bits", [32, 8])
def test_the_moments_type_cannot_change(device, bits):
    """Moments of 8 bits read as 32 would lie past their buffers' ends."""
    opt = device.layers.AdamW([torch.ones(300)], state_bits=bits)
    with pytest.raises(AttributeError):
        opt.state_bits = 40 - bits
    opt.step([torch.ones(300)])
    assert opt.state_bits == bits and len(device.library.named("zo_adamw")) == 1
