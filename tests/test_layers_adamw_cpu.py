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


def test_parameters_that_share_memory_are_refused(device):
    """Tied tensors, the same one twice and views that overlap in part: one launch would write their values in any order."""
    flat = torch.ones(64)
    for params in ([flat, flat], [flat[:40], flat[39:]], [flat[8:16], torch.ones(5), flat], [flat.view(8, 8), flat[63:]]):
        with pytest.raises(ValueError, match="share memory"):
            device.layers.AdamW(params)
    for params in ([flat[:40], flat[40:]], [flat[40:], flat[:0], flat[:40], flat[3:3]], [flat]):
        device.layers.AdamW(params)


def _adamw(layers, *tensors):
    """zo_adamw's status for tensors of (address, values, state_offset[, type]); every pointer is refused before use."""
    import ctypes as C
    from paper_2505_17852_amd import zo
    cfg = layers._AdamWConfig(1e-3, 0.9, 0.999, 1e-8, 1, 32)
    table = (layers._Tensor * len(tensors))(*(layers._Tensor(p, 0x10000000, n, off, 0.0, *(t or (0,)), 0)
                                              for p, n, off, *t in tensors))
    st = layers.lib().zo_adamw(C.byref(cfg), table, len(tensors), 0x20000000, 0x30000000, None, None, None, None, None)
    return st, zo.lib().zo_last_error().decode()


@pytest.mark.parametrize("tensors,word", [
    ([(0x10000, 8, 0), (0x10000, 8, 256)], "param"),
    ([(0x10000, 8, 0), (0x1001c, 8, 256)], "param"),
    ([(0x10000, 8, 0, 1), (0x1000e, 8, 256, 1)], "param"),
    ([(0x20000, 8, 0), (0x10000, 1 << 20, 256)], "param"),
    ([(0x10000 + 0x800 * (399 - i), 1024 if i == 200 else 8, 1024 * i) for i in range(400)], "param"),
    ([(0x10000 + 0x800 * i, 8, 1024 * (i ^ 1) if i < 398 else 1024) for i in range(400)], "moments"),
    ([(0x10000, 8, 0), (0x20000, 8, 0)], "moments"),
    ([(0x10000, 257, 0), (0x20000, 8, 256)], "moments"),
    ([(0x10000, 8, 512), (0x20000, 600, 0)], "moments"),
])
def test_the_library_refuses_tensors_that_share_memory(tensors, word):
    """Parameters, or the moments' whole blocks, that overlap in any order of the tensors."""
    from paper_2505_17852_amd import layers
    st, said = _adamw(layers, *tensors)
    assert st == -1 and word in said and "overlap" in said
