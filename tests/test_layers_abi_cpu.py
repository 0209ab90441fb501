"""Host-side checks of the layers' C ABI (no GPU needed): exported symbols, sizes and
refusals, which are reported before anything touches a device."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "zo_layers.h")
FAKE = 0x10000


@pytest.fixture(scope="module")
def layers():
    from paper_2505_17852_amd import layers as m
    from paper_2505_17852_amd import zo
    if not os.path.exists(zo.LIB_PATH):
        from paper_2505_17852_amd import build
        build.build()
    m.lib()
    return m


def test_library_exports_every_declared_symbol(layers):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(zo_[a-z_0-9]+)\s*\(", text)))
    assert len(names) >= 9
    for n in names:
        assert hasattr(layers.lib(), n), n


def test_header_is_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "abi.c"
    src.write_text('#include "zo_layers.h"\nint main(void) { zo_linattn s = {1, 1, 1, 1, 8, 8, ZO_WFP32, 1.0f}; '
                   "return s.batch - 1; }\n")
    subprocess.run([gcc, "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o",
                    str(tmp_path / "abi.o")], check=True)


def shape(layers, **kw):
    s = dict(batch=2, length=8, q_heads=4, kv_heads=2, key_dim=32, value_dim=32, dtype=0, scale=1.0)
    s.update(kw)
    return layers._SHAPE.pack(*s.values())


def heads(layers, data=FAKE):
    return layers._HEADS.pack(data or 0, 1, 1, 1)


def attention(layers, s, data=FAKE, decay=FAKE, lengths=None, initial=None, final=None, ws=FAKE, wn=1 << 40):
    h = heads(layers, data)
    return layers.lib().zo_linear_attention(s, h, h, h, h, decay, lengths, initial, final, ws, wn, None)


def error():
    from paper_2505_17852_amd import zo
    return zo.lib().zo_last_error().decode()


@pytest.mark.parametrize("bad,status,word", [
    (dict(batch=-1), -1, "batch"), (dict(length=-1), -1, "length"), (dict(q_heads=3), -1, "multiple"),
    (dict(kv_heads=0), -1, "kv_heads"), (dict(q_heads=0), -1, "q_heads"), (dict(key_dim=0), -1, "key_dim"),
    (dict(value_dim=257), -2, "value_dim"), (dict(key_dim=1000), -2, "key_dim"), (dict(dtype=2), -1, "dtype"),
    (dict(scale=float("nan")), -1, "scale"), (dict(scale=float("inf")), -1, "scale"),
    (dict(batch=1 << 20, q_heads=1 << 14), -2, "batch"),
    (dict(length=(1 << 30) + 1), -2, "length"),
])
def test_linear_attention_shapes_are_refused(layers, bad, status, word):
    L, h = layers.lib(), heads(layers)
    s = shape(layers, **bad)
    assert attention(layers, s) == status and word in error()
    assert L.zo_linear_attention_backward(s, h, h, h, h, h, h, h, FAKE, None, None, None, None, FAKE, 1 << 40,
                                          None) == status
    assert L.zo_linear_attention_step(s, h, h, h, h, FAKE, FAKE, 1 << 30, None, None) == status
    assert L.zo_linear_attention_workspace_bytes(s, 0) == 0


def test_linear_attention_pointers_are_refused(layers):
    L, s, h = layers.lib(), shape(layers), heads(layers)
    assert attention(layers, s, data=None) == -1 and "data" in error()
    assert attention(layers, s, data=FAKE + 2) == -1 and "aligned" in error()
    assert attention(layers, s, decay=None) == -1 and "log_decay" in error()
    for name in ("decay", "lengths", "initial", "final"):
        assert attention(layers, s, **{name: FAKE + 2}) == -1 and "aligned" in error()
    assert attention(layers, s, ws=FAKE + 8) == -1 and "workspace" in error()
    assert attention(layers, s, initial=FAKE, final=FAKE) == -1 and "different" in error()
    assert L.zo_linear_attention_backward(s, h, h, h, h, h, h, h, FAKE, None, None, FAKE, FAKE, FAKE, 1 << 40,
                                          None) == -1 and "different" in error()
    far = layers._HEADS.pack(FAKE, 1, (1 << 24) + 1, 1)
    assert L.zo_linear_attention(s, h, far, h, h, FAKE, None, None, None, FAKE, 1 << 40, None) == -2
    assert L.zo_linear_attention(s, None, h, h, h, FAKE, None, None, None, FAKE, 1 << 40, None) == -1
    assert L.zo_linear_attention(None, h, h, h, h, FAKE, None, None, None, FAKE, 1 << 40, None) == -1
    assert L.zo_linear_attention_backward(s, h, h, h, None, h, h, h, FAKE, None, None, None, None, FAKE,
                                          1 << 40, None) == -1
    step = L.zo_linear_attention_step
    assert step(s, h, h, h, h, FAKE, FAKE, 1, None, None) == -1 and "n_slots" in error()
    assert step(s, h, h, h, h, FAKE, FAKE, -1, FAKE, None) == -1
    assert step(s, h, h, h, h, FAKE, None, 4, None, None) == -1
    assert step(s, h, h, h, h, FAKE, FAKE, 4, FAKE + 1, None) == -1 and "slots" in error()
    need = L.zo_linear_attention_workspace_bytes(shape(layers, batch=1, length=1 << 16, dtype=1), 0)
    if need:
        big = shape(layers, batch=1, length=1 << 16, dtype=1)
        assert attention(layers, big, wn=need - 1) == -4 and attention(layers, big, ws=None, wn=need) == -1


def norm(layers, xt=0, wt=0, rows=4, D=8, x=FAKE, w=None, b=None, eps=1e-5, y=FAKE, mean=None, rstd=None):
    return layers.lib().zo_layer_norm(xt, wt, rows, D, x, D, w, b, eps, y, D, mean, rstd, None)


@pytest.mark.parametrize("bad,status", [
    (dict(xt=3), -1), (dict(wt=-1), -1), (dict(rows=-1), -1), (dict(D=0), -1), (dict(D=1 << 31), -2),
    (dict(rows=1 << 40), -2), (dict(x=None), -1), (dict(y=None), -1), (dict(mean=FAKE), -1), (dict(rstd=FAKE), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(x=FAKE + 2), -1), (dict(xt=1, x=FAKE + 1), -1),
    (dict(w=FAKE + 2), -1), (dict(b=FAKE + 2), -1), (dict(mean=FAKE + 1, rstd=FAKE), -1),
])
def test_layer_norm_arguments_are_refused(layers, bad, status):
    assert norm(layers, **bad) == status and error()


def test_layer_norm_backward_arguments_are_refused(layers):
    L = layers.lib()
    need = L.zo_layer_norm_workspace_bytes(1000, 64)
    assert need > 0 and L.zo_layer_norm_workspace_bytes(-1, 64) == 0

    def call(rows=1000, dy=FAKE, x=FAKE, mean=FAKE, rstd=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, wn=need):
        return L.zo_layer_norm_backward(0, 0, rows, 64, dy, 64, x, 64, None, mean, rstd, dx, 64, dw, db, ws, wn, None)

    for name in ("dy", "x", "mean", "rstd", "dx"):
        assert call(**{name: None}) == -1
        assert call(**{name: FAKE + 2}) == -1
    assert call(dw=FAKE + 2) == -1 and call(rows=-1) == -1
    assert call(ws=None) == -1 and call(ws=FAKE + 4) == -1 and call(wn=need - 1) == -4


def adamw(layers, cfg=(), tensor=(), n=1, m=FAKE, v=FAKE, ms=None, vs=None, gs=None, sk=None, tensors=True):
    c = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, state_bits=32)
    c.update(cfg)
    t = dict(param=FAKE, grad=FAKE, n=8, state_offset=0, weight_decay=0.0, pdtype=0, gdtype=0)
    t.update(tensor)
    table = (layers._Tensor * 1)(layers._Tensor(*t.values()))
    return layers.lib().zo_adamw(C.byref(layers._AdamWConfig(*c.values())), table if tensors else None, n, m, v, ms, vs,
                                 gs, sk, None)


@pytest.mark.parametrize("kw", [
    dict(cfg=dict(lr=float("nan"))), dict(cfg=dict(eps=-1.0)), dict(cfg=dict(beta1=1.0)), dict(cfg=dict(beta2=-0.1)),
    dict(cfg=dict(beta1=float("nan"))), dict(cfg=dict(step=0)), dict(cfg=dict(state_bits=16)), dict(n=-1),
    dict(tensors=False), dict(tensor=dict(n=-1)), dict(tensor=dict(n=1 << 60)), dict(tensor=dict(pdtype=2)),
    dict(tensor=dict(gdtype=-1)), dict(tensor=dict(param=None)), dict(tensor=dict(grad=None)),
    dict(tensor=dict(param=FAKE + 2)), dict(tensor=dict(gdtype=1, grad=FAKE + 1)), dict(tensor=dict(state_offset=8)),
    dict(tensor=dict(state_offset=-256)), dict(tensor=dict(weight_decay=float("inf"))), dict(m=None), dict(v=None),
    dict(m=FAKE + 4), dict(cfg=dict(state_bits=8)), dict(ms=FAKE, vs=FAKE), dict(gs=FAKE + 1), dict(sk=FAKE + 2),
])
def test_adamw_arguments_are_refused(layers, kw):
    assert adamw(layers, **kw) == -1 and error()


def test_adamw_moments_arguments_are_refused(layers):
    f = layers.lib().zo_adamw_moments
    assert f(255, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == -1
    assert f(-256, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == -1
    assert f(256, FAKE, FAKE, FAKE, FAKE, None, FAKE, None) == -1
    assert f(256, FAKE, FAKE, FAKE, FAKE, FAKE + 4, FAKE, None) == -1


def test_binding_refuses_what_does_not_fit(layers):
    """The binding's own checks: host tensors, types and shapes."""
    x = torch.zeros(2, 8, 4, 32)
    with pytest.raises(ValueError, match="device"):
        layers.linear_attention(x, x, x, torch.zeros(4))
    with pytest.raises(ValueError, match="device"):
        layers.linear_attention_step(x[:, 0], x[:, 0], x[:, 0], torch.zeros(4), torch.zeros(2, 4, 32, 32))
    with pytest.raises(ValueError, match="device"):
        layers.layer_norm(x)
    with pytest.raises(ValueError, match="device"):
        layers.layer_norm_backward(x, x, None, x, x)
    with pytest.raises(ValueError, match="device"):
        layers.AdamW([x])
    with pytest.raises(ValueError, match="no parameters"):
        layers.AdamW([])
    with pytest.raises(ValueError, match="state_bits"):
        layers.AdamW([x], state_bits=4)


def test_performance_cases_import_without_a_gpu():
    import importlib.util
    spec = importlib.util.spec_from_file_location("operators", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    cases = m.listed()
    assert len({c["name"] for c in cases}) == len(cases)
    assert all(m.work(c)["bytes"] > 0 for c in cases)


def test_states_that_share_memory_in_part_are_refused(layers):
    states = 2 * 2 * 32 * 32 * 4  # bytes of shape()'s states
    s, h = shape(layers), heads(layers)
    for a, b in ((FAKE, FAKE + 4), (FAKE + states - 4, FAKE), (FAKE, FAKE + states // 2)):
        assert attention(layers, s, initial=a, final=b) == -1 and "different" in error()
        st = layers.lib().zo_linear_attention_backward(s, h, h, h, h, h, h, h, FAKE, None, None, a, b, FAKE, 1 << 40,
                                                       None)
        assert st == -1 and "different" in error()


def test_no_kernel_that_no_call_reaches(layers):
    """Slices of 128 columns have 256 workgroups and more, which are never split into segments: no kernel for both."""
    from paper_2505_17852_amd import zo
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    names = subprocess.run([nm, "-C", zo.LIB_PATH], check=True, capture_output=True, text=True).stdout
    chunks = set(re.findall(r"linattn_chunk_kernel<([^>]*)>", names))
    assert any(x.endswith("128, 128, true, false") for x in chunks)
    assert not [x for x in chunks if x.endswith(("128, 128, true, true", "128, 128, false, true"))]
