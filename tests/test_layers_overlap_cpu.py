"""Outputs of the layers that share memory with what the call reads, or with one another, are refused on the host.
Every call here is one that is refused."""
import pytest

FAKE = 0x10000000
B, T, HQ, HKV, D = 2, 8, 4, 2, 32
SHAPE = dict(batch=B, length=T, q_heads=HQ, kv_heads=HKV, key_dim=D, value_dim=D, dtype=0, scale=1.0)


@pytest.fixture(scope="module")
def layers():
    import os
    from paper_2505_17852_amd import layers as m
    from paper_2505_17852_amd import zo
    if not os.path.exists(zo.LIB_PATH):
        from paper_2505_17852_amd import build
        build.build()
    m.lib()
    return m


def error():
    from paper_2505_17852_amd import zo
    return zo.lib().zo_last_error().decode()


def heads(layers, n, values=0, at=1, strides=None):
    """A contiguous [B][T][n][D] at buffer `at`, moved by `values`."""
    return layers._HEADS.pack(FAKE + at * 0x1000000 + 4 * values, *(strides or (T * n * D, n * D, D)))


def forward(layers, **kw):
    t = dict(q=heads(layers, HQ, at=1), k=heads(layers, HKV, at=2), v=heads(layers, HKV, at=3), o=heads(layers, HQ, at=4))
    t.update(kw)
    return layers.lib().zo_linear_attention(layers._SHAPE.pack(*SHAPE.values()), t["q"], t["k"], t["v"], t["o"], FAKE,
                                            None, None, None, FAKE, 1 << 40, None)


def backward(layers, **kw):
    t = {n: heads(layers, HQ if n in ("do", "q", "dq") else HKV, at=i + 1)
         for i, n in enumerate(("do", "q", "k", "v", "dq", "dk", "dv"))}
    t.update(kw)
    return layers.lib().zo_linear_attention_backward(layers._SHAPE.pack(*SHAPE.values()), *t.values(), FAKE, None, None,
                                                     None, None, FAKE, 1 << 40, None)


WIDE = (T * 8 * D, 8 * D, D)  # heads of one projection [B][T][8][D]


def test_outputs_of_linear_attention(layers):
    h = lambda *a, **kw: heads(layers, *a, **kw)  # noqa: E731
    size = B * T * HQ * D
    assert forward(layers, o=h(HQ, at=1)) == -1 and "o and q" in error()
    assert forward(layers, o=h(HQ, size - 1, at=1)) == -1 and "o and q" in error()
    assert forward(layers, o=h(HQ, -size + 1, at=3)) == -1 and "o and v" in error()
    # slices of one projection whose heads overlap by one, and by one value
    assert forward(layers, k=h(HKV, 4 * D, at=6, strides=WIDE), o=h(HQ, D, at=6, strides=WIDE)) == -1 and "k" in error()
    assert forward(layers, k=h(HKV, 4 * D - 1, at=6, strides=WIDE), o=h(HQ, 0, at=6, strides=WIDE)) == -1
    # the last position's values reach into the next sequence's first
    assert forward(layers, v=h(HKV, 7 * D, at=6, strides=WIDE), o=h(HQ, 0, at=6, strides=WIDE)) == -1
    # backwards in memory
    assert forward(layers, q=h(HQ, size - D, at=1, strides=(-T * HQ * D, -HQ * D, -D)), o=h(HQ, 5, at=1)) == -1
    # all sequences of one output in one place
    assert forward(layers, o=h(HQ, at=4, strides=(0, HQ * D, D))) == -1 and "o" in error()


def test_gradients_of_linear_attention(layers):
    h = lambda *a, **kw: heads(layers, *a, **kw)  # noqa: E731
    for out, n in (("dq", HQ), ("dk", HKV), ("dv", HKV)):
        for i, name in enumerate(("do", "q", "k", "v")):
            assert backward(layers, **{out: h(n, at=i + 1)}) == -1 and f"{out} and {name}" in error()
    assert backward(layers, dk=h(HKV, at=5)) == -1 and "dk and dq" in error()
    assert backward(layers, dv=h(HKV, D, at=6)) == -1 and "dv and dk" in error()
    assert backward(layers, dk=h(HKV, 4 * D, at=9, strides=WIDE), dv=h(HKV, 5 * D, at=9, strides=WIDE)) == -1


def test_the_output_of_a_step(layers):
    f = layers.lib().zo_linear_attention_step
    t = [layers._HEADS.pack(FAKE + i * 0x1000000, n * D, 0, D) for i, n in enumerate((HQ, HKV, HKV))]
    for i in range(3):
        assert f(layers._SHAPE.pack(*SHAPE.values()), *t, t[i], FAKE, FAKE, B, None, None) == -1 and "o and" in error()


def norm(layers, x=FAKE, xs=64, y=FAKE + 0x1000000, ys=64, rows=10, D=64):
    return layers.lib().zo_layer_norm(0, 0, rows, D, x, xs, None, None, 1e-5, y, ys, None, None, None)


def test_rows_of_a_norm(layers):
    """In place as a whole is allowed; anything else that shares memory is not."""
    assert norm(layers, y=FAKE + 4) == -1 and "y and x" in error()
    assert norm(layers, y=FAKE + 4 * 64) == -1 and "y and x" in error()
    assert norm(layers, xs=64, ys=128, y=FAKE) == -1
    assert norm(layers, xs=200, ys=200, y=FAKE + 4 * 137) == -1
    assert norm(layers, ys=0) == -1 and "y" in error()
    need = layers.lib().zo_layer_norm_workspace_bytes(10, 64)
    for dx in (FAKE + 4, FAKE + 0x1000000 + 4 * 63):
        st = layers.lib().zo_layer_norm_backward(0, 0, 10, 64, FAKE, 64, FAKE + 0x1000000, 64, None, FAKE + 0x2000000,
                                                 FAKE + 0x3000000, dx, 64, FAKE + 0x4000000, FAKE + 0x5000000,
                                                 FAKE + 0x6000000, need, None)
        assert st == -1 and "dx and" in error()
