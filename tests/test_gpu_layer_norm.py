"""Layer norm on the GPU, forward and backward, against 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layers_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_17852_amd import layers as m
    m.lib()
    return m


def rand(rng, shape, dtype="f32", scale=1.0, shift=0.0):
    t = torch.from_numpy((scale * rng.standard_normal(shape) + shift).astype(np.float32)).to(DT[dtype])
    return t.cuda(), t.float().numpy()


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def close(name, got, want, bound):
    off = np.abs(host(got) - want)
    worst = float((off / bound).max()) if off.size else 0.0
    print(f"{name}: worst error {worst:.3f} of its bound", flush=True)
    assert np.isfinite(host(got)).all() and worst <= 1.0, name


def check(layers, rng, rows, D, dtype, wdtype, shift=0.3, weight=True):
    """Bounds: mean and variance are sums of D terms in fp32, in a tree over threads of at
    most 16 + ceil(D / 8192) 8 terms each, joined by at most 22 more additions."""
    x_d, x = rand(rng, (rows, D), dtype, 1.5, shift)
    dy_d, dy = rand(rng, (rows, D), dtype)
    w_d, w = rand(rng, D, wdtype, 0.3, 1.0) if weight else (None, None)
    b_d, b = rand(rng, D, wdtype, 0.3) if weight else (None, None)
    y, mean, rstd = layers.layer_norm(x_d, w_d, b_d, eps=EPS)
    dx, dw, db = layers.layer_norm_backward(dy_d, x_d, w_d, mean, rstd)
    want, xhat, wmean, wrstd = ref.norm(x, w, b, EPS)
    wdx, wdw, wdb = ref.norm_backward(dy, x, w, EPS)
    u, n = ref.unit(dtype), 40 + 8 * (D // 8192)
    # the mean's error, against the row's mean size; xhat takes it times rstd
    merr = ref.ulps(n) * np.abs(x).mean(1)
    close("mean", mean, wmean, merr + 1e-37)
    # the variance's relative error: n roundings, and the mean's error squared against the variance
    rerr = ref.ulps(n) + (merr * wrstd) ** 2
    close("rstd", rstd, wrstd, rerr * wrstd)
    xerr = (merr * wrstd)[:, None] + (rerr[:, None] + ref.ulps(4)) * (np.abs(xhat) + np.abs(x * wrstd[:, None]) * 2 ** -20)
    wa = 1.0 if w is None else np.abs(w)
    close("y", y, want, u * np.abs(want) + xerr * wa + ref.ulps(4) * (np.abs(xhat) * wa + np.abs(want)) + 1e-37)
    g = np.abs(dy) * wa
    m0, m1 = g.mean(1, keepdims=True), (g * np.abs(xhat)).mean(1, keepdims=True)
    gerr = (g * xerr).mean(1, keepdims=True)
    spread = g + m0 + np.abs(xhat) * m1
    close("dx", dx, wdx, u * np.abs(wdx) + wrstd[:, None] * ((ref.ulps(n + 8) + rerr[:, None]) * spread + xerr * m1
                                                              + np.abs(xhat) * gerr) + 1e-37)
    # columns: a workgroup's rows one after another, then the workgroups (at most 2,048 of them)
    m = 24 + rows // 256 + min(rows, 2048) // 4
    close("dw", dw, wdw, ref.ulps(m) * (np.abs(dy) * np.abs(xhat)).sum(0) + (np.abs(dy) * xerr).sum(0) + 1e-37)
    close("db", db, wdb, ref.ulps(m) * np.abs(dy).sum(0) + 1e-37)


SIZES = [(1, 1), (3, 2), (5, 7), (64, 64), (33, 100), (257, 256), (130, 1003), (4, 1024), (9, 1025), (70, 2048),
         (31, 4096), (5, 4097), (18, 8192), (3, 8193), (6, 20000), (2049, 40), (5000, 96)]


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,D", SIZES)
def test_forward_and_backward(layers, rows, D, types):
    check(layers, np.random.default_rng(rows + D), rows, D, *types)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_weight_and_with_a_large_mean(layers, dtype):
    check(layers, np.random.default_rng(2), 40, 500, dtype, dtype, weight=False)
    check(layers, np.random.default_rng(3), 40, 500, "f32", "f32", shift=1000.0)


def test_constant_rows(layers):
    """No variance: xhat is zero, y the bias, and eps alone holds the gradient finite."""
    x = torch.full((3, 200), 5.0, device="cuda")
    b = torch.randn(200, device="cuda")
    y, mean, rstd = layers.layer_norm(x, None, b, eps=1e-5)
    assert torch.equal(y, b.expand(3, 200)) and bool((mean == 5.0).all())
    dx, dw, _ = layers.layer_norm_backward(torch.ones_like(x), x, None, mean, rstd)
    assert not dx.any() and not dw.any()


def test_a_row_that_is_not_finite_is_alone(layers):
    x = torch.randn(8, 300, device="cuda")
    good, mean, rstd = layers.layer_norm(x)
    x[3, 299] = float("nan")
    x[5, 0] = float("inf")
    y, mean, rstd = layers.layer_norm(x)
    rows = [0, 1, 2, 4, 6, 7]
    assert torch.equal(y[rows], good[rows]) and torch.isnan(y[3]).all() and not torch.isfinite(y[5]).any()
    dx, _, _ = layers.layer_norm_backward(torch.ones_like(x), x, None, mean, rstd)
    assert torch.isfinite(dx[rows]).all() and torch.isnan(dx[3]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [96, 1003, 4096, 9000])
def test_strided_rows_and_in_place(layers, dtype, D):
    rng = np.random.default_rng(D)
    wide, _ = rand(rng, (50, 2 * D + 3), dtype)
    x, dy = wide[:, 1:D + 1], wide[:, D + 2:2 * D + 2]
    w, _ = rand(rng, D, dtype, 0.2, 1.0)
    want = layers.layer_norm(x.contiguous(), w)
    got = layers.layer_norm(x, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    grads = layers.layer_norm_backward(dy.contiguous(), x.contiguous(), w, *want[1:])
    for out in (dy, x):
        held = wide.clone()
        x2, dy2 = held[:, 1:D + 1], held[:, D + 2:2 * D + 2]
        res = layers.layer_norm_backward(dy2, x2, w, *want[1:], out=dy2 if out is dy else x2)
        assert all(torch.equal(a, b) for a, b in zip(res, grads))
    y = x
    layers.layer_norm(x, w, out=y)
    assert torch.equal(x, want[0])
    assert torch.equal(wide[:, 0], wide[:, 0]) and torch.equal(layers.layer_norm(
        want[0].view(5, 10, D), w)[0].view(50, D), layers.layer_norm(want[0], w)[0])


def test_gradients_against_differences(layers):
    """Directional differences in x, w and b (fp32). With steps of 1e-2 the third derivative
    leaves at most 1e-3 of the change, and rounding 1e-4."""
    rng = np.random.default_rng(4)
    (x, _), (w, _), (b, _), (dy, _) = (rand(rng, (60, 130), scale=2.0), rand(rng, 130, shift=1.0), rand(rng, 130),
                                       rand(rng, (60, 130)))
    _, mean, rstd = layers.layer_norm(x, w, b, eps=EPS)
    grads = layers.layer_norm_backward(dy, x, w, mean, rstd)

    def loss(x, w, b):
        return float((layers.layer_norm(x, w, b, eps=EPS)[0].double() * dy.double()).sum())

    for i, g in enumerate(grads):
        d = g / g.norm() * np.sqrt(g.numel())

        def f(z):
            a = [x, w, b]
            a[i] = z
            return loss(*a)
        want = ref.finite_difference(f, (x, w, b)[i], d, 1e-2)
        got = float((g.double() * d.double()).sum())
        print(f"{got} difference {want}", flush=True)
        assert abs(got - want) <= 2e-3 * abs(want)


def test_the_same_bits_on_another_stream_and_in_a_graph(layers):
    rng = np.random.default_rng(9)
    (x, _), (dy, _), (w, _) = rand(rng, (3000, 512), "bf16"), rand(rng, (3000, 512), "bf16"), rand(rng, 512, "bf16")

    def call(stream=None):
        y, mean, rstd = layers.layer_norm(x, w, stream=stream)
        return [y, *layers.layer_norm_backward(dy, x, w, mean, rstd, stream=stream)]

    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        for t in held:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_no_rows(layers):
    x = torch.zeros(0, 64, device="cuda")
    y, mean, rstd = layers.layer_norm(x)
    dx, dw, db = layers.layer_norm_backward(x, x, None, mean, rstd)
    assert y.shape == x.shape == dx.shape and not dw.any() and not db.any()


@pytest.mark.parametrize("D", [100, 96, 250])
def test_constant_rows_whose_mean_times_rstd_overflows(layers, D):
    """Rows of 2^120 (sums and means are exact): xhat is zero, dx = rstd (dy - avg(dy)), though 2^120 rstd is not finite.
    The average carries at most 38 roundings of sums and a division, dx four more."""
    x = torch.full((5, D), 2.0 ** 120, device="cuda")
    dy, dy_h = rand(np.random.default_rng(D), (5, D))
    y, mean, rstd = layers.layer_norm(x, eps=EPS)
    assert not y.any() and bool((mean == 2.0 ** 120).all())
    dx, dw, db = layers.layer_norm_backward(dy, x, None, mean, rstd)
    g, r = dy_h.astype(np.float64), 1.0 / np.sqrt(EPS)
    want = r * (g - g.mean(1, keepdims=True))
    close("dx", dx, want, 43 * ref.unit("f32") * r * (np.abs(g) + np.abs(g).mean(1, keepdims=True)))
    assert not dw.any() and torch.isfinite(db).all()


def test_rows_between_the_input_s_rows(layers):
    """Input, output and gradient as columns of one buffer share no value, and are taken; shifted by one they are refused."""
    from paper_2505_17852_amd import zo
    rng = np.random.default_rng(14)
    wide, _ = rand(rng, (40, 300))
    x, y, dx = wide[:, :96], wide[:, 96:192], wide[:, 204:300]
    want = layers.layer_norm(x.contiguous())
    got = layers.layer_norm(x, out=y)
    assert torch.equal(y, want[0]) and got[0] is y
    dy = torch.ones_like(want[0])
    grads = layers.layer_norm_backward(dy, x.contiguous(), None, *want[1:])
    assert torch.equal(layers.layer_norm_backward(dy, x, None, *want[1:], out=dx)[0], grads[0]) and torch.equal(dx, grads[0])
    for out in (wide[:, 1:97], wide[:, 95:191], torch.zeros(1, 96, device="cuda").expand(40, 96)):
        with pytest.raises(zo.ZoError, match="share memory|one place"):
            layers.layer_norm(x, out=out)


def test_a_row_past_the_threads_of_one_grid_dimension(layers):
    """One row of 2^28 + 65 values: the column sums (of one row) are dy xhat and dy, all of them, xhat by the mean and rstd
    that the call keeps. Here and in torch's, three roundings each of values up to 6.5 |dy|: 6 x 6.5 x 2^-24 |dy|."""
    D = (1 << 28) + 65
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(1, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn(1, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    _, mean, rstd = layers.layer_norm(x)
    _, dw, db = layers.layer_norm_backward(dy, x, None, mean, rstd)
    assert torch.equal(db, dy[0].float())
    assert float(((dw - dy[0].float() * ((x[0].float() - mean) * rstd)).abs() / dy[0].float().abs().clamp(min=1e-3)).max()) <= 39 * 2.0 ** -24


MANY_ROWS = [(1300, 1025), (2100, 2048), (1100, 8192), (600, 9000), (2500, 4096)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,D", MANY_ROWS)
def test_several_rows_for_each_workgroup(layers, rows, D, dtype):
    """More rows than workgroups where several waves share one."""
    check(layers, np.random.default_rng(rows), rows, D, dtype, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,D", MANY_ROWS)
def test_several_rows_in_place_between_gaps(layers, rows, D, dtype):
    """dx in place of dy and of x, y in place of x: the same bits as apart, and no other value of the buffer changes."""
    rng = np.random.default_rng(D)
    wide, _ = rand(rng, (rows, 2 * D + 5), dtype)
    w, _ = rand(rng, D, dtype, 0.2, 1.0)
    at = {"x": slice(1, D + 1), "dy": slice(D + 3, 2 * D + 3)}
    x, dy = (wide[:, at[n]].contiguous() for n in ("x", "dy"))
    y, mean, rstd = layers.layer_norm(x, w)
    grads = layers.layer_norm_backward(dy, x, w, mean, rstd)

    def others(buffer, name):
        kept = torch.ones(buffer.shape[1], dtype=torch.bool, device="cuda")
        kept[at[name]] = False
        return torch.equal(buffer[:, kept], wide[:, kept])

    for name in ("dy", "x"):
        held = wide.clone()
        got = layers.layer_norm_backward(held[:, at["dy"]], held[:, at["x"]], w, mean, rstd, out=held[:, at[name]])
        assert all(torch.equal(a, b) for a, b in zip(got, grads)) and others(held, name)
        assert torch.equal(held[:, at[name]], grads[0])
    held = wide.clone()
    layers.layer_norm(held[:, at["x"]], w, out=held[:, at["x"]])
    assert torch.equal(held[:, at["x"]], y) and others(held, "x")
