"""AdamW over many tensors on the GPU against 64 bits, with 32-bit and 8-bit moments."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layers_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, BETAS, EPS, DECAY = 3e-3, (0.9, 0.99), 1e-8, 0.1


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_17852_amd import layers as m
    m.lib()
    return m


def rand(rng, n, dtype="f32", scale=1.0):
    return torch.from_numpy((scale * rng.standard_normal(n)).astype(np.float32)).to(DT[dtype]).cuda()


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def within(name, got, want, bound):
    off = np.abs(got - want)
    worst = float((off / bound).max()) if off.size else 0.0
    print(f"{name}: worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, name


SETS = {
    "one": [1],
    "sizes": [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 5000, 0, 33],
    "many": [3 + 37 * i % 600 for i in range(150)],
    "large": [300_001, 64, 1_000_000],
}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,gdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("name", list(SETS))
def test_steps(layers, name, dtype, gdtype, bits):
    """Several steps; each is held to 64 bits from the state that the kernel itself was in."""
    rng = np.random.default_rng(len(name) + bits)
    sizes = SETS[name]
    params = [rand(rng, n, dtype, 0.1) for n in sizes]
    decay = [DECAY if i % 2 else 0.0 for i in range(len(sizes))]
    opt = layers.AdamW(params, lr=LR, betas=BETAS, eps=EPS, weight_decay=decay, state_bits=bits)
    for step in range(1, 4):
        before = [host(p) for p in params]
        m0, v0 = (host(x) for x in opt.moments())
        if bits == 8:
            m0, v0 = ref.decode_moments(*(x.cpu().numpy() for x in (opt.m, opt.v, opt.m_scale, opt.v_scale)))
        grads = [rand(rng, n, gdtype, 10.0 ** -step) for n in sizes]
        opt.step(grads)
        assert opt.step_count == step
        m1, v1 = (host(x) for x in opt.moments())
        for i, (p, g, at) in enumerate(zip(params, grads, opt.offsets)):
            n = p.numel()
            if n == 0:
                continue
            s = slice(at, at + n)
            wp, wm, wv = ref.adamw(before[i], host(g), m0[s], v0[s], step, LR, *BETAS, EPS, decay[i])
            # m and v: 3 roundings of their terms (and 5 of the decoded moments); the change: 8 more
            merr = ref.ulps(9) * (np.abs(m0[s]) * BETAS[0] + (1 - BETAS[0]) * np.abs(host(g))) + 1e-44
            verr = ref.ulps(10) * wv + 1e-44
            den = np.sqrt(wv / (1 - BETAS[1] ** step)) + EPS
            change = LR * np.abs(wm) / (1 - BETAS[0] ** step) / den
            cerr = LR * merr / (1 - BETAS[0] ** step) / den + ref.ulps(20) * change
            within(f"p[{i}]", host(p), wp, ref.unit(dtype) * np.abs(wp) + ref.ulps(3) * np.abs(before[i]) + cerr
                   + ref.unit(dtype) * cerr + 1e-40)
            if bits == 32:
                within(f"m[{i}]", m1[s], wm, merr)
                within(f"v[{i}]", v1[s], wv, verr)
            else:
                # half a step of the code at the value, in the root's scale, and the scale's own error
                for what, got, want, err, levels, power in (("m", m1[s], wm, merr, 127, 2), ("v", v1[s], wv, verr, 255, 4)):
                    pad = np.zeros(-n % 256)
                    top = np.abs(np.concatenate([want, pad])).reshape(-1, 256).max(1).repeat(256)[:n] + 1e-300
                    root = (np.abs(want) / top) ** (1.0 / power)
                    reach = top * ((root + 0.502 / levels) ** power - root ** power) + ref.ulps(16) * top * root ** power
                    least = top * (1.0 / levels) ** power if what == "v" else 0.0
                    within(f"{what}[{i}]", got, want, np.maximum(reach, least) + err * 2 + 1e-44)
                    assert what == "m" or (got[want > 1e-40] > 0).all()


def test_codes_are_the_nearest(layers):
    """From given moments and a zero gradient, codes of the decayed moments: beta1 = beta2 = 0.5
    halves exactly, so every block's maximum halves and every code stays."""
    rng = np.random.default_rng(1)
    p = rand(rng, 256 * 40)
    opt = layers.AdamW([p], lr=0.0, betas=(0.5, 0.5), state_bits=8)
    opt.m.copy_(torch.from_numpy(rng.integers(-127, 128, 256 * 40).astype(np.int8)))
    opt.v.copy_(torch.from_numpy(rng.integers(0, 256, 256 * 40).astype(np.uint8)))
    opt.m.view(-1, 256)[:, 7] = 127
    opt.v.view(-1, 256)[:, 9] = 255
    opt.m_scale.uniform_(1e-4, 1.0)
    opt.v_scale.uniform_(1e-8, 1.0)
    m, v, ms, vs = (x.clone() for x in (opt.m, opt.v, opt.m_scale, opt.v_scale))
    opt.step([torch.zeros_like(p)])
    assert torch.equal(opt.m, m) and torch.equal(opt.v, v)
    assert torch.allclose(opt.m_scale, ms / 2, rtol=1e-6) and torch.allclose(opt.v_scale, vs / 2, rtol=1e-6)


@pytest.mark.parametrize("bits", [32, 8])
def test_views_of_one_vector_at_odd_addresses(layers, bits):
    """Tensors that are slices of a flat vector, at any address of their type: the same values as apart."""
    rng = np.random.default_rng(6)
    sizes = [5, 1000, 3, 4099]
    flat = rand(rng, sum(sizes) + 1, "bf16")
    grads = rand(rng, sum(sizes) + 1, "bf16", 0.01)
    views, gviews, at = [], [], 1
    for n in sizes:
        views.append(flat[at:at + n])
        gviews.append(grads[at:at + n])
        at += n
    apart = [v.clone() for v in views]
    first = flat[0].clone()
    for params, gs in ((views, gviews), (apart, [g.clone() for g in gviews])):
        opt = layers.AdamW(params, lr=LR, weight_decay=DECAY, state_bits=bits)
        for _ in range(2):
            opt.step(gs)
    assert all(torch.equal(a, b) for a, b in zip(views, apart)) and torch.equal(flat[0], first)


@pytest.mark.parametrize("bits", [32, 8])
def test_grad_scale_and_skipping(layers, bits):
    rng = np.random.default_rng(7)
    p0, g = rand(rng, 3000), rand(rng, 3000)

    def fresh():
        p = p0.clone()
        return p, layers.AdamW([p], lr=LR, betas=BETAS, weight_decay=DECAY, state_bits=bits)

    (a, oa), (b, ob) = fresh(), fresh()
    skipped = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    oa.step([g * 0.25])
    ob.step([g], grad_scale=torch.tensor([0.25], device="cuda"), skipped=skipped)
    assert torch.equal(a, b) and torch.equal(oa.m, ob.m) and torch.equal(oa.v, ob.v) and int(skipped) == 0
    for bad in (float("nan"), float("inf"), -float("inf")):
        held = [x.clone() for x in (b, ob.m, ob.v)]
        skipped.fill_(7)
        ob.step([g], grad_scale=torch.tensor([bad], device="cuda"), skipped=skipped)
        assert int(skipped) == 1 and all(torch.equal(x, y) for x, y in zip(held, (b, ob.m, ob.v)))
    none = torch.zeros(0, device="cuda")
    opt = layers.AdamW([none], state_bits=bits)
    opt.step([none], skipped=skipped.fill_(7))
    assert int(skipped) == 0


def test_a_bad_gradient_poisons_its_block_alone(layers):
    rng = np.random.default_rng(8)
    for bad in (float("nan"), float("inf")):
        p, g = rand(rng, 1000), rand(rng, 1000)
        g[300] = bad
        opt = layers.AdamW([p], state_bits=8)
        opt.step([g])
        m, v = opt.moments()
        for x in (m, v):
            assert torch.isnan(x[256:512]).all() and torch.isfinite(x[:256]).all() and torch.isfinite(x[512:]).all()
        assert int((~torch.isfinite(p)).sum()) == 1


def test_a_graph_and_another_stream(layers):
    rng = np.random.default_rng(10)
    p0, g = rand(rng, 10_000, "bf16"), rand(rng, 10_000, "bf16")
    p = p0.clone()
    opt = layers.AdamW([p], lr=LR, state_bits=8)
    opt.step([g])
    want = [x.clone() for x in (p, opt.m, opt.v, *opt.moments())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p.copy_(p0)
    q = p0.clone()
    other = layers.AdamW([q], lr=LR, state_bits=8)
    torch.cuda.synchronize()
    other.step([g], stream=side)
    got = other.moments(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (q, other.m, other.v, *got)))
    for x in (opt.m, opt.v, opt.m_scale, opt.v_scale):
        x.zero_()
    opt.step_count = 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g])
        held = opt.moments()
    for _ in range(3):
        p.copy_(p0)
        for x in (opt.m, opt.v, opt.m_scale, opt.v_scale):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (p, opt.m, opt.v, *held)))


@pytest.mark.parametrize("bits", [32, 8])
def test_what_changed_since_construction_is_refused(layers, bits):
    """A parameter whose storage was exchanged, and moments that cannot be: refused on the host, nothing counted."""
    sizes = [300, 40, 1000]
    for change in (lambda p: p.bfloat16(), lambda p: p[:-1].clone(), lambda p: p.cpu(), lambda p: p.repeat(2)[::2]):
        params = [torch.ones(n, device="cuda") for n in sizes]
        grads = [torch.ones(n, device="cuda") for n in sizes]
        opt = layers.AdamW(params, state_bits=bits)
        opt.step(grads)
        keep = params[0].clone()
        params[1].data = change(params[1])
        with pytest.raises(ValueError, match="parameter"):
            opt.step(grads)
        assert opt.step_count == 1 and torch.equal(params[0], keep)
    for name in ("m", "v", "m_scale", "v_scale"):
        with pytest.raises(AttributeError):
            setattr(opt, name, torch.zeros(1))


def test_gradients_that_do_not_fit_are_refused(layers):
    params = [torch.ones(6, 8, device="cuda"), torch.ones(40, device="cuda")]
    opt = layers.AdamW(params)
    good = [torch.ones_like(p) for p in params]
    for bad in (good[0][:, :7], good[0].view(48), good[0].double(), good[0].cpu(), torch.ones(8, 6, device="cuda").t(),
                good[0].int()):
        with pytest.raises(ValueError, match=r"grads\[0\]"):
            opt.step([bad, good[1]])
    with pytest.raises(ValueError, match="1 gradients"):
        opt.step(good[:1])
    assert opt.step_count == 0
    opt.step(good)
    assert opt.step_count == 1


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-25, 1e-18])
def test_second_moments_and_denominators_below_the_normal_range(layers, eps, bits):
    """First steps from gradients of 3e-20 to 1e-17, whose squares are subnormal or near it, and (but for eps = 0, where
    the quotient has no value) zero. Roundings of the subnormal square and product are of 2^-150 each; with bias
    correction the second moment is off by c2 (2^-150 (1 + 0.01) and 4 units), the change by what that makes of the
    quotient and 8 units more."""
    rng = np.random.default_rng(12)
    g = (10.0 ** rng.uniform(np.log10(3e-20), -17, 3000) * rng.choice([-1, 1], 3000)).astype(np.float32)
    if eps:
        g[::7] = 0.0
    p = torch.ones(3000, device="cuda")
    opt = layers.AdamW([p], lr=LR, betas=BETAS, eps=eps, state_bits=bits)
    opt.step([torch.from_numpy(g).cuda()])
    e = float(np.float32(eps))
    ge = g.astype(np.float64)
    off = 1.02 * 2.0 ** -150 / (1 - BETAS[1]) + ref.ulps(4) * ge ** 2
    lo, hi = (LR * np.abs(ge) / np.maximum(np.sqrt(np.maximum(ge ** 2 + s * off, 0)) + e, 1e-300) for s in (1, -1))
    change = LR * np.abs(ge) / np.maximum(np.sqrt(ge ** 2) + e, 1e-300)
    bound = np.maximum(change - lo, hi - change) + ref.ulps(8) * change + ref.ulps(2)
    within("p", host(p), 1.0 - np.sign(ge) * change, bound)


def test_parameters_that_require_gradients(layers):
    """The values of a step on tensors that require none, and the change is known to torch."""
    rng = np.random.default_rng(15)
    p0, g = rand(rng, 500), rand(rng, 500)
    p, w = p0.clone(), p0.clone().requires_grad_(True)
    layers.AdamW([p], lr=LR).step([g])
    held = (w * w).sum()
    layers.AdamW([w], lr=LR).step([g])
    assert torch.equal(w.detach(), p)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        held.backward()
