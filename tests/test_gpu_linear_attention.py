"""Linear attention with a decay for each head on the GPU (forward, backward and
the step for single tokens) against the recurrence in 64 bits, at the lengths,
head sizes, layouts and masks where it can go wrong."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layers_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_17852_amd import layers as m
    m.lib()
    return m


def rand(rng, shape, dtype="f32", scale=1.0):
    """(device tensor, its values on the host)."""
    t = torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).to(DT[dtype])
    return t.cuda(), t.float().numpy()


def host(t):
    return None if t is None else t.detach().float().cpu().numpy()


def close(name, got, want, bound):
    off = np.abs(host(got).astype(np.float64) - want)
    worst = float((off / bound).max()) if off.size else 0.0
    print(f"{name}: worst error {worst:.3f} of its bound", flush=True)
    assert np.isfinite(host(got)).all() and worst <= 1.0, name


def make(rng, dtype, B, T, Hq, Hkv, Dk, Dv, state=False, lengths=None, decay=None):
    s = dict(dtype=dtype, scale=ref.default_scale(Dk), log_decay=ref.log_decays(Hkv) if decay is None else decay)
    for name, shape in (("q", (B, T, Hq, Dk)), ("k", (B, T, Hkv, Dk)), ("v", (B, T, Hkv, Dv)),
                        ("do", (B, T, Hq, Dv))):
        s[name + "_d"], s[name] = rand(rng, shape, dtype)
    for name in ("initial", "dfinal"):
        s[name + "_d"], s[name] = rand(rng, (B, Hkv, Dk, Dv)) if state else (None, None)
    s["lengths"] = lengths
    s["lengths_d"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["decay_d"] = torch.from_numpy(np.asarray(s["log_decay"], dtype=np.float32)).cuda()
    return s


def check_forward(layers, s, **kw):
    B, T, Hq, Dk = s["q"].shape
    Dv = s["v"].shape[3]
    o, final = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], scale=s["scale"],
                                       initial_state=s["initial_d"], lengths=s["lengths_d"], return_state=True, **kw)
    want, wfinal, mag, fmag = ref.attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"], s["lengths"])
    n = ref.attention_terms(T, Dk, Dv)
    close("o", o, want, ref.attention_bound(want, mag, s["dtype"], n))
    close("final", final, wfinal, ref.state_bound(fmag, s["dtype"], n))
    return o, final


def check_backward(layers, s):
    B, T, Hq, Dk = s["q"].shape
    Hkv, Dv = s["v"].shape[2:]
    got = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"], scale=s["scale"],
                                           initial_state=s["initial_d"], lengths=s["lengths_d"],
                                           dfinal_state=s["dfinal_d"], return_dinitial=True)
    want, mag = ref.attention_backward(s["do"], s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"],
                                       s["lengths"], s["dfinal"])
    n = ref.attention_terms(T * Hq // Hkv, Dk, Dv)
    for name, g in zip(("dq", "dk", "dv"), got):
        close(name, g, want[name], ref.attention_bound(want[name], mag[name], s["dtype"], n))
    close("dinitial", got[3], want["dinitial"], ref.state_bound(mag["dinitial"], s["dtype"], n))
    return got


# B, T, Hq, Hkv, Dk, Dv, state, lengths
SHAPES = {
    "one_token": (2, 1, 2, 2, 64, 64, True, None),
    "one_value": (1, 5, 1, 1, 1, 1, True, None),
    "two_tokens": (1, 2, 4, 1, 32, 32, False, None),
    "odd_heads": (2, 37, 3, 3, 40, 24, True, None),
    "prime": (1, 67, 2, 1, 53, 61, True, None),
    "unequal": (2, 64, 2, 2, 128, 32, True, None),
    "unequal_other": (1, 65, 2, 2, 32, 128, False, None),
    "chunks": (1, 192, 2, 2, 64, 64, False, None),
    "shared": (2, 130, 6, 2, 64, 64, True, None),
    "wide": (1, 129, 2, 2, 128, 128, True, None),
    "widest": (1, 70, 2, 1, 256, 256, True, None),
    "wide_odd": (1, 70, 1, 1, 200, 129, True, None),
    "ragged": (6, 150, 4, 2, 64, 64, True, [0, 1, 150, 64, 65, 127]),
    "ragged_no_state": (3, 100, 2, 2, 32, 48, False, [99, 0, 33]),
    "empty_all": (2, 20, 2, 1, 32, 32, True, [0, 0]),
    "lengths_outside": (3, 40, 1, 1, 64, 64, True, [-5, 1000, 40]),
    "long": (1, 1500, 2, 1, 64, 64, True, None),
    "long_ragged": (2, 1111, 1, 1, 128, 128, True, [1111, 600]),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_forward_and_backward(layers, name, dtype):
    B, T, Hq, Hkv, Dk, Dv, state, lengths = SHAPES[name]
    s = make(np.random.default_rng(len(name) + 17), dtype, B, T, Hq, Hkv, Dk, Dv, state, lengths)
    check_forward(layers, s)
    check_backward(layers, s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv,T,state,ragged", [(64, 64, 70, True, True), (40, 24, 65, False, False),
                                                  (128, 128, 130, True, True), (96, 128, 64, False, False),
                                                  (64, 104, 33, True, False), (33, 64, 40, True, False), (8, 8, 1, True, False)])
def test_many_states(layers, dtype, Dk, Dv, T, state, ragged):
    """Enough states to fill the chip, heads that share none: the gradients of k and v from one walk."""
    B, H = 16, 17
    lengths = [0, 1, T] + [T - 3 * b for b in range(B - 3)] if ragged else None
    s = make(np.random.default_rng(Dk + T), dtype, B, T, H, H, Dk, Dv, state, lengths)
    check_forward(layers, s)
    check_backward(layers, s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_a_bad_value_among_many_states(layers, dtype, D):
    """Values that are not finite in q, k, v or do of some heads: gradients of the others, and those of
    positions that they do not reach, keep their bits."""
    B, T, H = 16, 130, 17
    s = make(np.random.default_rng(D), dtype, B, T, H, H, D, D, False)
    args = dict(scale=s["scale"])
    base = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    at = 70
    # what a bad value at a position reaches: dq from it on (k, v) or there alone (do), dk and dv up to it (q, do)
    # or there alone (k, v); and q no dq, k no dk, v no dv at all
    before, after, there, none = slice(0, at), slice(at + 1, T), slice(at, at + 1), slice(0, 0)
    kept = {"q": (none, after, after), "do": (None, after, after), "k": (before, none, None), "v": (before, None, none)}
    for name in ("q", "do", "k", "v"):
        for bad in (float("nan"), float("inf")):
            x = {n: s[n + "_d"].clone() for n in ("do", "q", "k", "v")}
            x[name][3, at, 5, 7] = bad
            got = layers.linear_attention_backward(x["do"], x["q"], x["k"], x["v"], s["decay_d"], **args)
            for g, w, part in zip(got, base, kept[name]):
                others = torch.ones(B, H, dtype=torch.bool, device="cuda")
                others[3, 5] = False
                assert torch.equal(g.transpose(1, 2)[others], w.transpose(1, 2)[others]), name
                if part is None:  # that position alone
                    assert torch.equal(g[3, before, 5], w[3, before, 5]) and torch.equal(g[3, after, 5], w[3, after, 5]), name
                    assert not torch.isfinite(g[3, there, 5]).all()
                elif part is not none:
                    assert torch.equal(g[3, part, 5], w[3, part, 5]), name
                    assert not torch.isfinite(g[3, there, 5]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_at_their_ends(layers, dtype):
    """No decay, total decay (log 0), and one that underflows within a chunk."""
    decay = np.array([0.0, -np.inf, -3.0, -40.0], dtype=np.float32)
    s = make(np.random.default_rng(3), dtype, 2, 150, 4, 4, 32, 32, True, [150, 77], decay)
    check_forward(layers, s)
    check_backward(layers, s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slices_strides_and_orders(layers, dtype):
    """q, k and v as slices of one projection, batch and position swapped in memory, odd addresses."""
    B, T, Hq, Hkv, D = 3, 70, 4, 2, 40
    rng = np.random.default_rng(5)
    flat, _ = rand(rng, T * B * (Hq + 2 * Hkv) * D + 1, dtype)
    qkv = flat[1:].view(T, B, (Hq + 2 * Hkv), D).transpose(0, 1)
    s = make(rng, dtype, B, T, Hq, Hkv, D, D, True)
    for name, at, n in (("q", 0, Hq), ("k", Hq, Hkv), ("v", Hq + Hkv, Hkv)):
        s[name + "_d"] = qkv[:, :, at:at + n]
        s[name] = host(s[name + "_d"])
    o, _ = check_forward(layers, s)
    check_backward(layers, s)
    # the output into a view: heads reversed in memory by their order, gaps between positions
    room = torch.full((B, T, 2, Hq, D), 7.0, dtype=DT[dtype], device="cuda")
    o2, _ = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], scale=s["scale"],
                                    initial_state=s["initial_d"], out=room[:, :, 0])
    assert torch.equal(o2, o) and bool((room[:, :, 1] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_past_the_lengths_are_never_used(layers, dtype):
    """NaN and infinities past the lengths change nothing; outputs and gradients there are zero."""
    lengths = [0, 1, 63, 64, 100]
    s = make(np.random.default_rng(8), dtype, 5, 130, 2, 1, 64, 64, True, lengths)
    a = [*check_forward(layers, s), *check_backward(layers, s)]
    for name in ("q", "k", "v", "do"):
        for b, n in enumerate(lengths):
            s[name + "_d"][b, n:] = float("nan") if b % 2 else float("inf")
    o, final = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], scale=s["scale"],
                                       initial_state=s["initial_d"], lengths=s["lengths_d"], return_state=True)
    grads = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"], scale=s["scale"],
                                             initial_state=s["initial_d"], lengths=s["lengths_d"],
                                             dfinal_state=s["dfinal_d"], return_dinitial=True)
    for x, y in zip(a, (o, final, *grads)):
        assert torch.equal(x, y)
    for b, n in enumerate(lengths):
        assert not o[b, n:].any() and not any(g[b, n:].any() for g in grads[:3])
    assert torch.equal(final[0], s["initial_d"][0]) and torch.equal(grads[3][0], s["dfinal_d"][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 9, 63, 64, 100])
def test_a_bad_value_leaves_earlier_positions_alone(layers, dtype, bad, at):
    """A value that is not finite, in v, k or q, reaches outputs from its position on only,
    and in the backward pass (in do) gradients of k and v up to its position only."""
    s = make(np.random.default_rng(13), dtype, 1, 130, 1, 1, 64, 64, False)
    args = dict(scale=s["scale"])
    base, _ = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    for name in ("v", "k", "q"):
        x = {n: s[n + "_d"].clone() for n in "qkv"}
        x[name][0, at, 0, 5] = bad
        o, _ = layers.linear_attention(x["q"], x["k"], x["v"], s["decay_d"], **args)
        assert torch.equal(o[:, :at], base[:, :at]), name
        assert not torch.isfinite(o[0, at]).all(), name
        if name == "q":
            assert torch.equal(o[:, at + 1:], base[:, at + 1:])
        if name == "v":
            other = torch.ones(64, dtype=torch.bool, device="cuda")
            other[5] = False
            assert torch.equal(o[..., other], base[..., other]) and not torch.isfinite(o[0, at:, 0, 5]).any()
    grads = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    x = s["do_d"].clone()
    x[0, at, 0, 5] = bad
    got = layers.linear_attention_backward(x, s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    for g, w in zip(got[1:3], grads[1:3]):
        assert torch.equal(g[:, at + 1:], w[:, at + 1:])
    for t in (slice(0, at), slice(at + 1, None)):
        assert torch.equal(got[0][:, t], grads[0][:, t])


def test_gradients_against_differences(layers):
    """Directional differences of a loss of the output and the final state (fp32): f is
    quadratic in q, k and v together, so central differences are exact but for rounding,
    which the step size keeps at 1e-3 of the change."""
    s = make(np.random.default_rng(21), "f32", 2, 90, 4, 2, 32, 32, True, [90, 51])
    rng = np.random.default_rng(22)
    grads = dict(zip(("q", "k", "v", "initial"), layers.linear_attention_backward(
        s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"], scale=s["scale"], initial_state=s["initial_d"],
        lengths=s["lengths_d"], dfinal_state=s["dfinal_d"])))

    def loss(name, x):
        a = {n: s[n + "_d"] for n in ("q", "k", "v", "initial")}
        a[name] = x
        o, final = layers.linear_attention(a["q"], a["k"], a["v"], s["decay_d"], scale=s["scale"],
                                           initial_state=a["initial"], lengths=s["lengths_d"], return_state=True)
        return float((o.double() * s["do_d"].double()).sum() + (final.double() * s["dfinal_d"].double()).sum())

    for name in grads:
        d = grads[name] + 0.3 * grads[name].norm() / np.sqrt(grads[name].numel()) * rand(rng, s[name].shape)[0]
        want = ref.finite_difference(lambda x: loss(name, x), s[name + "_d"], d, 0.5 / float(d.abs().max()))
        got = float((grads[name].double() * d.double()).sum())
        print(f"d{name}: {got} difference {want}", flush=True)
        assert abs(got - want) <= 2e-3 * abs(want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_prompt_in_parts_is_the_prompt(layers, dtype):
    """The state handed from part to part, then to single tokens, in place."""
    B, T, Hq, Hkv, D = 2, 140, 4, 2, 64
    s = make(np.random.default_rng(31), dtype, B, T, Hq, Hkv, D, D, True)
    want, wfinal, mag, fmag = ref.attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"])
    state, parts = s["initial_d"].clone(), []
    for a, b in ((0, 1), (1, 70), (70, 70), (70, 134)):
        o, final = layers.linear_attention(s["q_d"][:, a:b], s["k_d"][:, a:b], s["v_d"][:, a:b], s["decay_d"],
                                           scale=s["scale"], initial_state=state, final_state=state)
        assert final is state
        parts.append(o)
    for t in range(134, T):
        parts.append(layers.linear_attention_step(s["q_d"][:, t], s["k_d"][:, t], s["v_d"][:, t], s["decay_d"], state,
                                                  scale=s["scale"]).unsqueeze(1))
    n = ref.attention_terms(T, D, D)
    close("o", torch.cat(parts, 1), want, ref.attention_bound(want, mag, dtype, n))
    close("state", state, wfinal, ref.state_bound(fmag, dtype, n))


@pytest.mark.parametrize("shape", [(1, 2500, 8, 2, 64), (3, 500, 8, 1, 128), (1, 1400, 1, 1, 200)])
def test_states_advanced_in_place(layers, shape):
    """The final state into the initial one's buffer, with query heads and segments that read it too."""
    B, T, Hq, Hkv, D = shape
    s = make(np.random.default_rng(T), "bf16", B, T, Hq, Hkv, D, D, True)
    want = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], initial_state=s["initial_d"],
                                   return_state=True)
    state = s["initial_d"].clone()
    o, final = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], initial_state=state,
                                       final_state=state)
    assert final is state and torch.equal(o, want[0]) and torch.equal(state, want[1])


STEPS = {
    "one": (1, 1, 1, 1, 1),
    "small": (3, 2, 2, 32, 32),
    "odd": (5, 6, 3, 53, 61),
    "unaligned": (2, 3, 1, 129, 66),
    "shared": (4, 18, 2, 64, 64),
    "wide": (2, 2, 2, 256, 256),
    "plain": (7, 4, 4, 128, 128),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(STEPS))
def test_step(layers, name, dtype):
    B, Hq, Hkv, Dk, Dv = STEPS[name]
    s = make(np.random.default_rng(len(name)), dtype, B, 1, Hq, Hkv, Dk, Dv, True)
    want, wfinal, mag, fmag = ref.attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"])
    state = s["initial_d"].clone()
    o = layers.linear_attention_step(s["q_d"][:, 0], s["k_d"][:, 0], s["v_d"][:, 0], s["decay_d"], state,
                                     scale=s["scale"])
    n = ref.attention_terms(1, Dk, Dv)
    # everything in fp32, the output rounded once
    close("o", o, want[:, 0], ref.unit(dtype) * np.abs(want[:, 0]) + n * 2.0 ** -24 * mag[:, 0] + 1e-37)
    close("state", state, wfinal, ref.state_bound(fmag, "f32", n))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_with_slots(layers, dtype):
    """States anywhere in a pool, sequences without one, and slots that do not exist."""
    B, Hq, Hkv, Dk, Dv, n = 6, 4, 2, 64, 40, 9
    rng = np.random.default_rng(77)
    s = make(rng, dtype, B, 1, Hq, Hkv, Dk, Dv)
    pool, pool_h = rand(rng, (n, Hkv, Dk, Dv))
    slots = [8, -1, 0, 9, 3, -2]
    o = layers.linear_attention_step(s["q_d"][:, 0], s["k_d"][:, 0], s["v_d"][:, 0], s["decay_d"], pool,
                                     scale=s["scale"], slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    live = [b for b, x in enumerate(slots) if 0 <= x < n]
    at = [slots[b] for b in live]
    want, wfinal, mag, fmag = ref.attention(s["q"][live], s["k"][live], s["v"][live], s["log_decay"], s["scale"],
                                            pool_h[at])
    t = ref.attention_terms(1, Dk, Dv)
    close("o", o[live], want[:, 0], ref.unit(dtype) * np.abs(want[:, 0]) + t * 2.0 ** -24 * mag[:, 0] + 1e-37)
    close("state", pool[at], wfinal, ref.state_bound(fmag, "f32", t))
    rest = [i for i in range(n) if i not in at]
    assert np.array_equal(host(pool)[rest], pool_h[rest])
    assert not o[1].any() and torch.isnan(o[3]).all() and torch.isnan(o[5]).all()


def test_the_same_bits_every_time(layers):
    s = make(np.random.default_rng(41), "bf16", 2, 500, 4, 2, 64, 64, True, [500, 321])
    runs = []
    for _ in range(2):
        runs.append([*layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], initial_state=s["initial_d"],
                                              lengths=s["lengths_d"], return_state=True),
                     *layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"],
                                                       initial_state=s["initial_d"], lengths=s["lengths_d"],
                                                       dfinal_state=s["dfinal_d"])])
    assert all(torch.equal(x, y) for x, y in zip(*runs))


def test_another_stream_and_a_graph(layers):
    """On a stream of the caller's, and captured: every replay gives the eager result."""
    s = make(np.random.default_rng(51), "bf16", 2, 700, 4, 2, 64, 64, True)
    args = (s["q_d"], s["k_d"], s["v_d"], s["decay_d"])

    def call(**kw):
        return [*layers.linear_attention(*args, initial_state=s["initial_d"], return_state=True, **kw),
                *layers.linear_attention_backward(s["do_d"], *args, initial_state=s["initial_d"],
                                                  dfinal_state=s["dfinal_d"], **kw)]

    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        for t in held:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))


def test_nothing_to_do(layers):
    """No sequences, or no positions: the states pass through."""
    z = torch.zeros(0, 4, 2, 32, device="cuda")
    decay = torch.zeros(2, device="cuda")
    o, final = layers.linear_attention(z, z, z, decay, return_state=True)
    assert o.shape == (0, 4, 2, 32) and final.shape == (0, 2, 32, 32)
    z = torch.zeros(3, 0, 2, 32, device="cuda")
    initial = torch.randn(3, 2, 32, 32, device="cuda")
    o, final = layers.linear_attention(z, z, z, decay, initial_state=initial, return_state=True)
    assert torch.equal(final, initial)
    got = layers.linear_attention_backward(z, z, z, z, decay, dfinal_state=initial, return_dinitial=True)
    assert torch.equal(got[3], initial)
    e = torch.zeros(0, 2, 32, device="cuda")
    assert layers.linear_attention_step(e, e, e, decay, initial).shape == (0, 2, 32)


def test_a_final_state_that_overlaps_the_initial_one_in_part(layers):
    """States of one buffer, moved up by one sequence: the values before the call are the ones that count."""
    B, T, Hq, Hkv, D = 3, 300, 4, 2, 64
    s = make(np.random.default_rng(77), "f32", B, T, Hq, Hkv, D, D, True)
    want = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], initial_state=s["initial_d"],
                                   return_state=True)
    pool = torch.zeros(B + 1, Hkv, D, D, device="cuda")
    pool[:B] = s["initial_d"]
    o, final = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], initial_state=pool[:B],
                                       final_state=pool[1:])
    assert torch.equal(o, want[0]) and torch.equal(pool[1:], want[1]) and torch.equal(pool[0], s["initial_d"][0])


@pytest.mark.parametrize("name", ["odd_heads", "unequal", "shared", "wide", "widest", "wide_odd", "ragged", "long",
                                  "long_ragged"])
def test_bf16_results_as_near_as_fp32_operands_leave_them(layers, name):
    """Scores and states meet the bf16 inputs as two bf16 parts each: what is left out of an operand is at most
    unit(bf16) of its first part's own rounding, unit(bf16)^2 = 2^-16; the rest is fp32 sums and the output's rounding."""
    B, T, Hq, Hkv, Dk, Dv, state, lengths = SHAPES[name]
    s = make(np.random.default_rng(len(name) + 90), "bf16", B, T, Hq, Hkv, Dk, Dv, state, lengths)
    _near_fp32(layers, s)


@pytest.mark.parametrize("D,T", [(64, 130), (96, 70), (128, 200), (104, 65)])
def test_bf16_results_of_many_states_as_near(layers, D, T):
    """The same where there are states enough for the wider slices."""
    _near_fp32(layers, make(np.random.default_rng(D), "bf16", 16, T, 17, 17, D, D, True))


def _near_fp32(layers, s):
    B, T, Hq, Dk = s["q"].shape
    Hkv, Dv = s["v"].shape[2:]
    args = dict(scale=s["scale"], initial_state=s["initial_d"], lengths=s["lengths_d"])
    o, _ = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    want, _, mag, _ = ref.attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"], s["lengths"])
    n = ref.attention_terms(T, Dk, Dv)
    u = ref.unit("bf16")

    def bound(value, magnitude, terms):
        return u * np.abs(value) + (u * u + terms * 2.0 ** -24) * magnitude + 1e-37

    close("o", o, want, bound(want, mag, n))
    got = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"],
                                           dfinal_state=s["dfinal_d"], **args)
    want, mag = ref.attention_backward(s["do"], s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"],
                                       s["lengths"], s["dfinal"])
    n = ref.attention_terms(T * Hq // Hkv, Dk, Dv)
    for name, g in zip(("dq", "dk", "dv"), got):
        close(name, g, want[name], bound(want[name], mag[name], n))


def test_a_call_on_another_stream_takes_no_block_that_queued_work_still_uses(layers):
    """Tensors of the outputs' size are freed while the current stream's work on them is pending; a call on another stream
    gets other memory, and the right values."""
    s = make(np.random.default_rng(61), "bf16", 2, 1024, 16, 16, 64, 64)
    args = (s["q_d"], s["k_d"], s["v_d"], s["decay_d"])
    want, _ = layers.linear_attention(*args)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = [torch.zeros_like(want) for _ in range(3)]
    freed = {b.data_ptr() for b in busy}
    for b in busy:
        for _ in range(200):
            b.add_(1.0)
    del busy, b
    o, _ = layers.linear_attention(*args, stream=side)
    side.synchronize()
    assert o.data_ptr() not in freed and torch.equal(o, want)
    torch.cuda.synchronize()
    assert torch.equal(o, want)


@pytest.mark.parametrize("at_once", [0, 1, 4])
def test_thousands_of_single_tokens_do_not_drift(layers, at_once):
    """States that only decay, 2,000 tokens: each step rounds a value within 2^-24 of it. Where gamma's significand is full,
    to either side as often, so that the mean over 16,384 values of a head is known to 6 sqrt(2000) 2^-24 / sqrt(3) / 128 =
    7.3e-8 (bound 1.5e-7). Where gamma is 1 - 2^-b, one product in 2^b is a tie, which may always fall the same way, by
    half a unit: 2000 2^-b 2^-24 more. A decay of half a unit in the last place off, at every token, would be 6e-5."""
    rng = np.random.default_rng(71)
    B, H, D, n = 4, 8, 64, 2000
    state, start = rand(rng, (B, H, D, D))
    ld = ref.log_decays(H, 6.0, 11.0)
    zero = torch.zeros(B, H, D, device="cuda")
    decay = torch.from_numpy(ld).cuda()
    if at_once:  # as sequences of that many positions
        zero, other = zero.unsqueeze(1).expand(B, at_once, H, D).contiguous(), torch.empty_like(state)
        for _ in range(n // at_once):
            layers.linear_attention(zero, zero, zero, decay, initial_state=state, final_state=other)
            state, other = other, state
    else:
        for _ in range(n):
            layers.linear_attention_step(zero, zero, zero, decay, state)
    want = start.astype(np.float64) * np.exp(n * ld.astype(np.float64))[None, :, None, None]
    off = (host(state) / want - 1.0).mean(axis=(0, 2, 3))
    print(off, flush=True)
    bits = np.linspace(6.0, 11.0, H)
    ties = np.where(bits == np.round(bits), n * 2.0 ** -bits * 2.0 ** -24, 0.0)
    assert (np.abs(off) <= 1.5e-7 + ties).all()


@pytest.mark.parametrize("at_once", [0, 1])
@pytest.mark.parametrize("log_decay", [0.0, -float("inf"), -0.25, -0.75, -30.0, 0.25])
def test_a_token_on_states_that_are_not_finite(layers, log_decay, at_once):
    """Infinities stay what they are under a decay, NaN stays NaN, and the values beside them are as alone."""
    rng = np.random.default_rng(72)
    state, _ = rand(rng, (1, 1, 8, 8))
    q, k, v = (rand(rng, (1, 1, 8))[0] for _ in range(3))
    decay = torch.tensor([log_decay], device="cuda")

    def token(state):
        if at_once:
            layers.linear_attention(q.unsqueeze(1), k.unsqueeze(1), v.unsqueeze(1), decay, initial_state=state,
                                    final_state=state)
        else:
            layers.linear_attention_step(q, k, v, decay, state)

    alone = state.clone()
    token(alone)
    state[0, 0, 2, 3], state[0, 0, 4, 5], state[0, 0, 6, 7] = float("inf"), -float("inf"), float("nan")
    token(state)
    bad = torch.zeros(8, 8, dtype=torch.bool, device="cuda")
    bad[2, 3] = bad[4, 5] = bad[6, 7] = True
    assert torch.equal(state[0, 0][~bad], alone[0, 0][~bad]) and torch.isnan(state[0, 0, 6, 7])
    if log_decay > -float("inf"):
        assert state[0, 0, 2, 3] == float("inf") and state[0, 0, 4, 5] == -float("inf")
    else:
        assert torch.isnan(state[0, 0, 2, 3]) and torch.isnan(state[0, 0, 4, 5])


def test_one_position_at_any_distance(layers):
    """The distance between positions is free where there is one, or none: in the binding, and in a step's tensors."""
    B, H, D = 3, 2, 32
    s = make(np.random.default_rng(81), "f32", B, 1, H, H, D, D, True)
    want = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], initial_state=s["initial_d"],
                                   return_state=True)
    far = [s[n + "_d"].as_strided((B, 1, H, D), (H * D, 1 << 40, D, 1)) for n in ("q", "k", "v", "do")]
    out = torch.empty(B, 1, H, D, device="cuda").as_strided((B, 1, H, D), (H * D, 1 << 30, D, 1))
    o, final = layers.linear_attention(*far[:3], s["decay_d"], initial_state=s["initial_d"], return_state=True, out=out)
    assert torch.equal(o, want[0]) and torch.equal(final, want[1])
    grads = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"])
    got = layers.linear_attention_backward(far[3], *far[:3], s["decay_d"])
    assert all(torch.equal(a, b) for a, b in zip(got[:3], grads[:3]))
    none = [x[:, :0] for x in far[:3]]
    assert layers.linear_attention(*none, s["decay_d"])[0].shape == (B, 0, H, D)
    state, o1 = s["initial_d"].clone(), torch.empty(B, H, D, device="cuda")
    heads = [layers._HEADS.pack(t.data_ptr(), H * D, 1 << 40, D) for t in (s["q_d"], s["k_d"], s["v_d"], o1)]
    shape = layers._SHAPE.pack(B, 0, H, H, D, D, 0, s["scale"])
    layers._check(layers.lib().zo_linear_attention_step(shape, *heads, s["decay_d"].data_ptr(), state.data_ptr(), B,
                                                        None, layers._stream(o1)))
    n = ref.attention_terms(1, D, D)
    wo, wfinal, mag, fmag = ref.attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["initial"])
    close("o", o1, wo[:, 0], ref.unit("f32") * np.abs(wo[:, 0]) + n * 2.0 ** -24 * mag[:, 0] + 1e-37)
    close("state", state, wfinal, ref.state_bound(fmag, "f32", n))


@pytest.mark.parametrize("order", ["heads", "time", "apart"])
def test_outputs_between_the_inputs_values(layers, order):
    """Outputs in the gaps of the inputs' buffer, in any order of its dimensions, are taken; on its values they are refused."""
    from paper_2505_17852_amd import zo
    B, T, H, D = 2, 70, 3, 40
    s = make(np.random.default_rng(91), "f32", B, T, H, H, D, D)
    want = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"])[0]
    grads = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"])
    if order == "heads":
        room = torch.zeros(B, T, 7 * H, D, device="cuda").view(B, T, 7, H, D).permute(2, 0, 1, 3, 4)
    elif order == "time":
        room = torch.zeros(T, B, H, 7, D, device="cuda").permute(3, 1, 0, 2, 4)
    else:
        room = torch.zeros(7, B, T, H, D, device="cuda")
    for i, name in enumerate(("q", "k", "v")):
        room[i].copy_(s[name + "_d"])
    q, k, v, o = room[:4]
    layers.linear_attention(q, k, v, s["decay_d"], out=o)
    layers.linear_attention_backward(s["do_d"], q, k, v, s["decay_d"], dq=room[4], dk=room[5], dv=room[6])
    assert torch.equal(o, want) and all(torch.equal(a, b) for a, b in zip(room[4:], grads))
    assert all(torch.equal(a, s[n + "_d"]) for a, n in zip((q, k, v), "qkv"))
    for out in (q, v, torch.zeros(D, device="cuda").expand(B, T, H, D)):
        with pytest.raises(zo.ZoError, match="share memory|one place"):
            layers.linear_attention(q, k, v, s["decay_d"], out=out)
    with pytest.raises(zo.ZoError, match="dv and dk share memory"):
        layers.linear_attention_backward(s["do_d"], q, k, v, s["decay_d"], dk=o, dv=o)


# B, T, Hq, Hkv, Dk, Dv, lengths: up to four positions (times the query heads of a state: up to 4, up to 16, and past it)
FEW = {
    "two": (3, 2, 2, 2, 53, 61, None),
    "three": (4, 3, 3, 3, 128, 96, [0, 1, 3, 2]),
    "four": (5, 4, 2, 2, 64, 64, [4, 0, 1, 3, 2]),
    "four_wide": (2, 4, 1, 1, 256, 200, [3, 4]),
    "one_shared": (3, 1, 8, 2, 96, 128, [1, 0, 1]),
    "two_shared": (3, 2, 8, 1, 33, 130, [2, 1, 0]),
    "three_shared": (2, 3, 8, 2, 200, 40, None),
    "four_shared": (4, 4, 8, 2, 64, 120, [0, 1, 3, 4]),
    "four_shared_past": (4, 4, 10, 2, 64, 120, [0, 1, 3, 4]),
    "two_shared_past": (2, 2, 9, 1, 40, 256, [2, 1]),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("name", list(FEW))
def test_few_positions(layers, name, state, dtype):
    """With and without states, lengths inside, heads that share, odd sizes."""
    B, T, Hq, Hkv, Dk, Dv, lengths = FEW[name]
    s = make(np.random.default_rng(len(name) + 5 * state), dtype, B, T, Hq, Hkv, Dk, Dv, state, lengths)
    o, final = check_forward(layers, s)
    grads = check_backward(layers, s)
    _near_fp32(layers, s) if dtype == "bf16" else None
    for b, n in enumerate(lengths or []):
        assert not o[b, n:].any() and not any(g[b, n:].any() for g in grads[:3])
        if n == 0 and state:
            assert torch.equal(final[b], s["initial_d"][b]) and torch.equal(grads[3][b], s["dfinal_d"][b])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3, 4])
def test_decays_at_their_ends_over_few_positions(layers, T, dtype):
    decay = np.array([0.0, -np.inf, -3.0, -40.0], dtype=np.float32)
    s = make(np.random.default_rng(T), dtype, 2, T, 8, 4, 40, 24, True, [T, T - 1], decay)
    check_forward(layers, s)
    check_backward(layers, s)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [0, 1, 3])
def test_a_bad_value_among_few_positions(layers, at, bad):
    """As over many: outputs from its position on only, gradients of k and v up to it only; past a length it is not read."""
    s = make(np.random.default_rng(17), "bf16", 2, 4, 2, 2, 64, 64, False, [4, at])
    args = dict(scale=s["scale"], lengths=s["lengths_d"])
    base, _ = layers.linear_attention(s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    grads = layers.linear_attention_backward(s["do_d"], s["q_d"], s["k_d"], s["v_d"], s["decay_d"], **args)
    for name in ("q", "k", "v", "do"):
        x = {n: s[n + "_d"].clone() for n in ("q", "k", "v", "do")}
        x[name][:, at, 0, 5] = bad
        o, _ = layers.linear_attention(x["q"], x["k"], x["v"], s["decay_d"], **args)
        got = layers.linear_attention_backward(x["do"], x["q"], x["k"], x["v"], s["decay_d"], **args)
        for a, w in zip((o, *got[:3]), (base, *grads[:3])):
            assert torch.equal(a[1], w[1]) and torch.equal(a[0, :, 1], w[0, :, 1]), name
        if name != "do":
            assert torch.equal(o[0, :at], base[0, :at]) and not torch.isfinite(o[0, at, 0]).all(), name
        if name in ("q", "do"):
            assert all(torch.equal(a[0, at + 1:], w[0, at + 1:]) for a, w in zip(got[1:3], grads[1:3])), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_segments(layers, dtype):
    """One sequence of 5,000 positions in 19 segments, and one that ends within them."""
    s = make(np.random.default_rng(27), dtype, 1, 5000, 1, 1, 64, 64, True)
    check_forward(layers, s)
    check_backward(layers, s)
    s["lengths"], s["lengths_d"] = [3333], torch.tensor([3333], dtype=torch.int32, device="cuda")
    check_forward(layers, s)
    check_backward(layers, s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(64, 64), (50, 64), (100, 128), (190, 200)])
def test_states_are_as_exact_as_their_factors(layers, T, D, dtype):
    """Keys and queries of one 1 each, at a row of its own: every value of a final state (or an initial one's gradient) is one
    value times a power of gamma. Within its chunk that is two powers (each: an exponent under 1 rounded to 2^-23, the power
    to 2^-23), two products, and the value in parts, 2^-24 left out: 5 of 2^-23; 3 more for each chunk after it."""
    H = 3
    s = make(np.random.default_rng(T + D), dtype, 2, T, H, H, D, D, False, None, ref.log_decays(H, 8.0, 11.0))
    hot = torch.zeros(T, D, device="cuda", dtype=s["q_d"].dtype)
    hot[torch.arange(T), torch.arange(T)] = 1.0
    hot = hot.view(1, T, 1, D).expand(2, T, H, D).contiguous()
    unit = (5 + 3 * ((T - 1) // 64)) * 2.0 ** -23
    ld = s["log_decay"].astype(np.float64)[None, :, None, None]
    _, final = layers.linear_attention(hot, hot, s["v_d"], s["decay_d"], scale=1.0, return_state=True)
    left = T - 1 - np.arange(T)
    want = s["v"].astype(np.float64).transpose(0, 2, 1, 3) * np.exp(ld * left[None, None, :, None])
    close("final", final[:, :, :T], want, unit * np.abs(want) + 1e-37)
    assert not final[:, :, T:].any()
    got = layers.linear_attention_backward(s["do_d"], hot, hot, s["v_d"], s["decay_d"], scale=1.0, return_dinitial=True)[3]
    want = s["do"].astype(np.float64).transpose(0, 2, 1, 3) * np.exp(ld * (np.arange(T) + 1)[None, None, :, None])
    close("dinitial", got[:, :, :T], want, unit * np.abs(want) + 1e-37)
    assert not got[:, :, T:].any()


def test_a_graph_captured_with_its_stream_named(layers):
    """The capturing stream passed to each call: every replay, with eager work between, gives the eager result."""
    s = make(np.random.default_rng(101), "bf16", 2, 300, 4, 2, 64, 64, True)
    args = (s["q_d"], s["k_d"], s["v_d"], s["decay_d"])

    def call(stream=None):
        o, final = layers.linear_attention(*args, initial_state=s["initial_d"], return_state=True, stream=stream)
        y, mean, rstd = layers.layer_norm(o, stream=stream)
        return [o, final, y, *layers.linear_attention_backward(y, *args, initial_state=s["initial_d"], stream=stream)]

    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call(torch.cuda.current_stream())
    for _ in range(3):
        for t in held:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
        assert all(torch.equal(x, y) for x, y in zip(call(), want))
