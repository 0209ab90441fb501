"""The linear-attention language model end to end: its gradients against differences, a
training run that learns a batch, and single tokens against the whole sequence."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

CFG = dict(n_layers=2, vocab=50, embed=64, hidden=128, wdtype=0, probe=0)


@pytest.fixture(scope="module")
def rec():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_17852_amd import recurrent
    return recurrent


def batch(B=4, T=70, V=50, seed=3):
    rng = np.random.default_rng(seed)
    tokens = torch.from_numpy(rng.integers(0, V, (B, T + 1)).astype(np.int32)).cuda()
    mask = torch.from_numpy((rng.random((B, T)) < 0.7).astype(np.uint8)).cuda()
    return tokens, mask


def test_gradients_against_differences(rec):
    """Each tensor's gradient along itself, by central differences of the fp32 loss with steps h of 1%
    of the tensor's size and h / 2, extrapolated so that their third-order terms cancel;
    what is left and rounding within 3%."""
    model = rec.LinearLM(CFG, seed=1, kv_heads=1)
    tokens, mask = batch()
    _, grads = model.loss_and_gradients(tokens, mask)
    for (name, p), g in zip(model.p.items(), grads):
        n = float(g.norm())
        assert n > 0, name
        h = 0.01 * max(float(p.norm()), 1.0) / n
        keep = p.clone()

        def difference(h):
            ends = []
            for sign in (1, -1):
                p.copy_(keep + sign * h * g)
                ends.append(float(model.loss_and_gradients(tokens, mask)[0].double()))
            p.copy_(keep)
            return (ends[0] - ends[1]) / (2 * h)

        whole, half = difference(h), difference(h / 2)
        want, got = (4 * half - whole) / 3, n * n
        print(f"{name}: {got} differences {whole} {half} extrapolated {want}", flush=True)
        assert abs(got - want) <= 3e-2 * abs(got) + 3e-5 / h, name


@pytest.mark.parametrize("wdtype,bits", [(0, 32), (0, 8), (1, 32)])
def test_training_learns_a_batch(rec, wdtype, bits):
    model = rec.LinearLM(dict(CFG, wdtype=wdtype), seed=2, lr=5e-3, state_bits=bits)
    tokens, mask = batch()
    losses = [float(model.train_step(tokens, mask)) for _ in range(60)]
    print(losses[::10], losses[-1], flush=True)
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0]


def test_single_tokens_continue_a_prompt(rec):
    """Prompts of their own lengths, then tokens one by one: the logits are the whole sequences' (fp32,
    sums in another order through two layers)."""
    model = rec.LinearLM(CFG, seed=4, kv_heads=1)
    tokens, _ = batch(B=3, T=90)
    lengths = [40, 1, 64]
    whole, _ = model.forward(tokens)
    padded = tokens[:, :64].clone()
    logits, states = model.forward(padded, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    for b, n in enumerate(lengths):
        assert torch.allclose(logits[b, :n], whole[b, :n], atol=1e-4, rtol=1e-4)
    for t in range(20):
        now = torch.stack([tokens[b, n + t] for b, n in enumerate(lengths)])
        got = model.step(now, states)
        want = torch.stack([whole[b, n + t] for b, n in enumerate(lengths)])
        assert torch.allclose(got, want, atol=1e-4, rtol=1e-4), t


def test_a_bad_gradient_skips_the_step(rec):
    model = rec.LinearLM(CFG, seed=5)
    tokens, mask = batch()
    model.train_step(tokens, mask)
    keep = [x.clone() for x in (model.theta, model.opt.m, model.opt.v)]
    model.p["head_b"][0] = float("nan")
    keep[0][-CFG["vocab"]] = float("nan")
    model.train_step(tokens, mask)
    for a, b in zip(keep, (model.theta, model.opt.m, model.opt.v)):
        assert torch.equal(torch.nan_to_num(a, 7.0), torch.nan_to_num(b, 7.0))


def test_prompts_without_a_last_token_are_refused(rec):
    """A length of 0 has no token to continue from, one past the prompts' columns no logits."""
    model = rec.LinearLM(CFG, seed=6)
    tokens, _ = batch(B=3, T=20)
    good = torch.tensor([20, 1, 7], dtype=torch.int32, device="cuda")
    assert rec.answer(model, tokens[:, :20], good, 3).shape == (3, 3)
    for bad in ([0, 5, 20], [5, -1, 3], [5, 21, 3]):
        with pytest.raises(ValueError, match="lengths"):
            rec.answer(model, tokens[:, :20], torch.tensor(bad, dtype=torch.int32, device="cuda"), 3)
    with pytest.raises(ValueError, match="prompts"):
        rec.answer(model, tokens[:, :0], None, 3)


def test_training_asks_for_no_final_states(rec, monkeypatch):
    """Nothing reads them there; a prompt's are wanted."""
    asked = []
    whole = rec.layers.linear_attention
    monkeypatch.setattr(rec.layers, "linear_attention", lambda *a, **kw: asked.append(kw["return_state"]) or whole(*a, **kw))
    model = rec.LinearLM(CFG, seed=7)
    tokens, mask = batch()
    model.loss_and_gradients(tokens, mask)
    assert asked == [False] * CFG["n_layers"]
    _, states = model.forward(tokens)
    assert asked[CFG["n_layers"]:] == [True] * CFG["n_layers"] and all(s.dim() == 4 for s in states)


def test_the_head_by_parts_is_the_head(rec, monkeypatch):
    """Logits of 37 positions at a time against all 280 at once (fp32): the same sums in another order. A loss or gradient
    is a sum of at most 280 such terms, each through fp32 sums of at most 280 + 128 + 50 values: 1,000 units."""
    model = rec.LinearLM(CFG, seed=8)
    tokens, mask = batch()
    want, wgrads = model.loss_and_gradients(tokens, mask)
    monkeypatch.setattr(rec, "HEAD_VALUES", 37 * CFG["vocab"] + 3)
    got, grads = model.loss_and_gradients(tokens, mask)
    unit = 1000 * 2.0 ** -24
    assert abs(float(got) - float(want)) <= unit * abs(float(want))
    for name, a, b in zip(model.p, grads, wgrads):
        assert a.dtype == torch.float32 and a.shape == b.shape
        assert float((a - b).norm()) <= 8 * unit * float(b.norm()), name


def test_the_head_s_memory_is_bounded(rec):
    """16,384 positions of 50,000 logits: 3.3 GB each time they are held in fp32. A part holds at most HEAD_VALUES of them,
    six times over at its peak; the rest of the model and its gradients is under 0.5 GB."""
    model = rec.LinearLM(dict(n_layers=1, vocab=50_000, embed=64, hidden=64, wdtype=0), seed=9)
    tokens, _ = batch(B=16, T=1024, V=50_000)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    loss, _ = model.loss_and_gradients(tokens, None)
    assert np.isfinite(float(loss))
    peak = torch.cuda.max_memory_allocated() - before
    print(f"{peak / 2 ** 30:.2f} GiB", flush=True)
    assert peak <= 6 * 4 * (1 << 27) + (1 << 29)
