"""The decoding loop with drawn tokens, several samples of a prompt and 4-bit weights: reservation, copies, verification by sampling, release and
compaction, and the products together.

As in tests/test_speculate_gpu.py the model is computed once more in float64 over the finished texts, without cache and drafts.  A logit is off by
sqrt(20) u s rms there (u: unit roundoff, s: spread of the logits), the largest of ~1000 by four times that, e = 4 sqrt(20) u s; a weight exp(x / T) then changes by
a factor within exp(+-e / T), and a share of their sum by at most exp(2 e / T) - 1.  So the random number of a token has to lie within that of the
token's share of the distribution.  A drawn token that has nothing to do with its random number is off by a third on the average.
"""
import types

import numpy as np
import pytest

from tests.test_speculate_gpu import logits64

pytestmark = pytest.mark.gpu


def in_16_bits(model):
    """The model with the values of its weights, whatever they are held in (for logits64)."""
    from paper_2502_15572_b200 import binding
    from tests.test_w4_gpu import weights64
    value = lambda w: weights64(w.codes, w.scales, w.group).T if isinstance(w, binding.W4) else w
    m = types.SimpleNamespace(heads=model.heads, kv_heads=model.kv_heads, head_dim=model.head_dim, layers=model.layers, embed=model.embed, w_vocab=value(model.w_vocab))
    for name in ("w_qkv", "w_out", "w_up", "w_down"):
        setattr(m, name, [value(w) for w in getattr(model, name)])
    return m


def check_drawn(model, dtype, quantised, prompt, text, random, temperature):
    unit = 2.0 ** -11 if dtype == "f16" and not quantised else 2.0 ** -8
    x = logits64(model, np.array(prompt + text[:-1]), quantised, dtype)[len(prompt) - 1:]
    p = np.exp((x - x.max(-1, keepdims=True)) / temperature)
    run = (p / p.sum(-1, keepdims=True)).cumsum(-1)
    at = np.arange(len(text))
    lo, hi = np.where(np.array(text) > 0, run[at, np.array(text) - 1], 0), run[at, text]
    off = np.maximum(np.maximum(lo - random, random - hi), 0)
    assert off.max() <= np.expm1(2 * 4 * np.sqrt(20) * unit * x.std() / temperature), off.max()


@pytest.mark.parametrize("dtype,quantised,group,n,L,page,samples", [
    ("f16", False, 0, 4, 5, 16, 1),
    ("f16", False, 32, 3, 4, 32, 3),
    ("bf16", False, 128, 2, 3, 64, 2),
    ("f16", True, 64, 2, 6, 16, 4),
])
def test_drawn_texts(dtype, quantised, group, n, L, page, samples):
    import torch
    from paper_2502_15572_b200 import speculate
    model = speculate.Decoder(dtype=dtype, seed=7, group=group)
    gen = torch.Generator().manual_seed(8)
    prompts = [torch.randint(model.vocab, (m,), generator=gen).tolist() for m in (1, 16, 37)]
    count, T = 24, 0.8
    how = dict(page_size=page, quantised=quantised, samples=samples, temperature=T, seed=9)
    one = speculate.Speculator(model, prompts, count + L + 1, **how)
    plain, steps = one.run(count)
    store = speculate.make_datastore(model, [prompts[i // samples] + t for i, t in enumerate(plain)], L + 1)
    spec = speculate.Speculator(model, prompts, count + L + 1, store, n, L, **how)
    # right after the prompts are read: full pages are shared by the samples, nothing is copied yet
    assert sorted(spec.refs[spec.refs > 0].tolist()) == sorted(samples for p in prompts for _ in range(-(-len(p) // page)))
    width = min(one.random.shape[1], spec.random.shape[1])
    assert torch.equal(one.random[:, :width], spec.random[:, :width]) and width >= max(map(len, prompts)) + count
    drafted, fewer = spec.run(count)
    store.status()
    assert steps == count - 1 and fewer < steps, "no draft was ever accepted"
    reference = in_16_bits(model)
    for s, texts in ((one, plain), (spec, drafted)):
        numbers = s.random.cpu().numpy()
        for i, text in enumerate(texts):
            prompt = prompts[i // samples]
            check_drawn(reference, dtype, quantised, prompt, text, numbers[i, len(prompt):len(prompt) + count], T)
    if samples > 1:
        texts = [tuple(t) for t in drafted]
        assert len(set(texts)) == len(texts), "samples of a prompt are alike"
    # every place of every sequence is held by a page of its own or shared with samples of the same prompt
    held = (spec.refs > 0).sum().item()
    chosen = torch.arange(0, spec.B, samples, device="cuda")
    before = [spec.cache.read(0, kept(spec, spec.ctx, chosen))[0].clone(), spec.cache.read(1, kept(spec, spec.ctx, chosen))[1].clone()]
    ctx = spec.ctx.clone()
    used = spec.end(chosen)
    assert used == sum(-(-int(c) // page) for c in ctx[chosen]) <= held
    assert int(spec.table.max()) == used - 1 and spec.refs[:used].tolist() == [1] * used and int(spec.refs[used:].abs().sum()) == 0
    assert torch.equal(spec.cache.read(0, kept(spec, ctx, chosen))[0], before[0]) and torch.equal(spec.cache.read(1, kept(spec, ctx, chosen))[1], before[1])
    with pytest.raises(ValueError):
        spec.step()


def kept(spec, ctx, chosen):
    """The chosen sequences' tokens as a batch to be read."""
    import torch
    from paper_2502_15572_b200 import binding
    length = torch.zeros_like(ctx)
    length[chosen] = ctx[chosen]
    start = torch.cat((torch.zeros(1, dtype=torch.int32, device="cuda"), length.cumsum(0).int()))
    kept.alive = torch.zeros_like(ctx)                        # borrowed by the batch
    return binding.KvBatch(spec.table, kept.alive, start, rows=int(start[-1]))


@pytest.mark.parametrize("dtype,group", [("f16", 64), ("bf16", 32)])
def test_largest_logits_with_4_bit_weights(dtype, group):
    """The bound of tests/test_speculate_gpu.py, of a model whose weights are the quantised ones."""
    import torch
    from paper_2502_15572_b200 import speculate
    model = speculate.Decoder(dtype=dtype, seed=5, group=group)
    prompts, count = [[3, 5, 7], [11] * 20], 20
    plain, _ = speculate.Speculator(model, prompts, count + 1).run(count)
    store = speculate.make_datastore(model, [p + t for p, t in zip(prompts, plain)], 5)
    drafted, _ = speculate.Speculator(model, prompts, count + 5, store, 2, 4).run(count)
    reference = in_16_bits(model)
    for texts in (plain, drafted):
        for prompt, text in zip(prompts, texts):
            x = logits64(reference, np.array(prompt + text[:-1]), False, dtype)[len(prompt) - 1:]
            gap = x.max(-1) - x[np.arange(count), text]
            assert gap.max() <= 16 * np.sqrt(20) * (2.0 ** -11 if dtype == "f16" else 2.0 ** -8) * x.std()


def test_a_pool_that_is_too_small_is_reported():
    import torch
    from paper_2502_15572_b200 import speculate
    model = speculate.Decoder()
    spec = speculate.Speculator(model, [[1, 2, 3]], 40, page_size=16)
    spec.refs[1:] = 1                                         # as if others held the rest
    with pytest.raises(RuntimeError):
        spec.run(40)


def test_a_sequence_far_ahead_of_the_others():
    """Its drafts are all accepted, the other's never: what it writes beyond its room disturbs nobody."""
    import torch
    from paper_2502_15572_b200 import speculate
    model = speculate.Decoder(seed=5)
    prompts, count = [[3, 5, 7], [11] * 20], 30
    plain, _ = speculate.Speculator(model, prompts, count + 1, page_size=16).run(count)
    store = speculate.make_datastore(model, [prompts[0] + speculate.Speculator(model, prompts, 121, page_size=16).run(120)[0][0]], 9)
    spec = speculate.Speculator(model, prompts, count + 1, store, 2, 8, page_size=16)
    drafted, steps = spec.run(count)
    assert steps > 20
    reference = in_16_bits(model)
    for prompt, text in zip(prompts, drafted):
        x = logits64(reference, np.array(prompt + text[:-1]), False, "f16")[len(prompt) - 1:]
        gap = x.max(-1) - x[np.arange(count), text]
        assert gap.max() <= 16 * np.sqrt(20) * 2.0 ** -11 * x.std()


def test_commands():
    from paper_2502_15572_b200 import speculate
    speculate.main(["--group", "64", "--sequences", "2", "--tokens", "20", "--drafts", "2", "--draft-len", "3", "--temperature", "0.7", "--top-p", "0.95",
                    "--samples", "3"])
    speculate.main(["--sequences", "2", "--tokens", "12", "--drafts", "2", "--draft-len", "3", "--temperature", "1.2", "--top-k", "5", "--quantised"])
