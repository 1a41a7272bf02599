"""The cache, its attention and the draft calls as one decoding loop: every token it writes is the model's own.

The model is computed once more in float64, without a cache and without drafts, over the finished texts; the token
that the loop wrote has to be the largest logit there, up to what 16-bit arithmetic moves logits by.  Bound: a
logit passes about 10 roundings per layer (products, sums of the residual stream, norms, keys and values, weights of the
attention) of half a unit in the last place u each, relative to numbers of its own size, two layers, independent:
sqrt(20) u rms of the logits' spread s; the largest of ~1000 logits against ~4 standard deviations of the difference of two:
16 sqrt(20) u s.  8-bit rows are quantised in the float64 computation too; their codes may flip where a rounding lies on an edge, so
they get the bound of bf16.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def logits64(model, text, quantised, dtype):
    import torch
    from tests.test_kv_cache_gpu import ref_quantise, ref_values
    w = lambda t: t.double().cpu().numpy()
    rows, H, Hkv, d = len(text), model.heads, model.kv_heads, model.head_dim
    norm = lambda x: x / np.sqrt(np.square(x).mean(-1, keepdims=True) + 1e-6)
    angle = np.arange(rows)[:, None] * (10000.0 ** (-np.arange(0, d, 2) / d))

    def turn(x):
        lo, hi = x[..., :d // 2], x[..., d // 2:]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        return np.concatenate((lo * c - hi * s, hi * c + lo * s), -1)

    def held(x):
        return ref_values(*ref_quantise(x, dtype)) if quantised else x

    x = w(model.embed)[text]
    for layer in range(model.layers):
        q, k, v = np.split(norm(x) @ w(model.w_qkv[layer]), (H * d, (H + Hkv) * d), -1)
        q, k, v = turn(q.reshape(rows, H, d)), held(turn(k.reshape(rows, Hkv, d))), held(v.reshape(rows, Hkv, d))
        s = np.einsum("ihgd,jhd->hgij", q.reshape(rows, Hkv, H // Hkv, d), k) / np.sqrt(d)
        s = np.where(np.tri(rows, dtype=bool), s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        mixed = np.einsum("hgij,jhd->ihgd", p / p.sum(-1, keepdims=True), v).reshape(rows, H * d)
        x = x + mixed @ w(model.w_out[layer])
        x = x + np.maximum(norm(x) @ w(model.w_up[layer]), 0) @ w(model.w_down[layer])
    return norm(x) @ w(model.w_vocab)


@pytest.mark.parametrize("dtype,quantised,n,L,page,head_dim,kv_heads", [
    ("f16", False, 4, 5, 16, 64, 2),       # 21 tokens x 4 heads a key/value head: the many-row kernel
    ("bf16", False, 3, 2, 32, 128, 4),     # 7 x 2: the few-row kernel
    ("f16", True, 2, 9, 64, 128, 2),
    ("bf16", True, 1, 3, 128, 64, 8),
])
def test_decoding_with_drafts_writes_the_models_own_tokens(dtype, quantised, n, L, page, head_dim, kv_heads):
    import torch
    from paper_2502_15572_b200 import speculate
    model = speculate.Decoder(dtype=dtype, seed=5, head_dim=head_dim, kv_heads=kv_heads)
    gen = torch.Generator().manual_seed(6)
    prompts = [torch.randint(model.vocab, (m,), generator=gen).tolist() for m in (1, 17, 40)]
    count = 24
    plain, steps = speculate.Speculator(model, prompts, count + 1, page_size=page, quantised=quantised).run(count)
    store = speculate.make_datastore(model, [p + t for p, t in zip(prompts, plain)], L + 1)
    spec = speculate.Speculator(model, prompts, count + L + 1, store, n, L, page_size=page, quantised=quantised)
    drafted, fewer = spec.run(count)
    store.status()
    assert steps == count - 1 and fewer < steps, "no draft was ever accepted"
    unit = 2.0 ** -11 if dtype == "f16" and not quantised else 2.0 ** -8
    for texts in (plain, drafted):
        for prompt, text in zip(prompts, texts):
            logits = logits64(model, np.array(prompt + text[:-1]), quantised, dtype)[len(prompt) - 1:]
            gap = logits.max(-1) - logits[np.arange(count), text]
            assert gap.max() <= 16 * np.sqrt(20) * unit * logits.std(), (gap.max(), logits.std())


def test_command():
    from paper_2502_15572_b200 import speculate
    speculate.main(["--quantised", "--sequences", "2", "--tokens", "20", "--drafts", "2", "--draft-len", "3"])
