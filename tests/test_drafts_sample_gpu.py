"""Verification by sampling: the definition in numpy (weights as whole numbers, sums exact) on the CPU.

Tokens, lengths and drafts have to be equal.  A weight is 2^42 exp(.) rounded to a whole number; here exp is float64's, the kernel's is off by up to 2^-28 of
itself.  At a border R between tokens, u S against R then moves by at most 2 u (1 - u) 2^-28 S, and a random number lies between the two places with
a probability of no more than that; over V borders, and u anywhere, V 2^-28 / 3.  That is for errors of one sign.  They change sign from logit to logit, and these
rows have their weight on N > 2^10 of V logits, so the sums' errors are sqrt(N) times smaller: V 2^-34 or so, 2^-14 for the longest rows here
(2^20), of which there are four random numbers, and 2^-17 for the few hundred of some 10^5.  Inputs are fixed, so equality that holds stays.
Log-probabilities, x - ln S in units of the temperature: one rounding to fp32, 2^-24 of the value, and ln S is off by at most 2^-28 of itself (the largest logit's
weight is exact: S = 1 + R, off by 2^-28 R, and ln(1 + R) >= R / (1 + R)), so by at most 2^-28 of the value, which is not smaller.  The tolerance
leaves 2^-40 for that in place of 2^-28 of the value, again since errors of both signs meet in a sum; tests/test_drafts_sample_edges_gpu.py has the full
bound, and the weights' own.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ONE = 2.0 ** 42


# ---- the definition ------------------------------------------------------------------------------------------------
def ref_row(x, u, temperature=1.0, top_k=0, top_p=1.0):
    """x: float64 logits of a row -> (token, log-probability)."""
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    if not (x > -np.inf).any():
        return -1, 0.0
    top = x.max()
    if not temperature > 0:
        return int(np.argmax(x)), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        below = np.where(x == top, 0.0, (x - top) / np.float64(min(temperature, 1e36)))
        below = np.where(x == -np.inf, -np.inf, below)
    w = np.rint(ONE * np.exp(below)).astype(np.int64)
    order = np.lexsort((np.arange(len(x)), -x))                # descending, then by index
    order = order[x[order] > -np.inf]
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        run = np.cumsum(w[order])
        target = max(int(np.ceil(max(np.float64(top_p), 0.0) * np.float64(run[-1]))), 1)
        order = order[:int(np.searchsorted(run, target)) + 1]
    kept = np.zeros(len(x), dtype=np.int64)
    kept[order] = w[order]
    run = np.cumsum(kept)
    u = np.float64(min(max(np.float32(u), np.float32(0)), np.float32(1 - 2.0 ** -24))) if u == u else 0.0
    y = int(np.searchsorted(run, int(u * np.float64(run[-1])), side="right"))
    return y, below[y] - np.log(run[-1] / ONE)


def ref_sample(logits, uniform, drafts, valid, temperature, top_k, top_p):
    """numpy: logits [B][rows][V] float64 ... -> best, length, tokens, logprobs."""
    B, L = uniform.shape[0], uniform.shape[1] - 1
    n = 0 if drafts is None else drafts.shape[1]
    best, length = np.full(B, -1), np.zeros(B, dtype=int)
    tokens, logs = np.full((B, L + 1), -1), np.zeros((B, L + 1))
    for b in range(B):
        live = [r for r in range(n) if valid[b, r] != 0]
        for t in range(L + 1):
            if live:
                best[b] = live[0]
            row = 0 if t == 0 else 1 + live[0] * L + t - 1
            tokens[b, t], logs[b, t] = ref_row(logits[b, row], uniform[b, t], temperature[b], top_k[b], top_p[b])
            length[b] = t + 1
            live = [r for r in live if t < L and tokens[b, t] >= 0 and drafts[b, r, t] == tokens[b, t]]
            if not live:
                break
    return best, length, tokens, logs


def vector(x, B, dtype):
    return np.full(B, x, dtype=dtype) if np.isscalar(x) else np.asarray(x, dtype=dtype)


def check(logits, uniform, drafts=None, valid=None, temperature=1.0, top_k=0, top_p=1.0, **kwargs):
    """logits: CUDA tensor [B][rows][V]; the others numpy or numbers."""
    B = logits.shape[0]
    t, k, p = vector(temperature, B, np.float32), vector(top_k, B, np.int32), vector(top_p, B, np.float32)
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    uniform = np.asarray(uniform, dtype=np.float32)
    got = binding.drafts_sample(logits, dev(uniform), dev(drafts), dev(valid), temperature=dev(t), top_k=dev(k), top_p=dev(p), **kwargs)
    torch.cuda.synchronize()
    best, length, tokens, logs = (x.cpu().numpy() for x in got)
    want = ref_sample(logits.double().cpu().numpy(), uniform, drafts, valid, t, k, p)
    np.testing.assert_array_equal(tokens, want[2])
    np.testing.assert_array_equal(length, want[1])
    np.testing.assert_array_equal(best, want[0])
    assert (np.abs(logs - want[3]) <= 2.0 ** -24 * np.abs(want[3]) + 2.0 ** -40).all(), np.abs(logs - want[3]).max()
    return got


def chunk(B, n, L, V, dtype, seed, agree=2.0):
    """Logits, drafts of few distinct tokens (so that prefixes agree) and which are valid; the drafts' tokens are likely."""
    g = np.random.default_rng(seed)
    logits = torch.from_numpy(g.standard_normal((B, 1 + n * L, V)).astype(np.float32) * 2)
    drafts = g.integers(0, min(V, 3), (B, n, L)).astype(np.int32)
    logits[..., :3] += agree + np.log(V)
    valid = (g.random((B, n)) < 0.8).astype(np.int32)
    return logits.to(DT[dtype]).cuda(), g.random((B, L + 1)), drafts, valid


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 33, 1000, 4099, 20011])
@pytest.mark.parametrize("top_k,top_p", [(0, 1.0), (5, 1.0), (0, 0.6), (17, 0.8)])
def test_single_tokens(dtype, V, top_k, top_p):
    g = np.random.default_rng(V + top_k)
    B = 9
    logits = torch.from_numpy(g.standard_normal((B, 1, V)).astype(np.float32) * 3).to(DT[dtype]).cuda()
    check(logits, g.random((B, 1)), temperature=[0.7, 1, 0.2, 5, 0, -1, np.nan, np.inf, 1e-40], top_k=top_k, top_p=top_p)


@pytest.mark.gpu
@pytest.mark.parametrize("B,n,L,V,dtype", [(1, 10, 10, 3001, "f16"), (5, 3, 20, 517, "bf16"), (3, 32, 2, 64, "f32"), (40, 1, 1, 130, "f16"),
                                           (2, 4, 3, 33001, "bf16"), (200, 2, 4, 999, "f16")])
@pytest.mark.parametrize("temperature,top_k,top_p", [(1.0, 0, 1.0), (0.7, 0, 0.95), (1.3, 50, 1.0), (0.0, 0, 1.0)])
def test_chains_of_drafts(B, n, L, V, dtype, temperature, top_k, top_p):
    logits, uniform, drafts, valid = chunk(B, n, L, V, dtype, B + n + L)
    got = check(logits, uniform, drafts, valid, temperature, top_k, top_p)
    if temperature == 1.0 and B > 4:                       # (of three sequences each may well end at once)
        assert got[1].max() > 1 and got[1].min() < L + 1, "every sequence ended at the same depth"


@pytest.mark.gpu
@pytest.mark.parametrize("V,B", [(151001, 3), (262144, 1), (1 << 20, 1), (100003, 40), (50000, 90)])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_large_vocabularies(V, B, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = (torch.randn((B, 1, V), device="cuda", generator=g) * 2).to(DT[dtype])
    u = np.random.default_rng(V).random((B, 1))
    check(logits, u)
    check(logits, u, temperature=0.8, top_k=1000, top_p=0.9)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("order", ["mixed", "falling", "rising", "few values", "one value", "few left"])
def test_the_largest_few_of_long_rows(dtype, order):
    """Short lists of what is left, and rows whose largest logits all lie in one place, or are too many of a kind, for them."""
    g = torch.Generator(device="cuda").manual_seed(2)
    B, V = 40, 70003
    x = torch.randn((B, 1, V), device="cuda", generator=g) * 2
    if order in ("falling", "rising"):
        x = x.sort(-1, descending=order == "falling").values
    elif order == "few values":
        x = (x * 2).round()
    elif order == "one value":
        x = torch.ones_like(x)
    elif order == "few left":
        x[:, :, 37:] = -float("inf")
    u = np.random.default_rng(7).random((B, 1))
    k = np.array([1, 2, 7, 40, 100, 127, 128, 129, 300, 5000] * 4)
    check(x.to(DT[dtype]), u, temperature=0.9, top_k=k)
    check(x.to(DT[dtype]), u, temperature=0.9, top_k=k, top_p=0.7)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("top", [0.0, 2.0, np.inf])
@pytest.mark.parametrize("equal", [1, 59, 60, 61, 511, 512, 513, 1500])
def test_equal_logits_around_top_k(dtype, top, equal):
    """More or fewer of the largest than top_k takes, and than are looked at together; zeros of both signs, NaN among them."""
    g = np.random.default_rng(equal)
    B, V, k = 6, 9001, np.array([60, 60, 128, 1, 100, 60])
    x = -1 - np.abs(g.standard_normal((B, 1, V)))
    for b in range(B):
        at = g.permutation(V)
        x[b, 0, at[:equal]] = top
        x[b, 0, at[:equal:2]] = top if top else -0.0
        x[b, 0, at[equal:equal + 50]] = np.nan
        x[b, 0, at[equal + 50:equal + 90]] = -np.inf
    logits = torch.from_numpy(x).float().to(DT[dtype]).cuda()
    for u in (g.random((B, 1)), np.zeros((B, 1)), np.full((B, 1), 1 - 2.0 ** -24)):
        check(logits, u, temperature=0.8, top_k=k)
        check(logits, u, temperature=[0.8, 2.0, 1e-3, 1.0, 50.0, np.inf], top_k=k, top_p=[0.5, 0.99, 0.9, 0.1, 0.7, 1e-9])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_any_address_and_distance(dtype):
    """Rows that begin at every element of a 16-byte block, with strangers between them that would win."""
    g = np.random.default_rng(8)
    V = 1003
    for shift in range(9):
        wide = torch.full((2, 3, V + 13), 60.0, dtype=DT[dtype], device="cuda")
        logits = wide[:, :, shift:shift + V]
        logits.copy_(torch.from_numpy(g.standard_normal((2, 3, V))).to(DT[dtype]))
        drafts = g.integers(0, V, (2, 2, 1)).astype(np.int32)
        drafts[:, 0, 0] = [ref_row(logits[b, 0].double().cpu().numpy(), 0.5)[0] for b in range(2)]
        check(logits, np.full((2, 2), 0.5), drafts, np.ones((2, 2), np.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_masks_infinities_nan_and_equal_logits(dtype):
    inf, nan, V = float("inf"), float("nan"), 2500
    low = torch.finfo(DT[dtype]).min
    x = torch.zeros((12, 1, V))
    x[0] = -inf                                            # nothing
    x[1] = nan
    x[2] = -inf
    x[2, 0, 1700] = -3.0                                   # one
    x[3] = low                                             # all the lowest finite value
    x[4] = low
    x[4, 0, 77] = 0.0
    x[5, 0, 5:9] = inf                                     # infinities share everything
    x[6, 0, ::2] = nan
    x[6, 0, 1::2] = -inf
    x[6, 0, 2001] = 1.0
    x[7, 0, ::3] = -0.0                                    # zeros of both signs are equal
    x[8, 0, 1000:] = 1.0                                   # large classes of equal logits
    x[9, 0, :] = torch.arange(V) % 5
    x[10, 0, -1] = 10.0
    x[11, 0, 0] = -inf
    logits = x.to(DT[dtype]).cuda()
    g = np.random.default_rng(3)
    for top_k, top_p in ((0, 1.0), (1, 1.0), (3, 1.0), (1200, 1.0), (V, 1.0), (V + 9, 0.9), (-4, 0.5), (0, 0.0), (0, -1.0), (0, np.nan), (0, 1e-9), (1300, 0.3)):
        for temperature in (1.0, 0.0):
            check(logits, g.random((12, 1)), temperature=temperature, top_k=top_k, top_p=top_p)


@pytest.mark.gpu
def test_random_numbers_at_their_ends():
    g = np.random.default_rng(5)
    u = np.array([0.0, 1.0, 1 - 2.0 ** -24, 2.0, -1.0, np.nan, np.inf, 2.0 ** -149])[:, None]
    logits = torch.from_numpy(g.standard_normal((8, 1, 777))).half().cuda()
    check(logits, u)
    check(logits, u, top_k=3)
    logits[:, :, -4:] = -float("inf")                      # the last token with weight is not the last one
    got = check(logits, u, top_p=0.99)
    assert got[2].max() < 773


@pytest.mark.gpu
def test_equal_weights_are_shared_out_exactly():
    """1024 equal logits: u = k / 1024 is the first random number of token k, and top_p = 0.5 keeps the first 512."""
    u = (np.arange(1024) / 1024)[:, None]
    logits = torch.zeros((1024, 1, 1024), dtype=torch.float16, device="cuda")
    got = check(logits, u)
    assert got[2][:, 0].tolist() == list(range(1024))
    got = check(logits, u, top_p=0.5)
    assert got[2][:, 0].tolist() == [k // 2 for k in range(1024)]


@pytest.mark.gpu
def test_a_row_without_tokens_ends_its_sequence():
    logits, uniform, drafts, valid = chunk(2, 2, 3, 50, "f32", 1, agree=30.0)
    drafts[:], valid[:] = 1, 1
    logits[:] = -20.0
    logits[:, :, 1] = 20.0                                 # the drafts' token, certainly
    logits[0, 2] = -float("inf")                           # behind the second token of the first sequence's draft
    best, length, tokens, logs = check(logits, uniform, drafts, valid)
    assert tokens.tolist() == [[1, 1, -1, -1], [1, 1, 1, 1]] and length.tolist() == [3, 4] and best.tolist() == [0, 0]


@pytest.mark.gpu
def test_greedy_agrees_with_the_greedy_call():
    """Rows of equal prefixes are equal here, so the longest accepted draft is the same."""
    g = np.random.default_rng(2)
    B, n, L, V = 6, 4, 5, 40
    drafts = g.integers(0, 2, (B, n, L)).astype(np.int32)
    valid = np.ones((B, n), np.int32)
    valid[1] = 0
    table = torch.from_numpy(g.standard_normal((B, 2 ** (L + 1), V)) + 4 * (np.arange(V) < 2)).half().cuda()
    logits = torch.empty((B, 1 + n * L, V), dtype=torch.float16, device="cuda")
    for b in range(B):
        logits[b, 0] = table[b, 1]
        for r in range(n):
            node = 1
            for t in range(L):
                node = 2 * node + int(drafts[b, r, t])
                logits[b, 1 + r * L + t] = table[b, node]
    best, length, tokens, _ = check(logits, np.zeros((B, L + 1)), drafts, valid, temperature=0.0)
    own = logits.argmax(-1).int()
    llm = torch.cat((own[:, :1, None].expand(B, n, 1), own[:, 1:].view(B, n, L)), 2).contiguous()
    b2, l2, t2 = torch.empty_like(best), torch.empty_like(length), torch.empty_like(tokens)
    d, v = torch.from_numpy(drafts).cuda(), torch.from_numpy(valid).cuda()
    binding.dresd_drafts_accept(d.data_ptr(), v.data_ptr(), llm.data_ptr(), B, n, L, b2.data_ptr(), l2.data_ptr(), t2.data_ptr(),
                                torch.cuda.current_stream().cuda_stream)
    assert torch.equal(best, b2) and torch.equal(length, l2) and torch.equal(tokens, t2)
    assert int(length.max()) > 2


@pytest.mark.gpu
def test_a_token_does_not_depend_on_its_batch():
    """The same rows alone (many CTAs a sequence), and in a batch of 300 (one)."""
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = (torch.randn((300, 1, 9000), device="cuda", generator=g) * 2).bfloat16()
    u = torch.rand((300, 1), device="cuda", generator=g)
    p = torch.full((300,), 0.9, device="cuda")
    _, _, tokens, logs = binding.drafts_sample(logits, u, top_p=p)
    for b in (0, 7, 299):
        _, _, t, l = binding.drafts_sample(logits[b:b + 1], u[b:b + 1], top_p=p[b:b + 1])
        assert torch.equal(t, tokens[b:b + 1]) and torch.equal(l, logs[b:b + 1])


@pytest.mark.gpu
def test_other_stream_and_captured_calls():
    logits, uniform, drafts, valid = chunk(4, 3, 4, 5000, "f16", 11)
    u, d, v = (torch.from_numpy(a).cuda() for a in (uniform.astype(np.float32), drafts, valid))
    want = binding.drafts_sample(logits, u, d, v)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = binding.drafts_sample(logits, u, d, v, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = binding.drafts_sample(logits, u, d, v)
        two = binding.drafts_sample(logits, u, d, v)
    logits2, uniform2, _, _ = chunk(4, 3, 4, 5000, "f16", 12)
    logits.copy_(logits2)
    u.copy_(torch.from_numpy(uniform2.astype(np.float32)))
    graph.replay()
    graph.replay()
    want = binding.drafts_sample(logits, u, d, v)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, one, two))


@pytest.mark.gpu
def test_optional_arguments_and_empty_batches():
    logits = torch.randn((3, 1, 100), device="cuda")
    u = torch.rand((3, 1), device="cuda")
    full = binding.drafts_sample(logits, u, temperature=torch.ones(3, device="cuda"), top_k=torch.zeros(3, dtype=torch.int32, device="cuda"),
                                 top_p=torch.ones(3, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(full, binding.drafts_sample(logits, u)))
    none = torch.zeros((3, 0, 4), dtype=torch.int32, device="cuda")
    assert torch.equal(binding.drafts_sample(logits, u, none, none[:, :, 0])[2], full[2])
    empty = binding.drafts_sample(logits[:0], u[:0])
    assert [tuple(x.shape) for x in empty] == [(0,), (0,), (0, 1), (0, 1)]


@pytest.mark.gpu
def test_refusals():
    logits, u = torch.zeros((2, 3, 10), device="cuda"), torch.zeros((2, 2), device="cuda")
    d, v = torch.zeros((2, 2, 1), dtype=torch.int32, device="cuda"), torch.ones((2, 2), dtype=torch.int32, device="cuda")
    binding.drafts_sample(logits, u, d, v)
    half = torch.zeros(2, dtype=torch.float16, device="cuda")
    for args, kwargs in [((logits.cpu(), u, d, v), {}), ((logits.double(), u, d, v), {}), ((logits[0], u, d, v), {}), ((logits, u, d, None), {}),
                         ((logits[:, :2], u, d, v), {}), ((logits, u[:, :1], d, v), {}), ((logits, u.double(), d, v), {}), ((logits, u, d.long(), v), {}),
                         ((logits, u, d, v[:, :1]), {}), ((logits, u, d, v), dict(temperature=half)), ((logits, u, d, v), dict(top_k=half)),
                         ((logits, u, d, v), dict(top_p=u)), ((logits.transpose(1, 2), u, d, v), {}), ((logits, u.cpu(), d, v), {}),
                         ((logits[:1].expand(2, 3, 10), u, d, v), {}), ((logits, None, d, v), {})]:
        with pytest.raises(binding.DresdError) as e:
            binding.drafts_sample(*args, **kwargs)
        assert e.value.status == -1


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), -1), (dict(B=-1), -1), (dict(V=0), -1), (dict(n=-1), -1), (dict(n=2, L=0), -1), (dict(n=0, L=2), -1), (dict(n=33), -2),
    (dict(L=65537), -2), (dict(V=(1 << 20) + 1, row_stride=1 << 21, chunk_stride=1 << 30), -2), (dict(B=65536), -2), (dict(row_stride=9), -1),
    (dict(chunk_stride=9), -1), (dict(chunk_stride=1 << 40), -1)])
def test_refusals_need_no_device(change, status):
    from paper_2502_15572_b200 import build
    build.build()
    a = dict(dtype=1, chunk_stride=100, row_stride=10, V=10, B=2, n=2, L=3)
    a.update(change)
    with pytest.raises(binding.DresdError) as e:
        binding.dresd_drafts_sample(0x1000, a["dtype"], a["chunk_stride"], a["row_stride"], a["V"], 0x1000, 0x1000, 0x1000, None, None, None,
                                    a["B"], a["n"], a["L"], 0x1000, 0x1000, 0x1000, None)
    assert e.value.status == status
