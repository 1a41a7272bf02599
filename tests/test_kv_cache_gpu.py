"""The paged key/value cache: append, read, keep_draft and the attention over it, against plain statements of the
same definitions in float64 on the CPU.

Tolerances (derived, not fitted).  Let u = 2^-11 (fp16) or 2^-8 (bf16) be the unit roundoff of the type, V the largest
finite |v| a row sees.  The exact result is o = sum p_j v_j / sum p_j.  The kernels round each weight p_j to the type once
(relative error u), accumulate in fp32, and round the result (relative error u):
    |out - o| <= u V (weights; sum p_j u |v_j| / l <= u V) + u |o| + fp32 terms,
where the fp32 terms are: the score error |ds| <= (d + 4) 2^-24 sum |q_i k_i| scale (a chain of d products) plus 2^-22 of
the exponential, which moves a weight by at most a factor 1 +- (ds + 2^-21) and hence o by 2 (ds + 2^-21) V, and the
chain of the sums themselves, at most (longest row) 2^-24 V.  That last term also covers fp16 weights below 2^-14, whose
absolute step is 2^-24 (the weight sum is at least 1).  lse is off by ds + 2^-20 + 2^-23 |lse|.
fp16 results below 2^-14 have an absolute step of 2^-24, added as is.
The cache calls are exact: bit for bit.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


# ---- plain statements (CPU, float64) ----------------------------------------------------------------------------
def e4m3_values():
    v = np.zeros(256)
    for c in range(256):
        m, e = c & 7, (c >> 3) & 15
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        v[c] = -x if c >= 128 else x
    return v


E4M3 = e4m3_values()


def ref_quantise(x, dtype):
    """x float64 [..., d] -> codes uint8 [..., d], exponent bytes uint8 [...]: by search over the 127 magnitudes."""
    bound, least = (61440.0, -24) if dtype == "f16" else (1.875 * 2.0 ** 127, -126)
    x = np.clip(x, -bound, bound)
    amax = np.abs(x).max(-1)
    e = np.where(amax > 0, least, 0)
    for k in range(least, 128):
        e = np.where((amax > 448 * 2.0 ** (k - 1)) & (amax <= 448 * 2.0 ** k), k, e)
    y = np.abs(x) / (2.0 ** e)[..., None]
    mags = E4M3[:127]                                         # ascending, code = index
    hi = np.clip(np.searchsorted(mags, y), 1, 126)
    lo = hi - 1
    up = (y - mags[lo] > mags[hi] - y) | ((y - mags[lo] == mags[hi] - y) & (hi % 2 == 0))
    code = np.where(up, hi, lo).astype(np.uint8)
    return code | np.where(np.signbit(x), 128, 0).astype(np.uint8), (e + 127).astype(np.uint8)


def ref_values(codes, exps):
    return E4M3[codes] * (2.0 ** (exps.astype(np.int64) - 127))[..., None]


def ref_attend(q, k, v, ctx, seen, scale):
    """One sequence, float64: q [n][Hq][d], k, v [ctx + n][Hkv][d], seen bool [n][ctx + n].  Values not seen are left out."""
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    out, lse, bound, dsum = np.zeros(q.shape), np.full((n, Hq), -np.inf), np.zeros((n, Hq)), np.zeros((n, Hq))
    for h in range(Hq):
        for i in range(n):
            js = np.nonzero(seen[i])[0]
            if len(js) == 0:
                continue
            kk, vv = k[js, h // G], v[js, h // G]
            s = scale * (kk @ q[i, h])
            m = s.max()
            p = np.exp(s - m)
            with np.errstate(invalid="ignore"):
                out[i, h] = (p[:, None] * vv).sum(0) / p.sum()
            lse[i, h] = m + np.log(p.sum())
            bound[i, h] = np.abs(vv[np.isfinite(vv)]).max(initial=0)
            dsum[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, lse, bound, dsum


# ---- set-up -------------------------------------------------------------------------------------------------------
class Case:
    """A cache of random contents with the tokens of every sequence in it, on the GPU and as float64 on the CPU."""

    def __init__(self, dtype, d, page, Hkv, ctx, chunk, quantised=False, layers=1, layer=0, seed=0, spare=3, amp=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.d, self.page, self.Hkv, self.layer, self.q8 = dtype, d, page, Hkv, layer, quantised
        self.ctx, self.chunk, self.B = list(ctx), list(chunk), len(ctx)
        need = [-(-(c + n) // page) for c, n in zip(ctx, chunk)]
        self.pages = sum(need) + spare
        width = max(1, max(need))
        order = rng.permutation(self.pages)
        table = np.full((self.B, width), -1, dtype=np.int32)  # places no token reaches hold no page
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = order[at:at + m]
            at += m
        self.table_np, self.start_np = table, np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
        self.rows = int(self.start_np[-1])
        shape = (layers, self.pages, Hkv, page, d)
        self.t = {}
        for name in ("k", "v"):
            x = torch.from_numpy((rng.standard_normal(shape) * amp).astype(np.float32)).to(DT[dtype])
            if quantised:
                codes, exps = ref_quantise(x.double().numpy(), dtype)
                self.t[name], self.t[name + "_exp"] = torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda()
            else:
                self.t[name], self.t[name + "_exp"] = x.cuda(), None
        self.cache = binding.KvCache(self.t["k"], self.t["v"], dtype, k_exps=self.t["k_exp"], v_exps=self.t["v_exp"])
        dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()
        self.batch = binding.KvBatch(dev(table), dev(ctx), dev(self.start_np), rows=self.rows,
                                     max_chunk=max(chunk) if chunk else 0)

    def values(self, name, layer=None):
        """float64 [pages][Hkv][page][d] of a layer."""
        layer = self.layer if layer is None else layer
        x = self.t[name][layer]
        if not self.q8:
            return x.cpu().double().numpy()
        return ref_values(x.cpu().numpy(), self.t[name + "_exp"][layer].cpu().numpy())

    def place(self, b, p):
        return self.table_np[b, p // self.page], p % self.page

    def sequence(self, name, b, upto=None, layer=None):
        """float64 [tokens][Hkv][d] of a sequence."""
        n = self.ctx[b] + self.chunk[b] if upto is None else upto
        x = self.values(name, layer)
        return np.stack([x[pg, :, off] for pg, off in (self.place(b, p) for p in range(n))]) if n else np.zeros((0, self.Hkv, self.d))

    def queries(self, Hq, seed=1, amp=1.0):
        rng = np.random.default_rng(seed)
        return torch.from_numpy((rng.standard_normal((self.rows, Hq, self.d)) * amp).astype(np.float32)).to(DT[self.dtype]).cuda()


def causal(ctx, n):
    return np.arange(ctx + n)[None] <= ctx + np.arange(n)[:, None]


def check_attend(case, q, scale=None, seen=None, mask=None, lse=True, q_view=None):
    """seen: bool [chunk][ctx + chunk] per sequence (None = causal)."""
    d, dt = case.d, case.dtype
    scale = d ** -0.5 if scale is None else scale
    out_lse = torch.full((case.rows, q.shape[1]), 7.0, device="cuda") if lse else None
    out = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda")
    got = case.cache.attend(case.layer, q if q_view is None else q_view, case.batch, scale=scale, mask=mask, out=out, lse=out_lse)
    torch.cuda.synchronize()
    case.cache.status()
    got, got_lse = got.cpu().double().numpy(), None if out_lse is None else out_lse.cpu().double().numpy()
    qn, u = q.cpu().double().numpy(), U[dt]
    for b in range(case.B):
        if case.chunk[b] == 0:
            continue
        s, e = case.start_np[b], case.start_np[b + 1]
        vis = causal(case.ctx[b], case.chunk[b]) if seen is None else seen[b]
        want, wlse, V, ds = ref_attend(qn[s:e], case.sequence("k", b), case.sequence("v", b), case.ctx[b], vis, scale)
        ds = (d + 4) * 2.0 ** -24 * ds
        n = vis.shape[1]
        tol = u * V[..., None] + u * np.abs(want) + ((2 * (ds + 2.0 ** -21) + n * 2.0 ** -24) * V)[..., None] + 2.0 ** -24
        fin = np.isfinite(want)
        assert np.array_equal(np.isfinite(got[s:e]), fin), f"sequence {b}: non-finite places differ"
        err = np.abs(got[s:e][fin] - want[fin]) - tol[fin]
        assert err.max(initial=-1) <= 0, f"sequence {b}: {err.max()} beyond the tolerance"
        if got_lse is not None:
            some = vis.any(1)
            assert np.all(np.isneginf(got_lse[s:e][~some])) and np.all(got[s:e][~some] == 0)
            off = np.abs(got_lse[s:e][some] - wlse[some]) - (ds[some] + 2.0 ** -20 + 2.0 ** -23 * np.abs(wlse[some]))
            assert off.max(initial=-1) <= 0, f"sequence {b}: lse {off.max()} beyond the tolerance"
    return got


def bits_of(seen):
    """bool [rows][places] -> int32 [rows][words] on the GPU."""
    words = (seen.shape[1] + 31) // 32
    full = np.zeros((seen.shape[0], words * 32), dtype=np.uint8)
    full[:, :seen.shape[1]] = seen
    return torch.from_numpy(np.ascontiguousarray(np.packbits(full, axis=1, bitorder="little").view("<i4"))).cuda()


# ---- attention ----------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,quantised", [(t, d, q) for t in ("f16", "bf16") for d in (64, 128) for q in (False, True)])
@pytest.mark.parametrize("page", [16, 128])
def test_single_tokens_of_ragged_sequences(dtype, d, quantised, page):
    """One token each behind contexts from nothing to several pages, odd ones among them; 7 heads per kv head."""
    ctx = [0, 1, 15, 16, 17, 63, 64, 65, 130, 511, 700]
    case = Case(dtype, d, page, 2, ctx, [1] * len(ctx), quantised, seed=d + page)
    check_attend(case, case.queries(14))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,quantised", [("f16", False), ("bf16", True)])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (16, 2), (9, 1), (16, 1), (17, 1), (64, 1), (40, 10)])
def test_head_groups(dtype, quantised, Hq, Hkv):
    case = Case(dtype, 128, 32, Hkv, [33, 200], [1, 1], quantised, seed=Hq)
    check_attend(case, case.queries(Hq))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,quantised", [("f16", 128, False), ("bf16", 64, False), ("bf16", 128, True), ("f16", 64, True)])
def test_chunks_of_every_length(dtype, d, quantised):
    """Causal chunks that start anywhere in a page and end anywhere in a tile, an empty one among them."""
    chunk = [1, 2, 0, 7, 31, 64, 65, 129, 200]
    ctx = [0, 5, 40, 127, 128, 1, 100, 63, 37]
    case = Case(dtype, d, 64, 2, ctx, chunk, quantised, seed=3)
    check_attend(case, case.queries(6))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,quantised", [("f16", False), ("bf16", True)])
@pytest.mark.parametrize("n,L", [(10, 10), (3, 20), (2, 1), (1, 5), (12, 10)])
def test_draft_chunks(dtype, quantised, n, L):
    size = 1 + n * L
    ctx = [0, 75, 301]
    case = Case(dtype, 128, 16, 2, ctx, [size] * 3, quantised, seed=n)
    tree = np.zeros((size, size), dtype=bool)
    tree[:, 0] = True
    for i in range(1, size):
        first = 1 + (i - 1) // L * L
        tree[i, first:i + 1] = True
    mask = binding.draft_mask(n, L)
    assert torch.equal(mask.cpu(), bits_of(tree).cpu())
    seen = [np.concatenate([np.ones((size, c), dtype=bool), tree], 1) for c in ctx]
    check_attend(case, case.queries(4), seen=seen, mask=mask.repeat(3, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("Hq", [2, 16])
def test_masks_that_leave_rows_empty_and_short_masks(Hq):
    """Random bits: rows that see nothing (no context, no bit), and fewer words than the chunk has tokens."""
    rng = np.random.default_rng(5)
    ctx, chunk = [0, 0, 40], [50, 1, 70]
    case = Case("f16", 64, 32, 2, ctx, chunk, seed=6)
    bits = rng.random((case.rows, 64)) < 0.3
    bits[::3] = False
    bits[50] = False                                          # the second sequence's only token sees nothing at all
    seen = []
    for b in range(3):
        s, n = case.start_np[b], chunk[b]
        own = np.zeros((n, n), dtype=bool)
        own[:, :min(n, 64)] = bits[s:s + n, :min(n, 64)]
        seen.append(np.concatenate([np.ones((n, ctx[b]), dtype=bool), own], 1))
    got = check_attend(case, case.queries(Hq), seen=seen, mask=bits_of(bits))
    assert np.all(got[50] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,quantised,chunk,Hq", [("f16", False, 1, 2), ("bf16", True, 1, 2), ("f16", True, 1, 2), ("bf16", False, 70, 4),
                                                      ("f16", True, 70, 4), ("bf16", True, 70, 4)])
def test_unused_places_may_hold_anything(dtype, quantised, chunk, Hq):
    """NaN (and its code) in every place of the pool that no token occupies."""
    ctx = [30, 77, 3]
    case = Case(dtype, 128, 32, 2, ctx, [chunk] * 3, quantised, seed=8)
    used = np.zeros((case.pages, 32), dtype=bool)
    for b in range(3):
        for p in range(ctx[b] + chunk):
            used[case.place(b, p)] = True
    free = torch.from_numpy(~used).cuda()[None, :, None, :].expand(1, -1, 2, -1)
    for name in ("k", "v"):
        case.t[name][free] = 0x7F if quantised else float("nan")
        if quantised:
            case.t[name + "_exp"][free] = 255
    got = check_attend(case, case.queries(Hq))
    assert np.isfinite(got).all()


@pytest.mark.gpu
@pytest.mark.parametrize("chunk,G", [(5, 1), (100, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_tokens_that_do_not_see_a_bad_one_are_not_touched(chunk, G, bad):
    """A chunk token whose key and value are not finite: earlier tokens and those whose mask leaves it out stay exact;
    those that see it get non-finite numbers."""
    ctx = 20
    case = Case("bf16", 64, 16, 2, [ctx], [chunk], seed=9)
    at = ctx + chunk // 2
    pg, off = case.place(0, at)
    case.t["v"][0, pg, 1, off, 5] = bad                       # one element of one head's value
    case.t["v"][0, pg, 1, off, 40] = -bad
    q = case.queries(2 * G)
    got = check_attend(case, q)                               # compares the non-finite places too
    assert np.isfinite(got[:chunk // 2]).all() and not np.isfinite(got[chunk // 2:, G:, 5]).any()
    assert np.isfinite(got[chunk // 2:, G:, 6]).all()
    case.t["k"][0, pg, 1, off, 5] = bad                       # and its key: those that see it have no finite weights
    tree = np.tri(chunk, dtype=bool)
    tree[:, chunk // 2] = False
    seen = [np.concatenate([np.ones((chunk, ctx), dtype=bool), tree], 1)]
    got = check_attend(case, q, seen=seen, mask=bits_of(tree))
    assert np.isfinite(got).all()


@pytest.mark.gpu
def test_large_scores_and_types_lowest_values():
    """Scores far beyond the exponential's range, in both directions and rising from tile to tile."""
    case = Case("bf16", 64, 16, 1, [300, 299], [1, 40], seed=10)
    k = case.t["k"]
    for b in range(2):
        for p in range(300):
            pg, off = case.place(b, p)
            k[0, pg, 0, off] *= (p if b == 0 else 300 - p) / 10
    check_attend(case, case.queries(2, amp=30.0))
    lowest = torch.finfo(torch.bfloat16).min
    for p in range(0, 290):
        pg, off = case.place(0, p)
        k[0, pg, 0, off] = 0
        k[0, pg, 0, off, 0] = lowest                          # scores near the type's lowest value: weight zero
    q = case.queries(2)
    q[:, :, 0] = q[:, :, 0].abs() + 1
    check_attend(case, q)


@pytest.mark.gpu
@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("dtype,d,page,quantised", [("f16", 64, 32, False), ("bf16", 128, 16, False), ("bf16", 64, 128, True), ("f16", 128, 64, True)])
def test_either_kernel_takes_any_batch(path, dtype, d, page, quantised):
    """Both kernels on single tokens, short and long chunks in one batch; more rows than the largest row tile."""
    ctx, chunk = [0, 130, 1000, 17, 255, 60], [1, 1, 3, 0, 300, 129]
    case = Case(dtype, d, page, 2, ctx, chunk, quantised, seed=60)
    case.cache.set_option("attend_path", path)
    check_attend(case, case.queries(6))


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
def test_scales(scale):
    case = Case("f16", 64, 16, 2, [50, 9], [40, 33], seed=61)
    check_attend(case, case.queries(4, amp=0.5), scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("stage", [1, 2, 7])
def test_a_wait_that_runs_out_is_reported(quantised, stage):
    """The first CTA never receives one of its tiles: the call ends, the status says so, the next call is right again."""
    case = Case("bf16", 128, 32, 4, [30000, 200], [40, 64], quantised, seed=62)
    q = case.queries(8)
    first = case.cache.attend(0, q, case.batch)
    case.cache.set_option("wait_ms", 20)
    case.cache.set_option("debug_lose_stage", stage)
    case.cache.attend(0, q, case.batch)
    with pytest.raises(binding.DresdError) as e:
        case.cache.status()
    assert e.value.status == -5
    case.cache.set_option("debug_lose_stage", 0)
    case.cache.set_option("wait_ms", 0)
    assert torch.equal(case.cache.attend(0, q, case.batch), first)
    case.cache.status()
    with pytest.raises(binding.DresdError):
        case.cache.set_option("no_such_option", 1)


@pytest.mark.gpu
@pytest.mark.parametrize("chunk", [1, 90])
def test_strided_queries_layers_and_streams(chunk):
    """Queries as a slice of a joint projection, a middle layer, a side stream."""
    case = Case("f16", 128, 64, 2, [100, 3], [chunk, chunk], layers=3, layer=1, seed=11)
    wide = torch.randn(case.rows, 12, 128, device="cuda").half()
    q = wide[:, 3:9]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check_attend(case, q.contiguous(), q_view=q)


@pytest.mark.gpu
@pytest.mark.parametrize("chunk,Hq", [(1, 8), (40, 8)])
def test_attention_is_repeatable_and_can_be_captured(chunk, Hq):
    case = Case("bf16", 128, 32, 4, [3000, 11, 700], [chunk] * 3, seed=12)
    q = case.queries(Hq)
    first = case.cache.attend(0, q, case.batch)
    for _ in range(5):
        assert torch.equal(case.cache.attend(0, q, case.batch), first)
    out = torch.empty_like(first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        case.cache.attend(0, q, case.batch, out=out)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    q.mul_(0.5)                                               # the replay reads the queries as they are then
    g.replay()
    assert torch.equal(out, case.cache.attend(0, q, case.batch))


@pytest.mark.gpu
def test_rows_far_into_a_large_pool():
    """Offsets beyond 2^31 bytes and elements: the last pages of a 9 GB pool against the same pages in a small one."""
    small = Case("f16", 128, 128, 8, [500], [1], seed=13, spare=0)
    n = small.pages
    big_pages = 17000                                         # x 8 x 128 x 128 elements = 2.2e9
    big = {x: torch.zeros((1, big_pages, 8, 128, 128), dtype=torch.float16, device="cuda") for x in "kv"}
    for x in "kv":
        big[x][0, big_pages - n:] = small.t[x][0]
    table = small.batch.page_table + (big_pages - n)
    cache = binding.KvCache(big["k"], big["v"], "f16")
    batch = binding.KvBatch(table, small.batch.ctx, small.batch.start, rows=1, max_chunk=1)
    q = small.queries(16)
    want = small.cache.attend(0, q, small.batch)
    assert torch.equal(cache.attend(0, q, batch), want)
    k, v = torch.randn(2, 1, 8, 128, device="cuda").half()
    cache.append(0, k, v, batch)
    pg, off = small.place(0, 500)
    assert torch.equal(big["k"][0, big_pages - n + pg, :, off], k[0]) and torch.equal(big["v"][0, big_pages - n + pg, :, off], v[0])
    rk, rv = cache.read(0, batch)
    assert torch.equal(rk, k) and torch.equal(rv, v)
    cache.close()


@pytest.mark.gpu
@pytest.mark.parametrize("chunk", [1, 64])
def test_bad_batches_touch_nothing_outside(chunk):
    """Page numbers outside the pool, a table that is too narrow, lengths that contradict each other: results are
    unspecified, the arrays beside the cache stay as they are."""
    case = Case("f16", 64, 16, 2, [40, 40], [chunk, chunk], seed=14)
    case.batch.page_table[0, 1] = 10 ** 6
    case.batch.page_table[1, 0] = -5
    k = torch.randn(case.rows, 2, 64, device="cuda").half()
    before = {x: case.t[x].clone() for x in "kv"}
    case.cache.attend(0, case.queries(4), case.batch)
    rk, _ = case.cache.read(0, case.batch)
    case.batch.ctx.fill_(100000)                              # beyond the table: nothing is written, zeros are read
    case.cache.append(0, k, k, case.batch)
    assert all(torch.equal(case.t[x], before[x]) for x in "kv")
    assert not case.cache.read(0, case.batch)[0].any()
    case.cache.attend(0, case.queries(4), case.batch)
    case.batch.ctx.fill_(-3)                                  # counts as 0
    case.batch.start[0] = -7
    case.batch.start[2] = 10 ** 6
    case.cache.attend(0, case.queries(4), case.batch)
    torch.cuda.synchronize()
    case.cache.status()


# ---- the cache ----------------------------------------------------------------------------------------------------
def special_rows(T, Hkv, d, dtype, seed):
    """Rows of very different sizes, zeros, the type's extremes, and ties of the 8-bit rounding."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, Hkv, d)) * 2.0 ** rng.integers(-12, 12, size=(T, Hkv, 1))
    x[0] = 0
    if T > 3:
        x[1] = 2.0 ** -20 * rng.integers(-8, 9, size=(Hkv, d))
        x[2, :, 0] = 448.0
        x[3] = (rng.integers(0, 64, size=(Hkv, d)) + 0.5) * 4
    if T > 5:
        x[4, :, 1] = 65504.0 if dtype == "f16" else 3e38
        x[5, :, 2] = float("inf")
        x[5, :, 3] = float("-inf")
    return torch.from_numpy(x).to(DT[dtype]).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,quantised", [(t, d, q) for t in ("f16", "bf16") for d in (64, 128) for q in (False, True)])
def test_append_and_read_back(dtype, d, quantised):
    """Bit for bit, ragged chunks, slices of a joint projection; nothing else in the cache changes."""
    ctx, chunk = [0, 5, 16, 33, 2], [20, 1, 0, 40, 9]
    for Hkv in (1, 3, 8):
        case = Case(dtype, d, 16, Hkv, ctx, chunk, quantised, layers=2, layer=1, seed=20 + Hkv)
        k = special_rows(case.rows, Hkv, d, dtype, 1)
        wide = torch.zeros((case.rows, 2 * Hkv + 1, d), dtype=DT[dtype], device="cuda")
        wide[:, 1:1 + Hkv] = special_rows(case.rows, Hkv, d, dtype, 2)
        v = wide[:, 1:1 + Hkv]
        want = {x: t.clone() for x, t in case.t.items() if t is not None}
        for name, new in (("k", k), ("v", v)):
            codes, exps = ref_quantise(new.cpu().double().numpy(), dtype) if quantised else (None, None)
            for b in range(case.B):
                for i in range(chunk[b]):
                    pg, off = case.place(b, ctx[b] + i)
                    r = case.start_np[b] + i
                    if quantised:
                        want[name][1, pg, :, off] = torch.from_numpy(codes[r]).cuda()
                        want[name + "_exp"][1, pg, :, off] = torch.from_numpy(exps[r]).cuda()
                    else:
                        want[name][1, pg, :, off] = new[r]
        case.cache.append(1, k, v, case.batch)
        for x, t in want.items():
            assert torch.equal(case.t[x].view(torch.uint8), t.view(torch.uint8)), x
        rk, rv = case.cache.read(1, case.batch)
        for name, got, new in (("k", rk, k), ("v", rv, v)):
            if quantised:
                full = np.concatenate([case.sequence(name, b)[ctx[b]:] for b in range(case.B)])
                assert np.isfinite(full).all() and np.array_equal(got.cpu().double().numpy(), full), name
            else:
                assert torch.equal(got.view(torch.int16), new.contiguous().view(torch.int16)), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,page,quantised", [("f16", 128, 16, False), ("bf16", 64, 32, True), ("bf16", 64, 128, False), ("f16", 128, 64, True)])
@pytest.mark.parametrize("n,L", [(10, 10), (3, 20), (4, 1)])
def test_keep_draft(dtype, d, page, quantised, n, L):
    rng = np.random.default_rng(30 + n)
    B, size = 9, 1 + n * L
    ctx = [int(x) for x in rng.integers(0, 50, B)]
    case = Case(dtype, d, page, 2, ctx, [size] * B, quantised, layers=3, seed=31)
    best = np.array([-1, 0, 1, n - 1, n - 1, 1, n // 2, 0, n - 1], dtype=np.int32)
    length = np.array([1, L + 1, L + 1, L + 1, 1, 2, 1 + L // 2, 1, L], dtype=np.int32)
    want = {x: t.clone() for x, t in case.t.items() if t is not None}
    for b in range(B):
        if best[b] < 0:
            continue
        for t in range(length[b] - 1):
            (pf, of), (pt, ot) = case.place(b, ctx[b] + 1 + best[b] * L + t), case.place(b, ctx[b] + 1 + t)
            for x in want:
                want[x][:, pt, :, ot] = case.t[x][:, pf, :, of]
    dev = lambda a: torch.from_numpy(a).cuda()
    case.cache.keep_draft(case.batch, dev(best), dev(length), n, L)
    torch.cuda.synchronize()
    for x, t in want.items():
        assert torch.equal(case.t[x], t), x


@pytest.mark.gpu
def test_a_verified_draft_goes_on_as_if_it_had_been_read_token_by_token():
    """append -> attend (drafts) -> accept -> keep_draft -> append -> attend, against the accepted text read in one
    causal chunk: the same attention result for the next token."""
    n, L, Hkv, Hq, d = 3, 4, 2, 4, 64
    size, ctx = 1 + n * L, 37
    case = Case("f16", d, 16, Hkv, [ctx], [size + L], seed=40)            # room for the next step
    rng = torch.Generator(device="cuda").manual_seed(1)
    new = torch.randn((size, 2 * Hkv, d), device="cuda", generator=rng).half()
    batch = binding.KvBatch(case.batch.page_table, case.batch.ctx, torch.tensor([0, size], dtype=torch.int32, device="cuda"), size, size)
    case.cache.append(0, new[:, :Hkv], new[:, Hkv:], batch)
    q = torch.randn((size, Hq, d), device="cuda", generator=rng).half()
    drafted = case.cache.attend(0, q, batch, mask=binding.draft_mask(n, L))
    best, length = torch.tensor([2], dtype=torch.int32, device="cuda"), torch.tensor([4], dtype=torch.int32, device="cuda")
    case.cache.keep_draft(batch, best, length, n, L)
    keep = [0] + [1 + 2 * L + t for t in range(3)]
    text = binding.KvBatch(case.batch.page_table, case.batch.ctx, torch.tensor([0, 4], dtype=torch.int32, device="cuda"), 4, 4)
    again = case.cache.attend(0, q[keep].contiguous(), text)
    scale = case.values("v")
    tol = 4 * U["f16"] * np.abs(scale).max()
    assert (again - drafted[keep]).abs().max().item() <= tol
    k, v = case.cache.read(0, text)
    assert torch.equal(k, new[keep, :Hkv]) and torch.equal(v, new[keep, Hkv:])


# ---- refusals ---------------------------------------------------------------------------------------------------
def test_refusals_without_a_device():
    from paper_2502_15572_b200 import build as lib_build
    lib_build.build()
    good = dict(k_pages_ptr=0x1000, v_pages_ptr=0x2000, k_exps_ptr=None, v_exps_ptr=None, layers=1, num_pages=4, kv_heads=2,
                page_size=16, head_dim=64, dtype=binding.DRESD_F16)
    for change, status in [(dict(k_pages_ptr=0), -1), (dict(v_pages_ptr=0x2008), -1), (dict(k_exps_ptr=0x3000), -1),
                           (dict(dtype=binding.DRESD_F32), -2), (dict(dtype=9), -1), (dict(layers=0), -1), (dict(num_pages=0), -1),
                           (dict(kv_heads=0), -1), (dict(head_dim=96), -2), (dict(head_dim=-1), -1), (dict(page_size=24), -2),
                           (dict(page_size=256), -2), (dict(num_pages=2 ** 31, layers=80), -2), (dict(), -1)]:
        with pytest.raises(binding.DresdError) as e:          # the last: the addresses are not device memory
            binding.dresd_kv_create(**dict(good, **change))
        assert e.value.status == status, (change, e.value)
    b = binding.dresd_kv_batch(0x1000, 0x1000, 0x1000, 1, 1, 1, 1)
    for call in (lambda: binding.dresd_kv_append(0, 0, b, 0, 64, 64, 0, 64, 64), lambda: binding.dresd_kv_read(0, 0, b, 0, 0),
                 lambda: binding.dresd_kv_attend(0, 0, b, 0, 64, 64, 1, 1.0, None, 0, 0, None),
                 lambda: binding.dresd_kv_keep_draft(0, b, 0, 0, 1, 1), lambda: binding.dresd_kv_status(0)):
        with pytest.raises(binding.DresdError) as e:
            call()
        assert e.value.status == -1 and "NULL" in e.value.message
    binding.dresd_kv_destroy(0)
    assert binding.dresd_kv_last_launches(0) == 0


@pytest.mark.gpu
def test_refusals():
    case = Case("f16", 64, 16, 2, [3], [2], seed=50)
    c, b = case.cache, case.batch
    q, k = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    bad = [
        lambda: c.append(1, k, k, b), lambda: c.append(-1, k, k, b), lambda: c.append(0, k.bfloat16(), k, b),
        lambda: c.append(0, k.cpu(), k, b), lambda: c.append(0, k[:1], k, b), lambda: c.append(0, q, k, b),
        lambda: c.append(0, torch.zeros((2, 2, 128), dtype=torch.float16, device="cuda")[:, :, ::2], k, b),
        lambda: c.append(0, torch.zeros(2 * 2 * 64 + 8, dtype=torch.float16, device="cuda")[1:257].view(2, 2, 64), k, b),
        lambda: c.append(0, torch.zeros((2, 2, 68), dtype=torch.float16, device="cuda")[:, :, :64], k, b),
        lambda: c.read(0, b, out=(k, k[:1])), lambda: c.read(2, b),
        lambda: c.attend(0, q[:, :3].contiguous(), b), lambda: c.attend(0, q, b, out=q[:, :2]), lambda: c.attend(0, q, b, scale=float("nan")),
        lambda: c.attend(0, q, b, scale=float("inf")), lambda: c.attend(0, q, b, mask=i32(1)), lambda: c.attend(0, q, b, mask=torch.zeros((2, 1), device="cuda")),
        lambda: c.attend(0, q, b, lse=torch.zeros(2, 2, device="cuda")), lambda: c.attend(0, q.expand(2, 4, 64).float(), b),
        lambda: c.keep_draft(b, i32(1), i32(1, 2), 2, 2), lambda: c.keep_draft(b, i32(1), i32(1), 0, 2), lambda: c.keep_draft(b, i32(1), i32(1), 2, 0),
        lambda: binding.KvBatch(b.page_table, b.ctx, i32(0), 2), lambda: binding.KvBatch(b.page_table.cpu(), b.ctx, b.start, 2),
        lambda: binding.KvBatch(b.page_table.long(), b.ctx, b.start, 2), lambda: c.attend(0, q, binding.KvBatch(b.page_table, b.ctx, b.start, 2, 3)),
        lambda: binding.KvCache(case.t["k"], case.t["v"][:, :1], "f16"), lambda: binding.KvCache(case.t["k"], case.t["v"], "bf16"),
        lambda: binding.dresd_kv_attend(c.handle, 0, b.c, 0, 256, 64, 4, 1.0, None, 0, q.data_ptr(), None),
        lambda: binding.dresd_kv_attend(c.handle, 0, b.c, q.data_ptr(), 256, 32, 4, 1.0, None, 0, q.data_ptr(), None),
        lambda: binding.dresd_kv_attend(c.handle, 0, b.c, q.data_ptr(), -256, 64, 4, 1.0, None, 0, q.data_ptr(), None),
        lambda: binding.dresd_kv_attend(c.handle, 0, b.c, q.data_ptr(), 256, 64, 4, 1.0, None, 0, q.data_ptr() + 2, None),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.DresdError) as e:
            call()
        assert e.value.status == -1, (i, e.value)
    for call in (lambda: c.attend(0, torch.zeros((2, 130, 64), dtype=torch.float16, device="cuda"), b),
                 lambda: c.keep_draft(b, i32(1), i32(1), 33, 2), lambda: binding.KvCache(case.t["k"], case.t["v"], "f32")):
        with pytest.raises(binding.DresdError) as e:
            call()
        assert e.value.status == -2, e.value
    c.status()
    empty = binding.KvBatch(b.page_table[:0].contiguous(), b.ctx[:0], i32(0), 0)
    assert c.attend(0, q[:0], empty).shape == (0, 4, 64) and c.last_launches() == 0
    c.append(0, k[:0], k[:0], empty)
    c.keep_draft(empty, i32(), i32(), 2, 2)
