"""Attention over the paged cache where a worker goes through several segments, where 8-bit rows differ in size by
powers of two, and where masked rows hold anything: against float64 on the GPU, vectorised (the definitions and the
derivation of the tolerance are those of test_kv_cache_gpu).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding
from tests.test_kv_cache_gpu import DT, U, Case, bits_of, ref_quantise

pytestmark = pytest.mark.gpu


class Large(Case):
    """A case whose pool is made on the GPU (random rows; quantised by the definition, in torch)."""

    def __init__(self, dtype, d, page, Hkv, ctx, chunk, quantised=False, seed=0):
        super().__init__(dtype, d, page, 1, [0] * len(ctx), [0] * len(ctx), quantised, seed=seed)      # handles of an empty pool
        self.cache.close()
        rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
        self.Hkv, self.ctx, self.chunk = Hkv, list(ctx), list(chunk)
        need = [-(-(c + n) // page) for c, n in zip(ctx, chunk)]
        self.pages, at = sum(need) + 3, 0
        order = rng.permutation(self.pages)
        self.table_np = np.full((self.B, max(need)), -1, dtype=np.int32)
        for b, m in enumerate(need):
            self.table_np[b, :m] = order[at:at + m]
            at += m
        self.start_np = np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
        self.rows = int(self.start_np[-1])
        for name in ("k", "v"):
            x = torch.randn((1, self.pages, Hkv, page, d), device="cuda", generator=gen).to(DT[dtype])
            self.t[name], self.t[name + "_exp"] = x, None
            if quantised:
                m, e = torch.frexp(x.float().abs().amax(-1))          # 448 = 0.875 2^9
                e = torch.where(m <= 0.875, e - 9, e - 8)
                self.t[name] = torch.ldexp(x.float(), -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
                self.t[name + "_exp"] = (e + 127).to(torch.uint8)
        self.cache = binding.KvCache(self.t["k"], self.t["v"], dtype, k_exps=self.t["k_exp"], v_exps=self.t["v_exp"])
        dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()
        self.batch = binding.KvBatch(dev(self.table_np), dev(ctx), dev(self.start_np), rows=self.rows, max_chunk=max(chunk))


def held_rows(case, name, b, upto):
    """float64 [upto][Hkv][d] of a sequence, on the GPU."""
    p = np.arange(upto)
    page, off = torch.from_numpy(case.table_np[b, p // case.page].astype(np.int64)).cuda(), torch.from_numpy(p % case.page).cuda()
    x = case.t[name][case.layer][page, :, off]
    if not case.q8:
        return x.double()
    c = x.long()
    man, ex = (c & 7).double(), (c >> 3) & 15
    mag = torch.where(ex > 0, (8 + man) * torch.pow(2.0, (ex - 10).double()), man * 2.0 ** -9)
    e = case.t[name + "_exp"][case.layer][page, :, off].double() - 127
    return torch.where(c >= 128, -mag, mag) * torch.pow(2.0, e)[..., None]


def expected(case, q, b, see, scale):
    """One sequence: out [n][Hq][d], lse, the largest |v| seen, the largest sum |q k| scale of those positions whose weight is
    more than e^-40 of the largest (the score errors of the others move nothing); see: bool [n][S]."""
    s, e, S = case.start_np[b], case.start_np[b + 1], see.shape[1]
    n, Hq, G = int(e - s), q.shape[1], q.shape[1] // case.Hkv
    k, v, x = held_rows(case, "k", b, S), held_rows(case, "v", b, S), q[s:e].double().view(n, case.Hkv, G, case.d)
    sc = (torch.einsum("ihgd,jhd->ihgj", x, k) * scale).masked_fill(~see[:, None, None], -np.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(m > -np.inf, m, torch.zeros_like(m)))
    l = p.sum(-1, keepdim=True)
    v = torch.where(torch.isfinite(v), v, torch.zeros_like(v))        # rows that see them are not compared
    out = torch.einsum("ihgj,jhd->ihgd", p, v) / torch.where(l > 0, l, torch.ones_like(l))
    lse = (m + l.log()).squeeze(-1)
    big = torch.where(see[:, None], v.abs().amax(-1).T[None], 0.0).amax(-1)                      # [n][Hkv]
    ds = torch.einsum("ihgd,jhd->ihgj", x.abs(), k.abs()).mul(abs(scale))
    ds = ds.masked_fill(~(see[:, None, None] & (sc + case.d * 2.0 ** -23 * ds > m - 40)), 0).amax(-1)
    shape = lambda t: t.reshape(n, Hq, *t.shape[3:])
    return shape(out), shape(lse), shape(big[:, :, None].expand(n, case.Hkv, G)), shape(ds)


def causal_of(c, n):
    return torch.arange(c + n, device="cuda")[None] <= c + torch.arange(n, device="cuda")[:, None]


def check(case, q, seen=None, mask=None, scale=None, leave=()):
    """leave: rows that are not compared."""
    d, u = case.d, U[case.dtype]
    scale = d ** -0.5 if scale is None else scale
    lse = torch.full((case.rows, q.shape[1]), 7.0, device="cuda")
    got = case.cache.attend(case.layer, q, case.batch, scale=scale, mask=mask, lse=lse)
    torch.cuda.synchronize()
    case.cache.status()
    for b in range(case.B):
        c, n = case.ctx[b], case.chunk[b]
        if n == 0:
            continue
        s, e = case.start_np[b], case.start_np[b + 1]
        want, wlse, V, ds = expected(case, q, b, causal_of(c, n) if seen is None else seen[b], scale)
        ds = (d + 4) * 2.0 ** -24 * ds
        tol = u * V[..., None] + u * want.abs() + ((2 * (ds + 2.0 ** -21) + (c + n) * 2.0 ** -24) * V)[..., None]
        if case.dtype == "f16":
            tol = tol + 2.0 ** -24                            # the type's step below its normal numbers
        rows = [i for i in range(n) if s + i not in leave]
        err, tol = (got[s:e].double() - want).abs()[rows], tol[rows]
        assert torch.isfinite(got[s:e][rows]).all(), f"sequence {b}: not finite"
        assert (err <= tol).all(), f"sequence {b}: {(err / tol).max().item()} tolerances"
        off = (lse[s:e].double() - wlse).abs() <= ds + 2.0 ** -20 + 2.0 ** -23 * wlse.abs()
        assert (off | (lse[s:e].double() == wlse))[rows].all(), f"sequence {b}: lse"
    return got


def ragged(seed, B, lo, hi):
    rng = np.random.default_rng(seed)
    return [int(x) for x in rng.integers(lo, hi + 1, B)]


# ---- several segments a worker ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,quantised", [("bf16", 64, True), ("bf16", 128, True), ("f16", 64, True), ("bf16", 128, False),
                                               ("f16", 64, False)])
@pytest.mark.parametrize("tree", [False, True])
def test_many_row_items_of_ragged_batches(dtype, d, quantised, tree):
    """More items than SMs, lengths that share no cut: a CTA has the tail of one item, whole ones and the head of another.
    The queries of every sequence have a size of their own."""
    B, Hkv, G = 30, 4, 3
    ctx, chunk = ragged(1, B, 0, 2500), ragged(2, B, 40, 200)
    ctx[3], chunk[5], chunk[6] = 0, 0, 1
    case = Large(dtype, d, 64, Hkv, ctx, chunk, quantised, seed=70)
    q = case.queries(Hkv * G)
    for b in range(B):
        q[case.start_np[b]:case.start_np[b + 1]] *= 2.0 ** (b % 7 - 4)
    seen = mask = None
    if tree:                                                  # random bits, but every token sees itself
        g = torch.Generator(device="cuda").manual_seed(3)
        bits = torch.rand((case.rows, max(chunk)), device="cuda", generator=g) < 0.5
        for b in range(B):
            i = torch.arange(chunk[b], device="cuda")
            bits[int(case.start_np[b]) + i, i] = True
        mask = bits_of(bits.cpu().numpy())
        seen = [torch.cat([torch.ones((chunk[b], ctx[b]), dtype=torch.bool, device="cuda"),
                           bits[int(case.start_np[b]):int(case.start_np[b + 1]), :chunk[b]]], 1) for b in range(B)]
    first = check(case, q, seen, mask)
    for _ in range(3):
        assert torch.equal(case.cache.attend(0, q, case.batch, mask=mask), first)


@pytest.mark.parametrize("dtype,d,quantised", [("f16", 128, False), ("bf16", 128, True), ("bf16", 64, False), ("f16", 64, True)])
@pytest.mark.parametrize("B,Hkv,G,hi,longest", [(70, 4, 4, 800, 9000), (160, 8, 7, 150, 3000), (300, 8, 1, 60, 1000), (60, 4, 12, 500, 5000)])
def test_single_tokens_of_large_ragged_batches(dtype, d, quantised, B, Hkv, G, hi, longest):
    """Groups of four, two and one warps with tiles of 8 rows, and of four with tiles of 16; several segments each."""
    ctx = ragged(B, B, 0, hi)
    ctx[0], ctx[B // 2] = 0, longest
    case = Large(dtype, d, 32, Hkv, ctx, [1] * B, quantised, seed=71)
    q = case.queries(Hkv * G)
    check(case, q)


@pytest.mark.parametrize("dtype,quantised", [("f16", False), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("chunk,path", [(1, 0), (33, 0), (2, 2), (33, 1)])
def test_long_contexts(dtype, quantised, chunk, path):
    """Parts of a long item joined through clusters and global memory."""
    case = Large(dtype, 128, 128, 2, [40000, 9999], [chunk] * 2, quantised, seed=72)
    case.cache.set_option("attend_path", path)
    check(case, case.queries(8))


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("f16", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("path,B,lo,hi", [(1, 30, 2, 30), (2, 30, 40, 150), (2, 3, 20, 60)])
def test_bad_values_in_several_segments(dtype, d, path, B, lo, hi):
    """16-bit values that are not finite, in the middle of every second chunk: tokens before them are untouched, through clusters,
    several segments and parts."""
    Hkv, ctx, chunk = 4, ragged(4, B, 0, 1500), ragged(5, B, lo, hi)
    case = Large(dtype, d, 32, Hkv, ctx, chunk, seed=84)
    case.cache.set_option("attend_path", path)
    leave = set()
    for b in range(0, B, 2):
        bad = chunk[b] // 2
        pg, off = case.place(b, ctx[b] + bad)
        case.t["v"][0, pg, :, off, ::7] = float("nan") if b % 4 else float("inf")
        leave |= {int(case.start_np[b]) + i for i in range(bad, chunk[b])}
    check(case, case.queries(3 * Hkv), leave=leave)


# ---- 8-bit rows of very different sizes -----------------------------------------------------------------------
BOTH = [("f16", 64), ("f16", 128), ("bf16", 64), ("bf16", 128)]


def put(case, name, b, p, x):
    """Row of token p of sequence b: x float64 [Hkv][d], as append holds it."""
    codes, exps = ref_quantise(np.broadcast_to(x, (case.Hkv, case.d)).astype(np.float64), case.dtype)
    pg, off = case.place(b, p)
    case.t[name][case.layer, pg, :, off] = torch.from_numpy(codes).cuda()
    case.t[name + "_exp"][case.layer, pg, :, off] = torch.from_numpy(exps).cuda()


def pathed(path, *args, **kw):
    case = Case(*args, quantised=True, **kw)
    case.cache.set_option("attend_path", path)
    return case


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("dtype,d", BOTH)
@pytest.mark.parametrize("chunk,G,peak", [(1, 4, 1.0), (30, 2, 6.0), (150, 1, 1.0), (1, 12, 6.0)])
def test_zero_rows_among_small_values(path, dtype, d, chunk, G, peak):
    """Rows of zeros (whose exponent byte is that of values near 448) among keys and values of 2^-10 (fp16) and 2^-20 (bf16), one
    of them first, one in the chunk; even weights and peaked ones."""
    amp = 2.0 ** (-10 if dtype == "f16" else -20)
    case = pathed(path, dtype, d, 32, 2, [900, 40, 0], [chunk] * 3, amp=amp, seed=75)
    for b in range(3):
        for p in (0, 17, 130, 131, 400, case.ctx[b] + chunk // 2):
            if p < case.ctx[b] + chunk - (chunk > 1):
                put(case, "v", b, p, 0.0)
                put(case, "k", b, p + (p > 0), 0.0)
    check(case, case.queries(2 * G, amp=peak), scale=d ** -0.5 / amp)


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("dtype,d", BOTH)
@pytest.mark.parametrize("chunk,G", [(5, 1), (30, 2), (100, 1), (90, 4)])
@pytest.mark.parametrize("what", ["k", "v", "kv"])
def test_tokens_that_are_not_seen_may_have_any_size(path, dtype, d, chunk, G, what):
    """A chunk token whose key or value is infinite (held as the bound): earlier tokens and those whose mask leaves it
    out are as if it were not there."""
    case = pathed(path, dtype, d, 16, 2, [300, 20], [chunk] * 2, seed=76)
    bad = chunk // 2
    for b in range(2):
        for name in what:
            put(case, name, b, case.ctx[b] + bad, np.where(np.arange(d) % 3 == 0, -np.inf, np.inf))
    q = case.queries(2 * G)
    check(case, q, leave={int(case.start_np[b]) + i for b in range(2) for i in range(bad, chunk)})
    tree = np.tri(chunk, dtype=bool)
    tree[:, bad] = False
    seen = [torch.from_numpy(np.concatenate([np.ones((chunk, c), dtype=bool), tree], 1)).cuda() for c in case.ctx]
    check(case, q, seen=seen, mask=bits_of(np.concatenate([tree, tree])))


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("dtype,d", BOTH)
@pytest.mark.parametrize("chunk,G", [(1, 4), (40, 3)])
def test_rows_of_very_different_sizes(path, dtype, d, chunk, G):
    """Values from 2^-12 to 2^12, and a key 2^10 (fp16) or 2^30 (bf16) above the others whose weight is zero for every query."""
    case = pathed(path, dtype, d, 64, 2, [500, 130], [chunk] * 2, seed=77)
    rng = np.random.default_rng(78)
    q = case.queries(2 * G)
    q[:, :, 0] = q[:, :, 0].abs() + 1
    for b in range(2):
        for p in range(case.ctx[b] + chunk):
            put(case, "v", b, p, rng.standard_normal((2, d)) * 2.0 ** rng.integers(-12, 13))
        x = np.zeros((2, d))
        x[:, 0] = -(2.0 ** (14 if dtype == "f16" else 30))
        put(case, "k", b, 70, x)
    check(case, q)


# ---- a long tail of small weights -------------------------------------------------------------------------------
@pytest.mark.parametrize("path,chunk", [(1, 1), (1, 9), (2, 40)])
@pytest.mark.parametrize("dtype,quantised", [("f16", False), ("f16", True), ("bf16", True), ("bf16", False)])
def test_tails_below_the_types_last_bit(dtype, quantised, path, chunk):
    """One position in 64 has e^18 = 2^26 times the weight of the others, whose values are large: what the tail adds up
    to is all that most elements of the result have.  Weights are off by u of themselves or by 2^-32 of the largest:
    |out - o| <= u sum p |v| / l + 2^-32 sum |v| / l + u |o| + fp32 terms, the weights p and their sum l relative to the largest;
    sum p |v| / l is |o|, as every element's values have one sign."""
    S, d = 8000, 64
    case = Case(dtype, d, 64, 1, [S], [chunk], quantised, seed=79)
    case.cache.set_option("attend_path", path)
    k, v = np.zeros((S + chunk, 1, d)), np.full((S + chunk, 1, d), 28672.0)
    k[::64, :, 0], v[::64, :, 1:], v[:, :, 0] = 18, 0, 0
    v[::64, :, 0] = 1
    for name, x in (("k", k), ("v", v)):
        page, off = zip(*(case.place(0, p) for p in range(S + chunk)))
        if quantised:
            codes, exps = ref_quantise(x, dtype)
            case.t[name][0, page, :, off] = torch.from_numpy(codes).cuda()
            case.t[name + "_exp"][0, page, :, off] = torch.from_numpy(exps).cuda()
        else:
            case.t[name][0, page, :, off] = torch.from_numpy(x).to(DT[dtype]).cuda()
    q = torch.zeros((chunk, 2, d), dtype=DT[dtype], device="cuda")
    q[:, :, 0] = 8
    lse = torch.empty((chunk, 2), device="cuda")
    got = case.cache.attend(0, q, case.batch, lse=lse).double()
    want, wlse, V, ds = expected(case, q, 0, causal_of(S, chunk), d ** -0.5)
    u, ds, l = U[dtype], (d + 4) * 2.0 ** -24 * ds[..., None], torch.exp(wlse - 18)[..., None]
    step = 0 if dtype == "bf16" and not quantised else 2.0 ** -32 * (S + chunk) * V[..., None] / l
    tol = (2 * u + 2 * (ds + 2.0 ** -21) + (S + chunk) * 2.0 ** -24) * want.abs() + step + 2.0 ** -24
    assert want[0, 0, 1] > 20 * tol[0, 0, 1] or dtype == "bf16"
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()
    assert ((lse - wlse).abs() <= ds[..., 0] + 2.0 ** -20 + 2.0 ** -23 * wlse.abs()).all()


# ---- the same call, the same bits -------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,quantised", [("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("G,chunk,path", [(3, 50, 2), (7, 20, 2), (12, 200, 2), (3, 1, 1), (5, 4, 1), (7, 30, 1)])
def test_repeatable_whatever_ran_before(dtype, quantised, G, chunk, path):
    """Groups that do not divide a row tile, and other calls in between whose queries are very large or very small."""
    case = Large(dtype, 64, 16, 3, [700, 90, 2100, 0], [chunk, 1, chunk, chunk // 2 + 1], quantised, seed=73)
    other = Large(dtype, 64, 16, 2, [600] * 80, [8 * chunk // G + 1] * 80, quantised, seed=74)
    case.cache.set_option("attend_path", path)
    other.cache.set_option("attend_path", path)
    q = case.queries(3 * G)
    first = check(case, q)
    for amp in (1e-3, 8.0, 200.0):
        other.cache.attend(0, other.queries(2 * 8, amp=amp), other.batch)
        assert torch.equal(case.cache.attend(0, q, case.batch), first)


# ---- waits that run out -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("B,chunk,path,stage", [(2, 1, 1, 1), (2, 1, 1, 3), (60, 1, 1, 1), (60, 1, 1, 3)] +
                         [(b, c, p, s) for b, c, p in ((2, 50, 1), (2, 30, 2), (12, 90, 2)) for s in (1, 3, 11)])
def test_waits_that_run_out_in_either_kernel(B, chunk, path, stage, quantised):
    """A warp (K11) or CTA (K12) never receives one of its tiles -- alone, in a cluster, in one group of several --: the call ends,
    the status says so once, and the next call is right again."""
    ctx = [30000] + [600] * (B - 1)
    case = Large("bf16", 128, 32, 4, ctx, [chunk] * B, quantised, seed=80)
    case.cache.set_option("attend_path", path)
    q = case.queries(8)
    first = case.cache.attend(0, q, case.batch)
    case.cache.status()
    case.cache.set_option("wait_ms", 20)
    case.cache.set_option("debug_lose_stage", stage)
    case.cache.attend(0, q, case.batch)
    with pytest.raises(binding.DresdError) as e:
        case.cache.status()
    assert e.value.status == -5
    case.cache.set_option("debug_lose_stage", 0)
    case.cache.set_option("wait_ms", 0)
    for _ in range(2):
        assert torch.equal(case.cache.attend(0, q, case.batch), first)
        case.cache.status()


# ---- lengths that cannot be --------------------------------------------------------------------------------------
@pytest.mark.parametrize("path,chunk", [(1, 1), (1, 40), (2, 40), (2, 200)])
@pytest.mark.parametrize("ctx", [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 4097, 10 ** 6])
@pytest.mark.parametrize("quantised,masked", [(False, False), (False, True), (True, False)])
def test_contexts_beyond_the_table(path, chunk, ctx, quantised, masked):
    """A sequence whose ctx is far beyond its table, as far as 31 bits go: its own result is unspecified, the
    other sequences' are what they are, nothing is written to the cache."""
    case = Case("f16", 64, 16, 2, [37, 500, 90], [chunk] * 3, quantised, seed=81)
    case.cache.set_option("attend_path", path)
    q = case.queries(6)
    mask = bits_of(np.concatenate([np.tri(chunk, dtype=bool)] * 3)) if masked else None
    want = case.cache.attend(0, q, case.batch, mask=mask)
    case.batch.ctx[1] = ctx
    held = {x: t.clone() for x, t in case.t.items() if t is not None}
    got = case.cache.attend(0, q, case.batch, mask=mask)
    good = torch.ones(case.rows, dtype=torch.bool, device="cuda")
    good[chunk:2 * chunk] = False
    # the work is divided otherwise, so the sums may be in another order: two roundings, and the weights'
    most = held_rows(case, "v", 0, 37 + chunk).abs().max(), held_rows(case, "v", 2, 90 + chunk).abs().max()
    assert ((got[good].double() - want[good].double()).abs() <= 4 * U["f16"] * max(most)).all()
    k = torch.zeros((case.rows, 2, 64), dtype=torch.float16, device="cuda")
    case.batch.ctx.fill_(ctx)
    case.cache.append(0, k, k, case.batch)
    case.cache.keep_draft(case.batch, torch.ones(3, dtype=torch.int32, device="cuda"), torch.full((3,), 3, dtype=torch.int32, device="cuda"), 2, 2)
    assert not case.cache.read(0, case.batch)[0].any()
    assert all(torch.equal(case.t[x], t) for x, t in held.items())
    case.cache.status()


@pytest.mark.parametrize("path,chunk", [(1, 1), (1, 20), (2, 50)])
def test_tables_so_wide_that_the_plan_counts_in_64_bits(path, chunk):
    B, Hkv = 200, 4
    ctx = ragged(82, B, 0, 200)
    case = Case("f16", 64, 16, Hkv, ctx, [chunk] * B, seed=82)
    case.cache.set_option("attend_path", path)
    q = case.queries(2 * Hkv)
    check(case, q)
    table = torch.full((B, 1 << 18), -1, dtype=torch.int32, device="cuda")
    table[:, :case.batch.page_table.shape[1]] = case.batch.page_table
    case.batch = binding.KvBatch(table, case.batch.ctx, case.batch.start, rows=case.rows, max_chunk=chunk)
    check(case, q)


@pytest.mark.parametrize("path", [1, 2])
def test_starts_that_contradict_each_other(path):
    """Every second sequence has all rows: unspecified results, but an end, and nothing written beside them."""
    B, rows = 41, 60
    case = Case("bf16", 64, 32, 2, [100] * B, [rows] * B, seed=83)
    case.cache.set_option("attend_path", path)
    start = torch.tensor([rows * (b % 2) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    batch = binding.KvBatch(case.batch.page_table, case.batch.ctx, start, rows=rows, max_chunk=0)
    out = torch.full((3 * rows, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    case.cache.attend(0, case.queries(4)[:rows], batch, out=out[rows:2 * rows])
    case.cache.status()
    assert (out[:rows] == 7).all() and (out[2 * rows:] == 7).all()
