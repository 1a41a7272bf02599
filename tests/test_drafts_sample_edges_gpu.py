"""Verification by sampling where few calls go: CTAs that begin late, rows so long that an entry stands for several steps, temperatures at
their ends, and the weights themselves."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding
from tests.test_drafts_sample_gpu import DT, ONE, chunk, ref_row

pytestmark = pytest.mark.gpu


def test_clusters_of_a_busy_gpu():
    """Calls whose CTAs begin while others of all sizes still run, one behind the other and on two streams: what each gives alone."""
    g = torch.Generator(device="cuda").manual_seed(6)
    calls = []
    for B, V in ((1, 32000), (9, 20001), (17, 9000), (40, 33001), (150, 2500)):
        logits = (torch.randn((B, 1, V), device="cuda", generator=g) * 2).half()
        u, p = torch.rand((B, 1), device="cuda", generator=g), torch.full((B,), 0.9, device="cuda")
        calls.append(lambda x=logits, u=u, p=p: binding.drafts_sample(x, u, top_p=p))
    logits, uniform, drafts, valid = chunk(7, 3, 5, 12001, "bf16", 4)
    u, d, v = (torch.from_numpy(a).cuda() for a in (uniform.astype(np.float32), drafts, valid))
    calls.append(lambda: binding.drafts_sample(logits, u, d, v))
    want = []
    for call in calls:
        want.append(call())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(20):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                i = (turn * (1 + 2 * s) + s) % len(calls)
                got.append((i, calls[i]()))
    torch.cuda.synchronize()
    for i, outs in got:
        assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))


# ---- temperatures at their ends ------------------------------------------------------------------------------------
def check_clipped(logits, uniform, temperature, top_k=0, top_p=1.0):
    """check() with temperatures brought into 10^-36 .. 10^33; a weight is off by 2^-28, so the logarithm of their sum by less than 2^-27."""
    B = logits.shape[0]
    new = lambda x, dtype: torch.full((B,), x, dtype=dtype, device="cuda")
    got = binding.drafts_sample(logits, torch.from_numpy(uniform.astype(np.float32)).cuda(), temperature=torch.from_numpy(temperature).cuda(),
                                top_k=new(top_k, torch.int32), top_p=new(top_p, torch.float32))
    x = logits.double().cpu().numpy()
    for b in range(B):
        T = min(max(np.float64(temperature[b]), np.float64(np.float32(1e-36))), np.float64(np.float32(1e33)))
        token, log = ref_row(x[b, 0], np.float32(uniform[b, 0]), T, top_k, np.float32(top_p))
        assert int(got[2][b, 0]) == token, (b, T, int(got[2][b, 0]), token)
        assert abs(float(got[3][b, 0]) - log) <= 2.0 ** -24 * abs(log) + 2.0 ** -27, (b, T, float(got[3][b, 0]), log)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_k,top_p", [(0, 1.0), (7, 1.0), (300, 0.8), (0, 0.7)])
@pytest.mark.parametrize("temperature", [2.0 ** -149, 1e-45, 1e-42, 1e-40, 1e-38, 1e-37, 1e-36, 1e-35])
def test_small_temperatures(temperature, top_k, top_p, dtype):
    """Logits within a few hundred temperatures of each other, subnormal numbers among them, around zero and away from it.  (Of 1000 borders one
    is next to a random number, within 2^-28 of the whole, with a probability of 2^-18.)"""
    g = np.random.default_rng(11)
    T = np.float32(temperature)
    x = -np.abs(g.standard_normal((6, 1, 1000))) * 20 * max(np.float64(T), 2e-44)
    x[1] += 5 * np.float64(T)
    x[2, 0, ::3] = 0
    x[3] = np.float32(-2.0 ** -149) * g.integers(0, 9, 1000)
    x[4, 0, 500:] = -np.inf
    x[5] *= 1e8
    check_clipped(torch.from_numpy(x).to(DT[dtype]).cuda(), g.random((6, 1)), np.full(6, T), top_k, top_p)


@pytest.mark.parametrize("top_k,top_p", [(0, 1.0), (7, 1.0), (0, 0.7)])
@pytest.mark.parametrize("temperature", [1e30, 1e33, 1e34, 1e35, 1e36, 1e38, np.inf])
def test_large_temperatures(temperature, top_k, top_p):
    g = np.random.default_rng(12)
    T = np.float32(temperature)
    x = g.standard_normal((4, 1, 1000)) * 5 * min(np.float64(T), 1e33)
    x[1] *= 100
    x[2] = np.where(g.random((1, 1000)) < 0.5, 3e38, -3e38)
    x[3] = x[3] / 1e20
    check_clipped(torch.from_numpy(x).float().cuda(), g.random((4, 1)), np.full(4, T), top_k, top_p)


# ---- rows so long that an entry of a warp's sums stands for several of its steps -----------------------------------
def alone(logits, u, settings, size):
    """The same rows, `size` at a time: more CTAs a row, and fewer steps of each."""
    parts = [binding.drafts_sample(logits[b:b + size], u[b:b + size], **{k: v[b:b + size] for k, v in settings.items()}) for b in range(0, logits.shape[0], size)]
    return [torch.cat(p) for p in zip(*parts)]


@pytest.mark.parametrize("dtype,V", [("bf16", 151937), ("f16", 262147), ("f32", 70001), ("f32", 200003)])
@pytest.mark.parametrize("values", ["many", "few"])
def test_one_cta_for_a_long_row(dtype, V, values):
    """One CTA has more than 16384 blocks of 16 bytes: entries of 2 or 4 steps."""
    B = 152
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((B, 1, V), device="cuda", generator=g) * 2
    logits = (x.round() if values == "few" else x).to(DT[dtype])
    del x
    random = np.random.default_rng(V)
    u = random.random((B, 1)).astype(np.float32)
    u[:4, 0] = 0, 1 - 2.0 ** -24, 2.0 ** -24, 0.5
    kind = np.arange(B) % 4                                   # all tokens, top_p, top_k and top_p, the largest
    t, k, p = np.where(kind == 3, 0, 0.9).astype(np.float32), np.where(kind == 2, 1000, 0).astype(np.int32), np.where(kind % 3 == 0, 1, 0.9).astype(np.float32)
    settings = dict(temperature=torch.from_numpy(t).cuda(), top_k=torch.from_numpy(k).cuda(), top_p=torch.from_numpy(p).cuda())
    ud = torch.from_numpy(u).cuda()
    got = binding.drafts_sample(logits, ud, **settings)
    for a, b in zip(got, alone(logits, ud, settings, 8)):
        assert torch.equal(a, b)
    for b in list(range(12)) + [B - 1]:
        token, log = ref_row(logits[b, 0].double().cpu().numpy(), u[b, 0], np.float64(t[b]), k[b], p[b])
        assert int(got[2][b, 0]) == token
        assert abs(float(got[3][b, 0]) - log) <= 2.0 ** -24 * abs(log) + 2.0 ** -27


def test_one_cta_for_the_longest_row():
    """2^20 logits in fp32: entries of 16 steps or 32.  The last token with weight lies at the very end, in a step that is not full."""
    B, V = 150, 1 << 20
    wide = torch.randn((B, 1, V + 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    logits = wide[:, :, 1:] if wide.data_ptr() % 16 == 0 else wide[:, :, :V]        # rows begin anywhere in a block
    u = torch.rand((B, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    u[0], u[1] = 0, 1 - 2.0 ** -24
    logits[2, 0, :-1] = -float("inf")
    for p in (1.0, 0.5):
        settings = dict(top_p=torch.full((B,), p, device="cuda"))
        got = binding.drafts_sample(logits, u, **settings)
        for a, b in zip(got, alone(logits, u, settings, 6)):
            assert torch.equal(a, b)
        assert int(got[2][2, 0]) == V - 1


# ---- the weights -----------------------------------------------------------------------------------------------------
def brackets(w, N, M, g, below):
    """(u, j) for a row of N logits of weight W, w or nearly, and M of 2^42 behind them: u S >= j W exactly if W <= theta = u M 2^42 / (j - u N).  theta
    lies beyond what W may be, w (1 +- 2^-28) and half a unit: by 2^-29 at most (or 1/4)."""
    edge = w * (1 - 2.0 ** -28) - 0.5 if below else w * (1 + 2.0 ** -28) + 0.5
    room = max(w * 2.0 ** -29, 0.25)
    q = M * 2.0 ** 42 / (edge + (-0.5 if below else 0.5) * room)      # j - u N over u
    scale = 2.0 ** -np.ceil(max(0.0, np.log2((N + q) / N)))
    for _ in range(4):
        u = g.integers(1 << 23, 1 << 24, 1 << 20) * 2.0 ** -24 * scale
        j = np.rint(u * (N + q))
        with np.errstate(divide="ignore"):
            theta = u * M * 2.0 ** 42 / (j - u * N)           # j, u N: exact in 53 bits; relative error 2^-51
        off = (edge - theta if below else theta - edge)
        fits = np.flatnonzero((off > room * 2.0 ** -6) & (off < room) & (j >= 1) & (j <= N))
        if len(fits):
            return u[fits[0]], int(j[fits[0]])
    return None


@pytest.mark.parametrize("temperature,top", [(1.0, 0.0), (0.7, 3.25), (0.05, -11.5), (1.3, 100.0), (0.7, 5000.0), (0.1, -900.0), (1e-36, 7e-36), (1e33, 2e34), (1e-30, 1e-26)])
def test_a_weight_is_off_by_less_than_its_bound(temperature, top):
    """The documented bound, 2^-28 of the weight and the rounding to a whole number, from both sides: a random number that draws a
    token for every weight within the bound, and one that does not.  (log_probabilities in fp32 are too coarse to show it.)  |top| / T above
    2^12 ln 2 takes another form of the difference."""
    g = np.random.default_rng(3)
    T, rows = np.float64(np.float32(temperature)), []
    N, top = 1 << 14, np.float32(top)
    gaps = np.concatenate((np.geomspace(1e-3, 26, 24), np.arange(1, 9) * np.log(2) / 64 * 7.5))
    for gap in gaps:
        x = np.float32(np.float64(top) - gap * T)
        if x == top:
            continue
        w = ONE * np.exp((np.float64(x) - np.float64(top)) / T)
        for below in (False, True):
            M, found = 0, None
            while found is None:                              # (some M have few random numbers that come near)
                M = int(max(1, g.uniform(0.7, 1.3) * 2.0 ** 13 * w / ONE))
                found = brackets(w, N, M, g, below)
            rows.append((x, M, below, *found))
    most = N + max(r[1] for r in rows)
    logits = np.full((len(rows), 1, most), -np.inf, dtype=np.float32)
    for i, (x, M, _, _, _) in enumerate(rows):
        logits[i, 0, :N] = x
        logits[i, 0, N:N + M] = top
    u = np.array([r[3] for r in rows])
    assert (u == u.astype(np.float32)).all()
    got = binding.drafts_sample(torch.from_numpy(logits).cuda(), torch.from_numpy(u.astype(np.float32)[:, None]).cuda(),
                                temperature=torch.full((len(rows),), float(T), device="cuda"))[2][:, 0].tolist()
    assert len(rows) > 20
    for y, (x, M, below, _, j) in zip(got, rows):
        # the token is the first one whose running sum exceeds floor(u S): j or later exactly if j W <= u S
        assert (y >= j) is (not below), (x, y, j, below)
