"""What the paged key/value cache and its attention are measured on.

The language model that verifies retrieved drafts keeps its keys and values in a paged cache.  Four operators work on
it: `append` writes (and quantises) the keys and values of new tokens, `read` brings a range of positions back,
`attend` is the attention of a chunk of new tokens over the cache (one token per sequence, a chunk of drafts with a
visibility mask, or a piece of a prompt), and `keep` moves the accepted draft's tokens into place.

A cache is [layers][pages][kv heads][page][d], keys and values apart, in fp16 / bf16, or in 8 bits (E4M3) with one
power-of-two scale per token and head.  Chunk token i of sequence b has position ctx[b] + i; its row in the dense
tensors is start[b] + i.
"""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of one sequence behind a prompt of ordinary length, every head its own keys: latency
        dict(name="decode 1 x 700", op="attend", B=1, heads=32, kv_heads=32, d=128, page=16, dtype="f16", quantised=False,
             drafts=0, draft_len=0, chunk_lo=1, chunk_hi=1, ctx_lo=700, ctx_hi=700),
        # a serving batch of very different lengths, one of them just begun, on an 8-bit cache with grouped heads
        dict(name="decode ragged 48 e4m3", op="attend", B=48, heads=32, kv_heads=8, d=128, page=64, dtype="bf16",
             quantised=True, drafts=0, draft_len=0, chunk_lo=1, chunk_hi=1, ctx_lo=0, ctx_hi=8191),
        # two long documents: the bytes of the cache are the cost
        dict(name="decode 2 x 131071", op="attend", B=2, heads=64, kv_heads=8, d=128, page=128, dtype="bf16",
             quantised=False, drafts=0, draft_len=0, chunk_lo=1, chunk_hi=1, ctx_lo=131071, ctx_hi=131071),
        # batch verification of ten drafts of ten tokens (and the token before them) by one sequence
        dict(name="verify 10 x 10", op="attend", B=1, heads=32, kv_heads=32, d=128, page=16, dtype="f16", quantised=False,
             drafts=10, draft_len=10, chunk_lo=101, chunk_hi=101, ctx_lo=1999, ctx_hi=1999),
        # three drafts of twenty tokens for sixteen sequences, heads of 64, 8-bit cache
        dict(name="verify 3 x 20 e4m3", op="attend", B=16, heads=40, kv_heads=10, d=64, page=32, dtype="bf16",
             quantised=True, drafts=3, draft_len=20, chunk_lo=61, chunk_hi=61, ctx_lo=500, ctx_hi=4035),
        # a piece of a long prompt, as the hidden states of a datastore's corpus are computed
        dict(name="prompt 2047 at 12345", op="attend", B=1, heads=32, kv_heads=8, d=128, page=64, dtype="bf16",
             quantised=False, drafts=0, draft_len=0, chunk_lo=2047, chunk_hi=2047, ctx_lo=12345, ctx_hi=12345),
        # the tokens of one verification step, written as they are
        dict(name="append 101", op="append", B=1, kv_heads=32, heads=32, d=128, page=16, dtype="f16", quantised=False,
             chunk_lo=101, chunk_hi=101, ctx_lo=299, ctx_hi=299),
        # prompts of four sequences, quantised as they are written
        dict(name="append 4 x 8000 e4m3", op="append", B=4, kv_heads=8, heads=32, d=128, page=64, dtype="bf16",
             quantised=True, chunk_lo=7001, chunk_hi=9001, ctx_lo=0, ctx_hi=77),
        # a short range back out of an 8-bit cache
        dict(name="read 300 e4m3", op="read", B=1, kv_heads=8, heads=8, d=128, page=64, dtype="f16", quantised=True,
             chunk_lo=300, chunk_hi=300, ctx_lo=53, ctx_hi=53),
        # whole sequences back out of a 16-bit cache, to be kept elsewhere
        dict(name="read 3 x 20000", op="read", B=3, kv_heads=8, heads=8, d=128, page=32, dtype="bf16", quantised=False,
             chunk_lo=15001, chunk_hi=25000, ctx_lo=0, ctx_hi=0),
        # the accepted tokens of one verified step, every layer
        dict(name="keep 10 x 10", op="keep", B=1, kv_heads=8, d=128, page=16, dtype="f16", quantised=False, layers=32,
             drafts=10, draft_len=10, ctx_lo=211, ctx_hi=211),
        # the same for a batch on an 8-bit cache
        dict(name="keep 32 of 3 x 20 e4m3", op="keep", B=32, kv_heads=10, d=64, page=32, dtype="bf16", quantised=True,
             layers=40, drafts=3, draft_len=20, ctx_lo=50, ctx_hi=300),
    ]


def spread(rng, lo, hi):
    """A whole number in lo .. hi, spread over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "append", "read", "keep"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 10, 16, 32])
    case = dict(op=op, kv_heads=kv_heads, d=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
                dtype=rng.choice(["f16", "bf16"]), quantised=rng.random() < 0.5)
    if op == "keep":
        n = rng.randint(2, 12)
        ctx = spread(rng, 1, 300)
        return dict(case, B=spread(rng, 1, 32), kv_heads=min(kv_heads, 10), layers=spread(rng, 2, 40), drafts=n,
                    draft_len=rng.randint(1, 120 // n), ctx_lo=ctx // 3, ctx_hi=ctx)
    if op in ("append", "read"):
        tokens = spread(rng, 1, 32000)
        B = min(spread(rng, 1, 32), tokens)
        each = max(1, tokens // B)
        return dict(case, B=B, heads=kv_heads * rng.choice([1, 2, 4]), chunk_lo=max(1, each * 3 // 4),
                    chunk_hi=max(1, each * 5 // 4), ctx_lo=0, ctx_hi=spread(rng, 1, 500))
    case["heads"] = kv_heads * rng.choice([1, 1, 2, 4, 7, 8] if kv_heads <= 8 else [1, 2, 4])
    form = rng.choice(["decode", "verify", "prompt"])
    if form == "verify":
        n = rng.randint(2, 12)
        L = rng.randint(1, 120 // n)
        B, chunk, hi = spread(rng, 1, 24), 1 + n * L, spread(rng, 30, 16000)
    else:
        n = L = 0
        B = spread(rng, 1, 64) if form == "decode" else spread(rng, 1, 4)
        chunk, hi = 1 if form == "decode" else spread(rng, 16, 2047 // B), spread(rng, 20, 131071 if form == "decode" else 12345)
    # the cache of the longest sequences stays within that of the largest listed case, the scores too
    room = min(2.1e8 / (B * kv_heads * case["d"]), 9.4e8 / (B * chunk * case["heads"]))
    hi = max(1, min(hi, int(room)))
    return dict(case, B=B, drafts=n, draft_len=L, chunk_lo=chunk if n else max(1, chunk * 2 // 3), chunk_hi=chunk,
                ctx_lo=rng.choice([0, hi // 9, hi]), ctx_hi=hi)


def lengths(lo, hi, count):
    """`count` lengths from lo to hi, evenly over the logarithm, in a mixed order that the case alone decides."""
    if count == 1:
        return [hi]
    a = [min(hi, max(lo, round((lo + 1) * ((hi + 1) / (lo + 1)) ** (i / (count - 1)) - 1))) for i in range(count)]
    random.Random(97 * count + hi).shuffle(a)
    return a


def accepted(case):
    """Per sequence: the accepted draft (-1: none) and the accepted tokens (the matched ones and the model's own)."""
    n, L = case["drafts"], case["draft_len"]
    best = [(3 * b + n - 1) % (n + 1) - (1 if b % 5 == 4 else 0) for b in range(case["B"])]
    best = [min(b, n - 1) for b in best]
    return best, [1 if best[b] < 0 else 1 + (3 * b + L) % (L + 1) for b in range(case["B"])]


def geometry(case):
    ctx = lengths(case["ctx_lo"], case["ctx_hi"], case["B"])
    if case["op"] == "keep":
        chunk = [1 + case["drafts"] * case["draft_len"]] * case["B"]
    else:
        chunk = lengths(case["chunk_lo"], case["chunk_hi"], case["B"])
    return ctx, chunk


def draft_mask(n, L):
    """[1 + n L][words] int32: bit j of row i: chunk token i sees chunk token j (the first token, and its own draft so far)."""
    size = 1 + n * L
    words = (size + 31) // 32
    rows = []
    for i in range(size):
        bits = 1
        if i:
            first = 1 + (i - 1) // L * L
            bits |= ((1 << (i - first + 1)) - 1) << first
        row = [(bits >> (32 * w)) & 0xFFFFFFFF for w in range(words)]
        rows.append([x - (1 << 32) if x >> 31 else x for x in row])
    return torch.tensor(rows, dtype=torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, d, Hkv, page, B = DTYPES[case["dtype"]], case["d"], case["kv_heads"], case["page"], case["B"]
    ctx, chunk = geometry(case)
    layers = case.get("layers", 1)
    width = max(-(-(c + n) // page) for c, n in zip(ctx, chunk))
    used = sum(-(-(c + n) // page) for c, n in zip(ctx, chunk))
    pages = used + 2
    # the pages of a sequence lie anywhere; places of the table that no token reaches hold page 0
    order = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        n = -(-(ctx[b] + chunk[b]) // page)
        table[b, :n] = order[at:at + n]
        at += n
    shape = (layers, pages, Hkv, page, d)
    s = dict(case=case, table=table, ctx=torch.tensor(ctx, dtype=torch.int32, device="cuda"), max_chunk=max(chunk),
             start=torch.tensor([sum(chunk[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda"), rows=sum(chunk))

    def filled(wide):
        """Cache contents; with `wide`, every sixteenth channel is larger than the others, as keys have them."""
        x = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
        return x.mul_((1 + wide * (torch.arange(d, device="cuda") % 16 == 3)).to(dtype))

    for name, wide in (("k", 3.0), ("v", 0.0)):
        if case["quantised"]:
            # bytes over the range that quantised rows use (largest magnitude 224 .. 448), exponents of ordinary rows
            x = (torch.empty(shape, dtype=torch.float16, device="cuda").normal_(generator=g) * 100).clamp_(-448, 448)
            s[name] = x.to(torch.float8_e4m3fn).view(torch.uint8)
            s[name + "_exp"] = torch.randint(127 - 8, 127 - 5, shape[:4], dtype=torch.uint8, device="cuda", generator=g)
            del x
        else:
            s[name] = filled(wide)
            s[name + "_exp"] = None
    T = s["rows"]
    if case["op"] == "append":
        # the projection of a layer: queries, keys and values of a token side by side
        wide = torch.randn((T, case["heads"] + 2 * Hkv, d), dtype=torch.float32, device="cuda", generator=g).to(dtype)
        s["new_k"], s["new_v"] = wide[:, case["heads"]:case["heads"] + Hkv], wide[:, case["heads"] + Hkv:]
    if case["op"] == "attend":
        s["q"] = torch.randn((T, case["heads"], d), dtype=torch.float32, device="cuda", generator=g).to(dtype)
        s["scale"] = 1 / math.sqrt(d)
        s["mask"] = None
        if case["drafts"]:
            s["mask"] = draft_mask(case["drafts"], case["draft_len"]).cuda().repeat(B, 1)
    if case["op"] == "keep":
        best, length = accepted(case)
        s["best"] = torch.tensor(best, dtype=torch.int32, device="cuda")
        s["length"] = torch.tensor(length, dtype=torch.int32, device="cuda")
    if own:
        from paper_2502_15572_b200 import binding
        s["cache"] = binding.KvCache(s["k"], s["v"], case["dtype"], k_exps=s["k_exp"], v_exps=s["v_exp"])
        s["batch"] = binding.KvBatch(s["table"], s["ctx"], s["start"], rows=T, max_chunk=s["max_chunk"])
    return s


def contents(s):
    """The cache as values: 8-bit codes as E4M3 numbers beside their exponent bytes."""
    if s["case"]["quantised"]:
        return [s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["k_exp"], s["v_exp"]]
    return [s["k"], s["v"]]


def run(s):
    op, case = s["case"]["op"], s["case"]
    if own:
        cache, batch = s["cache"], s["batch"]
        if op == "attend":
            return cache.attend(0, s["q"], batch, scale=s["scale"], mask=s["mask"])
        if op == "read":
            return cache.read(0, batch)
        if op == "append":
            cache.append(0, s["new_k"], s["new_v"], batch)
        else:
            cache.keep_draft(batch, s["best"], s["length"], case["drafts"], case["draft_len"])
        return contents(s)
    if op == "attend":
        return plain_attend(s)
    if op == "read":
        return plain_read(s)
    plain_append(s) if op == "append" else plain_keep(s)
    return contents(s)


# ---- the plain forms ---------------------------------------------------------------------------------------------
def row_owner(s):
    """The sequence of every dense row, and its place in the chunk."""
    t = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(s["start"][1:].contiguous(), t.to(torch.int32), right=True)
    return b, t - s["start"].long()[b]


def row_place(s):
    """Page and offset in the page of every dense row's token."""
    b, i = row_owner(s)
    p = s["ctx"].long()[b] + i
    return s["table"].long()[b, p // s["case"]["page"]], p % s["case"]["page"]


def as_float(codes, exps):
    if exps is None:
        return codes.float()
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), exps.int()[..., None] - 127)


def quantise(x):
    """E4M3 codes (as bytes) and exponent bytes of rows along the last dimension."""
    x = x.float()
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)                                  # amax = m 2^e, m in [0.5, 1): 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.zeros_like(e))
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def plain_append(s):
    page, off = row_place(s)
    for name, new in (("k", s["new_k"]), ("v", s["new_v"])):
        if s["case"]["quantised"]:
            codes, exps = quantise(new)
            s[name][0][page, :, off] = codes
            s[name + "_exp"][0][page, :, off] = exps
        else:
            s[name][0][page, :, off] = new


def plain_read(s):
    page, off = row_place(s)
    dtype = DTYPES[s["case"]["dtype"]]
    out = []
    for name in ("k", "v"):
        exps = s[name + "_exp"]
        out.append(as_float(s[name][0][page, :, off], None if exps is None else exps[0][page, :, off]).to(dtype))
    return out


def plain_keep(s):
    case = s["case"]
    L, size = case["draft_len"], case["page"]
    t = torch.arange(L, device="cuda")[None]
    best, kept = s["best"].long()[:, None], s["length"].long()[:, None] - 1
    moved = (t < kept) & (best >= 0)
    dst = s["ctx"].long()[:, None] + 1 + t
    src = torch.where(moved, dst + best * L, dst)             # a token that is not kept moves onto itself
    table = s["table"].long()
    sp, dp = table.gather(1, src // size), table.gather(1, dst // size)
    for name in ("k", "v"):
        s[name][:, dp, :, dst % size] = s[name][:, sp, :, src % size]
        if case["quantised"]:
            s[name + "_exp"][:, dp, :, dst % size] = s[name + "_exp"][:, sp, :, src % size]


def plain_attend(s):
    case = s["case"]
    dtype, d, Hkv, page = DTYPES[case["dtype"]], case["d"], case["kv_heads"], case["page"]
    G, M, B, T = case["heads"] // Hkv, s["max_chunk"], case["B"], s["rows"]
    table = s["table"].long()

    def dense(name):
        exps = s[name + "_exp"]
        x = as_float(s[name][0][table], None if exps is None else exps[0][table])      # [B][width][Hkv][page][d]
        return x.transpose(1, 2).reshape(B, Hkv, -1, d)

    start, ctx = s["start"].long(), s["ctx"].long()
    rows = start[:-1, None] + torch.arange(M, device="cuda")                            # [B][M]
    inside = rows < start[1:, None]
    rows = rows.clamp(max=T - 1)
    q = s["q"].float()[rows].view(B, M, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, M * G, d)
    scores = torch.matmul(q, dense("k").transpose(2, 3)) * s["scale"]
    S = scores.shape[-1]
    j = torch.arange(S, device="cuda")[None, None] - ctx[:, None, None]                 # place in the chunk, < 0: context
    if s["mask"] is None:
        seen = j <= torch.arange(M, device="cuda")[None, :, None]
    else:
        words = s["mask"][rows]                                                        # [B][M][words]
        w = (j.clamp(min=0) // 32).clamp(max=words.shape[-1] - 1).expand(B, M, S)
        seen = (j < 0) | (((words.gather(2, w) >> (j.clamp(min=0) % 32).int()) & 1) != 0)
    seen = seen & (j < (start[1:] - start[:-1])[:, None, None]) & inside[:, :, None]
    seen = seen[:, None, :, None].expand(B, 1, M, G, S).reshape(B, 1, M * G, S)
    scores.masked_fill_(~seen, float("-inf"))
    m = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(m > float("-inf"), m, torch.zeros_like(m))).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, dense("v")) / torch.where(l > 0, l, torch.ones_like(l))
    o = o.view(B, Hkv, M, G, d).permute(0, 2, 1, 3, 4).reshape(B, M, Hkv * G, d)
    b, i = row_owner(s)
    return o[b, i].to(dtype)


# ---- what cannot be done without ----------------------------------------------------------------------------------
def work(case):
    ctx, chunk = geometry(case)
    d, Hkv, T = case["d"], case["kv_heads"], sum(chunk)
    per_row = d + 1 if case["quantised"] else 2 * d            # bytes of one token's head in the cache, keys or values
    if case["op"] == "keep":
        best, length = accepted(case)
        moved = sum(n - 1 for b, n in zip(best, length) if b > 0)
        return {"bytes": max(1, 4 * moved * case["layers"] * Hkv * per_row + 8 * case["B"]), "flops": 0}
    if case["op"] in ("append", "read"):
        return {"bytes": 2 * T * Hkv * (2 * d + per_row), "flops": 0}
    pairs = 0
    for c, n in zip(ctx, chunk):
        if case["drafts"]:
            L = case["draft_len"]
            pairs += n * c + 1 + case["drafts"] * (L + L * (L + 1) // 2)
        else:
            pairs += n * c + n * (n + 1) // 2
    tokens = sum(ctx) + T
    return {"bytes": 2 * tokens * Hkv * per_row + 4 * T * case["heads"] * d, "flops": 4 * d * case["heads"] * pairs}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def value64(codes, exps):
    """Values of cache rows: E4M3 codes taken apart by sign, exponent (bias 7) and three mantissa bits."""
    if exps is None:
        return codes.double()
    c = codes.to(torch.int64)
    man, ex = (c & 7).double(), (c >> 3) & 15
    mag = torch.where(ex > 0, (8 + man) * torch.pow(2.0, (ex - 10).double()), man * 2.0 ** -9)
    return torch.where(c >= 128, -mag, mag) * torch.pow(2.0, exps[..., None].double() - 127)


def nearest64(x, bits, least):
    """x rounded to `bits` significant bits, ties to even, multiples of 2^least at the finest."""
    e = torch.floor(torch.log2(x.abs().clamp(min=1e-300)))
    e = torch.where(torch.pow(2.0, e) > x.abs(), e - 1, e)
    e = torch.where(torch.pow(2.0, e + 1) <= x.abs(), e + 1, e)
    step = torch.pow(2.0, torch.clamp(e - (bits - 1), min=least))
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    ctx, chunk = geometry(case)
    d, Hkv, size = case["d"], case["kv_heads"], case["page"]
    first = [sum(chunk[:b]) for b in range(case["B"])]
    q8 = case["quantised"]

    def places(b, lo, hi):
        p = torch.arange(lo, hi, device="cuda")
        return s["table"][b].long()[p // size], p % size

    if case["op"] == "attend":
        G = case["heads"] // Hkv
        pairs = sum(n * (c + n) for c, n in zip(ctx, chunk)) * case["heads"]
        if pairs * d > 5e12:
            return None
        out = torch.zeros((s["rows"], case["heads"], d), dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            c, n = ctx[b], chunk[b]
            page, off = places(b, 0, c + n)
            k, v = (value64(s[x][0][page, :, off], s[x + "_exp"][0][page, :, off] if q8 else None) for x in ("k", "v"))
            see = torch.ones((n, c + n), dtype=torch.bool, device="cuda")
            if case["drafts"]:
                L = case["draft_len"]
                draft = torch.tensor([-1] + [r for r in range(case["drafts"]) for _ in range(L)], device="cuda")
                i = torch.arange(n, device="cuda")
                see[:, c:] = (i[None] <= i[:, None]) & ((draft[None] == draft[:, None]) | (i[None] == 0))
            else:
                see[:, c:] = torch.tril(see[:, c:])
            for h in range(Hkv):
                for r0 in range(0, n, 512):
                    r1 = min(n, r0 + 512)
                    q = s["q"][first[b] + r0:first[b] + r1, h * G:(h + 1) * G].double()
                    x = torch.einsum("igd,jd->igj", q, k[:, h]) / math.sqrt(d)
                    x = x.masked_fill(~see[r0:r1, None], float("-inf")).softmax(-1)
                    out[first[b] + r0:first[b] + r1, h * G:(h + 1) * G] = torch.einsum("igj,jd->igd", x, v[:, h])
        return out
    if case["op"] == "read":
        out = [torch.empty((s["rows"], Hkv, d), dtype=torch.float64, device="cuda") for _ in "kv"]
        for b in range(case["B"]):
            page, off = places(b, ctx[b], ctx[b] + chunk[b])
            for o, x in zip(out, "kv"):
                o[first[b]:first[b] + chunk[b]] = value64(s[x][0][page, :, off], s[x + "_exp"][0][page, :, off] if q8 else None)
        return out
    ones = torch.full(s["k"].shape[:4], 127, dtype=torch.uint8, device="cuda")
    if s["k"].numel() > 2e8:
        return None
    out = [value64(s[x], ones if q8 else None) for x in "kv"]
    if case["op"] == "keep":
        best, length = accepted(case)
        for b in range(case["B"]):
            for t in range(length[b] - 1 if best[b] >= 0 else 0):
                to = ctx[b] + 1 + t
                (p0, o0), (p1, o1) = (places(b, x, x + 1) for x in (to + best[b] * case["draft_len"], to))
                for o in out:
                    o[:, p1, :, o1] = o[:, p0, :, o0]
    else:
        for b in range(case["B"]):
            page, off = places(b, ctx[b], ctx[b] + chunk[b])
            for o, x in zip(out, ("new_k", "new_v")):
                new = s[x][first[b]:first[b] + chunk[b]].double()
                if q8:
                    e = torch.ceil(torch.log2(new.abs().amax(-1, keepdim=True).clamp(min=1e-300) / 448))
                    new = nearest64(new / torch.pow(2.0, e), 4, -9)
                o[0][page, :, off] = new
    return out + [None, None] if q8 else out
