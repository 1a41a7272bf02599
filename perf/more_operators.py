"""What the operators of a sampled decoding step are measured on.

The language model that verifies retrieved drafts draws its tokens from a distribution, writes several continuations of one
prompt, and is bound by its weights.  Three operators serve it:

`sample`   verification of drafts against the model's probabilities from given random numbers (none: plain sampling).
           Sequence b has a row of logits behind its last token and one behind every draft token, as the verification
           chunk lies: row 0, and row 1 + r L + t behind token t of draft r.  At depth t one token is drawn, with the random
           number u[b][t], from the row behind the best-ranked draft that agrees with all that was drawn so far; the
           sequence ends where no draft agrees any more.  A row's distribution: temperature, then the top_k largest
           logits, then the shortest prefix of these (by logit, then by index) that holds top_p of their weight.
           Weights are whole multiples of 2^-42 of the largest, so that sums do not depend on their order; the token is
           the first one, by index, whose running sum exceeds u times the sum.
`pages`    pages of the paged key/value cache, counted in refs[page] = rows of the table that hold it.  "fork": rows
           become copies of other rows and share their pages, the places of the next chunk are made their own (absent pages
           are taken, shared ones with tokens in them copied), and all of that is given back.  "compact": the used pages
           move to the lowest page numbers.
`product`  x W^T with weights of 4 bits, one scale for a group of inputs: y[t][o] = sum_i s[o][i / group] (c[o][i] - 8) x[t][i],
           two codes a byte, the even input in the low half; with the residual added where there is one.
"""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ONE = 2.0 ** 42                      # the largest weight of a row


def listed():
    return [
        # one token of one sequence, nucleus sampling: latency
        dict(name="sample 1 of 32000", op="sample", B=1, n=0, L=0, V=32000, dtype="f16", temperature=0.7, top_k=0, top_p=0.95, agree=0.0),
        # ten drafts of ten tokens for one sequence
        dict(name="verify 10 x 10 of 32000", op="sample", B=1, n=10, L=10, V=32000, dtype="f16", temperature=0.7, top_k=0, top_p=0.95, agree=0.6),
        # three drafts of twenty tokens for sixteen sequences, a large vocabulary of odd size
        dict(name="verify 16 of 3 x 20 of 100003", op="sample", B=16, n=3, L=20, V=100003, dtype="bf16", temperature=1.0, top_k=0, top_p=1.0, agree=0.6),
        # a serving batch without drafts, its logits in 32 bits, the forty best
        dict(name="sample 64 of 151001 f32", op="sample", B=64, n=0, L=0, V=151001, dtype="f32", temperature=0.9, top_k=40, top_p=0.9, agree=0.0),
        # eight continuations of one prompt: the last, partly filled page is copied for each
        dict(name="fork 1 to 8", op="fork", prompts=1, copies=8, tokens=1999, chunk=1, layers=32, heads=8, d=128, page=16, dtype="f16",
             quantised=False, spare=40),
        # twenty-four prompts, three continuations each with room for a chunk of drafts, an 8-bit cache
        dict(name="fork 24 to 72 e4m3", op="fork", prompts=24, copies=3, tokens=1501, chunk=61, layers=16, heads=8, d=128, page=64, dtype="bf16",
             quantised=True, spare=300),
        # a small pool after some sequences have gone
        dict(name="compact 700 pages", op="compact", pages=700, used=0.4, rows=9, layers=16, heads=4, d=128, page=16, dtype="f16", quantised=False),
        # a large pool of which a third is in use
        dict(name="compact 2500 pages", op="compact", pages=2500, used=0.35, rows=40, layers=4, heads=8, d=128, page=64, dtype="bf16", quantised=False),
        # one token through a square projection: latency
        dict(name="product 1 x 4096 x 4096", op="product", rows=1, inputs=4096, outputs=4096, group=128, dtype="f16", residual=False),
        # a few sequences' tokens through a wide layer
        dict(name="product 7 x 4096 x 11008", op="product", rows=7, inputs=4096, outputs=11008, group=64, dtype="bf16", residual=False),
        # the chunk of a verification step through the layer that leads back, onto the residual stream
        dict(name="product 101 x 11008 x 4096", op="product", rows=101, inputs=11008, outputs=4096, group=128, dtype="f16", residual=True),
        # a piece of a prompt
        dict(name="product 2047 x 4096 x 11008", op="product", rows=2047, inputs=4096, outputs=11008, group=128, dtype="bf16", residual=False),
    ]


def spread(rng, lo, hi):
    """A whole number in lo .. hi, spread over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "fork", "compact", "product", "product"])
    if op == "sample":
        V = spread(rng, 500, 151001)
        n = rng.choice([0, 0, rng.randint(1, 12)])
        L = rng.randint(1, 60 // n) if n else 0
        # rows that are held, and rows that are walked through, stay within those of the largest listed case
        most = min(64, int(9.7e7 / ((1 + n * L) * V)), int(9.6e6 / V) if n == 0 else 64)
        return dict(op=op, B=spread(rng, 1, max(1, most)), n=n, L=L, V=V, dtype=rng.choice(["f16", "bf16", "f32"]),
                    temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 1.3]), top_k=rng.choice([0, 0, 1, rng.randint(2, 200)]),
                    top_p=rng.choice([1.0, 1.0, 0.95, round(rng.uniform(0.3, 0.99), 2)]), agree=round(rng.uniform(0.2, 0.8), 1) if n else 0.0)
    if op == "product":
        group = rng.choice([32, 64, 128])
        inputs = group * spread(rng, 2, 11008 // group)
        rows, outputs = spread(rng, 1, 2047), spread(rng, 7, 11008)
        rows = max(1, min(rows, int(9.2e10 / (inputs * outputs))))
        return dict(op=op, rows=rows, inputs=inputs, outputs=outputs, group=group, dtype=rng.choice(["f16", "bf16"]), residual=rng.random() < 0.4)
    geometry = dict(layers=spread(rng, 1, 32), heads=rng.choice([1, 2, 4, 8, 10]), d=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
                    dtype=rng.choice(["f16", "bf16"]), quantised=rng.random() < 0.5)
    # bytes of one page in all layers, keys and values
    each = geometry["layers"] * 2 * geometry["heads"] * geometry["page"] * geometry["d"] * (1 if geometry["quantised"] else 2)
    if op == "fork":
        prompts, copies = spread(rng, 1, 24), spread(rng, 1, 12)
        prompts = max(1, min(prompts, int(1.5e8 / (copies * each))))
        tokens, chunk = spread(rng, 1, 1999), spread(rng, 1, 130)
        held = prompts * (tokens // geometry["page"] + 1) + prompts * copies * (chunk // geometry["page"] + 2)
        while held * each > 2.5e9 and tokens > 1:
            tokens //= 2
            held = prompts * (tokens // geometry["page"] + 1) + prompts * copies * (chunk // geometry["page"] + 2)
        return dict(op=op, prompts=prompts, copies=copies, tokens=tokens, chunk=chunk, spare=rng.randint(0, 50), **geometry)
    pages = max(8, min(spread(rng, 20, 2500), int(2.5e9 / each)))
    return dict(op=op, pages=pages, used=round(rng.uniform(0.1, 0.9), 2), rows=rng.randint(1, 40), **geometry)


# ---- inputs --------------------------------------------------------------------------------------------------------
def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    op = case["op"]
    s = prepare_sample(case, seed) if op == "sample" else prepare_product(case, seed) if op == "product" else prepare_pages(case, seed)
    s["case"] = case
    return s


def prepare_sample(case, seed):
    g = generator(seed)
    B, n, L, V = case["B"], case["n"], case["L"], case["V"]
    rows = 1 + n * L
    # most of the mass on a few tokens, a long tail behind
    logits = torch.randn((B, rows, V), device="cuda", generator=g).mul_(2.0)
    s = dict(uniform=torch.rand((B, L + 1), device="cuda", generator=g), drafts=None, valid=None)
    if n:
        drafts = torch.randint(V, (B, n, L), device="cuda", generator=g, dtype=torch.int32)
        # neighbours of one state begin alike: draft r follows draft 0 for a while
        alike = torch.randint(L + 1, (B, n, 1), device="cuda", generator=g)
        drafts = torch.where(torch.arange(L, device="cuda") < alike, drafts[:, :1], drafts)
        valid = (torch.rand((B, n), device="cuda", generator=g) < 0.9).to(torch.int32)
        # the row behind a prefix favours the token that the draft goes on with, so that it is drawn about every `agree`-th time
        t = case["temperature"] or 1.0
        height = t * (math.log(V) + 2.0 / t ** 2 + math.log(case["agree"] / (1 - case["agree"])))
        after = torch.cat((drafts[:, 0, :1], torch.cat((drafts[:, :, 1:], drafts[:, :, :1]), 2).reshape(B, n * L)), 1).long()
        logits.scatter_(2, after[:, :, None], height)
        # equal prefixes have equal rows
        same = (drafts[:, :, None] == drafts[:, None]).long().cumprod(-1)               # [B][n][n][L]: r and r' alike up to place t
        first = same.argmax(2)                                                          # the first draft that begins alike
        row = torch.cat((torch.zeros((B, 1), dtype=torch.long, device="cuda"), (1 + first * L + torch.arange(L, device="cuda")).reshape(B, n * L)), 1)
        logits = logits[torch.arange(B, device="cuda")[:, None], row]
        s.update(drafts=drafts, valid=valid)
    s["logits"] = logits.to(DTYPES[case["dtype"]])
    s["temperature"] = torch.full((B,), case["temperature"], device="cuda")
    s["top_k"] = torch.full((B,), case["top_k"], device="cuda", dtype=torch.int32)
    s["top_p"] = torch.full((B,), case["top_p"], device="cuda")
    return s


def prepare_product(case, seed):
    g = generator(seed)
    dtype, o, i = DTYPES[case["dtype"]], case["outputs"], case["inputs"]
    s = dict(x=torch.randn((case["rows"], i), device="cuda", generator=g).to(dtype), residual=None)
    # codes as rounded normal numbers have them
    s["codes"] = (torch.randn((o, i // 2, 2), device="cuda", generator=g) * 2.6 + 8).round_().clamp_(0, 15).to(torch.uint8)
    s["codes"] = s["codes"][..., 0] | s["codes"][..., 1] << 4
    s["scales"] = ((0.5 + torch.rand((o, i // case["group"]), device="cuda", generator=g)) * (0.4 / math.sqrt(i))).to(dtype)
    if case["residual"]:
        s["residual"] = torch.randn((case["rows"], o), device="cuda", generator=g).to(dtype)
    if own:
        from paper_2502_15572_b200 import binding
        s["w"] = binding.W4(s["codes"], s["scales"], case["dtype"])
    return s


def prepare_pages(case, seed):
    g = generator(seed)
    page, fork = case["page"], case["op"] == "fork"
    rng = random.Random(1000 * case["layers"] + page)          # the geometry is the case's alone
    if fork:
        full = [max(1, case["tokens"] - rng.randint(0, case["tokens"] // 3)) for _ in range(case["prompts"])]
        own_pages = [-(-m // page) for m in full]
        children = case["prompts"] * case["copies"]
        places = (case["tokens"] + case["chunk"]) // page + 2
        pages = sum(own_pages) + children * (case["chunk"] // page + 2) + case["spare"]
        rows = case["prompts"] + children
    else:
        pages, rows = case["pages"], case["rows"]
        held = max(1, int(pages * case["used"]))
        cuts = sorted(rng.randint(0, held) for _ in range(rows - 1))
        own_pages = [b - a for a, b in zip([0] + cuts, cuts + [held])]
        places = max(own_pages) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((rows, places), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(own_pages):
        table[b, :m] = order[at:at + m]
        at += m
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order[:at].long()] = 1
    shape = (case["layers"], pages, case["heads"], page, case["d"])
    s = dict(table=table, refs=refs, k_exp=None, v_exp=None)
    for name in ("k", "v"):
        if case["quantised"]:
            s[name] = torch.randint(0, 127, shape, dtype=torch.uint8, device="cuda", generator=g)
            s[name + "_exp"] = torch.randint(119, 130, shape[:4], dtype=torch.uint8, device="cuda", generator=g)
        else:
            s[name] = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=g)
    if fork:
        s["ctx"] = torch.tensor(full + [0] * children, dtype=torch.int32, device="cuda")
        s["parent"] = torch.tensor([-1] * case["prompts"] + [c // case["copies"] for c in range(children)], dtype=torch.int32, device="cuda")
        # the prompts' own rows stand still, their copies go on
        s["start"] = torch.tensor([0] * case["prompts"] + [case["chunk"] * c for c in range(children + 1)], dtype=torch.int32, device="cuda")
        s["keep"] = torch.tensor(full + [0] * children, dtype=torch.int32, device="cuda")
    else:
        s["table_before"], s["refs_before"] = table.clone(), refs.clone()
    if own:
        from paper_2502_15572_b200 import binding
        cache = binding.KvCache(s["k"], s["v"], case["dtype"], k_exps=s["k_exp"], v_exps=s["v_exp"])
        s["pages"] = binding.KvPages(cache, table, refs)
        if fork:
            s["batch"] = binding.KvBatch(table, s["ctx"], s["start"], rows=children * case["chunk"], max_chunk=case["chunk"])
    return s


def contents(s):
    """The cache as values: 8-bit codes as E4M3 numbers beside their exponent bytes."""
    if s["case"]["quantised"]:
        return [s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["k_exp"], s["v_exp"]]
    return [s["k"], s["v"]]


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if op == "sample":
        if own:
            from paper_2502_15572_b200 import binding
            return list(binding.drafts_sample(s["logits"], s["uniform"], s["drafts"], s["valid"], temperature=s["temperature"],
                                              top_k=s["top_k"], top_p=s["top_p"]))
        return plain_sample(s)
    if op == "product":
        if own:
            return s["w"].matmul(s["x"], residual=s["residual"])
        return plain_product(s)
    if op == "fork":
        if own:
            pages = s["pages"]
            pages.fork(s["ctx"], s["parent"])
            missing = pages.reserve(s["batch"])
            between = s["table"].clone()                       # what the steps until the release work with
            pages.release(s["keep"])
        else:
            plain_fork(s)
            missing = plain_reserve(s)
            between = s["table"].clone()
            plain_release(s)
        return contents(s) + [between, missing, s["table"], s["refs"], s["ctx"]]
    s["table"].copy_(s["table_before"])                        # the same sequences are there again
    s["refs"].copy_(s["refs_before"])
    used = s["pages"].compact() if own else plain_compact(s)
    return contents(s) + [s["table"], s["refs"], used]


# ---- the plain forms -----------------------------------------------------------------------------------------------
def ordered(x):
    """Logits as numbers whose order is total: NaN below everything."""
    x = x.double()
    return torch.where(x.isnan(), torch.full_like(x, -math.inf), x)


def plain_rows(x, u, temperature, top_k, top_p):
    """Tokens and logarithms of their probabilities for rows [N][V], each with its own random number and settings."""
    x = ordered(x)
    N, V = x.shape
    top = x.amax(-1, keepdim=True)
    greedy = ~(temperature > 0)
    t = torch.where(greedy, torch.ones_like(temperature), temperature).double()[:, None]
    below = torch.where(x == top, torch.zeros_like(x), (x - top) / t)
    w = torch.where(x > -math.inf, below.exp().mul_(ONE).round_(), torch.zeros_like(x)).long()
    w = torch.where(greedy[:, None], torch.where(x == top, w, torch.zeros_like(w)), w)
    top_k = torch.where(greedy, torch.ones_like(top_k), torch.where(top_k > 0, top_k, torch.full_like(top_k, V)))
    by = torch.sort(x, dim=-1, descending=True, stable=True).indices
    w_by = w.gather(1, by)
    w_by = torch.where(torch.arange(V, device=x.device) < top_k[:, None], w_by, torch.zeros_like(w_by))
    total = w_by.sum(-1)
    target = (top_p.double() * total.double()).ceil().long()
    off = ~(top_p < 1)
    before = w_by.cumsum(-1) - w_by
    keep = off[:, None] | (before < target[:, None])
    keep[:, 0] = True
    w_by = torch.where(keep, w_by, torch.zeros_like(w_by))
    kept = torch.zeros_like(w).scatter_(1, by, w_by)
    total = kept.sum(-1)
    aim = (u.clamp(0, 1 - 2.0 ** -24).double() * total.double()).long()
    y = (kept.cumsum(-1) > aim[:, None]).to(torch.int8).argmax(-1)
    y = torch.where(total > 0, y, torch.full_like(y, -1))
    log = below.gather(1, y.clamp(min=0)[:, None])[:, 0] - (total.double() / ONE).log()
    return y.to(torch.int32), torch.where(total > 0, log, torch.zeros_like(log)).float()


def plain_sample(s):
    """Every row is drawn from, then the drafts are followed: all drafts that begin alike take the row of the first."""
    B, n, L = s["case"]["B"], s["case"]["n"], s["case"]["L"]
    rows = 1 + n * L
    depth = torch.cat((torch.zeros(1, dtype=torch.long), torch.arange(1, L + 1).repeat(n))).cuda()
    u = s["uniform"][:, depth].reshape(-1)
    per = [x[:, None].expand(B, rows).reshape(-1) for x in (s["temperature"], s["top_k"], s["top_p"])]
    y, log = (x.view(B, rows) for x in plain_rows(s["logits"].reshape(B * rows, -1), u, *per))
    if n == 0:
        return [torch.full((B,), -1, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda"), y, log]
    drafts, valid = s["drafts"], s["valid"] != 0
    same = (drafts[:, :, None] == drafts[:, None]).long().cumprod(-1) * valid[:, None, :, None]
    first = same.argmax(2)                                                               # [B][n][L]
    row = torch.cat((torch.zeros((B, n, 1), dtype=torch.long, device="cuda"), 1 + first * L + torch.arange(L, device="cuda")), 2)
    drawn = y.gather(1, row.view(B, -1)).view(B, n, L + 1)
    matched = (drafts == drawn[:, :, :L]).long().cumprod(-1).sum(-1)
    matched = torch.where(valid, matched, torch.full_like(matched, -1))
    length, best = matched.amax(1), matched.argmax(1)
    at = row.gather(1, best[:, None, None].expand(B, 1, L + 1))[:, 0]
    inside = torch.arange(L + 1, device="cuda") <= length.clamp(min=0)[:, None]
    tokens = torch.where(inside, y.gather(1, at), torch.full_like(at, -1, dtype=torch.int32))
    logs = torch.where(inside, log.gather(1, at), torch.zeros_like(at, dtype=torch.float32))
    best = torch.where(length >= 0, best, torch.full_like(best, -1))
    return [best.to(torch.int32), (length.clamp(min=0) + 1).to(torch.int32), tokens, logs]


def plain_product(s):
    case = s["case"]
    codes = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).view(case["outputs"], -1, case["group"])
    w = (codes.float() - 8).mul_(s["scales"].float()[..., None]).view(case["outputs"], -1)
    y = s["x"].float() @ w.t()
    if s["residual"] is not None:
        y += s["residual"].float()
    return y.to(s["x"].dtype)


def plain_fork(s):
    table, refs, ctx, parent = s["table"], s["refs"], s["ctx"], s["parent"].long()
    p = parent.clamp(min=0)
    fork = (parent >= 0) & (parent[p] < 0)
    new = torch.where(torch.arange(table.shape[1], device="cuda") < ((ctx + s["case"]["page"] - 1) // s["case"]["page"])[p, None],
                      table[p], torch.full_like(table, -1))
    shared = new[fork]
    refs.index_add_(0, shared[shared >= 0].long(), torch.ones_like(shared[shared >= 0]))
    table.copy_(torch.where(fork[:, None], new, table))
    ctx.copy_(torch.where(fork, ctx[p], ctx))


def plain_reserve(s):
    """Wanted places in order of rows and places; one that is shared still after the earlier ones have left it is copied."""
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    ctx, length = s["ctx"].long(), (s["start"][1:] - s["start"][:-1]).long()
    place = torch.arange(table.shape[1], device="cuda")
    wanted = (length > 0)[:, None] & (place >= (ctx // page)[:, None]) & (place <= ((ctx + length - 1) // page)[:, None])
    beyond = torch.where(length > 0, (ctx + length - 1) // page + 1 - table.shape[1], torch.zeros_like(ctx)).clamp(min=0)
    b, i = wanted.nonzero(as_tuple=True)
    old = table[b, i].long()
    by = torch.sort(old, stable=True).indices                  # wishes for one page side by side, in their order
    run = old[by]
    rank = torch.arange(len(by), device="cuda") - torch.searchsorted(run, run)
    earlier = torch.empty_like(rank).scatter_(0, by, rank)
    absent = old < 0
    take = absent | (refs[old.clamp(min=0)] - earlier > 1)
    b, i, old, absent = b[take], i[take], old[take], absent[take]
    free = (refs == 0).nonzero()[:, 0]
    missing = (beyond.sum() + (len(b) - len(free)) * (len(b) > len(free))).to(torch.int32).view(1)
    if int(missing):
        return missing
    new = free[:len(b)]
    filled = ~absent & (i * page < ctx[b])
    src, dst = old[filled], new[filled]
    for name in ("k", "v", "k_exp", "v_exp"):
        if s[name] is not None:
            s[name][:, dst] = s[name][:, src]
    refs.index_add_(0, old[~absent], torch.full_like(old[~absent], -1, dtype=torch.int32))
    refs[new] = 1
    table[b, i] = new.to(torch.int32)
    return missing


def plain_release(s):
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    gone = (torch.arange(table.shape[1], device="cuda") >= ((s["keep"] + page - 1) // page)[:, None]) & (table >= 0)
    left = table[gone].long()
    refs.index_add_(0, left, torch.full_like(left, -1, dtype=torch.int32))
    table.masked_fill_(gone, -1)


def plain_compact(s):
    table, refs = s["table"], s["refs"]
    used = refs > 0
    count = used.sum()
    number = torch.arange(len(refs), device="cuda")
    src, dst = (used & (number >= count)).nonzero()[:, 0], (~used & (number < count)).nonzero()[:, 0]
    for name in ("k", "v", "k_exp", "v_exp"):
        if s[name] is not None:
            s[name][:, dst] = s[name][:, src]
    to = number.to(torch.int32)
    to[src] = dst.to(torch.int32)
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))
    refs[dst] = refs[src]
    refs[src] = 0
    return count.to(torch.int32).view(1)


# ---- what cannot be done without -----------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "sample":
        size = 4 if case["dtype"] == "f32" else 2
        walked = sum(case["agree"] ** t for t in range(case["L"] + 1))       # rows on the path of a sequence, on the average
        return {"bytes": int(case["B"] * (walked * case["V"] * size + 8 * case["L"] + 24)), "flops": 0}
    if op == "product":
        t, i, o = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": o * i // 2 + 2 * o * (i // case["group"]) + 2 * t * i + 2 * t * o * (2 if case["residual"] else 1), "flops": 2 * t * i * o}
    each = case["layers"] * 2 * case["heads"] * case["page"] * (case["d"] + 1 if case["quantised"] else 2 * case["d"])
    if op == "fork":
        rng = random.Random(1000 * case["layers"] + case["page"])
        full = [max(1, case["tokens"] - rng.randint(0, case["tokens"] // 3)) for _ in range(case["prompts"])]
        moved = sum(case["copies"] for m in full if m % case["page"])
    else:
        held = max(1, int(case["pages"] * case["used"]))
        moved = held * (case["pages"] - held) // case["pages"]               # used pages above `held`, on the average
    return {"bytes": max(1, 2 * moved * each), "flops": 0}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        c = s["codes"].to(torch.int16)
        y = torch.zeros((case["rows"], case["outputs"]), dtype=torch.float64, device="cuda")
        for half in range(2):                                  # the even inputs, then the odd ones
            w = ((c >> (4 * half)) % 16 - 8).double() * s["scales"].double().repeat_interleave(case["group"] // 2, 1)
            y += s["x"].double()[:, half::2] @ w.T
        return y if s["residual"] is None else y + s["residual"].double()
    if op == "sample":
        return exact_sample(case, s)
    return None


def exact_sample(case, s):
    """One sequence after the other, one depth after the other; the distribution by sorting and by sums of real numbers."""
    B, n, L, T = case["B"], case["n"], case["L"], case["temperature"]
    best, length = torch.full((B,), -1, dtype=torch.int32), torch.ones(B, dtype=torch.int32)
    tokens, logs = torch.full((B, L + 1), -1, dtype=torch.int32), torch.zeros((B, L + 1), dtype=torch.float64)
    drafts = s["drafts"].tolist() if n else [[]] * B
    valid = s["valid"].tolist() if n else [[]] * B
    for b in range(B):
        live = [r for r in range(n) if valid[b][r]]
        for t in range(L + 1):
            x = s["logits"][b, 0 if t == 0 else 1 + live[0] * L + t - 1].double()
            if T == 0:
                y, log = int((x == x.max()).nonzero()[0]), 0.0
            else:
                value, index = torch.sort(x, dim=0, descending=True, stable=True)
                p = torch.exp((value - value[0]) / s["temperature"][b].double())
                if case["top_k"]:
                    p = p[:case["top_k"]]
                p = p / p.sum()
                if case["top_p"] < 1:
                    p = p[:1 + int((p.cumsum(0) < s["top_p"][b].double()).sum())]
                    p = p / p.sum()
                index, order = index[:len(p)].sort()
                run = p[order].cumsum(0)
                at = min(int((run <= s["uniform"][b, t].double() * run[-1]).sum()), len(run) - 1)
                y, log = int(index[at]), math.log(float(p[order][at]))
            tokens[b, t], logs[b, t] = y, log
            length[b] = t + 1
            if live:
                best[b] = live[0]
            live = [r for r in live if t < L and drafts[b][r][t] == y]
            if not live:
                break
    return [best.cuda(), length.cuda(), tokens.cuda(), logs.cuda()]
