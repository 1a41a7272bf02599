"""Speculative decoding with dense retrieval, all of its device steps together (Algorithm 1 of arxiv 2502.15572).

    python -m paper_2502_15572_b200.speculate [--quantised] [--group G] [--sequences B] [--tokens T]
                                              [--temperature T --top-p P --top-k K --samples S]

A small decoder with random weights (token mixing by the paged cache's attention; products plain library ones, or with
4-bit weights) writes some texts token by token; its hidden states and the tokens behind them become a datastore; then the
same prompts are continued with drafts.  A step of ``Speculator`` is

    retrieve_filtered      hidden state, last token -> n continuations that begin with the last token
    drafts_prepare         -> n drafts of L tokens
    reserve                pages for the step's chunk; those that sequences still share are copied
    append, attend         per layer: the chunk [last token, drafts] behind the tokens already read, under draft_mask
    drafts_accept          the longest draft that the model agrees with, and the model's own next token; or
    drafts_sample          the same for a model that draws its tokens, from given random numbers
    keep_draft             the accepted tokens' keys and values into place; the sequence counts on from them

Nothing waits for the device between these; lengths live there.  Several samples of a prompt read it once (fork); when one of
them has been chosen, the others' pages are given back and the pool is compacted.
"""
import argparse
import math

from . import binding


class Decoder:
    """Pre-norm decoder with grouped heads and rotary positions; random weights from `seed`.  group: 0 = weights in `dtype`; 32, 64
    or 128 = of 4 bits with a scale for so many inputs (all but the embeddings)."""

    def __init__(self, vocab=997, width=256, layers=2, heads=8, kv_heads=2, head_dim=64, dtype="f16", seed=0, device="cuda", group=0):
        import torch
        self.torch_dtype = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        self.dtype, self.vocab, self.width, self.layers = dtype, vocab, width, layers
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        gen = torch.Generator().manual_seed(seed)

        def new(*shape):
            w = (torch.randn(shape, generator=gen) / math.sqrt(shape[0])).to(self.torch_dtype).to(device)
            return binding.W4.quantise(w, group) if group else w

        self.embed = (torch.randn((vocab, width), generator=gen)).to(self.torch_dtype).to(device)
        self.w_qkv = [new(width, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.w_out = [new(heads * head_dim, width) for _ in range(layers)]
        self.w_up = [new(width, 2 * width) for _ in range(layers)]
        self.w_down = [new(2 * width, width) for _ in range(layers)]
        self.w_vocab = new(width, vocab)
        self.rates = (10000.0 ** (-torch.arange(0, head_dim, 2) / head_dim)).to(device)

    @staticmethod
    def product(x, w, residual=None, relu=False):
        if isinstance(w, binding.W4):
            return w.matmul(x, residual=residual, relu=relu)
        y = x @ w
        y = y.relu() if relu else y
        return y if residual is None else residual + y

    def norm(self, x):
        x = x.float()
        return (x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()).to(self.torch_dtype)

    def rotate(self, x, positions):
        """x [rows][heads][head_dim]: pairs (j, j + head_dim / 2) turned by position x rate_j."""
        import torch
        angle = (positions[:, None] * self.rates)[:, None, :]
        lo, hi = x.float().chunk(2, -1)
        return torch.cat((lo * angle.cos() - hi * angle.sin(), hi * angle.cos() + lo * angle.sin()), -1).to(self.torch_dtype)

    def forward(self, cache, batch, tokens, positions, mask=None):
        """tokens, positions [rows] of the batch's chunks -> hidden states [rows][width], logits [rows][vocab]."""
        rows, q_size, kv_size = tokens.shape[0], self.heads * self.head_dim, self.kv_heads * self.head_dim
        x = self.embed[tokens]
        for layer in range(self.layers):
            q, k, v = self.product(self.norm(x), self.w_qkv[layer]).split((q_size, kv_size, kv_size), -1)
            q = self.rotate(q.view(rows, self.heads, -1), positions)
            k = self.rotate(k.view(rows, self.kv_heads, -1), positions)
            cache.append(layer, k, v.view(rows, self.kv_heads, -1), batch)       # v: a slice of the joint projection
            mixed = cache.attend(layer, q, batch, mask=mask)
            x = self.product(mixed.view(rows, q_size), self.w_out[layer], residual=x)
            x = self.product(self.product(self.norm(x), self.w_up[layer], relu=True), self.w_down[layer], residual=x)
        hidden = self.norm(x)
        return hidden, self.product(hidden, self.w_vocab)


class Speculator:
    """Continues prompts with drafts of a datastore (or without, n = 0): a cache, its pages and the sequences' state.

    room: places behind a prompt, so texts of up to room + 1 tokens (the last one needs no place).  A sequence whose drafts are accepted may be ahead of the
    others: what ``step`` returns of it beyond its room is not part of its text.
    samples: sequences of every prompt, one after the other (sequence b * samples + s); the prompt is read once.  temperature > 0: tokens are drawn
    (top_k, top_p as in dresd_drafts_sample), the token at place p of sequence q with the random number random[q][p] that
    `seed` gives, so that a text does not depend on its drafts; 0: the largest logit, and samples are alike."""

    def __init__(self, model, prompts, room: int, store=None, n: int = 4, L: int = 8, eos_id: int = -1,
                 page_size: int = 64, quantised: bool = False, samples: int = 1, temperature: float = 0.0, top_k: int = 0,
                 top_p: float = 1.0, seed: int = 0):
        import torch
        if not prompts or not all(prompts):
            raise ValueError("every sequence needs a prompt of at least one token")
        if samples < 1:
            raise ValueError("a prompt needs a sample at least")
        device = model.embed.device
        self.model, self.store, self.n, self.L, self.eos_id = model, store, n if store else 0, L if store else 0, eos_id
        self.samples, self.B, self.chunk = samples, len(prompts) * samples, 1 + self.n * self.L
        if store:
            store.enable_first_token_filter()
        # pages for the prompt, what is to be written and one chunk behind it; full pages of the prompt are shared
        need = [-(-(len(p) + room + self.chunk) // page_size) for p in prompts]
        full = [len(p) // page_size for p in prompts]
        pages = sum(f + samples * (m - f) for m, f in zip(need, full))
        self.table = torch.full((self.B, max(need)), -1, dtype=torch.int32, device=device)
        shape = (model.layers, pages, model.kv_heads, page_size, model.head_dim)
        held = torch.uint8 if quantised else model.torch_dtype
        k, v = torch.zeros(shape, dtype=held, device=device), torch.zeros(shape, dtype=held, device=device)
        exps = [torch.zeros(shape[:4], dtype=torch.uint8, device=device) for _ in range(2)] if quantised else [None, None]
        self.cache = binding.KvCache(k, v, model.dtype, *exps)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)
        self.pages = binding.KvPages(self.cache, self.table, self.refs)
        self.missing = torch.zeros(1, dtype=torch.int32, device=device)
        self.ctx = torch.zeros(self.B, dtype=torch.int32, device=device)
        self.sampling = temperature > 0
        if self.sampling:
            new = lambda x, dtype: torch.full((self.B,), x, dtype=dtype, device=device)
            self.settings = dict(temperature=new(temperature, torch.float32), top_k=new(top_k, torch.int32), top_p=new(top_p, torch.float32))
            most = max(map(len, prompts)) + room + self.chunk + 1
            # place by place, so that they are the same whatever the room
            self.random = torch.rand((most, self.B), generator=torch.Generator().manual_seed(seed)).t().contiguous().to(device)
        # a sequence may be ahead of the others when they are done: what it writes beyond its room takes the same places again
        self.limit = torch.tensor([len(p) + room for p in prompts], dtype=torch.int32, device=device).repeat_interleave(samples)
        self.steps_left = room                                 # a step writes a token at least: then every sequence is at its limit
        self.logs = torch.zeros((self.B, 1), device=device)        # of the last tokens' probabilities, where tokens are drawn
        # places of a step's chunk: of its first token on, in the sequence
        self.offset = torch.tensor([0] + [1 + t for _ in range(self.n) for t in range(self.L)], device=device).repeat(self.B)
        self.mask = binding.draft_mask(self.n, self.L, device).repeat(self.B, 1) if self.n else None
        self.start = torch.arange(0, (self.B + 1) * self.chunk, self.chunk, dtype=torch.int32, device=device)
        self.batch = binding.KvBatch(self.table, self.ctx, self.start, rows=self.B * self.chunk, max_chunk=self.chunk)
        self.read(prompts)

    def reserve(self, batch):
        self.missing = self.missing + self.pages.reserve(batch)

    def read(self, prompts):
        """The prompts, in one piece, for the first sample of each; the others become copies of it."""
        import torch
        device, lengths, S = self.ctx.device, [len(p) for p in prompts], self.samples
        chunks = torch.tensor(lengths, dtype=torch.int32)[:, None] * (torch.arange(S) == 0)
        start = torch.cat((torch.zeros(1, dtype=torch.int32), chunks.view(-1).cumsum(0).int())).to(device)
        tokens = torch.tensor([t for p in prompts for t in p], device=device)
        positions = torch.cat([torch.arange(m) for m in lengths]).to(device)
        batch = binding.KvBatch(self.table, self.ctx, start, rows=sum(lengths), max_chunk=max(lengths))
        self.reserve(batch)
        hidden, logits = self.model.forward(self.cache, batch, tokens, positions)
        self.ctx.copy_(start[1:] - start[:-1])
        if S > 1:
            of = torch.arange(self.B, dtype=torch.int32, device=device)
            self.pages.fork(self.ctx, torch.where(of % S == 0, -1, of // S * S))
        ends = torch.tensor(lengths, device=device).cumsum(0).repeat_interleave(S) - 1
        self.hidden, logits = hidden[ends].contiguous(), logits[ends]
        if self.sampling:
            _, _, token, self.logs = binding.drafts_sample(logits[:, None], self.numbers(1, 0), **self.settings)
            self.last = token[:, 0].contiguous()
        else:
            self.last = logits.argmax(-1).int()

    def numbers(self, count, ahead):
        """Random numbers of the `count` places from the sequences' lengths + `ahead` on."""
        import torch
        at = self.ctx.long()[:, None] + ahead + torch.arange(count, device=self.ctx.device)
        return self.random.gather(1, at.clamp(max=self.random.shape[1] - 1))

    def step(self):
        """One step; returns ``(tokens [B][L + 1], length [B])``: the tokens behind the last one, -1 behind `length` of them."""
        import torch
        if self.pages is None:
            raise ValueError("the sequences have ended")
        if self.steps_left < 1:
            raise ValueError("no sequence has room for another token")
        self.steps_left -= 1
        B, n, L = self.B, self.n, self.L
        chunk, drafts, valid = self.last[:, None], None, None
        if n:
            ids, _, found = self.store.retrieve_filtered(self.hidden, self.last, n, L + 1)
            found = found[:, :, 1:].contiguous()              # the first one is the last token itself
            drafts, valid = torch.empty_like(found), torch.empty_like(ids)
            stream = binding._raw_stream(self.ctx.device.index, None)
            binding.dresd_drafts_prepare(found.data_ptr(), ids.data_ptr(), B, n, L, self.eos_id, drafts.data_ptr(),
                                         valid.data_ptr(), stream)
            chunk = torch.cat((chunk, drafts.view(B, n * L)), 1)
        tokens = chunk.reshape(-1).long().clamp_min(0)         # missing neighbours hold no token
        positions = (self.ctx.long()[:, None] + self.offset.view(B, -1)).view(-1)
        self.reserve(self.batch)
        hidden, logits = self.model.forward(self.cache, self.batch, tokens, positions, self.mask)
        hidden = hidden.view(B, self.chunk, -1)
        best, length = torch.empty_like(self.last), torch.ones_like(self.last)
        if self.sampling:
            best, length, out, self.logs = binding.drafts_sample(logits.view(B, self.chunk, -1), self.numbers(L + 1, 1), drafts, valid, **self.settings)
        else:
            out = own = logits.argmax(-1).int().view(B, -1)
            if n:
                # the model's token at draft r's place t: behind the last token (t = 0), behind the draft's token t - 1
                behind = own[:, 1:].view(B, n, L)
                llm = torch.cat((own[:, :1, None].expand(B, n, 1), behind), 2).contiguous()
                out = torch.empty((B, L + 1), dtype=torch.int32, device=own.device)
                binding.dresd_drafts_accept(drafts.data_ptr(), valid.data_ptr(), llm.data_ptr(), B, n, L, best.data_ptr(),
                                            length.data_ptr(), out.data_ptr(), stream)
        at = torch.zeros_like(self.last).long()
        if n:
            self.cache.keep_draft(self.batch, best, length, n, L)
            at = torch.where(length > 1, best * L + length - 1, 0).long()
        rows = torch.arange(B, device=out.device)
        self.hidden = hidden[rows, at].contiguous()
        self.last = out[rows, length.long() - 1]
        # the last token and what it led to, but for the new last one
        self.ctx.copy_(torch.minimum(self.ctx + length, self.limit))
        return out, length

    def run(self, count: int):
        """At least `count` tokens for every sequence, from its last one on: lists of tokens, and the steps that it took.  ``score``: the
        logarithms of their probabilities, where tokens are drawn."""
        import torch
        left = int((self.limit - self.ctx).min())
        if count > left + 1:
            raise ValueError(f"{count} tokens for sequences with room for {left + 1}")
        texts, logs, steps = [[int(t)] for t in self.last.tolist()], [row[:1] for row in self.logs.tolist()], 0
        while min(map(len, texts)) < count:
            out, length = self.step()
            steps += 1
            for text, row, m in zip(texts, out.tolist(), length.tolist()):
                text += row[:m]
            if self.sampling:
                for log, row, m in zip(logs, self.logs.tolist(), length.tolist()):
                    log += row[:m]
        self.cache.status()
        if isinstance(self.model.w_vocab, binding.W4):
            binding.dresd_w4_status(torch.cuda.current_stream().cuda_stream)
        if int(self.missing):
            raise RuntimeError(f"the pool had {int(self.missing)} pages too few")
        self.score = [sum(log[:count]) for log in logs]
        return [text[:count] for text in texts], steps

    def end(self, chosen):
        """Ends all sequences, gives back the pages of those that are not `chosen` and compacts the pool; returns the pages in use
        (the first ones).  The chosen ones' rows of `table` stay as they are read with ``cache.read``."""
        import torch
        keep = torch.zeros_like(self.ctx)
        keep[chosen] = self.ctx[chosen]
        self.pages.release(keep)
        used = int(self.pages.compact())
        self.cache.status()
        self.ctx.copy_(keep)
        self.pages = None
        return used


def make_datastore(model, texts, stored_len: int):
    """Keys: unit hidden states of every place of the texts; values: the `stored_len` tokens that follow."""
    import torch
    device = model.embed.device
    lengths = [len(t) for t in texts]
    pages = [-(-m // 64) for m in lengths]
    table = torch.full((len(texts), max(pages)), -1, dtype=torch.int32)
    for b, m in enumerate(pages):
        table[b, :m] = torch.arange(m) + sum(pages[:b])
    shape = (model.layers, sum(pages), model.kv_heads, 64, model.head_dim)
    cache = binding.KvCache(*(torch.zeros(shape, dtype=model.torch_dtype, device=device) for _ in range(2)), model.dtype)
    start = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).int().to(device)
    batch = binding.KvBatch(table.to(device), torch.zeros(len(texts), dtype=torch.int32, device=device), start,
                            rows=sum(lengths), max_chunk=max(lengths))
    tokens = torch.tensor([t for text in texts for t in text], device=device)
    positions = torch.cat([torch.arange(m) for m in lengths]).to(device)
    hidden, _ = model.forward(cache, batch, tokens, positions)
    cache.status()
    keep, following, at = [], [], 0
    for text in texts:
        for i in range(len(text) - stored_len):
            keep.append(at + i)
            following.append(text[i + 1:i + 1 + stored_len])
        at += len(text)
    keys = torch.nn.functional.normalize(hidden[keep].float(), dim=-1).to(model.torch_dtype).contiguous()
    return binding.Store(keys, torch.tensor(following, dtype=torch.int32, device=device), model.dtype)


def main(argv=None):
    import torch
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--quantised", action="store_true", help="hold the cache in 8 bits")
    p.add_argument("--sequences", type=int, default=4)
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--drafts", type=int, default=4)
    p.add_argument("--draft-len", type=int, default=8)
    p.add_argument("--group", type=int, default=0, help="4-bit weights with a scale for so many inputs (32, 64, 128)")
    p.add_argument("--temperature", type=float, default=0.0, help="draw tokens")
    p.add_argument("--top-k", type=int, default=0)
    p.add_argument("--top-p", type=float, default=1.0)
    p.add_argument("--samples", type=int, default=1, help="texts of every prompt")
    a = p.parse_args(argv)
    model = Decoder(group=a.group)
    how = dict(quantised=a.quantised, temperature=a.temperature, top_k=a.top_k, top_p=a.top_p, samples=a.samples)
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(model.vocab, (20 + 7 * b,), generator=gen).tolist() for b in range(a.sequences)]
    plain, steps = Speculator(model, prompts, a.tokens + 1, **how).run(a.tokens)
    store = make_datastore(model, [prompts[i // a.samples] + y for i, y in enumerate(plain)], a.draft_len + 1)
    room = a.tokens + a.draft_len + 1
    spec = Speculator(model, prompts, room, store, a.drafts, a.draft_len, **how)
    drafted, fewer = spec.run(a.tokens)
    store.status()
    same = sum(x == y for t, u in zip(plain, drafted) for x, y in zip(t, u)) / (len(plain) * a.tokens)
    print(f"{len(plain)} sequences of {a.tokens} tokens: {steps} steps token by token, {fewer} with {a.drafts} drafts of "
          f"{a.draft_len}; {100 * same:.1f}% of the tokens alike")
    if a.samples > 1:
        held = int((spec.refs > 0).sum())
        likely = [max(range(b, b + a.samples), key=spec.score.__getitem__) for b in range(0, spec.B, a.samples)]
        used = spec.end(torch.tensor(likely, device=spec.ctx.device))
        print(f"the likeliest of {a.samples} samples kept: {held} pages in use before, {used} now")


if __name__ == "__main__":
    main()
