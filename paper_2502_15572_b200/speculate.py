"""Speculative decoding with dense retrieval, all of its device steps together (Algorithm 1 of arxiv 2502.15572).

    python -m paper_2502_15572_b200.speculate [--quantised] [--sequences B] [--tokens T]

A small decoder with random weights (token mixing by the paged cache's attention, everything else plain library
products) writes some texts token by token; its hidden states and the tokens behind them become a datastore; then the
same prompts are continued with drafts.  A step of ``Speculator`` is

    retrieve_filtered      hidden state, last token -> n continuations that begin with the last token
    drafts_prepare         -> n drafts of L tokens
    append, attend         per layer: the chunk [last token, drafts] behind the tokens already read, under draft_mask
    drafts_accept          the longest draft that the model agrees with, and the model's own next token
    keep_draft             the accepted tokens' keys and values into place; the sequence counts on from them

Nothing waits for the device between these; lengths live there.
"""
import argparse
import math

from . import binding


class Decoder:
    """Pre-norm decoder with grouped heads and rotary positions; random weights from `seed`."""

    def __init__(self, vocab=997, width=256, layers=2, heads=8, kv_heads=2, head_dim=64, dtype="f16", seed=0, device="cuda"):
        import torch
        self.torch_dtype = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        self.dtype, self.vocab, self.width, self.layers = dtype, vocab, width, layers
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        gen = torch.Generator().manual_seed(seed)
        new = lambda *shape: (torch.randn(shape, generator=gen) / math.sqrt(shape[0])).to(self.torch_dtype).to(device)
        self.embed = (torch.randn((vocab, width), generator=gen)).to(self.torch_dtype).to(device)
        self.w_qkv = [new(width, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.w_out = [new(heads * head_dim, width) for _ in range(layers)]
        self.w_up = [new(width, 2 * width) for _ in range(layers)]
        self.w_down = [new(2 * width, width) for _ in range(layers)]
        self.w_vocab = new(width, vocab)
        self.rates = (10000.0 ** (-torch.arange(0, head_dim, 2) / head_dim)).to(device)

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
            q, k, v = (self.norm(x) @ self.w_qkv[layer]).split((q_size, kv_size, kv_size), -1)
            q = self.rotate(q.view(rows, self.heads, -1), positions)
            k = self.rotate(k.view(rows, self.kv_heads, -1), positions)
            cache.append(layer, k, v.view(rows, self.kv_heads, -1), batch)       # v: a slice of the joint projection
            mixed = cache.attend(layer, q, batch, mask=mask)
            x = x + mixed.view(rows, q_size) @ self.w_out[layer]
            x = x + (self.norm(x) @ self.w_up[layer]).relu() @ self.w_down[layer]
        hidden = self.norm(x)
        return hidden, hidden @ self.w_vocab


class Speculator:
    """Continues `B` prompts with drafts of a datastore (or without, n = 0): a cache, its pages and the sequences' state."""

    def __init__(self, model, prompts, room: int, store=None, n: int = 4, L: int = 8, eos_id: int = -1,
                 page_size: int = 64, quantised: bool = False):
        import torch
        if not prompts or not all(prompts):
            raise ValueError("every sequence needs a prompt of at least one token")
        device = model.embed.device
        self.model, self.store, self.n, self.L, self.eos_id = model, store, n if store else 0, L if store else 0, eos_id
        self.B, self.chunk = len(prompts), 1 + self.n * self.L
        if store:
            store.enable_first_token_filter()
        # pages for the prompt, what is to be written and one chunk behind it
        need = [-(-(len(p) + room + self.chunk) // page_size) for p in prompts]
        table = torch.full((self.B, max(need)), -1, dtype=torch.int32)
        order, at = torch.randperm(sum(need), generator=torch.Generator().manual_seed(0)).int(), 0
        for b, m in enumerate(need):
            table[b, :m] = order[at:at + m]
            at += m
        self.table = table.to(device)
        shape = (model.layers, at, model.kv_heads, page_size, model.head_dim)
        held = torch.uint8 if quantised else model.torch_dtype
        k, v = torch.zeros(shape, dtype=held, device=device), torch.zeros(shape, dtype=held, device=device)
        exps = [torch.zeros(shape[:4], dtype=torch.uint8, device=device) for _ in range(2)] if quantised else [None, None]
        self.cache = binding.KvCache(k, v, model.dtype, *exps)
        self.ctx = torch.zeros(self.B, dtype=torch.int32, device=device)
        # places of a step's chunk: of its first token on, in the sequence
        self.offset = torch.tensor([0] + [1 + t for _ in range(self.n) for t in range(self.L)], device=device).repeat(self.B)
        self.mask = binding.draft_mask(self.n, self.L, device).repeat(self.B, 1) if self.n else None
        self.start = torch.arange(0, (self.B + 1) * self.chunk, self.chunk, dtype=torch.int32, device=device)
        self.batch = binding.KvBatch(self.table, self.ctx, self.start, rows=self.B * self.chunk, max_chunk=self.chunk)
        self.read(prompts)

    def read(self, prompts):
        """The prompts, in one piece."""
        import torch
        device, lengths = self.ctx.device, [len(p) for p in prompts]
        start = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).int().to(device)
        tokens = torch.tensor([t for p in prompts for t in p], device=device)
        positions = torch.cat([torch.arange(m) for m in lengths]).to(device)
        batch = binding.KvBatch(self.table, self.ctx, start, rows=sum(lengths), max_chunk=max(lengths))
        hidden, logits = self.model.forward(self.cache, batch, tokens, positions)
        ends = start[1:].long() - 1
        self.hidden, self.last = hidden[ends].contiguous(), logits[ends].argmax(-1).int()
        self.ctx.copy_(start[1:] - start[:-1])

    def step(self):
        """One step; returns ``(tokens [B][L + 1], length [B])``: the tokens behind the last one, -1 behind `length` of them."""
        import torch
        B, n, L = self.B, self.n, self.L
        chunk = self.last[:, None]
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
        hidden, logits = self.model.forward(self.cache, self.batch, tokens, positions, self.mask)
        own, hidden = logits.argmax(-1).int().view(B, -1), hidden.view(B, self.chunk, -1)
        if n:
            # the model's token at draft r's place t: behind the last token (t = 0), behind the draft's token t - 1
            behind = own[:, 1:].view(B, n, L)
            llm = torch.cat((own[:, :1, None].expand(B, n, 1), behind), 2).contiguous()
            best, length = torch.empty_like(self.last), torch.empty_like(self.last)
            out = torch.empty((B, L + 1), dtype=torch.int32, device=own.device)
            binding.dresd_drafts_accept(drafts.data_ptr(), valid.data_ptr(), llm.data_ptr(), B, n, L, best.data_ptr(),
                                        length.data_ptr(), out.data_ptr(), stream)
            self.cache.keep_draft(self.batch, best, length, n, L)
            at = torch.where(length > 1, best * L + length - 1, 0).long()
        else:
            out, length, at = own, torch.ones_like(self.last), torch.zeros_like(self.last).long()
        rows = torch.arange(B, device=own.device)
        self.hidden = hidden[rows, at].contiguous()
        self.last = out[rows, length.long() - 1]
        self.ctx += length                                     # the last token and what it led to, but for the new last one
        return out, length

    def run(self, count: int):
        """At least `count` tokens for every sequence: lists of tokens, and the steps that it took."""
        texts, steps = [[int(t)] for t in self.last.tolist()], 0
        while min(map(len, texts)) < count:
            out, length = self.step()
            steps += 1
            for text, row, m in zip(texts, out.tolist(), length.tolist()):
                text += row[:m]
        self.cache.status()
        return [text[:count] for text in texts], steps


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
    a = p.parse_args(argv)
    model = Decoder()
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(model.vocab, (20 + 7 * b,), generator=gen).tolist() for b in range(a.sequences)]
    plain, steps = Speculator(model, prompts, a.tokens + 1, quantised=a.quantised).run(a.tokens)
    store = make_datastore(model, [x + y for x, y in zip(prompts, plain)], a.draft_len + 1)
    room = a.tokens + a.draft_len + 1
    drafted, fewer = Speculator(model, prompts, room, store, a.drafts, a.draft_len, quantised=a.quantised).run(a.tokens)
    store.status()
    same = sum(x == y for t, u in zip(plain, drafted) for x, y in zip(t, u)) / (a.sequences * a.tokens)
    print(f"{a.sequences} sequences of {a.tokens} tokens: {steps} steps token by token, {fewer} with {a.drafts} drafts of "
          f"{a.draft_len}; {100 * same:.1f}% of the tokens alike")


if __name__ == "__main__":
    main()
