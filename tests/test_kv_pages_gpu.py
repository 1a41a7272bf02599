"""Pages of the cache against plain loops over the same definitions (numpy, on the CPU): tables, counts and every byte of the pool."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding


# ---- the definitions -----------------------------------------------------------------------------------------------
class Model:
    """Pool contents are one number per layer and page: [layers][pages]."""

    def __init__(self, table, refs, ctx, page, layers):
        self.table, self.refs, self.ctx, self.page = table.copy(), refs.copy(), ctx.copy(), page
        self.pool = np.arange(layers * len(refs)).reshape(layers, len(refs))

    def is_page(self, e):
        return 0 <= e < len(self.refs)

    def fork(self, parent):
        before, ctx = self.table.copy(), self.ctx.copy()
        for b, p in enumerate(parent):
            if 0 <= p < len(parent) and parent[p] < 0:
                held = -(-max(ctx[p], 0) // self.page)
                self.table[b] = [e if i < held else -1 for i, e in enumerate(before[p])]
                for e in self.table[b]:
                    self.refs[e] += self.is_page(e)
                self.ctx[b] = ctx[p]

    def reserve(self, chunk):
        table, refs, pool = self.table.copy(), self.refs.copy(), self.pool.copy()
        free, missing = [p for p in range(len(refs)) if refs[p] <= 0], 0
        for b, n in enumerate(chunk):
            c = max(self.ctx[b], 0)
            for i in range(c // self.page, (c + n - 1) // self.page + 1) if n else []:
                if i >= table.shape[1]:
                    missing += 1
                    continue
                e = table[b, i]
                if self.is_page(e) and refs[e] <= 1:
                    continue
                if not free:
                    missing += 1
                    if self.is_page(e):
                        refs[e] -= 1
                    continue
                new = free.pop(0)
                if self.is_page(e):
                    refs[e] -= 1
                    if i * self.page < c:
                        pool[:, new] = pool[:, e]
                refs[new], table[b, i] = 1, new
        if missing == 0:
            self.table, self.refs, self.pool = table, refs, pool
        return missing

    def release(self, keep):
        for b, k in enumerate(keep):
            for i in range(-(-max(k, 0) // self.page), self.table.shape[1]):
                e = self.table[b, i]
                if self.is_page(e):
                    self.refs[e] -= 1
                    self.table[b, i] = -1

    def compact(self):
        used = int((self.refs > 0).sum())
        src = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        dst = [p for p in range(used) if self.refs[p] <= 0]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.pool[:, d] = self.pool[:, s]
            self.refs[d], self.refs[s] = self.refs[s], 0
        self.table = np.vectorize(lambda e: to.get(e, e))(self.table).astype(np.int32)
        return used


class Both:
    """The calls on both sides, compared after each."""

    def __init__(self, rows, width, pages, page=16, layers=2, heads=2, d=64, dtype="f16", quantised=False, seed=0):
        g = np.random.default_rng(seed)
        self.g, self.rows, self.page = g, rows, page
        held = torch.uint8 if quantised else {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        shape = (layers, pages, heads, page, d)
        # every byte of a page says which page of which layer it was, and where in the page it lies
        def filled(shape, what, factor):
            size = int(np.prod(shape[2:])) * factor
            a = (np.arange(size)[None, None] * 7 + np.arange(layers)[:, None, None] * 101 + np.arange(pages)[None, :, None] * 13 + what) % 120
            return torch.from_numpy(a.astype(np.uint8)).cuda()
        self.k, self.v = (filled(shape, i, 1 if quantised else 2).view(held).view(shape) for i in (0, 50))
        self.exps = [filled(shape[:4], i, 1).view(shape[:4]) for i in (3, 9)] if quantised else [None, None]
        self.start_bytes = [self.bytes(x) for x in self.arrays()]
        self.table, self.refs, self.ctx = (torch.full((rows, width), -1, dtype=torch.int32, device="cuda"), torch.zeros(pages, dtype=torch.int32, device="cuda"),
                                           torch.zeros(rows, dtype=torch.int32, device="cuda"))
        self.cache = binding.KvCache(self.k, self.v, dtype, *self.exps)
        self.pages = binding.KvPages(self.cache, self.table, self.refs)
        self.model = Model(self.table.cpu().numpy(), self.refs.cpu().numpy(), self.ctx.cpu().numpy(), page, layers)

    def arrays(self):
        return [x for x in (self.k, self.v, *self.exps) if x is not None]

    def bytes(self, x):
        return x.view(x.shape[0], x.shape[1], -1).view(torch.uint8).cpu().numpy().copy()

    def int32(self, a):
        return torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()

    def load(self):
        """The model's table, counts and lengths onto the GPU."""
        for t, a in ((self.table, self.model.table), (self.refs, self.model.refs), (self.ctx, self.model.ctx)):
            t.copy_(torch.from_numpy(a))

    def compare(self):
        torch.cuda.synchronize()
        self.cache.status()
        np.testing.assert_array_equal(self.table.cpu().numpy(), self.model.table)
        np.testing.assert_array_equal(self.refs.cpu().numpy(), self.model.refs)
        np.testing.assert_array_equal(self.ctx.cpu().numpy(), self.model.ctx)
        layer, page = np.divmod(self.model.pool, self.model.pool.shape[1])
        for x, start in zip(self.arrays(), self.start_bytes):
            np.testing.assert_array_equal(self.bytes(x), start[layer, page])

    def fork(self, parent):
        self.pages.fork(self.ctx, self.int32(parent))
        self.model.fork(list(parent))
        self.compare()

    def reserve(self, chunk):
        start = np.concatenate(([0], np.cumsum(chunk)))
        self.batch = binding.KvBatch(self.table, self.ctx, self.int32(start), rows=int(start[-1]), max_chunk=int(max(chunk)))
        missing = int(self.pages.reserve(self.batch))
        assert missing == self.model.reserve(list(chunk))
        self.compare()
        return missing

    def grow(self, chunk):
        """Reserves the chunks and counts on over them."""
        missing = self.reserve(chunk)
        if missing == 0:
            self.model.ctx = self.model.ctx + np.asarray(chunk, dtype=np.int32)
            self.load()
        return missing

    def release(self, keep):
        self.pages.release(self.int32(keep))
        self.model.release(list(keep))
        self.compare()
        self.model.ctx = np.minimum(self.model.ctx, np.maximum(keep, 0)).astype(np.int32)
        self.load()

    def compact(self):
        assert int(self.pages.compact()) == self.model.compact()
        self.compare()


GEOMETRIES = [dict(page=16, layers=3, heads=1, d=64), dict(page=128, layers=1, heads=3, d=128, dtype="bf16"), dict(page=32, layers=2, heads=5, d=64, quantised=True),
              dict(page=64, layers=2, heads=8, d=128, quantised=True, dtype="bf16")]


@pytest.mark.gpu
@pytest.mark.parametrize("geometry", GEOMETRIES)
def test_a_sequences_life(geometry):
    page = geometry["page"]
    x = Both(rows=6, width=9, pages=40, **geometry)
    assert x.grow([page * 2 + 1, page, 1, 0, 0, 0]) == 0
    x.fork([-1, -1, -1, 0, 0, 1])                  # two copies of a partly filled page, one of a full one
    x.grow([1, 1, 0, 1, page + 3, 1])              # 0, 3 and 4 wish for one page: the last keeps it
    x.grow([0, page, 5, 1, 1, 2 * page])
    x.release([page + 1, 0, 0, 10 ** 9, page, -5])
    x.compact()
    x.grow([3, 70, 3, 1, 1, 1])
    x.compact()
    x.release([0] * 6)
    x.compact()
    assert int(x.refs.abs().sum()) == 0 and int(x.table.max()) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
def test_random_lives(seed):
    g = np.random.default_rng(seed)
    rows, pages = int(g.integers(1, 40)), int(g.integers(30, 400))
    x = Both(rows=rows, width=12, pages=pages, seed=seed, **GEOMETRIES[seed % 4])
    served = 0
    for _ in range(12):
        what = g.random()
        if what < 0.45:
            served += x.grow(g.integers(0, 2 * x.page, rows) * (g.random(rows) < 0.6)) == 0
        elif what < 0.65:
            # rows that are let go become copies of others
            child = g.random(rows) < 0.4
            others = np.nonzero(~child)[0]
            if len(others):
                x.release(np.where(child, 0, 2 ** 31 - 1))
                x.fork(np.where(child, g.choice(others, rows), -1))
        elif what < 0.85:
            x.release(np.where(g.random(rows) < 0.5, x.model.ctx, x.model.ctx // 2))
        else:
            x.compact()
    assert served > 0


@pytest.mark.gpu
@pytest.mark.parametrize("rows,chunk", [(1, 5000), (2000, 1), (3, 700), (70, 40)])
def test_many_pages_at_once(rows, chunk):
    """A long prompt; more rows than a CTA looks after at a time; a pool of more pages than the planning threads."""
    width, pages = 320, rows * (chunk // 16 + 2) + 9001
    x = Both(rows=rows, width=width, pages=pages, layers=1, heads=1, d=64, page=16)
    # free pages lie scattered
    held = np.nonzero(np.random.default_rng(rows).random(pages) < 0.5)[0][:9000]
    x.model.refs[held] = 1
    x.load()
    chunks = np.maximum(chunk - np.arange(rows) % 7, 0)
    assert x.grow(chunks) == 0
    x.grow(np.full(rows, 1))
    x.model.refs[held] = 0                         # as if rows elsewhere had let them go
    x.load()
    x.compact()


@pytest.mark.gpu
def test_many_copies_of_one_page():
    """299 copies share a page with the first row; all wish at once."""
    x = Both(rows=300, width=4, pages=400, page=16, layers=2, heads=2, d=64)
    x.grow([10] + [0] * 299)
    x.fork([-1] + [0] * 299)
    assert x.refs[0] == 300
    x.grow([1] * 300)
    assert x.refs[0] == 1 and x.table[299, 0] == 0
    x.release([0] * 150 + [11] * 150)
    x.compact()


@pytest.mark.gpu
def test_a_pool_that_is_too_small_changes_nothing():
    x = Both(rows=3, width=4, pages=5, page=16)
    x.grow([40, 0, 0])                             # three pages
    x.fork([-1, 0, 0])
    assert x.reserve([1, 40, 60]) > 0              # shared pages among the wishes: their counts stay
    assert x.reserve([0, 1, 1]) == 0               # the workspace is as it was
    x.release([40, 0, 0])
    assert x.reserve([16 * 4 - 40 + 1, 0, 0]) == 1          # a place behind the table
    assert x.reserve([16 * 4 - 40 + 16 * 20, 0, 16 * 7]) > 20
    assert x.reserve([16 * 4 - 40, 0, 16]) == 0


@pytest.mark.gpu
def test_rows_that_cannot_be_copied():
    x = Both(rows=6, width=4, pages=20)
    x.grow([20, 33, 0, 0, 0, 0])
    x.fork([-1, -1, 3, 0, 6, 5])                   # a copy of a copy, a row that is not there, oneself: only row 3 is copied
    assert x.table[2].tolist() == [-1] * 4 and x.table[3, 0] == x.table[0, 0] and x.table[5, 0] == -1
    x.fork([-1, -1, -2 ** 31, -7, 2 ** 31 - 1, 1])
    x.fork([-1] * 6)


@pytest.mark.gpu
def test_contradictions_stay_inside():
    """Counts that do not fit the tables, entries outside the pool, lengths below zero or far behind the table: no access outside the
    arrays (guards around them stay whole), and the calls come back."""
    pages, rows, width = 12, 5, 3
    guarded = torch.full((pages + 64,), 77, dtype=torch.int32, device="cuda")
    refs = guarded[32:32 + pages]
    wide = torch.full((rows * width + 64,), 77, dtype=torch.int32, device="cuda")
    table = wide[32:32 + rows * width].view(rows, width)
    k, v = (torch.zeros((1, pages, 1, 16, 64), dtype=torch.float16, device="cuda") for _ in range(2))
    cache = binding.KvCache(k, v, "f16")
    p = binding.KvPages(cache, table, refs)
    g = np.random.default_rng(0)
    for trial in range(20):
        refs.copy_(torch.from_numpy(g.integers(-2, 4, pages).astype(np.int32)))
        table.copy_(torch.from_numpy(g.choice([-1, -2 ** 31, 0, 1, 1, 5, 11, 12, 2 ** 31 - 1], (rows, width)).astype(np.int32)))
        ctx = torch.from_numpy(g.choice([-2 ** 31, -1, 0, 17, 40, 47, 48, 1000, 2 ** 31 - 1], rows).astype(np.int32)).cuda()
        start = torch.from_numpy(np.array([[0, 3, 9, 9, 30, 60], [-5, 70, 2, -1, 80, 10], [60, 50, 40, 30, 20, 10]][trial % 3], dtype=np.int32)).cuda()
        batch = binding.KvBatch(table, ctx, start, rows=60)
        p.reserve(batch)
        p.fork(ctx, torch.from_numpy(g.integers(-3, rows + 2, rows).astype(np.int32)).cuda())
        p.release(ctx)
        used = int(p.compact())
        cache.status()
        assert 0 <= used <= pages
        for t, n in ((guarded, pages), (wide, rows * width)):
            assert bool((t[:32] == 77).all()) and bool((t[32 + n:] == 77).all())


@pytest.mark.gpu
def test_appending_to_copies_leaves_the_others_alone():
    """Copies of one prompt write different tokens behind it; each reads its own, and the prompt is whole in all of them."""
    g = torch.Generator(device="cuda").manual_seed(0)
    x = Both(rows=4, width=6, pages=30, layers=2, heads=2, d=64, page=16)
    x.reserve([21, 0, 0, 0])
    token = lambda n: torch.randn((n, 2, 64), device="cuda", generator=g).half()
    prompt = token(21)
    for layer in range(2):
        x.cache.append(layer, prompt, prompt, x.batch)
    x.model.ctx[0] = 21
    x.load()
    x.pages.fork(x.ctx, x.int32([-1, 0, 0, 0]))
    start = x.int32([0, 20, 40, 60, 80])
    batch = binding.KvBatch(x.table, x.ctx, start, rows=80, max_chunk=20)
    assert int(x.pages.reserve(batch)) == 0
    new = token(80)
    for layer in range(2):
        x.cache.append(layer, new, -new, batch)
    whole = binding.KvBatch(x.table, x.int32([0] * 4), x.int32([0, 41, 82, 123, 164]), rows=164, max_chunk=41)
    for layer in range(2):
        k, v = x.cache.read(layer, whole)
        for b in range(4):
            assert torch.equal(k[41 * b:41 * b + 21], prompt) and torch.equal(v[41 * b:41 * b + 21], prompt)
            assert torch.equal(k[41 * b + 21:41 * b + 41], new[20 * b:20 * b + 20]) and torch.equal(v[41 * b + 21:41 * b + 41], -new[20 * b:20 * b + 20])
    used = int(x.pages.compact())
    assert used == int((x.refs > 0).sum()) and int(x.table.max()) == used - 1
    k, _ = x.cache.read(1, whole)
    assert all(torch.equal(k[41 * b + 21:41 * b + 41], new[20 * b:20 * b + 20]) for b in range(4))


@pytest.mark.gpu
def test_captured_calls_and_two_tables_of_one_cache():
    x = Both(rows=3, width=5, pages=30)
    x.grow([20, 0, 0])
    parent, keep, start = x.int32([-1, 0, 0]), x.int32([20, 0, 0]), x.int32([0, 0, 5, 10])
    batch = binding.KvBatch(x.table, x.ctx, start, rows=10, max_chunk=5)
    other_table, other_refs = torch.full((2, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(30, dtype=torch.int32, device="cuda")
    other = binding.KvPages(x.cache, other_table, other_refs)          # counts elsewhere, for the same cache
    other.release(x.int32([0, 0]))
    x.fork([-1, 0, 0])
    x.release([20, 0, 0])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        x.pages.fork(x.ctx, parent)
        missing = x.pages.reserve(batch)
        x.pages.release(keep)
        used = x.pages.compact()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        x.model.fork([-1, 0, 0])
        assert int(missing) == x.model.reserve([0, 5, 5])
        x.model.release([20, 0, 0])
        assert int(used) == x.model.compact()
        x.compare()
    assert int(other_refs.abs().sum()) == 0


@pytest.mark.gpu
def test_refusals():
    x = Both(rows=3, width=5, pages=30)
    cache, table, refs = x.cache, x.table, x.refs
    ones = x.int32([-1, -1, -1])
    for bad in [lambda: binding.KvPages(cache, table.long(), refs), lambda: binding.KvPages(cache, table[:, :3], refs), lambda: binding.KvPages(cache, table.cpu(), refs),
                lambda: binding.KvPages(cache, table, refs[:29]), lambda: binding.KvPages(cache, table, refs.float()), lambda: binding.KvPages(cache, table[0], refs),
                lambda: x.pages.fork(x.ctx, ones[:2]), lambda: x.pages.fork(x.ctx.long(), ones), lambda: x.pages.release(ones.cpu()),
                lambda: x.pages.reserve(binding.KvBatch(table.clone(), x.ctx, x.int32([0, 1, 2, 3]), rows=3))]:
        with pytest.raises(binding.DresdError) as e:
            bad()
        assert e.value.status == -1
    fresh = binding.KvCache(x.k, x.v, "f16")
    batch = binding.KvBatch(table, x.ctx, x.int32([0, 1, 2, 3]), rows=3)
    word = x.int32([0])
    for call in [lambda: binding.dresd_kv_reserve(fresh.handle, batch.c, word.data_ptr()), lambda: binding.dresd_kv_compact(fresh.handle, batch.c, word.data_ptr()),
                 lambda: binding.dresd_kv_release(fresh.handle, batch.c, ones.data_ptr()), lambda: binding.dresd_kv_fork(fresh.handle, batch.c, x.ctx.data_ptr(), ones.data_ptr()),
                 lambda: binding.dresd_kv_attach_pages(fresh.handle, 0), lambda: binding.dresd_kv_fork(cache.handle, batch.c, ones.data_ptr(), ones.data_ptr()),
                 lambda: binding.dresd_kv_reserve(cache.handle, batch.c, 0), lambda: binding.dresd_kv_compact(cache.handle, batch.c, 0),
                 lambda: binding.dresd_kv_release(cache.handle, batch.c, 0), lambda: binding.dresd_kv_reserve(0, batch.c, word.data_ptr())]:
        with pytest.raises(binding.DresdError) as e:
            call()
        assert e.value.status == -1
    x.compare()


@pytest.mark.gpu
def test_batches_without_rows():
    x = Both(rows=3, width=5, pages=30)
    x.grow([5, 0, 0])
    batch = binding.KvBatch(x.table, x.ctx, x.int32([0, 0, 0, 0]), rows=0)
    assert int(x.pages.reserve(batch)) == 0
    x.compare()
