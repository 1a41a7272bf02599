"""Results that a call allocates belong to the stream that writes them, and tensors to the device of their cache."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding


class Side:
    """Stands for a stream where there is no GPU."""
    cuda_stream = 77


@pytest.fixture
def recorded(monkeypatch):
    """Allocations as (stream they were made under), and a library whose calls do nothing."""
    under, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        under.append(stream)
        yield
        under.pop()

    real = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: (made.append(under[-1]), real(*a, **kw))[1])
    for name in ("dresd_kv_attend", "dresd_kv_read", "dresd_retrieve", "dresd_retrieve_filtered", "dresd_retrieve_quantised",
                 "dresd_preprocess", "dresd_quantise_keys", "dresd_store_attach_quantised"):
        monkeypatch.setattr(binding, name, lambda *a: None)
    monkeypatch.setattr(binding.KvCache, "_rows", lambda *a: (0, 0))
    return made


def calls():
    """name -> call with a stream (or None: of a cache, where that needs no GPU)."""
    cache = binding.KvCache.__new__(binding.KvCache)
    cache.k_pages, cache.torch_dtype, cache.kv_heads, cache.head_dim, cache.device_index = torch.zeros(1), torch.float16, 2, 64, 0
    store = binding.Store.__new__(binding.Store)
    store.keys, store.N, store.d, store.dtype = torch.zeros(1), 5, 4, "f16"
    cache.handle = store.handle = None
    batch = type("Batch", (), dict(rows=3, c=None, device_index=0))
    q, queries = torch.zeros((3, 4, 64), dtype=torch.float16), torch.zeros((2, 4))
    return {"attend": lambda s: cache.attend(0, q, batch, stream=s), "read": lambda s: cache.read(0, batch, stream=s),
            "retrieve": lambda s: store.retrieve(queries, 2, 2, stream=s),
            "retrieve_filtered": lambda s: store.retrieve_filtered(queries, None, 2, 2, stream=s),
            "retrieve_quantised": lambda s: store.retrieve_quantised(queries, 2, 2, 4, stream=s),
            "attach_quantised": lambda s: store.attach_quantised(stream=s), "preprocess": lambda s: store.preprocess(queries, stream=s)}


@pytest.mark.parametrize("name", ["attend", "read", "retrieve", "retrieve_filtered", "retrieve_quantised", "attach_quantised", "preprocess"])
def test_results_are_allocated_on_the_stream_that_writes_them(recorded, name):
    side = Side()
    calls()[name](side)
    assert recorded and all(s is side for s in recorded)


@pytest.mark.gpu
def test_results_on_another_stream_while_the_current_one_is_busy():
    """Memory that the current stream has freed but still writes to (behind a delay) is not given to a call on another stream."""
    from tests.test_kv_cache_gpu import Case
    case = Case("f16", 64, 16, 2, [300, 40], [1, 1], seed=90)
    q = case.queries(8)
    want, (want_k, want_v) = case.cache.attend(0, q, case.batch), case.cache.read(0, case.batch)
    side = torch.cuda.Stream()
    for call, right in ((lambda: case.cache.attend(0, q, case.batch, stream=side), want),
                        (lambda: case.cache.read(0, case.batch, stream=side)[0], want_k),
                        (lambda: case.cache.read(0, case.batch, stream=side)[1], want_v)):
        torch.cuda.synchronize()
        x = [torch.empty_like(want) for _ in range(64)]
        torch.cuda._sleep(100_000_000)                         # some 50 ms
        for t in x:
            t.fill_(7.0)
        del x, t
        got = call()
        torch.cuda.synchronize()
        assert torch.equal(got, right)
    case.cache.status()


class Tensor:
    """Stands for a CUDA tensor of device `at`."""
    is_cuda = True

    def __init__(self, at, dtype, *shape):
        self.at, self.dtype, self.shape = at, dtype, torch.Size(shape)
        self.device = torch.device("cuda", at)

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(torch.empty(self.shape, device="meta").stride())

    def data_ptr(self):
        return 4096


def test_tensors_of_another_device_are_refused(monkeypatch):
    for name in ("dresd_kv_attend", "dresd_kv_read", "dresd_kv_append", "dresd_kv_keep_draft", "_raw_stream"):
        monkeypatch.setattr(binding, name, lambda *a: 0)
    monkeypatch.setattr(binding, "dresd_kv_create", lambda *a: 0)
    i32, f16, u8, f32 = torch.int32, torch.float16, torch.uint8, torch.float32
    batch = lambda *at: binding.KvBatch(Tensor(at[0], i32, 2, 4), Tensor(at[1], i32, 2), Tensor(at[2], i32, 3), 5)
    pages = lambda at, dtype=f16: Tensor(at, dtype, 1, 9, 2, 16, 64)
    cache = binding.KvCache(pages(0), pages(0), "f16")
    here, there = batch(0, 0, 0), batch(1, 1, 1)
    k, q, best = (lambda at: Tensor(at, f16, 5, 2, 64)), (lambda at: Tensor(at, f16, 5, 4, 64)), (lambda at: Tensor(at, i32, 2))
    good = [lambda: cache.append(0, k(0), k(0), here), lambda: cache.read(0, here, out=(k(0), k(0))),
            lambda: cache.attend(0, q(0), here, out=q(0), lse=Tensor(0, f32, 5, 4), mask=Tensor(0, i32, 5, 1)),
            lambda: cache.keep_draft(here, best(0), best(0), 2, 2)]
    bad = [lambda: batch(0, 1, 0), lambda: batch(0, 0, 1), lambda: binding.KvCache(pages(0), pages(1), "f16"),
           lambda: binding.KvCache(pages(0, u8), pages(0, u8), "f16", Tensor(1, u8, 1, 9, 2, 16), Tensor(0, u8, 1, 9, 2, 16)),
           lambda: cache.append(0, k(1), k(0), here), lambda: cache.append(0, k(0), k(1), here), lambda: cache.append(0, k(0), k(0), there),
           lambda: cache.read(0, there, out=(k(0), k(0))), lambda: cache.read(0, here, out=(k(0), k(1))),
           lambda: cache.attend(0, q(1), here, out=q(0)), lambda: cache.attend(0, q(0), there, out=q(0)), lambda: cache.attend(0, q(0), here, out=q(1)),
           lambda: cache.attend(0, q(0), here, out=q(0), lse=Tensor(1, f32, 5, 4)),
           lambda: cache.attend(0, q(0), here, out=q(0), mask=Tensor(1, i32, 5, 1)),
           lambda: cache.keep_draft(there, best(0), best(0), 2, 2), lambda: cache.keep_draft(here, best(1), best(0), 2, 2)]
    for call in good:
        call()
    for i, call in enumerate(bad):
        with pytest.raises(binding.DresdError) as e:
            call()
        assert e.value.status == -1, i
