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
