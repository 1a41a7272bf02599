"""Calls of sampled verification, pages and 4-bit products at their edges: misaligned addresses, two calls at once, the first call of a
process inside a capture, and the pages' tests under the bounds-checked build."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2502_15572_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def env(**more):
    return dict(os.environ, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""), **more)


@pytest.mark.gpu
def test_misaligned_words_are_refused():
    new = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="cuda")
    logits, uniform, setting, words = new(1, 3, 64, dtype=torch.float16), new(4, dtype=torch.float32), new(4, dtype=torch.float32), new(16)
    p, w = logits.data_ptr(), words.data_ptr()
    args = [p, binding.DRESD_F16, 192, 64, 64, w, w + 16, uniform.data_ptr(), setting.data_ptr(), w + 32, setting.data_ptr(), 1, 1, 2, w + 40, w + 44, w + 48, 0]
    for i in (5, 6, 7, 8, 9, 10, 14, 15, 16, 17):
        bad = list(args)
        bad[i] = (bad[i] or w) + 2
        with pytest.raises(binding.DresdError) as e:
            binding.dresd_drafts_sample(*bad)
        assert e.value.status == -1
    k, v = (new(1, 4, 1, 16, 64, dtype=torch.float16) for _ in range(2))
    cache = binding.KvCache(k, v, "f16")
    refs, table, start = new(5), new(8), new(3)
    with pytest.raises(binding.DresdError):
        binding.dresd_kv_attach_pages(cache.handle, refs.data_ptr() + 2)
    binding.dresd_kv_attach_pages(cache.handle, refs.data_ptr())
    batch = lambda t=0, c=0, s=0: binding.dresd_kv_batch(table.data_ptr() + t, w + c, start.data_ptr() + s, 1, 4, 1, 0)
    for call in [lambda: binding.dresd_kv_reserve(cache.handle, batch(), w + 2), lambda: binding.dresd_kv_compact(cache.handle, batch(), w + 2),
                 lambda: binding.dresd_kv_release(cache.handle, batch(), w + 2), lambda: binding.dresd_kv_fork(cache.handle, batch(), w, w + 2),
                 lambda: binding.dresd_kv_reserve(cache.handle, batch(t=2), w), lambda: binding.dresd_kv_reserve(cache.handle, batch(c=2), w),
                 lambda: binding.dresd_kv_reserve(cache.handle, batch(s=2), w), lambda: binding.dresd_kv_release(cache.handle, batch(t=2), w)]:
        with pytest.raises(binding.DresdError) as e:
            call()
        assert e.value.status == -1
    assert not any(int(t.abs().sum()) for t in (words, refs, table))


def operators():
    """Calls on fixed inputs, as functions that return their results."""
    gen = torch.Generator().manual_seed(5)
    rand = lambda *shape, dtype=torch.float16: torch.randn(shape, generator=gen).to(dtype).cuda()
    w = binding.W4.quantise(rand(2048, 4096, dtype=torch.bfloat16), 64)
    x = {rows: rand(rows, 2048, dtype=torch.bfloat16) for rows in (1, 20, 300)}
    logits, uniform = 4 * rand(3, 5, 40001), torch.rand((3, 5), generator=gen).cuda()
    drafts = torch.randint(40001, (3, 1, 4), generator=gen).int().cuda()
    valid, p = torch.ones((3, 1), dtype=torch.int32, device="cuda"), torch.full((3,), 0.9, device="cuda")
    calls = [lambda r=r: (w.matmul(x[r]),) for r in x]
    return calls + [lambda: binding.drafts_sample(logits, uniform, drafts, valid, top_p=p), lambda: binding.drafts_sample(logits[:, :1], uniform[:, :1].contiguous(), top_p=p)]


@pytest.mark.gpu
def test_two_calls_at_once():
    calls = operators()
    want = [call() for call in calls]
    torch.cuda.synchronize()
    streams, graphs, results = [torch.cuda.Stream() for _ in range(2)], [], []
    for turn, stream in enumerate(streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            order = range(len(calls)) if turn == 0 else reversed(range(len(calls)))
            results.append({i: calls[i]() for _ in range(3) for i in order})
        graphs.append(graph)
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for result in results:
        for i, outs in result.items():
            assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))
    binding.dresd_w4_status()


CAPTURED_FIRST = r'''
import torch
from tests.test_decode_edges_gpu import operators
from paper_2502_15572_b200 import binding
calls = operators()
torch.cuda.synchronize()
graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
with torch.cuda.graph(graph, stream=stream):
    results = [call() for call in calls]
graph.replay()
torch.cuda.synchronize()
for call, outs in zip(calls, results):
    assert all(torch.equal(a, b) for a, b in zip(call(), outs))
binding.dresd_w4_status()
print("captured first")
'''


@pytest.mark.gpu
def test_the_first_call_of_a_process_may_be_captured():
    r = subprocess.run([sys.executable, "-c", CAPTURED_FIRST], capture_output=True, text=True, env=env(), cwd=ROOT, timeout=600)
    assert r.returncode == 0 and "captured first" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])


@pytest.mark.gpu
def test_pages_under_the_bounds_checked_build():
    code = ("import sys, pytest; from paper_2502_15572_b200 import binding, build; build.build(debug=True); assert binding.dresd_debug_build() == 1;"
            "sys.exit(pytest.main(['-x', '-q', '-m', 'gpu', '-p', 'no:cacheprovider', 'tests/test_kv_pages_gpu.py']))")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, env=env(DRESD_DEBUG="1"), cwd=ROOT, timeout=900)
    assert r.returncode == 0 and "passed" in r.stdout, (r.stdout[-3000:], r.stderr[-3000:])
