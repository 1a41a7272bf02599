"""Products with 4-bit weights and their status, when several threads and streams call."""
import subprocess
import sys
import threading

import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding
from tests.test_decode_edges_gpu import ROOT, env
from tests.test_w4_gpu import exact_inputs, option  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def status(stream=0):
    try:
        binding.dresd_w4_status(stream)
    except binding.DresdError as e:
        return e.status
    return 0


def test_every_thread_is_told_of_a_wait_that_ran_out(option):
    """Whoever asks first does not take the report from the others; each is told once."""
    x, codes, scales = exact_inputs(40, 4096, 600, 128, "f16", 4)
    w = binding.W4(codes, scales, "f16")
    want = w.matmul(x)
    ask, answers = [threading.Event() for _ in range(3)], []

    def other():
        torch.cuda.set_device(0)
        answers.append(status())
        ask[0].set()
        for turn in (1, 2):
            assert ask[turn].wait(120)
            answers.append(status())

    thread = threading.Thread(target=other, daemon=True)
    thread.start()
    assert ask[0].wait(120)
    status()                                                  # what earlier calls left
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    option("w4_path", 2)
    option("w4_wait_ms", 20)
    option("w4_debug_lose_stage", 1)
    w.matmul(x, stream=side)
    option("w4_debug_lose_stage", 0)
    side.synchronize()
    assert status(torch.cuda.current_stream().cuda_stream) == -5       # of another stream: the device's
    ask[1].set()
    while len(answers) < 2 and thread.is_alive():
        thread.join(0.05)
    assert answers[1] == -5
    ask[2].set()
    thread.join(120)
    assert answers[2] == 0 and status(side.cuda_stream) == 0
    assert torch.equal(w.matmul(x), want) and status() == 0

FIRST_CALLS = r'''
import threading
import torch
from tests.test_w4_gpu import exact_inputs, weights64
from paper_2502_15572_b200 import binding
x, codes, scales = exact_inputs(40, 1024, 600, 128, "f16", 4)
w = binding.W4(codes, scales, "f16")
binding.dresd_set_global_option("w4_path", 2)
torch.cuda.synchronize()
results, begin = [None] * 8, threading.Barrier(8)
def call(i):
    torch.cuda.set_device(0)
    stream = torch.cuda.Stream()
    begin.wait()
    results[i] = w.matmul(x, stream=stream)
    stream.synchronize()
threads = [threading.Thread(target=call, args=(i,)) for i in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
want = (x.cpu().double() @ weights64(codes, scales, 128).T).half()
assert all(torch.equal(r.cpu(), want) for r in results)
binding.dresd_w4_status()
print("threads agree")
'''


def test_first_calls_of_several_threads():
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, env=env(), cwd=ROOT, timeout=600)
    assert r.returncode == 0 and "threads agree" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])
