"""The status of products with 4-bit weights when several threads and streams ask for it."""
import threading

import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding
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
