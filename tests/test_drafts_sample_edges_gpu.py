"""Verification by sampling where few calls go: CTAs that begin late, rows so long that an entry stands for several steps, temperatures at
their ends, and the weights themselves."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding
from tests.test_drafts_sample_gpu import DT, ONE, check, chunk, ref_row

pytestmark = pytest.mark.gpu


def test_clusters_of_a_busy_gpu():
    """Calls whose CTAs begin while others of all sizes still run, one behind the other and on two streams: what each gives alone."""
    g = torch.Generator(device="cuda").manual_seed(6)
    calls = []
    for B, V in ((1, 32000), (9, 20001), (17, 9000), (40, 33001), (150, 2500)):
        logits = (torch.randn((B, 1, V), device="cuda", generator=g) * 2).half()
        u, p = torch.rand((B, 1), device="cuda", generator=g), torch.full((B,), 0.9, device="cuda")
        calls.append(lambda x=logits, u=u, p=p: binding.drafts_sample(x, u, top_p=p))
    logits, uniform, drafts, valid = chunk(7, 3, 5, 12001, "bf16", 4)
    u, d, v = (torch.from_numpy(a).cuda() for a in (uniform.astype(np.float32), drafts, valid))
    calls.append(lambda: binding.drafts_sample(logits, u, d, v))
    want = []
    for call in calls:
        want.append(call())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(20):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                i = (turn * (1 + 2 * s) + s) % len(calls)
                got.append((i, calls[i]()))
    torch.cuda.synchronize()
    for i, outs in got:
        assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))
