"""The paged cache's kernels under the bounds-checked debug build (libdresd_debug.so): the tests of the cache and its
attention, those of contradictory batches among them, run in a child process with DRESD_DEBUG=1.  Every one of them ends
with a status call, which reports the first check that failed.
"""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SELFTEST = r'''
import torch
from paper_2502_15572_b200 import binding
assert binding.dresd_debug_build() == 1, "the release library was loaded"
pages = [torch.zeros((1, 4, 2, 16, 64), dtype=torch.float16, device="cuda") for _ in range(2)]
cache = binding.KvCache(*pages, "f16")
binding.dresd_kv_debug_selftest(cache.handle)
try:
    cache.status()
    raise SystemExit("the failed check was not reported")
except binding.DresdError as e:
    assert e.status == -6 and "check 7" in e.message, (e.status, e.message)
cache.status()                                # the word is cleared
print("reported")
'''


def child(*args):
    from paper_2502_15572_b200 import build as lib_build
    lib_build.build(debug=True)
    env = dict(os.environ, DRESD_DEBUG="1", PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    r = subprocess.run([sys.executable, *args], capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-2000:])
    return r.stdout


@pytest.mark.gpu
def test_a_failed_check_is_reported_by_the_cache():
    assert "reported" in child("-c", SELFTEST)


@pytest.mark.gpu
def test_no_check_of_the_caches_kernels_fails():
    chosen = ("chunks_of_every_length or draft_chunks or masks_that or either_kernel or far_into or bad_batches or append_and_read or "
              "test_keep_draft or (large_ragged and f16) or (many_row and 64) or long_contexts or contexts_beyond or contradict or zero_rows")
    out = child("-m", "pytest", "tests/test_kv_cache_gpu.py", "tests/test_kv_attend_gpu.py", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider",
                "-k", chosen)
    assert " passed" in out and "skipped" not in out


@pytest.mark.gpu
def test_the_release_build_has_no_self_test():
    import torch
    from paper_2502_15572_b200 import binding
    if binding.dresd_debug_build():
        return
    cache = binding.KvCache(*(torch.zeros((1, 4, 2, 16, 64), dtype=torch.float16, device="cuda") for _ in range(2)), "f16")
    with pytest.raises(binding.DresdError) as e:
        binding.dresd_kv_debug_selftest(cache.handle)
    assert e.value.status == -2
