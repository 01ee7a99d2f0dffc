"""Chunks and weights behind a wait that gave up: while the device status word is set their tcgen05 kernels return without computing, everything else in the call runs as ever, and once
the word has been read calls are right again.  As in test_gpu_wait_limit.py a child process loads the copy of the library with a short limit."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys
sys.path.insert(0, "tests")
import torch
import paper_2310_05869_b200 as ha
import chunk_util as CU
import test_gpu_cache_chunk as TC
L = ha.lib()
g = torch.Generator(device="cuda"); g.manual_seed(3)
q, k, v = (torch.randn((1, 4, 4096, 64), device="cuda", generator=g).to(torch.bfloat16) for _ in range(3))
lens, counts = [300, 40, 1000], [300, 2, 700]
x, cache, table, K, V, (out, lse), _ = TC.both(lens, counts, (4, 2, 64), 16, torch.bfloat16)
lengths, cu = CU.ints(lens), CU.offsets(counts)
w = ha.cache_weights(x, cache, table, lengths, lse, cu)
torch.cuda.synchronize()
assert ha.last_device_status() == 0
assert L.hyperattn_test_arm_drop(1) == 0
ha.forward(q, k, v, 256, 256, 7, causal=True, n0=1024)          # gives up, and sets the word
before = cache.clone()
for _ in range(5):
    ha.cache_chunk_attention(x, cache, table, lengths, cu)
    ha.cache_weights(x, cache, table, lengths, lse, cu)
torch.cuda.synchronize()
assert torch.equal(cache, before)
assert ha.last_device_status() == -6 and ha.last_device_status() == 0
again = ha.cache_chunk_attention(x, cache, table, lengths, cu)
assert torch.equal(again[0], out) and torch.equal(again[1], lse)
assert torch.equal(ha.cache_weights(x, cache, table, lengths, lse, cu), w)
assert ha.last_device_status() == 0
print("serving behind a wait that gave up ok")
"""


def test_chunks_and_weights_behind_a_wait_that_gave_up():
    from paper_2310_05869_b200 import build as B
    lib = B.WAIT_TEST_LIB if os.path.exists(B.WAIT_TEST_LIB) else B.build_wait_test_library()
    env = dict(os.environ, HYPERATTN_LIB=lib, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    res = subprocess.run([sys.executable, "-c", CHILD], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    assert "serving behind a wait that gave up ok" in res.stdout
