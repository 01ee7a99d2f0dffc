"""Calls on a stream of the caller's while torch's current one is busy: nothing of theirs may wait for it, or run on it."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def check(call, after=None, off=0.0):
    """call(**kw) -> tensors; after(): what the call has changed; off: what two calls may differ by, relative (sums whose order is anybody's)."""
    got = call()
    want = [x.clone() for x in (after() if after else got)]
    side = torch.cuda.Stream()
    for _ in range(3):
        for x in (after() if after else ()):
            x.zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(400_000_000)                   # some tenths of a second
        got = call(stream=side.cuda_stream)
        with torch.cuda.stream(side):
            got = [x.clone() for x in (after() if after else got)]
        side.synchronize()
        busy = not torch.cuda.current_stream().query()
        torch.cuda.synchronize()
        if busy:                                         # the current stream was still at it (something else may have held the call up)
            break
    assert len(got) == len(want) and all(torch.equal(a, b) if not off else ((a - b).abs() <= off * b.abs()).all() for a, b in zip(got, want))


# strides that a call has to copy for: an odd address, rows that are all the same one, coordinates that are not next to each other
def odd(x):
    wide = torch.zeros(*x.shape[:-1], x.shape[-1] + 1, dtype=x.dtype, device=x.device)
    wide[..., 1:] = x
    return wide[..., 1:]


COPIES = {"odd": odd, "one row": lambda x: x[:1].expand_as(x), "turned": lambda x: x.transpose(-1, -2).contiguous().transpose(-1, -2)}


@pytest.mark.parametrize("kind", list(COPIES))
@pytest.mark.parametrize("d", [64, 128])
def test_tensors_that_are_copied(kind, d):
    make = COPIES[kind]
    T, H, page = 3000, 4, 64
    q, k, v = (make(torch.randn(T, H, d, device="cuda").bfloat16()) for _ in range(3))
    cu = ints([0, 1000, 3000])
    check(lambda **kw: ha.prompt_attention(q, k, v, cu, **kw))
    cache = ha.cache_pages(T // page + 1, H, d, page)
    slots = ints(np.arange(T))
    check(lambda **kw: ha.cache_store(cache, k, v, slots, **kw), lambda: [cache])
    table, lengths = ints(np.arange(T // page))[None].repeat(40, 1), ints(np.arange(40) * 60)
    check(lambda **kw: ha.cache_attention(q[:40], cache, table, lengths, **kw))
    rows = ints(np.arange(41) * 50)
    check(lambda **kw: ha.cache_read(cache, table, rows, 2000, **kw))


def test_plans_of_some_requests_and_of_none():
    rng = np.random.default_rng(0)
    for R in (0, 5):
        lengths, new, table = ints(rng.integers(0, 40, R)), ints(rng.integers(-1, 9, R)), ints(np.arange(R * 4).reshape(R, 4))
        free, n_free = ints(np.arange(30, 60)), ints([30])
        check(lambda **kw: ha.cache_plan(lengths, new, table, free, n_free, 16, 50, **kw))


def test_the_default_stream_from_another_one():
    q, k, v = (torch.randn(500, 2, 64, device="cuda").bfloat16() for _ in range(3))
    cu = ints([0, 500])
    want = ha.prompt_attention(q, k, v, cu)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        q = odd(q)
        torch.cuda.synchronize()
        got = ha.prompt_attention(q, k, v, cu, stream=torch.cuda.default_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_the_approximation_its_gradients_and_its_parts():
    q, k, v, dout = (torch.randn(3000, 1, 2, 64, device="cuda").bfloat16().permute(1, 2, 0, 3) for _ in range(4))       # (copied: rows are not next to each other)
    check(lambda **kw: ha.forward(q, k, v, 256, 256, 7, causal=True, n0=1024, **kw))
    check(lambda **kw: tuple(x for x in ha.forward(q, k, v, 256, 256, 7, debug=True, **kw)[:2]))
    out, lse = ha.forward(q, k, v, 256, 256, 7)
    x = q[0, 0, :, :]
    check(lambda **kw: ha.sortlsh_noalloc(x, 7, **kw))
    check(lambda **kw: (ha.alpha(q, k, **kw),), off=3000 * 2.0 ** -24)          # (a column's sum over the rows, in any order)
    grads = ha.backward(q, k, v, out, lse, dout, 256, 256, 7)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)
    got = ha.backward(q, k, v, out, lse, dout, 256, 256, 7, stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(got, grads):                         # (sums of the key's gradients come in any order)
        assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()


FIRST = r"""
import torch
import paper_2310_05869_b200 as ha
q, k, v = (torch.randn(1000, 4, 64, device="cuda").bfloat16() for _ in range(3))
cu = torch.tensor([0, 1000], dtype=torch.int32, device="cuda")
x = torch.full((1 << 26,), -1, dtype=torch.int32, device="cuda")       # memory that is not zero goes back to the driver
del x
torch.cuda.synchronize()
torch.cuda.empty_cache()
side = torch.cuda.Stream()
torch.cuda._sleep(400_000_000)                                          # the default stream is busy
with torch.cuda.stream(side):
    got = ha.prompt_attention(q, k, v, cu)
    side.synchronize()
    assert ha.last_device_status() == 0
    torch.cuda.synchronize()
    want = ha.prompt_attention(q, k, v, cu)
    side.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool(got[0].any())
print("first call ok")
"""


def test_the_first_call_on_a_device_beside_a_busy_default_stream():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, PYTHONPATH=root + os.pathsep + os.environ.get("PYTHONPATH", ""))
    res = subprocess.run([sys.executable, "-c", FIRST], env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "first call ok" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]
