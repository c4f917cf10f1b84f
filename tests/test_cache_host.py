"""Host-side tests of the 4-bit cache: what the C entry points and the binding
refuse before anything is launched, and the sizes they give. Runs without a
GPU: pointers are stand-ins that a refused call never reads."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_2507_16676_amd as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096          # an aligned pointer, never read
BIG = 1 << 40


def test_cache_bytes():
    lib = F.lib()
    # per tile of 64 slots: codes of K and V, K's block scales, V's scales, two sums of two bf16
    for d in (64, 96, 128, 256):
        tile = 64 * (d + d // 32 + 2 + 8)
        assert lib.fabft_cache_bytes(1, 1, 64, d) == tile
        assert lib.fabft_cache_bytes(3, 5, 640, d) == 150 * tile
    for args in ((0, 1, 64, 64), (1, 0, 64, 64), (1, 1, 0, 64), (1, 1, 100, 64), (1, 1, -64, 64),
                 (1, 1, (1 << 30) + 64, 64), (1 << 20, 1 << 20, 64, 64),
                 (1 << 12, 1 << 12, 1 << 30, 256)):      # the last: past 2^61 bytes
        assert lib.fabft_cache_bytes(*args) == F.E_SHAPE, args
    assert lib.fabft_cache_bytes(1, 1, 64, 80) == F.E_HEADDIM
    assert lib.fabft_cache_bytes(1 << 12, 1 << 11, 1 << 28, 256) == (1 << 23) * (1 << 22) * 17536


def test_workspace_bytes():
    f = F.cache_workspace_bytes
    assert f(2, 3, 4, 5, 64, 1) == 0
    assert f(2, 3, 4, 5, 64, 1, True) == 2 * 3 * 4 * 5 * 16
    # records of d + 4 floats, and 8 bytes for each head's row tile (20 rows: one), per split
    assert f(2, 3, 4, 5, 64, 7) == 120 * 7 * 68 * 4 + 6 * 7 * 8
    assert f(2, 3, 4, 5, 64, 7, True) == 120 * 7 * 68 * 4 + 120 * 16 + 6 * 7 * 8
    for args in ((0, 1, 1, 1, 64, 1), (1, 1, 1, 1, 64, 0), (1, 1, 1, 1, 64, 65), (1, 1, 0, 1, 64, 1),
                 (1 << 10, 1 << 10, 1 << 10, 2, 64, 1), (1, 1, 1, 1, 80, 1)):
        with pytest.raises(F.FabftError):
            f(*args)


def test_splits():
    """At least one, at most 64, never more than there are tiles, no more work than the chip
    holds once the heads and rows fill it."""
    for B in (1, 3, 16, 300):
        for H in (1, 8, 32):
            for G, Lq in ((1, 1), (4, 1), (8, 4), (1, 700)):
                for cap in (64, 128, 4096, 32768, 1 << 20):
                    n = F.cache_splits(B, H, G, Lq, cap)
                    assert 1 <= n <= 64 and n <= cap // 64
                    if B * H >= 1024:
                        assert n == 1
    for args in ((0, 1, 1, 1, 64), (1, 1, 1, 0, 64), (1, 1, 1 << 20, 1 << 20, 64), (1, 1, 1, 1, 0)):
        with pytest.raises(F.FabftError):
            F.cache_splits(*args)


def append(**kw):
    a = dict(cache=P, B=1, H=1, capacity=64, d=64, k=P, v=P, n=1, strides=None, start=P, counts=None)
    a.update(kw)
    if a["strides"]:
        a["strides"] = (ctypes.c_longlong * 6)(*a["strides"])
    return F.lib().fabft_cache_append(*a.values())


def read(**kw):
    a = dict(cache=P, B=1, H=1, capacity=64, d=64, k=P, v=P, n=1, start=P, counts=None)
    a.update(kw)
    return F.lib().fabft_cache_read(*a.values())


def attn(**kw):
    a = dict(q=P, cache=P, o=P, resid=P, flags=P, B=1, H=1, G=1, Lq=1, capacity=64, d=64, lengths=P,
             counts=None, causal=0, scale=1.0, weight=None, decay=1.0, nsplit=1, workspace=P,
             workspace_bytes=BIG)
    a.update(kw)
    return F.lib().fabft_attn_fwd_cache(*a.values())


def evict(**kw):
    a = dict(cache=P, B=1, H=1, capacity=128, d=64, weight=BIG, lengths=P, keep=10, recent=0,
             into=2 * BIG, into_capacity=64, into_weight=3 * BIG, index=P, new_lengths=4 * P)
    a.update(kw)
    return F.lib().fabft_cache_evict(*a.values())


@pytest.mark.parametrize("call,kw,code", [
    (append, dict(cache=0), F.E_NULL), (append, dict(k=0), F.E_NULL), (append, dict(v=0), F.E_NULL),
    (append, dict(start=0), F.E_NULL), (append, dict(d=80), F.E_HEADDIM),
    (append, dict(capacity=100), F.E_SHAPE), (append, dict(n=0), F.E_SHAPE),
    (append, dict(B=0), F.E_SHAPE), (append, dict(cache=P + 8), F.E_ALIGN),
    (append, dict(k=P + 2), F.E_ALIGN), (append, dict(v=P + 8), F.E_ALIGN),
    (append, dict(strides=[0, 0, 60, 0, 0, 64]), F.E_ALIGN),
    (append, dict(strides=[0, 0, 64, 4, 0, 64]), F.E_ALIGN),
    (read, dict(cache=0), F.E_NULL), (read, dict(k=0), F.E_NULL), (read, dict(start=0), F.E_NULL),
    (read, dict(n=-1), F.E_SHAPE), (read, dict(v=P + 8), F.E_ALIGN), (read, dict(d=0), F.E_HEADDIM),
    (attn, dict(q=0), F.E_NULL), (attn, dict(cache=0), F.E_NULL), (attn, dict(o=0), F.E_NULL),
    (attn, dict(resid=0), F.E_NULL), (attn, dict(flags=0), F.E_NULL), (attn, dict(lengths=0), F.E_NULL),
    (attn, dict(nsplit=2, workspace=0), F.E_NULL), (attn, dict(weight=P, workspace=0), F.E_NULL),
    (attn, dict(d=512), F.E_HEADDIM), (attn, dict(G=0), F.E_SHAPE), (attn, dict(Lq=0), F.E_SHAPE),
    (attn, dict(capacity=96), F.E_SHAPE), (attn, dict(nsplit=0), F.E_SHAPE),
    (attn, dict(nsplit=65), F.E_SHAPE), (attn, dict(G=1 << 20, Lq=1 << 20), F.E_SHAPE),
    (attn, dict(scale=-1.0), F.E_SCALE), (attn, dict(scale=float("nan")), F.E_SCALE),
    (attn, dict(scale=float("inf")), F.E_SCALE), (attn, dict(weight=P, decay=-0.5), F.E_SCALE),
    (attn, dict(weight=P, decay=float("nan")), F.E_SCALE),
    (attn, dict(q=P + 8), F.E_ALIGN), (attn, dict(o=P + 2), F.E_ALIGN),
    (attn, dict(nsplit=2, workspace=P + 4), F.E_ALIGN),
    (attn, dict(nsplit=2, workspace_bytes=2 * 68 * 4 - 1), F.E_WORKSPACE),
    (attn, dict(weight=P, workspace_bytes=15), F.E_WORKSPACE),
    (evict, dict(cache=0), F.E_NULL), (evict, dict(weight=0), F.E_NULL), (evict, dict(into=0), F.E_NULL),
    (evict, dict(into_weight=0), F.E_NULL), (evict, dict(index=0), F.E_NULL),
    (evict, dict(new_lengths=0), F.E_NULL), (evict, dict(keep=0), F.E_SHAPE),
    (evict, dict(keep=65), F.E_SHAPE), (evict, dict(recent=11), F.E_SHAPE),
    (evict, dict(recent=-1), F.E_SHAPE), (evict, dict(into_capacity=100), F.E_SHAPE),
    # overlapping caches, weights, lengths
    (evict, dict(into=P), F.E_SHAPE), (evict, dict(into=P + 4864), F.E_SHAPE),
    (evict, dict(into=P, into_capacity=128), F.E_SHAPE),
    (evict, dict(into_weight=BIG + 508), F.E_SHAPE), (evict, dict(new_lengths=P), F.E_SHAPE),
    (evict, dict(into=2 * BIG + 8), F.E_ALIGN),
], ids=str)
def test_refused_by_the_library(call, kw, code):
    assert call(**kw) == code, kw


PROLOGUE = """
import torch
import paper_2507_16676_amd as F

class T(torch.Tensor):
    # a CPU tensor that says it is on a GPU: enough to be refused for something else
    is_cuda = True

def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(T)

i = lambda n=2: t(n, dtype=torch.int32)
n = F.lib().fabft_cache_bytes(2, 3, 64, 64)
c = F.Cache(t(2, 3, 1, n // 6, dtype=torch.uint8), 2, 3, 64, 64)
w = t(2, 3, 64, dtype=torch.float32)
bad = object()
for call in CALLS:
    try:
        eval(call)
        print("passed:", call)
    except (ValueError, TypeError, F.FabftError) as e:
        print("refused:", type(e).__name__)
"""

CALLS = [
    "F.cache_append(bad, t(2, 3, 1, 64), t(2, 3, 1, 64), i())",
    "F.cache_append(c, t(2, 3, 1, 64, dtype=torch.float32), t(2, 3, 1, 64), i())",
    "F.cache_append(c, t(2, 3, 1, 64), t(2, 3, 2, 64), i())",
    "F.cache_append(c, t(2, 4, 1, 64), t(2, 4, 1, 64), i())",
    "F.cache_append(c, t(2, 3, 1, 96), t(2, 3, 1, 96), i())",
    "F.cache_append(c, t(2, 3, 64, 1).expand(2, 3, 64, 64), t(2, 3, 64, 64), i())",
    "F.cache_append(c, t(2, 3, 1, 64), t(2, 3, 1, 64), t(2))",
    "F.cache_append(c, t(2, 3, 1, 64), t(2, 3, 1, 64), i(3))",
    "F.cache_append(c, t(2, 3, 1, 64), t(2, 3, 1, 64), 5)",
    "F.cache_append(c, t(2, 3, 1, 64), t(2, 3, 1, 64), i(), counts=i(1))",
    "F.cache_append(F.Cache(c.data, 2, 3, 128, 64), t(2, 3, 1, 64), t(2, 3, 1, 64), i())",
    "F.cache_append(F.Cache(c.data, 2, 3, 100, 64), t(2, 3, 1, 64), t(2, 3, 1, 64), i())",
    "F.cache_read(c, i(), -1)",
    "F.cache_read(c, i(), 2, out=(t(2, 3, 2, 64), t(2, 3, 3, 64)))",
    "F.cache_read(c, i(), 2, out=(t(2, 3, 2, 64),))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), bad, i())",
    "F.attn_fwd_cache(t(2, 4, 1, 64), c, i())",
    "F.attn_fwd_cache(t(2, 2, 1, 64), c, i())",
    "F.attn_fwd_cache(t(1, 3, 1, 64), c, i())",
    "F.attn_fwd_cache(t(2, 3, 1, 128), c, i())",
    "F.attn_fwd_cache(t(2, 3, 0, 64), c, i())",
    "F.attn_fwd_cache(t(2, 3, 1, 64, dtype=torch.float16), c, i())",
    "F.attn_fwd_cache(t(2, 3, 64, 1).transpose(2, 3), c, i(1))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, torch.zeros(2, dtype=torch.int64))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), counts=i(5))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), weight=t(2, 3, 63, dtype=torch.float32))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), weight=t(2, 3, 64))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), nsplit=0)",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), nsplit=2, workspace=t(10, dtype=torch.uint8))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), nsplit=2, workspace=bad)",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), out=(t(2, 3, 1, 64), bad, bad))",
    "F.attn_fwd_cache(t(2, 3, 1, 64), c, i(), out=(t(2, 3, 1, 64),))",
    "F.cache_evict(c, w, i(), 0)",
    "F.cache_evict(c, w, i(), 65)",
    "F.cache_evict(c, w, i(), 10, recent=11)",
    "F.cache_evict(c, w, i(), 10, into=c)",
    "F.cache_evict(c, w, i(), 10, into_weight=w)",
    "F.cache_evict(c, w, i(), 10, into=bad, into_weight=w)",
    "F.cache_evict(c, w, i(), 10, into=c, into_weight=t(2, 3, 63, dtype=torch.float32))",
    "F.cache_evict(c, t(2, 3, 64), i(), 10)",
    "F.cache_evict(c, w, i(3), 10)",
    "F.cache_new(1, 1, 64, 80)",
    "F.cache_new(0, 1, 64, 64)",
    "F.cache_new(1, 1, 0, 64)",
    "F.cache_new(1, 1, 64, 64, device='cpu')",
]


def test_refused_by_the_binding():
    r = subprocess.run([sys.executable, "-c", f"CALLS = {CALLS!r}\n" + PROLOGUE], cwd=ROOT, text=True,
                       capture_output=True, timeout=600)
    lines = r.stdout.splitlines()
    assert r.returncode == 0 and len(lines) == len(CALLS), r.stdout + r.stderr
    assert all(x.startswith("refused:") for x in lines), "\n".join(lines)


@pytest.mark.parametrize("call", [
    "F.cache_new(0, 1, 1, 64)", "F.cache_splits(0, 1, 1, 1, 64)",
    "F.cache_workspace_bytes(0, 1, 1, 1, 64, 1)",
    "F.cache_append(bad, bad, bad, bad)", "F.cache_read(bad, bad, 1)",
    "F.attn_fwd_cache(bad, bad, bad)", "F.cache_evict(bad, bad, bad, 1)",
], ids=lambda c: c[2:c.index("(")])
def test_first_call_of_a_process(call):
    code = f"""
import paper_2507_16676_amd as F
bad = object()
try:
    {call}
except (F.FabftError, TypeError) as e:
    print("refused:", e)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, text=True, capture_output=True, timeout=600)
    assert r.returncode == 0 and r.stdout.startswith("refused:"), r.stdout + r.stderr


@pytest.mark.parametrize("call,kw", [
    # rows whose 32-bit indexes would overflow
    (append, dict(n=(1 << 30) + 1)), (append, dict(n=(1 << 31) - 1, strides=[0] * 6)),
    (read, dict(n=(1 << 31) - 1)), (attn, dict(Lq=(1 << 31) - 1)), (attn, dict(G=(1 << 30) + 1)),
    # more workgroups than a grid holds: 2^24 of 256 threads, 2^22 of 1,024
    (append, dict(B=1 << 12, H=1 << 12, n=64)), (append, dict(B=1 << 12, H=1 << 11, d=256, n=63)),
    (attn, dict(B=1 << 12, H=1 << 12)), (attn, dict(B=1 << 10, H=1 << 10, nsplit=16, capacity=1024)),
    (attn, dict(B=1 << 12, H=1 << 12, G=64)), (attn, dict(B=1 << 12, H=1 << 12, weight=P)),
    (evict, dict(B=1 << 10, H=1 << 11, weight=BIG, into=1 << 50, into_weight=1 << 60)),
], ids=str)
def test_more_than_a_launch_holds(call, kw):
    assert call(**kw) == F.E_SHAPE


def test_row_counts_of_the_sizes():
    for f, last in ((F.cache_workspace_bytes, (64, 2)), (F.cache_splits, (64,))):
        assert f(1, 1, 1, 1 << 30, *last) > 0 and f(1, 1, 1 << 15, 1 << 15, *last) > 0
        for args in ((1, 1, 1, (1 << 31) - 1), (1, 1, 1 << 15, (1 << 15) + 1), (2, 1, 1, 1 << 30)):
            with pytest.raises(F.FabftError):
                f(*args, *last)


@pytest.mark.parametrize("weight", [None, BIG])
@pytest.mark.parametrize("q,o", [(P, P), (P, P + 16), (P + 2 * 3 * 4 * 5 * 128 - 16, P)])
def test_outputs_over_the_queries_are_refused(q, o, weight):
    """The second pass of a call with weights reads q again."""
    assert attn(q=q, o=o, B=2, H=3, G=4, Lq=5, weight=weight) == F.E_SHAPE


def test_outputs_over_the_queries_are_refused_by_the_binding():
    code = f"CALLS = {['f(q, 0)', 'f(q, 0, weight=w)', 'f(q, 64)', 'f(q, -64)']!r}\n" + PROLOGUE.split("bad = object()")[0] + """
buf = t(3 * 2 * 3 * 4 * 64)
n = 2 * 3 * 4 * 64
q = buf[n:2 * n].view(2, 3, 4, 64)
def f(q, by, **kw):
    out = (buf[n + by:2 * n + by].view(2, 3, 4, 64), t(2, 3, 4, dtype=torch.float32),
           t(2, 3, 4, dtype=torch.uint8))
    return F.attn_fwd_cache(q, c, i(), out=out, **kw)
for call in CALLS:
    try:
        eval(call)
        print("passed")
    except ValueError as e:
        print("overlap" in str(e))
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, text=True, capture_output=True, timeout=600)
    assert r.returncode == 0 and r.stdout.split() == ["True"] * 4, r.stdout + r.stderr


def test_workspace_error_names_its_sizes():
    with pytest.raises(F.FabftError, match="fabft_cache_workspace_bytes"):
        F._check(attn(nsplit=2, workspace_bytes=0), "fabft_attn_fwd_cache")
