"""The 4-bit key/value cache on the GPU through the package: append and read
value by value, the attention against the fp64 oracle on the cache's values,
the keys' weights, eviction, and a decode loop that uses all of them."""
import math

import numpy as np
import pytest
import torch

import oracle
import workloads as W
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu

F = pytest.importorskip("paper_2507_16676_amd")


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def draw(seed, *shape, spread=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape).astype(np.float32)
    if spread:
        x *= (2.0 ** rng.integers(-spread, spread + 1, size=shape[:-1] + (1,))).astype(np.float32)
    return G.to_dev(W.f32_to_bf16_bits(x))


def values(k, v):
    """The values that the cache holds of rows k and v, by the oracle."""
    return oracle.cache_k(G.from_dev_bf16(k)), oracle.cache_v(G.from_dev_bf16(v))


def filled(B, H, cap, d, seed, n=None, spread=0, k=None):
    """A cache of n rows, and their values (fp64)."""
    n = cap if n is None else n
    k = draw(seed, B, H, n, d, spread=spread) if k is None else k
    v = draw(seed + 1, B, H, n, d, spread=spread)
    c = F.cache_new(B, H, cap, d)
    F.cache_append(c, k, v, ints([0] * B))
    return (c, *values(k, v))


# ---- append and read

@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_values(d):
    """What is read is what the oracle says, bit for bit: sizes from 2^-30 to 2^30 row by row,
    borders between codes, tiny and huge values, zeros."""
    k, v = draw(1, 2, 3, 130, d, spread=30), draw(2, 2, 3, 130, d, spread=30)
    edge = torch.tensor([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 6.5, 7, -.25, -.75, -5, .126, -6],
                        dtype=torch.bfloat16, device="cuda").repeat(d // 16)
    for i, f in enumerate((1.0, 2.0 ** 100, 2.0 ** -98, 2.0 ** -104, 2.0 ** -126, 3.0, 0.0, 2.0 ** 125,
                           5.0 / 7)):
        k[0, 0, i], v[0, 0, i] = edge * f, edge * f
        k[0, 1, i], v[0, 1, i] = edge[:16].repeat(d // 16) * f, (edge / 8 * f)
    c = F.cache_new(2, 3, 192, d)
    F.cache_append(c, k, v, ints([0, 60]))
    kr, vr = F.cache_read(c, ints([0, 60]), 130)
    ke, ve = values(k, v)
    assert np.array_equal(G.from_dev_bf16(kr), ke)
    assert np.array_equal(G.from_dev_bf16(vr), ve)


def test_every_bf16_number():
    """All 65,536 patterns as the largest of a row (the others at ratios of it), both halves of a
    row; NaN and infinities make K's 32 channels, and V's row, NaN."""
    u = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    x = W.bf16_bits_to_f32(u)
    ratio = np.linspace(0, 1, 32, dtype=np.float32)
    with np.errstate(all="ignore"):
        row = x[:, None] * ratio[None, ::-1]
    row = np.concatenate([row, np.full_like(row, 0.3)], axis=1).reshape(1, 1, 65536, 64)
    t = G.to_dev(W.f32_to_bf16_bits(row))
    c = F.cache_new(1, 1, 65536, 64)
    F.cache_append(c, t, t, ints([0]))
    kr, vr = F.cache_read(c, ints([0]), 65536)
    ke, ve = values(t, t)
    assert np.array_equal(G.from_dev_bf16(kr), ke, equal_nan=True)
    assert np.array_equal(G.from_dev_bf16(vr), ve, equal_nan=True)


@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("n", [1, 3, 64, 70])
def test_append_touches_its_rows_only(n, d):
    """Rows at any slot, a padded batch, rows before slot 0 and past the capacity: what other slots
    hold stays, bit for bit."""
    B, H, cap = 4, 2, 128
    c, k0, v0 = filled(B, H, cap, d, 3)
    k, v = draw(5, B, H, n, d), draw(6, B, H, n, d)
    start, counts = [61, -2, cap - 1, 5], [n, n, n, (n + 1) // 2]
    F.cache_append(c, k, v, ints(start), counts=ints(counts))
    ke, ve = values(k, v)
    for b in range(B):
        for i in range(counts[b]):
            s = start[b] + i
            if 0 <= s < cap:
                k0[b, :, s], v0[b, :, s] = ke[b, :, i], ve[b, :, i]
    kr, vr = F.cache_read(c, ints([0] * B), cap)
    assert np.array_equal(G.from_dev_bf16(kr), k0)
    assert np.array_equal(G.from_dev_bf16(vr), v0)


def test_read_zeros_outside():
    c, k0, v0 = filled(2, 1, 64, 64, 7)
    kr, vr = F.cache_read(c, ints([-3, 60]), 10, counts=ints([10, 3]))
    k, v = G.from_dev_bf16(kr), G.from_dev_bf16(vr)
    assert np.all(k[0, 0, :3] == 0) and np.array_equal(k[0, 0, 3:], k0[0, 0, :7])
    assert np.array_equal(v[1, 0, :3], v0[1, 0, 60:63]) and np.all(v[1, 0, 3:] == 0)


def test_read_of_more_than_a_grid_dimension():
    """More rows than one dimension of a grid has workgroups for: 2^29 before the cache's 64."""
    far = 1 << 29
    if torch.cuda.mem_get_info()[0] < 180 << 30:
        pytest.skip("needs 130 GiB of device memory")
    c, k0, v0 = filled(1, 1, 64, 64, 8)
    kr, vr = F.cache_read(c, ints([-far - 36]), far + 100)
    for x, e in ((kr, k0), (vr, v0)):
        assert np.array_equal(G.from_dev_bf16(x[:, :, far + 36:]), e)
        y = x[0, 0, :far + 36].view(torch.int32).flatten()
        assert not any(bool(p.any()) for p in y.split(1 << 30))
    del kr, vr, x, y
    torch.cuda.empty_cache()


def test_append_strides():
    """[B, n, H, d] projections seen as [B, H, n, d], a slice of wider rows, one row for all heads."""
    B, H, n, d = 2, 3, 5, 96
    kw, vw = draw(8, B, n, H, 2 * d), draw(9, B, 1, n, d)
    k, v = kw.transpose(1, 2)[..., d:], vw.expand(B, H, n, d)
    c = F.cache_new(B, H, 64, d)
    F.cache_append(c, k, v, ints([0, 7]))
    kr, vr = F.cache_read(c, ints([0, 7]), n)
    ke, ve = values(k.contiguous(), v.contiguous())
    assert np.array_equal(G.from_dev_bf16(kr), ke)
    assert np.array_equal(G.from_dev_bf16(vr), ve)


# ---- attention

def check_attention(q, c, ke, ve, lengths, counts, causal, scale, weight=None, decay=1.0, rows=None,
                    **kw):
    """One call against the oracle, element by element. The bounds: a softmax weight is rounded
    to bf16 once (half a step: 2^-8 of it) and O once more; the scores' fp32 products are off by at
    most 2^-23 d sum |q||k|, which an exponential and its sum turn into twice that times the scale,
    relative to P; 2^-18 covers the fp32 sums, exponentials and the division."""
    B, HG, Lq, d = q.shape
    H = c.H
    w0 = None if weight is None else weight.double().cpu().numpy().copy()
    o, resid, flags = F.attn_fwd_cache(q, c, ints(lengths), causal=causal, scale=scale, weight=weight,
                                       decay=decay, counts=None if counts is None else ints(counts),
                                       **kw)
    torch.cuda.synchronize()
    O, r = G.from_dev_bf16(o).reshape(B, H, -1, Lq, d), resid.cpu().numpy().reshape(B, H, -1, Lq)
    Q = G.from_dev_bf16(q).reshape(B, H, -1, Lq, d)
    assert int(flags.sum()) == 0
    wn = None if weight is None else weight.double().cpu().numpy()
    for b in range(B):
        m = Lq if counts is None else counts[b]
        for h in range(H):
            eo, ea, pred, ew = oracle.cache_attention(Q[b, h], ke[b, h], ve[b, h], lengths[b], m, causal,
                                                      scale)
            n = max(1, lengths[b])
            qk = (np.abs(np.nan_to_num(Q[b, h])) @ np.abs(ke[b, h, :n]).T).max()
            rel = 2.0 * scale * 2.0 ** -23 * d * qk + 2.0 ** -18
            lim = 2.0 ** -8 * (1 + 2.0 ** -8) * (ea + np.abs(eo)) + rel * ea
            bad = np.abs(O[b, h] - eo) > lim
            assert not bad.any(), (b, h, np.argwhere(bad)[:3], np.abs(O[b, h] - eo).max())
            M = np.abs(eo).sum(-1) + np.abs(pred)
            assert np.all(np.abs(r[b, h]) <= F.get_threshold()[0] / 4 * M + 1e-30)
            if weight is not None:
                want = ew if decay == 0 else decay * w0[b, h] + ew
                # the sum of Lq G terms and the product and sum with the old weight
                lim = rel * ew + 2.0 ** -24 * (Lq * Q.shape[2] + 2) * np.abs(want) + 1e-30
                at = slice(0, lengths[b])
                assert np.all(np.abs(wn[b, h] - want)[at] <= lim[at])
                assert np.array_equal(wn[b, h, lengths[b]:], w0[b, h, lengths[b]:])
    return o, resid, flags


CASES = [
    # B, H, G, Lq, capacity, d, causal, lengths, counts, nsplit
    (1, 1, 1, 1, 64, 128, False, [1], None, None),
    (1, 1, 1, 1, 64, 64, True, [64], None, None),
    (2, 3, 1, 1, 320, 128, True, [257, 64], None, 1),
    (2, 3, 1, 1, 1024, 64, False, [1000, 65], None, 3),
    (3, 2, 4, 1, 640, 96, True, [640, 1, 63], None, 4),
    (2, 2, 3, 1, 704, 256, False, [700, 129], None, None),
    (1, 2, 8, 2, 512, 128, True, [500], None, 2),          # 16 rows
    (1, 2, 1, 17, 320, 128, True, [300], None, 1),         # 17 rows: two operands
    (2, 1, 4, 5, 512, 256, True, [512, 5], None, 5),
    (1, 2, 3, 33, 1100, 64, True, [1087], None, 3),        # row tiles that span two heads
    (2, 8, 1, 70, 384, 96, True, [384, 200], None, 2),     # eight heads per XCD round, several tiles
    (2, 4, 2, 129, 320, 128, True, [320, 129], None, None),
    (1, 1, 2, 40, 256, 256, False, [255], None, 1),
    (4, 2, 2, 4, 256, 128, True, [200, 4, 3, 0], [4, 2, 4, 1], 2),    # padding, rows without keys
    (3, 1, 1, 6, 192, 64, False, [192, 100, 7], [0, 6, 9], 3),        # no row; a count past Lq
    (2, 1, 2, 1, 256, 96, True, [-5, 1000], None, 2),                 # lengths are clamped
    (1, 2, 2, 1, 4160, 128, False, [4150], None, 64),                 # more splits than work for
    (1, 8, 2, 1, 8192, 64, True, [70], None, 32),                     # a nearly empty cache
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "b{}h{}g{}q{}c{}d{}".format(*c[:6]))
def test_attention(case):
    B, H, Gq, Lq, cap, d, causal, lengths, counts, ns = case
    print(f"[cache attention] {case}", flush=True)
    c, ke, ve = filled(B, H, -(-cap // 64) * 64, d, 11)
    q = draw(13, B, H * Gq, Lq, d)
    weight = torch.rand((B, H, c.capacity), device="cuda")
    lens = [min(max(n, 0), c.capacity) for n in lengths]
    cnt = None if counts is None else [min(n, Lq) for n in counts]
    args = dict(lengths=lens, counts=cnt, causal=causal, scale=d ** -0.5)
    if lens != lengths or cnt != counts:     # as given: the kernel clamps them
        o1, _, _ = F.attn_fwd_cache(q, c, ints(lengths), causal=causal, nsplit=ns,
                                    counts=None if counts is None else ints(counts))
        o2, _, _ = F.attn_fwd_cache(q, c, ints(lens), causal=causal, nsplit=ns,
                                    counts=None if cnt is None else ints(cnt))
        assert torch.equal(o1, o2)
    a = check_attention(q, c, ke, ve, nsplit=ns, weight=weight, decay=0.75, **args)
    # without the weights, and again: bit for bit
    b = F.attn_fwd_cache(q, c, ints(lens), causal=causal, nsplit=ns,
                         counts=None if cnt is None else ints(cnt))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # the mean of all visible keys
    check_attention(q, c, ke, ve, lens, cnt, causal, 0.0, weight=weight, decay=0.0, nsplit=ns)


# more than 12 tiles: the splits are merged, in the last workgroup, or with many rows and splits
# by a launch of their own; 1, up to 4, 8, 16 and 32 rows a workgroup, and several of those
MERGES = [
    # B, H, G, Lq, capacity, d, lengths, nsplit
    (2, 2, 1, 1, 2048, 128, [2047, 833], None),
    (4, 1, 1, 1, 3200, 64, [3200, 70, 0, 1500], 13),
    (1, 3, 3, 1, 1600, 96, [1599], 5),
    (2, 8, 2, 2, 1024, 256, [1024, 900], 4),
    (1, 2, 8, 1, 6400, 128, [6399], 64),          # apart
    (3, 1, 2, 4, 1500, 64, [1500, 2, 1100], 7),
    (1, 1, 4, 4, 5000, 256, [4999], 32),          # apart
    (2, 2, 5, 2, 1700, 96, [1700, 1300], 9),
    (1, 1, 2, 16, 2100, 128, [2050], 3),
    (1, 2, 1, 29, 2304, 64, [2304], 31),          # apart
    (2, 1, 3, 37, 1100, 128, [1100, 850], 4),     # several row tiles
    (1, 1, 1, 70, 1300, 256, [1290], 5),
]


@pytest.mark.parametrize("case", MERGES, ids=lambda c: "b{}h{}g{}q{}c{}d{}".format(*c[:6]))
def test_merge(case):
    B, H, Gq, Lq, cap, d, lengths, ns = case
    print(f"[cache merge] {case}", flush=True)
    c, ke, ve = filled(B, H, -(-cap // 64) * 64, d, 35)
    q = draw(36, B, H * Gq, Lq, d)
    weight = torch.rand((B, H, c.capacity), device="cuda")
    w0 = weight.clone()
    a = check_attention(q, c, ke, ve, lengths, None, True, d ** -0.5, weight=weight, nsplit=ns)
    for _ in range(5):     # whichever workgroup comes last: bit for bit
        w = w0.clone()
        b = F.attn_fwd_cache(q, c, ints(lengths), causal=True, nsplit=ns, weight=w)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(w, weight)
    # and as without splits, to rounding
    one, _, _ = F.attn_fwd_cache(q, c, ints(lengths), causal=True, nsplit=1)
    assert float((one.float() - a[0].float()).abs().max()) <= 2.0 ** -6 * float(one.float().abs().max())


def test_longest_first():
    """More workgroups than fit at once, of sequences of different lengths and row counts."""
    B, H, Gq, Lq, cap, d = 4, 16, 2, 192, 448, 64
    c, ke, ve = filled(B, H, cap, d, 37)
    check_attention(draw(38, B, H * Gq, Lq, d), c, ke, ve, [200, 448, 0, 448], [192, 100, 7, 192], True,
                    d ** -0.5, weight=torch.zeros((B, H, cap), device="cuda"))


def test_large_caches():
    """Caches beside which the memory-side cache is small are read, filled and listed as streams:
    the results are those of a small one, bit for bit."""
    H, d, n = 8, 128, 1100
    c, ke, ve = filled(1, H, 1152, d, 39)
    big = F.cache_new(1, H, 131072, d)
    k, v = F.cache_read(c, ints([0]), n)
    F.cache_append(big, k, v, ints([0]))      # (the values are their own nearest ones)
    for G, Lq in ((1, 1), (4, 1), (8, 1), (4, 4)):
        q = draw(40, 1, H * G, Lq, d)
        for ns in (1, 4):
            a = F.attn_fwd_cache(q, c, ints([n]), causal=True, nsplit=ns)
            b = F.attn_fwd_cache(q, big, ints([n]), causal=True, nsplit=ns)
            assert torch.equal(a[0], b[0]) and int(b[2].sum()) == 0
    n, d = 98_500, 256
    k, v = draw(41, 1, 1, n, d), draw(42, 1, 1, n, d)
    c = F.cache_new(1, 1, n, d)
    F.cache_append(c, k, v, ints([0]))
    kr, vr = F.cache_read(c, ints([0]), n)
    for at in (0, 40_000, n - 3000):
        part = F.cache_new(1, 1, 3008, d)
        F.cache_append(part, k[:, :, at:at + 3000], v[:, :, at:at + 3000], ints([0]))
        kp, vp = F.cache_read(part, ints([0]), 3000)
        assert torch.equal(kr[:, :, at:at + 3000], kp) and torch.equal(vr[:, :, at:at + 3000], vp)


@pytest.mark.parametrize("rows", [(1, 3), (4, 17)])
def test_nan_keys_leave_the_weights(rows):
    """Keys of NaN in the middle of the cache: all rows that see them are flagged and add nothing,
    the keys' own weights included; rows that do not see them add theirs."""
    G, Lq = rows
    H, cap, d = 2, 320, 64
    k, v = draw(43, 1, H, cap, d), draw(44, 1, H, cap, d)
    k[0, 0, 100, 5] = float("nan")
    v[0, 1, 305, 7] = float("inf")
    c = F.cache_new(1, H, cap, d)
    F.cache_append(c, k, v, ints([0]))
    w = torch.full((1, H, cap), 0.5, device="cuda")
    q = draw(45, 1, H * G, Lq, d)
    o, _, flags = F.attn_fwd_cache(q, c, ints([cap]), causal=True, weight=w)
    assert bool((flags[:, :G] & F.FLAG_NONFINITE).bool().all()) and bool((w[:, 0] == 0.5).all())
    seen = torch.arange(cap - Lq, cap, device="cuda") >= 305
    assert torch.equal((flags[0, G:] != 0), seen.expand(G, Lq))
    assert bool(torch.isfinite(w).all())
    assert abs(float(w[0, 1].double().sum()) - 0.5 * cap - G * int((~seen).sum())) < 1e-3


@pytest.mark.parametrize("nsplit", [1, 16])
@pytest.mark.parametrize("G_,Lq", [(1, 1), (2, 2), (8, 5)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_scores_that_overflow(d, G_, Lq, nsplit):
    """Rows whose scores are all -inf have no weights: NaN and flagged, and they add nothing to
    the keys' weights; with some at -inf those keys have the weight 0."""
    cap, n = 4096, 4000
    x = torch.full((1, 2, n, d), 1e38, dtype=torch.bfloat16, device="cuda")
    x[0, 1, ::2] = 2.0 ** -100      # head 1: every other key has a finite score, about 0
    v = draw(33, 1, 2, n, d)
    c = F.cache_new(1, 2, cap, d)
    F.cache_append(c, x, v, ints([0]))
    q = torch.full((1, 2 * G_, Lq, d), -1e38, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(1, 2, cap, device="cuda")
    o, _, flags = F.attn_fwd_cache(q, c, ints([n]), scale=2.0 ** -40, weight=w, nsplit=nsplit)
    assert bool(torch.isnan(o[:, :G_]).all()) and bool((flags[:, :G_] == 3).all())
    assert bool((w[0, 0] == 0).all())
    assert int(flags[:, G_:].sum()) == 0
    mean = oracle.cache_v(G.from_dev_bf16(v))[0, 1, ::2].mean(axis=0)
    # the weights are equal: fp32 sums of 2,000 of them, and the rounding of O
    err = np.abs(G.from_dev_bf16(o[:, G_:]) - mean)
    assert np.all(err <= 2.0 ** -8 * np.abs(mean) + 2.0 ** -12 * np.abs(v.float().cpu().numpy()).max())
    assert bool((w[0, 1, 1::2] == 0).all())
    assert torch.allclose(w[0, 1, :n:2], torch.tensor(G_ * Lq / 2000.0, device="cuda"), rtol=2.0 ** -10)


@pytest.mark.parametrize("nsplit", [1, 4])
@pytest.mark.parametrize("G_,Lq", [(1, 1), (2, 2), (2, 9)])
def test_huge_scores(G_, Lq, nsplit):
    """Scores of 2^20 to 2^60 whose largest is 2^-3 of them or more above the others: O is the V row of
    that key, and from 2^31 on that or NaN and flagged."""
    H, cap, n, d = 2, 1024, 1000, 64
    at = 777
    k = (torch.rand((1, H, n, 1), device="cuda") - 0.5).to(torch.bfloat16).expand(1, H, n, d).contiguous()
    k[:, :, at] = 0.75                      # (the others: 0.5 at most)
    v = draw(34, 1, H, n, d)
    q = torch.ones((1, H * G_, Lq, d), dtype=torch.bfloat16, device="cuda")
    c = F.cache_new(1, H, cap, d)
    F.cache_append(c, k, v, ints([0]))
    ve = oracle.cache_v(G.from_dev_bf16(v))[0, :, at]
    for e in (20, 27, 30, 31, 33, 45, 60):
        for sign in (1.0, 1.0 + 2.0 ** -20, 1.5):
            scale = sign * 2.0 ** e * math.log(2) / (0.75 * d)
            o, _, flags = F.attn_fwd_cache(q, c, ints([n]), scale=scale, nsplit=nsplit)
            O = G.from_dev_bf16(o).reshape(H, -1, d)
            f = flags.cpu().numpy().reshape(H, -1)
            assert np.all((f == 0) | (f & F.FLAG_NONFINITE != 0))
            if e <= 30:
                assert np.all(f == 0)
            for h in range(H):
                ok = f[h] == 0
                # one weight, rounded to bf16, and the rounding of O
                assert np.all(np.abs(O[h][ok] - ve[h]) <= 2.0 ** -6 * np.abs(ve[h]))


@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_attention_peaked(d):
    """Scores that jump late past the lazily kept maximum, and far below it."""
    B, H, cap = 2, 2, 1536
    k = draw(15, B, H, cap, d)
    k[:, :, 700:1400:50] *= 8
    c, ke, ve = filled(B, H, cap, d, 15, k=k)
    for Lq in (1, 20):
        check_attention(draw(16, B, 2 * H, Lq, d), c, ke, ve, [1500, 900], None, True, d ** -0.5,
                        weight=torch.zeros((B, H, cap), device="cuda"))


def test_attention_value_sizes():
    """V rows of sizes from 2^-20 to 2^20 side by side, and all near the smallest scale."""
    B, H, cap, d = 1, 2, 256, 128
    for f in (1.0, 2.0 ** -90, 2.0 ** 90):
        k, v = draw(17, B, H, cap, d), draw(18, B, H, cap, d, spread=20) * f
        c = F.cache_new(B, H, cap, d)
        F.cache_append(c, k, v, ints([0]))
        check_attention(draw(19, B, H, 3, d), c, *values(k, v), [250], None, True, d ** -0.5)


@pytest.mark.parametrize("nsplit", [1, 2])
@pytest.mark.parametrize("G_,Lq", [(1, 1), (2, 2), (1, 8), (2, 8), (4, 8)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_values_up_to_the_bound(d, G_, Lq, nsplit):
    """Keys times the largest sum of |v| over a row just below 2^118, with scores that rise by
    almost 8 (base 2) behind every wave's first tile, where the kept maximum does not follow: right.
    Far above: rows whose sums overflow are flagged, and the others right."""
    H, cap = 2, 1024
    n = 1000
    k = torch.zeros((1, H, n, d), dtype=torch.bfloat16, device="cuda")
    k[:, :, 64 * 4 * nsplit:] = 1.0
    q = torch.ones((1, H * G_, Lq, d), dtype=torch.bfloat16, device="cuda")
    scale = 7.9 * math.log(2) / d
    v0 = draw(20, 1, H, n, d).abs().clamp(0.25, 4.0)
    total = float(oracle.cache_v(G.from_dev_bf16(v0)).sum(-1).max()) * n
    top = 117 - math.floor(math.log2(total))
    assert 2.0 ** 117 <= total * 2.0 ** top < 2.0 ** 118
    for e in (top, -90):
        c = F.cache_new(1, H, cap, d)
        v = v0 * 2.0 ** e
        F.cache_append(c, k, v, ints([0]))
        whole = (np.pad(x, ((0, 0), (0, 0), (0, cap - n), (0, 0))) for x in values(k, v))
        check_attention(q, c, *whole, [n], None, False, scale, nsplit=nsplit,
                        weight=torch.zeros((1, H, cap), device="cuda"))
    for e in range(top + 1, 125, 3):
        c = F.cache_new(1, H, cap, d)
        v = v0 * 2.0 ** e
        F.cache_append(c, k, v, ints([0]))
        o, _, flags = F.attn_fwd_cache(q, c, ints([n]), scale=scale, nsplit=nsplit)
        bad = (flags & F.FLAG_NONFINITE) != 0
        assert bool(torch.isfinite(o)[~bad].all())
        eo, ea, _, _ = oracle.cache_attention(np.ones((G_, Lq, d)), *(x[0, 0] for x in values(k, v)), n, Lq,
                                              False, scale)
        err = np.abs(G.from_dev_bf16(o[:, :G_])[0] - eo)[~bad[0, :G_].cpu().numpy()]
        assert np.all(err <= 2.0 ** -6 * ea.max())


def test_same_as_the_bf16_forward_on_the_read_values():
    """attn_fwd_splitkv over what cache_read gives: the same to the rounding of the weights."""
    B, H, cap, d = 2, 4, 2048, 128
    c, ke, ve = filled(B, H, cap, d, 21)
    q = draw(22, B, H, 4, d)
    k, v = F.cache_read(c, ints([0, 0]), cap)
    o, _, flags = F.attn_fwd_cache(q, c, ints([cap, cap]), causal=True)
    ref, _, rflags = F.attn_fwd_splitkv(q, k, v, causal=True)
    assert int(flags.sum()) == 0 and int(rflags.sum()) == 0
    err = (o.float() - ref.float()).abs()
    assert float(err.max()) <= 2.0 ** -6 * float(ref.float().abs().max())


def test_masked_places_hold_anything():
    """Bytes of all ones (NaN scales) behind the lengths, NaN rows of padding queries, and keys of
    NaN that a causal row does not see, change nothing."""
    B, H, cap, d, Lq = 2, 2, 320, 128, 5
    for d in (64, 96, 128, 256):
        k, v = draw(23, B, H, cap, d), draw(24, B, H, cap, d)
        lengths, counts = [200, 131], [5, 3]
        q = draw(25, B, 2 * H, Lq, d)
        c = F.cache_new(B, H, cap, d)
        c.data.fill_(255)
        for b in range(B):
            F.cache_append(c, k[:, :, :lengths[b]], v[:, :, :lengths[b]],
                           ints([0 if i == b else cap for i in range(B)]))
        ke, ve = values(k, v)
        w = torch.full((B, H, cap), float("nan"), device="cuda")
        for b in range(B):
            w[b, :, :lengths[b]] = 0.25
        q[1, :, 3:] = float("nan")
        weight = w.clone()
        o, resid, flags = F.attn_fwd_cache(q, c, ints(lengths), counts=ints(counts), causal=True,
                                           weight=weight)
        assert int(flags.sum()) == 0 and bool(torch.all(o[1, :, 3:] == 0))
        assert bool(torch.all(resid[1, :, 3:] == 0))
        for b in range(B):
            assert bool(torch.isfinite(weight[b, :, :lengths[b]]).all())
            assert bool(torch.isnan(weight[b, :, lengths[b]:]).all())
        # key 198 is seen by rows 3 and 4 of sequence 0 alone
        k[0, 1, 198, 3] = float("inf")
        v[0, 0, 198, 3] = float("nan")
        F.cache_append(c, k[:, :, 198:199], v[:, :, 198:199], ints([198, cap]))
        w2 = w.clone()
        o2, _, f2 = F.attn_fwd_cache(q, c, ints(lengths), counts=ints(counts), causal=True, weight=w2)
        hit = torch.zeros_like(flags, dtype=torch.bool)
        hit[0, :, 3:] = True
        assert bool(torch.all(((f2 & F.FLAG_NONFINITE) != 0) == hit))
        assert torch.equal(o2[~hit], o[~hit])
        # the rows with a flag add nothing to the weights
        assert bool(torch.isfinite(w2[0, :, :200]).all())
        assert bool((w2[0, :, :200].sum(-1) - 0.25 * 200 - 6).abs().max() < 1e-3)


# Row tiles with rows that see no key, where splits are merged: rows of a workgroup (1 has no
# such row beside others), a merge in the last workgroup and by a launch of its own
PADDED = [
    # B, H, G, Lq, capacity, d, causal, lengths, counts, nsplit
    (4, 2, 1, 1, 1088, 128, True, [1088, 1000, 833, 900], [1, 0, 1, 0], 4),
    (3, 2, 1, 4, 1088, 128, True, [1088, 1000, 833], [2, 0, 9], 4),
    (2, 1, 3, 2, 1600, 96, False, [1599, 900], [1, 2], 6),
    (2, 2, 2, 4, 1152, 256, False, [1150, 1000], [3, 1], 5),
    (2, 2, 4, 3, 2048, 64, True, [2000, 850], [1, 2], 8),            # 12 rows: apart
    (2, 1, 2, 8, 1344, 256, False, [1344, 1100], [5, 8], 4),         # 16 rows: apart
    (3, 1, 1, 20, 1280, 64, True, [1280, 900, 1000], [7, 19, 0], 5),
    (2, 2, 3, 30, 1408, 128, False, [1400, 1000], [29, 3], 4),       # several row tiles
    (1, 1, 2, 801, 832, 64, True, [800], [801], 4),                  # row 0 sees no key beside row 800
]


@pytest.mark.parametrize("case", PADDED, ids=lambda c: "b{}h{}g{}q{}c{}d{}".format(*c[:6]))
def test_rows_without_keys_beside_others(case):
    """Rows behind the counts, and causal rows before the first key, are O = 0, resid = 0, flag 0
    whatever their q holds, and change nothing else: bit for bit as with zeros there."""
    B, H, Gq, Lq, cap, d, causal, lengths, counts, ns = case
    print(f"[cache rows without keys] {case}", flush=True)
    assert ns > 1 and min(lengths) > 12 * F.CACHE_TILE      # (fewer tiles are not split)
    c, ke, ve = filled(B, H, cap, d, 47)
    q = draw(48, B, H * Gq, Lq, d)
    cnt = [min(n, Lq) for n in counts]
    none = torch.zeros((B, Lq), dtype=torch.bool)
    for b in range(B):
        for i in range(Lq):
            none[b, i] = i >= cnt[b] or (causal and lengths[b] - cnt[b] + i < 0)
    none = none[:, None].expand(B, H * Gq, Lq).cuda()
    assert bool(none.any()) and not bool(none.all())
    q[none] = 0
    w0 = torch.rand((B, H, cap), device="cuda")
    weight = w0.clone()
    a = check_attention(q, c, ke, ve, lengths, cnt, causal, d ** -0.5, weight=weight, nsplit=ns)
    assert not bool(a[0][none].any()) and not bool(a[1][none].any())
    inf = float("inf")
    for x in (inf, -inf, 3e38, -3e38, float("nan")):
        for every in (1, 7):              # the whole row, or some channels (NaN from inf * 0 too)
            p, w = q.clone(), w0.clone()
            p[none] = torch.where(torch.arange(d, device="cuda") % every == 0, x, 0.5).to(p.dtype)
            o, resid, flags = F.attn_fwd_cache(p, c, ints(lengths), counts=ints(counts), causal=causal,
                                               scale=d ** -0.5, nsplit=ns, weight=w)
            assert not bool(flags.any()), (x, every, flags.nonzero()[:3])
            assert torch.equal(o, a[0]) and torch.equal(resid, a[1]) and torch.equal(w, weight)


@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_changed_codes_are_flagged(d):
    """A bit of V's codes, or of their sums, that changed in memory since the append fails the
    check of every row that sees it; the paper's check and the weighted one."""
    B, H, cap, n = 1, 2, 192, 150
    c, ke, ve = filled(B, H, cap, d, 27)
    q = draw(28, B, H, 2, d)
    rb = d // 2
    vcode = 64 * rb + 64 * (d // 32)         # tile layout: K codes, K scales, V codes, ...
    vsum = vcode + 64 * rb + 128
    clean = c.data.clone()
    F.set_weighted_check(True)
    try:
        for tile, row, off, bit in ((0, 5, vcode + 5 * rb + 7, 6), (1, 70, vcode + 6 * rb + rb - 1, 1),
                                    (2, 140, vcode + 12 * rb, 2), (1, 70, vsum + 2 * 6 + 1, 6),
                                    (0, 9, vsum + 256 + 2 * 9 + 1, 6)):
            c.data.copy_(clean)
            c.data[0, 1, tile, off] ^= 1 << bit
            _, resid, flags = F.attn_fwd_cache(q, c, ints([n]), scale=0.0)
            assert int(flags[0, 0].sum()) == 0
            assert bool((flags[0, 1] != 0).all()), (tile, off, bit)
        c.data.copy_(clean)
        _, _, flags = F.attn_fwd_cache(q, c, ints([n]))
        assert int(flags.sum()) == 0
    finally:
        F.set_weighted_check(False)


def test_workspace_and_out():
    B, H, cap, d = 2, 2, 1024, 64
    c, ke, ve = filled(B, H, cap, d, 31)
    q = draw(32, B, 2 * H, 1, d)
    need = F.cache_workspace_bytes(B, H, 2, 1, d, 4, True)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out = (torch.empty_like(q), torch.full((B, 2 * H, 1), float("nan"), device="cuda"),
           torch.full((B, 2 * H, 1), 77, dtype=torch.uint8, device="cuda"))
    w = torch.zeros((B, H, cap), device="cuda")
    check_attention(q, c, ke, ve, [1000, 3], None, True, 0.125, weight=w, nsplit=4, workspace=ws,
                    out=out)
    # a second, smaller call in the same workspace
    o, _, _ = F.attn_fwd_cache(q, c, ints([3, 100]), nsplit=3, workspace=ws)
    o2, _, _ = F.attn_fwd_cache(q, c, ints([3, 100]), nsplit=3)
    assert torch.equal(o, o2)


def test_output_beside_the_queries():
    """q and o next to each other in one buffer, either way round; over each other they are refused."""
    B, H, cap, d, Lq = 2, 2, 1024, 64, 3
    c, ke, ve = filled(B, H, cap, d, 45)
    n = B * 2 * H * Lq * d
    x = draw(46, B, 2 * H, Lq, d)
    for at, to in ((0, n), (n, 0)):
        buf = torch.zeros(2 * n, dtype=torch.bfloat16, device="cuda")
        q, o = (buf[i:i + n].view(B, 2 * H, Lq, d) for i in (at, to))
        q.copy_(x)
        out = (o, torch.empty((B, 2 * H, Lq), device="cuda"),
               torch.empty((B, 2 * H, Lq), dtype=torch.uint8, device="cuda"))
        check_attention(q, c, ke, ve, [1000, 900], None, True, 0.125, nsplit=4, out=out,
                        weight=torch.zeros((B, H, cap), device="cuda"))
        assert torch.equal(q, x)
        for bad in (q, buf[n // 2:n // 2 + n].view_as(q)):
            with pytest.raises(ValueError):
                F.attn_fwd_cache(q, c, ints([1000, 900]), out=(bad, *out[1:]))


def test_offsets_past_32_bits():
    """One head of 34 million slots (4.8 GB): rows at its far end are written, read and attended."""
    cap, d, n = 34_000_000 // 64 * 64, 128, 100
    c = F.cache_new(1, 1, cap, d)
    assert c.data.numel() > 2 ** 32
    k, v = draw(33, 1, 1, n, d), draw(34, 1, 1, n, d)
    F.cache_append(c, k, v, ints([cap - n]))
    ke, ve = values(k, v)
    kr, vr = F.cache_read(c, ints([cap - n]), n)
    assert np.array_equal(G.from_dev_bf16(kr), ke) and np.array_equal(G.from_dev_bf16(vr), ve)
    q = 8 * k[:, :, -1:].contiguous()        # scores of its own key far above the others'
    w = torch.zeros((1, 1, cap), device="cuda")
    o, resid, flags = F.attn_fwd_cache(q, c, ints([cap]), scale=1.0, weight=w)
    assert int(flags.sum()) == 0
    assert np.abs(G.from_dev_bf16(o)[0, 0, 0] - ve[0, 0, -1]).max() <= 2.0 ** -7 * np.abs(ve).max()
    assert float(w[0, 0, -1]) > 0.99 and abs(float(w.double().sum()) - 1) < 1e-3
    idx, new = F.cache_evict(c, w, ints([cap]), 5, recent=1, into=F.cache_new(1, 1, 64, d),
                             into_weight=torch.empty((1, 1, 64), device="cuda"))
    assert int(idx[0, 0, -1]) == cap - 1 and int(new) == 5


# ---- eviction

EVICT = [
    # B, H, capacity, d, lengths, keep, recent
    (1, 1, 64, 64, [10], 4, 0),
    (2, 3, 256, 128, [256, 100], 100, 10),
    (3, 2, 2240, 96, [2240, 64, 1], 1500, 1500),
    (2, 2, 2048, 256, [2047, 0], 1025, 1),
    (2, 1, 5056, 64, [5000, 4097], 4096, 64),
    (1, 2, 4096, 128, [4096], 1, 0),
    (1, 2, 4096, 128, [4096], 4095, 0),
]


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("case", EVICT, ids=lambda c: "b{}h{}c{}d{}".format(*c[:4]))
def test_evict(case, ties):
    """Into another cache, then in place: the same slots, values, sums and weights as the oracle's
    choice; nothing else moves."""
    B, H, cap, d, lengths, keep, recent = case
    c, ke, ve = filled(B, H, cap, d, 41)
    rng = np.random.default_rng(42)
    w = rng.standard_normal((B, H, cap)).astype(np.float32)
    if ties:
        w = np.round(w)                # few values, -0 among them
        w[:, :, 3::50] = np.inf
        w[:, :, 7::90] = np.nan
    weight = torch.from_numpy(w).cuda()
    into = F.cache_new(B, H, keep + 70, d)
    into.data.fill_(255)
    iw = torch.full((B, H, into.capacity), 9.0, device="cuda")
    before = c.data.clone()
    index, new = F.cache_evict(c, weight, ints(lengths), keep, recent=recent, into=into, into_weight=iw)
    assert torch.equal(c.data, before)
    assert np.array_equal(weight.cpu().numpy(), w, equal_nan=True)
    behind = c.data.clone()
    index2, new2 = F.cache_evict(c, weight, ints(lengths), keep, recent=recent)
    assert torch.equal(index, index2) and torch.equal(new, new2)
    assert new.tolist() == [min(n, keep) for n in lengths]
    zero, n = ints([0] * B), min(keep + 64, cap)
    kr, vr = (G.from_dev_bf16(t) for t in F.cache_read(into, zero, keep, counts=new))
    ki, vi = (G.from_dev_bf16(t) for t in F.cache_read(c, zero, keep, counts=new))
    got, nw, nwi = index.cpu().numpy(), iw.cpu().numpy(), weight.cpu().numpy()
    for b in range(B):
        for h in range(H):
            at = oracle.cache_keep(w[b, h].astype(np.float64), lengths[b], keep, recent)
            m = len(at)
            assert got[b, h, :m].tolist() == at.tolist() and np.all(got[b, h, m:] == -1)
            for kk, vv in ((kr, vr), (ki, vi)):
                assert np.array_equal(kk[b, h, :m], ke[b, h, at])
                assert np.array_equal(vv[b, h, :m], ve[b, h, at])
            for x in (nw, nwi):
                assert np.array_equal(x[b, h, :m], w[b, h, at], equal_nan=True)
                assert np.all(x[b, h, m:] == 0)
    # the row sums moved along: no flag
    q = draw(43, B, H, 1, d)
    a = F.attn_fwd_cache(q, into, new)
    b = F.attn_fwd_cache(q, c, new)
    assert int(a[2].sum()) == 0 and int(b[2].sum()) == 0
    assert torch.equal(a[0], b[0])


# ---- together

def decode_loop(steps, B, H, Gq, d, cap, budget, recent, run):
    """A prompt and single tokens over a cache of `cap` slots that is cut to `budget` whenever it is
    full; `run` makes one step's calls."""
    k, v = draw(51, B, H, 40, d), draw(52, B, H, 40, d)
    c = F.cache_new(B, H, cap, d)
    w = torch.zeros((B, H, c.capacity), device="cuda")
    lengths = ints([40, 29][:B])
    F.cache_append(c, k, v, ints([0] * B), counts=lengths)
    ke, ve = values(k, v)
    kept = [[list(zip(ke[b, h], ve[b, h]))[:int(lengths[b])] for h in range(H)] for b in range(B)]
    for s in range(steps):
        q, k, v = draw(60 + s, B, H * Gq, 1, d), draw(90 + s, B, H, 1, d), draw(120 + s, B, H, 1, d)
        o, _, flags = run(c, q, k, v, lengths, w)
        lengths = lengths + 1
        ke, ve = values(k, v)
        O, Q, host_w = G.from_dev_bf16(o), G.from_dev_bf16(q), w.double().cpu().numpy()
        assert int(flags.sum()) == 0
        for b in range(B):
            for h in range(H):
                kept[b][h].append((ke[b, h, 0], ve[b, h, 0]))
                K, V = (np.array(x) for x in zip(*kept[b][h]))
                assert len(K) == int(lengths[b])
                qq = Q[b, h * Gq:h * Gq + Gq]
                eo, ea, _, _ = oracle.cache_attention(qq, K, V, len(K), 1, True, d ** -0.5)
                lim = 2.0 ** -8 * (1 + 2.0 ** -8) * (ea + np.abs(eo)) + 2.0 ** -10 * ea
                assert np.all(np.abs(O[b, h * Gq:h * Gq + Gq] - eo) <= lim)
        # every row of every step left a sum of 1 in the weights; evicted ones took theirs along
        if int(lengths.max()) >= cap:
            for b in range(B):
                for h in range(H):
                    n = int(lengths[b])
                    kept[b][h] = [kept[b][h][i] for i in
                                  oracle.cache_keep(host_w[b, h], n, budget, recent)]
            _, lengths = F.cache_evict(c, w, lengths, budget, recent=recent)
    return c, w, lengths


def one_step(c, q, k, v, lengths, w):
    F.cache_append(c, k, v, lengths)
    return F.attn_fwd_cache(q, c, lengths + 1, causal=True, weight=w, decay=0.95)


@pytest.mark.parametrize("d", [64, 128])
def test_decode_with_eviction(d):
    decode_loop(60, 2, 2, 2, d, 64, 48, 16, one_step)


@pytest.mark.parametrize("cap,Gq,n", [(640, 2, 500), (4096, 2, 3000), (4160, 12, 4100)])
def test_decode_from_a_graph(cap, Gq, n):
    """The step captured once on another stream, replayed with new tokens and lengths between eager
    work (one workgroup a head, the merge of splits in the last one, and apart); every replay
    against an eager twin, bit for bit."""
    B, H, d = 2, 2, 128
    caches = [filled(B, H, cap, d, 53)[0] for _ in range(2)]
    ws = [torch.zeros((B, H, cap), device="cuda") for _ in range(2)]
    q, k, v = draw(60, B, H * Gq, 1, d), draw(61, B, H, 1, d), draw(62, B, H, 1, d)
    lengths = ints([n, 63])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one_step(caches[0], q, k, v, lengths, ws[0])      # loads the kernels
    torch.cuda.current_stream().wait_stream(side)
    ws[0].zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        o, resid, flags = one_step(caches[0], q, k, v, lengths, ws[0])
    for i in range(5):
        q.copy_(draw(70 + i, B, H * Gq, 1, d))
        k.copy_(draw(80 + i, B, H, 1, d))
        v.copy_(draw(90 + i, B, H, 1, d))
        g.replay()
        eo, er, ef = one_step(caches[1], q, k, v, lengths, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(o, eo) and torch.equal(resid, er) and torch.equal(flags, ef)
        assert torch.equal(ws[0], ws[1])
        lengths += 1
    assert int(flags.sum()) == 0


def test_two_streams_at_once():
    """Calls of two caches on two streams, interleaved: each call has its own workspace."""
    B, H, d, cap = 2, 4, 96, 2048
    sets = []
    for i in range(2):
        c, _, _ = filled(B, H, cap, d, 54 + 10 * i)
        sets.append((c, draw(56 + i, B, 2 * H, 1, d)))
    n = ints([2000, 1234])
    want = [F.attn_fwd_cache(q, c, n)[0] for c, q in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, (c, q) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                got[i].append(F.attn_fwd_cache(q, c, n)[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_two_graphs_share_a_workspace():
    """Captured calls of different shapes, splits and merges with one workspace, replayed in turn
    and between eager calls with it: each result is the one of a call by itself."""
    calls, graphs = [], []
    shapes = [(2, 2, 1, 1, 4096, 128, 8), (1, 3, 4, 2, 2048, 64, 16), (2, 1, 4, 8, 2048, 128, 5),
              (3, 2, 2, 1, 1024, 256, 4)]
    need = max(F.cache_workspace_bytes(B, H, Gq, Lq, d, ns, True) for B, H, Gq, Lq, _, d, ns in shapes)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for i, (B, H, Gq, Lq, cap, d, ns) in enumerate(shapes):
        c = filled(B, H, cap, d, 60 + 3 * i)[0]
        q, lens = draw(80 + i, B, H * Gq, Lq, d), ints([cap - 5 * b for b in range(B)])
        w = torch.zeros((B, H, cap), device="cuda")
        kw = dict(causal=True, nsplit=ns, decay=0.0)
        w1 = torch.full_like(w, 7)      # (slots behind the lengths stay as they are below)
        alone = (*F.attn_fwd_cache(q, c, lens, weight=w1, **kw), w1)
        out = tuple(torch.empty_like(x) for x in alone[:3])
        call = lambda q=q, c=c, lens=lens, w=w, out=out, kw=kw: F.attn_fwd_cache(
            q, c, lens, weight=w, workspace=ws, out=out, **kw)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        graphs.append(g)
        calls.append((call, (*out, w), alone))
    n = len(calls)
    for turn in range(12):
        for j in range(n):
            i = (j * (1 + turn % 3) + turn) % n
            call, got, alone = calls[i]
            for x in got:
                x.fill_(7)
            graphs[i].replay() if (turn + j) % 3 else call()
            assert all(torch.equal(x, y) for x, y in zip(got, alone)), (turn, i)
