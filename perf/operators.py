"""Performance cases of the 4-bit key/value cache: filling it, attention over it,
and eviction from it, through the package's public entry points.

The cache holds a row of K in blocks of 32 channels, each with a power of two as
its scale, and a row of V with one scale; a value is a number of the grid 0, 0.5,
1, 1.5, 2, 3, 4, 6 (and its negatives) times the scale:

* K: 2^e with e the smallest integer >= -100 that has max|x| < 7 * 2^e;
* V: s, the smallest number of six significant bits >= max|x| / 6 (and >= 2^-100);

x / scale goes to the nearest number of the grid, ties to the even code. All
values are bfloat16 numbers.

A case has a kind:

* ``append``: n new tokens per sequence go into the cache; their values are read back;
* ``attend``: Lq query rows of H * G query heads over H key/value heads. ``causal``:
  the query rows are the last tokens of their sequence. ``pad``: sequences have 1 to
  Lq query rows (a padded batch). ``weight``: every key's softmax weight, summed over
  the query rows and the heads of its group, is added to a running one;
* ``step``: the tokens are appended and attended, with ``weight``;
* ``evict``: the ``recent`` last keys and the others of the largest weight, ``keep`` in
  all, go to a smaller cache, whose values are read back.

``ragged`` sequences have lengths from 1 to L. Inputs are seeded: N(0, 1) in bfloat16,
K with channels of log-normal size and 1% of the keys 4 times as large (sinks). Each
flag says whether a row's output failed its checksum: none does. The residuals are the
rounding of the sums (their exact value is 0) and are not among the outputs.
"""
from __future__ import annotations

import math

import torch

own = False

DIMS = (64, 96, 128, 256)
MOST_BYTES = 6 << 28
MOST_FLOPS = 1.4e11
MOST_PAIRS = 1 << 28        # (query row, key) pairs of all heads


def _case(name, kind, B, H, G, d, L, Lq=1, causal=True, pad=False, weight=False, ragged=False,
          keep=0, recent=0):
    c = dict(kind=kind, B=B, H=H, G=G, d=d, L=L, Lq=Lq, causal=causal, pad=pad, weight=weight,
             ragged=ragged, keep=keep, recent=recent)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one new token per sequence goes into the cache of a 32-head decoder
        _case("append_token", "append", 4, 32, 1, 128, 4096, 1, ragged=True),
        # the prompt batch of the benchmark workload goes into it
        _case("append_l4096", "append", 4, 32, 1, 128, 4096, 4096),
        # the next token over a short cache of 12 heads of 64: launch and latency
        _case("attend_k512_d64", "attend", 1, 12, 1, 64, 512),
        # decode of one sequence over an ordinary cache, odd length
        _case("attend_k4097", "attend", 1, 32, 1, 128, 4097),
        # decode over a long cache
        _case("attend_k32768", "attend", 4, 32, 1, 128, 32768),
        # a serving batch: shared key/value heads, lengths of all sizes
        _case("attend_ragged_g4", "attend", 16, 8, 4, 128, 8192, ragged=True),
        # four drafted tokens per sequence, heads of 256
        _case("attend_q4_d256", "attend", 2, 4, 4, 256, 20011, 4),
        # the next part of several prompts, padded, over a cache
        _case("chunk_q256_k8192", "attend", 4, 8, 4, 128, 8192, 256, pad=True, ragged=True),
        # one layer's whole step at heads of 96: append, attend, keep the weights
        _case("step_d96", "step", 2, 32, 1, 96, 2047, 1, weight=True),
        # the last 32 tokens of a prompt say which keys matter
        _case("observe_q32_k16384", "attend", 2, 8, 4, 128, 16384, 32, weight=True),
        # an ordinary cache is cut to a quarter
        _case("evict_l4096", "evict", 4, 32, 1, 128, 4096, keep=1024, recent=64),
        # a long prompt's caches, of uneven lengths, are cut to a budget
        _case("evict_k32768", "evict", 2, 8, 4, 128, 32768, ragged=True, keep=4001, recent=500),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("append", "attend", "attend", "attend", "step", "evict"))
        B, H, G = _log_int(rng, 1, 24), rng.choice((1, 2, 3, 5, 8, 12, 16, 32)), 1
        d, L = rng.choice(DIMS), _log_int(rng, 100, 65536)
        ragged = rng.random() < 0.5
        if kind == "append":
            c = _case("", kind, B, H, G, d, L, min(L, _log_int(rng, 1, 5000)), ragged=ragged)
        elif kind == "evict":
            keep = max(1, int(L * rng.uniform(0.05, 0.9)))
            c = _case("", kind, B, H, G, d, L, ragged=ragged, keep=keep,
                      recent=int(keep * rng.uniform(0.0, 0.5)))
        else:
            G = rng.choice((1, 1, 2, 3, 4, 6, 8, 16))
            Lq = min(L, rng.choice((1, 1, 1, 2, 4, _log_int(rng, 2, 600))))
            c = _case("", kind, B, H, G, d, L, Lq, rng.random() < 0.7 or kind == "step",
                      Lq > 1 and rng.random() < 0.4, kind == "step" or rng.random() < 0.3, ragged)
        w = work(c)
        if (1 << 16) <= w["bytes"] and B * H * L * (d + d // 32 + 2) <= MOST_BYTES and \
                w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and \
                (kind in ("append", "evict") or B * H * G * c["Lq"] * L <= MOST_PAIRS):
            return c


def _sizes(case):
    return tuple(case[k] for k in ("B", "H", "G", "d", "L", "Lq"))


def _slots(case):
    """Slots per head of the cache before the call. All Lq rows of a padded step are appended and
    read back, those behind a sequence's own ones too: they have room."""
    room = case["Lq"] if case["kind"] == "step" and case["pad"] else 0
    return -(-(case["L"] + room) // 64) * 64


def _host_lengths(case, seed):
    """Keys per sequence, and query rows (or new tokens) per sequence."""
    B, L, Lq = case["B"], case["L"], case["Lq"]
    g = torch.Generator().manual_seed(int(seed) * 2 + 1)
    counts = torch.full((B,), Lq)
    if case["pad"]:
        counts = torch.randint(1, Lq + 1, (B,), generator=g)
        counts[0] = Lq
    lengths = torch.full((B,), L)
    if case["ragged"]:
        lengths = (torch.rand((B,), generator=g) * (L - counts + 1)).long() + counts
        lengths[-1] = L
    return lengths, counts


def _inputs(case, seed):
    """The bfloat16 rows of one call: q, and K and V of all L keys (of an append, the new ones)."""
    B, H, G, d, L, Lq = _sizes(case)
    L = Lq if case["kind"] == "append" else L
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    q = normal(B, H * G, Lq, d) if case["kind"] in ("attend", "step") else None
    k, v = normal(B, H, L, d), normal(B, H, L, d)
    k *= torch.exp(0.5 * normal(1, H, 1, d))
    k *= 1 + 3 * (torch.rand((B, H, L, 1), generator=g, device="cuda") < 0.01)
    w = torch.exp(torch.randn((B, H, _slots(case)), generator=g, device="cuda"))
    return q, k, v, w


def prepare(case, seed):
    B, H, G, d, L, Lq = _sizes(case)
    kind, C = case["kind"], _slots(case)
    q, k, v, w = _inputs(case, seed)
    lengths, counts = _host_lengths(case, seed)
    dev = {"device": "cuda", "dtype": torch.int32}
    s = {"case": case, "q": q, "scale": 1.0 / math.sqrt(d), "weight": w,
         "lengths": lengths.to(**dev), "counts": counts.to(**dev),
         "start": (lengths - counts).to(**dev)}
    if kind in ("append", "step"):
        s["k"], s["v"] = k[:, :, :Lq].contiguous(), v[:, :, :Lq].contiguous()
    # the cache as it is before the call
    s["cache"] = _new_cache(B, H, C, d)
    if kind != "append":
        _fill(s["cache"], k, v, torch.zeros((B,), **dev))
    if kind == "evict":
        # the smaller cache, with room for the tokens to come
        s["into"] = _new_cache(B, H, -(-case["keep"] // 64) * 64 + 64, d)
        s["into_weight"] = torch.zeros((B, H, s["into"]["C"]), device="cuda")
        s["first"] = torch.zeros((B,), **dev)
    return s


def _new_cache(B, H, C, d):
    if own:
        import paper_2507_16676_amd as F
        return {"C": C, "own": F.cache_new(B, H, C, d)}
    u8 = {"device": "cuda", "dtype": torch.uint8}
    return {"C": C, "kc": torch.zeros((B, H, C, d // 2), **u8),
            "ke": torch.zeros((B, H, C, d // 32), device="cuda", dtype=torch.int8),
            "vc": torch.zeros((B, H, C, d // 2), **u8),
            "vs": torch.zeros((B, H, C), device="cuda", dtype=torch.bfloat16)}


def _fill(cache, k, v, start):
    if own:
        import paper_2507_16676_amd as F
        F.cache_append(cache["own"], k, v, start)
        return
    for b in range(len(k)):      # (one at a time: the temporaries)
        one = {n: x[b:b + 1] for n, x in cache.items() if n != "C"}
        _append(one, k[b:b + 1], v[b:b + 1], start[b:b + 1])


# ---- the plain forms

def _codes(x, scale):
    """Codes (0 to 15, two a byte) of x / scale, whose borders c * scale are exact."""
    a, neg = x.abs(), x < 0
    n = torch.zeros(x.shape, dtype=torch.uint8, device=x.device)
    for c, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False),
                  (3.5, True), (5.0, False)):
        n += (a >= c * scale) if up else (a > c * scale)
    n += 8 * (neg & (n > 0))
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _quantise(k, v):
    B, H, n, d = k.shape
    x = k.float().view(B, H, n, d // 32, 32)
    top = x.abs().amax(-1)
    # a = m * 2^p with 0.5 <= m < 1: a < 7 * 2^e for e = p - 3, or p - 2 from m = 0.875 on
    m, p = torch.frexp(top)
    e = torch.where(top > 0, p - 3 + (m >= 0.875), -100).clamp(min=-100)
    kc = _codes(x, torch.ldexp(torch.ones_like(top), e).unsqueeze(-1)).view(B, H, n, d // 2)
    y = v.float()
    s = (y.abs().amax(-1) / 6).clamp(min=2.0 ** -100)
    s = ((s.view(torch.int32) + 0x3ffff) & ~0x3ffff).view(torch.float32)
    return kc, e.to(torch.int8), _codes(y, s.unsqueeze(-1)), s.to(torch.bfloat16)


def _append(c, k, v, start):
    B, H, n, _ = k.shape
    at = (start.long().view(B, 1) + torch.arange(n, device=k.device)).view(B, 1, n)
    b = torch.arange(B, device=k.device).view(B, 1, 1)
    h = torch.arange(H, device=k.device).view(1, H, 1)
    for name, x in zip(("kc", "ke", "vc", "vs"), _quantise(k, v)):
        c[name][b, h, at] = x


def _values(codes, scale):
    """codes [..., d / 2] times scale [..., d / 32 or 1], in 32 bits."""
    grid = torch.tensor([0., .5, 1., 1.5, 2., 3., 4., 6.], device=codes.device)
    grid = torch.cat((grid, -grid))
    x = torch.stack((grid[(codes & 15).int()], grid[(codes >> 4).int()]), dim=-1).flatten(-2)
    return (x.unflatten(-1, (scale.shape[-1], -1)) * scale.unsqueeze(-1)).flatten(-2)


def _dequantise(kc, ke, vc, vs):
    one = torch.ones((), device=kc.device)
    return _values(kc, torch.ldexp(one, ke.int())), _values(vc, vs.float().unsqueeze(-1))


def _read(c, start, n):
    B, H = c["kc"].shape[:2]
    at = (start.long().view(B, 1) + torch.arange(n, device=start.device)).view(B, 1, n)
    b = torch.arange(B, device=start.device).view(B, 1, 1)
    h = torch.arange(H, device=start.device).view(1, H, 1)
    ok = (at < c["C"]).unsqueeze(-1)
    at = at.clamp(max=c["C"] - 1)
    k, v = _dequantise(*(c[x][b, h, at] for x in ("kc", "ke", "vc", "vs")))
    return (k * ok).to(torch.bfloat16), (v * ok).to(torch.bfloat16)


def _attend(q, c, lengths, counts, causal, scale, weight):
    B, HG, Lq, d = q.shape
    H, L = c["kc"].shape[1:3]
    G = HG // H
    k, v = _dequantise(c["kc"], c["ke"], c["vc"], c["vs"])
    x = torch.matmul(q.float().view(B, H, G * Lq, d), k.transpose(2, 3)) * scale
    i = torch.arange(Lq, device=q.device)
    last = (lengths - counts).unsqueeze(1) + i if causal else \
        (lengths - 1).unsqueeze(1).expand(B, Lq)
    last = torch.where(i < counts.unsqueeze(1), last, -1).view(B, 1, 1, Lq, 1)
    seen = (torch.arange(L, device=q.device) <= last).expand(B, 1, G, Lq, L).reshape(
        B, 1, G * Lq, L)
    x = x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp_(x.sub_(torch.where(top > -math.inf, top, torch.zeros_like(top))))
    p /= p.sum(-1, keepdim=True).clamp(min=1e-30)
    if weight is not None:
        weight += p.sum(2)
    flags = torch.zeros((B, HG, Lq), dtype=torch.uint8, device=q.device)
    return torch.matmul(p, v).to(torch.bfloat16).view(B, HG, Lq, d), flags


def _evict(c, w, lengths, keep, recent, into, into_weight):
    B, H, C = w.shape
    slot, n = torch.arange(C, device=w.device), lengths.long().view(B, 1, 1)
    key = torch.where(slot >= n - recent, math.inf, w)
    key = torch.where(slot < n, key, -1.0)
    kept = n.clamp(max=keep)
    best = key.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    rank = torch.arange(best.shape[-1], device=w.device)
    index = torch.where(rank < kept, best, C).sort(dim=-1).values
    ok = index < C
    b = torch.arange(B, device=w.device).view(B, 1, 1)
    h = torch.arange(H, device=w.device).view(1, H, 1)
    at = index.clamp(max=C - 1)
    for x in ("kc", "ke", "vc", "vs"):
        rows = c[x][b, h, at]
        into[x][:, :, :at.shape[-1]] = torch.where(
            ok.unsqueeze(-1) if rows.dim() == 4 else ok, rows, torch.zeros_like(rows))
    into_weight[:, :, :at.shape[-1]] = torch.where(ok, w[b, h, at], 0.0)
    return torch.where(ok, index, -1).int(), kept.view(B).int()


# ---- one pass

def run(state):
    case, cache = state["case"], state["cache"]
    kind, n = case["kind"], case["Lq"]
    weight = state["weight"] if case["weight"] else None
    if own:
        import paper_2507_16676_amd as F
        c = cache["own"]
        if kind == "evict":
            index, lengths = F.cache_evict(c, state["weight"], state["lengths"], case["keep"],
                                           recent=case["recent"], into=state["into"]["own"],
                                           into_weight=state["into_weight"])
            k, v = F.cache_read(state["into"]["own"], state["first"], case["keep"],
                                counts=lengths)
            return {"index": index, "lengths": lengths, "weight": state["into_weight"],
                    "k": k, "v": v}
        out = {}
        if kind != "attend":
            F.cache_append(c, state["k"], state["v"], state["start"])
            out["k"], out["v"] = F.cache_read(c, state["start"], n)
        if kind != "append":
            out["o"], _, out["flags"] = F.attn_fwd_cache(
                state["q"], c, state["lengths"], counts=state["counts"], causal=case["causal"],
                scale=state["scale"], weight=weight)
    else:
        if kind == "evict":
            index, lengths = _evict(cache, state["weight"], state["lengths"], case["keep"],
                                    case["recent"], state["into"], state["into_weight"])
            k, v = _read(state["into"], state["first"], case["keep"])
            return {"index": index, "lengths": lengths, "weight": state["into_weight"],
                    "k": k, "v": v}
        out = {}
        if kind != "attend":
            _append(cache, state["k"], state["v"], state["start"])
            out["k"], out["v"] = _read(cache, state["start"], n)
        if kind != "append":
            out["o"], out["flags"] = _attend(state["q"], cache, state["lengths"],
                                             state["counts"], case["causal"], state["scale"],
                                             weight)
    if weight is not None:
        out["weight"] = weight
    return out


def work(case):
    """Bytes: the inputs' and outputs' 2 a value, the cache's codes and scales once, 4 a
    weight. Ragged and padded sequences are on average half as long."""
    B, H, G, d, L, Lq = _sizes(case)
    kind, slot = case["kind"], d + d // 32 + 2
    n, f = 0.0, 0.0
    keys = B * H * L * (0.5 if case["ragged"] and B > 1 else 1.0)
    if kind == "evict":
        kept = B * H * min(case["keep"], L)
        return {"bytes": float(4 * keys + kept * (2 * slot + 4 + 4 * d + 4)), "flops": float(keys)}
    rows = B * H * Lq
    if kind in ("append", "step"):
        n += rows * (4 * d + slot + 4 * d)
        f += 8.0 * rows * d
    if kind in ("attend", "step"):
        rows *= G * (0.5 if case["pad"] and B > 1 else 1.0)
        n += keys * slot + rows * (4 * d + 1) + (8 * keys if case["weight"] else 0)
        f += 4.0 * d * rows * keys / (B * H)
    return {"bytes": n, "flops": f}


# ---- the definition in 64 bits, without the packed form

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest64(x, scale):
    """scale times the number of the grid nearest to x / scale (ties: the even one)."""
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    y = x / scale
    lo = (torch.searchsorted(grid, y.abs(), right=True) - 1).clamp(0, 6)
    below, above = y.abs() - grid[lo], grid[lo + 1] - y.abs()
    up = (above < below) | ((above == below) & (lo % 2 == 1))
    return torch.sign(y) * grid[lo + up] * scale


def _rows64(k, v):
    x = k.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.log2(top.clamp(min=2.0 ** -120) / 7).floor() + 1
    e = torch.where(top >= 7 * torch.exp2(e), e + 1, e)
    e = torch.where(top < 7 * torch.exp2(e - 1), e - 1, e).clamp(min=-100)
    y = v.double()
    s = (y.abs().amax(-1, keepdim=True) / 6).clamp(min=2.0 ** -100)
    step = torch.exp2(torch.log2(s).floor() - 5)
    return _nearest64(x, torch.exp2(e)).flatten(-2), _nearest64(y, torch.ceil(s / step) * step)


def exact(case, seed):
    B, H, G, d, L, Lq = _sizes(case)
    kind = case["kind"]
    q, k, v, w = _inputs(case, seed)
    lengths, counts = (x.tolist() for x in _host_lengths(case, seed))
    if kind == "append":
        ks, vs = zip(*(_rows64(k[b, :, :Lq], v[b, :, :Lq]) for b in range(B)))
        return {"k": torch.stack(ks), "v": torch.stack(vs)}
    if kind == "evict":
        keep, recent = case["keep"], case["recent"]
        out = {n: torch.zeros((B, H, keep, d), dtype=torch.float64, device="cuda") for n in "kv"}
        nw = torch.zeros((B, H, -(-keep // 64) * 64 + 64), dtype=torch.float64, device="cuda")
        for b in range(B):
            n = min(keep, lengths[b])
            old = max(0, lengths[b] - recent)
            for h in range(H):
                # the order of (largest weight, lowest slot)
                take = torch.argsort(-w[b, h, :old].double(), stable=True)[
                    :n - (lengths[b] - old)].sort().values
                at = torch.cat((take, torch.arange(old, lengths[b], device="cuda")))
                out["k"][b, h, :n], out["v"][b, h, :n] = _rows64(k[b, h, at], v[b, h, at])
                nw[b, h, :n] = w[b, h, at].double()
        return {"index": None, "lengths": None, "weight": nw, **out}
    res = {"o": torch.zeros((B, H * G, Lq, d), dtype=torch.float64, device="cuda"), "flags": None}
    if case["weight"]:
        res["weight"] = w.double()
    if kind == "step":
        ks, vs = zip(*(_rows64(k[b, :, :Lq], v[b, :, :Lq]) for b in range(B)))
        res["k"], res["v"] = torch.stack(ks), torch.stack(vs)
    for b in range(B):
        n, m = lengths[b], counts[b]
        keys = torch.arange(n, device="cuda")
        last = torch.arange(n - m, n, device="cuda") if case["causal"] else \
            torch.full((m,), n, device="cuda")
        for h in range(H):
            kk, vv = _rows64(k[b, h, :n], v[b, h, :n])
            if kind == "step":
                kk[n - m:], vv[n - m:] = res["k"][b, h, :m], res["v"][b, h, :m]
            for g in range(h * G, h * G + G):
                x = (q[b, g, :m].double() @ kk.t().contiguous()) / math.sqrt(d)
                p = torch.softmax(x.masked_fill(keys > last.unsqueeze(1), -math.inf), dim=-1)
                res["o"][b, g, :m] = p @ vv
                if case["weight"]:
                    res["weight"][b, h, :n] += p.sum(0)
    return res
