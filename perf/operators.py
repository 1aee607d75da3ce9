"""Performance cases of the operators on the paged cache: decode attention of one new token over
pages, the same with the attention weights of the cached rows accumulated, and the eviction of a
cache down to a budget by those weights.

A paged cache keeps the rows of a sequence in pages of a pool shared by all sequences; a table
names each sequence's pages in order.  Cases are what a serving loop calls once per token (or
once per eviction): one layer, as a model calls it between its other kernels, and whole stacks of
layers, with the heads of this package's workloads, one to sixteen query heads per KV head, head
dimensions 64 and 128, float32 and bf16 caches, pages of 16 to 256 rows, lengths from a few rows
to beyond a hundred thousand, with and without a sliding window and its sinks.

`listed` names the fixed cases, `draw` gives more of the same ranges, `prepare` builds a case's
inputs from a seed, `run` makes one pass (the plain form, or with `own` the library's calls),
`exact` computes the same outputs in float64 and `work` counts what a pass cannot do without.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
GB = 1e9


def _heads(layers, batch, h_q, h_kv, d, dtype, page):
    return {"layers": layers, "batch": batch, "h_q": h_q, "h_kv": h_kv, "d": d, "dtype": dtype, "page": page}


def listed():
    return [
        # ---- decode attention of one new token over a paged cache
        # The Tiny workload's layer (float32): one call of almost no data, its latency counts.
        {"name": "decode_tiny_f32", "kind": "decode", **_heads(1, 1, 8, 2, 64, "f32", 16), "lo": 512, "hi": 512,
         "window": 0, "sinks": 0, "ragged": False},
        # One layer of the 7B-class heads after compression: what a model calls between its other
        # kernels, 32 units for 152 SMs.
        {"name": "decode_layer_7b", "kind": "decode", **_heads(1, 8, 28, 4, 128, "bf16", 16), "lo": 3800, "hi": 4700,
         "window": 0, "sinks": 0, "ragged": False},
        # One long sequence, one layer of the 32B-class heads: few units, cut over their length.
        {"name": "decode_long_b1", "kind": "decode", **_heads(1, 1, 40, 8, 128, "bf16", 32), "lo": 100000, "hi": 131072,
         "window": 0, "sinks": 0, "ragged": False},
        # The 7B-class stack uncompressed, all layers in one call: the largest cache of the list.
        {"name": "decode_stack_7b", "kind": "decode", **_heads(28, 8, 28, 4, 128, "bf16", 64), "lo": 15000, "hi": 16384,
         "window": 0, "sinks": 0, "ragged": False},
        # 16 layers of the 32B-class heads with a sliding window and a few sinks, per-unit lengths.
        {"name": "decode_window_32b", "kind": "decode", **_heads(16, 4, 40, 8, 128, "bf16", 16), "lo": 20000, "hi": 32768,
         "window": 4000, "sinks": 4, "ragged": True},
        # The 1.5B-class stack after compression in float32, lengths that end inside a page.
        {"name": "decode_f32", "kind": "decode", **_heads(28, 4, 12, 2, 128, "f32", 32), "lo": 800, "hi": 1500,
         "window": 0, "sinks": 0, "ragged": False},
        # ---- the same with every row's attention weight accumulated
        # The Tiny layer.
        {"name": "weights_tiny_f32", "kind": "weights", **_heads(1, 1, 8, 2, 64, "f32", 16), "lo": 512, "hi": 512,
         "window": 0, "sinks": 0, "ragged": False},
        # One layer, sixteen sequences of very different lengths with a window and sinks.
        {"name": "weights_layer_7b", "kind": "weights", **_heads(1, 16, 28, 4, 128, "bf16", 16), "lo": 90, "hi": 4000,
         "window": 2000, "sinks": 8, "ragged": False},
        # The 7B-class stack between two evictions.
        {"name": "weights_stack_7b", "kind": "weights", **_heads(28, 8, 28, 4, 128, "bf16", 64), "lo": 3800, "hi": 4700,
         "window": 0, "sinks": 0, "ragged": False},
        # ---- eviction down to a budget by accumulated weight
        # The Tiny layer, a quarter kept.
        {"name": "evict_tiny_f32", "kind": "evict", **_heads(1, 1, 8, 2, 64, "f32", 16), "lo": 512, "hi": 512,
         "w": 16, "sinks": 4, "ratio": 0.25, "cut": 1},
        # One layer, half of sixteen sequences over their budget by a few hundred rows.
        {"name": "evict_layer_7b", "kind": "evict", **_heads(1, 16, 28, 4, 128, "bf16", 16), "lo": 4200, "hi": 4600,
         "w": 32, "sinks": 4, "ratio": 0.9, "cut": 8},
        # The 7B-class stack, every sequence cut to a quarter.
        {"name": "evict_stack_7b", "kind": "evict", **_heads(28, 8, 28, 4, 128, "bf16", 64), "lo": 15000, "hi": 16384,
         "w": 32, "sinks": 4, "ratio": 0.25, "cut": 8},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: any operator, type, head shape, page and length."""
    kind = rng.choice(["decode", "decode", "weights", "weights", "evict"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    h_kv = rng.choice([1, 2, 3, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 12, 16])
    d = 64 if rng.random() < 0.3 else 128
    layers = 1 if rng.random() < 0.5 else rng.randint(2, 28)
    c = {"kind": kind, **_heads(layers, _log_int(rng, 1, 24), G * h_kv, h_kv, d, dtype, rng.choice([16, 32, 64, 128, 256]))}
    units = c["layers"] * c["batch"] * h_kv
    most = int(min(131072, max(96, 3.0 * GB / (units * 2 * d * (4 if dtype == "f32" else 2)))))
    hi = _log_int(rng, 32, most)
    c["lo"], c["hi"] = max(24, hi // rng.choice([1, 1, 2, 4, 16])), hi
    if kind == "evict":
        c["w"] = rng.randint(1, max(1, min(64, c["lo"] // 4)))
        c["sinks"] = rng.choice([0, 0, 1, 4, 5])
        c["ratio"] = round(rng.uniform(0.2, 0.98), 3)
        c["cut"] = rng.randint(1, c["batch"])
        return c
    c["window"], c["sinks"] = 0, 0
    if rng.random() < 0.4:
        c["window"] = _log_int(rng, 1, 2 * hi)
        c["sinks"] = rng.choice([0, 1, 4, 17, 64])
    c["ragged"] = rng.random() < 0.5
    return c


# ---------------------------------------------------------------- inputs
class State:
    pass


def _np(seed, stream):
    return np.random.Generator(np.random.PCG64([int(seed), stream]))


def _to(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _lens(c, seed):
    """[layers, B, h_kv] lengths, one per sequence or (ragged) one per unit, spread over their logarithm."""
    rng = _np(seed, 1)
    Ly, B, H = c["layers"], c["batch"], c["h_kv"]
    shape = (Ly, B, H) if c.get("ragged") else (1, B, 1)
    n = np.exp(rng.uniform(math.log(c["lo"]), math.log(c["hi"] + 1), shape)).astype(np.int64)
    return np.ascontiguousarray(np.broadcast_to(np.clip(n, c["lo"], c["hi"]), (Ly, B, H)), dtype=np.int32)


def _paged_state(c, seed):
    """Pool, table and lengths.  The table gives each sequence its pages in a random order over
    the pool, which holds a few more than are in use."""
    s = State()
    s.case = c
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s.gen = g
    Ly, B, H, d, page = c["layers"], c["batch"], c["h_kv"], c["d"], c["page"]
    s.dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    lens = _lens(c, seed)
    per = c["hi"] // page + 1  # pages of the longest unit with its new token
    rng = _np(seed, 2)
    s.table = _to(rng.permutation(B * per + 3)[:B * per].astype(np.int32).reshape(B, per))
    shape = (Ly, B * per + 3, H, page, d)
    s.K = torch.randn(shape, generator=g, device=DEV, dtype=s.dt)
    s.V = torch.randn(shape, generator=g, device=DEV, dtype=s.dt)
    s.lens0 = _to(lens)
    s.lens = s.lens0.clone()
    s.cap = per * page
    if own:
        from paper_2608_04771_gb300 import reco
        s.reco = reco
        s.kv = reco.make_paged_kv(s.K, s.V, s.table, c["h_q"])
        op = {"decode": reco.RECO_OP_PAGED_DECODE, "weights": reco.RECO_OP_PAGED_WEIGHTS,
              "evict": reco.RECO_OP_PAGED_EVICT}[c["kind"]]
        s.ws = reco.paged_workspace(op, s.kv, DEV)
    return s


def prepare(c, seed):
    s = _paged_state(c, seed)
    Ly, B, H, Hq, d = c["layers"], c["batch"], c["h_kv"], c["h_q"], c["d"]
    rand = lambda *shape: torch.randn(shape, generator=s.gen, device=DEV, dtype=s.dt)  # noqa: E731
    if c["kind"] == "evict":
        # weights as many tokens' attention leaves them: positive and skewed, the first rows largest
        s.weights = torch.exp(1.5 * torch.randn((Ly, B, H, s.cap), generator=s.gen, device=DEV))
        s.weights[..., :4] += 20.0
        rng = _np(seed, 3)
        lens = s.lens0[0, :, 0].cpu().numpy()
        budget = np.full(B, s.cap, np.int32)  # these sequences are not over their budget
        for b in rng.permutation(B)[:c["cut"]]:
            budget[b] = max(c["w"] + c["sinks"], int(lens[b] * min(1.0, c["ratio"] * rng.uniform(0.95, 1.02))))
        s.budget = _to(budget)
        s.kept = torch.zeros((Ly, B, H, s.cap), dtype=torch.int32, device=DEV)
        return s
    s.scale = 1.0 / math.sqrt(d)
    s.q, s.kn, s.vn = rand(Ly, B, Hq, d), rand(Ly, B, H, d), rand(Ly, B, H, d)
    s.out = torch.empty((Ly, B, Hq, d), dtype=s.dt, device=DEV)
    s.lse = torch.empty((Ly, B, Hq), dtype=torch.float32, device=DEV)
    if c["kind"] == "weights":
        s.weights = torch.rand((Ly, B, H, s.cap), generator=s.gen, device=DEV) * (8.0 / c["hi"])
    return s


# ---------------------------------------------------------------- the plain form
def _rows(pool, table):
    """[layers, B, h_kv, capacity, d] float32 rows of every sequence, in order."""
    x = pool[:, table.long()]  # [layers, B, pages, h_kv, page, d]
    return x.permute(0, 1, 3, 2, 4, 5).flatten(3, 4).float()


def _place(s, at):
    """Pool indices (layer, page, head, row) of row `at` [layers, B, h_kv, ...] of every unit."""
    c = s.case
    extra = (1,) * (at.dim() - 3)
    ly = torch.arange(c["layers"], device=DEV).view(-1, 1, 1, *extra)
    b = torch.arange(c["batch"], device=DEV).view(1, -1, 1, *extra)
    h = torch.arange(c["h_kv"], device=DEV).view(1, 1, -1, *extra)
    pages = s.table.long()[b, at // c["page"]]
    return ly.expand(at.shape), pages, h.expand(at.shape), at % c["page"]


def _decode_plain(s):
    c = s.case
    Ly, B, H, Hq, d = c["layers"], c["batch"], c["h_kv"], c["h_q"], c["d"]
    at = s.lens.long()
    place = _place(s, at)
    s.K[place], s.V[place] = s.kn, s.vn
    s.lens += 1
    n = at.unsqueeze(-1) + 1
    j = torch.arange(s.cap, device=DEV)
    seen = j < n
    if c["window"]:
        seen = seen & ((j < c["sinks"]) | (j >= n - c["window"]))
    q = s.q.float().view(Ly, B, H, Hq // H, d)
    x = torch.matmul(q, _rows(s.K, s.table).transpose(3, 4)) * s.scale
    x = torch.where(seen.unsqueeze(3), x, -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    p = e / z
    v = torch.where(seen.unsqueeze(-1), _rows(s.V, s.table), 0.0)
    s.out.copy_(torch.matmul(p, v).view(Ly, B, Hq, d))
    s.lse.copy_((m + torch.log(z)).view(Ly, B, Hq))
    if c["kind"] == "weights":  # the new row starts with its own weight
        s.weights.copy_(torch.where(seen, torch.where(j == n - 1, 0.0, s.weights) + p.mean(3), s.weights))


def _evict_plain(s):
    c = s.case
    L = s.lens.long().unsqueeze(-1)
    m = s.budget.long().view(1, -1, 1, 1).expand(L.shape)
    j = torch.arange(s.cap, device=DEV)
    over = L > m
    fixed = (j < c["sinks"]) | ((j >= L - c["w"]) & (j < L))
    order = torch.sort(torch.where(fixed, math.inf, torch.where(j < L, s.weights, -math.inf)), dim=-1,
                       descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, j.expand(order.shape))
    kept = torch.sort(torch.where(rank < m, j, s.cap), dim=-1).values  # kept rows in order, then s.cap
    moved = over & (j < m)
    source = torch.where(moved, kept, j)
    s.kept.copy_(torch.where(moved, kept.int(), s.kept))
    src, dst = _place(s, source), _place(s, j.expand(source.shape))
    s.K[dst], s.V[dst] = s.K[src], s.V[src]
    s.weights.copy_(s.weights.gather(-1, source))
    s.lens.copy_(torch.where(over, m, L).squeeze(-1))


def run(s):
    """One token (at the same length in every pass), or one eviction (from the same length)."""
    c = s.case
    s.lens.copy_(s.lens0)
    if c["kind"] == "evict":
        if own:
            s.reco.reco_paged_evict(s.kv, s.weights, s.lens, s.budget, c["w"], c["sinks"], s.kept, s.ws)
        else:
            _evict_plain(s)
        return {"K": s.K, "V": s.V, "weights": s.weights, "lens": s.lens, "kept": s.kept}
    r = {"out": s.out, "lse": s.lse, "lens": s.lens, "K": s.K, "V": s.V}
    if c["kind"] == "weights":
        r["weights"] = s.weights
    if not own:
        _decode_plain(s)
    elif c["kind"] == "weights":
        s.reco.reco_paged_decode_attn_weights(s.kv, s.q, s.kn, s.vn, s.lens, s.scale, s.out, s.lse, s.weights, s.ws,
                                              window=c["window"], sinks=c["sinks"])
    else:
        s.reco.reco_paged_decode_attn(s.kv, s.q, s.kn, s.vn, s.lens, s.scale, s.out, s.lse, s.ws,
                                      window=c["window"], sinks=c["sinks"])
    return r


# ---------------------------------------------------------------- the same in float64
def exact(c, seed):
    if c["kind"] == "evict":  # moves rows, computes no numbers
        return None
    s = prepare(c, seed)
    Ly, B, H, G, d, page = c["layers"], c["batch"], c["h_kv"], c["h_q"] // c["h_kv"], c["d"], c["page"]
    out = torch.zeros((Ly, B, H * G, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((Ly, B, H * G), dtype=torch.float64, device=DEV)
    weights = s.weights.double() if c["kind"] == "weights" else None
    lens, table = s.lens0.cpu().numpy(), s.table.long()
    for b in range(B):
        for ly in range(Ly):
            n = lens[ly, b]  # [h_kv] lengths before the token
            top = int(n.max())
            ids = table[b, :top // page + 1]
            k = s.K[ly, ids].double().transpose(0, 1).reshape(H, -1, d)[:, :top + 1].clone()
            v = s.V[ly, ids].double().transpose(0, 1).reshape(H, -1, d)[:, :top + 1].clone()
            last = _to(n.astype(np.int64))
            heads = torch.arange(H, device=DEV)
            k[heads, last], v[heads, last] = s.kn[ly, b].double(), s.vn[ly, b].double()
            pos = torch.arange(top + 1, device=DEV).view(1, -1)
            hide = pos > last.view(-1, 1)
            if c["window"] > 0:
                hide = hide | ((pos >= c["sinks"]) & (pos <= last.view(-1, 1) - c["window"]))
            logit = torch.einsum("hgd,hjd->hgj", s.q[ly, b].double().view(H, G, d), k) * s.scale
            logit = logit.masked_fill(hide.unsqueeze(1), -math.inf)
            norm = torch.logsumexp(logit, -1)
            prob = torch.exp(logit - norm.unsqueeze(-1))
            v = v.masked_fill(hide.unsqueeze(-1), 0.0)
            out[ly, b] = torch.einsum("hgj,hjd->hgd", prob, v).reshape(H * G, d)
            lse[ly, b] = norm.reshape(H * G)
            if weights is not None:
                weights[ly, b][heads, last] = 0.0
                weights[ly, b, :, :top + 1] += prob.sum(1) / G
    r = {"out": out, "lse": lse, "lens": None, "K": None, "V": None}
    if weights is not None:
        r["weights"] = weights
    return r


# ---------------------------------------------------------------- what a pass cannot do without
def _mean(c):
    """Mean length of the log-uniform draw of lengths."""
    lo, hi = c["lo"], c["hi"]
    return float(lo) if hi <= lo else (hi - lo) / math.log(hi / lo)


def work(c):
    Ly, B, H, d = c["layers"], c["batch"], c["h_kv"], c["d"]
    G, es = c["h_q"] // H, 4 if c["dtype"] == "f32" else 2
    units, n = Ly * B * H, _mean(c)
    if c["kind"] == "evict":  # scores of the units that are cut, their kept rows read and written
        m = max(c["w"] + c["sinks"], n * min(1.0, c["ratio"]))
        units *= c["cut"] / B
        return {"bytes": units * (4 * n + 4 * m + 4 * m + 4 * m * d * es), "flops": 0.0}
    seen = n + 1 if not c["window"] else min(n + 1, c["window"] + c["sinks"])
    by = units * (2 * seen * d * es + 2 * G * d * es + 4 * G + 4 * d * es + 8) + 4 * B * seen / c["page"]
    if c["kind"] == "weights":
        by += units * 8 * seen
    return {"bytes": by, "flops": 4.0 * units * G * seen * d}
