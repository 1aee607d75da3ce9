"""Performance cases of what fills a paged cache and of what reads one prompt for many answers: the
append of new tokens' keys and values with the position rotation applied on the way, and decode
attention of a batch whose sequences share the rows of a prefix.

An append takes the tokens of all sequences one after the other (`starts` says whose they are),
keys, values and queries as views into the output of one projection, [tokens, all heads, d], and
rotates keys and queries by their positions.  The cases are one token per sequence, as a serving
loop appends them, and prompts or pieces of prompts.

Attention over a shared prefix serves several answers to one question: the sequences of a group
hold the question's rows once, in pages that all of them name, and their own rows behind them.

Heads are those of this package's workloads, one to sixteen query heads per KV head, head
dimensions 64 and 128, float32 and bf16, pages of 16 to 256 rows.

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


def _heads(layers, batch, h_q, h_kv, d, dtype, page):
    return {"layers": layers, "batch": batch, "h_q": h_q, "h_kv": h_kv, "d": d, "dtype": dtype, "page": page}


def _append(heads, lo, hi, have, rot, interleaved=False, base=1e6, far=0):
    """lo..hi new tokens per sequence behind up to `have` cached rows, positions from `far` on."""
    return {"kind": "append", **heads, "lo": lo, "hi": hi, "have": have, "rot": rot, "interleaved": interleaved,
            "base": base, "far": far}


def _prefix(heads, groups, p_lo, p_hi, lo, hi, ragged=False, append=True, out_f32=False):
    """`groups` runs of sequences, prefixes of p_lo..p_hi rows, lo..hi rows of their own behind them."""
    return {"kind": "prefix", **heads, "groups": groups, "p_lo": p_lo, "p_hi": p_hi, "lo": lo, "hi": hi,
            "ragged": ragged, "append": append, "out_f32": out_f32}


def listed():
    return [
        # ---- append with rotation
        # One token of one sequence, the Tiny workload's layer: a call of almost no data, its latency counts.
        {"name": "append_tiny_f32", **_append(_heads(1, 1, 8, 2, 64, "f32", 16), 1, 1, 512, 64, base=1e4)},
        # One token of eight sequences, a 7B-class layer: once per layer and token in a serving loop.
        {"name": "append_token_7b", **_append(_heads(1, 8, 28, 4, 128, "bf16", 16), 1, 1, 4000, 128)},
        # One token of forty sequences, sixteen 32B-class layers in one call, positions beyond a hundred thousand.
        {"name": "append_token_32b", **_append(_heads(16, 40, 40, 8, 128, "bf16", 32), 1, 1, 2000, 128, far=100000)},
        # Ragged pieces of prompts, one 7B-class layer.
        {"name": "append_prompt_7b", **_append(_heads(1, 8, 28, 4, 128, "bf16", 16), 90, 4001, 700, 128)},
        # float32, pairs of neighbours and only half of the dimensions rotated, a 1.5B-class layer.
        {"name": "append_prompt_f32", **_append(_heads(1, 4, 12, 2, 128, "f32", 64), 500, 2000, 0, 64, True, 1e4)},
        # A prompt through all layers of the 7B-class stack: the most data of the appends.
        {"name": "append_stack_7b", **_append(_heads(28, 1, 28, 4, 128, "bf16", 64), 4096, 4096, 0, 128)},
        # ---- decode attention over a shared prefix
        # Two answers to a short question, the Tiny layer.
        {"name": "prefix_tiny_f32", **_prefix(_heads(1, 2, 8, 2, 64, "f32", 16), 1, 512, 512, 20, 40)},
        # Sixteen answers to one question, a 7B-class layer, ragged answers.
        {"name": "prefix_layer_7b", **_prefix(_heads(1, 16, 28, 4, 128, "bf16", 16), 1, 4001, 4001, 200, 2000)},
        # Four questions with eight answers each, prefixes and answers of many lengths, one 7B-class layer.
        {"name": "prefix_groups_7b", **_prefix(_heads(1, 32, 28, 4, 128, "bf16", 16), 4, 900, 9000, 1, 1500, True)},
        # Sixty-four samples over one long document, a 32B-class layer: as much arithmetic as data.
        {"name": "prefix_long_32b", **_prefix(_heads(1, 64, 40, 8, 128, "bf16", 32), 1, 100001, 100001, 16, 500)},
        # Eight samples, all layers of the 7B-class stack in one call.
        {"name": "prefix_stack_7b", **_prefix(_heads(28, 8, 28, 4, 128, "bf16", 64), 1, 16001, 16001, 1000, 4000)},
        # The 1.5B-class stack in float32, two questions with four answers.
        {"name": "prefix_f32", **_prefix(_heads(28, 8, 12, 2, 128, "f32", 32), 2, 1500, 2000, 100, 400)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: either operator, any type, head shape, page and length."""
    kind = rng.choice(["append", "prefix"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    es = 4 if dtype == "f32" else 2
    h_kv = rng.choice([1, 2, 3, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 12, 16])
    d = 64 if rng.random() < 0.3 else 128
    layers = 1 if rng.random() < 0.5 else rng.randint(2, 28)
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        heads = _heads(layers, batch, G * h_kv, h_kv, d, dtype, page)
        most = 2.0e9 / (layers * batch * 2 * (G + 2) * h_kv * d * es)  # the largest listed append's bytes
        hi = 1 if rng.random() < 0.35 else _log_int(rng, 1, max(2, min(8192, int(most))))
        lo = hi if hi == 1 else max(0, hi // rng.choice([1, 2, 4, 50, 10000]))
        rot = rng.choice([d, d, d // 2, 16, d - 16])
        return _append(heads, lo, hi, _log_int(rng, 1, 3000) - 1, rot, rng.random() < 0.4,
                       rng.choice([1e4, 5e5, 1e6]), rng.choice([0, 0, 1000, 100000, 1000000]))
    groups = rng.choice([1, 1, 1, 2, 3, 6])
    batch = max(groups, _log_int(rng, 1, 80))
    heads = _heads(layers, batch, G * h_kv, h_kv, d, dtype, page)
    row = layers * h_kv * 2 * d * es
    # bytes and products below those of the largest listed ones (float32 products cost several times as much)
    flops = 1.0e10 if dtype == "f32" else 1.2e11
    most = min(131072, 2.0e9 / (row * groups), flops / (4.0 * layers * batch * G * h_kv * d))
    p_hi = _log_int(rng, 16, max(17, most))
    own_most = min(8192, 8.0e8 / (row * batch), 0.3 * flops / (4.0 * layers * batch * G * h_kv * d))
    hi = _log_int(rng, 1, max(2, own_most))
    append = rng.random() < 0.7
    lo = max(0 if append else 1, hi // rng.choice([1, 2, 8, 100000]))
    p_lo = max(0, p_hi // rng.choice([1, 1, 2, 8, 1000000]))
    return _prefix(heads, groups, p_lo, p_hi, lo, hi, rng.random() < 0.4, append, rng.random() < 0.3)


# ---------------------------------------------------------------- inputs
class State:
    pass


def _np(seed, stream):
    return np.random.Generator(np.random.PCG64([int(seed), stream]))


def _to(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _spread(rng, lo, hi, shape):
    """Whole numbers of lo..hi, spread over their logarithm."""
    n = np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2), shape)).astype(np.int64) - 1
    return np.clip(n, lo, hi)


def _new_state(c, seed):
    s = State()
    s.case = c
    s.gen = torch.Generator(device=DEV)
    s.gen.manual_seed(int(seed))
    s.dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    return s


def _pool(s, n_pages):
    c = s.case
    shape = (c["layers"], n_pages, c["h_kv"], c["page"], c["d"])
    s.K = torch.randn(shape, generator=s.gen, device=DEV, dtype=s.dt)
    s.V = torch.randn(shape, generator=s.gen, device=DEV, dtype=s.dt)


def _prepare_append(c, seed):
    s = _new_state(c, seed)
    Ly, B, H, Hq, d, page = c["layers"], c["batch"], c["h_kv"], c["h_q"], c["d"], c["page"]
    # new tokens of each sequence: the same lengths for every seed, in another order
    n = _np(seed, 1).permutation(_spread(_np(0, 1), c["lo"], c["hi"], B))
    have = _spread(_np(seed, 2), 0, c["have"], (Ly, B, H))  # rows of each unit, as compression leaves them
    starts = np.concatenate([[0], np.cumsum(n)])
    s.T = max(1, int(starts[-1]))
    per = (c["have"] + int(n.max()) + page - 1) // page
    s.table = _to(_np(seed, 3).permutation(B * per + 3)[:B * per].astype(np.int32).reshape(B, per))
    _pool(s, B * per + 3)
    # positions run on from the tokens that a sequence has seen, whatever compression kept of them
    pos = np.zeros(s.T, np.int32)
    for b in range(B):
        first = c["far"] + int(have[:, b].max()) + 17 * b
        pos[starts[b]:starts[b + 1]] = first + np.arange(n[b])
    s.starts, s.pos = _to(starts.astype(np.int32)), _to(pos)
    s.inv_freq = _to((c["base"] ** (-np.arange(0, c["rot"], 2) / c["rot"])).astype(np.float32))
    s.lens0 = _to(have.astype(np.int32))
    s.lens = s.lens0.clone()
    # queries, keys and values as a fused projection leaves them
    s.qkv = torch.randn((Ly, s.T, Hq + 2 * H, d), generator=s.gen, device=DEV, dtype=s.dt)
    s.q_out = torch.zeros((Ly, s.T, Hq, d), dtype=s.dt, device=DEV)
    if own:
        from paper_2608_04771_gb300 import reco
        s.reco = reco
        s.kv = reco.make_paged_kv(s.K, s.V, s.table, Hq)
        s.ws = reco.paged_workspace(reco.RECO_OP_PAGED_APPEND, s.kv, DEV)
    return s


def _prepare_prefix(c, seed):
    s = _new_state(c, seed)
    Ly, B, H, Hq, d, page, groups = (c["layers"], c["batch"], c["h_kv"], c["h_q"], c["d"], c["page"], c["groups"])
    rng = _np(seed, 1)
    cuts = np.sort(rng.permutation(B - 1)[:groups - 1] + 1) if groups > 1 else np.zeros(0, np.int64)
    s.first = np.concatenate([[0], cuts, [B]]).astype(np.int64)  # first sequence of each group, then B
    p = _spread(rng, c["p_lo"], c["p_hi"], groups)
    shape = (Ly, B, H) if c["ragged"] else (1, B, 1)
    mine = np.broadcast_to(_spread(rng, c["lo"], c["hi"], shape), (Ly, B, H))
    if not c["append"]:
        mine = np.maximum(mine, 1)
    group = np.repeat(np.arange(groups), np.diff(s.first))
    shared = p[group]
    lens = shared.reshape(1, B, 1) + mine
    # A sequence names the group's pages for whole pages of the prefix and pages of its own behind them (the page
    # that the prefix ends in belongs to it, the first sequence of the group holds the prefix's last rows there).
    per = (c["p_hi"] + max(1, c["hi"]) + page) // page
    n_pages = groups * (c["p_hi"] // page) + B * ((max(1, c["hi"]) + 2 * page - 1) // page + 1) + 3
    need = [int((lens[:, b].max() + 1 + page - 1) // page) for b in range(B)]
    fresh = [need[b] - (0 if b in s.first else int(shared[b]) // page) for b in range(B)]
    ids = iter(_np(seed, 2).permutation(n_pages)[:sum(fresh)].tolist())
    table = np.full((B, per), -1, np.int32)
    for b in range(B):
        lead = int(s.first[group[b]])
        whole = 0 if b == lead else int(shared[b]) // page
        table[b, :whole] = table[lead, :whole]
        table[b, whole:need[b]] = [next(ids) for _ in range(need[b] - whole)]
    s.table = _to(table)
    _pool(s, n_pages)
    s.p, s.most = p.tolist(), int(mine.max()) + 1
    s.group, s.shared = _to(group.astype(np.int32)), _to(shared.astype(np.int32))
    s.lens0 = _to(lens.astype(np.int32))
    s.lens = s.lens0.clone()
    s.scale = 1.0 / math.sqrt(d)
    rand = lambda *shape: torch.randn(shape, generator=s.gen, device=DEV, dtype=s.dt)  # noqa: E731
    s.q, s.kn, s.vn = rand(Ly, B, Hq, d), rand(Ly, B, H, d), rand(Ly, B, H, d)
    if not c["append"]:
        s.kn = s.vn = None
    s.out = torch.empty((Ly, B, Hq, d), dtype=torch.float32 if c["out_f32"] else s.dt, device=DEV)
    s.lse = torch.empty((Ly, B, Hq), dtype=torch.float32, device=DEV)
    if own:
        from paper_2608_04771_gb300 import reco
        s.reco = reco
        s.kv = reco.make_paged_kv(s.K, s.V, s.table, Hq)
        s.ws = reco.paged_workspace(reco.RECO_OP_PAGED_PREFIX, s.kv, DEV)
    return s


def prepare(c, seed):
    return _prepare_append(c, seed) if c["kind"] == "append" else _prepare_prefix(c, seed)


# ---------------------------------------------------------------- the plain form
def _turn(x, cos, sin, rot, interleaved):
    """Rotates the first `rot` elements of float rows x [..., T, heads, d] by cos, sin [T, 1, rot / 2]."""
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


def _append_plain(s):
    c = s.case
    H, Hq, page = c["h_kv"], c["h_q"], c["page"]
    n_all = s.qkv.shape[1]
    angle = (s.pos.double().view(-1, 1) * s.inv_freq.double()).unsqueeze(1)  # far positions: 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    t = torch.arange(n_all, device=DEV)
    b = torch.searchsorted(s.starts[1:].contiguous(), t, right=True)  # the token's sequence, B behind the last one
    there = b < c["batch"]
    t, b = t[there], b[there]
    cos, sin = cos[there], sin[there]
    for ly in range(c["layers"]):  # a layer at a time: float32 copies of all of them would be large
        x = s.qkv[ly, t].float()
        s.q_out[ly, t] = _turn(x[:, :Hq], cos, sin, c["rot"], c["interleaved"]).to(s.dt)
        k = _turn(x[:, Hq:Hq + H], cos, sin, c["rot"], c["interleaved"]).to(s.dt)
        row = s.lens[ly, b].long() + (t - s.starts[b]).unsqueeze(1)  # [T, H]
        at = s.table[b.unsqueeze(1), row // page].long(), torch.arange(H, device=DEV).expand(row.shape), row % page
        s.K[ly][at] = k
        s.V[ly][at] = s.qkv[ly, t, Hq + H:]
    s.lens += (s.starts[1:] - s.starts[:-1]).view(1, -1, 1)


def _prefix_plain(s):
    c = s.case
    Ly, B, H, Hq, d, page = c["layers"], c["batch"], c["h_kv"], c["h_q"], c["d"], c["page"]
    ly = torch.arange(Ly, device=DEV).view(-1, 1, 1)
    heads = torch.arange(H, device=DEV).view(1, 1, -1)
    if c["append"]:
        at = s.lens.long()
        pg = s.table.long()[torch.arange(B, device=DEV).view(1, -1, 1), at // page]
        place = ly.expand(at.shape), pg, heads.expand(at.shape), at % page
        s.K[place], s.V[place] = s.kn, s.vn
        s.lens += 1
    q = s.q.float().view(Ly, B, H, Hq // H, d)
    for g, p in enumerate(s.p):
        b0, b1 = int(s.first[g]), int(s.first[g + 1])
        n = b1 - b0
        # the prefix, once for the group
        ids = s.table[b0, :(p + page - 1) // page].long()
        kp = s.K[:, ids].permute(0, 2, 1, 3, 4).reshape(Ly, H, ids.numel() * page, d)[:, :, :p].float()
        vp = s.V[:, ids].permute(0, 2, 1, 3, 4).reshape(Ly, H, ids.numel() * page, d)[:, :, :p].float()
        qg = q[:, b0:b1].permute(0, 2, 1, 3, 4).reshape(Ly, H, n * Hq // H, d)
        xp = torch.matmul(qg, kp.transpose(2, 3)) * s.scale  # [Ly, H, n * G, p]
        # each sequence's own rows
        j = p + torch.arange(s.most, device=DEV)
        seen = j < s.lens[:, b0:b1].unsqueeze(-1)  # [Ly, n, H, most]
        pg = s.table[b0:b1].long()[:, (j // page).clamp(max=s.table.shape[1] - 1)].clamp(min=0).view(1, n, 1, -1)
        where = (ly.unsqueeze(-1), pg, heads.unsqueeze(-1), (j % page).view(1, 1, 1, -1))
        kg, vg = s.K[where].float(), s.V[where].float()  # [Ly, n, H, most, d]
        vg = torch.where(seen.unsqueeze(-1), vg, 0.0)
        xo = torch.matmul(q[:, b0:b1], kg.transpose(3, 4)) * s.scale  # [Ly, n, H, G, most]
        xo = torch.where(seen.unsqueeze(3), xo, -math.inf)
        xp = xp.view(Ly, H, n, Hq // H, p).permute(0, 2, 1, 3, 4)  # [Ly, n, H, G, p]
        m = xo.amax(-1, keepdim=True)
        if p > 0:
            m = torch.maximum(m, xp.amax(-1, keepdim=True))
        ep, eo = torch.exp(xp - m), torch.exp(xo - m)
        z = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
        acc = torch.matmul(ep.permute(0, 2, 1, 3, 4).reshape(Ly, H, n * Hq // H, p), vp)
        acc = acc.view(Ly, H, n, Hq // H, d).permute(0, 2, 1, 3, 4) + torch.matmul(eo, vg)
        s.out[:, b0:b1] = (acc / z).reshape(Ly, n, Hq, d).to(s.out.dtype)
        s.lse[:, b0:b1] = (m + torch.log(z)).view(Ly, n, Hq)


def run(s):
    """One append, or one token's attention (from the same lengths in every pass)."""
    c = s.case
    s.lens.copy_(s.lens0)
    if c["kind"] == "append":
        if own:
            q, k, v = s.qkv.split([c["h_q"], c["h_kv"], c["h_kv"]], dim=2)
            s.reco.reco_paged_append(s.kv, k, v, s.starts, s.lens, s.ws, pos=s.pos, inv_freq=s.inv_freq, q=q,
                                     q_out=s.q_out, interleaved=c["interleaved"])
        else:
            _append_plain(s)
        return {"K": s.K, "V": s.V, "q": s.q_out, "lens": s.lens}
    if own:
        s.reco.reco_paged_prefix_attn(s.kv, s.q, s.kn, s.vn, s.lens, s.group, s.shared, s.scale, s.out, s.lse, s.ws)
    else:
        _prefix_plain(s)
    return {"out": s.out, "lse": s.lse, "lens": s.lens, "K": s.K, "V": s.V}


# ---------------------------------------------------------------- the same in float64
def _exact_append(c, seed):
    s = prepare(c, seed)
    H, Hq, page, rot = c["h_kv"], c["h_q"], c["page"], c["rot"]
    K, q_out = s.K.double(), s.q_out.double()
    starts, lens, table = s.starts.tolist(), s.lens0.cpu().numpy(), s.table.cpu().numpy()
    f = np.asarray(s.inv_freq.cpu().numpy(), np.float64)
    z = np.exp(1j * s.pos.cpu().numpy().astype(np.float64)[:, None] * f)  # a rotation is a complex product
    z = _to(z).view(-1, 1, rot // 2)
    lo = torch.arange(0, rot, 2, device=DEV) if c["interleaved"] else torch.arange(rot // 2, device=DEV)
    hi = lo + (1 if c["interleaved"] else rot // 2)
    for ly in range(c["layers"]):
        x = s.qkv[ly, :, :Hq + H].double()
        turned = torch.complex(x[..., lo], x[..., hi]) * z
        x[..., lo], x[..., hi] = turned.real, turned.imag
        for b in range(c["batch"]):
            t0, t1 = starts[b], starts[b + 1]
            q_out[ly, t0:t1] = x[t0:t1, :Hq]
            for h in range(H):
                rows = np.arange(lens[ly, b, h], lens[ly, b, h] + t1 - t0)
                K[ly, _to(table[b][rows // page].astype(np.int64)), h, _to(rows % page)] = x[t0:t1, Hq + h]
    return {"K": K, "V": None, "q": q_out, "lens": None}


def _exact_prefix(c, seed):
    s = prepare(c, seed)
    Ly, B, H, G, d, page = c["layers"], c["batch"], c["h_kv"], c["h_q"] // c["h_kv"], c["d"], c["page"]
    out = torch.zeros((Ly, B, H * G, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((Ly, B, H * G), dtype=torch.float64, device=DEV)
    lens, table, group = s.lens0.cpu().numpy(), s.table.cpu().numpy(), s.group.tolist()
    for b in range(B):
        lead = group.index(group[b])
        p = int(s.shared[b])
        for ly in range(Ly):
            n = lens[ly, b]  # [H] rows without the new one
            j = np.arange(int(n.max()))
            ids = np.where(j < p, table[lead][j // page], table[b][j // page])
            ids, at = _to(ids.astype(np.int64)), _to(j % page)
            k, v = s.K[ly, ids, :, at].double(), s.V[ly, ids, :, at].double()  # [rows, H, d]
            hide = _to(j[:, None] >= n[None, :])
            if c["append"]:
                k, v = torch.cat([k, s.kn[ly, b].double()[None]]), torch.cat([v, s.vn[ly, b].double()[None]])
                hide = torch.cat([hide, torch.zeros((1, H), dtype=torch.bool, device=DEV)])
            logit = torch.einsum("hgd,jhd->hgj", s.q[ly, b].double().view(H, G, d), k) * s.scale
            logit = logit.masked_fill(hide.T.unsqueeze(1), -math.inf)
            norm = torch.logsumexp(logit, -1)
            prob = torch.exp(logit - norm.unsqueeze(-1))
            out[ly, b] = torch.einsum("hgj,jhd->hgd", prob, v.masked_fill(hide.unsqueeze(-1), 0.0)).reshape(H * G, d)
            lse[ly, b] = norm.reshape(H * G)
    return {"out": out, "lse": lse, "lens": None, "K": None, "V": None}


def exact(c, seed):
    return _exact_append(c, seed) if c["kind"] == "append" else _exact_prefix(c, seed)


# ---------------------------------------------------------------- what a pass cannot do without
def _mean(lo, hi):
    """Mean of _spread's whole numbers (log-uniform)."""
    return float(lo) if hi <= lo else (hi - lo) / math.log((hi + 2) / (lo + 1))


def work(c):
    Ly, B, H, Hq, d = c["layers"], c["batch"], c["h_kv"], c["h_q"], c["d"]
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "append":  # projections read, rows and queries written
        n = B * _mean(c["lo"], c["hi"])
        return {"bytes": n * (Ly * 2 * (2 * H + Hq) * d * es + 4) + 8 * Ly * B * H,
                "flops": 3.0 * n * Ly * (Hq + H) * c["rot"]}
    p, mine = _mean(c["p_lo"], c["p_hi"]), _mean(c["lo"], c["hi"]) + (1 if c["append"] else 0)
    rows = Ly * H * (c["groups"] * p + B * mine)  # the prefix once per group
    by = rows * 2 * d * es + Ly * B * Hq * (d * es + d * (4 if c["out_f32"] else es) + 4) + Ly * B * H * (4 * d * es + 8)
    return {"bytes": by + 4 * rows / (H * Ly * c["page"]), "flops": 4.0 * Ly * B * Hq * d * (p + mine)}
