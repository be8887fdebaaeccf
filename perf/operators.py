"""Performance cases of the paged key-value cache and of the attention that
reads it: the calls of one decode instance between two rescheduling rounds, at
the sizes of the repository's workloads and over the ranges around them.

Kinds of case, each one pass through the public entry points of
``paper_2510_13668_amd.star``:

* ``decode``: attention of one new token a request over its cached pages; the
  token's keys and values join the cache in the same call.
* ``prompt``: attention of several new tokens a request (a prompt, or the next
  chunk of one), with the tokens' keys and values written to the cache.
* ``assign``: pages for the requests' next lengths: growth, release, forks and
  the migrations of a plan.
* ``compact``: the live pages of each instance to its lowest indices.

Where ``own`` is false a pass computes the same in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# (query heads, key-value heads, head width) of the repository's hidden widths
HEADS = {"1024": (16, 16, 64), "3584": (28, 4, 128), "4096": (32, 8, 128), "5120": (40, 8, 128),
         "8192": (64, 8, 128), "narrow": (8, 2, 64), "wide": (8, 4, 256), "one_kv": (20, 1, 128)}
LARGEST_KV = 2.3e9          # bytes of keys and values the largest decode case reads
LARGEST_FLOPS = 5.5e11      # the largest prompt case
LARGEST_POOL = 2.0e9        # bytes of the largest page pool of assign and compact


def listed():
    return [
        # the smallest decode step: one fp32 instance of the 64-request cluster
        dict(name="decode_tiny_f32", kind="decode", n_seq=16, heads="1024", dtype="f32", page=16,
             lo=1, hi=2048, window=0, sinks=0, empty=0, lse=True),
        # one instance of the headline batch (1024 requests on 8), a padded batch
        dict(name="decode_continuous", kind="decode", n_seq=128, heads="4096", dtype="bf16",
             page=16, lo=128, hi=8192, window=0, sinks=0, empty=3, lse=False),
        # two requests with the longest caches: few rows, a long axis
        dict(name="decode_two_long", kind="decode", n_seq=2, heads="3584", dtype="bf16", page=64,
             lo=60001, hi=65536, window=0, sinks=0, empty=0, lse=False),
        # the long-reasoning batch of one instance under a sliding window with
        # four first tokens that stay visible
        dict(name="decode_window", kind="decode", n_seq=256, heads="5120", dtype="bf16", page=16,
             lo=256, hi=16384, window=1000, sinks=4, empty=0, lse=True),
        # a handful of prompts of the simulator's lengths, admitted together
        dict(name="prompt_ragged", kind="prompt", n_seq=6, heads="3584", dtype="bf16", page=16,
             q_lo=128, q_hi=4096, past=0, window=0, sinks=0, lse=False),
        # the largest: one prompt of 8192 tokens
        dict(name="prompt_long", kind="prompt", n_seq=1, heads="4096", dtype="bf16", page=64,
             q_lo=8191, q_hi=8191, past=0, window=0, sinks=0, lse=False),
        # the next chunk of four long prompts, windowed with sinks
        dict(name="prompt_chunk_window", kind="prompt", n_seq=4, heads="5120", dtype="bf16",
             page=16, q_lo=500, q_hi=515, past=12000, window=4096, sinks=4, lse=True),
        # every decode step: each of 1024 requests grows by one token, some
        # finish, new ones take their slots; nothing is copied
        dict(name="assign_step", kind="assign", n_seq=1024, n_inst=8, page=16, n_pages=65536,
             layers=1, page_bytes=256, len_hi=2000, grow=1, fork=0.0, move=0.0, drop=0.02),
        # a plan's migrations: a few requests' pages follow, over all layers
        dict(name="assign_migrate", kind="assign", n_seq=96, n_inst=8, page=16, n_pages=2048,
             layers=28, page_bytes=32768, len_hi=400, grow=1, fork=0.0, move=0.2, drop=0.02),
        # parallel samples: half the slots become forks of another one
        dict(name="assign_fork", kind="assign", n_seq=512, n_inst=1, page=64, n_pages=2048,
             layers=8, page_bytes=65536, len_hi=300, grow=1, fork=0.5, move=0.0, drop=0.0),
        # a small pool, half full
        dict(name="compact_small", kind="compact", n_seq=64, n_inst=1, page=16, n_pages=1024,
             layers=4, page_bytes=8192, len_hi=256),
        # the largest: eight instances' pools over all layers
        dict(name="compact_large", kind="compact", n_seq=256, n_inst=8, page=16, n_pages=2048,
             layers=28, page_bytes=32768, len_hi=130),
    ]


# ---------------------------------------------------------------------------
# more cases of the same ranges
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_attention(rng, kind):
    heads, dtype = rng.choice(sorted(HEADS)), rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = dict(kind=kind, heads=heads, dtype=dtype, page=rng.choice([16, 32, 64, 128]),
             window=rng.choice([0, 0, _log(rng, 1, 4096)]), sinks=rng.choice([0, 1, 4, 50]),
             lse=rng.random() < 0.5)
    while True:
        if kind == "decode":
            c.update(n_seq=_log(rng, 1, 512), hi=_log(rng, 1, 65536))
            c.update(lo=rng.randint(1, c["hi"]), empty=rng.choice([0, 0, 1, 5]))
            ok = _kv_bytes(c, c["n_seq"] * c["hi"]) <= LARGEST_KV
        else:
            c.update(n_seq=_log(rng, 1, 16), q_hi=_log(rng, 2, 8192),
                     past=rng.choice([0, _log(rng, 1, 16384)]))
            c["q_lo"] = rng.randint(1, c["q_hi"])
            Hq = HEADS[heads][0]
            area = 4.0 * c["n_seq"] * Hq * c["q_hi"] * (c["past"] + c["q_hi"])  # plain scores
            ok = (work(c)["flops"] <= LARGEST_FLOPS / (16 if dtype == "f32" else 1) and
                  area <= 1.2e10)
        if ok:
            return c


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "prompt", "prompt", "prompt", "assign",
                       "assign", "compact"])
    if kind in ("decode", "prompt"):
        return _draw_attention(rng, kind)
    while True:
        c = dict(kind=kind, n_seq=_log(rng, 1, 4096), n_inst=rng.choice([1, 1, 2, 8]),
                 page=rng.choice([16, 32, 64, 128]), layers=rng.randint(1, 28),
                 page_bytes=16 * _log(rng, 1, 4096), len_hi=_log(rng, 16, 8192))
        P = 1 + int(1.5 * c["n_seq"] / c["n_inst"] * (c["len_hi"] / (2 * c["page"]) + 1))
        c["n_pages"] = c["n_inst"] * P
        if c["n_pages"] * c["layers"] * c["page_bytes"] <= LARGEST_POOL and c["n_pages"] <= 262144:
            break
    if kind == "assign":
        c.update(grow=rng.choice([1, 1, rng.randint(2, 64)]), fork=rng.choice([0.0, 0.0, 0.3]),
                 move=rng.choice([0.0, 0.1]) if c["n_inst"] > 1 else 0.0,
                 drop=rng.choice([0.0, 0.05]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n whole numbers spread evenly over lo..hi, the same for every seed."""
    return np.floor(lo + (hi - lo + 1) * (np.arange(n) + 0.5) / max(n, 1)).astype(np.int64)


def _lengths(c):
    """(cached tokens after the call, new tokens) of each request, unshuffled."""
    n = c["n_seq"]
    if c["kind"] == "decode":
        total = _spread(c["lo"], c["hi"], n)
        total[: min(c["empty"], n - 1)] = 0
        return total, np.minimum(total, 1)
    new = _spread(c["q_lo"], c["q_hi"], n)
    return new + _spread(0, c["past"], n) * (c["past"] > 0), new


def _dev(a, dt=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dt).to(DEV)


def _normal(g, shape, dt, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=dt) * scale


def _attention_inputs(c, seed):
    """q ~ N(0, 2^2), k and v ~ N(0, 1); a request's pages lie anywhere in the pool."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    Hq, Hkv, D = HEADS[c["heads"]]
    dt, ps, n = DTYPES[c["dtype"]], c["page"], c["n_seq"]
    total, new = _lengths(c)
    order = rng.permutation(n)
    total, new = total[order], new[order]
    used = -(-total // ps)
    M, n_pages = int(max(1, used.max())), int(used.sum()) + 8
    where = rng.permutation(n_pages)
    first = np.cumsum(used) - used
    j = np.arange(M)[None, :]
    table = np.where(j < used[:, None], where[np.minimum(first[:, None] + j, n_pages - 1)], -1)
    rows = n if c["kind"] == "decode" else int(new.sum())
    # queries, keys and values are columns of one projection's output
    qkv = _normal(g, (rows, Hq + 2 * Hkv, D), dt)
    qkv[:, :Hq] *= 2.0
    return dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:],
                kv=_normal(g, (n_pages, 2, Hkv, ps, D), dt), table=_dev(table),
                seq_len=_dev(total), q_start=_dev(np.concatenate([[0], np.cumsum(new)])),
                new_len=_dev(new), max_new=int(new.max()), n_pages=n_pages, max_pages=M,
                scale=D ** -0.5, out=torch.zeros((rows, Hq, D), dtype=dt, device=DEV),
                lse=torch.zeros((rows, Hq), dtype=torch.float32, device=DEV) if c["lse"] else None)


def _pool_inputs(c, seed):
    """Requests in blocks over the instances, pages anywhere in the instance's
    range; every fourth request shares its first pages with the one before."""
    rng = np.random.default_rng(seed)
    n, I, ps, P = c["n_seq"], c["n_inst"], c["page"], c["n_pages"] // c["n_inst"]
    M = -(-(c["len_hi"] + c.get("grow", 0)) // ps)
    inst = (np.arange(n) * I) // n
    length = rng.permutation(_spread(1, c["len_hi"], n))
    most = int(0.8 * P) // max(1, -(-n // I))          # pages a request may hold
    length = np.minimum(length, np.maximum(rng.integers(1, 2 * most + 1, n), 1) * ps)
    used = -(-length // ps)
    for i in range(I):                                  # what does not fit waits outside
        at = np.flatnonzero(inst == i)
        length[at[np.cumsum(used[at]) > 0.8 * P]] = 0
    used = -(-length // ps)
    where = np.stack([i * P + rng.permutation(P) for i in range(I)])
    first = np.zeros(n, np.int64)
    for i in range(I):
        at = inst == i
        first[at] = np.cumsum(used[at]) - used[at]
    j = np.arange(M)[None, :]
    table = where[inst[:, None], np.minimum(first[:, None] + j, P - 1)]
    back = np.maximum(np.arange(n) - 1, 0)
    share = np.where((np.arange(n) % 4 == 3) & (inst == inst[back]),
                     np.minimum(length, length[back]) // ps, 0)
    table = np.where(j < share[:, None], table[back], table)
    held = j < used[:, None]
    table = np.where(held, table, -1)
    refs = np.bincount(table[held], minlength=I * P)
    s = dict(n_pages=I * P, max_pages=M, table=_dev(table), seq_len=_dev(length),
             seq_inst=_dev(inst), refs=_dev(refs),
             kv=torch.randint(-32768, 32768, (c["layers"], I * P, c["page_bytes"] // 2),
                              generator=torch.Generator(device=DEV).manual_seed(seed),
                              dtype=torch.int16, device=DEV))
    if c["kind"] == "assign":
        parent, to, new = np.arange(n), inst.copy(), length + c["grow"]
        pick = rng.random(n)
        fork = (pick < c["fork"]) & (n > 1)
        parent[fork] = rng.integers(0, n, int(fork.sum()))
        new[fork] = length[parent[fork]] + c["grow"]
        drop = (pick >= c["fork"]) & (pick < c["fork"] + c["drop"])
        parent[drop] = -1                               # the slot starts anew, or stays empty
        new[drop] = np.where(rng.random(int(drop.sum())) < 0.5, 0, rng.integers(1, c["len_hi"] + 1))
        move = pick > 1.0 - c["move"]
        to[move] = rng.integers(0, I, int(move.sum()))
        s.update(parent=_dev(parent), new_len=_dev(np.minimum(new, M * ps)), inst_of=_dev(to),
                 forks=bool(fork.any() or drop.any()), seq_len_out=torch.zeros_like(s["seq_len"]),
                 seq_inst_out=torch.zeros_like(s["seq_inst"]))
    else:
        s["n_live"] = torch.zeros(I, dtype=torch.int32, device=DEV)
    s.update(table_out=s["table"].clone(), refs_out=torch.zeros_like(s["refs"]))
    return s


def prepare(case, seed):
    c = case
    attention = c["kind"] in ("decode", "prompt")
    s = _attention_inputs(c, seed) if attention else _pool_inputs(c, seed)
    s["c"] = c
    if own:
        from paper_2510_13668_amd import star
        if attention:
            Hq, Hkv, D = HEADS[c["heads"]]
            s["p"] = star.attend_params(
                c["n_seq"], s["q"].shape[0], Hq, Hkv, D, star.BF16 if c["dtype"] == "bf16"
                else star.F32, c["page"], s["n_pages"], s["max_pages"], s["scale"], c["window"],
                c["sinks"], q_stride=s["q"].stride(0), kv_stride=s["k"].stride(0))
            size = (star.attend_decode_workspace_size if c["kind"] == "decode" else
                    star.attend_prompt_workspace_size)(s["p"])
        else:
            s["p"] = star.pages_params(c["n_seq"], s["max_pages"], s["n_pages"], c["page"],
                                       c["layers"], c["page_bytes"], n_inst=c["n_inst"])
            size = (star.assign_pages_workspace_size if c["kind"] == "assign" else
                    star.compact_pages_workspace_size)(s["p"])
        s["ws"] = star.Workspace(size)
    return s


# ---------------------------------------------------------------------------
# one pass in elementary operations
# ---------------------------------------------------------------------------
def _store(kv, table, at, slot, k, v):
    """Keys and values of tokens at positions `at` of requests `slot`."""
    ps = kv.shape[3]
    page = table[slot, at // ps].long()
    kv[page, 0, :, at % ps] = k
    kv[page, 1, :, at % ps] = v


def _attend(s, q, first_pos, rows_mask):
    """q [n, Hkv, r, D] in 32 bits, row r of request b at position first_pos[b, r]."""
    c, kv = s["c"], s["kv"]
    n, Hkv, R, D = q.shape
    pages = kv[s["table"].clamp(min=0).long()]                   # [n, M, 2, Hkv, ps, D]
    k, v = (pages[:, :, x].float().transpose(1, 2).reshape(n * Hkv, -1, D) for x in (0, 1))
    z = torch.bmm(q.reshape(n * Hkv, R, D) * s["scale"], k.transpose(1, 2)).view(n, Hkv, R, -1)
    j = torch.arange(z.shape[-1], device=DEV)
    p = first_pos[:, :, None]
    see = (j <= p) & rows_mask[:, :, None]
    if c["window"]:
        see &= (j > p - c["window"]) | (j < c["sinks"])
    z = z.masked_fill(~see[:, None], -math.inf)
    top = z.amax(dim=-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(z - top)
    total = e.sum(dim=-1, keepdim=True)
    o = torch.bmm(e.view(n * Hkv, R, -1), v).view(n, Hkv, R, D) / total.clamp(min=1e-30)
    return o, (top + torch.log(total)).squeeze(-1)


def _plain_decode(s):
    q, L = s["q"], s["seq_len"].long()
    n, Hq, D = q.shape
    Hkv = s["k"].shape[1]
    live = torch.nonzero(L > 0).squeeze(1)
    _store(s["kv"], s["table"], L[live] - 1, live, s["k"][live], s["v"][live])
    pos = (L - 1)[:, None].expand(n, Hq // Hkv)
    o, lse = _attend(s, q.float().reshape(n, Hkv, Hq // Hkv, D), pos, pos >= 0)
    return o.reshape(n, Hq, D).to(q.dtype), lse.reshape(n, Hq)


def _plain_prompt(s):
    q, L, new = s["q"], s["seq_len"].long(), s["new_len"].long()
    Hq, D, n, T = q.shape[1], q.shape[2], len(new), s["max_new"]
    Hkv = s["k"].shape[1]
    slot = torch.repeat_interleave(torch.arange(n, device=DEV), new)
    i = torch.arange(q.shape[0], device=DEV) - s["q_start"].long()[slot]
    _store(s["kv"], s["table"], (L - new)[slot] + i, slot, s["k"], s["v"])
    wide = torch.zeros((n, T, Hq, D), device=DEV)
    wide[slot, i] = q.float()
    g = Hq // Hkv
    wide = wide.view(n, T, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(n, Hkv, T * g, D)
    row = torch.arange(T, device=DEV).repeat_interleave(g)[None, :]
    o, lse = _attend(s, wide, (L - new)[:, None] + row, row < new[:, None])
    o = o.view(n, Hkv, T, g, D).permute(0, 2, 1, 3, 4).reshape(n, T, Hq, D)
    lse = lse.view(n, Hkv, T, g).permute(0, 2, 1, 3).reshape(n, T, Hq)
    return o[slot, i].to(q.dtype), lse[slot, i].contiguous()


def _count(table, held, n_pages):
    """How often each page stands in the held places of a table."""
    page = torch.where(held, table, n_pages).long().reshape(-1)
    return torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV).index_add_(
        0, page, torch.ones_like(page, dtype=torch.int32))[:n_pages]


def _plain_assign(s):
    c, table, refs, length = s["c"], s["table"].long(), s["refs"], s["seq_len"].long()
    n, M, ps, I, P = c["n_seq"], s["max_pages"], c["page"], c["n_inst"], s["n_pages"] // c["n_inst"]
    me, j = torch.arange(n, device=DEV), torch.arange(M, device=DEV)[None, :]
    a, new, to = s["parent"].long(), s["new_len"].long(), s["inst_of"].long()
    from_ = a.clamp(min=0)
    keep = torch.minimum(new, torch.where(a >= 0, length[from_], 0))
    same = (a >= 0) & (s["seq_inst"].long()[from_] == to)
    full, part = keep // ps, keep % ps > 0
    last = table[from_, full.clamp(max=M - 1)].clamp(min=0)
    shared = torch.where(same, full + (part & (a == me) & (refs[last] == 1)), 0)
    pages, kept = -(-new // ps), -(-keep // ps)
    need = pages - shared
    order = torch.argsort((refs.view(I, P) != 0).int(), dim=1, stable=True)   # free ones first
    free = (refs.view(I, P) == 0).sum(dim=1)
    mine = torch.where(to[:, None] == torch.arange(I, device=DEV), need[:, None], 0)
    upto = mine.cumsum(dim=0)[me, to]
    served = (need == 0) | (upto <= free[to])
    rank = (upto - need)[:, None] + j - shared[:, None]
    fresh = to[:, None] * P + order[to[:, None], rank.clamp(0, P - 1)]
    held, old = j < pages[:, None], j < -(-length // ps)[:, None]
    row = torch.where(j < shared[:, None], table[from_], fresh)
    row = torch.where(held & served[:, None], row, table)
    b, x = torch.nonzero((j >= shared[:, None]) & (j < kept[:, None]) & served[:, None],
                         as_tuple=True)
    s["kv"][:, row[b, x]] = s["kv"][:, table[from_[b], x]]
    now = torch.where(served[:, None], held, old)
    return (row.int(), torch.where(served, new, length).int(),
            torch.where(served, to, s["seq_inst"].long()).int(),
            refs + _count(row, now, s["n_pages"]) - _count(table, old, s["n_pages"]))


def _plain_compact(s):
    c, refs, I = s["c"], s["refs"], s["c"]["n_inst"]
    P = s["n_pages"] // I
    live = refs.view(I, P) != 0
    n_live = live.sum(dim=1)
    # live pages of an instance keep their place below n_live; the others
    # take the holes there in order
    order = torch.arange(P, device=DEV)[None, :]
    low = order < n_live[:, None]
    hole, high = low & ~live, ~low & live
    i, x = torch.nonzero(high, as_tuple=True)
    src = i * P + x
    i, x = torch.nonzero(hole, as_tuple=True)
    dst = i * P + x
    to = torch.arange(s["n_pages"], device=DEV)
    to[src] = dst
    s["kv"][:, dst] = s["kv"][:, src]
    out = refs.clone()
    out[dst] = refs[src]
    out[src] = 0
    table = s["table"].long()
    held = torch.arange(s["max_pages"], device=DEV) < -(-s["seq_len"].long() // c["page"])[:, None]
    return torch.where(held, to[table.clamp(min=0)], table).int(), out, n_live.int()


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _bits(kv):
    return kv if kv.dtype == torch.int16 else kv.view(
        torch.int16 if kv.dtype == torch.bfloat16 else torch.int32)


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        from paper_2510_13668_amd import star
    if kind in ("decode", "prompt"):
        if own and kind == "decode":
            star.attend_decode(s["p"], s["q"], s["k"], s["v"], s["kv"], s["table"], s["seq_len"],
                               s["out"], s["lse"], s["ws"])
        elif own:
            star.attend_prompt(s["p"], s["q"], s["k"], s["v"], s["kv"], s["table"], s["seq_len"],
                               s["q_start"], s["out"], s["lse"], s["ws"])
        else:
            s["out"], lse = (_plain_decode if kind == "decode" else _plain_prompt)(s)
            s["lse"] = lse if c["lse"] else None
        out = {"out": s["out"], "kv": _bits(s["kv"])}
        if c["lse"]:
            out["lse"] = s["lse"]
        return out
    if kind == "assign":
        if own:
            star.assign_pages(s["p"], s["parent"] if s["forks"] else None, s["new_len"],
                              s["inst_of"], s["table"], s["seq_len"], s["seq_inst"], s["refs"],
                              s["kv"], s["table_out"], s["seq_len_out"], s["seq_inst_out"],
                              s["refs_out"], s["ws"])
        else:
            (s["table_out"], s["seq_len_out"], s["seq_inst_out"],
             s["refs_out"]) = _plain_assign(s)
        return {"table": s["table_out"], "seq_len": s["seq_len_out"],
                "seq_inst": s["seq_inst_out"], "refs": s["refs_out"], "kv": s["kv"]}
    if own:
        star.compact_pages(s["p"], s["table"], s["seq_len"], s["refs"], s["kv"], s["table_out"],
                           s["refs_out"], s["n_live"], s["ws"])
    else:
        s["table_out"], s["refs_out"], s["n_live"] = _plain_compact(s)
    return {"table": s["table_out"], "refs": s["refs_out"], "n_live": s["n_live"], "kv": s["kv"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def _kv_bytes(c, tokens):
    _, Hkv, D = HEADS[c["heads"]]
    return 2.0 * tokens * Hkv * D * (2 if c["dtype"] == "bf16" else 4)


def work(c):
    if c["kind"] in ("decode", "prompt"):
        Hq, Hkv, D = HEADS[c["heads"]]
        total, new = _lengths(c)
        W, S = c["window"] or 1 << 40, c["sinks"]
        pairs = read = 0
        for L, T in zip(total.tolist(), new.tolist()):
            p = np.arange(L - T, L, dtype=np.int64)          # row positions
            pairs += int(np.where(p + 1 <= W + S, p + 1, W + S).sum())
            lo = max(0, L - T - W + 1) if T else L           # keys of the window
            read += L - lo + min(lo, S) if T else 0
        e = 2 if c["dtype"] == "bf16" else 4
        rows = int(new.sum()) if c["kind"] == "prompt" else c["n_seq"]
        byte = _kv_bytes(c, read) + 2 * rows * Hq * D * e + 2 * _kv_bytes(c, int(new.sum()))
        byte += 4 * rows * Hq * c["lse"] + 4 * sum(-(-t // c["page"]) for t in total.tolist())
        return {"bytes": byte, "flops": 4.0 * pairs * Hq * D}
    # page tables, lengths and counts once in and once out, and the pages that
    # have to be copied: expected shares of the requests' pages
    n, ps = c["n_seq"], c["page"]
    M = -(-(c["len_hi"] + c.get("grow", 0)) // ps)
    most = max(1, int(0.8 * (c["n_pages"] // c["n_inst"])) // max(1, -(-n // c["n_inst"])))
    per = min(c["len_hi"] / (2.0 * ps) + 0.5, M, most)       # pages a request holds
    index = 8.0 * n * per + 8.0 * c["n_pages"] + 16.0 * n
    if c["kind"] == "assign":
        copied = n * (c["fork"] + c["move"] * per * (1.0 - 1.0 / c["n_inst"]))
    else:
        full = min(1.0, n * per / c["n_pages"])
        copied = c["n_pages"] * full * (1.0 - full)          # live pages above the line
    return {"bytes": index + 2.0 * copied * c["layers"] * c["page_bytes"], "flops": 0}


# ---------------------------------------------------------------------------
# the attention in 64 bits (page tables and copies are exact already)
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    if c["kind"] not in ("decode", "prompt"):
        return None
    x = _attention_inputs(c, seed)
    Hq, Hkv, D = HEADS[c["heads"]]
    g, ps = Hq // Hkv, c["page"]
    total, start = x["seq_len"].tolist(), x["q_start"].tolist()
    o = torch.zeros((x["q"].shape[0], Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((x["q"].shape[0], Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, L in enumerate(total):
        if L == 0:
            continue
        rows = slice(b, b + 1) if c["kind"] == "decode" else slice(start[b], start[b + 1])
        T = rows.stop - rows.start
        pages = x["table"][b, : -(-L // ps)].long()
        # the pages' tokens in order, the new tokens' own keys and values last
        k, v = (torch.cat([x["kv"][pages, w].transpose(0, 1).reshape(Hkv, -1, D)[:, : L - T],
                           x["k" if w == 0 else "v"][rows].transpose(0, 1)], dim=1).double()
                for w in (0, 1))
        j = torch.arange(L, device=DEV)
        for h in range(Hkv):
            for at in range(0, T, 1024):
                q = x["q"][rows][at:at + 1024, h * g:(h + 1) * g].double()
                pos = torch.arange(L - T + at, L - T + at + q.shape[0], device=DEV)[:, None]
                hidden = j > pos
                if c["window"]:
                    hidden |= (j <= pos - c["window"]) & (j >= c["sinks"])
                z = (q.reshape(-1, D) @ k[h].t()).view(q.shape[0], g, L) * x["scale"]
                z = torch.where(hidden[:, None], -math.inf, z)
                to = slice(rows.start + at, rows.start + at + q.shape[0])
                lse[to, h * g:(h + 1) * g] = torch.logsumexp(z, dim=-1)
                o[to, h * g:(h + 1) * g] = (torch.softmax(z, dim=-1).view(-1, L) @ v[h]).view(
                    q.shape[0], g, D)
    return {"out": o, "kv": None, "lse": lse} if c["lse"] else {"out": o, "kv": None}
