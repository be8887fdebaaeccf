"""Plain restatement of the paged cache's operators -- TEST INFRASTRUCTURE.

Page tables: one slot and one page after the other, in order.  Attention: one
request after the other over its tokens in a plain row, in 64 bits.  Host tensors in and out; nothing here imports the HIP
path.
"""
from __future__ import annotations

import math

import torch

BAD_INST, BAD_LEN, BAD_PAGE, BAD_PARENT, NO_PAGES = 1, 8, 16, 32, 64


def _ceil(a, b):
    return -(-a // b)


def assign(table, seq_len, seq_inst, refs, kv, new_len, parent=None, inst_of=None, *, n_inst,
           page_size):
    """(table, seq_len, seq_inst, refs, kv, flags) after star_assign_pages; kv [layers, pages, ...]."""
    n, M = table.shape
    ps, P, n_pages = page_size, refs.numel() // n_inst, refs.numel()
    t_in, L, I, R = (x.tolist() for x in (table, seq_len, seq_inst, refs))
    t_out, L_out, I_out, R_out = [list(r) for r in t_in], list(L), list(I), list(R)
    kv_out = kv.clone()
    free = [[x for x in range(i * P, (i + 1) * P) if R[x] == 0] for i in range(n_inst)]
    run, flags = [0] * n_inst, 0
    fine = lambda x: 0 <= x < n_pages
    source = lambda b: b if parent is None else int(parent[b])
    target = lambda b: I[b] if inst_of is None else int(inst_of[b])

    def whole(b):
        """Pages of its source that slot b may share in any case: full ones, and in
        a fork or a cut not that of its last token."""
        a, want = source(b), int(new_len[b])
        if a != b or want < L[a]:
            return max(0, min(want - 1, L[a]) // ps)
        return L[a] // ps

    taken = [0] * n                    # pages of a slot that forks share
    for c in range(n):
        a = source(c)
        if (0 <= a < n and a != c and 0 <= int(new_len[c]) <= M * ps and
                all(0 <= L[x] <= M * ps and 0 <= I[x] < n_inst for x in (a, c)) and
                I[a] == target(c)):
            taken[a] = max(taken[a], whole(c))
    for b in range(n):
        a, want, to = source(b), int(new_len[b]), target(b)
        ok = True
        if not (0 <= L[b] <= M * ps and 0 <= want <= M * ps):
            ok, flags = False, flags | BAD_LEN
        if not (0 <= I[b] < n_inst and 0 <= to < n_inst):
            ok, flags = False, flags | BAD_INST
        if not -1 <= a < n:
            ok, flags = False, flags | BAD_PARENT
        if ok and a >= 0 and a != b:
            if not 0 <= L[a] <= M * ps:
                ok, flags = False, flags | BAD_LEN
            if not 0 <= I[a] < n_inst:
                ok, flags = False, flags | BAD_INST
        if not ok:
            continue
        keep = min(want, L[a]) if a >= 0 else 0
        shared = 0
        if a >= 0 and I[a] == to:
            shared = whole(b)
            if (a == b and shared * ps < keep and fine(t_in[b][shared]) and
                    R[t_in[b][shared]] == 1 and taken[b] <= shared):
                shared += 1
        kept, pages, old = _ceil(keep, ps), _ceil(want, ps), _ceil(L[b], ps)
        need = pages - shared
        first = run[to]
        run[to] += need
        if need and run[to] > len(free[to]):
            flags |= NO_PAGES
            continue
        row = [t_in[a][j] for j in range(shared)]
        row += free[to][first:first + need]
        for j in range(shared, kept):
            if fine(t_in[a][j]):
                kv_out[:, row[j]] = kv[:, t_in[a][j]]
            else:
                flags |= BAD_PAGE
        stays = shared if a == b else 0          # pages that the row keeps
        for j in range(stays, old):
            if fine(t_in[b][j]):
                R_out[t_in[b][j]] -= 1
            else:
                flags |= BAD_PAGE
        for j in range(stays, pages):
            if fine(row[j]):
                R_out[row[j]] += 1
            else:
                flags |= BAD_PAGE
        t_out[b][:pages] = row
        L_out[b], I_out[b] = want, to
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)
    return i32(t_out).reshape(n, M), i32(L_out), i32(I_out), i32(R_out), kv_out, flags


def compact(table, seq_len, refs, kv, *, n_inst, page_size):
    """(table, refs, n_live, kv, flags) after star_compact_pages."""
    P, n_pages = refs.numel() // n_inst, refs.numel()
    n, M = table.shape
    R, R_out, kv_out, flags = refs.tolist(), refs.tolist(), kv.clone(), 0
    move, n_live = {}, []
    for i in range(n_inst):
        live = [x for x in range(i * P, (i + 1) * P) if R[x] != 0]
        line = i * P + len(live)
        holes = [x for x in range(i * P, line) if R[x] == 0]
        for src, dst in zip([x for x in live if x >= line], holes):
            move[src] = dst
            R_out[dst], R_out[src] = R[src], 0
            kv_out[:, dst] = kv[:, src]
        n_live.append(len(live))
    t = table.tolist()
    for b in range(n):
        if not 0 <= int(seq_len[b]) <= M * page_size:
            flags |= BAD_LEN
            continue
        for j in range(_ceil(int(seq_len[b]), page_size)):
            if 0 <= t[b][j] < n_pages:
                t[b][j] = move.get(t[b][j], t[b][j])
            else:
                flags |= BAD_PAGE
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)
    return i32(t).reshape(n, M), i32(R_out), i32(n_live), kv_out, flags


def attend(q, k_new, v_new, kv, table, seq_len, q_start=None, *, scale, window=0, sinks=0):
    """Attention of new tokens over one layer's pages [n_pages, 2, n_kv, page_size, D].

    Returns a dict: out and lse in 64 bits, `written` (the rows that are), kv
    afterwards, `mass` = sum_j p_j |v_j| and `reach` = the largest
    scale sum |q||k| of a row (what error bounds are made of), and flags.
    """
    n_pages, _, n_kv, ps, D = kv.shape
    n, M = table.shape
    n_rows, Hq = q.shape[0], q.shape[1]
    g, kv_out, flags = Hq // n_kv, kv.clone(), 0
    out = torch.zeros((n_rows, Hq, D), dtype=torch.float64)
    written = torch.zeros(n_rows, dtype=torch.bool)
    mass = torch.zeros((n_rows, Hq, D), dtype=torch.float64)
    lse = torch.full((n_rows, Hq), -math.inf, dtype=torch.float64)
    reach = torch.zeros((n_rows, Hq), dtype=torch.float64)
    plan = []
    for b in range(n):
        L = int(seq_len[b])
        lo, hi = (b, b + 1) if q_start is None else (int(q_start[b]), int(q_start[b + 1]))
        T = hi - lo
        if not (0 <= L <= M * ps and 0 <= lo <= hi <= n_rows and (q_start is None or T <= L)):
            flags |= BAD_LEN
            continue
        written[lo:hi] = True
        if L == 0:
            continue
        plan.append((b, L, lo, T))
        for i in range(T):
            j = L - T + i
            page = int(table[b, j // ps])
            if 0 <= page < n_pages:
                kv_out[page, 0, :, j % ps] = k_new[lo + i]
                kv_out[page, 1, :, j % ps] = v_new[lo + i]
    for b, L, lo, T in plan:
        k = torch.zeros((n_kv, L, D), dtype=torch.float64)
        v = torch.zeros((n_kv, L, D), dtype=torch.float64)
        there = torch.zeros(L, dtype=torch.bool)
        seen = torch.zeros(L, dtype=torch.bool)
        j = torch.arange(L)
        for i in range(T):
            p = L - T + i
            see = j <= p
            if window:
                see &= (j > p - window) | (j < sinks)
            seen |= see
        for x in range(_ceil(L, ps)):
            at = slice(x * ps, min(L, (x + 1) * ps))
            page = int(table[b, x])
            if 0 <= page < n_pages:
                k[:, at] = kv_out[page, 0, :, : at.stop - at.start].double()
                v[:, at] = kv_out[page, 1, :, : at.stop - at.start].double()
                there[at] = True
            elif seen[at].any():
                flags |= BAD_PAGE
        def visible(p):
            see = (j <= p) & there
            return see & ((j > p - window) | (j < sinks)) if window else see

        # query head h reads key-value head h // g
        kg, vg = (t.repeat_interleave(g, dim=0) for t in (k, v))
        # values that are not finite reach the rows that see them, as by a positive weight
        odd = ~torch.isfinite(vg)
        vf = vg.masked_fill(odd, 0.0)
        for at in range(0, T, 64):
            rows = slice(lo + at, lo + min(T, at + 64))
            pos = torch.arange(L - T + at, L - T + at + rows.stop - rows.start)
            see = torch.stack([visible(int(p)) for p in pos])          # [rows, L]
            qh = q[rows].double().transpose(0, 1)                      # [Hq, rows, D]
            z = (scale * (qh @ kg.transpose(1, 2))).masked_fill(~see, -math.inf)
            top = z.max(dim=2).values
            e = torch.exp(z - top.clamp(min=-1e300)[..., None])
            total = e.sum(2)
            pr = e / total.clamp(min=1e-300)[..., None]
            o = pr @ vf
            if odd.any():
                for x, here in ((math.inf, vg == math.inf), (-math.inf, vg == -math.inf),
                                (math.nan, torch.isnan(vg))):
                    o = torch.where(see.double() @ here.double() > 0, o + x, o)
            out[rows] = o.transpose(0, 1)
            mass[rows] = (pr @ vf.abs()).transpose(0, 1)
            lse[rows] = (top + torch.log(total)).transpose(0, 1)
            span = (abs(scale) * (qh.abs() @ kg.abs().transpose(1, 2))).masked_fill(~see, 0.0)
            reach[rows] = span.max(dim=2).values.transpose(0, 1)
    return dict(out=out, lse=lse, written=written, mass=mass, reach=reach, kv=kv_out, flags=flags)
