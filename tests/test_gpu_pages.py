"""Page tables of the cache on the GPU against the oracle: every integer and
every byte of the pool."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_13668_amd import star

pytestmark = pytest.mark.gpu
DEV = "cuda"


class State:
    """A random, consistent cache: pages anywhere, some rows sharing their first
    pages with the row before; `fill` of each instance's pages in use at most."""

    def __init__(self, seed, n, M, P, n_inst=1, ps=16, layers=2, page_bytes=64, fill=0.6,
                 len_hi=None):
        rng = np.random.default_rng(seed)
        self.n, self.M, self.P, self.n_inst, self.ps = n, M, P, n_inst, ps
        self.layers, self.page_bytes = layers, page_bytes
        inst = rng.integers(0, n_inst, n)
        length = rng.integers(0, (len_hi or M * ps) + 1, n)
        table = rng.integers(-5, n_inst * P + 5, (n, M))     # entries past the end: anything
        refs = np.zeros(n_inst * P, np.int64)
        free = [list(i * P + rng.permutation(P)) for i in range(n_inst)]
        room = [int(fill * P)] * n_inst
        for b in range(n):
            pages = -(-int(length[b]) // ps)
            share = 0
            if b and inst[b] == inst[b - 1] and rng.random() < 0.4:
                share = min(int(length[b]), int(length[b - 1])) // ps
            if pages - share > room[inst[b]]:
                length[b] = pages = share = 0
            room[inst[b]] -= pages - share
            row = list(table[b - 1, :share]) + [free[inst[b]].pop() for _ in range(pages - share)]
            table[b, :pages] = row
            refs[row] += 1
        i32 = lambda a: torch.from_numpy(np.asarray(a).astype(np.int32))
        self.table, self.len, self.inst, self.refs = map(i32, (table, length, inst, refs))
        self.kv = torch.from_numpy(
            rng.integers(-30000, 30000, (layers, n_inst * P, page_bytes // 2)).astype(np.int16))
        self.rng = rng

    def params(self):
        return star.pages_params(self.n, self.M, self.n_inst * self.P, self.ps, self.layers,
                                 self.page_bytes, n_inst=self.n_inst)


def _assign(s, new, parent=None, inst_of=None, in_place=False, stream=None):
    p = s.params()
    dev = lambda t: None if t is None else t.to(DEV)
    table, length, inst, refs, kv = map(dev, (s.table, s.len, s.inst, s.refs, s.kv))
    if in_place:
        t2, l2, i2, r2 = table, length, inst, refs
    else:
        t2, l2, i2, r2 = s.table.to(DEV), *(torch.full_like(x, -9) for x in (length, inst, refs))
    ws = star.Workspace(star.assign_pages_workspace_size(p))
    star.assign_pages(p, dev(parent), dev(new), dev(inst_of), table, length, inst, refs, kv, t2, l2,
                      i2, r2, ws, stream)
    torch.cuda.synchronize()
    got = [x.cpu() for x in (t2, l2, i2, r2, kv)]
    return got + [ws.read_device_error()]


def _check_assign(s, new, parent=None, inst_of=None, in_place=False):
    got = _assign(s, new, parent, inst_of, in_place)
    ref = paged.assign(s.table, s.len, s.inst, s.refs, s.kv, new, parent, inst_of,
                       n_inst=s.n_inst, page_size=s.ps)
    for name, x, y in zip(("table", "seq_len", "seq_inst", "refs", "kv"), got, ref):
        assert torch.equal(x, y), (name, torch.nonzero(x != y)[:5], x[x != y][:5], y[x != y][:5])
    assert got[5] == ref[5]
    return ref


@pytest.mark.parametrize("n,M,P,n_inst,ps,layers,page_bytes", [
    (1, 1, 3, 1, 16, 1, 16), (7, 3, 40, 1, 16, 3, 48), (64, 6, 100, 4, 32, 2, 4096),
    (300, 9, 700, 3, 16, 2, 80), (1500, 4, 5000, 1, 64, 1, 16), (33, 70, 1025, 2, 128, 2, 32768),
])
@pytest.mark.parametrize("what", ["grow", "release", "fork", "move", "all"])
def test_assign(n, M, P, n_inst, ps, layers, page_bytes, what):
    s = State(n + M, n, M, P, n_inst, ps, layers, page_bytes, fill=0.5,
              len_hi=max(1, min(M * ps, P * n_inst * ps // (2 * n))))
    print(f"assign {what} n={n} M={M} P={P} inst={n_inst} ps={ps}", flush=True)
    rng, most = s.rng, M * ps
    new = s.len.numpy().astype(np.int64)
    parent = inst_of = None
    if what in ("grow", "all"):
        new = new + rng.integers(0, 2 * ps, n)
    if what in ("release", "all"):
        cut = rng.random(n) < 0.4
        new[cut] = (new[cut] * rng.random(int(cut.sum()))).astype(np.int64)
        new[rng.random(n) < 0.2] = 0
    if what in ("fork", "all"):
        parent = np.where(rng.random(n) < 0.5, np.arange(n), rng.integers(-1, n, n))
        new = np.where(rng.random(n) < 0.5, s.len.numpy()[np.maximum(parent, 0)] + 1, new)
        parent = torch.from_numpy(parent.astype(np.int32))
    if what in ("move", "all"):
        inst_of = torch.from_numpy(np.where(rng.random(n) < 0.3, rng.integers(0, n_inst, n),
                                            s.inst.numpy()).astype(np.int32))
    new = torch.from_numpy(np.minimum(new, most).astype(np.int32))
    _check_assign(s, new, parent, inst_of)
    if parent is None:
        _check_assign(s, new, parent, inst_of, in_place=True)


def test_assign_when_pages_run_out():
    s = State(3, 50, 8, 90, 2, fill=1.0, len_hi=60)
    ref = _check_assign(s, torch.clamp(s.len + 40, max=128).to(torch.int32))
    assert ref[5] & paged.NO_PAGES and (ref[1] != s.len).any() and (ref[1] == s.len).any()


def test_assign_bad_contents_are_reported_and_left_out():
    s = State(4, 20, 4, 60, 2, fill=1.0, len_hi=40)
    two, one = (int(torch.nonzero(s.len > k)[x]) for k, x in ((16, 0), (0, -1)))
    s.table[two, 1], s.table[one, 0] = 999, -1          # a bad page copied, one given up
    new = torch.clamp(s.len + 1, max=64).to(torch.int32)
    inst_of = s.inst.clone()
    inst_of[two], new[one] = 1 - s.inst[two], 0
    parent = torch.arange(20, dtype=torch.int32)
    low, high, off, up = [b for b in range(20) if b not in (two, one)][:4]
    new[low], new[high], inst_of[off], parent[up] = -1, 65, 2, 20
    ref = _check_assign(s, new, parent, inst_of)
    assert ref[5] & 63 == paged.BAD_INST | paged.BAD_LEN | paged.BAD_PAGE | paged.BAD_PARENT


def test_assign_follows_a_plan_and_the_cache_stays_consistent():
    """Twenty steps of growth, forks, moves and ends: counts always equal what
    the rows hold."""
    s = State(5, 40, 12, 200, 4, fill=0.3, len_hi=60)
    for step in range(20):
        print("step", step, flush=True)
        rng = s.rng
        new = s.len.numpy() + 1 + rng.integers(0, 20, s.n)
        new[rng.random(s.n) < 0.15] = 0
        parent = np.where(rng.random(s.n) < 0.15, rng.integers(0, s.n, s.n), np.arange(s.n))
        inst_of = np.where(rng.random(s.n) < 0.1, rng.integers(0, 4, s.n), s.inst.numpy())
        i32 = lambda a: torch.from_numpy(np.asarray(a).astype(np.int32))
        ref = _check_assign(s, i32(np.minimum(new, 12 * 16)), i32(parent), i32(inst_of))
        s.table, s.len, s.inst, s.refs, s.kv = ref[:5]
        held = torch.arange(s.M)[None] < -(-s.len // s.ps)[:, None]
        assert torch.equal(torch.bincount(s.table[held].long(), minlength=800),
                           s.refs.long())
        where = s.table // s.P
        assert (where[held] == s.inst[:, None].expand_as(where)[held]).all()


@pytest.mark.parametrize("n,M,P,n_inst,ps,page_bytes", [
    (1, 1, 1, 1, 16, 16), (9, 4, 50, 1, 16, 48), (60, 6, 300, 4, 32, 4096),
    (500, 5, 3000, 2, 16, 160), (40, 90, 4097, 1, 256, 32768),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(n, M, P, n_inst, ps, page_bytes, in_place):
    s = State(n + P, n, M, P, n_inst, ps, 2, page_bytes, fill=0.7)
    print(f"compact n={n} M={M} P={P} inst={n_inst}", flush=True)
    p = s.params()
    table, length, refs, kv = (x.to(DEV) for x in (s.table, s.len, s.refs, s.kv))
    t2 = table if in_place else s.table.to(DEV)
    r2, n_live = torch.full_like(refs, -9), torch.full((n_inst,), -9, dtype=torch.int32, device=DEV)
    ws = star.Workspace(star.compact_pages_workspace_size(p))
    star.compact_pages(p, table, length, refs, kv, t2, r2, n_live, ws)
    torch.cuda.synchronize()
    ref = paged.compact(s.table, s.len, s.refs, s.kv, n_inst=n_inst, page_size=ps)
    for name, x, y in zip(("table", "refs", "n_live", "kv"), (t2, r2, n_live, kv), ref):
        assert torch.equal(x.cpu(), y), name
    assert ws.read_device_error() == ref[4] == 0


def test_compact_full_empty_and_bad_rows():
    for fill in (0.0, 1.0):
        s = State(11, 30, 4, 64, 2, fill=fill)
        if fill:
            s.refs[:] = 1
        p = s.params()
        args = [x.to(DEV) for x in (s.table, s.len, s.refs, s.kv, s.table, s.refs)]
        n_live = torch.zeros(2, dtype=torch.int32, device=DEV)
        ws = star.Workspace(star.compact_pages_workspace_size(p))
        star.compact_pages(p, *args[:4], args[4], args[5], n_live, ws)
        assert n_live.tolist() == ([64, 64] if fill else [0, 0])
        assert torch.equal(args[4].cpu(), s.table) and torch.equal(args[5].cpu(), s.refs)
        assert torch.equal(args[3].cpu(), s.kv)
    s = State(12, 30, 4, 64, 2, fill=0.5)
    s.len[4], s.len[5], s.len[6] = 65, -1, 30
    s.table[6, 1] = 128
    ref = paged.compact(s.table, s.len, s.refs, s.kv, n_inst=2, page_size=16)
    p = s.params()
    args = [x.to(DEV) for x in (s.table, s.len, s.refs, s.kv, s.table, s.refs)]
    n_live = torch.zeros(2, dtype=torch.int32, device=DEV)
    ws = star.Workspace(star.compact_pages_workspace_size(p))
    star.compact_pages(p, *args[:4], args[4], args[5], n_live, ws)
    for x, y in zip((args[4], args[5], n_live, args[3]), ref):
        assert torch.equal(x.cpu(), y)
    assert ws.read_device_error() == ref[4] == paged.BAD_LEN | paged.BAD_PAGE


def test_strided_pool_and_nothing_to_do():
    """Pages of all layers side by side ([pages, layers, bytes]) and gaps stay
    as they are; no slots, no copies."""
    s = State(13, 24, 4, 80, 2, layers=3, page_bytes=64, fill=0.5)
    wide = torch.from_numpy(s.rng.integers(-9, 9, (160, 3, 48)).astype(np.int16))  # 96-byte steps
    wide[:, :, :32] = s.kv.transpose(0, 1)
    inst_of = 1 - s.inst
    new = s.len.clone()
    ref = paged.assign(s.table, s.len, s.inst, s.refs, s.kv, new, None, inst_of, n_inst=2,
                       page_size=16)
    p = star.pages_params(24, 4, 160, 16, 3, 64, n_inst=2, page_stride=3 * 96, layer_stride=96)
    d = [x.to(DEV) for x in (s.table, s.len, s.inst, s.refs, wide)]
    ws = star.Workspace(star.assign_pages_workspace_size(p))
    star.assign_pages(p, None, new.to(DEV), inst_of.to(DEV), *d, *d[:4], ws)
    got = d[4].cpu()
    assert torch.equal(got[:, :, :32].transpose(0, 1), ref[4])
    assert torch.equal(got[:, :, 32:], wide[:, :, 32:])
    assert torch.equal(d[0].cpu(), ref[0]) and torch.equal(d[3].cpu(), ref[3])

    p = star.pages_params(0, 1, 10, 16, 1, 16)
    refs = torch.arange(10, dtype=torch.int32, device=DEV) % 2
    kv = torch.zeros((10, 8), dtype=torch.int16, device=DEV)
    empty, out = torch.zeros(0, dtype=torch.int32, device=DEV), torch.zeros_like(refs)
    ws = star.Workspace(star.assign_pages_workspace_size(p))
    star.assign_pages(p, None, empty, None, empty, empty, None, refs, kv, empty, empty, None, out,
                      ws)
    assert torch.equal(out, refs) and ws.read_device_error() == 0


def test_assign_replayed_from_a_graph():
    """A captured in-place growth step, replayed with eager work between."""
    s = State(14, 60, 10, 400, 2, fill=0.3, len_hi=50)
    p = s.params()
    table, length, inst, refs, kv = (x.to(DEV) for x in (s.table, s.len, s.inst, s.refs, s.kv))
    ws = star.Workspace(star.assign_pages_workspace_size(p))
    new = torch.empty_like(length)
    g = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=stream):
        torch.add(length, 7, out=new)
        star.assign_pages(p, None, new, None, table, length, inst, refs, kv, table, length, inst,
                          refs, ws)
    for _ in range(5):
        g.replay()
        torch.cuda.synchronize()
        ref = paged.assign(s.table, s.len, s.inst, s.refs, s.kv, s.len + 7, n_inst=2, page_size=16)
        s.table, s.len, s.inst, s.refs, s.kv = ref[:5]
        for x, y in zip((table, length, inst, refs, kv), ref):
            assert torch.equal(x.cpu(), y)
        torch.rand(1000, device=DEV).sum().item()
