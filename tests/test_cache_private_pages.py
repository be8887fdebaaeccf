"""The page that attention stores to next is never a shared one, also after cuts
and forks: hand-worked tables (CPU), the kernel against the oracle over random
cuts beside forks, and attention from the other holder of the pages."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_13668_amd import star
from test_gpu_cache_flow import Instance, N
from test_gpu_pages import State, _check_assign

i32 = lambda *x: torch.tensor(x, dtype=torch.int32)


def _assign(lens, rows, new, parent=None, n_pages=12):
    """The oracle's call for slots on one instance, pages of 16; kv[0, x] = x."""
    table = torch.full((len(rows), 5), -1, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    for b, row in enumerate(rows):
        table[b, : len(row)] = i32(*row)
        refs[row] += 1
    kv = torch.arange(n_pages, dtype=torch.int16).reshape(1, n_pages, 1)
    t, L, _, R, kv2, flags = paged.assign(
        table, i32(*lens), i32(*[0] * len(rows)), refs, kv, i32(*new),
        None if parent is None else i32(*parent), n_inst=1, page_size=16)
    held = [t[b, : -(-int(L[b]) // 16)].tolist() for b in range(len(rows))]
    count = np.bincount(sum(held, []), minlength=n_pages)
    assert flags == 0 and L.tolist() == list(new) and R.tolist() == count.tolist()
    return held, kv2[0, :, 0].tolist()


def test_a_cut_beside_a_fork_of_the_whole_leaves_the_page_to_the_fork():
    held, kv = _assign([32, 0], [[0, 1], []], [20, 33], [0, 0])
    assert held == [[0, 2], [0, 1, 3]] and kv[2] == 1
    # a fork that stops before the page does not take it
    held, _ = _assign([32, 0], [[0, 1], []], [20, 17], [0, 0])
    assert held == [[0, 1], [0, 2]]


@pytest.mark.parametrize("cut,shared", [(1, 0), (15, 0), (16, 0), (17, 1), (31, 1), (32, 1)])
def test_a_cut_to_shared_pages_copies_the_one_of_its_last_token(cut, shared):
    held, kv = _assign([33, 33], [[0, 1, 2], [0, 1, 3]], [cut, 33])
    assert held == [[0, 1][:shared] + [4], [0, 1, 3]] and kv[4] == shared
    # pages of its own stay
    held, _ = _assign([33, 33], [[0, 1, 2], [5, 6, 3]], [cut, 33])
    assert held[0] == [0, 1][: shared + 1]


def test_a_fork_that_does_not_grow_copies_the_page_of_its_last_token():
    for new, want in ((32, [0, 3]), (16, [3]), (33, [0, 1, 3]), (48, [0, 1, 3]), (49, [0, 1, 2, 3])):
        held, kv = _assign([48, 0], [[0, 1, 2], []], [49, new], [0, 0])
        # (slot 0 grows first, into page 3)
        assert held[0] == [0, 1, 2, 3] and held[1] == [x + (x == 3) for x in want], new
        assert new == 49 or kv[4] == (new - 1) // 16


def test_slots_that_keep_their_length_or_end_keep_and_free_pages():
    held, _ = _assign([32, 33], [[0, 1], [0, 1, 2]], [32, 33])
    assert held == [[0, 1], [0, 1, 2]]
    held, _ = _assign([32, 33], [[0, 1], [0, 1, 2]], [0, 34], [-1, 1])
    assert held == [[], [0, 1, 2]]


@pytest.mark.gpu
@pytest.mark.parametrize("n,M,P,n_inst,ps,move", [
    (2, 3, 12, 1, 16, 0.0), (40, 6, 300, 1, 16, 0.0), (300, 9, 2000, 3, 16, 0.1),
    (1500, 4, 9000, 1, 64, 0.0), (5000, 3, 9000, 2, 32, 0.1)])
def test_cuts_beside_forks(n, M, P, n_inst, ps, move):
    s = State(n + M, n, M, P, n_inst, ps, fill=0.45)
    rng = s.rng
    print(f"cuts n={n} M={M} P={P} inst={n_inst} ps={ps}", flush=True)
    for step in range(3):
        lens = s.len.numpy().astype(np.int64)
        pick = rng.random(n)
        parent = np.where(pick < 0.35, rng.integers(0, n, n), np.arange(n))
        base = lens[parent]
        new = np.where(pick < 0.2, base, base + 1)               # forks whole, and growing
        cut = pick > 0.6
        new[cut] = (base[cut] * rng.random(int(cut.sum()))).astype(np.int64)
        border = pick > 0.8                                      # whole pages
        new[border] = new[border] // ps * ps
        to = np.where(rng.random(n) < move, rng.integers(0, n_inst, n), s.inst.numpy())
        dev = lambda a: torch.from_numpy(a.astype(np.int32))
        new = dev(np.minimum(new, M * ps))
        ref = _check_assign(s, new, dev(parent), dev(to))
        assert ref[5] == 0 or step
        changed = (parent != np.arange(n)) | (new.numpy() != lens)
        for b in np.flatnonzero(changed & (new.numpy() > 0) & (ref[5] == 0)):
            assert ref[3][ref[0][b, (int(new[b]) - 1) // ps]] == 1, b
        s.table, s.len, s.inst, s.refs, s.kv = ref[:5]
        if step == 0 and n > 2:                                  # and without forks
            cuts = dev(np.where(rng.random(n) < 0.5, s.len.numpy() // ps * ps, s.len.numpy()))
            _check_assign(s, cuts)
            _check_assign(s, cuts, in_place=True)


@pytest.mark.gpu
def test_cuts_and_forks_when_pages_run_out():
    """What has no page for its copy stays as it was."""
    n, M, P, ps = 60, 6, 110, 16
    s = State(9, n, M, P, 1, ps, fill=1.0)
    lens = s.len.numpy().astype(np.int64)
    parent = np.where(s.rng.random(n) < 0.4, s.rng.integers(0, n, n), np.arange(n))
    new = np.where(s.rng.random(n) < 0.5, lens[parent] // ps * ps, lens[parent])
    new[::3] = lens[::3] // 2 // ps * ps
    parent[::3] = np.arange(n)[::3]
    dev = lambda a: torch.from_numpy(a.astype(np.int32))
    ref = _check_assign(s, dev(new), dev(parent))
    assert ref[5] == paged.NO_PAGES and (ref[1] == dev(new)).any()
    _check_assign(s, dev(np.where(s.rng.random(n) < 0.5, lens // ps * ps, lens)))


@pytest.mark.gpu
def test_cuts_beside_forks_replayed_from_a_graph():
    """Whatever an earlier call left in the workspace."""
    n, M, P, ps = 200, 5, 900, 16
    s = State(10, n, M, P, 2, ps, fill=0.4)
    p = s.params()
    ws = star.Workspace(star.assign_pages_workspace_size(p))
    d = [x.to("cuda") for x in (s.table, s.len, s.inst, s.refs, s.kv)]
    out = [d[0].clone(), *(torch.zeros_like(x) for x in d[1:4])]
    parent, new = torch.zeros_like(d[1]), torch.zeros_like(d[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        star.assign_pages(p, parent, new, None, *d, *out, ws)
    for seed in range(4):
        rng = np.random.default_rng(seed)
        a = np.where(rng.random(n) < 0.4, rng.integers(0, n, n), np.arange(n))
        lens = s.len.numpy()
        want = np.where(rng.random(n) < 0.4, lens[a] * rng.random(n), lens[a] + rng.integers(0, 2, n))
        a, want = (torch.from_numpy(x.astype(np.int32)) for x in (a, np.minimum(want, M * ps)))
        parent.copy_(a)
        new.copy_(want)
        for x, y in zip((*out[:1], d[4]), (s.table, s.kv)):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        ref = paged.assign(s.table, s.len, s.inst, s.refs, s.kv, want, a, n_inst=2, page_size=ps)
        for x, y in zip((*out, d[4]), ref):
            assert torch.equal(x.cpu(), y)
        assert ws.read_device_error() == ref[5] == 0
        torch.rand(1000, device="cuda").sum().item()


def _grow(s, slots):
    lens = s.len.tolist()
    return [x + (b in slots) for b, x in enumerate(lens)]


def _step(s, new):
    """Every slot's last token is (or is written) anew."""
    s.rows = [[tuple(t[: max(0, new[b] - 1)] for t in layer[b]) for b in range(N)]
              for layer in s.rows]
    s.step([min(x, 1) for x in new])


@pytest.mark.gpu
@pytest.mark.parametrize("cut", [1, 15, 16, 17, 31, 32])
def test_attention_after_a_cut_of_shared_rows(cut):
    s = Instance("f32", 0, 0, seed=cut)
    lens = [32] + [0] * (N - 1)
    s.assign(lens)
    s.step(lens)
    keep = list(range(N))
    new = [33, 0, 33] + [0] * (N - 3)                            # slot 2 (the same instance)
    s.assign(new, keep[:2] + [0] + keep[3:])
    _step(s, new)
    new[0], new[2] = cut, 34
    s.assign(new)
    _step(s, new)
    for _ in range(2):
        new = _grow(s, (0, 2))
        s.assign(new)
        _step(s, new)


@pytest.mark.gpu
@pytest.mark.parametrize("cut", [1, 16, 20, 32, 33, 47])
def test_attention_after_a_cut_beside_a_fork(cut):
    s = Instance("bf16", 0, 0, seed=cut)
    lens = [48] + [0] * (N - 1)
    s.assign(lens)
    s.step(lens)
    keep = list(range(N))
    # slots 2 and 4 take all of slot 0's tokens, 6 what it keeps; it writes its
    # last token anew
    new = [cut, 0, 49, 0, 48, 0, cut] + [0] * (N - 7)
    s.assign(new, [0, 1, 0, 3, 0, 5, 0] + keep[7:])
    for _ in range(3):
        _step(s, new)
        new = _grow(s, (0, 2, 4, 6))
        s.assign(new)
