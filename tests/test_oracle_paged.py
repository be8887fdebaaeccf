"""Pins of the paged cache's oracle: hand-worked page tables, and attention
against closed forms."""
import math

import torch

from oracle import paged

i32 = lambda *x: torch.tensor(x, dtype=torch.int32)


def _pool(n_pages, layers=2):
    return torch.arange(layers * n_pages * 8, dtype=torch.int16).reshape(layers, n_pages, 8)


def test_assign_worked_example():
    """Two instances of six pages of 16 tokens.  Slot 0 grows across a page
    border, slot 1 moves to instance 1 with its two pages, slot 2 becomes a
    fork of slot 0 (shares its full page, copies the partly filled one), slot 3
    ends."""
    table = torch.full((4, 4), -1, dtype=torch.int32)
    table[0, :2], table[1, :2], table[2, :1], table[3, :1] = i32(4, 0), i32(2, 3), i32(1), i32(8)
    refs = torch.zeros(12, dtype=torch.int32)
    refs[[0, 1, 2, 3, 4, 8]] = 1
    kv = _pool(12)
    t, L, I, R, kv2, flags = paged.assign(
        table, i32(24, 20, 5, 9), i32(0, 0, 0, 1), refs, kv, i32(33, 21, 25, 0),
        i32(0, 1, 0, 3), i32(0, 1, 0, 1), n_inst=2, page_size=16)
    # instance 0 has page 5 alone free: slot 0 takes it, slot 2 waits; slot 1
    # takes 6 and 7 of instance 1
    assert flags == paged.NO_PAGES
    assert L.tolist() == [33, 21, 5, 0] and I.tolist() == [0, 1, 0, 1]
    assert t[0, :3].tolist() == [4, 0, 5]
    assert t[1, :2].tolist() == [6, 7] and t[2, 0] == 1
    assert R.tolist() == [1, 1, 0, 0, 1, 1, 1, 1, 0, 0, 0, 0]
    assert torch.equal(kv2[:, 6], kv[:, 2]) and torch.equal(kv2[:, 7], kv[:, 3])
    # one step later the pages that slot 1 left serve the fork
    t, L, I, R, kv3, flags = paged.assign(
        t, L, I, R, kv2, i32(33, 21, 25, 0), i32(0, 1, 0, 3), n_inst=2, page_size=16)
    assert flags == 0 and L.tolist() == [33, 21, 25, 0]
    assert t[2, :2].tolist() == [4, 2] and R.tolist() == [1, 0, 1, 0, 2, 1, 1, 1, 0, 0, 0, 0]
    assert torch.equal(kv3[:, 2], kv2[:, 0])


def test_assign_never_leaves_the_next_token_on_a_shared_page():
    """Slots 0 and 1 share page 3; both cut it short and go on: each gets a
    copy, and the shared page is free afterwards."""
    refs = torch.zeros(8, dtype=torch.int32)
    refs[3] = 2
    t, L, I, R, kv, flags = paged.assign(
        torch.tensor([[3, -1], [3, -1]], dtype=torch.int32), i32(16, 16), i32(0, 0), refs,
        _pool(8), i32(10, 12), n_inst=1, page_size=16)
    assert flags == 0 and t[:, 0].tolist() == [0, 1]
    assert R.tolist() == [1, 1, 0, 0, 0, 0, 0, 0]


def test_compact_worked_example():
    table = torch.tensor([[5, 2], [7, 5]], dtype=torch.int32)
    refs = i32(0, 0, 1, 0, 0, 2, 0, 1)
    kv = _pool(8)
    t, R, n_live, kv2, flags = paged.compact(table, i32(20, 32), refs, kv, n_inst=1, page_size=16)
    assert flags == 0 and n_live.tolist() == [3]
    assert t.tolist() == [[0, 2], [1, 0]] and R.tolist() == [2, 1, 1, 0, 0, 0, 0, 0]
    assert torch.equal(kv2[:, 0], kv[:, 5]) and torch.equal(kv2[:, 1], kv[:, 7])


def _attend_case(L, T, window=0, sinks=0, zero_q=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    ps, D = 16, 8
    M = -(-L // ps)
    kv = torch.randn((M + 1, 2, 1, ps, D), generator=g)
    table = torch.randperm(M + 1, generator=g)[:M].to(torch.int32)[None]
    q = torch.zeros((T, 2, D)) if zero_q else torch.randn((T, 2, D), generator=g)
    k, v = torch.randn((T, 1, D), generator=g), torch.randn((T, 1, D), generator=g)
    r = paged.attend(q, k, v, kv, table, i32(L), i32(0, T), scale=0.5, window=window, sinks=sinks)
    rows = r["kv"][table[0].long(), 1, 0].reshape(-1, D)[:L].double()
    return r, rows, v


def test_equal_scores_give_the_mean_of_the_visible_values():
    r, v, _ = _attend_case(40, 3)
    for i, p in enumerate((37, 38, 39)):
        torch.testing.assert_close(r["out"][i, 1], v[: p + 1].mean(0))
        assert abs(r["lse"][i, 0].item() - math.log(p + 1)) < 1e-12
    r, v, _ = _attend_case(40, 3, window=5, sinks=2)
    for i, p in enumerate((37, 38, 39)):
        see = list(range(2)) + list(range(p - 4, p + 1))
        torch.testing.assert_close(r["out"][i, 0], v[see].mean(0))


def test_new_tokens_are_in_the_cache_and_the_whole_prompt_equals_its_last_rows():
    r, v, new = _attend_case(33, 33, zero_q=False)
    torch.testing.assert_close(v, new[:, 0].double())
    # a row alone, over the cache that the prompt left, gives the same
    g = torch.Generator().manual_seed(0)
    assert r["flags"] == 0 and torch.isfinite(r["out"]).all()
    torch.testing.assert_close(r["out"][0, 0], new[0, 0].double())    # the first sees itself


def test_empty_and_refused_slots():
    kv = torch.zeros((2, 2, 1, 16, 8))
    q, k = torch.ones((3, 1, 8)), torch.ones((3, 1, 8))
    table = torch.tensor([[0], [1], [1]], dtype=torch.int32)
    r = paged.attend(q, k, k, kv, table, i32(0, 17, 3), scale=1.0)
    assert r["out"][0].abs().max() == 0 and r["lse"][0, 0] == -math.inf
    assert r["written"].tolist() == [True, False, True] and r["flags"] == paged.BAD_LEN
    assert torch.isfinite(r["out"][2]).all()
    table[2, 0] = 9
    r = paged.attend(q, k, k, kv, table, i32(0, 16, 3), scale=1.0)
    assert r["flags"] == paged.BAD_PAGE and r["out"][2].abs().max() == 0
