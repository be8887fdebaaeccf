"""Visible values that are not finite leave the rows that see them infinite or NaN in
their columns, however far their scores lie below the row's maximum and wherever the
keys are cut (infinity times a weight that has run down to 0 is no number), and touch
no other row or column: against the oracle, whose weights are positive in 64 bits
(e^-300 and the like)."""
import math

import pytest
import torch

from oracle import paged
from paper_2510_13668_amd import star
from test_gpu_attend import WIDE, Cache, compare, run, tiled

pytestmark = pytest.mark.gpu
INF = math.inf


def _far(c, low, high):
    """Queries of ones and the key of token j (of every request) at j's level:
    scores about 300 (in e's powers) lower at `low` than at `high`, others between."""
    q, k, v = c.split(c.qkv)
    q[:] = 1.0
    c.scale = 1.0
    for b, L in enumerate(c.lens):
        first = L - c.new[b]
        row0 = int(c.start[b])
        for j in range(L):
            # (D keys of this size, times ones: the score; 16-bit types hold it)
            x = {low: -150.0, high: 150.0}.get(j, 0.0) / c.D
            if j >= first:
                k[row0 + j - first] = x
            else:
                c.kv[int(c.table[b, j // c.ps]), 0, :, j % c.ps] = x


def _value(c, b, j, head, d, x):
    first = c.lens[b] - c.new[b]
    if j >= first:
        c.split(c.qkv)[2][int(c.start[b]) + j - first, head, d] = x
    else:
        c.kv[int(c.table[b, j // c.ps]), 1, head, j % c.ps, d] = x


def _both(c, decode, what, low, high):
    _far(c, low, high)
    for b, L in enumerate(c.lens):
        if low < L:
            _value(c, b, low, 0, 3, INF)
            _value(c, b, low, c.Hkv - 1, c.D - 1, -INF)
        if high < L:
            _value(c, b, high, 0, 8, -INF)
            _value(c, b, high, 0, 9, INF)
            if low < L:
                _value(c, b, low, 0, 9, -INF)
    print(what, str(c.lens)[:60], low, high, c.D, flush=True)
    out, lse, _, err = run(c, decode)
    q, k, v = c.split(c.qkv)
    r = paged.attend(q, k, v, c.kv, c.table, c.len, None if decode else c.start, scale=c.scale)
    odd = ~torch.isfinite(r["out"])
    assert err == r["flags"] == 0 and odd.any() and not odd.all()
    assert torch.equal(~torch.isfinite(out), odd)
    out[odd], r["out"][odd], r["mass"][odd] = 0.0, 0.0, 0.0
    compare(out, lse, r, c, decode)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (256, "bf16"), (64, "f32"),
                                     (128, "f32"), (256, "f32")])
@pytest.mark.parametrize("low,high", [(3, 130), (130, 3), (20, 21), (200, 3)])
def test_decode_far_below_the_maximum(D, dtype, low, high):
    c = Cache(D + low, [131, 260, 5, 700], [1] * 4, 4, 2, D, dtype)
    _both(c, True, "far", low, high)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low,high", [(5, 8000), (8000, 5), (8999, 4), (4, 8999)])
def test_decode_far_below_the_maximum_in_another_part(dtype, low, high):
    c = Cache(low, [9000], [1], 8, 2, 64, dtype, ps=64)
    _both(c, True, "parts", low, high)


def test_decode_blocks_of_a_wave_each():
    """So many short requests that every block is one wave's."""
    lens = [30 - b % 3 for b in range(600)]
    c = Cache(1, lens, [1] * 600, 4, 2, 64)
    _both(c, True, "short", 2, 20)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("low,high", [(3, 60), (60, 3)])
def test_prompt_by_row_blocks(D, dtype, low, high):
    c = Cache(D + low, [100, 61], [50, 40], 4, 2, D, dtype)
    assert not tiled(c)
    _both(c, False, "rows", low, high)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (256, "bf16"), (64, "f32"),
                                     (128, "f32")])
@pytest.mark.parametrize("low,high", [(3, 300), (300, 3), (150, 151), (3, 5), (341, 3)])
def test_prompt_tiled(D, dtype, low, high):
    """At tiles that every row sees and at tiles that some do."""
    c = Cache(D + low, [350, 170], [60, 40], WIDE, WIDE, D, dtype, ps=32)
    assert tiled(c)
    _both(c, False, "tiles", low, high)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (64, "f32")])
@pytest.mark.parametrize("low,high", [(3, 3000), (3000, 3), (1500, 3199), (2000, 2001)])
def test_prompt_tiled_with_keys_cut(D, dtype, low, high):
    heads = 28 if dtype == "bf16" else 40
    c = Cache(D + low, [3200], [500], heads, heads, D, dtype, ps=64)
    assert tiled(c) and star.attend_prompt_workspace_size(c.params(0, 0)) > 1 << 20
    _both(c, False, "cut", low, high)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("decode", [True, False])
def test_rows_whose_visible_scores_are_all_minus_infinity(dtype, decode):
    """They are 0 but where a value is not finite."""
    for heads in (2, WIDE):
        c = Cache(2, [90, 70], [1, 1] if decode else [70, 40], heads, heads, 64, dtype)
        q, k, v = c.split(c.qkv)
        q[:] = 1.0
        last = int(c.start[1]) - 1                      # the first request's last token
        k[last, 0], v[last, 0, 7], v[last, 1, 7] = -INF, INF, INF
        out, lse, _, err = run(c, decode, 1, 0)
        assert err == 0 and lse[last, 0] == -INF
        assert not torch.isfinite(out[last, 0, 7]) and out[last, 1, 7] == INF
        out[last, :2, 7] = 0.0
        assert (out[last, 0] == 0).all() and torch.isfinite(out).all()
