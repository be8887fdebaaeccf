"""Which kernel takes a prompt call, what precision it has there, and the paths of
cut keys that lengths, windows and many requests open."""
import pytest
import torch

from oracle import paged
from paper_2510_13668_amd import star
from test_gpu_attend import WIDE, Cache, check, compare, run, tiled

pytestmark = pytest.mark.gpu


def in_pairs(c, window=0, sinks=0):
    """A prompt call on the row-block kernel: bf16 probabilities as hi + lo pairs add
    2^-16 of the mass, where one bf16 would add 2^-8."""
    assert not tiled(c)
    out, lse, _, err = run(c, False, window, sinks)
    q, k, v = c.split(c.qkv)
    r = paged.attend(q, k, v, c.kv, c.table, c.len, c.start, scale=c.scale, window=window,
                     sinks=sinks)
    assert err == r["flags"] == 0
    compare(out, lse, r, c, True)                       # (the bounds of pairs)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (28, 4, 128), (4, 2, 256)])
def test_prompts_by_row_blocks_have_pairs(Hq, Hkv, D):
    in_pairs(Cache(Hq, [300, 61, 5], [150, 40, 2], Hq, Hkv, D))


def rows_many(c, window=0, sinks=0):
    """The header's rule for calls with many rows."""
    n_blocks = (c.qkv.shape[0] * (c.Hq // c.Hkv) + 64 * len(c.lens)) // 128 * c.Hkv
    keys = c.M * c.ps
    return n_blocks >= 112 or (n_blocks >= 56 and min(keys, window + sinks if window else keys)
                               >= 4096)


@pytest.mark.parametrize("lens,new,Hq,Hkv,wide", [
    ([90] * 28, [1] * 28, 8, 8, 0),                     # 8 (14.2) blocks: 112
    ([90] * 27, [1] * 27, 8, 8, 0),                     # 8 (13.7): 104
    ([200], [193], 224, 56, 0), ([300], [208], 32, 8, 4096), ([300], [207], 32, 8, 4096),
    ([300], [208], 32, 8, 4080), ([40, 0, 31], [3, 0, 9], 4, 4, 8192)])
def test_rows_decide_the_kernel_and_its_precision(lens, new, Hq, Hkv, wide):
    """At the borders of the rule, also where the table is wider than its requests."""
    c = Cache(len(lens), lens, new, Hq, Hkv, 64)
    if wide:
        c.table = torch.cat([c.table, torch.full((len(lens), wide // 16 - c.M), -3,
                                                 dtype=torch.int32)], dim=1)
        c.M = wide // 16
    assert tiled(c) == rows_many(c)
    if tiled(c):
        check(c, False)
    else:
        in_pairs(c)


def test_a_window_narrows_the_keys_that_rows_can_see():
    for window, sinks, many in ((4000, 96, True), (4000, 95, False), (5000, 0, True)):
        c = Cache(3, [4500], [700], 16, 16, 64, ps=64)
        assert rows_many(c, window, sinks) == many
        size = star.attend_prompt_workspace_size(c.params(window, sinks))
        # (the row-block kernel's parts: two of 16 rows for each of 512 workgroups)
        rows = star.STAR_WS_HEADER_BYTES + 2 * 512 * (16 * 64 + 4 * 16) * 4
        assert (size != rows) == many
        check(c, False, window, sinks)


def cut(c, window=0, sinks=0):
    """The call holds room for parts of cut blocks."""
    assert tiled(c)
    assert star.attend_prompt_workspace_size(c.params(window, sinks)) > 1 << 20
    a = check(c, False, window, sinks)
    b = run(c, False, window, sinks)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])   # no order of arrival in it


@pytest.mark.parametrize("Hq,Hkv,D,T,past,window,sinks,dtype", [
    (32, 16, 128, 450, 2600, 2100, 9, "bf16"), (16, 16, 64, 900, 2900, 2300, 0, "bf16"),
    (28, 28, 256, 490, 1500, 1100, 5, "bf16"), (24, 24, 64, 900, 2800, 2500, 3, "f32"),
    (48, 24, 128, 450, 2000, 1600, 70, "f32")])
def test_keys_cut_under_a_window(Hq, Hkv, D, T, past, window, sinks, dtype):
    cut(Cache(6, [past + T], [T], Hq, Hkv, D, dtype, ps=64, peak=3.0), window, sinks)


@pytest.mark.parametrize("Hkv,D,dtype", [(2, 64, "bf16"), (3, 64, "f32"), (2, 128, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2200, 7)])
def test_keys_cut_of_more_than_64_requests(Hkv, D, dtype, window, sinks):
    new = [70 + b % 5 for b in range(70)]
    past = [3000 * (b * 7 % 23) // 22 for b in range(70)]
    lens = [n + m for n, m in zip(new, past)]
    cut(Cache(8, lens, new, Hkv, Hkv, D, dtype, ps=64, peak=3.0), window, sinks)


def test_single_tokens_beside_a_chunk():
    new = [1] * 40 + [300] + [1] * 40
    lens = [1 + 29 * b % 200 for b in range(40)] + [900] + [1 + 31 * b % 150 for b in range(40)]
    for dtype in ("bf16", "f32"):
        check(Cache(9, lens, new, 28, 4, 128, dtype), False)


def test_a_table_wider_than_its_requests():
    """Columns that no request reaches may hold anything."""
    for Hq, Hkv in ((8, 2), (WIDE, WIDE)):
        c = Cache(10, [200, 77, 0, 31], [130, 77, 0, 1], Hq, Hkv, 64)
        c.table = torch.cat([c.table, torch.full((4, 300), -3, dtype=torch.int32)], dim=1)
        c.M = c.table.shape[1]
        check(c, False)
        check(c, False, window=40, sinks=4)
        d = Cache(10, [200, 77, 0, 31], [1] * 4, Hq, Hkv, 64)
        d.table = torch.cat([d.table, torch.full((4, 300), 10 ** 6, dtype=torch.int32)], dim=1)
        d.M = d.table.shape[1]
        check(d, True)


def test_an_error_is_kept_until_it_is_read():
    """Calls of either kind between do not lose it, the read clears it."""
    ws = star.Workspace(1 << 25)

    def call(c, decode):
        p, (q, k, v) = c.params(0, 0), c.split(c.qkv.to("cuda"))
        out = torch.empty((c.qkv.shape[0], c.Hq, c.D), dtype=c.qkv.dtype, device="cuda")
        args = [t.to("cuda") for t in (c.kv, c.table, c.len)]
        if decode:
            star.attend_decode(p, q, k, v, *args, out, None, ws)
        else:
            star.attend_prompt(p, q, k, v, *args, c.start.to("cuda"), out, None, ws)

    good = Cache(16, [3000, 5], [1, 1], 4, 1, 64), Cache(17, [300], [300], 4, 1, 64)
    short, page = Cache(16, [40, 5], [1, 1], 4, 1, 64), Cache(17, [60], [50], 4, 1, 64)
    short.len[1], page.table[0, 1] = -1, -1
    for bad, decode, flag in ((short, True, star.DEV_BAD_LEN), (page, False, star.DEV_BAD_PAGE)):
        call(bad, decode)
        call(good[0], True)
        call(good[1], False)
        assert ws.read_device_error() == flag
        call(good[0], True)
        assert ws.read_device_error() == 0
