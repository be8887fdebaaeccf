"""Attention over the paged cache against the oracle (64 bits).

Error bounds, from the arithmetic (u = 2^-24, reach = the largest
scale sum |q||k| of a row, mass = sum_j p_j |v_j|):
* a score's fp32 sum of D products and its scaling are off by at most
  (D + 4) u reach, the exponent's argument by 2 u more times the distance to
  the maximum (at most 2 reach); a probability is then off by twice that
  relative (its own and the sum's), and a few u of exp2 and the joins;
* the second product and the joins sum at most L + 64 terms in fp32:
  (L + 64) u mass;
* bf16: the probabilities as hi + lo pairs add 2^-16 mass, as one bf16 (long
  prompts) half a step, 2^-8 mass; the output's own rounding half a step,
  2^-8 (bf16) or u (fp32) of its value.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_13668_amd import star

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = {"bf16": (torch.bfloat16, star.BF16), "f32": (torch.float32, star.F32)}


class Cache:
    """One layer's pages with everything that no token holds at NaN, and rows
    of new tokens as columns of one wider array."""

    def __init__(self, seed, lens, new, Hq, Hkv, D, dtype="bf16", ps=16, spare=3, peak=1.0):
        g = torch.Generator().manual_seed(seed)
        dt, self.code = TYPES[dtype]
        self.lens, self.new, self.ps, self.D, self.Hq, self.Hkv = lens, new, ps, D, Hq, Hkv
        n = len(lens)
        used = [-(-x // ps) for x in lens]
        self.M = max(1, *used)
        self.n_pages = sum(used) + spare
        where = torch.randperm(self.n_pages, generator=g).tolist()
        self.table = torch.full((n, self.M), -7, dtype=torch.int32)
        self.kv = torch.full((self.n_pages, 2, Hkv, ps, D), math.nan, dtype=dt)
        for b in range(n):
            for j in range(used[b]):
                page = where.pop()
                self.table[b, j] = page
                k = min(lens[b] - new[b] - j * ps, ps)
                if k > 0:
                    self.kv[page, :, :, :k] = torch.randn((2, Hkv, k, D), generator=g).to(dt)
        rows = sum(new)
        qkv = torch.randn((rows, Hq + 2 * Hkv + 1, D), generator=g)
        qkv[:, :Hq] *= peak
        self.qkv = qkv.to(dt)
        self.len = torch.tensor(lens, dtype=torch.int32)
        self.start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        self.scale = D ** -0.5

    def split(self, qkv):
        return qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:-1]

    def params(self, window, sinks):
        return star.attend_params(len(self.lens), self.qkv.shape[0], self.Hq, self.Hkv, self.D,
                                  self.code, self.ps, self.n_pages, self.M, self.scale, window,
                                  sinks, q_stride=self.qkv.stride(0), kv_stride=self.qkv.stride(0))


def run(c, decode, window=0, sinks=0, lse=True, ws=None):
    p = c.params(window, sinks)
    qkv, kv = c.qkv.to(DEV), c.kv.to(DEV)
    q, k, v = c.split(qkv)
    out = torch.full((qkv.shape[0], c.Hq, c.D), 77.0, dtype=qkv.dtype, device=DEV)
    z = torch.full((qkv.shape[0], c.Hq), 77.0, device=DEV) if lse else None
    size = star.attend_decode_workspace_size if decode else star.attend_prompt_workspace_size
    ws = ws or star.Workspace(size(p))
    if decode:
        star.attend_decode(p, q, k, v, kv, c.table.to(DEV), c.len.to(DEV), out, z, ws)
    else:
        star.attend_prompt(p, q, k, v, kv, c.table.to(DEV), c.len.to(DEV), c.start.to(DEV), out, z,
                           ws)
    torch.cuda.synchronize()
    return out.cpu(), None if z is None else z.cpu(), kv.cpu(), ws.read_device_error()


def check(c, decode, window=0, sinks=0, flags=0, what=""):
    print(f"{'decode' if decode else 'prompt'} {what} lens={str(c.lens)[:60]} window={window} "
          f"sinks={sinks} heads={c.Hq}/{c.Hkv} D={c.D}", flush=True)
    out, lse, kv, err = run(c, decode, window, sinks)
    q, k, v = c.split(c.qkv)
    r = paged.attend(q, k, v, c.kv, c.table, c.len, None if decode else c.start, scale=c.scale,
                     window=window, sinks=sinks)
    assert err == r["flags"] == flags
    assert torch.equal(kv.view(torch.uint8), r["kv"].view(torch.uint8)), "cache"
    compare(out, lse, r, c, decode)
    return out, lse


def compare(out, lse, r, c, decode):
    left = ~r["written"]
    assert (out[left] == 77.0).all() and (lse[left] == 77.0).all()
    out, lse = out[r["written"]], lse[r["written"]]
    r = {x: r[x][r["written"]] for x in ("out", "lse", "mass", "reach")}
    L = max(1, max(c.lens))
    score = ((c.D + 8) + 8) * U * r["reach"] + 16 * U
    bf = c.code == star.BF16
    one = (2.0 ** -16 if decode else 2.0 ** -8) if bf else 0.0
    bound = ((2 * score + (L + 64) * U + one)[..., None] * r["mass"] +
             (2.0 ** -8 if bf else 2 * U) * r["out"].abs() + 1e-30)
    off = (out.double() - r["out"]).abs()
    fine = torch.isfinite(r["out"])
    assert torch.equal(torch.isnan(out), torch.isnan(r["out"]))
    inf = torch.isinf(r["out"])
    assert torch.equal(out[inf].double(), r["out"][inf])
    assert (off[fine] <= bound[fine]).all(), (off / bound)[fine].max()
    seen = torch.isfinite(r["lse"])
    assert torch.equal(torch.isnan(lse), torch.isnan(r["lse"]))
    z_bound = score + (L + 64) * U + 4 * U * r["lse"].abs()
    assert ((lse.double() - r["lse"]).abs()[seen] <= z_bound[seen]).all()
    empty = torch.isinf(r["lse"])
    assert torch.equal(lse[empty].double(), r["lse"][empty])


HEADS = [(1, 1, 64), (28, 4, 128), (8, 2, 64), (20, 1, 128), (6, 2, 256), (33, 1, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [16, 64])
def test_decode_lengths(Hq, Hkv, D, dtype, ps):
    lens = [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 0, 300, 777]
    new = [1] * len(lens)
    check(Cache(Hq + ps, lens, new, Hq, Hkv, D, dtype, ps), True)
    check(Cache(Hq + ps + 1, lens, new, Hq, Hkv, D, dtype, ps, peak=4.0), True, window=40, sinks=5)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 33), (64, 4), (500, 100),
                                          (2 ** 31 - 1, 0), (100, 2 ** 31 - 1), (0, 7)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_windows(window, sinks, dtype):
    lens = [1, 16, 40, 111, 300, 301, 620]
    check(Cache(window % 97, lens, [1] * 7, 12, 3, 64, dtype), True, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_long_and_short_together(dtype):
    """One cache that many workgroups share beside ones that share a workgroup."""
    lens = [9000] + [3] * 40 + [2500, 0, 1, 4100]
    c = Cache(1, lens, [1] * len(lens), 8, 2, 128, dtype, ps=32, peak=3.0)
    a = check(c, True)
    b = check(c, True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])   # no order of arrival in it
    check(c, True, window=1000, sinks=3)


def test_decode_pages_out_of_the_window_may_be_gone():
    c = Cache(2, [200, 150], [1, 1], 4, 2, 64)
    keep = run(c, True, window=40, sinks=20)
    c.table[0, 2:10], c.table[1, 2:6] = -1, 10 ** 6      # tokens 32..159 and 32..95
    out, lse, _, err = run(c, True, window=40, sinks=20)
    assert err == 0 and torch.equal(out, keep[0]) and torch.equal(lse, keep[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_bad_contents(dtype):
    lens = [50, 100, 30, 60, 20, 64]
    c = Cache(3, lens, [1] * 6, 4, 2, 64, dtype)
    c.len[1], c.len[2] = -1, c.M * 16 + 1               # left out
    c.table[3, 1] = c.n_pages                           # 16 tokens left out
    c.table[4, 1] = -1                                  # the new token's page
    c.table[5, :] = -2                                  # nothing left to see
    out, lse = check(c, True, flags=star.DEV_BAD_LEN | star.DEV_BAD_PAGE)
    assert (out[5] == 0).all() and torch.isinf(lse[5]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("decode", [True, False])
def test_infinities_and_nans_stay_with_the_rows_that_see_them(dtype, decode):
    """Keys and values that are not finite, at tokens that some rows see and
    others do not."""
    new = [1, 1, 1] if decode else [70, 5, 33]
    lens = [150, 40, 90] if decode else [150, 40, 33]
    c = Cache(4, lens, new, 4, 2, 64, dtype)
    c.scale = 0.05
    inf, nan = math.inf, math.nan
    at = lambda b, j: (int(c.table[b, j // 16]), j % 16)
    if decode:
        page, slot = at(0, 3)
        c.kv[page, 1, 0, slot, 5] = inf                 # visible: out becomes infinite
        page, slot = at(0, 80)
        c.kv[page, 1, 1, slot, :] = nan                 # behind the window
        c.kv[page, 0, 1, slot, :] = nan
        page, slot = at(2, 20)
        c.kv[page, 1, 0, slot, 7] = -inf                # behind the window
        check(c, True, window=30, sinks=4)
        check(c, True, window=30, sinks=0)
        return
    q, k, v = c.split(c.qkv)
    v[40, 0, 9], v[41, 1, 3], v[60, 0, 11] = inf, nan, -inf     # slot 0's new tokens
    k[55, 1, :] = nan
    v[75 + 20, 1, 2] = inf                                       # slot 2's
    check(c, False)
    check(c, False, window=25, sinks=2)


PROMPTS = [([1], [1]), ([2, 1, 3], [2, 1, 3]), ([17, 64, 5], [17, 30, 1]), ([100], [100]),
           ([333, 0, 16, 80], [200, 0, 16, 33]), ([700], [3]), ([513], [513])]


@pytest.mark.parametrize("lens,new", PROMPTS)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (28, 4, 128), (20, 1, 128), (4, 2, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt(lens, new, Hq, Hkv, D, dtype):
    c = Cache(len(lens), lens, new, Hq, Hkv, D, dtype, ps=16 if D < 256 else 32, peak=2.0)
    check(c, False)
    check(c, False, window=29, sinks=3)


# Enough key-value heads put small prompts on the tiled kernel, which takes
# calls of many workgroups (128 rows of one head each).
WIDE = 160


def tiled(c):
    """The call is the tiled kernel's: no workspace but the parts of cut blocks."""
    size = star.attend_prompt_workspace_size(c.params(0, 0)) - star.STAR_WS_HEADER_BYTES
    return size % (4096 * (c.D // 8 + 1)) == 0


@pytest.mark.parametrize("lens,new", [([1], [64]), ([17, 64, 5], [17, 30, 1]), ([100], [100]),
                                      ([200, 0, 16, 80], [130, 0, 16, 33]), ([260], [129])])
@pytest.mark.parametrize("g,D,dtype", [(1, 64, "bf16"), (2, 128, "bf16"), (1, 256, "bf16"),
                                       (2, 64, "f32"), (1, 128, "f32")])
def test_prompt_tiled(lens, new, g, D, dtype):
    lens = [max(a, b) for a, b in zip(lens, new)]
    c = Cache(sum(lens), lens, new, WIDE * g, WIDE, D, dtype, ps=16 if D < 256 else 32, peak=2.0)
    assert tiled(c)
    check(c, False)
    check(c, False, window=29, sinks=3)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (64, 0), (70, 70), (64, 1),
                                          (2 ** 31 - 1, 3), (50, 2 ** 31 - 1), (100, 33)])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (64, "f32"), (128, "f32")])
def test_prompt_tiled_windows(window, sinks, D, dtype):
    c = Cache(7, [190, 160], [100, 31], WIDE, WIDE, D, dtype)
    c.scale = -0.2                                     # and the least products first
    assert tiled(c)
    check(c, False, window, sinks)


@pytest.mark.parametrize("ps", [128, 256])
@pytest.mark.parametrize("scale", [0.0, -0.3, 0.3])
def test_large_pages_and_scales(ps, scale):
    lens = [1, 127, 128, 129, 400, 513]
    for c, decode in ((Cache(18, lens, [1] * 6, 6, 2, 64, ps=ps), True),
                      (Cache(19, lens, [1, 100, 1, 129, 30, 64], 4, 2, 128, ps=ps), False),
                      (Cache(20, lens, [1, 20, 1, 9, 30, 64], WIDE, WIDE, 64, ps=ps), False)):
        c.scale = scale
        check(c, decode)
        check(c, decode, window=70, sinks=3)


def test_tiled_pages_out_of_the_window_may_be_gone():
    c = Cache(21, [300, 150], [60, 40], WIDE, WIDE, 64)
    assert tiled(c)
    keep = run(c, False, window=40, sinks=20)
    c.table[0, 2:12], c.table[1, 2:4] = -1, 10 ** 6      # tokens 32..191 and 32..63
    out, lse, _, err = run(c, False, window=40, sinks=20)
    assert err == 0 and torch.equal(out, keep[0]) and torch.equal(lse, keep[1])


def test_very_many_requests():
    """More requests than threads, waves and lanes hold one each, short ones
    and some long ones: values that are the same for all of a request's tokens
    come back whatever the weights."""
    n, rng = 20000, np.random.default_rng(22)
    lens = rng.integers(0, 3, n)
    lens[rng.integers(0, n, 40)] = rng.integers(100, 400, 40)
    used = -(-lens // 16)
    M, pages = int(used.max()), int(used.sum())
    j = np.arange(M)[None]
    table = np.where(j < used[:, None], (np.cumsum(used) - used)[:, None] + j, -1)
    value = torch.randint(-99, 100, (n,)).float()
    owner = torch.from_numpy(np.repeat(np.arange(n), used))
    kv = torch.randn((pages, 2, 1, 16, 64))
    kv[:, 1] = value[owner][:, None, None, None]
    for dtype in ("bf16", "f32"):
        dt, code = TYPES[dtype]
        p = star.attend_params(n, n, 2, 1, 64, code, 16, pages, M, 0.1)
        dev = lambda t: t.to(DEV)
        v_new = value[:, None, None].expand(n, 1, 64).to(dt).contiguous()
        out = torch.full((n, 2, 64), 77.0, dtype=dt, device=DEV)
        ws = star.Workspace(star.attend_decode_workspace_size(p))
        print("many", dtype, flush=True)
        star.attend_decode(p, dev(torch.randn((n, 2, 64)).to(dt)),
                           dev(torch.randn((n, 1, 64)).to(dt)), dev(v_new), dev(kv.to(dt)),
                           dev(torch.from_numpy(table.astype(np.int32))),
                           dev(torch.from_numpy(lens.astype(np.int32))), out, None, ws)
        want = torch.where(torch.from_numpy(lens) > 0, value, torch.zeros(()))
        # sums of up to 400 probabilities over their own sum (bf16 pairs: 2^-16)
        tol = 99 * (2.0 ** -8 + 2.0 ** -16 if dtype == "bf16" else 500 * U)
        assert (out.cpu().double() - want[:, None, None]).abs().max() <= tol
        assert ws.read_device_error() == 0


def test_two_streams_with_workspaces_of_their_own():
    a = Cache(23, [2000, 40], [1, 1], 8, 2, 64)
    b = Cache(24, [300, 200], [250, 90], 8, 2, 64)
    want = run(a, True)[0], run(b, False)[0]
    pa, pb = a.params(0, 0), b.params(0, 0)
    wa = star.Workspace(star.attend_decode_workspace_size(pa))
    wb = star.Workspace(star.attend_prompt_workspace_size(pb))
    xa, xb, ka, kb = (t.to(DEV) for t in (a.qkv, b.qkv, a.kv, b.kv))
    ta, la, tb, lb, sb = (t.to(DEV) for t in (a.table, a.len, b.table, b.len, b.start))
    oa, ob = torch.empty_like(want[0], device=DEV), torch.empty_like(want[1], device=DEV)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        star.attend_decode(pa, *a.split(xa), ka, ta, la, oa, None, wa, s1)
        star.attend_prompt(pb, *b.split(xb), kb, tb, lb, sb, ob, None, wb, s2)
    torch.cuda.synchronize()
    assert torch.equal(oa.cpu(), want[0]) and torch.equal(ob.cpu(), want[1])


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (64, "f32"), (128, "f32")])
def test_prompt_tiled_infinities_and_bad_contents(D, dtype):
    c = Cache(4, [150, 40, 90], [70, 5, 33], WIDE, WIDE, D, dtype)
    c.scale = 0.05
    assert tiled(c)
    q, k, v = c.split(c.qkv)
    inf, nan = math.inf, math.nan
    v[40, 0, 9], v[41, 1, 3], v[60, 0, 11], v[69, 5, 63] = inf, nan, -inf, inf
    k[55, 1, :] = nan
    v[75 + 20, 1, 2] = inf
    page = int(c.table[0, 1])
    c.kv[page, 1, 2, 3, 30], c.kv[page, 0, 3, 3, 30] = nan, nan         # token 19
    check(c, False)
    check(c, False, window=25, sinks=2)
    check(c, False, window=25, sinks=20)
    c.len[1] = 4                                       # more new tokens than tokens
    c.table[2, 1], c.table[0, 6] = -1, 10 ** 6         # cached tokens and new ones
    check(c, False, flags=star.DEV_BAD_LEN | star.DEV_BAD_PAGE)
    check(c, False, window=25, sinks=2, flags=star.DEV_BAD_LEN | star.DEV_BAD_PAGE)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_tiled_many_requests(dtype):
    new = [1 + 37 * b % 40 for b in range(70)]
    c = Cache(5, [n + b % 3 * 20 for b, n in enumerate(new)], new, 32, 16, 64, dtype)
    assert tiled(c)
    check(c, False)


@pytest.mark.parametrize("Hq,Hkv,D,T,past,window,sinks,dtype", [
    (16, 16, 64, 900, 2000, 0, 0, "bf16"), (32, 16, 128, 450, 1700, 0, 0, "bf16"),
    (32, 16, 128, 450, 1900, 1700, 9, "bf16"), (28, 28, 256, 490, 700, 0, 0, "bf16"),
    (24, 24, 64, 900, 2000, 1990, 3, "f32"), (48, 24, 128, 450, 1700, 0, 0, "f32"),
    (8, 8, 64, 900, 4000, 0, 0, "bf16"), (96, 96, 64, 340, 5100, 0, 0, "bf16")])
def test_prompt_tiled_cut_keys(Hq, Hkv, D, T, past, window, sinks, dtype):
    """Few blocks over long caches: several workgroups share a block's keys."""
    c = Cache(6, [past + T], [T], Hq, Hkv, D, dtype, ps=64, peak=3.0)
    assert tiled(c) and star.attend_prompt_workspace_size(c.params(0, 0)) > 1 << 20
    a = check(c, False, window, sinks)
    b = run(c, False, window, sinks)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])   # no order of arrival in it


@pytest.mark.parametrize("Hq,Hkv,D,window,sinks,dtype", [
    (32, 32, 64, 0, 0, "bf16"), (40, 20, 128, 0, 0, "bf16"), (32, 32, 64, 3000, 70, "bf16"),
    (24, 24, 64, 0, 0, "f32"), (28, 28, 128, 0, 0, "f32"), (16, 16, 256, 0, 0, "bf16")])
def test_prompt_tiled_longer_blocks_are_cut(Hq, Hkv, D, window, sinks, dtype):
    """One launch of requests after long, middling and no prefixes: as many workgroups
    as a block's keys ask for."""
    new = [300, 200, 0, 100, 150]
    past = [4000, 100, 6000, 2500, 0]
    c = Cache(11, [n + m for n, m in zip(new, past)], new, Hq, Hkv, D, dtype, ps=64, peak=3.0)
    assert tiled(c) and star.attend_prompt_workspace_size(c.params(0, 0)) > 1 << 20
    a = check(c, False, window, sinks)
    b = run(c, False, window, sinks)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (64, 0), (100, 70), (128, 1),
                                          (2 ** 31 - 1, 3), (500, 2 ** 31 - 1)])
def test_prompt_windows(window, sinks):
    check(Cache(7, [400, 260], [300, 131], 8, 2, 64, "bf16"), False, window, sinks)
    check(Cache(8, [260], [131], 4, 2, 128, "f32"), False, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_bad_contents(dtype):
    c = Cache(9, [90, 50, 70, 64], [40, 50, 20, 10], 4, 2, 64, dtype)
    c.len[1] = 49                                       # more new tokens than tokens
    c.table[2, 0], c.table[2, 4] = -1, 10 ** 6          # cached tokens and new ones
    check(c, False, flags=star.DEV_BAD_LEN | star.DEV_BAD_PAGE)
    c = Cache(10, [90, 50, 70], [40, 50, 20], 4, 2, 64, dtype)
    c.start[2] = 30                                     # not ascending: slot 1 is left out
    check(c, False, flags=star.DEV_BAD_LEN)
    c.start[1:] = torch.tensor([40, 90, 111])           # past the last row: slot 2 too
    check(c, False, flags=star.DEV_BAD_LEN)


def test_rows_behind_the_last_request_stay():
    c = Cache(11, [40, 30], [12, 6], 4, 2, 64)
    c.qkv = torch.cat([c.qkv, c.qkv[:9]])               # a padded batch of rows
    out, _ = check(c, False)
    assert (out[18:] == 77.0).all()


def test_prompt_equals_its_tokens_one_by_one():
    """Decode calls over the cache that earlier ones left give the prompt's rows."""
    c = Cache(12, [45], [45], 8, 2, 64, "f32")
    whole, _, kv, _ = run(c, False)
    q, k, v = c.split(c.qkv.to(DEV))
    p = star.attend_params(1, 1, 8, 2, 64, star.F32, 16, c.n_pages, c.M, c.scale)
    ws, cache = star.Workspace(star.attend_decode_workspace_size(p)), c.kv.to(DEV)
    table = c.table.to(DEV)
    for t in range(45):
        out = torch.empty((1, 8, 64), device=DEV)
        n = torch.tensor([t + 1], dtype=torch.int32, device=DEV)
        star.attend_decode(p, q[t:t + 1].contiguous(), k[t:t + 1].contiguous(),
                           v[t:t + 1].contiguous(), cache, table, n, out, None, ws)
        torch.testing.assert_close(out[0].cpu(), whole[t], rtol=1e-5, atol=1e-6)
    held = ~torch.isnan(kv)
    assert torch.equal(torch.isnan(cache.cpu()), ~held)
    assert torch.equal(cache.cpu()[held], kv[held])


def test_strided_pages_far_offsets_and_side_streams():
    """One layer of a pool whose pages hold all layers (its own stride), pages
    whose offsets pass 32 bits, on a stream of its own."""
    c = Cache(13, [100, 37], [1, 1], 8, 2, 128)
    step = 2 * 2 * 16 * 128
    far = 2 ** 32 // (2 * 3 * step) + 5                 # pages before ours: over 4 GiB
    pool = torch.zeros((far + c.n_pages, 3, 2, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    pool[far:, 1] = c.kv.to(DEV)
    c2 = Cache(13, [100, 37], [1, 1], 8, 2, 128)
    p = star.attend_params(2, 2, 8, 2, 128, star.BF16, 16, far + c.n_pages, c.M, c.scale,
                           q_stride=c.qkv.stride(0), kv_stride=c.qkv.stride(0),
                           page_stride=3 * step * 2)
    q, k, v = c.split(c.qkv.to(DEV))
    table = torch.where(c.table >= 0, c.table + far, c.table).to(DEV)
    out, lens = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV), c.len.to(DEV)
    ws = star.Workspace(star.attend_decode_workspace_size(p))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    star.attend_decode(p, q, k, v, pool[:, 1], table, lens, out, None, ws, stream)
    torch.cuda.current_stream().wait_stream(stream)
    want = run(c2, True)
    assert torch.equal(out.cpu(), want[0])
    assert torch.equal(pool[far:, 1].cpu().view(torch.int16), want[2].view(torch.int16))
    assert not pool[:, 0].any() and not pool[:far].any()


def test_decode_and_prompt_replayed_from_a_graph():
    c = Cache(14, [500, 77, 0, 3000], [1, 1, 1, 1], 8, 2, 64)
    d = Cache(15, [200, 90], [150, 90], 8, 2, 64)
    ws = star.Workspace(1 << 25)
    p, pd = c.params(0, 0), d.params(64, 4)
    x, y = c.qkv.to(DEV), d.qkv.to(DEV)
    kv, kvd = c.kv.to(DEV), d.kv.to(DEV)
    args = [t.to(DEV) for t in (c.table, c.len, d.table, d.len, d.start)]
    out = torch.empty((4, 8, 64), dtype=torch.bfloat16, device=DEV)
    outd = torch.empty((d.qkv.shape[0], 8, 64), dtype=torch.bfloat16, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        star.attend_decode(p, *c.split(x), kv, args[0], args[1], out, None, ws)
        star.attend_prompt(pd, *d.split(y), kvd, args[2], args[3], args[4], outd, None, ws)
    for _ in range(4):
        x.normal_()
        y.normal_()
        g.replay()
        torch.cuda.synchronize()
        c.qkv, d.qkv = x.cpu(), y.cpu()
        assert torch.equal(out.cpu(), run(c, True)[0])
        assert torch.equal(outd.cpu(), run(d, False, 64, 4)[0])


def test_one_workspace_serves_both_and_errors_are_kept_until_read():
    ws = star.Workspace(1 << 25)
    c = Cache(16, [3000, 5], [1, 1], 4, 1, 64)
    d = Cache(17, [300], [300], 4, 1, 64)
    want = run(c, True)[0], run(d, False)[0]
    for _ in range(3):
        assert torch.equal(run(c, True, ws=ws)[0], want[0])
        assert torch.equal(run(d, False, ws=ws)[0], want[1])
