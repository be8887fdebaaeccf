"""Host-side contract of the cache's entry points: every call below is refused
by the checks that run before anything is launched (no GPU)."""
import ctypes
import os

import pytest
import torch

from paper_2510_13668_amd import star

FAKE = ctypes.c_void_p(1 << 20)          # never dereferenced
OTHER = ctypes.c_void_p(1 << 21)
ODD = ctypes.c_void_p((1 << 20) + 8)     # not 16-byte aligned
BIG = 1 << 34


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(star.LIB_PATH):
        from paper_2510_13668_amd import build
        build.build()
    return star.lib()


def _pages(**kw):
    base = dict(n_seq=8, max_pages=4, n_pages=64, page_size=16, n_layers=2, page_bytes=64)
    base.update(kw)
    return star.pages_params(**base)


def _assign(L, p, ws_bytes=BIG, ws=FAKE, **ptrs):
    a = dict.fromkeys(("parent", "new_len", "inst_of", "table", "seq_len", "seq_inst", "refs",
                       "kv", "table_out", "seq_len_out", "seq_inst_out", "refs_out"), FAKE)
    a["parent"] = None
    a.update(ptrs)
    return L.star_assign_pages(ctypes.byref(p) if p is not None else None, *a.values(), ws,
                               ws_bytes, None)


def _compact(L, p, ws_bytes=BIG, ws=FAKE, **ptrs):
    a = dict.fromkeys(("table", "seq_len", "refs", "kv", "table_out", "refs_out", "n_live"), FAKE)
    a["refs_out"] = OTHER
    a.update(ptrs)
    return L.star_compact_pages(ctypes.byref(p) if p is not None else None, *a.values(), ws,
                                ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_seq=-1), -1), (dict(max_pages=0), -1), (dict(n_pages=0), -1), (dict(n_inst=0), -1),
    (dict(n_inst=3), -1), (dict(page_size=0), -1), (dict(n_layers=0), -1), (dict(page_bytes=0), -1),
    (dict(page_stride=32), -1), (dict(layer_stride=32), -1), (dict(layer_stride=-64), -1),
    (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=512), -2),
    (dict(n_inst=2048, n_pages=2048), -2), (dict(page_bytes=24), -2), (dict(page_stride=72), -2),
    (dict(layer_stride=4104), -2), (dict(max_pages=(1 << 26) + 1), -2),
    (dict(page_stride=1 << 60, layer_stride=1 << 60), -3), (dict(n_seq=(1 << 30) + 1), -2),
])
def test_page_calls_reject_bad_scalars(L, kw, status):
    p = _pages(**kw)
    assert _assign(L, p) == status and _compact(L, p) == status
    assert star.assign_pages_workspace_size(p) == star.compact_pages_workspace_size(p) == 0


def test_page_calls_reject_null_pointers_overlaps_and_workspaces(L):
    p = _pages()
    assert _assign(L, None) == -1 and _compact(L, None) == -1
    for name in ("new_len", "table", "seq_len", "refs", "kv", "table_out", "seq_len_out",
                 "refs_out"):
        assert _assign(L, p, **{name: None}) == -1, name
    for name in ("table", "seq_len", "refs", "kv", "table_out", "refs_out", "n_live"):
        assert _compact(L, p, **{name: None}) == -1, name
    two = _pages(n_inst=2)
    assert _assign(L, two, seq_inst=None) == -1 and _assign(L, two, seq_inst_out=None) == -1
    assert _assign(L, p, parent=FAKE) == -1               # a parent's row would be overwritten
    assert _compact(L, p, refs_out=FAKE) == -1
    assert _assign(L, p, kv=ODD) == -2 and _compact(L, p, kv=ODD) == -2
    need = star.assign_pages_workspace_size(p)
    assert need == star.compact_pages_workspace_size(p) > star.STAR_WS_HEADER_BYTES + 64 * 12
    assert _assign(L, p, ws_bytes=need - 1) == -4 and _compact(L, p, ws_bytes=need - 1) == -4
    assert _assign(L, p, ws=None) == -4 and _compact(L, p, ws=ODD) == -4


def _attend(**kw):
    base = dict(n_seq=4, n_rows=4, n_heads=8, n_kv_heads=2, head_dim=128, dtype=star.BF16,
                page_size=16, n_pages=100, max_pages=9, scale=0.1)
    base.update(kw)
    return star.attend_params(**base)


def _decode(L, p, ws_bytes=BIG, ws=FAKE, **ptrs):
    a = dict.fromkeys(("q", "k_new", "v_new", "kv", "table", "seq_len", "out"), FAKE)
    a["lse"] = None
    a.update(ptrs)
    return L.star_attend_decode(ctypes.byref(p) if p is not None else None, *a.values(), ws,
                                ws_bytes, None)


def _prompt(L, p, ws_bytes=BIG, ws=FAKE, **ptrs):
    a = dict.fromkeys(("q", "k_new", "v_new", "kv", "table", "seq_len", "q_start", "out"), FAKE)
    a["lse"] = None
    a.update(ptrs)
    return L.star_attend_prompt(ctypes.byref(p) if p is not None else None, *a.values(), ws,
                                ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_seq=-1, n_rows=-1), -1), (dict(n_rows=-1), -1), (dict(n_heads=0), -1),
    (dict(n_kv_heads=0), -1), (dict(n_kv_heads=3), -1), (dict(head_dim=0), -1),
    (dict(dtype=7), -1), (dict(page_size=0), -1), (dict(n_pages=0), -1), (dict(max_pages=0), -1),
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(q_stride=1023), -1), (dict(kv_stride=255), -1),
    (dict(page_stride=2 * 2 * 16 * 128 * 2 - 16), -1),
    (dict(head_dim=80), -2), (dict(head_dim=512), -2), (dict(page_size=24), -2),
    (dict(page_size=512), -2), (dict(q_stride=1028), -2), (dict(kv_stride=260), -2),
    (dict(page_stride=(1 << 20) + 8), -2), (dict(max_pages=(1 << 26) + 1), -2),
    (dict(n_seq=1 << 28, n_rows=1 << 28), -3), (dict(page_stride=1 << 60), -3),
    (dict(n_seq=(1 << 30) + 1, n_rows=(1 << 30) + 1, n_heads=1, n_kv_heads=1), -2),
    (dict(n_heads=1 << 17), -2), (dict(scale=3e38), -1),
])
def test_attention_rejects_bad_scalars(L, kw, status):
    p = _attend(**kw)
    assert _decode(L, p) == status and _prompt(L, p) == status
    assert star.attend_decode_workspace_size(p) == star.attend_prompt_workspace_size(p) == 0


def test_attention_rejects_null_pointers_and_workspaces(L):
    p = _attend()
    assert _decode(L, None) == -1 and _prompt(L, None) == -1
    for name in ("q", "k_new", "v_new", "kv", "table", "seq_len", "out"):
        assert _decode(L, p, **{name: None}) == -1, name
        assert _prompt(L, p, **{name: None}) == -1, name
    assert _prompt(L, p, q_start=None) == -1
    for name in ("q", "k_new", "v_new", "kv", "out"):
        assert _decode(L, p, **{name: ODD}) == -2 and _prompt(L, p, **{name: ODD}) == -2, name
    assert _decode(L, _attend(n_rows=5)) == -1            # one row a slot
    assert star.attend_decode_workspace_size(_attend(n_rows=5)) == 0
    for call, size in ((_decode, star.attend_decode_workspace_size),
                       (_prompt, star.attend_prompt_workspace_size)):
        assert call(L, p, ws_bytes=size(p) - 1) == -4
        assert call(L, p, ws=None) == -4 and call(L, p, ws=ODD) == -4


def test_binding_checks_the_tensors():
    """Layouts that the pointers alone could not tell apart are refused."""
    rows = (1536, 128, 1)
    fake = lambda *shape: _Meta(torch.empty(shape, dtype=torch.bfloat16))
    qkv = torch.empty((4, 12, 128), dtype=torch.bfloat16)
    assert star._strided(_Meta(qkv[:, :8]), torch.bfloat16, (4, 8, 128), rows) == qkv.data_ptr()
    for bad in (fake(4, 8, 64), fake(4, 8, 128), _Meta(qkv[:, :8].float()),
                _Meta(qkv.transpose(0, 1)[:8].transpose(0, 1)[:, :, :64]),
                _Meta(torch.empty((4, 128, 8), dtype=torch.bfloat16).transpose(1, 2))):
        with pytest.raises(ValueError):
            star._strided(bad, torch.bfloat16, (4, 8, 128), rows)
    with pytest.raises(ValueError):
        star._strided(qkv[:, :8], torch.bfloat16, (4, 8, 128), rows)       # not on a GPU
    one = _Meta(torch.empty((1, 8, 128), dtype=torch.bfloat16))             # one row: any stride
    star._strided(one, torch.bfloat16, (1, 8, 128), (5, 128, 1))


def test_binding_refuses_another_device(monkeypatch):
    class On:
        def __init__(self, device):
            self.device_index = device

        def get_device(self):
            return self.device_index

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    star._same_device(On(1), None)
    star._same_device(On(1), On(1))
    for tensor, stream in ((On(0), None), (On(1), On(0)), (On(0), On(0))):
        with pytest.raises(ValueError):
            star._same_device(tensor, stream)


    star._same_device(On(1), None, On(1))
    with pytest.raises(ValueError):
        star._same_device(On(1), None, On(1), On(-1))


def test_binding_refuses_short_and_mistyped_arrays():
    class At(_Meta):
        def get_device(self):
            return 3

    i32 = torch.int32
    t = torch.zeros((4, 5), dtype=i32)
    assert star._arrays(3, ((i32, 80), (i32, 7)), At(t), None) == [t.data_ptr(), None]
    for bad, n in ((At(t), 81), (At(t.long()), 80), (At(t.t()), 80), (t, 80)):
        with pytest.raises(ValueError):
            star._arrays(3, ((i32, n),), bad)
    # a pool of two layers of ten pages
    pool = star._pages_layout(bytes(star.pages_params(1, 1, 10, 16, 2, 64)))[-1]
    assert pool == 1280
    kv = torch.empty(pool, dtype=torch.uint8)
    assert star._pool(kv, pool) == kv.data_ptr()
    for bad in (kv[1:], torch.empty((40, 64), dtype=torch.uint8).t()):
        with pytest.raises(ValueError):
            star._pool(bad, pool)


def test_binding_follows_changed_parameters():
    p = _attend()
    before = star._attend_layout(bytes(p))
    p.n_rows = p.n_seq = 5
    after = star._attend_layout(bytes(p))
    assert before[1] == (4, 8, 128) and after[1] == (5, 8, 128)
    assert star._attend_layout(bytes(_attend())) == before


class _Meta:
    """A host tensor that says it is on a GPU."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_attention_of_nothing_launches_nothing(L):
    assert _decode(L, _attend(n_seq=0, n_rows=0)) == 0
    assert _prompt(L, _attend(n_seq=0, n_rows=0)) == 0
    assert _prompt(L, _attend(n_seq=4, n_rows=0)) == 0


def test_binding_refuses_types_it_does_not_know(monkeypatch):
    """A type that is none of the two is a ValueError, as the other mistakes are."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class At(_Meta):
        def get_device(self):
            return 0

    t = At(torch.empty((4, 8, 128), dtype=torch.float16))
    t.buf = t
    for call, starts in ((star.attend_decode, ()), (star.attend_prompt, (t,))):
        with pytest.raises(ValueError):
            call(_attend(dtype=7), t, t, t, t, t, t, *starts, t, None, t)
