"""The C entry points over a paged cache reject bad arguments before touching the
device (CPU only, no compute), and their workspaces grow with their arguments."""
import ctypes
import os

import pytest

from paper_2609_28870_amd import pc

FAKE = 0x1000   # never dereferenced: every call below fails validation


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pc.LIB_PATH):
        pytest.fail("libpc.so is not built (run __graft_entry__.build())")
    return pc.lib()


def cache(**kw):
    d = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, stride_page=2048, stride_head=1024, stride_slot=64, dtype=0,
             n_pages=10, page_size=16, n_kv_heads=2, head_dim=64)
    d.update(kw)
    return pc._KvCache(*(d[name] for name, _ in pc._KvCache._fields_))


BAD_CACHES = [dict(k=None), dict(v=None), dict(dtype=3), dict(dtype=2), dict(k_scale=FAKE), dict(k_scale=FAKE, v_scale=FAKE),
              dict(dtype=2, k_scale=FAKE), dict(page_size=0), dict(page_size=65537), dict(n_kv_heads=0), dict(n_kv_heads=1025),
              dict(head_dim=8), dict(head_dim=72), dict(head_dim=272), dict(n_pages=0), dict(k=FAKE + 8), dict(v=FAKE + 2),
              dict(stride_page=2049), dict(stride_head=1028), dict(stride_slot=4),
              dict(dtype=2, k_scale=FAKE, v_scale=FAKE, stride_slot=72)]


def append(L, c=None, **kw):
    d = dict(table=FAKE, ts=4, kv=FAKE, off=FAKE, n_seqs=3, rows=5, max_kv=64, k=FAKE, kr=128, kh=64, v=FAKE, vr=128, vh=64,
             dtype=0, ws=FAKE, wsz=256)
    d.update(kw)
    return L.pc_kv_append(ctypes.byref(c or cache()), d["table"], d["ts"], d["kv"], d["off"], d["n_seqs"], d["rows"],
                          d["max_kv"], d["k"], d["kr"], d["kh"], d["v"], d["vr"], d["vh"], d["dtype"], d["ws"], d["wsz"], None)


def attn(L, c=None, **kw):
    d = dict(table=FAKE, ts=4, kv=FAKE, off=FAKE, n_seqs=3, rows=5, max_q=4, max_kv=64, q=FAKE, qr=256, qh=64, dtype=0,
             heads=4, scale=0.1, flags=1, window=0, out=FAKE, outr=256, outh=64, lse=None, w=None, wout=None, wstride=0,
             ws=FAKE, wsz=1 << 40)
    d.update(kw)
    return L.pc_attn_paged(ctypes.byref(c or cache()), d["table"], d["ts"], d["kv"], d["off"], d["n_seqs"], d["rows"],
                           d["max_q"], d["max_kv"], d["q"], d["qr"], d["qh"], d["dtype"], d["heads"], d["scale"], d["flags"],
                           d["window"], d["out"], d["outr"], d["outh"], d["lse"], d["w"], d["wout"], d["wstride"], d["ws"],
                           d["wsz"], None)


def evict(L, c=None, **kw):
    d = dict(table=FAKE, ts=4, kv=FAKE, n_seqs=3, max_kv=64, w=FAKE, wstride=64, budget=8, recent=2, dst=FAKE, dstride=1,
             kept=FAKE, wout=None, nl=FAKE, ws=FAKE, wsz=1 << 40)
    d.update(kw)
    return L.pc_kv_evict(ctypes.byref(c or cache()), d["table"], d["ts"], d["kv"], d["n_seqs"], d["max_kv"], d["w"],
                         d["wstride"], d["budget"], d["recent"], d["dst"], d["dstride"], d["kept"], d["wout"], d["nl"],
                         d["ws"], d["wsz"], None)


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_descriptor(L, bad):
    for call in (append, attn, evict):
        assert call(L, cache(**bad)) == -1


def test_no_descriptor(L):
    assert L.pc_kv_append(None, FAKE, 4, FAKE, FAKE, 3, 5, 64, FAKE, 128, 64, FAKE, 128, 64, 0, FAKE, 256, None) == -1
    assert append(L, cache(n_pages=0xFFFFFFFF)) == -2


def test_append_rejects(L):
    assert append(L, dtype=1) == -1            # not the cache's type
    assert append(L, dtype=2) == -1
    assert append(L, n_seqs=0x80000000) == -2
    assert append(L, rows=0x80000000) == -2
    assert append(L, max_kv=0x7FFF0001) == -2
    assert append(L, max_kv=65) == -1          # four pages of sixteen
    assert append(L, kv=None) == -1
    assert append(L, off=None) == -1
    assert append(L, table=None) == -1
    assert append(L, k=None) == -1
    assert append(L, v=None) == -1
    assert append(L, k=FAKE + 4) == -1
    assert append(L, vr=100) == -1
    assert append(L, n_seqs=0) == -1
    assert append(L, ws=None) == -3
    assert append(L, wsz=255) == -3


def test_attention_rejects(L):
    assert attn(L, dtype=1) == -1
    assert attn(L, heads=0) == -1
    assert attn(L, heads=3) == -1
    assert attn(L, heads=1026) == -1
    assert attn(L, flags=2) == -1
    assert attn(L, scale=float("nan")) == -1
    assert attn(L, scale=float("inf")) == -1
    assert attn(L, max_kv=65) == -1
    assert attn(L, max_kv=0x7FFF0001) == -2
    assert attn(L, rows=0x7FFFFFFF) == -2
    assert attn(L, w=FAKE) == -1               # weights without a place for them
    assert attn(L, wout=FAKE, wstride=63) == -1
    assert attn(L, max_q=0) == -1
    assert attn(L, q=None) == -1
    assert attn(L, out=None) == -1
    assert attn(L, kv=None) == -1
    assert attn(L, off=None) == -1
    assert attn(L, table=None) == -1
    assert attn(L, n_seqs=0) == -1
    assert attn(L, q=FAKE + 8) == -1
    assert attn(L, outh=60) == -1
    assert attn(L, ws=None) == -3
    need = L.pc_attn_paged_ws(3, 5, 4, 64, 4, 2, 64, 0)
    assert attn(L, wsz=need - 1) == -3
    more = L.pc_attn_paged_ws(3, 5, 4, 64, 4, 2, 64, 1)
    assert more > need and attn(L, wout=FAKE, wstride=64, wsz=more - 1) == -3


def test_eviction_rejects(L):
    assert evict(L, budget=0) == -1
    assert evict(L, recent=9) == -1
    assert evict(L, max_kv=0x7FFF0001) == -2
    assert evict(L, n_seqs=0x60000000) == -2
    assert evict(L, wstride=63) == -1
    assert evict(L, w=None) == -1
    assert evict(L, kept=None) == -1
    assert evict(L, nl=None) == -1
    assert evict(L, kv=None) == -1
    assert evict(L, budget=17) == -1           # one destination page of sixteen
    assert evict(L, max_kv=64, ts=3) == -1
    assert evict(L, ws=None) == -3
    assert evict(L, wsz=0) == -3


def test_workspaces(L):
    assert L.pc_kv_append_ws() >= 256
    assert L.pc_kv_evict_ws(4, 2, 1000) >= 256
    for max_q in (1, 5, 100):
        base = L.pc_attn_paged_ws(4, 4 * max_q, max_q, 4096, 16, 4, 128, 0)
        assert base >= 256
        assert L.pc_attn_paged_ws(4, 4 * max_q, max_q, 4096, 16, 4, 128, 1) > base
        assert L.pc_attn_paged_ws(4, 4 * max_q, max_q, 4096, 16, 4, 256, 0) >= base
