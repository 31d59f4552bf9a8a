"""Calls over a paged cache whose launches would hold 2^32 threads or more are refused as too
large before anything is enqueued (CPU only: every call below fails validation; one that
is just small enough gets as far as its missing workspace)."""
from test_kv_abi import FAKE, L, append, attn, evict   # noqa: F401


def test_append(L):   # noqa: F811
    assert append(L, rows=(1 << 28) - 16) == -2
    assert append(L, rows=(1 << 28) - 32, ws=None) == -3


def test_attention_rows(L):   # noqa: F811
    # few rows: a workgroup for every sequence and head
    assert attn(L, n_seqs=1 << 23, max_q=1, max_kv=16) == -2
    assert attn(L, n_seqs=(1 << 23) - 1024, max_q=1, max_kv=16, ws=None) == -3
    # chunks
    assert attn(L, n_seqs=1 << 23, max_q=100, max_kv=16) == -2
    assert attn(L, n_seqs=(1 << 23) - 1024, max_q=100, max_kv=16, ws=None) == -3


def test_attention_weights(L):   # noqa: F811
    long = dict(ts=1 << 17, max_kv=1 << 21, wout=FAKE, wstride=1 << 21)
    assert attn(L, n_seqs=1024, max_q=100, **long) == -2
    assert attn(L, n_seqs=1023, max_q=100, ws=None, **long) == -3
    assert attn(L, n_seqs=4096, max_q=1, **long) == -2


def test_eviction(L):   # noqa: F811
    assert evict(L, n_seqs=1 << 21, dst=None) == -2
    assert evict(L, n_seqs=(1 << 21) - 1, dst=None, ws=None) == -3
    long = dict(ts=1 << 16, max_kv=1 << 20, wstride=1 << 20, budget=1 << 20, dstride=1 << 16)
    assert evict(L, n_seqs=1 << 15, **dict(long, dst=None)) == -2
    assert evict(L, n_seqs=(1 << 15) - 1, ws=None, **dict(long, dst=None)) == -3
    assert evict(L, n_seqs=512, **long) == -2
    assert evict(L, n_seqs=511, ws=None, **long) == -3


def test_workspace_of_scores(L):   # noqa: F811
    """Few rows with weights: what holds their scores is bounded, whatever the room for slots is, and
    a workspace for some room holds out for less of it."""
    parts = L.pc_attn_paged_ws(96, 384, 4, 131072, 64, 8, 128, 0)
    assert L.pc_attn_paged_ws(96, 384, 4, 131072, 64, 8, 128, 1) <= parts + (4 << 30) + (1 << 20)
    sizes = [L.pc_attn_paged_ws(64, 256, 4, max_kv, 64, 8, 128, 1)
             for max_kv in (1, 1 << 10, 1 << 15, (1 << 16) - 1, 1 << 16, (1 << 16) + 1, 1 << 17, 1 << 20, 0x7FFF0000)]
    assert sizes == sorted(sizes) and 4 << 30 <= sizes[4] and sizes[-1] <= parts + (4 << 30) + (1 << 20)
