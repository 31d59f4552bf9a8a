"""Arrays of a call over a paged cache that share memory with what it writes are refused (CPU
only: every call below fails validation)."""
from test_kv_abi import FAKE, L, attn, evict   # noqa: F401


def test_eviction_results(L):   # noqa: F811
    """3 sequences, 2 heads: 64 weights and 8 kept slots each."""
    kept, weights = 6 * 8 * 4, 6 * 64 * 4
    far = dict(w=FAKE, kept=FAKE + 0x10000, nl=FAKE + 0x20000, wout=FAKE + 0x30000)

    def refused(**kw):
        assert evict(L, **dict(far, **kw)) == -1
    for at in (0, 4, kept - 4, 4 - kept):
        refused(wout=far["kept"] + at)
    for at in (0, -8, kept - 4):
        refused(nl=far["kept"] + at)
        refused(nl=far["wout"] + at)
    for at in (0, 4 - kept, weights - 4):
        refused(kept=FAKE + at)
        refused(wout=FAKE + at)
    for at in (0, -8, weights - 4):
        refused(nl=FAKE + at)
