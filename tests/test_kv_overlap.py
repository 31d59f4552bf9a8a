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


def test_attention_results(L):   # noqa: F811
    """5 rows of 4 heads of 64 elements, 2 bytes each: runs of 128 bytes."""
    def refused(out, **kw):
        assert attn(L, out=out, **kw) == -1
    for at in (16, 128, 512, 4 * 512 + 496, -16, -512, 16 - 2560):
        refused(FAKE + at)                                        # dense, at another place
    refused(FAKE, wout=FAKE + 0x10000, wstride=64)                # in place, with weights
    refused(FAKE, outr=512)                                       # in place, other strides
    refused(FAKE, outh=128, outr=512)
    wide = dict(qr=512, outr=512)                                 # rows of 1,024 bytes, half of them used
    for at in (0, 16, 496, 528, -16, 1024 + 16):
        refused(FAKE + at, wout=FAKE + 0x10000, wstride=64, **wide)
    heads_apart = dict(qh=128, outh=128, qr=512, outr=512)        # runs with gaps of their own length
    for at in (16, 112, 144, 256, -16):
        refused(FAKE + at, **heads_apart)
    heads_first = dict(qr=128, outr=128, qh=640, outh=640)        # [head][row], runs with gaps
    for at in (16, 112, 144, 256, -16):
        refused(FAKE + at, **heads_first)


def test_attention_weights(L):   # noqa: F811
    """3 sequences, 2 heads, 64 weights each: in place or apart."""
    size, far = 6 * 64 * 4, dict(out=FAKE + 0x10000, wstride=64)
    for at in (4, 256, size - 4, -4, 4 - size):
        assert attn(L, w=FAKE + 0x20000, wout=FAKE + 0x20000 + at, **far) == -1
