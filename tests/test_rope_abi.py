"""The rotation's C entry points, and the calls over a cache in 4 bits, reject bad arguments
before touching the device; the frequencies of a table (CPU only)."""
import ctypes

import numpy as np
import pytest

from paper_2609_28870_amd import pc
from test_kv_abi import FAKE, L, append, attn, cache, evict   # noqa: F401

FP4 = dict(dtype=3, k_scale=FAKE, v_scale=FAKE)


def rotation(**kw):
    d = dict(table=FAKE, pos=FAKE, n_pos=100, rot_dim=64, flags=0)
    d.update(kw)
    return pc._Rotation(*(d[name] for name, _ in pc._Rotation._fields_))


def rope(L, r=None, **kw):   # noqa: F811
    d = dict(x=FAKE, xr=256, xh=64, out=FAKE + 0x10000, outr=256, outh=64, dtype=0, rows=5, heads=4, dim=64, ws=FAKE, wsz=256)
    d.update(kw)
    return L.pc_rope(ctypes.byref(r or rotation()), d["x"], d["xr"], d["xh"], d["out"], d["outr"], d["outh"], d["dtype"], d["rows"],
                     d["heads"], d["dim"], d["ws"], d["wsz"], None)


def append_rope(L, c=None, r=None, **kw):   # noqa: F811
    d = dict(table=FAKE, ts=4, kv=FAKE, off=FAKE, n_seqs=3, rows=5, max_kv=64, k=FAKE, kr=128, kh=64, v=FAKE, vr=128, vh=64,
             q=FAKE + 0x10000, qr=256, qh=64, o=FAKE + 0x20000, orow=256, oh=64, heads=4, dtype=0, ws=FAKE, wsz=256)
    d.update(kw)
    return L.pc_kv_append_rope(ctypes.byref(c or cache()), d["table"], d["ts"], d["kv"], d["off"], d["n_seqs"], d["rows"],
                               d["max_kv"], ctypes.byref(r or rotation()), d["k"], d["kr"], d["kh"], d["v"], d["vr"], d["vh"],
                               d["q"], d["qr"], d["qh"], d["o"], d["orow"], d["oh"], d["heads"], d["dtype"], d["ws"], d["wsz"], None)


BAD_ROTATIONS = [dict(table=None), dict(table=FAKE + 4), dict(n_pos=0), dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=66),
                 dict(flags=4)]


@pytest.mark.parametrize("bad", BAD_ROTATIONS, ids=str)
def test_rotation(L, bad):   # noqa: F811
    assert rope(L, rotation(**bad)) == -1
    assert append_rope(L, r=rotation(**bad)) == -1


def test_rotations_that_are_too_large_or_not_there(L):   # noqa: F811
    assert rope(L, rotation(n_pos=0xFFFFFFFF)) == -2
    assert append_rope(L, r=rotation(n_pos=0xFFFFFFFF)) == -2
    assert append_rope(L, r=rotation(flags=2)) == -1          # a cache is not turned back
    assert L.pc_rope(None, FAKE, 256, 64, FAKE, 256, 64, 0, 5, 4, 64, FAKE, 256, None) == -1


def test_rope_rejects(L):   # noqa: F811
    assert rope(L, dtype=2) == -1
    assert rope(L, dtype=3) == -1
    assert rope(L, dim=4) == -1
    assert rope(L, dim=68) == -1
    assert rope(L, dim=264) == -1
    assert rope(L, heads=0) == -1
    assert rope(L, heads=1025) == -1
    assert rope(L, rows=0x80000000) == -2
    assert rope(L, rows=0x7FFFFFFF, heads=1024) == -2         # a launch of 2^32 threads
    assert rope(L, x=None) == -1
    assert rope(L, out=None) == -1
    assert rope(L, x=FAKE + 8) == -1
    assert rope(L, outh=60) == -1
    assert rope(L, xr=100) == -1
    assert rope(L, rotation(pos=None, n_pos=4)) == -1         # five rows at positions 0 to 4
    assert rope(L, ws=None) == -3
    assert rope(L, wsz=255) == -3
    for at in (16, 128, 512, -16, 4 * 512 + 496):
        assert rope(L, out=FAKE + at) == -1                   # over other rows
    assert rope(L, out=FAKE, outr=512) == -1                  # in place, other strides
    for kw in (dict(outh=0), dict(outr=0), dict(outh=56), dict(outr=248), dict(outr=64, outh=312)):
        assert rope(L, **kw) == -1                            # results over each other
    assert rope(L, outr=64, outh=320, ws=None) == -3          # [head, row]
    assert rope(L, x=FAKE, out=FAKE, xh=0, outh=0) == -1


def test_table_rejects(L):   # noqa: F811
    f = (ctypes.c_double * 4)(1.0, 0.1, 0.01, 0.001)

    def table(freq=f, n=4, first=0, pos=10, magnitude=1.0, out=FAKE):
        return L.pc_rope_table(freq, n, first, pos, magnitude, out, None)
    assert table(freq=None) == -1
    assert table(n=0) == -1
    assert table(n=129) == -1
    assert table(magnitude=float("nan")) == -1
    assert table(magnitude=float("inf")) == -1
    assert table(out=None) == -1
    assert table(out=FAKE + 4) == -1
    assert table(pos=0xFFFFFFFF) == -2
    assert table(first=0xFFFFFFFF) == -2
    assert table(first=0xFFFFFFF0, pos=16) == -2
    for bad in (float("nan"), float("inf"), 65537.0, -1e7):
        assert table(freq=(ctypes.c_double * 4)(1.0, bad, 0.01, 0.001)) == -1
    assert table(pos=0, out=None) == 0                        # nothing to do


def test_append_rejects(L):   # noqa: F811
    assert append_rope(L, dtype=1) == -1                      # not the cache's type
    assert append_rope(L, dtype=2) == -1
    assert append_rope(L, dtype=3) == -1
    assert append_rope(L, n_seqs=0x80000000) == -2
    assert append_rope(L, rows=0x80000000) == -2
    assert append_rope(L, max_kv=0x7FFF0001) == -2
    assert append_rope(L, max_kv=65) == -1
    for name in ("kv", "off", "table", "k", "v"):
        assert append_rope(L, **{name: None}) == -1
    assert append_rope(L, q=None) == -1                       # queries without a place, and the other way round
    assert append_rope(L, o=None) == -1
    assert append_rope(L, heads=0) == -1
    assert append_rope(L, heads=1025) == -1
    assert append_rope(L, n_seqs=0) == -1
    assert append_rope(L, ws=None) == -3
    assert append_rope(L, wsz=255) == -3
    for name in ("k", "v", "q"):
        assert append_rope(L, **{name: FAKE + 8}) == -1
    for name in ("kr", "kh", "vr", "vh", "qr", "qh", "orow", "oh"):
        assert append_rope(L, **{name: 68}) == -1


def test_queries_that_overlap(L):   # noqa: F811
    """5 rows: queries of 512 bytes, keys and values of 256."""
    far = dict(k=FAKE, v=FAKE + 0x10000, q=FAKE + 0x20000, o=FAKE + 0x30000)

    def refused(**kw):
        assert append_rope(L, **dict(far, **kw)) == -1
    for at in (0, 16, 256, 1264, -16, -2544):
        refused(o=far["k"] + at)
        refused(o=far["v"] + at)
    for at in (16, 512, -16):
        refused(o=far["q"] + at)
    # beside each other in a fused projection's rows of 1,024 bytes: only what lies in the gaps
    fused = dict(q=FAKE, o=FAKE, qr=512, orow=512, k=FAKE + 512, kr=512, v=FAKE + 768, vr=512)
    refused(**dict(fused, k=FAKE + 496))
    refused(**dict(fused, v=FAKE + 784))
    refused(**dict(fused, kr=1024))
    refused(**dict(fused, oh=128))
    refused(oh=0)
    refused(orow=0)
    assert append_rope(L, **dict(fused, ws=None)) == -3       # as they are meant


BAD_FP4 = [dict(k_scale=None), dict(v_scale=None), dict(head_dim=48), dict(head_dim=16), dict(stride_slot=80), dict(stride_page=2064),
           dict(k=FAKE + 8)]


@pytest.mark.parametrize("bad", BAD_FP4, ids=str)
def test_descriptor_of_4_bits(L, bad):   # noqa: F811
    bad = dict(FP4, **bad)
    for call in (append, attn, evict):
        assert call(L, cache(**bad)) == -1
    assert append_rope(L, cache(**bad)) == -1


def test_calls_on_4_bits(L):   # noqa: F811
    c = cache(**FP4)
    assert append(L, c, dtype=2) == -1
    assert append(L, c, dtype=3) == -1
    assert append(L, c, rows=(1 << 31) - 1, n_seqs=3) == -2   # more than a launch holds
    assert append(L, c, wsz=255) == -3
    assert append(L, c, dtype=1, wsz=255) == -3               # any of the two types of new tokens
    assert attn(L, c, dtype=3) == -1
    assert attn(L, c, ws=None) == -3
    assert evict(L, c, ws=None) == -3
    assert append_rope(L, c, ws=None) == -3


def test_workspaces(L):   # noqa: F811
    assert L.pc_rope_ws() >= 256 and L.pc_kv_append_rope_ws() >= 256


@pytest.mark.parametrize("rot", [2, 6, 64, 128])
def test_frequencies(rot):
    i = np.arange(rot // 2)
    plain = pc.rope_frequencies(rot, 500.0)
    assert np.allclose(plain, np.exp(-2 * i / rot * np.log(500.0)), rtol=1e-14)
    assert np.allclose(pc.rope_frequencies(rot, 500.0, "linear", 4.0), plain / 4, rtol=1e-14)
    grown = pc.rope_frequencies(rot, 500.0, "base", 4.0)
    assert grown[0] == 1 and (rot == 2 or np.isclose(grown[-1], plain[-1] / 4, rtol=1e-13))
    ramp = pc.rope_frequencies(rot, 500.0, "ramp", 4.0, trained=1000, slow=2.0, fast=20.0)
    for f, g in zip(plain, ramp):
        turns = 1000 * f / (2 * np.pi)
        keep = 1.0 if turns >= 20 else 0.0 if turns <= 2 else (turns - 2) / 18
        assert np.isclose(g, f * keep + f / 4 * (1 - keep), rtol=1e-13)
    assert np.allclose(pc.rope_frequencies(rot, 500.0, "ramp", 1.0, trained=1000), plain, rtol=1e-15)


def test_frequencies_refused():
    for kw in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=8, base=0.0), dict(rot_dim=8, base=float("nan")),
               dict(rot_dim=8, factor=0.0), dict(rot_dim=8, scaling="other"), dict(rot_dim=8, scaling="ramp"),
               dict(rot_dim=8, scaling="ramp", trained=10, slow=3.0, fast=3.0)):
        with pytest.raises(pc.PcError):
            pc.rope_frequencies(**kw)
