"""Where pc_kv_append_rope's queries may lie beside its keys and values: every layout that shares memory is refused,
and the layouts of fused projections are taken (CPU only: calls that pass every check of arguments stop at the
workspace)."""
import itertools

import numpy as np
import pytest

from test_kv_abi import FAKE, L, cache   # noqa: F401
from test_rope_abi import append_rope

FAR = FAKE + 0x100000
RUN = 128    # bytes of a head of 64


def runs(at, row, head, n_rows, heads):
    return {at + t * row + h * head for t, h in itertools.product(range(n_rows), range(heads))}


def share(a, b):
    """Whether runs of RUN bytes at two sets of multiples of RUN / 8 share a byte."""
    return any(abs(x - y) < RUN for x in a for y in b)


def call(L, n_rows, heads, kvh, q, k):   # noqa: F811
    """-1: refused, -3: fine but for the workspace.  q and k: (byte, row stride, head stride), queries in place."""
    return append_rope(L, cache(n_kv_heads=kvh), rows=n_rows, heads=heads, q=q[0], o=q[0], qr=q[1] // 2, orow=q[1] // 2, qh=q[2] // 2,
                       oh=q[2] // 2, k=k[0], kr=k[1] // 2, kh=k[2] // 2, v=FAR, vr=kvh * RUN // 2, vh=RUN // 2, ws=None)


@pytest.mark.parametrize("n_rows", [1, 2, 5])
@pytest.mark.parametrize("heads", [1, 4])
def test_a_heads_query_key_and_value_beside_each_other(L, n_rows, heads):   # noqa: F811
    """A fused projection as [row, head, 3, head_dim]."""
    row, head = heads * 3 * RUN, 3 * RUN
    for at in (RUN, 2 * RUN, -RUN):
        assert call(L, n_rows, heads, heads, (FAKE, row, head), (FAKE + at, row, head)) == -3
    for at in (0, 16, RUN - 16, 2 * RUN + 16, -16):
        if heads > 1 or abs(at) < RUN:
            assert call(L, n_rows, heads, heads, (FAKE, row, head), (FAKE + at, row, head)) == -1


def test_fewer_heads_of_keys_between_the_queries(L):   # noqa: F811
    row, head = 8 * 2 * RUN, 2 * RUN
    assert call(L, 3, 8, 2, (FAKE, row, head), (FAKE + RUN, row, head)) == -3
    assert call(L, 3, 8, 1, (FAKE, row, head), (FAKE + RUN, row, RUN)) == -3      # one head's stride is anything
    assert call(L, 3, 1, 1, (FAKE, row, RUN), (FAKE + RUN, row, RUN)) == -3
    assert call(L, 3, 8, 2, (FAKE, row, head), (FAKE + RUN - 16, row, head)) == -1


@pytest.mark.parametrize("seed", range(6))
def test_what_shares_memory_is_refused(L, seed):   # noqa: F811
    r = np.random.default_rng(seed)
    for _ in range(400):
        n_rows, heads, kvh = (int(x) for x in r.integers(1, 5, 3))
        q_head, k_head = (int(x) for x in r.integers(8, 40, 2) * 16)
        if r.integers(2):
            k_head = q_head
        q_row = int(r.integers(8, 160)) * 16
        k_row = q_row if r.integers(4) else int(r.integers(8, 160)) * 16
        at = int(r.integers(-60, 61)) * 16
        q, k = (FAKE, q_row, q_head), (FAKE + at, k_row, k_head)
        own = sorted(runs(*q, n_rows, heads))
        apart = len(own) == n_rows * heads and all(b - a >= RUN for a, b in zip(own, own[1:]))
        shared = share(own, runs(*k, n_rows, kvh))
        got = call(L, n_rows, heads, kvh, q, k)
        assert got in (-1, -3)
        assert got == -1 or (apart and not shared)
