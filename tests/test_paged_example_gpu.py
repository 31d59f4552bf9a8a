"""The paged-session example: pages are shared by key, budgets hold, and its last step's
attention is the definition's over what its cache then holds."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import kv_plain

pytestmark = pytest.mark.gpu


def test_sessions_share_pages_and_keep_their_budget():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_sessions.py")
    spec = importlib.util.spec_from_file_location("paged_sessions", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    server = example.run(sessions=5, steps=12, budget=128, recent=16, seed=3)
    torch.cuda.synchronize()
    assert server.shared_tokens == 4 * (200 // 16) * 16        # the system prompt's full blocks
    assert server.evictions >= 4 and server.len.max() <= 128 + 4 * 16 + 12
    held = [p for s in server.pages for p in s]
    assert sorted(set(held)) == sorted(np.flatnonzero(server.users).tolist())
    assert all(held.count(p) == server.users[p] for p in set(held))
    assert set(server.free).isdisjoint(held) and len(server.free) + len(set(held)) == server.users.size
    q, table, kv_len, q_off, out = server.last
    k, v = kv_plain.cache_values(server.cache.k, server.cache.v, None, None)
    (want, _, _), (tol, _, _) = kv_plain.attention(q, k, v, table.cpu().numpy(), kv_len.cpu().numpy(), q_off.cpu().numpy(),
                                                   q.shape[2] ** -0.5, True, 0)
    got = out.cpu().double().numpy()
    assert np.all(np.abs(got - want) <= tol)
    w = server.weight.cpu().numpy()
    assert np.isfinite(w).all() and (w >= 0).all()
