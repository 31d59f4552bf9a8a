"""Sessions over one paged cache: chained block keys find the pages that a prompt
shares with what is cached, only its other tokens are computed, their queries and keys
turned by their positions on the way into the cache, decode steps accumulate the
attention weight of every cached token, and sessions that outgrow their budget are
cut to the tokens with the most of it.

    python examples/paged_sessions.py [--sessions N] [--steps K] [--budget B] [--cache bf16|fp4]

One attention layer with random weights stands for a model.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_28870_amd import pc  # noqa: E402

PAGE = 16


class Server:
    def __init__(self, sessions, heads=8, kv_heads=2, dim=64, n_pages=4096, max_kv=2048, dtype=torch.bfloat16, seed=0,
                 cache="bf16", positions=8192):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.dtype = heads, kv_heads, dim, dtype
        width = heads * dim
        self.embed = torch.randn(32000, width, generator=g, device="cuda", dtype=dtype)
        self.qkv = torch.randn(width, (heads + 2 * kv_heads) * dim, generator=g, device="cuda", dtype=dtype) * width ** -0.5
        if cache == "fp4":      # two codes a byte, and the scale of every 32 of them
            codes, scales = (torch.zeros(2, n_pages, kv_heads, PAGE, n, device="cuda", dtype=torch.uint8) for n in (dim // 2, dim // 32))
            codes = codes.view(torch.float4_e2m1fn_x2)
            self.cache = pc.PagedCache(codes[0], codes[1], scales[0], scales[1])
        else:
            k = torch.zeros(n_pages, kv_heads, PAGE, dim, device="cuda", dtype=dtype)
            self.cache = pc.PagedCache(k, torch.zeros_like(k))
        self.angles = pc.rope_table(pc.rope_frequencies(dim), positions)
        self.free = list(range(n_pages - 1, -1, -1))
        self.users = np.zeros(n_pages, np.int64)      # sessions that hold a page
        self.page_of_key = {}                         # full blocks by their chained key
        self.key_of_page = {}
        self.max_kv = max_kv
        self.pages = [[] for _ in range(sessions)]
        self.len = np.zeros(sessions, np.int64)
        self.text = np.zeros(sessions, np.int64)      # tokens so far, the evicted ones among them: the next one's position
        self.weight = torch.zeros(sessions, kv_heads, max_kv, device="cuda")
        self.shared_tokens = self.evictions = 0

    def _take(self, session):
        page = self.free.pop()
        self.users[page] = 1
        self.pages[session].append(page)

    def _drop(self, page):
        self.users[page] -= 1
        if not self.users[page]:
            self.page_of_key.pop(self.key_of_page.pop(page, None), None)
            self.free.append(page)

    def _table(self):
        """Page tables on the device; entries past a session's pages are not read."""
        cols = self.max_kv // PAGE
        table = np.zeros((len(self.pages), cols), np.int32)
        for s, p in enumerate(self.pages):
            table[s, :len(p)] = p
        return torch.from_numpy(table).cuda()

    def _i32(self, x):
        return torch.from_numpy(np.asarray(x, np.int32)).cuda()

    def admit(self, prompts):
        """Attention of every prompt's tokens that are not cached.  A session gets the pages
        of its longest cached prefix; its last token is always computed."""
        lens = np.array([len(p) for p in prompts])
        blocks = lens // PAGE
        off = np.concatenate([[0], np.cumsum(blocks)])
        start = np.concatenate([[0], np.cumsum(lens)[:-1]])
        keys, _, _ = pc.hash_blocks(torch.from_numpy(np.concatenate(prompts).astype(np.int32)).cuda(), pc.to_dev_u64(start),
                                    pc.to_dev_u32(lens), pc.to_dev_u64(off), int(off[-1]), PAGE, want_depth=False)
        keys = pc.as_u64(keys)
        out = []
        for s, prompt in enumerate(prompts):          # one after the other, so that each finds the ones before
            mine = keys[off[s]:off[s + 1]]
            for key in mine[:(len(prompt) - 1) // PAGE]:
                page = self.page_of_key.get(int(key))
                if page is None:
                    break
                self.users[page] += 1
                self.pages[s].append(page)
            cached = len(self.pages[s]) * PAGE
            self.shared_tokens += cached
            self.len[s] = self.text[s] = cached
            out.append(self.step([s], [prompt[cached:]])[0])
            for i, key in enumerate(mine):
                if int(key) not in self.page_of_key:
                    self.page_of_key[int(key)] = self.pages[s][i]
                    self.key_of_page[self.pages[s][i]] = int(key)
        return out

    def step(self, sessions, tokens):
        """New tokens of some sessions into the cache, and their attention over it."""
        new = np.zeros(len(self.pages), np.int64)
        pos = []
        for s, t in sorted(zip(sessions, tokens), key=lambda x: x[0]):
            new[s] = len(t)
            pos.append(np.arange(self.text[s], self.text[s] + len(t)))
            self.len[s] += len(t)
            self.text[s] += len(t)
            while len(self.pages[s]) * PAGE < self.len[s]:
                self._take(s)
        order = [t for _, t in sorted(zip(sessions, tokens), key=lambda x: x[0])]
        x = self.embed[torch.from_numpy(np.concatenate(order).astype(np.int64)).cuda()] @ self.qkv
        x = x.view(-1, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = x.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        # a session that takes no part has no new rows, and keeps its weights
        table, kv_len, q_off = self._table(), self._i32(self.len), self._i32(np.concatenate([[0], np.cumsum(new)]))
        q, ws = pc.kv_append_rope(self.cache, table, kv_len, q_off, k, v, self.angles, pos=self._i32(np.concatenate(pos)), q=q, q_out=q)
        out, _, _, ws2 = pc.attn_paged(q, self.cache, table, kv_len, q_off, int(new.max()), max_kv=self.max_kv,
                                       weight=self.weight, weight_out=self.weight)
        for w in (ws, ws2):
            if pc.workspace_status(w):
                raise pc.PcError("a length or page does not fit")
        self.last = (q, table, kv_len, q_off, out)
        return out.split([int(new[s]) for s in sorted(sessions)])

    def evict(self, session, budget, recent):
        """The session's `budget` tokens of the most weight move to pages of their own."""
        old = self.pages[session]
        dst = [self.free.pop() for _ in range((budget + PAGE - 1) // PAGE)]
        r = pc.kv_evict(self.cache, self._table()[session:session + 1], self._i32(self.len[session:session + 1]),
                        self.weight[session:session + 1], budget, recent, dst_table=self._i32([dst]))
        if pc.workspace_status(r["ws"]):
            raise pc.PcError("a length or page does not fit")
        self.weight[session].zero_()
        self.weight[session, :, :budget] = r["weight"][0]
        self.users[dst] = 1
        self.pages[session], self.len[session] = dst, min(self.len[session], budget)
        for page in old:
            self._drop(page)
        self.evictions += 1


def run(sessions=6, steps=40, budget=256, recent=32, seed=0, cache="bf16"):
    r = np.random.default_rng(seed)
    server = Server(sessions, seed=seed, cache=cache)
    system = r.integers(0, 32000, 200)
    server.admit([np.concatenate([system, r.integers(0, 32000, int(r.integers(1, 400)))]) for _ in range(sessions)])
    for _ in range(steps):
        for s in range(sessions):
            if server.len[s] > budget + 4 * PAGE:
                server.evict(s, budget, recent)
        server.step(list(range(sessions)), [r.integers(0, 32000, 1) for _ in range(sessions)])
    return server


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--sessions", type=int, default=6)
    p.add_argument("--steps", type=int, default=40)
    p.add_argument("--budget", type=int, default=256)
    p.add_argument("--cache", choices=["bf16", "fp4"], default="bf16")
    a = p.parse_args()
    server = run(a.sessions, a.steps, a.budget, min(32, a.budget), cache=a.cache)
    print("%d sessions, %d decode steps: %d prompt tokens found in shared pages, %d evictions, lengths %s, %d pages in use" % (
        a.sessions, a.steps, server.shared_tokens, server.evictions, server.len.tolist(), int((server.users > 0).sum())))


if __name__ == "__main__":
    main()
