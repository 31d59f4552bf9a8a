"""Workloads that the operators over a paged cache of KV blocks are measured on:
writing new tokens into it, attention of new tokens over it (a chunk, drafted
tokens, one token), the attention weight that its tokens accumulate, and the
eviction of the tokens with the least of it.

``run`` makes the calls of ``paper_2609_28870_amd.pc`` where ``own`` is true,
and computes the same in elementary torch operations in 32 bits where it is
not.  Block sizes, context caps and the shared prefix are those of the
repository's traces; the 32 query heads over 4 key/value heads of 128 are the
geometry behind its 1.5 MiB a block of 48 layers.
"""
import math
import random

import torch

own = False

BF16, F16, FP8 = "bf16", "f16", "fp8"
TYPES = {BF16: torch.bfloat16, F16: torch.float16, FP8: torch.float8_e4m3fn}
SIZE = {BF16: 2, F16: 2, FP8: 1}
SHARED = 2048            # tokens of a system prompt that sequences share
E4M3_MAX = 448.0
PLAIN_SCORES = 3.0e9     # most (row, key) pairs that the plain form holds at once


def listed():
    usual = dict(heads=32, kv_heads=4, dim=128)
    return [
        # the new token of every running sequence goes into its last block
        dict(name="append_decode", kind="append", seqs=256, new=1, tail=96, mixed=True, page=16, cache=BF16, type=BF16, **usual),
        # a scheduler step of ragged prefill chunks into an 8-bit cache
        dict(name="append_chunks_fp8", kind="append", seqs=24, new=2048, tail=0, mixed=True, page=64, cache=FP8, type=BF16, **usual),
        # one user, one token: latency alone
        dict(name="decode_one", kind="attend", seqs=1, new=1, kv=1537, mixed=False, page=16, cache=BF16, type=BF16,
             window=0, causal=True, weights=False, **usual),
        # the decode step of a batch of chat sessions
        dict(name="decode_batch", kind="attend", seqs=64, new=1, kv=32768, mixed=True, page=16, cache=BF16, type=BF16,
             window=0, causal=True, weights=False, **usual),
        # agent sessions at their context cap over an 8-bit cache
        dict(name="decode_long_fp8", kind="attend", seqs=8, new=1, kv=131072, mixed=False, page=64, cache=FP8, type=BF16,
             window=0, causal=True, weights=False, **usual),
        # five drafted tokens a sequence, a key/value head for every query head, odd blocks
        dict(name="drafted", kind="attend", seqs=24, new=5, kv=6001, mixed=True, page=24, cache=F16, type=F16,
             window=0, causal=True, weights=False, heads=16, kv_heads=16, dim=64),
        # the missed suffix of a long agent turn over its cached prefix
        dict(name="chunk_long", kind="attend", seqs=1, new=2048, kv=32768, mixed=False, page=16, cache=BF16, type=BF16,
             window=0, causal=True, weights=False, **usual),
        # a step of ragged chunks and single tokens, a group of seven heads, a window
        dict(name="chunks_ragged", kind="attend", seqs=12, new=777, kv=8192, mixed=True, page=16, cache=F16, type=F16,
             window=4096, causal=True, weights=False, heads=28, kv_heads=4, dim=128),
        # a decode step that also accumulates the weights an eviction ranks by
        dict(name="decode_weights", kind="attend", seqs=32, new=1, kv=16384, mixed=True, page=16, cache=BF16, type=BF16,
             window=0, causal=True, weights=True, **usual),
        # a prefill chunk that does
        dict(name="chunk_weights", kind="attend", seqs=2, new=1024, kv=16384, mixed=False, page=64, cache=BF16, type=BF16,
             window=0, causal=True, weights=True, **usual),
        # one sequence of a chat turn cut to its budget
        dict(name="evict_one", kind="evict", seqs=1, kv=4099, mixed=False, budget=1024, recent=64, page=16, cache=BF16, **usual),
        # agent sessions cut to a fraction of their contexts, together
        dict(name="evict_batch", kind="evict", seqs=16, kv=65536, mixed=True, budget=8192, recent=1000, page=64, cache=BF16, **usual),
    ]


HEADS = [(32, 4, 128), (28, 4, 128), (16, 16, 64), (8, 1, 256), (64, 8, 128), (20, 4, 96), (12, 12, 80), (9, 3, 64)]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    bytes_most = max(work(c)["bytes"] for c in listed())
    flops_most = max(work(c)["flops"] for c in listed())
    while True:
        heads, kv_heads, dim = rng.choice(HEADS)
        kind = rng.choice(["append", "attend", "attend", "attend", "attend", "evict"])
        t = rng.choice([BF16, BF16, F16])
        case = dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([16, 16, 64, 256, 24, 10]),
                    cache=rng.choice([t, t, FP8]), seqs=log_int(1, 96), mixed=rng.random() < 0.7)
        if kind == "append":
            case.update(type=t, new=rng.choice([1, log_int(2, 4096)]), tail=log_int(1, 500))
        elif kind == "attend":
            case.update(type=t, new=rng.choice([1, rng.randint(2, 9), log_int(10, 4096)]), kv=log_int(16, 131072),
                        window=rng.choice([0, 0, 0, log_int(16, 8192)]), causal=rng.random() < 0.85,
                        weights=rng.random() < 0.3)
            case["new"] = min(case["new"], case["kv"])
        else:
            kv = log_int(64, 131072)
            case.update(kv=kv, budget=log_int(16, kv), recent=0)
            case["recent"] = rng.randint(0, case["budget"] // 2)
        w = work(case)
        new, kv = lengths(case)
        if w["bytes"] > bytes_most or w["flops"] > flops_most or not sum(kv):
            continue
        if kind == "attend" and len(kv) * max(new) * heads * max(kv) > PLAIN_SCORES:
            continue
        if len(kv) * max(kv) * kv_heads * dim * 8 > 24e9:
            continue
        return case


# ------------------------------------------------------------------ inputs

def lengths(case):
    """New tokens and cache length (new ones included) of every sequence: the
    largest first, the others spread over six octaves where the batch is mixed,
    an idle one (no tokens) among many."""
    r = random.Random("%s %s %s" % (case["kind"], case["seqs"], case.get("kv", case.get("new"))))
    n = case["seqs"]
    spread = [1.0] + [2.0 ** -r.uniform(0, 6) if case["mixed"] else 1.0 for _ in range(n - 1)]
    share = [1.0] + [r.uniform(0.02, 1) if case["mixed"] else 1.0 for _ in range(n - 1)]
    if case["kind"] == "append":
        new = [max(1, round(case["new"] * f)) for f in share]
        kv = [SHARED + case["tail"] + m for m in new]
    elif case["kind"] == "attend":
        kv = [max(1, round(case["kv"] * f)) for f in spread]
        new = [min(max(1, round(case["new"] * f)), c) for f, c in zip(share, kv)]
    else:
        kv = [max(1, round(case["kv"] * f)) for f in spread]
        new = [0] * n
    if case["mixed"] and n >= 16:
        new[n // 2] = kv[n // 2] = 0
    return new, kv


def _pages(tokens, page):
    return (tokens + page - 1) // page


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev, page, kvh, dim = "cuda", case["page"], case["kv_heads"], case["dim"]
    new, kv = lengths(case)
    n = len(kv)
    # pages: a shared prefix (append), every sequence's own in shuffled order, and for an eviction the pages it moves to
    shared = SHARED // page if case["kind"] == "append" else 0
    each = [max(0, _pages(c, page) - shared) if c else 0 for c in kv]
    used = shared + sum(each)
    keep = min(case["budget"], max(kv)) if case["kind"] == "evict" else 0
    fresh = n * _pages(keep, page)
    cols = max(1, max(_pages(c, page) for c in kv))
    order = torch.randperm(used - shared, generator=g, device=dev).to(torch.int32) + shared
    table = torch.zeros((n, cols), dtype=torch.int32, device=dev)
    prefix = torch.arange(shared, dtype=torch.int32, device=dev)
    at = 0
    for s in range(n):
        if kv[s]:
            table[s, :shared] = prefix
            table[s, shared:shared + each[s]] = order[at:at + each[s]]
        at += each[s]
    kind = TYPES[case["cache"]]
    quant = case["cache"] == FP8
    scales = [torch.full((kvh,), 0.02, device=dev) * (1 + torch.rand(kvh, generator=g, device=dev)) if quant else None
              for _ in range(2)]

    def values(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.bfloat16)

    def pool():
        x = torch.empty((used + fresh, kvh, page, dim), dtype=kind, device=dev)
        step = max(1, (1 << 28) // (kvh * page * dim))
        for a in range(0, used, step):
            b = min(used, a + step)
            v = values(b - a, kvh, page, dim)
            x[a:b] = ((v.float() * 40).clamp(-E4M3_MAX, E4M3_MAX) if quant else v).to(kind)
        x.view(torch.uint8)[used:] = 0
        return x

    k, v = pool(), pool()
    off = [0]
    for m in new:
        off.append(off[-1] + m)
    state = dict(case=case, k=k, v=v, k_scale=scales[0], v_scale=scales[1], table=table, used=used, shared=shared,
                 kv_len=torch.tensor(kv, dtype=torch.int32, device=dev), kv=kv, max_kv=max(kv),
                 q_off=torch.tensor(off, dtype=torch.int32, device=dev), off=off, max_q=max(new))
    if case["kind"] == "append":
        # the key and value thirds of one fused projection's output
        qkv = values(off[-1], case["heads"] + 2 * kvh, dim).to(TYPES[case["type"]])
        state["k_new"] = qkv[:, case["heads"]:case["heads"] + kvh]
        state["v_new"] = qkv[:, case["heads"] + kvh:]
    elif case["kind"] == "attend":
        # a few dimensions that every query shares, so that some keys gather much of the weight
        lean = values(1, case["heads"], dim) * (torch.rand(1, case["heads"], dim, generator=g, device=dev) < 0.05)
        state["q"] = (values(off[-1], case["heads"], dim) + 3 * lean).to(TYPES[case["type"]])
        if case["weights"]:
            w = torch.rand(n, kvh, max(kv), generator=g, device=dev)
            state["weight"] = torch.where(torch.arange(max(kv), device=dev) < state["kv_len"][:, None, None], w * w, 0)
    else:
        # heavy-tailed, as accumulated attention is, with ties and with tokens nothing attended to
        w = torch.randn(n, kvh, max(kv), generator=g, device=dev).mul_(2).exp_()
        w = torch.where(torch.rand(w.shape, generator=g, device=dev) < 0.1, (w * 4).round() / 4, w)
        state["weight"] = torch.where(torch.arange(max(kv), device=dev) < state["kv_len"][:, None, None], w, 0)
        state["dst"] = (torch.randperm(fresh, generator=g, device=dev).to(torch.int32) + used).view(n, -1)
    return state


# --------------------------------------------------------------------- run

def run(state):
    kind = state["case"]["kind"]
    return {"append": _append, "attend": _attend, "evict": _evict}[kind](state)


def _cache(state):
    from paper_2609_28870_amd import pc
    return pc, pc.PagedCache(state["k"], state["v"], state["k_scale"], state["v_scale"])


def _values(x, scale):
    """What cache entries [page, head, slot, dim] stand for."""
    return x.float() if scale is None else x.float() * scale[:, None, None]


def _raw(x):
    """Bytes where torch has no indexing for the type."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _append(state):
    k, v = state["k"], state["v"]
    if own:
        pc, cache = _cache(state)
        pc.kv_append(cache, state["table"], state["kv_len"], state["q_off"], state["k_new"], state["v_new"])
    else:
        page = state["case"]["page"]
        q_off = state["q_off"].long()
        count = q_off[1:] - q_off[:-1]
        seq = torch.repeat_interleave(torch.arange(count.numel(), device=k.device), count, output_size=state["off"][-1])
        slot = state["kv_len"].long()[seq] - q_off[seq + 1] + torch.arange(seq.numel(), device=k.device)
        at = state["table"].long()[seq, slot // page], slice(None), slot % page
        _raw(k)[at] = _raw(_stored(state["k_new"], k.dtype, state["k_scale"]))
        _raw(v)[at] = _raw(_stored(state["v_new"], v.dtype, state["v_scale"]))
    # the shared prefix's pages are not written
    k, v = k[state["shared"]:], v[state["shared"]:]
    return (k, v) if state["k_scale"] is None else (_values(k, state["k_scale"]), _values(v, state["v_scale"]))


def _stored(x, dtype, scale):
    if scale is None:
        return x.to(dtype)
    return (x.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)


def _attend(state):
    case = state["case"]
    scale = case["dim"] ** -0.5
    if own:
        pc, cache = _cache(state)
        out, lse, weight = pc.attn_paged(state["q"], cache, state["table"], state["kv_len"], state["q_off"],
                                         state["max_q"], max_kv=state["max_kv"], scale=scale, causal=case["causal"],
                                         window=case["window"], want_lse=True, weight=state.get("weight"))[:3]
        return (out, lse) if weight is None else (out, lse, weight)
    q, dev = state["q"], state["q"].device
    n, cols = state["table"].shape
    m, heads, kvh, dim, page = state["max_q"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    group, length = heads // kvh, state["max_kv"]
    q_off, kv_len = state["q_off"].long(), state["kv_len"].long()
    count = q_off[1:] - q_off[:-1]
    # queries padded to [sequence, kv head, group x row, dim], keys and values to [sequence, kv head, slot, dim]
    row = torch.arange(m, device=dev)
    there = row < count[:, None]
    at = (q_off[:-1, None] + row).clamp(max=q.shape[0] - 1)
    qp = q.float()[at].view(n, m, kvh, group, dim).permute(0, 2, 3, 1, 4).reshape(n, kvh, group * m, dim)
    pages = state["table"].long()

    def flat(x, s):
        x = _raw(x)[pages].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[pages]
        x = x.permute(0, 2, 1, 3, 4).float() if s is None else x.permute(0, 2, 1, 3, 4).float() * s[:, None, None, None]
        return x.reshape(n, kvh, cols * page, dim)[:, :, :length]

    scores = torch.matmul(qp * scale, flat(state["k"], state["k_scale"]).transpose(-1, -2))
    slot = torch.arange(length, device=dev)
    pos = (kv_len - count)[:, None] + row                                        # [sequence, row]
    seen = (slot < kv_len[:, None, None]) & there[:, :, None]
    if case["causal"]:
        seen &= slot <= pos[:, :, None]
    if case["window"]:
        seen &= slot > pos[:, :, None] - case["window"]
    scores = scores.view(n, kvh, group, m, length)
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    lse = top + total.log()
    scores.div_(total.clamp(min=1e-38))
    out = torch.matmul(scores.view(n, kvh, group * m, length), flat(state["v"], state["v_scale"]))
    rows = there.nonzero(as_tuple=True)
    out = out.view(n, kvh, group, m, dim).permute(0, 3, 1, 2, 4)[rows].reshape(-1, heads, dim).to(q.dtype)
    lse = lse.view(n, kvh, group, m).permute(0, 3, 1, 2)[rows].reshape(-1, heads)
    if "weight" not in state:
        return out, lse
    return out, lse, state["weight"] + scores.sum((2, 3))


def _evict(state):
    case = state["case"]
    k, v, weight = state["k"], state["v"], state["weight"]
    budget, recent, page, used = case["budget"], case["recent"], case["page"], state["used"]
    budget = min(budget, state["max_kv"])
    if own:
        pc, cache = _cache(state)
        r = pc.kv_evict(cache, state["table"], state["kv_len"], weight, budget, recent, dst_table=state["dst"],
                        max_kv=state["max_kv"])
        return r["new_len"], r["kept"], r["weight"], k[used:], v[used:]
    dev = k.device
    n, kvh, length = weight.shape
    kv_len = state["kv_len"].long()[:, None, None]
    slot = torch.arange(length, device=dev)
    new_len = kv_len.clamp(max=budget)
    by_weight = weight.sort(dim=-1, descending=True, stable=True).indices
    late = (by_weight < kv_len - recent).to(torch.uint8) + 2 * (by_weight >= kv_len).to(torch.uint8)
    first = by_weight.gather(-1, late.sort(dim=-1, stable=True).indices)[..., :budget]
    place = torch.arange(budget, device=dev)
    kept = torch.where(place < new_len, first, length).sort(-1).values          # unused places last
    real = (place < new_len).expand(n, kvh, budget)
    s, h, r = real.nonzero(as_tuple=True)
    j = kept[s, h, r]
    src, dst = state["table"].long()[s, j // page], state["dst"].long()[s, r // page]
    for x in (_raw(k), _raw(v)):
        x[dst, h, r % page] = x[src, h, j % page]
    moved = torch.where(real, weight.gather(-1, kept.clamp(max=length - 1)), 0)
    return new_len.view(n).to(torch.int32), torch.where(real, kept, -1).to(torch.int32), moved, k[used:], v[used:]


# -------------------------------------------------------------------- work

def _pairs(case, new, kv):
    """Visible (row, key) pairs and keys that any row sees, of one sequence."""
    j0, window = kv - new, case["window"]
    hi = (lambda i: j0 + i + 1) if case["causal"] else (lambda i: kv)
    lo = (lambda i: max(0, j0 + i - window + 1)) if window else (lambda i: 0)
    pairs = sum(max(0, hi(i) - lo(i)) for i in range(new))
    return pairs, (hi(new - 1) - lo(0) if new else 0)


def work(case):
    new, kv = lengths(case)
    kvh, dim, size = case["kv_heads"], case["dim"], SIZE[case["cache"]]
    if case["kind"] == "append":
        return {"bytes": 2 * sum(new) * kvh * dim * (2 + size), "flops": 0}
    if case["kind"] == "evict":
        kept = sum(min(c, case["budget"]) for c in kv)
        return {"bytes": kvh * (4 * sum(kv) + 8 * kept + 4 * kept * dim * size), "flops": 0}
    pairs = keys = 0
    for m, c in zip(new, kv):
        a, b = _pairs(case, m, c)
        pairs, keys = pairs + a, keys + b
    moved = 2 * keys * kvh * dim * size + sum(new) * case["heads"] * (4 * dim + 4)
    if case["weights"]:
        moved += 8 * sum(kv) * kvh
    return {"bytes": moved, "flops": 4 * pairs * case["heads"] * dim}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    if case["kind"] == "evict":
        return None           # nothing is computed: indexes and moved values
    state = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(state)
    return _exact_attend(state)


def _exact_append(state):
    case, page = state["case"], state["case"]["page"]
    out = []
    for name in ("k", "v"):
        x, scale = state[name][state["shared"]:].double(), state[name + "_scale"]
        rows = state[name + "_new"].double()
        if scale is not None:
            rows = _nearest_e4m3(rows / scale.double()[:, None])
        for s, c in enumerate(state["kv"]):
            a, b = state["off"][s], state["off"][s + 1]
            for p in range((c - (b - a)) // page, (c + page - 1) // page) if b > a else ():
                lo, hi = max(p * page, c - (b - a)), min((p + 1) * page, c)
                at = int(state["table"][s, p]) - state["shared"]
                x[at, :, lo - p * page:hi - p * page] = rows[a + lo - (c - (b - a)):a + hi - (c - (b - a))].transpose(0, 1)
        out.append(x if scale is None else x * scale.double()[:, None, None])
    return tuple(out)


def _nearest_e4m3(x):
    """Values rounded to the grid of 8-bit floats with 4 exponent and 3 fraction bits, ties to even."""
    a = x.abs().clamp(max=E4M3_MAX)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign((a / step).round() * step, x)


def _exact_attend(state):
    case = state["case"]
    heads, kvh, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    group = heads // kvh
    q = state["q"].double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    weight = state["weight"].double() if "weight" in state else None
    for s, c in enumerate(state["kv"]):
        a, b = state["off"][s], state["off"][s + 1]
        if a == b:
            continue
        ids = state["table"][s, :_pages(c, page)].long()
        j = torch.arange(c, device=q.device)
        pos = c - (b - a) + torch.arange(b - a, device=q.device)
        hide = (j > pos[:, None]) if case["causal"] else torch.zeros((b - a, c), dtype=torch.bool, device=q.device)
        if case["window"]:
            hide = hide | (j <= pos[:, None] - case["window"])
        for h in range(kvh):
            keys, vals = (_raw(state[x])[ids, h].view(state[x].dtype).reshape(-1, dim)[:c].double() for x in "kv")
            if state["k_scale"] is not None:
                keys, vals = keys * state["k_scale"][h].double(), vals * state["v_scale"][h].double()
            for e in range(h * group, (h + 1) * group):
                z = (q[a:b, e] @ keys.T / math.sqrt(dim)).masked_fill(hide, -math.inf)
                lse[a:b, e] = torch.logsumexp(z, -1)
                p = torch.exp(z - lse[a:b, e, None])
                out[a:b, e] = p @ vals
                if weight is not None:
                    weight[s, h, :c] += p.sum(0)
    return (out, lse) if weight is None else (out, lse, weight)
