"""Workloads for the position rotation and for a cache in 4 bits: tables of angles,
rows turned by them (and turned back, as a gradient is), new tokens written into the
paged cache with the rotation applied on the way, and attention over a cache whose
keys and values are 4-bit codes with a power-of-two scale for every 32 of them.

``run`` makes the calls of ``paper_2609_28870_amd.pc`` where ``own`` is true, and
computes the same in elementary torch operations where it is not: in 32 bits, and in
64 the angles, and what lies next to a border between two codes.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F16, FP8, FP4 = "bf16", "f16", "fp8", "fp4"
TYPES = {BF16: torch.bfloat16, F16: torch.float16, FP8: torch.float8_e4m3fn}
BITS = {BF16: 16, F16: 16, FP8: 8, FP4: 4.25}
SHARED = 2048            # tokens of a system prompt that sequences share
E4M3_MAX = 448.0
BASE = 10000.0
PLAIN_SCORES = 2.5e9     # most (row, key) pairs that the plain form holds at once
LARGEST = {BF16: 252, F16: 140}     # bounds of a scale's exponent byte, by the new tokens' type
SMALLEST = {BF16: 1, F16: 104}


def listed():
    usual = dict(heads=32, kv_heads=4, dim=128)
    return [
        # the queries of one decode step: latency alone
        dict(name="rope_step", kind="rope", rows=64, heads=32, dim=128, rot=128, interleaved=False, transpose=False, type=BF16),
        # the queries of a scheduler step's prefill chunks, inside the fused projection's output
        dict(name="rope_chunks", kind="rope", rows=16384, heads=32, dim=128, rot=128, interleaved=False, transpose=False, type=BF16),
        # the gradient of queries whose heads are turned in part, neighbours paired, an odd number of rows
        dict(name="rope_back_part", kind="rope", rows=8191, heads=20, dim=96, rot=64, interleaved=True, transpose=True, type=F16),
        # the angles up to a context cap, stretched for a context longer than the one that was trained
        dict(name="table_long", kind="table", positions=131072, rot=128, scaling="ramp", factor=16.0),
        # the new token of every running sequence, its queries turned in the same call
        dict(name="append_step", kind="append", seqs=256, new=1, tail=96, mixed=True, page=16, cache=BF16, type=BF16,
             rot=128, interleaved=False, given=False, **usual),
        # the new token of sequences that were cut to a budget: positions are not slots any more
        dict(name="append_step_fp4", kind="append", seqs=48, new=1, tail=30, mixed=True, page=64, cache=FP4, type=BF16,
             rot=128, interleaved=False, given=True, **usual),
        # ragged prefill chunks into an 8-bit cache, half of every head turned, neighbours paired
        dict(name="append_chunks_fp8", kind="append", seqs=24, new=1024, tail=0, mixed=True, page=64, cache=FP8, type=F16,
             rot=64, interleaved=True, given=True, **usual),
        # ragged prefill chunks into a 4-bit cache
        dict(name="append_chunks_fp4", kind="append", seqs=24, new=1024, tail=0, mixed=True, page=16, cache=FP4, type=BF16,
             rot=128, interleaved=False, given=False, **usual),
        # one user, one token over a 4-bit cache: latency alone
        dict(name="decode_one_fp4", kind="attend", seqs=1, new=1, kv=1537, mixed=False, page=16, type=BF16, window=0,
             causal=True, weights=False, **usual),
        # the decode step of a batch of chat sessions
        dict(name="decode_batch_fp4", kind="attend", seqs=64, new=1, kv=32768, mixed=True, page=16, type=BF16, window=0,
             causal=True, weights=False, **usual),
        # the missed suffix of a long agent turn over its cached prefix
        dict(name="chunk_long_fp4", kind="attend", seqs=1, new=2048, kv=32768, mixed=False, page=64, type=BF16, window=0,
             causal=True, weights=False, **usual),
        # drafted tokens, a group of seven heads, a window, and the weights that an eviction ranks by
        dict(name="drafted_weights_fp4", kind="attend", seqs=32, new=3, kv=16384, mixed=True, page=24, type=F16, window=6000,
             causal=True, weights=True, heads=28, kv_heads=4, dim=128),
    ]


HEADS = [(32, 4, 128), (28, 4, 128), (16, 16, 64), (8, 1, 256), (64, 8, 128), (20, 4, 96), (9, 3, 64), (12, 12, 32)]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    bytes_most = max(work(c)["bytes"] for c in listed())
    flops_most = max(work(c)["flops"] for c in listed())
    while True:
        heads, kv_heads, dim = rng.choice(HEADS)
        kind = rng.choice(["rope", "rope", "table", "append", "append", "append", "attend", "attend", "attend", "attend"])
        t, rot = rng.choice([BF16, BF16, F16]), rng.choice([dim, dim, dim // 2, dim // 4])
        case = dict(kind=kind)
        if kind == "table":
            case.update(positions=log_int(16, 131072), rot=rot, scaling=rng.choice(["none", "linear", "base", "ramp"]),
                        factor=rng.uniform(1, 32))
        elif kind == "rope":
            case.update(rows=log_int(1, 20000), heads=heads, dim=dim, rot=rot, interleaved=rng.random() < 0.5,
                        transpose=rng.random() < 0.3, type=t)
        else:
            case.update(heads=heads, kv_heads=kv_heads, dim=dim, type=t, page=rng.choice([16, 16, 64, 256, 24, 10]),
                        seqs=log_int(1, 96), mixed=rng.random() < 0.7)
            if kind == "append":
                case.update(cache=rng.choice([t, FP8, FP4, FP4]), new=rng.choice([1, log_int(2, 4096)]), tail=log_int(1, 500),
                            rot=rot, interleaved=rng.random() < 0.5, given=rng.random() < 0.5)
            else:
                case.update(new=rng.choice([1, rng.randint(2, 9), log_int(10, 4096)]), kv=log_int(16, 131072),
                            window=rng.choice([0, 0, 0, log_int(16, 8192)]), causal=rng.random() < 0.85,
                            weights=rng.random() < 0.3)
                case["new"] = min(case["new"], case["kv"])
        w = work(case)
        if w["bytes"] > bytes_most or w["flops"] > flops_most:
            continue
        if kind in ("append", "attend"):
            new, kv = lengths(case)
            if not sum(kv) or len(kv) * max(kv) * kv_heads * dim * 8 > 20e9:
                continue
            if kind == "append" and sum(kv) * kv_heads * dim > 2e8:
                continue
            if kind == "attend" and len(kv) * max(new) * heads * max(kv) > PLAIN_SCORES:
                continue
        return case


# ------------------------------------------------------------------ inputs

def lengths(case):
    """New tokens and cache length (new ones included) of every sequence: the largest first, the others spread over six
    octaves where the batch is mixed, an idle one (no tokens) among many."""
    r = random.Random("%s %s %s" % (case["kind"], case["seqs"], case.get("kv", case.get("new"))))
    n = case["seqs"]
    spread = [1.0] + [2.0 ** -r.uniform(0, 6) if case["mixed"] else 1.0 for _ in range(n - 1)]
    share = [1.0] + [r.uniform(0.02, 1) if case["mixed"] else 1.0 for _ in range(n - 1)]
    if case["kind"] == "append":
        new = [max(1, round(case["new"] * f)) for f in share]
        kv = [SHARED + case["tail"] + m for m in new]
    else:
        kv = [max(1, round(case["kv"] * f)) for f in spread]
        new = [min(max(1, round(case["new"] * f)), c) for f, c in zip(share, kv)]
    if case["mixed"] and n >= 16:
        new[n // 2] = kv[n // 2] = 0
    return new, kv


def _pages(tokens, page):
    return (tokens + page - 1) // page


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _angles(positions, rot):
    """A program's table of cosines and sines, made once: float32 [positions, rot / 2, 2]."""
    freq = BASE ** (torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / -rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([a.cos(), a.sin()], -1).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def values(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)

    if case["kind"] == "table":
        # another seed, another base: the frequencies are the inputs
        base = BASE * (1 + 0.01 * (seed % 1000))
        return dict(case=case, base=base, trained=max(2, int(case["positions"] / case["factor"])))
    if case["kind"] == "rope":
        rows, heads, dim = case["rows"], case["heads"], case["dim"]
        # sequences of the step restart their positions
        pos = torch.arange(rows, device="cuda") % 5000 + torch.randint(0, 3000, (1,), generator=g, device="cuda")
        return dict(case=case, x=values(rows, heads + 8, dim).to(TYPES[case["type"]])[:, :heads], pos=pos.to(torch.int32),
                    table=_angles(8192, case["rot"]))
    page, kvh, dim, append = case["page"], case["kv_heads"], case["dim"], case["kind"] == "append"
    new, kv = lengths(case)
    n, cache = len(kv), case.get("cache", FP4)
    # pages: a shared prefix (append), every sequence's own in shuffled order
    shared = SHARED // page if append else 0
    each = [max(0, _pages(c, page) - shared) if c else 0 for c in kv]
    used = shared + sum(each)
    cols = max(1, max(_pages(c, page) for c in kv))
    order = (torch.randperm(used - shared, generator=g, device="cuda") + shared).tolist()
    rows, at = [], 0
    for s in range(n):
        mine = list(range(shared)) + order[at:at + each[s]] if kv[s] else []
        rows.append(mine + [0] * (cols - len(mine)))
        at += each[s]
    off = [0]
    for m in new:
        off.append(off[-1] + m)
    state = dict(case=case, table=_i32(rows), kv_len=_i32(kv), kv=kv, max_kv=max(kv), q_off=_i32(off), off=off, max_q=max(new),
                 shared=shared, k_scale=None, v_scale=None)
    for name in "kv":
        x = torch.empty((used, kvh, page, dim // 2 if cache == FP4 else dim),
                        dtype=torch.uint8 if cache == FP4 else TYPES[cache], device="cuda")
        scale = None
        if cache == FP8:
            scale = torch.full((kvh,), 0.02, device="cuda") * (1 + torch.rand(kvh, generator=g, device="cuda"))
        elif cache == FP4:
            scale = torch.empty((used, kvh, page, dim // 32), dtype=torch.uint8, device="cuda")
        # heads' dimensions differ in size, as those of keys do
        size = (torch.randn(kvh, 1, dim, generator=g, device="cuda") * 0.7).exp()
        step = max(1, (1 << 26) // (kvh * page * dim))
        for a in range(0, used, step):
            y = values(min(used, a + step) - a, kvh, page, dim).float() * size
            if cache == FP4:
                x[a:a + step], scale[a:a + step] = _to_fp4(y, case["type"])
            else:
                x[a:a + step] = (y * 40).clamp(-E4M3_MAX, E4M3_MAX).to(x.dtype) if cache == FP8 else y.to(x.dtype)
        state[name], state[name + "_scale"] = x, scale
    if append:
        # queries, keys and values of one fused projection's output
        qkv = values(off[-1], case["heads"] + 2 * kvh, dim).to(TYPES[case["type"]])
        state["q"], state["k_new"], state["v_new"] = qkv.split([case["heads"], kvh, kvh], 1)
        if case["given"]:
            # sequences that were cut: every one's text is ahead of its slots by what it lost
            ahead = torch.randint(0, 9000, (n,), generator=g, device="cuda").tolist()
            pos = [c - m + i + ahead[s] for s, (c, m) in enumerate(zip(kv, new)) for i in range(m)]
            state["pos"] = _i32(pos)
        state["angles"] = _angles(16384, case["rot"])
    else:
        # a few dimensions that every query shares, so that some keys gather much of the weight
        lean = values(1, case["heads"], dim) * (torch.rand(1, case["heads"], dim, generator=g, device="cuda") < 0.05)
        state["q"] = (values(off[-1], case["heads"], dim) + 3 * lean).to(TYPES[case["type"]])
        if case["weights"]:
            w = torch.rand(n, kvh, max(kv), generator=g, device="cuda")
            state["weight"] = torch.where(torch.arange(max(kv), device="cuda") < state["kv_len"][:, None, None], w * w, 0)
    return state


# --------------------------------------------------------------------- run

def run(state):
    kind = state["case"]["kind"]
    return {"table": _table, "rope": _rope, "append": _append, "attend": _attend}[kind](state)


def _table(state):
    case = state["case"]
    rot, s, n = case["rot"], case["factor"], case["positions"]
    if own:
        from paper_2609_28870_amd import pc
        freq = pc.rope_frequencies(rot, base=state["base"], scaling=case["scaling"], factor=s, trained=state["trained"],
                                   slow=1.0, fast=32.0)
        return pc.rope_table(freq, n)
    base = state["base"] * s ** (rot / (rot - 2)) if case["scaling"] == "base" and rot > 2 else state["base"]
    freq = base ** (torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / -rot)
    if case["scaling"] == "linear":
        freq = freq / s
    elif case["scaling"] == "ramp":
        keep = ((state["trained"] * freq / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        freq = (1 - keep) * freq / s + keep * freq
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([a.cos(), a.sin()], -1).float()


def _turn(x, table, pos, interleaved, transpose=False):
    """Rows x [row, head, dim] turned by their positions' angles, in x's type."""
    c, s = table[pos].to(x.dtype).unsqueeze(1).unbind(-1)                # [row, 1, rot / 2]
    if transpose:
        s = -s
    half = c.shape[-1]
    y = x.clone()
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., first], x[..., second]
    y[..., first] = a * c - b * s
    y[..., second] = b * c + a * s
    return y


def _rope(state):
    case, x = state["case"], state["x"]
    if own:
        from paper_2609_28870_amd import pc
        return pc.rope(x, state["table"], state["pos"], interleaved=case["interleaved"], transpose=case["transpose"])[0]
    return _turn(x.float(), state["table"], state["pos"].long(), case["interleaved"], case["transpose"]).to(x.dtype)


def _cache(state):
    from paper_2609_28870_amd import pc
    k, v = state["k"], state["v"]
    if k.dtype == torch.uint8:
        k, v = k.view(torch.float4_e2m1fn_x2), v.view(torch.float4_e2m1fn_x2)
    return pc, pc.PagedCache(k, v, state["k_scale"], state["v_scale"])


def _to_fp4(y, kind):
    """Float values [..., dim] as 4-bit codes, two a byte, and the exponent bytes of the scales of 32 of them.  The scale is
    the power of two that leaves the largest below 7, so that the codes' largest, 6, is at most half a step off."""
    y = y.view(*y.shape[:-1], -1, 32)
    top = y.abs().amax(-1)
    e = (((top.view(torch.int32) + 0x200000) >> 23) - 2).clamp(SMALLEST[kind], LARGEST[kind])
    a = y.abs() / (e << 23).view(torch.float32)[..., None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) | (
        (y < 0).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., ::2] | code[..., 1::2] << 4, e.to(torch.uint8)


def _of_fp4(codes, scale, dtype):
    """The values that codes [..., dim / 2] and exponent bytes [..., dim / 32] stand for."""
    one = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device=codes.device)
    one = torch.cat([one, -one])
    two = torch.stack([one.repeat(16), one.repeat_interleave(16)], -1)   # of a byte, the low half first
    x = two[codes.int()].flatten(-2)
    s = (scale.int() << 23).view(torch.float32).to(dtype)
    return (x.view(*s.shape, 32) * s[..., None]).flatten(-2)


def _values(x, scale, dtype=torch.float32):
    """What cache entries [page, head, slot, dim] stand for."""
    if x.dtype == torch.uint8:
        return _of_fp4(x, scale, dtype)
    return x.float() if scale is None else x.float() * scale[:, None, None]


def _append(state):
    case, k, v, q = state["case"], state["k"], state["v"], state["q"]
    if own:
        pc, cache = _cache(state)
        q = pc.kv_append_rope(cache, state["table"], state["kv_len"], state["q_off"], state["k_new"], state["v_new"],
                              state["angles"], pos=state.get("pos"), interleaved=case["interleaved"], q=q)[0]
    else:
        page, q_off = case["page"], state["q_off"].long()
        count = q_off[1:] - q_off[:-1]
        seq = torch.repeat_interleave(torch.arange(count.numel(), device=k.device), count, output_size=state["off"][-1])
        slot = state["kv_len"].long()[seq] - q_off[seq + 1] + torch.arange(seq.numel(), device=k.device)
        pos = state["pos"].long() if "pos" in state else slot
        at = state["table"].long()[seq, slot // page], slice(None), slot % page
        q = _turn(q.float(), state["angles"], pos, case["interleaved"]).to(q.dtype)
        # turned in 64 bits where a code's border may be next to the value
        wide = torch.float32 if case["cache"] in (BF16, F16) else torch.float64
        new = {"k": _turn(state["k_new"].to(wide), state["angles"], pos, case["interleaved"]).float(),
               "v": state["v_new"].float()}
        for name, x in (("k", k), ("v", v)):
            scale = state[name + "_scale"]
            if case["cache"] == FP4:
                x[at], scale[at] = _to_fp4(new[name], case["type"])
            elif case["cache"] == FP8:
                x.view(torch.uint8)[at] = (new[name] / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(x.dtype).view(torch.uint8)
            else:
                x[at] = new[name].to(x.dtype)
    a = state["shared"]     # the shared prefix's pages are not written
    if case["cache"] in (BF16, F16):
        return q, k[a:], v[a:]
    if case["cache"] == FP8:
        return q, _values(k[a:], state["k_scale"]), _values(v[a:], state["v_scale"])
    return (q, _values(k[a:], state["k_scale"][a:], torch.bfloat16), _values(v[a:], state["v_scale"][a:], torch.bfloat16))


def _attend(state):
    case = state["case"]
    scale = case["dim"] ** -0.5
    if own:
        pc, cache = _cache(state)
        out, lse, weight = pc.attn_paged(state["q"], cache, state["table"], state["kv_len"], state["q_off"], state["max_q"],
                                         max_kv=state["max_kv"], scale=scale, causal=case["causal"], window=case["window"],
                                         want_lse=True, weight=state.get("weight"))[:3]
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

    def flat(name):
        x = _of_fp4(state[name][pages], state[name + "_scale"][pages], torch.float32)
        return x.permute(0, 2, 1, 3, 4).reshape(n, kvh, cols * page, dim)[:, :, :length]

    scores = torch.matmul(qp * scale, flat("k").transpose(-1, -2).contiguous())
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
    out = torch.matmul(scores.view(n, kvh, group * m, length), flat("v"))
    rows = there.nonzero(as_tuple=True)
    out = out.view(n, kvh, group, m, dim).permute(0, 3, 1, 2, 4)[rows].reshape(-1, heads, dim).to(q.dtype)
    lse = lse.view(n, kvh, group, m).permute(0, 3, 1, 2)[rows].reshape(-1, heads)
    if "weight" not in state:
        return out, lse
    return out, lse, state["weight"] + scores.sum((2, 3))


# -------------------------------------------------------------------- work

def _pairs(case, new, kv):
    """Visible (row, key) pairs and keys that any row sees, of one sequence."""
    j0, window = kv - new, case["window"]
    hi = (lambda i: j0 + i + 1) if case["causal"] else (lambda i: kv)
    lo = (lambda i: max(0, j0 + i - window + 1)) if window else (lambda i: 0)
    pairs = sum(max(0, hi(i) - lo(i)) for i in range(new))
    return pairs, (hi(new - 1) - lo(0) if new else 0)


def work(case):
    if case["kind"] == "table":
        pairs = case["positions"] * (case["rot"] // 2)
        return {"bytes": 8 * pairs, "flops": 3 * pairs}
    if case["kind"] == "rope":
        rows, heads = case["rows"], case["heads"]
        return {"bytes": rows * (4 * heads * case["dim"] + 4) + 4 * case["rot"] * min(rows, 5000),
                "flops": 3 * rows * heads * case["rot"]}
    new, kv = lengths(case)
    kvh, dim = case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        a_token = 4 * case["heads"] * dim + 2 * kvh * dim * (2 + BITS[case["cache"]] / 8) + 4 * case["rot"]
        return {"bytes": int(sum(new) * a_token), "flops": 3 * sum(new) * (case["heads"] + kvh) * case["rot"]}
    pairs = keys = 0
    for m, c in zip(new, kv):
        a, b = _pairs(case, m, c)
        pairs, keys = pairs + a, keys + b
    moved = int(2 * keys * kvh * dim * BITS[FP4] / 8) + sum(new) * case["heads"] * (4 * dim + 4)
    if case["weights"]:
        moved += 8 * sum(kv) * kvh
    return {"bytes": moved, "flops": 4 * pairs * case["heads"] * dim}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    state = prepare(case, seed)
    return {"table": _exact_table, "rope": _exact_rope, "append": _exact_append, "attend": _exact_attend}[case["kind"]](state)


def _exact_table(state):
    case = state["case"]
    rot, s = case["rot"], case["factor"]
    f = np.empty(rot // 2)
    for i in range(rot // 2):
        base = state["base"]
        if case["scaling"] == "base" and rot > 2:
            base *= s ** (rot / (rot - 2))
        f[i] = math.exp(-2 * i / rot * math.log(base))
        if case["scaling"] == "linear":
            f[i] /= s
        elif case["scaling"] == "ramp":
            turns = state["trained"] / (2 * math.pi / f[i])
            keep = min(1.0, max(0.0, (turns - 1) / (32 - 1)))
            f[i] *= keep + (1 - keep) / s
    z = np.exp(1j * np.multiply.outer(np.arange(case["positions"], dtype=np.float64), f))
    return torch.from_numpy(z.view(np.float64).reshape(*z.shape, 2)).cuda()


def _exact_turn(x, table, pos, rot, interleaved, transpose=False):
    """As complex numbers times another."""
    x, turn = x.double(), torch.view_as_complex(table.double().contiguous())[pos.long()][:, None]
    if transpose:
        turn = turn.conj()
    head, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(head[..., :rot // 2], head[..., rot // 2:]) * turn
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, rest], -1)


def _exact_rope(state):
    case = state["case"]
    return _exact_turn(state["x"], state["table"], state["pos"], case["rot"], case["interleaved"], case["transpose"])


def _nearest(x, grid):
    """Rounded to a grid of magnitudes (in the order of their codes), ties to the even code."""
    grid = torch.tensor(grid, dtype=torch.float64, device=x.device)
    a = x.abs().clamp(max=grid[-1])
    i = torch.searchsorted(grid, a).clamp(1, len(grid) - 1)
    lo, hi = grid[i - 1], grid[i]
    up = (hi - a < a - lo) | ((hi - a == a - lo) & (i % 2 == 0))
    return torch.copysign(torch.where(up, hi, lo), x)


def _exact_stored(rows, case, scale):
    """What a cache of the case's type holds of rows [row, head, dim]."""
    if case["cache"] == FP8:
        grid = [f * 2.0 ** -9 for f in range(8)] + [(8 + f) * 2.0 ** (e - 9) for e in range(15) for f in range(8)]
        # the rotated value and its quotient are numbers of 32 bits, by definition
        return _nearest((rows.float() / scale[:, None]).double(), grid[:grid.index(E4M3_MAX) + 1]) * scale.double()[:, None]
    if case["cache"] == FP4:
        y = rows.float().double().reshape(*rows.shape[:-1], -1, 32)
        top = y.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(top.clamp(min=1e-300))) - 2
        e = torch.where(top >= 7 * torch.exp2(e), e + 1, e).clamp(SMALLEST[case["type"]] - 127, LARGEST[case["type"]] - 127)
        return (_nearest(y / torch.exp2(e), [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]) * torch.exp2(e)).flatten(-2)
    return rows


def _exact_append(state):
    case, page = state["case"], state["case"]["page"]
    rows = torch.arange(state["off"][-1], device="cuda")
    first = torch.tensor([c - b for c, b in zip(state["kv"], state["off"][1:])], device="cuda")
    seq = torch.bucketize(rows, torch.tensor(state["off"][1:], device="cuda"), right=True)
    pos = state.get("pos", rows + first[seq])
    turned = _exact_turn(state["k_new"], state["angles"], pos, case["rot"], case["interleaved"])
    out = [_exact_turn(state["q"], state["angles"], pos, case["rot"], case["interleaved"])]
    for name, new in (("k", turned), ("v", state["v_new"].double())):
        scale, a = state[name + "_scale"], state["shared"]
        if case["cache"] == FP4:
            x = _of_fp4(state[name][a:], scale[a:], torch.float64)
        else:
            x = state[name][a:].double()
            if case["cache"] == FP8:
                x = x * scale.double()[:, None, None]
        new = _exact_stored(new, case, scale)
        for s, c in enumerate(state["kv"]):
            lo, hi = state["off"][s], state["off"][s + 1]
            for p in range((c - (hi - lo)) // page, _pages(c, page)) if hi > lo else ():
                j0, j1 = max(p * page, c - (hi - lo)), min((p + 1) * page, c)
                at = int(state["table"][s, p]) - a
                x[at, :, j0 - p * page:j1 - p * page] = new[hi - c + j0:hi - c + j1].transpose(0, 1)
        out.append(x)
    return tuple(out)


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
            keys, vals = (_of_fp4(state[x][ids, h], state[x + "_scale"][ids, h], torch.float64).reshape(-1, dim)[:c] for x in "kv")
            for e in range(h * group, (h + 1) * group):
                z = (q[a:b, e] @ keys.T / math.sqrt(dim)).masked_fill(hide, -math.inf)
                lse[a:b, e] = torch.logsumexp(z, -1)
                p = torch.exp(z - lse[a:b, e, None])
                out[a:b, e] = p @ vals
                if weight is not None:
                    weight[s, h, :c] += p.sum(0)
    return (out, lse) if weight is None else (out, lse, weight)
