"""Decode over selected blocks of the paged cache, with lengths that stay on the GPU: its operators as measurable cases.

A serving loop whose sequences grow on the GPU makes five calls for each layer's attention half:

  extend   block tables, slots and positions of the new tokens, from the sequences' lengths and a list of free blocks
  append   norms of the query and key heads, rotation, and the append of K and V to the paged cache
  bounds   for each block the largest and smallest key in every channel, in 8 bits
  select   for each sequence and kv-head the blocks whose bounds promise the largest scores
  attend   attention of one token per row over the selected blocks

  listed()             the cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  what the program holds before the call
  run(state)           one call and its outputs: in plain torch, or (own) through the library
  exact(case, seed)    the computed numbers from float64
  work(case)           bytes and operations the call cannot do without
"""
import math
import random

import torch

own = False

BK = 16  # tokens per block
MAX_POSITION = 1 << 17
# query heads, kv-heads, head size, theta, norms of query and key heads, eps, bf16
SHAPES = {
    "tiny": (4, 4, 64, 1e4, False, 1e-5, False),
    "llama8b": (32, 8, 128, 5e5, False, 1e-5, True),
    "qwen32b": (64, 8, 128, 1e6, True, 1e-6, True),
}


def listed():
    return [
        # A token step of a multi-agent server: 64 conversations, one new token each, one to eight agents answering.
        dict(name="extend_step", kind="extend", seqs=64, ctx_lo=1024, ctx_hi=16384, new_lo=1, new_hi=1, act_lo=1, act_hi=8, free=1.0),
        # A round of admissions: 256 conversations append prompts and observations of up to 500 tokens; the last ones find no block.
        dict(name="extend_admit", kind="extend", seqs=256, ctx_lo=0, ctx_hi=8192, new_lo=0, new_hi=500, act_lo=0, act_hi=0, free=0.9),
        # The same token step in a layer: 64 new tokens among the agents' rows.
        dict(name="append_step", kind="append", shape="llama8b", kv="same", seqs=64, ctx_lo=1024, ctx_hi=16384, new_lo=1, new_hi=1, act_lo=1, act_hi=8),
        # Four agents append an observation of 60-400 tokens each; norms of the heads, cache in FP8.
        dict(name="append_turn_fp8", kind="append", shape="qwen32b", kv="fp8", seqs=4, ctx_lo=600, ctx_hi=8192, new_lo=60, new_hi=400, act_lo=0, act_hi=0),
        # Chunked prefill of a full server.
        dict(name="append_prompt", kind="append", shape="llama8b", kv="same", seqs=32, ctx_lo=8192, ctx_hi=8192, new_lo=512, new_hi=512, act_lo=0, act_hi=0),
        # The smallest layer: one sequence in float32, one new token.
        dict(name="bounds_tiny_fp32", kind="bounds", shape="tiny", kv="same", seqs=1, ctx_lo=127, ctx_hi=127, new_lo=1, new_hi=1),
        # Whole prefixes whose keys have no bounds yet: 32 conversations of 8192 tokens.
        dict(name="bounds_prefix", kind="bounds", shape="llama8b", kv="same", seqs=32, ctx_lo=0, ctx_hi=0, new_lo=8192, new_hi=8192),
        # One long conversation, all eight agents answering: interactive latency.
        dict(name="select_one", kind="select", shape="qwen32b", seqs=1, ctx_lo=32768, ctx_hi=32768, act_lo=8, act_hi=8, top=128),
        # The mixed batch.
        dict(name="select_batch", kind="select", shape="llama8b", seqs=64, ctx_lo=1024, ctx_hi=16384, act_lo=1, act_hi=8, top=64),
        # One long conversation again.
        dict(name="attend_one", kind="attend", shape="llama8b", kv="same", seqs=1, ctx_lo=32768, ctx_hi=32768, act_lo=8, act_hi=8, top=128),
        # The mixed batch.
        dict(name="attend_batch", kind="attend", shape="llama8b", kv="same", seqs=64, ctx_lo=1024, ctx_hi=16384, act_lo=1, act_hi=8, top=64),
        # Long contexts on the larger model, all agents, cache in FP8, an eighth of the blocks.
        dict(name="attend_long_fp8", kind="attend", shape="qwen32b", kv="fp8", seqs=16, ctx_lo=32768, ctx_hi=32768, act_lo=8, act_hi=8, top=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["extend", "append", "append", "bounds", "select", "select", "attend", "attend", "attend"])
    shape = rng.choice(["llama8b", "llama8b", "qwen32b", "tiny"])
    kv = rng.choice(["same", "same", "fp8"])
    if kind in ("extend", "append"):
        seqs = _log_int(rng, 1, 300)
        act = rng.randint(0, 8)
        if rng.random() < 0.5:  # token steps
            lo, hi = 1, 1
        else:
            hi = _log_int(rng, 2, max(2, 16000 // seqs))
            lo, act = max(0 if seqs >= 32 else 1, int(hi * rng.uniform(0, 1))), 0
        ctx = rng.choice([0, _log_int(rng, 16, 30000)])
        if kind == "append":
            ctx = min(ctx, 60000 // seqs)
        c = dict(kind=kind, seqs=seqs, ctx_lo=int(ctx * rng.uniform(0.1, 1)), ctx_hi=ctx, new_lo=lo, new_hi=hi, act_lo=rng.randint(0, act), act_hi=act)
        if kind == "extend":
            c["free"] = rng.choice([1.0, round(rng.uniform(0.3, 1.2), 3)])
        else:
            c.update(shape=shape, kv=kv)
        return c
    if kind == "bounds":
        seqs = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 200000 // seqs)
        return dict(kind=kind, shape=shape, kv=kv, seqs=seqs, ctx_lo=0, ctx_hi=rng.choice([0, _log_int(rng, 16, 2000)]), new_lo=max(1, hi // 2), new_hi=hi)
    seqs = _log_int(rng, 1, 64)
    hi = _log_int(rng, 200, min(65536, 600000 // seqs))
    act = rng.randint(0, 8)
    top = max(3, min(512, 16000 // seqs, _log_int(rng, 8, 512)))
    c = dict(kind=kind, shape=shape, seqs=seqs, ctx_lo=max(1, int(hi * rng.uniform(0.06, 1))), ctx_hi=hi, act_lo=rng.randint(0, act), act_hi=act, top=top)
    if kind == "attend":
        c["kv"] = kv
    return c


# ---- the call's bookkeeping, from the case alone ------------------------------------------------------------------------

def _plan(case):
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    S = case["seqs"]
    p = {"ctx": [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(S)]}
    p["new"] = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(S)] if "new_lo" in case else [0] * S
    p["act"] = [r.randint(case["act_lo"], case["act_hi"]) for _ in range(S)] if "act_lo" in case else [0] * S
    p["end"] = [a + b for a, b in zip(p["ctx"], p["new"])]
    if "new_lo" in case:  # a sequence's new tokens, then a row for each agent at the last of them
        p["rows_of"] = [n + a if n else 0 for n, a in zip(p["new"], p["act"])]
    else:
        p["rows_of"] = [1 + a for a in p["act"]]
    p["rows"] = sum(p["rows_of"])
    p["max_blocks"] = max(1, max(-(-e // BK) for e in p["end"]))
    p["old"] = [-(-c // BK) for c in p["ctx"]]
    p["need"] = [-(-e // BK) - o for e, o in zip(p["end"], p["old"])]
    return p


def _elem(case):
    return {"fp8": 1}.get(case.get("kv", "same"), 2 if SHAPES[case["shape"]][6] else 4)


def work(case):
    p, S = _plan(case), case["seqs"]
    if case["kind"] == "extend":  # lengths in; per row its sequence, position and slot; the new entries of the tables and the ids they take
        return {"bytes": 12 * S + 8 * S + 16 * p["rows"] + 8 * sum(p["need"]), "flops": 0}
    Hq, Hkv, D, _, _, _, bf16 = SHAPES[case["shape"]]
    es = 2 if bf16 else 4
    if case["kind"] == "append":
        n = sum(p["new"])
        return {"bytes": 2 * p["rows"] * Hq * D * es + 2 * n * Hkv * D * (es + _elem(case)) + 12 * p["rows"],
                "flops": 6 * p["rows"] * Hq * D + 6 * n * Hkv * D}
    if case["kind"] == "bounds":
        blocks = sum(-(-e // BK) - c // BK for c, e in zip(p["ctx"], p["end"]))
        tokens = sum(e - c // BK * BK for c, e in zip(p["ctx"], p["end"]))
        return {"bytes": tokens * Hkv * D * _elem(case) + blocks * (Hkv * (2 * D + 4) + 4), "flops": 2 * tokens * Hkv * D}
    blocks = [-(-e // BK) for e in p["end"]]
    if case["kind"] == "select":
        return {"bytes": sum(blocks) * (Hkv * (2 * D + 4) + 4) + p["rows"] * Hq * D * es + S * Hkv * case["top"] * 4,
                "flops": sum(4 * D * b * n * Hq for b, n in zip(blocks, p["rows_of"]))}
    tokens = [min(e, case["top"] * BK) for e in p["end"]]
    return {"bytes": sum(tokens) * 2 * Hkv * D * _elem(case) + 2 * p["rows"] * Hq * D * es + 4 * Hkv * sum(min(b, case["top"]) for b in blocks),
            "flops": sum(4 * D * t * n * Hq for t, n in zip(tokens, p["rows_of"]))}


# ---- inputs, from the seed ----------------------------------------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    p, S = _plan(case), case["seqs"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"kind": case["kind"], "case": dict(case), "S": S, "rows": p["rows"], "group": max(p["rows_of"]), "ctx": _ints(p["ctx"]), "new": _ints(p["new"]), "act": _ints(p["act"]),
          "end": _ints(p["end"]), "max_blocks": p["max_blocks"], "max_new": max(p["new"])}
    start = [0]
    for n in p["rows_of"]:
        start.append(start[-1] + n)
    st["row_start"] = _ints(start)

    # Block ids: a random permutation of the pool, dealt to the sequences' tables.
    have = [o if case["kind"] == "extend" else o + n for o, n in zip(p["old"], p["need"])]
    taken = 3 if case["kind"] == "extend" else 0  # ids at the list's front that went before
    st["num_blocks"] = max(1, sum(p["old"]) + sum(p["need"]) + taken)
    perm = torch.randperm(st["num_blocks"], generator=gen, device="cuda").to(torch.int32)
    first = [0]
    for h in have:
        first.append(first[-1] + h)
    col = torch.arange(p["max_blocks"], device="cuda")
    at = (torch.tensor(first[:-1], device="cuda")[:, None] + col).clamp_(max=st["num_blocks"] - 1)
    st["table"] = torch.where(col < torch.tensor(have, device="cuda")[:, None], perm[at], -1).contiguous()
    if case["kind"] == "extend":
        st["free"] = perm[first[-1]:][:taken + int(sum(p["need"]) * case["free"])].contiguous()
        st["used"] = _ints([taken])
    else:
        _tensors(case, p, st, gen)
    if own:
        _handle(case, st)
    return st


def _tensors(case, p, st, gen):
    Hq, Hkv, D, _, norm, _, bf16 = SHAPES[case["shape"]]
    dt = torch.bfloat16 if bf16 else torch.float32
    kind, S = case["kind"], case["seqs"]

    def normal(*shape, std=1.0):
        t = torch.empty(shape, dtype=dt, device="cuda")
        flat = t.view(-1)
        for a in range(0, flat.numel(), 1 << 28):
            n = min(1 << 28, flat.numel() - a)
            flat[a:a + n] = torch.randn(n, generator=gen, device="cuda") * std
        return t

    def pool():  # N(0, 1) in every slot; the FP8 cache with scale 1
        t = normal(st["num_blocks"], Hkv, 2, BK * D)
        return t.to(torch.float8_e4m3fn).view(torch.uint8) if case.get("kv") == "fp8" else t

    if kind == "append":
        st["pool"] = pool()
        st["qkv"] = normal(p["rows"], (Hq + 2 * Hkv) * D)
        if norm:
            st["q_norm"], st["k_norm"] = 1 + normal(D, std=0.1), 1 + normal(D, std=0.1)
        pos, slot = [], []
        table = st["table"].tolist()
        for s in range(S):
            for t in range(p["ctx"][s], p["end"][s]):
                pos.append(t)
                slot.append(table[s][t // BK] * BK + t % BK)
            if p["new"][s]:
                pos += [p["end"][s] - 1] * p["act"][s]
                slot += [-1] * p["act"][s]
        st["pos"], st["slot"] = _ints(pos), torch.tensor(slot, dtype=torch.int64, device="cuda")
        st["out"] = torch.empty((p["rows"], Hq, D), dtype=dt, device="cuda")
    if kind in ("bounds", "attend"):
        st["pool"] = pool()
    if kind in ("bounds", "select"):
        # codes as keys from N(0, 1) give them: extremes of 16 values, in steps of a 32nd mostly
        wide = 57 + 13 * torch.randn((st["num_blocks"], Hkv, 2, D), generator=gen, device="cuda")
        wide[:, :, 1] *= -1
        st["codes"] = wide.round_().clamp_(-127, 127).to(torch.int8)
        st["scales"] = torch.exp2(-torch.randint(4, 7, (st["num_blocks"], Hkv), generator=gen, device="cuda").float())
    if kind in ("select", "attend"):
        st["q"] = normal(p["rows"], Hq, D)
        st["top"] = case["top"]
    if kind == "select":
        st["blocks"], st["counts"] = torch.empty((S, Hkv, case["top"]), dtype=torch.int32, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda")
    if kind == "attend":  # the first block, the last two, and others at random, ascending
        nb = ((st["end"] + BK - 1) // BK)[:, None, None]
        col = torch.arange(max(st["max_blocks"], case["top"]), device="cuda")
        rank = torch.rand((S, Hkv, col.numel()), generator=gen, device="cuda")
        rank = torch.where((col == 0) | (col >= nb - 2), 2.0, rank)
        rank = torch.where(col < nb, rank, -1.0)
        best = rank.topk(case["top"], dim=-1)
        ids = torch.where(best.values >= 0, best.indices, 1 << 30).sort(dim=-1).values
        st["blocks"] = torch.where(ids < 1 << 30, ids, -1).to(torch.int32).contiguous()
        st["counts"] = (st["blocks"][:, 0] >= 0).sum(-1).to(torch.int32)
        st["out"] = torch.empty_like(st["q"])


# ---- the library's calls ------------------------------------------------------------------------------------------------

def _handle(case, st):
    """The layer context and the buffers that a serving program keeps."""
    from paper_2603_13281_amd import binding

    Hq, Hkv, D, theta, norm, eps, bf16 = SHAPES[case.get("shape", "llama8b")]
    one = torch.zeros(256, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    weights = {n: one for n in binding.PROJ + ("norm_attn", "norm_ffn")}  # none of these calls reads a projection
    if norm:
        weights["q_norm"], weights["k_norm"] = st.get("q_norm", one), st.get("k_norm", one)
    st["layer"] = binding.IcarusLayer(binding.LayerConfig(
        d_model=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, d_ffn=256, block_size=BK, num_blocks=st["num_blocks"], bf16=bf16, qk_norm=norm,
        max_position=MAX_POSITION, rope_theta=theta, rms_eps=eps, kv_fp8=case.get("kv") == "fp8"), weights)
    if case["kind"] == "extend":
        st["map"] = binding.SequenceMap(st["S"], st["rows"], "cuda")


def _run_own(st):
    layer, kind = st["layer"], st["kind"]
    if kind == "extend":
        m = layer.extend_sequences(st["map"], st["ctx"], st["new"], st["table"], st["free"], st["used"], streams=st["act"])
        return {"kv_lens": m.kv_lens, "row_start": m.row_start, "row_seq": m.row_seq, "row_pos": m.row_pos, "row_slot": m.row_slot, "counts": m.counts,
                "table": st["table"]}
    if kind == "append":
        layer.rope_append(st["qkv"], st["pos"], st["slot"], st["pool"], st["out"])
        return {"q": st["out"], "cache": _cache(st)}
    if kind == "bounds":
        layer.key_bounds(st["pool"], st["table"], st["ctx"], st["end"], st["codes"], st["scales"], max_new=st["max_new"])
        return {"codes": st["codes"], "scales": st["scales"]}
    if kind == "select":
        layer.select_blocks(st["q"], st["codes"], st["scales"], st["table"], st["end"], st["row_start"], st["blocks"], st["counts"], first=1, last=2,
                            seq_rows=st["group"])
        return {"blocks": st["blocks"], "counts": st["counts"]}
    layer.attn_blocks(st["q"], st["pool"], st["table"], st["end"], st["row_start"], st["blocks"], st["counts"], st["out"], seq_rows=st["group"])
    return {"out": st["out"]}


# ---- plain torch --------------------------------------------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"extend": _extend, "append": _append, "bounds": _bounds, "select": _select, "attend": _attend}[st["kind"]](st)


def _cache(st):
    return st["pool"].view(torch.float8_e4m3fn) if st["pool"].dtype == torch.uint8 else st["pool"]


def _values(st, x):
    return (x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x).float()


def _extend(st):
    """A sequence's new tokens take the rest of its last block, then blocks from the free list, in the order of the sequences; one whose
    blocks would reach past the list's end gets none."""
    ctx, new, rows, table = st["ctx"].long(), st["new"].long(), st["rows"], st["table"]
    old, end = (ctx + BK - 1) // BK, ctx + new
    need = (end + BK - 1) // BK - old
    head = st["used"].long()
    last = head + need.cumsum(0)
    ok = (need == 0) | (last <= st["free"].numel())
    n = torch.where(new > 0, new + st["act"], 0)
    stop = n.cumsum(0)
    row = torch.arange(rows, device="cuda")
    s = torch.searchsorted(stop, row, right=True).clamp(max=st["S"] - 1)
    i = row - (stop - n)[s]
    pos = ctx[s] + torch.minimum(i, new[s] - 1)
    column = pos // BK
    good, col = ok[s], torch.arange(table.shape[1], device="cuda")
    fresh = (col >= old[:, None]) & (col < (old + need)[:, None]) & ok[:, None]
    take = ((last - need - old)[:, None] + col).clamp(0, st["free"].numel() - 1)
    table.copy_(torch.where(fresh, st["free"][take], table))
    slot = torch.where(good & (i < new[s]), table[s, column.clamp(max=table.shape[1] - 1)].long() * BK + pos % BK, -1)
    return {"kv_lens": torch.where(ok, end, ctx).int(), "row_start": torch.cat([stop.new_zeros(1), stop]).int(),
            "row_seq": torch.where(good, s, -1).int(), "row_pos": torch.where(good, pos, -1).int(), "row_slot": slot,
            "counts": torch.stack([torch.where(ok & (need > 0), last, head).amax(), (~ok).sum()]).int(), "table": table}


def _append(st):
    Hq, Hkv, D, theta, norm, eps, _ = SHAPES[st["case"]["shape"]]
    rows, pool = st["rows"], st["pool"]
    x = st["qkv"].float().view(rows, Hq + 2 * Hkv, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if norm:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + eps) * st["q_norm"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + eps) * st["k_norm"].float()
    half = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    angle = st["pos"].double()[:, None] * torch.exp2(-2.0 * half / D * math.log2(theta))
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotate(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    st["out"].copy_(rotate(q))
    to = torch.nonzero(st["slot"] >= 0)[:, 0]
    slot = st["slot"][to]
    block, off = slot // BK, slot % BK
    k, v = rotate(k)[to], v[to]
    if pool.dtype == torch.uint8:  # scale 1
        k, v = (t.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for t in (k, v))
    pool.view(-1, Hkv, 2, BK, D)[block, :, 0, off] = k.to(pool.dtype)
    pool.view(-1, Hkv, 2, D, BK)[block, :, 1, :, off] = v.to(pool.dtype)
    return {"q": st["out"], "cache": _cache(st)}


def _step(a):
    """2^e for the smallest e in -40 .. 40 with 127 * 2^e >= a."""
    m, x = torch.frexp(a)
    return torch.exp2(torch.where(a > 0, x - 7 + (m > 127 / 128).int(), -40).clamp(-40, 40).float())


def _finite(x):
    return torch.nan_to_num(x, nan=0.0)


def _bounds(st):
    Hq, Hkv, D = SHAPES[st["case"]["shape"]][:3]
    col = torch.arange(st["max_blocks"], device="cuda")
    touched = (col >= (st["ctx"] // BK)[:, None]) & (col < ((st["end"] + BK - 1) // BK)[:, None]) & (st["new"] > 0)[:, None]
    s, b = torch.nonzero(touched, as_tuple=True)
    ids = st["table"][s, b].long()
    n = (st["end"][s] - b * BK).clamp(max=BK)
    k = _finite(_values(st, st["pool"].view(-1, Hkv, 2, BK, D)[ids, :, 0]))
    there = torch.arange(BK, device="cuda")[None, None, :, None] < n[:, None, None, None]
    hi = torch.where(there, k, -math.inf).amax(2)
    lo = torch.where(there, k, math.inf).amin(2)
    step = _step(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    codes = torch.stack([torch.ceil(hi / step[..., None]), torch.floor(lo / step[..., None])], 2).clamp(-127, 127)
    st["codes"][ids] = codes.to(torch.int8)
    st["scales"][ids] = step
    return {"codes": st["codes"], "scales": st["scales"]}


def _stacked(st, q):
    """Rows of each sequence, stacked with the query heads of each kv-head: [S, Hkv, group * g, D], and which of them are there."""
    Hq, Hkv, D = SHAPES[st["case"]["shape"]][:3]
    row = st["row_start"][:-1, None].long() + torch.arange(st["group"], device="cuda")
    there = row < st["row_start"][1:, None]
    x = q[row.clamp(max=st["rows"] - 1)].float().view(st["S"], st["group"], Hkv, Hq // Hkv, D)
    return x.transpose(1, 2).reshape(st["S"], Hkv, -1, D), there.repeat_interleave(Hq // Hkv, 1)[:, None], row, there


def _select(st):
    """Score of a block: the largest, over the stacked queries, of the sum over channels of q * (the block's largest key where q is positive, its
    smallest where it is negative), with q and keys in 8 bits.  Sums of whole numbers below 2^23, times powers of two: exact in float32."""
    q, there, _, _ = _stacked(st, st["q"])
    q = _finite(q)
    step = _step(q.abs().amax(-1))
    q = torch.round(q / step[..., None]).clamp(-127, 127)
    ids = st["table"].long().clamp(min=0)
    codes = st["codes"][ids].float().permute(0, 2, 3, 1, 4)  # [S, Hkv, 2, blocks, D]
    dots = torch.matmul(q.clamp(min=0), codes[:, :, 0].transpose(2, 3)) + torch.matmul(q.clamp(max=0), codes[:, :, 1].transpose(2, 3))
    best = torch.where(there[..., None], dots * step[..., None], -math.inf).amax(2)
    score = best * st["scales"][ids].transpose(1, 2)
    nb = ((st["end"] + BK - 1) // BK)[:, None, None]
    col = torch.arange(score.shape[2], device="cuda")
    score = torch.where((col < 1) | (col >= nb - 2), math.inf, score)
    score = torch.where(col < nb, score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    far = 1 << 30
    order = torch.where(col < nb, order, far)[..., :st["top"]].sort(dim=-1).values
    st["blocks"].fill_(-1)
    st["blocks"][..., :order.shape[2]] = torch.where(order < far, order, -1)
    st["counts"].copy_(nb[:, 0, 0].clamp(max=st["top"]))
    return {"blocks": st["blocks"], "counts": st["counts"]}


def _attend(st):
    Hq, Hkv, D = SHAPES[st["case"]["shape"]][:3]
    q, there, row, real = _stacked(st, st["q"])
    S, top = st["S"], st["top"]
    listed_ = st["blocks"].long()
    ids = st["table"].long().gather(1, listed_.clamp(min=0).view(S, -1)).view(S, Hkv, top)
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    k = _values(st, st["pool"].view(-1, Hkv, 2, BK, D)[ids, head, 0]).reshape(S, Hkv, top * BK, D)
    v = _values(st, st["pool"].view(-1, Hkv, 2, D, BK)[ids, head, 1]).transpose(3, 4).reshape(S, Hkv, top * BK, D)
    pos = listed_[..., None] * BK + torch.arange(BK, device="cuda")
    seen = ((listed_ >= 0)[..., None] & (pos < st["end"][:, None, None, None])).view(S, Hkv, 1, top * BK)
    score = torch.where(seen, torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D)), -math.inf)
    p = torch.where(seen, torch.exp(score - score.amax(-1, keepdim=True)), 0.0)
    out = torch.matmul(p / p.sum(-1, keepdim=True), v)  # every sequence has a token
    out = out.view(S, Hkv, st["group"], Hq // Hkv, D).transpose(1, 2).reshape(S, st["group"], Hq, D)
    st["out"].copy_(out[real])
    return {"out": st["out"]}


# ---- float64 ------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] in ("extend", "select"):
        return None  # whole numbers
    st, p = prepare(case, seed), _plan(case)
    Hq, Hkv, D, theta, norm, eps, _ = SHAPES[case["shape"]]
    if case["kind"] == "bounds":
        scales = st["scales"].double()
        for s in range(case["seqs"]):
            for b in range(p["ctx"][s] // BK, -(-p["end"][s] // BK), 4096):
                last = min(b + 4096, -(-p["end"][s] // BK))
                ids = st["table"][s, b:last].long()
                k = st["pool"][ids][:, :, 0].reshape(last - b, Hkv, BK, D)
                k = (k.view(torch.float8_e4m3fn) if k.dtype == torch.uint8 else k).double().abs()
                pos = torch.arange(b * BK, last * BK, device="cuda").view(last - b, 1, BK, 1)
                a = torch.where(pos < p["end"][s], k, 0.0).amax((2, 3))
                scales[ids] = torch.exp2(torch.ceil(torch.log2(a / 127)))
        return {"codes": None, "scales": scales}
    if case["kind"] == "append":
        x = st["qkv"].double().view(-1, Hq + 2 * Hkv, D)
        turn = st["pos"].double()[:, None] * theta ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        w = torch.polar(torch.ones_like(turn), turn)[:, None]
        heads = x[:, :Hq + Hkv]
        if norm:
            gain = torch.cat([st["q_norm"].double().expand(Hq, D), st["k_norm"].double().expand(Hkv, D)])
            heads = heads / torch.sqrt(heads.square().sum(-1, keepdim=True) / D + eps) * gain
        z = torch.complex(heads[..., :D // 2].contiguous(), heads[..., D // 2:].contiguous()) * w
        heads = torch.cat([z.real, z.imag], -1)
        cache = st["pool"].view(torch.float8_e4m3fn).double() if st["pool"].dtype == torch.uint8 else st["pool"].double()
        k, v = cache.view(-1, Hkv, 2, BK, D)[:, :, 0], cache.view(-1, Hkv, 2, D, BK)[:, :, 1]
        to = st["slot"] >= 0
        slot = st["slot"][to]
        k.index_put_((slot // BK, torch.arange(Hkv, device="cuda")[:, None], slot % BK), heads[to, Hq:].transpose(0, 1))
        v.permute(0, 1, 3, 2).index_put_((slot // BK, torch.arange(Hkv, device="cuda")[:, None], slot % BK), x[to, Hq + Hkv:].transpose(0, 1))
        return {"q": heads[:, :Hq], "cache": cache}
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for s in range(case["seqs"]):
        n, q = p["rows_of"][s], st["q"][at:at + p["rows_of"][s]].double()
        for c in range(Hkv):
            b = st["blocks"][s, c, :int(st["counts"][s])].long()
            kv = st["pool"][st["table"][s][b].long(), c]
            kv = (kv.view(torch.float8_e4m3fn) if kv.dtype == torch.uint8 else kv).double()
            pos = (b[:, None] * BK + torch.arange(BK, device="cuda")).view(-1)
            k = kv[:, 0].reshape(-1, D)[pos < p["end"][s]]
            v = kv[:, 1].reshape(-1, D, BK).permute(0, 2, 1).reshape(-1, D)[pos < p["end"][s]]
            g = Hq // Hkv
            a = torch.softmax(q[:, c * g:(c + 1) * g].reshape(-1, D) @ k.T / math.sqrt(D), -1)
            out[at:at + n, c * g:(c + 1) * g] = (a @ v).view(n, g, D)
        at += n
    return {"out": out}
