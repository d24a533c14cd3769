"""Sequences that branch over a shared prefix: the operators of beam search and of batches with a common prefix as measurable cases.

A decoding loop whose sequences fork on the GPU makes four calls a step beside the ones of operators.py:

  choose   the best continuations of each group of beams, from the logits of the whole vocabulary
  fork     new block tables from the chosen parents: shared blocks, places for the copies, blocks that nobody holds any more
  copy     the blocks that may no longer be shared, in the pools of all layers
  attend   attention of one token per row, the blocks that a group of sequences shares read once for all of its rows

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
EOS = 2
# query heads, kv-heads, head size, bf16
SHAPES = {
    "tiny": (4, 4, 64, False),
    "llama8b": (32, 8, 128, True),
    "qwen32b": (64, 8, 128, True),
}


def listed():
    return [
        # One question, four beams, over the vocabulary of the layer stack: interactive latency.
        dict(name="choose_one", kind="choose", groups=1, width=4, vocab=128256, bf16=False, act=1, done=0.0),
        # A full server, an encoder and a decoder row to each beam; some beams have ended.
        dict(name="choose_batch", kind="choose", groups=64, width=8, vocab=128256, bf16=False, act=1, done=0.1),
        # Logits in bfloat16, where many are equal; an odd vocabulary.
        dict(name="choose_bf16", kind="choose", groups=24, width=5, vocab=50021, bf16=True, act=0, done=0.05),
        # Eight beams of one long conversation.
        dict(name="fork_one", kind="fork", groups=1, width=8, ctx_lo=32768, ctx_hi=32768, spread=0, shared=0.98, gone=0.0),
        # A full server; some beams end for good.
        dict(name="fork_batch", kind="fork", groups=64, width=8, ctx_lo=1024, ctx_hi=16384, spread=40, shared=0.8, gone=0.05),
        # The copies of that one conversation, in eight layers.
        dict(name="copy_one", kind="copy", shape="llama8b", kv="same", layers=8, entries=8, real=0.75),
        # Those of the full server.
        dict(name="copy_batch", kind="copy", shape="llama8b", kv="same", layers=8, entries=512, real=0.6),
        # The smallest layer: three samples of one short prompt in float32.
        dict(name="attend_tiny_fp32", kind="attend", shape="tiny", kv="same", groups=1, seqs_lo=3, seqs_hi=3, pre_lo=100, pre_hi=100, tail_lo=1, tail_hi=30, act_lo=0, act_hi=0),
        # One long conversation, eight beams of a base and a task model each.
        dict(name="attend_beams", kind="attend", shape="llama8b", kv="same", groups=1, seqs_lo=8, seqs_hi=8, pre_lo=32000, pre_hi=32000, tail_lo=20, tail_hi=300, act_lo=1, act_hi=1),
        # The mixed batch: 64 conversations over eight system prompts, one to eight agents answering.
        dict(name="attend_batch", kind="attend", shape="llama8b", kv="same", groups=8, seqs_lo=4, seqs_hi=12, pre_lo=1024, pre_hi=8192, tail_lo=50, tail_hi=2000, act_lo=1, act_hi=8),
        # One long system prompt for a crowd of conversations.
        dict(name="attend_crowd", kind="attend", shape="llama8b", kv="same", groups=1, seqs_lo=128, seqs_hi=128, pre_lo=8192, pre_hi=8192, tail_lo=0, tail_hi=500, act_lo=1, act_hi=1),
        # Long contexts on the larger model, all agents, cache in FP8.
        dict(name="attend_long_fp8", kind="attend", shape="qwen32b", kv="fp8", groups=2, seqs_lo=8, seqs_hi=8, pre_lo=32768, pre_hi=32768, tail_lo=1, tail_hi=1000, act_lo=8, act_hi=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["choose", "choose", "fork", "copy", "attend", "attend", "attend"])
    if kind == "choose":
        vocab, width = _log_int(rng, 500, 160000), rng.randint(1, 16)
        return dict(kind=kind, groups=_log_int(rng, 1, max(1, min(64, 65000000 // (vocab * width)))), width=width, vocab=vocab, bf16=rng.random() < 0.4, act=rng.randint(0, 2),
                    done=rng.choice([0.0, round(rng.uniform(0, 0.4), 2)]))
    if kind == "fork":
        groups, width = _log_int(rng, 1, 64), rng.randint(2, 24)
        hi = _log_int(rng, 20, min(65536, 8000000 // (groups * width)))
        return dict(kind=kind, groups=groups, width=width, ctx_lo=int(hi * rng.uniform(0.1, 1)), ctx_hi=hi, spread=rng.choice([0, 40]), shared=round(rng.uniform(0, 0.99), 2),
                    gone=rng.choice([0.0, 0.1]))
    shape, kv = rng.choice(["llama8b", "llama8b", "qwen32b", "tiny"]), rng.choice(["same", "same", "fp8"])
    if kind == "copy":
        layers = rng.randint(1, 24)
        return dict(kind=kind, shape=shape, kv=kv, layers=layers, entries=_log_int(rng, 1, 4096 // layers), real=round(rng.uniform(0.2, 1), 2))
    groups = _log_int(rng, 1, 16)
    seqs = _log_int(rng, 1, 128 // groups)
    act = rng.randint(0, 8) if seqs * groups <= 64 else rng.randint(0, 2)
    rows = seqs * groups * (act + 1) * (2 if shape == "qwen32b" else 1)
    hi = _log_int(rng, 16, min(65536, 400000 // groups, 9000000 // rows))
    tail = _log_int(rng, 1, min(2000, 160000 // (seqs * groups)))
    return dict(kind=kind, shape=shape, kv=kv, groups=groups, seqs_lo=max(1, seqs // 2), seqs_hi=seqs, pre_lo=int(hi * rng.uniform(0.2, 1)), pre_hi=hi, tail_lo=rng.randint(0, tail), tail_hi=tail,
                act_lo=rng.randint(0, act), act_hi=act)


# ---- the call's bookkeeping, from the case alone ------------------------------------------------------------------------

def _blocks(n):
    return -(-n // BK)


def _plan(case):
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    G, p = case["groups"], {}
    if case["kind"] == "fork":
        W = case["width"]
        base = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(G)]
        p["shared"] = [int(b * case["shared"]) // BK for b in base]
        p["len"] = [b + r.randint(0, case["spread"]) for b in base for _ in range(W)]
        p["apart"] = [r.randint(p["shared"][i // W], _blocks(n)) for i, n in enumerate(p["len"])]  # the column from which a beam has blocks of its own
        p["parents"] = [-1 if r.random() < case["gone"] else int(W * r.random() ** 2) for _ in range(G * W)]
        p["max_blocks"] = max(1, max(_blocks(n) for n in p["len"]))
        return p
    n_seqs = [r.randint(case["seqs_lo"], case["seqs_hi"]) for _ in range(G)]
    p["group_start"] = [sum(n_seqs[:i]) for i in range(G + 1)]
    p["pre"] = [r.randint(case["pre_lo"], case["pre_hi"]) for _ in range(G)]
    p["group"] = [i for i, n in enumerate(n_seqs) for _ in range(n)]
    p["tail"] = [r.randint(case["tail_lo"], case["tail_hi"]) for _ in p["group"]]
    p["len"] = [p["pre"][g] + t for g, t in zip(p["group"], p["tail"])]
    p["rows_of"] = [1 + r.randint(case["act_lo"], case["act_hi"]) for _ in p["group"]]
    p["rows"] = sum(p["rows_of"])
    p["max_blocks"] = max(1, max(_blocks(n) for n in p["len"]))
    return p


def _elem(case):
    return 1 if case["kv"] == "fp8" else 2 if SHAPES[case["shape"]][3] else 4


def work(case):
    if case["kind"] == "choose":
        rows = case["groups"] * case["width"]
        return {"bytes": rows * (case["vocab"] * (2 if case["bf16"] else 4) + 4 + 4 + 16), "flops": 0}
    if case["kind"] == "copy":
        Hq, Hkv, D, _ = SHAPES[case["shape"]]
        real = max(1, int(case["entries"] * case["real"]))
        return {"bytes": 2 * real * case["layers"] * Hkv * 2 * BK * D * _elem(case) + 8 * case["entries"], "flops": 0}
    p = _plan(case)
    if case["kind"] == "fork":  # each table read and each written once; parents and lengths in, lengths and copies out
        W = case["width"]
        new = sum(_blocks(p["len"][i // W * W + q]) for i, q in enumerate(p["parents"]) if q >= 0)
        return {"bytes": 4 * (sum(_blocks(n) for n in p["len"]) + new) + 20 * len(p["len"]), "flops": 0}
    Hq, Hkv, D, bf16 = SHAPES[case["shape"]]
    pre = sum(n // BK * BK for n in p["pre"])
    tails = sum(n - p["pre"][g] // BK * BK for g, n in zip(p["group"], p["len"]))
    return {"bytes": (pre + tails) * 2 * Hkv * D * _elem(case) + 2 * p["rows"] * Hq * D * (2 if bf16 else 4),
            "flops": sum(4 * D * Hq * n * r for n, r in zip(p["len"], p["rows_of"]))}


# ---- inputs, from the seed ----------------------------------------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(gen, dt, *shape):
    t = torch.empty(shape, dtype=dt, device="cuda")
    flat = t.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=gen, device="cuda")
    return t


def _pool(gen, case, num_blocks):
    """N(0, 1) in every slot; the FP8 cache with scale 1."""
    Hq, Hkv, D, bf16 = SHAPES[case["shape"]]
    t = _normal(gen, torch.bfloat16 if bf16 else torch.float32, num_blocks, Hkv, 2, BK * D)
    return t.to(torch.float8_e4m3fn).view(torch.uint8) if case["kv"] == "fp8" else t


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"kind": case["kind"], "case": dict(case), "num_blocks": 1}
    {"choose": _choose_state, "fork": _fork_state, "copy": _copy_state, "attend": _attend_state}[case["kind"]](case, st, gen)
    if own:
        _handle(case, st)
    return st


def _choose_state(case, st, gen):
    """Logits as a trained model gives them: a wide bell and some dozens of tokens that stand out of it."""
    S, per = case["groups"] * case["width"], 1 + case["act"]
    logits = _normal(gen, torch.float32, S * per, case["vocab"]) * 2
    top = torch.randint(case["vocab"], (S * per, 48), generator=gen, device="cuda")
    logits.scatter_add_(1, top, 9 * torch.rand(top.shape, generator=gen, device="cuda"))
    st["logits"] = logits.bfloat16() if case["bf16"] else logits
    st["row_start"] = _ints([per * i for i in range(S + 1)])
    st["scores"] = -25 * torch.rand(S, generator=gen, device="cuda")
    st["done"] = (torch.rand(S, generator=gen, device="cuda") < case["done"]).int()


def _fork_state(case, st, gen):
    """Beams of a group share the columns before the one at which they came apart; the list holds every block, those in use before its head."""
    p, G, W = _plan(case), case["groups"], case["width"]
    st["max_blocks"], C = p["max_blocks"], p["max_blocks"]
    col, n = torch.arange(C, device="cuda"), torch.tensor(p["len"], device="cuda")
    nb = (n + BK - 1) // BK
    first = torch.arange(G * W, device="cuda") // W * W
    alone = col >= torch.tensor(p["apart"], device="cuda")[:, None]
    longest = nb.view(G, W).amax(1).repeat_interleave(W)[:, None]
    home = (col < longest) & (torch.arange(G * W, device="cuda") == first)[:, None]  # the blocks that beams share stand in the first beam's row
    wanted = (home | (alone & (col < nb[:, None]))).view(-1)
    used = int(wanted.sum())
    st["num_blocks"] = used + 2 * G * W + 5
    perm = torch.randperm(st["num_blocks"], generator=gen, device="cuda").to(torch.int32)
    ids = torch.full((G * W * C,), -1, dtype=torch.int32, device="cuda")
    ids[wanted] = perm[:used]
    ids = ids.view(G * W, C)
    st["table"] = torch.where(col < nb[:, None], torch.where(alone, ids, ids[first]), -1).contiguous()
    st["free"], st["used"] = perm.clone(), _ints([used])
    st["len"], st["parents"], st["shared"] = _ints(p["len"]), _ints(p["parents"]), _ints(p["shared"])
    st["out"] = torch.full_like(st["table"], -1)


def _copy_state(case, st, gen):
    n, real = case["entries"], max(1, int(case["entries"] * case["real"]))
    st["num_blocks"] = 2 * n + 3
    st["pools"] = [_pool(gen, case, st["num_blocks"]) for _ in range(case["layers"])]
    perm = torch.randperm(st["num_blocks"], generator=gen, device="cuda").to(torch.int32)
    there = torch.randperm(n, generator=gen, device="cuda") < real
    st["src"], st["dst"] = (torch.where(there, perm[a:a + n], -1).contiguous() for a in (0, n))


def _attend_state(case, st, gen):
    p, S = _plan(case), len(_plan(case)["len"])
    Hq, Hkv, D, bf16 = SHAPES[case["shape"]]
    own_from = [p["pre"][g] // BK for g in p["group"]]
    need = [_blocks(n) - a for n, a in zip(p["len"], own_from)]
    whole = [n // BK for n in p["pre"]]
    at_group = [sum(whole[:i]) for i in range(len(whole))]
    at_seq = [sum(whole) + sum(need[:i]) for i in range(S)]
    st["num_blocks"] = max(1, sum(whole) + sum(need))
    perm = torch.randperm(st["num_blocks"], generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(p["max_blocks"], device="cuda")
    a, b, c, e = (torch.tensor(v, device="cuda")[:, None] for v in ([at_group[g] for g in p["group"]], at_seq, own_from, [_blocks(n) for n in p["len"]]))
    at = torch.where(col < c, a + col, b + col - c).clamp(0, st["num_blocks"] - 1)
    st["table"] = torch.where(col < e, perm[at], -1).contiguous()
    st["pool"] = _pool(gen, case, st["num_blocks"])
    st["q"] = _normal(gen, torch.bfloat16 if bf16 else torch.float32, p["rows"], Hq, D)
    st["out"] = torch.empty_like(st["q"])
    start = [0]
    for r in p["rows_of"]:
        start.append(start[-1] + r)
    st["row_start"], st["group_start"], st["pre"], st["len"] = _ints(start), _ints(p["group_start"]), _ints(p["pre"]), _ints(p["len"])
    st["rows"], st["seqs"] = p["rows"], S
    st["most_rows"] = max(p["rows_of"])
    st["most_group"] = max(start[y] - start[x] for x, y in zip(p["group_start"], p["group_start"][1:]))
    st["most_tail"] = max(n - a * BK for n, a in zip(p["len"], own_from))
    st["most_whole"] = max(whole)


# ---- the library's calls ------------------------------------------------------------------------------------------------

def _handle(case, st):
    """The layer context and the buffers that a serving program keeps."""
    from paper_2603_13281_amd import binding

    Hq, Hkv, D, bf16 = SHAPES[case.get("shape", "llama8b")]
    one = torch.zeros(256, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    weights = {n: one for n in binding.PROJ + ("norm_attn", "norm_ffn")}  # none of these calls reads a projection
    st["layer"] = binding.IcarusLayer(binding.LayerConfig(
        d_model=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, d_ffn=256, block_size=BK, num_blocks=st["num_blocks"], bf16=bf16,
        max_position=MAX_POSITION, kv_fp8=case.get("kv") == "fp8"), weights)
    if case["kind"] == "choose":
        st["map"] = binding.BeamMap(case["groups"], case["width"], "cuda")
    if case["kind"] == "fork":
        st["map"] = binding.ForkMap(case["groups"], case["width"], st["max_blocks"], "cuda")
        st["map"].block_tables.fill_(-1)


def _run_own(st):
    layer, kind = st["layer"], st["kind"]
    if kind == "choose":
        m = layer.beam_select(st["logits"], st["scores"], st["map"], row_start=st["row_start"], done=st["done"], eos=EOS)
        return {"parents": m.parents, "tokens": m.tokens, "scores": m.scores, "done": m.done}
    if kind == "fork":
        m = layer.fork_sequences(st["parents"], st["len"], st["table"], st["map"], st["free"], st["used"], shared=st["shared"])
        return {"kv_lens": m.kv_lens, "tables": m.block_tables, "copy_src": m.copy_src, "copy_dst": m.copy_dst, "counts": m.counts, "free": st["free"]}
    if kind == "copy":
        layer.copy_blocks(st["pools"], st["src"], st["dst"])
        return {"pools": [_values(x) for x in st["pools"]]}
    layer.attn_prefix(st["q"], st["pool"], st["table"], st["len"], st["row_start"], st["group_start"], st["pre"], st["out"])
    return {"out": st["out"]}


# ---- plain torch --------------------------------------------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"choose": _choose, "fork": _fork, "copy": _copy, "attend": _attend}[st["kind"]](st)


def _values(x):
    return x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x


def _choose(st):
    """A beam continues with each token at its score plus the token's log-probability; one that is done stays as it is, as its end token.  In 64 bits: a choice
    hangs on the last digits of the normalisers."""
    G, W, V = (st["case"][k] for k in ("groups", "width", "vocab"))
    x = st["logits"][(st["row_start"][1:] - 1).long()].double()
    most = x.amax(-1, keepdim=True)
    norm = most + torch.exp(x - most).sum(-1, keepdim=True).log()
    score = x.sub_(norm).add_(st["scores"].double()[:, None])
    done = st["done"].bool()[:, None]
    end = torch.arange(V, device="cuda") == EOS
    score = torch.where(done, torch.where(end, st["scores"].double()[:, None], -math.inf), score).view(G, W * V)
    best = torch.sort(score, dim=-1, descending=True, stable=True)
    value, at = best.values[:, :W], best.indices[:, :W]
    none = value == -math.inf
    parent, token = torch.where(none, -1, at // V), torch.where(none, -1, at % V)
    was = st["done"].view(G, W).gather(1, parent.clamp(min=0)) > 0
    ended = ~none & (was | (token == EOS))
    return {"parents": parent.int().view(-1), "tokens": token.int().view(-1), "scores": value.float().view(-1), "done": ended.int().view(-1)}


def _fork(st):
    """Child i of a group takes the table of its parent.  A block that is partly filled goes to the parent's first child, the others get a fresh one and a copy.  Blocks behind
    the shared columns that no child names any more go before the head of the free list, by group, column and beam; the fresh ones are taken from there."""
    G, W, C = st["case"]["groups"], st["case"]["width"], st["max_blocks"]
    parent, n = st["parents"].view(G, W).long(), st["len"].view(G, W)
    col = torch.arange(C, device="cuda")
    old = st["table"].view(G, W, C)
    have = (col < ((n + BK - 1) // BK)[..., None]) & (col >= st["shared"].view(G, 1, 1))
    child = parent[:, None, :] == torch.arange(W, device="cuda")[:, None]  # [G, beam, child]
    same = (old[:, :, None] == old[:, None]) & have[:, :, None] & have[:, None]  # [G, beam, other, column]
    held = (same & child.any(-1)[:, None, :, None]).any(2)
    before = torch.ones(W, W, dtype=torch.bool, device="cuda").tril(-1)
    free = have & ~held & ~(same & before[:, :, None]).any(2)
    freed = old.transpose(1, 2)[free.transpose(1, 2)]  # by group, column, beam
    head = st["used"].long() - freed.numel()
    st["free"][head + torch.arange(freed.numel(), device="cuda")] = freed
    ok = parent >= 0
    up = parent.clamp(min=0)
    length = torch.where(ok, n.gather(1, up), 0)
    first = (child & (child.cumsum(-1) == 1)).any(1)
    part = length % BK != 0
    last = length // BK
    fresh = (part & (~first | (last < st["shared"].view(G, 1)))).view(-1)
    at = head + fresh.cumsum(0) - 1
    refused = fresh & (at >= st["free"].numel())
    take = fresh & ~refused
    block = st["free"][at.clamp(0, st["free"].numel() - 1)]
    source = old.gather(1, up[..., None].expand(G, W, C)).view(-1, C)
    new_len = torch.where(refused, 0, length.view(-1))
    table = torch.where((col == last.view(-1, 1)) & take[:, None], block[:, None], source)
    st["out"].copy_(torch.where(col < ((new_len + BK - 1) // BK)[:, None], table, st["out"]))
    lent = source.gather(1, last.view(-1, 1).clamp(max=C - 1))[:, 0]
    counts = torch.stack([(head[0] + fresh.sum()).clamp(max=st["free"].numel()), refused.sum(), (free.sum())])
    return {"kv_lens": new_len.int(), "tables": st["out"], "copy_src": torch.where(take, lent, -1), "copy_dst": torch.where(take, block, -1), "counts": counts.int(), "free": st["free"]}


def _copy(st):
    there = st["src"] >= 0
    src, dst = st["src"][there].long(), st["dst"][there].long()
    for pool in st["pools"]:
        pool[dst] = pool[src]
    return {"pools": [_values(x) for x in st["pools"]]}


def _stacked(x, start, most, heads):
    """Rows start[i] .. start[i + 1] - 1 of each i, stacked with the query heads of each kv-head: [n, heads, most * g, D], the rows, and which of them are there."""
    row = start[:-1, None].long() + torch.arange(most, device="cuda")
    there = row < start[1:, None]
    R, Hq, D = x.shape
    y = x[row.clamp(max=R - 1)].float().view(len(row), most, heads, Hq // heads, D)
    return y.transpose(1, 2).reshape(len(row), heads, -1, D), there


def _unstacked(y, there, heads, Hq):
    """The other way: [rows, Hq, last] of what is there."""
    n, _, _, D = y.shape
    y = y.view(n, heads, there.shape[1], Hq // heads, D).transpose(1, 2).reshape(n, there.shape[1], Hq, D)
    return y[there]


def _part(q, ids, seen, pool, heads, D):
    """Maximum, sum and sum of values of the queries q over the tokens of the blocks ids that are seen [n, tokens]."""
    n, nb = ids.shape
    ids = ids.clamp(min=0)
    k = _values(pool)[ids, :, 0].float().view(n, nb, heads, BK, D).transpose(1, 2).reshape(n, heads, nb * BK, D)
    v = _values(pool)[ids, :, 1].float().view(n, nb, heads, D, BK).permute(0, 2, 1, 4, 3).reshape(n, heads, nb * BK, D)
    score = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).masked_fill_(~seen[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True).clamp(min=-1e30)
    w = score.sub_(most).exp_()
    return most, w.sum(-1, keepdim=True), torch.matmul(w, v)


def _attend(st):
    Hq, Hkv, D, _ = SHAPES[st["case"]["shape"]]
    whole = st["pre"] // BK
    group = torch.repeat_interleave(torch.arange(len(whole), device="cuda"), (st["group_start"][1:] - st["group_start"][:-1]).long(), output_size=st["seqs"])
    col = torch.arange(max(1, st["most_whole"]), device="cuda")
    ids = st["table"][st["group_start"][:-1].long()][:, col].long()
    q, there = _stacked(st["q"], st["row_start"][st["group_start"].long()], st["most_group"], Hkv)
    m, l, o = (_unstacked(x, there, Hkv, Hq) for x in _part(q, ids, (col < whole[:, None]).repeat_interleave(BK, 1), st["pool"], Hkv, D))
    at = whole[group][:, None] + torch.arange(max(1, _blocks(st["most_tail"])), device="cuda")
    ids = st["table"].gather(1, at.clamp(max=st["table"].shape[1] - 1).long()).long()
    seen = (at[..., None] * BK + torch.arange(BK, device="cuda") < st["len"][:, None, None]).flatten(1)
    q, there = _stacked(st["q"], st["row_start"], st["most_rows"], Hkv)
    m2, l2, o2 = (_unstacked(x, there, Hkv, Hq) for x in _part(q, ids, seen, st["pool"], Hkv, D))
    most = torch.maximum(m, m2)
    a, b = torch.exp(m - most), torch.exp(m2 - most)
    st["out"].copy_((a * o + b * o2) / (a * l + b * l2))  # every sequence has a token
    return {"out": st["out"]}


# ---- float64 ------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "fork":
        return None  # whole numbers
    st = prepare(case, seed)
    if case["kind"] == "copy":
        src, dst = st["src"].tolist(), st["dst"].tolist()
        pools = [_values(x).double() for x in st["pools"]]
        for new, old in zip(pools, st["pools"]):
            for s, d in zip(src, dst):
                if s >= 0:
                    new[d] = _values(old)[s].double()
        return {"pools": pools}
    if case["kind"] == "choose":
        W = case["width"]
        scores = []
        for g in range(case["groups"]):
            some = []
            for s in range(g * W, g * W + W):
                x = st["logits"][int(st["row_start"][s + 1]) - 1].double()
                score = float(st["scores"][s])
                some.append(torch.full((1,), score, dtype=torch.float64, device="cuda") if int(st["done"][s]) else (torch.log_softmax(x, 0) + score).topk(W).values)
            some = torch.cat(some).sort(descending=True).values[:W]
            scores.append(torch.nn.functional.pad(some, (0, W - len(some)), value=-math.inf))
        return {"parents": None, "tokens": None, "scores": torch.cat(scores), "done": None}
    Hq, Hkv, D, _ = SHAPES[case["shape"]]
    p, g = _plan(case), Hq // Hkv
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for s, (n, rows) in enumerate(zip(p["len"], p["rows_of"])):
        q = st["q"][at:at + rows].double()
        for c in range(Hkv):
            kv = _values(st["pool"])[st["table"][s, :_blocks(n)].long(), c].double()
            k = kv[:, 0].reshape(-1, D)[:n]
            v = kv[:, 1].reshape(-1, D, BK).permute(0, 2, 1).reshape(-1, D)[:n]
            w = torch.softmax(q[:, c * g:(c + 1) * g].reshape(-1, D) @ k.T / math.sqrt(D), -1)
            out[at:at + rows, c * g:(c + 1) * g] = (w @ v).view(rows, g, D)
        at += rows
    return {"out": out}
