"""icarus_branches.h without a GPU: the plain references against brute force, and every refusal that the host makes."""
import ctypes as C
import itertools
import math

import numpy as np
import pytest
import torch

import branch_reference as ref
from paper_2603_13281_amd import binding
from paper_2603_13281_amd.binding import IcarusLayer, LayerConfig

A = 0x1000000  # 16-byte aligned, never read


def _layer(**kw):
    cfg = dict(d_model=256, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ffn=256, block_size=16, num_blocks=64, max_position=4096)
    cfg.update(kw)
    return IcarusLayer(LayerConfig(**cfg), {p: A for p in binding.PROJ + ("norm_attn", "norm_ffn")})


def _refused(layer, rc, status):
    assert binding.STATUS[rc] == status, (binding.STATUS[rc], binding._lib.icarus_last_error(layer._h))


def test_beam_refusals():
    layer, call = _layer(), binding._lib.icarus_beam_select
    good = dict(x=A, dt=0, vocab=100, ld=100, R=6, G=2, W=3, rows=A + (1 << 16), scores=A + (2 << 16), done=A + (3 << 16), eos=2, p=A + (4 << 16), t=A + (5 << 16), so=A + (6 << 16),
                do=A + (7 << 16), ws=A + (8 << 16), n=binding._lib.icarus_beam_workspace_bytes(layer._h, 2, 3, 100))
    assert good["n"] > 0

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, call(layer._h, a["x"], a["dt"], a["vocab"], a["ld"], a["R"], a["G"], a["W"], a["rows"], a["scores"], a["done"], a["eos"], a["p"], a["t"], a["so"], a["do"],
                             a["ws"], a["n"], None), status)
    run("OK", G=0)
    run("INVALID_ARG", dt=2)
    for name in ("R", "G", "W", "vocab"):
        run("INVALID_ARG", **{name: -1})
    run("INVALID_ARG", W=0)
    run("UNSUPPORTED", W=65)
    run("UNSUPPORTED", G=32768, W=2)
    run("UNSUPPORTED", vocab=(1 << 24) + 1, ld=1 << 25)
    run("SHAPE", ld=99)
    run("INVALID_ARG", eos=100)
    run("INVALID_ARG", eos=-2)
    run("INVALID_ARG", eos=-1)                    # beams may be done, but as which token
    for name in ("x", "scores", "p", "t", "so", "ws"):
        run("INVALID_ARG", **{name: None})
    for name in ("x", "ws"):
        run("ALIGNMENT", **{name: good[name] + 8})
    for name in ("rows", "scores", "done", "p", "t", "so", "do"):
        run("ALIGNMENT", **{name: good[name] + 2})
    run("INVALID_ARG", p=good["scores"])
    run("INVALID_ARG", so=good["scores"] + 20)    # the scores are read while others are written
    run("INVALID_ARG", do=good["done"])
    run("INVALID_ARG", t=good["rows"] + 24)
    run("INVALID_ARG", t=good["p"] + 4)
    run("INVALID_ARG", p=good["x"] + 2396)
    run("CAPACITY", n=good["n"] - 1)
    assert binding._lib.icarus_beam_workspace_bytes(layer._h, 1, 65, 100) == 0
    assert binding._lib.icarus_beam_workspace_bytes(layer._h, -1, 1, 100) == 0
    layer.close()


def test_fork_refusals():
    layer, call = _layer(), binding._lib.icarus_fork_sequences
    good = dict(G=2, W=3, par=A, kv=A + (1 << 16), bt=A + (2 << 16), mb=10, sh=A + (3 << 16), free=A + (4 << 16), nf=50, used=A + (5 << 16), nl=A + (6 << 16), nt=A + (7 << 16),
                src=A + (8 << 16), dst=A + (9 << 16), cnt=A + (10 << 16), ws=A + (11 << 16), n=binding._lib.icarus_fork_workspace_bytes(layer._h, 2, 3, 10))

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, call(layer._h, a["G"], a["W"], a["par"], a["kv"], a["bt"], a["mb"], a["sh"], a["free"], a["nf"], a["used"], a["nl"], a["nt"], a["src"], a["dst"], a["cnt"],
                             a["ws"], a["n"], None), status)
    run("OK", G=0)
    for name in ("G", "W", "mb", "nf"):
        run("INVALID_ARG", **{name: -1})
    run("INVALID_ARG", W=0)
    run("UNSUPPORTED", W=65)
    run("UNSUPPORTED", G=65536, W=1)
    run("UNSUPPORTED", mb=(1 << 22) + 1)
    run("UNSUPPORTED", G=1000, W=2, mb=1 << 15)
    run("UNSUPPORTED", nf=(1 << 29) + 1)
    for name in ("par", "kv", "bt", "free", "used", "nl", "nt", "src", "dst", "cnt", "ws"):
        run("INVALID_ARG", **{name: None})
    for name in ("par", "kv", "bt", "sh", "free", "used", "nl", "nt", "src", "dst", "cnt"):
        run("ALIGNMENT", **{name: good[name] + 2})
    run("ALIGNMENT", ws=good["ws"] + 8)
    for o, i in itertools.product(("nl", "nt", "src", "dst", "cnt", "free"), ("par", "kv", "bt", "sh", "used")):
        run("INVALID_ARG", **{o: good[i]})
    run("INVALID_ARG", nt=good["bt"] + 4 * 59)    # in place: a parent's table is read while its child's is written
    for o, i in itertools.combinations(("nl", "nt", "src", "dst", "cnt", "free"), 2):
        run("INVALID_ARG", **{o: good[i]})
    run("CAPACITY", n=good["n"] - 1)
    assert binding._lib.icarus_fork_workspace_bytes(layer._h, 1, 65, 10) == 0
    layer.close()


def test_copy_refusals():
    layer, call = _layer(), binding._lib.icarus_copy_blocks

    def run(status, at=(A, A + 4096), size=(1024, 16), src=A, dst=A + 64, n=3, k=None):
        k = len(at) if k is None else k
        _refused(layer, call(layer._h, (C.c_void_p * len(at))(*at) if at is not None else None, (C.c_int64 * len(size))(*size) if size is not None else None, k, src, dst, n, None), status)
    run("OK", n=0)
    run("OK", k=0)
    run("INVALID_ARG", n=-1)
    run("INVALID_ARG", k=-1)
    run("UNSUPPORTED", n=(1 << 20) + 1)
    run("INVALID_ARG", src=None)
    run("INVALID_ARG", dst=None)
    run("INVALID_ARG", at=(A, None))
    run("INVALID_ARG", size=None)
    run("ALIGNMENT", src=A + 2)
    run("ALIGNMENT", dst=A + 2)
    run("ALIGNMENT", at=(A, A + 2))
    run("SHAPE", size=(1024, 0))
    run("SHAPE", size=(1024, 18))
    run("UNSUPPORTED", size=(1024, (1 << 30) + 4))
    layer.close()


def test_prefix_attention_refusals():
    layer, call = _layer(), binding._lib.icarus_attn_prefix
    good = dict(q=A, pool=A + (1 << 20), bt=A + (2 << 20), mb=10, S=4, kv=A + (3 << 20), R=8, rows=A + (4 << 20), G=2, gs=A + (5 << 20), pre=A + (6 << 20), out=A + (7 << 20), ws=A + (8 << 20),
                n=binding._lib.icarus_attn_prefix_workspace_bytes(layer._h, 4, 2, 8, 10))

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, call(layer._h, a["q"], a["pool"], a["bt"], a["mb"], a["S"], a["kv"], a["R"], a["rows"], a["G"], a["gs"], a["pre"], a["out"], a["ws"], a["n"], None), status)
    for name in ("S", "R", "G"):
        run("OK", **{name: 0})
        run("INVALID_ARG", **{name: -1})
    run("INVALID_ARG", mb=-1)
    run("UNSUPPORTED", S=65536)
    run("UNSUPPORTED", G=65536)
    run("UNSUPPORTED", R=(1 << 28) + 1)           # four queries to a kv-head
    run("UNSUPPORTED", mb=(1 << 22) + 1)
    for name in ("q", "pool", "bt", "kv", "rows", "gs", "pre", "out", "ws"):
        run("INVALID_ARG", **{name: None})
    for name in ("q", "pool", "out", "ws"):
        run("ALIGNMENT", **{name: good[name] + 8})
    for name in ("bt", "kv", "rows", "gs", "pre"):
        run("ALIGNMENT", **{name: good[name] + 2})
    run("INVALID_ARG", out=good["q"] + 8 * 8 * 64 * 2 - 16)
    run("CAPACITY", n=good["n"] - 1)
    assert binding._lib.icarus_attn_prefix_workspace_bytes(layer._h, 65536, 1, 1, 1) == 0
    layer.close()


def test_prefix_attention_workspace_of_most_parts():
    """A plan counts parts of rows in sums that stop below 2^30; sizes that could reach that are refused, and the largest below it are not."""
    layer, need = _layer(n_q_heads=1, n_kv_heads=1, head_dim=128), binding._lib.icarus_attn_prefix_workspace_bytes
    assert need(layer._h, 2, 1, 1 << 28, 10) == 0
    some = [need(layer._h, 2, 1, r << 20, 10) for r in (1, 16, 64, 128, 168)]  # 6 (R / 128) 129 parts, at most: 2^30 at R = 169.3 * 2^20
    assert all(0 < a < b for a, b in zip(some, some[1:])) and some[-1] < (1 << 30) * (128 * 4 + 8) * 1.01
    layer.close()


def test_binding_refuses_tensors_of_the_host():
    layer = _layer()
    beams, forked = binding.BeamMap(2, 3, "cpu"), binding.ForkMap(2, 3, 4, "cpu")
    i, f = torch.zeros(6, dtype=torch.int32), torch.zeros(6)
    for call in (lambda: layer.beam_select(torch.zeros(6, 10), f, beams), lambda: layer.fork_sequences(i, i, torch.zeros(6, 4, dtype=torch.int32), forked, i, i[:1]),
                 lambda: layer.copy_blocks([], i, i), lambda: layer.attn_prefix(torch.zeros(2, 8, 64, dtype=torch.bfloat16), None, torch.zeros(2, 4, dtype=torch.int32), i, i, i, i)):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(TypeError):
        layer.beam_select(torch.zeros(6, 10, dtype=torch.float16), f, beams)
    layer.close()


# ---- the references --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("seed", range(6))
def test_reference_of_the_choice(seed):
    """Against all continuations, sorted."""
    rng = np.random.default_rng(seed)
    G, W, V, eos = 3, 4, 9, 5
    x = rng.standard_normal((G * W, V)).round(1 if seed % 2 else 6).astype(np.float32)
    x[rng.random(x.shape) < 0.2] = -np.inf
    scores = (-3 * rng.random(G * W)).astype(np.float32)
    scores[1] = -np.inf
    done = (rng.random(G * W) < 0.3).astype(int)
    p, t, v, d, _ = ref.choose(x, None, scores, done, eos, G, W)
    for g in range(G):
        every = []
        for b in range(W):
            s = g * W + b
            if scores[s] == -np.inf:
                continue
            y = x[s].astype(float)
            with np.errstate(divide="ignore"):
                lp = y - y.max() - np.log(np.exp(y - y.max()).sum())
            every += [(scores[s], b, eos)] if done[s] else [(scores[s] + lp[k], b, k) for k in range(V) if lp[k] > -np.inf]
        every.sort(key=lambda e: (-round(e[0], 9), e[1], e[2]))
        for i in range(W):
            s = g * W + i
            if i >= len(every):
                assert (p[s], t[s], v[s], d[s]) == (-1, -1, -math.inf, 0)
                continue
            assert (p[s], t[s]) == every[i][1:] and abs(v[s] - every[i][0]) < 1e-9
            assert d[s] == (done[g * W + p[s]] != 0 or t[s] == eos)


@pytest.mark.parametrize("seed", range(8))
def test_reference_of_the_fork(seed):
    """Every block of the pool is free, in the common prefix, or in some table; children hold their parents' tokens; no block that a child still fills is in two tables."""
    rng = np.random.default_rng(seed)
    G, W, bk, mb, shared = 3, 4, 4, 12, 2
    num = G * (shared + W * mb)
    ids = list(rng.permutation(num))
    table, kv = np.full((G * W, mb), -9), np.zeros(G * W, dtype=int)
    prefix = [[ids.pop() for _ in range(shared)] for _ in range(G)]
    text = {b: [("p", b, j) for j in range(bk)] for pre in prefix for b in pre}
    for g in range(G):
        apart = int(rng.integers(shared, mb - 1))
        trunk = [ids.pop() for _ in range(apart - shared)]
        for i in range(W):
            s = g * W + i
            kv[s] = rng.integers(apart * bk, mb * bk + 1)
            own = [ids.pop() for _ in range(ref.blocks_of(kv[s], bk) - apart)]
            row = prefix[g] + trunk + own
            table[s, :len(row)] = row
    for b in range(num):
        text.setdefault(b, [(b, j) for j in range(bk)])
    used = num - len(ids)
    free = np.concatenate([np.full(used, -5), np.array(ids, dtype=int)])
    parents = rng.integers(-1, W, G * W)
    got = ref.fork(parents, kv, table, np.full(G, shared), free, used, bk, num, W, np.full((G * W, mb), -9))
    assert got["counts"][1] == 0
    for s, d in zip(got["copy_src"], got["copy_dst"]):
        if s >= 0:
            text[int(d)] = list(text[int(s)])

    def words(t, n):
        return [text[int(t[p // bk])][p % bk] for p in range(n)]
    live, last = set(), []
    for s in range(G * W):
        n, P = got["kv_lens"][s], s // W * W + parents[s]
        assert n == (kv[P] if parents[s] >= 0 else 0)
        row = got["block_tables"][s, :ref.blocks_of(n, bk)]
        live |= set(row.tolist())
        last += [int(row[-1])] if n % bk else []
        if n:
            old = [("x", int(b), j) for b in table[P] for j in range(bk)]
            assert len(words(row, n)) == n and len(old) >= n
            assert [w for w in words(row, n)] == [w for w in words(table[P], n)]
    assert len(last) == len(set(last))
    left = set(got["free"][got["counts"][0]:].tolist())
    assert len(left) == num - got["counts"][0] and not left & live
    assert left | live | {b for pre in prefix for b in pre} == set(range(num))


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("samples", [False, True])
def test_reference_of_forks_from_one_prompt(samples, seed):
    """Beams (children of one live sequence) and samples (each its own parent, the prompt's last block a shared column for the first fork) of a prompt that ends inside a block: no block
    that a child fills is in two tables or the prompt's, and every block is the prompt's, in a table, or free."""
    rng = np.random.default_rng(seed)
    W, bk, cols, num = 5, 4, 12, 90
    n = 4 * bk + int(rng.integers(1, bk))
    ids = rng.permutation(num)
    table = np.full((W, cols), -1)
    table[:, :5] = ids[:5]
    prompt = set(ids[:5 if samples else 4].tolist())
    kv, free, used, parents, shared = np.full(W, n), ids, 5, np.arange(W) if samples else np.zeros(W, dtype=int), 5 if samples else 4
    for step in range(8):
        got = ref.fork(parents, kv, table, np.array([shared]), free, used, bk, num, W, np.full((W, cols), -1))
        kv, table, free, used = got["kv_lens"].copy(), got["block_tables"].copy(), got["free"], int(got["counts"][0])
        filled = [int(table[s, kv[s] // bk]) for s in range(W) if kv[s] % bk]
        assert len(filled) == len(set(filled)) and not prompt & set(filled), step
        for s in np.flatnonzero((kv > 0) & (kv < cols * bk)):
            if kv[s] % bk == 0:
                table[s, kv[s] // bk] = free[used]
                used += 1
            kv[s] += 1
        held = {int(b) for s in range(W) for b in table[s, :ref.blocks_of(kv[s], bk)]}
        left = free[used:].tolist()
        assert len(left) == len(set(left)) and not (held | prompt) & set(left) and held | prompt | set(left) == set(range(num)), step
        parents, shared = rng.integers(-1, W, W), 4
