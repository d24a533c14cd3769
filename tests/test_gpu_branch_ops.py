"""The operators of include/icarus_branches.h on the GPU against plain float64 (branch_reference.py), at the sizes and contents where they can go
wrong.  Whole numbers and copied bytes are equal; floats are within bounds that are derived beside them."""
import math

import numpy as np
import pytest
import torch

import branch_reference as ref
from block_reference import blocks_of
from paper_2603_13281_amd import binding
from test_gpu_block_ops import DEV, E24, host, i32, make, pool_values, random_pool

pytestmark = pytest.mark.gpu


# ---- choice of the continuations ----------------------------------------------------------------------------------------

def run_choose(layer, logits, groups, width, scores, row_start=None, done=None, eos=-1):
    beams = binding.BeamMap(groups, width, DEV)
    for t in (beams.parents, beams.tokens, beams.done):
        t.fill_(-77)
    beams.scores.fill_(7.0)
    layer.beam_select(logits, torch.tensor(scores, dtype=torch.float32, device=DEV), beams, None if row_start is None else i32(row_start), None if done is None else i32(done), eos)
    torch.cuda.synchronize()
    p, t, v, d, gaps = ref.choose(host(logits), row_start, np.asarray(scores, dtype=np.float32), done, eos, groups, width)
    # A sum of exponentials, each to 2^-37, and its logarithm are off by less than 2^-36 and 2^-50 of the numbers added: where no two candidates of different beams are nearer than
    # 2^-30 the order is the reference's.
    assert all(x == 0.0 or x > 2.0 ** -30 for x in gaps)
    got = [x.cpu().numpy() for x in (beams.parents, beams.tokens, beams.done)]
    for a, b, name in zip(got, (p, t, d), ("parents", "tokens", "done")):
        assert np.array_equal(a, b), (name, np.argwhere(a != b)[:5].ravel(), a[:20], b[:20])
    s = host(beams.scores)
    there = p >= 0
    assert (s[~there] == -math.inf).all()
    assert (np.abs(s[there] - v[there]) <= E24 * np.abs(v[there]) + 2.0 ** -34).all()
    return beams


def words(rng, rows, vocab, dt):
    x = rng.standard_normal((rows, vocab)) * 2
    top = rng.integers(0, vocab, (rows, 20))
    np.put_along_axis(x, top, np.take_along_axis(x, top, 1) + 9 * rng.random(top.shape), 1)
    return torch.tensor(x, dtype=torch.float32).to(dt).to(DEV)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("groups,width,vocab", [(1, 1, 1), (2, 3, 2), (1, 64, 5), (3, 5, 301), (1, 4, 2048), (2, 64, 4099), (5, 2, 8193), (20, 3, 50021), (2, 16, 128256)])
def test_choose(groups, width, vocab, dt):
    print("case:", groups, width, vocab, dt, flush=True)
    layer, rng = make(), np.random.default_rng(vocab + width)
    S = groups * width
    logits = words(rng, S, vocab, dt)
    scores = -20 * rng.random(S)
    run_choose(layer, logits, groups, width, scores)
    eos = vocab // 2
    run_choose(layer, logits, groups, width, scores, done=(rng.random(S) < 0.3).astype(int), eos=eos)
    start = np.concatenate([[0], np.cumsum(rng.integers(0, 4, S))])       # some beams have no row, the others take their last
    run_choose(layer, words(rng, int(start[-1]) + 1, vocab, dt), groups, width, scores, row_start=start, eos=eos)
    layer.close()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("vocab,gap", [(5000, 3), (5000, 1), (4096, 64), (333, 0)])
def test_choose_strided_rows(vocab, gap, dt):
    """Rows at any distance, what lies between them is not read as logits."""
    layer, rng = make(), np.random.default_rng(gap)
    whole = torch.full((9, vocab + gap), 1e30, dtype=dt, device=DEV)
    logits = whole[:, :vocab]
    logits.copy_(words(rng, 9, vocab, dt))
    run_choose(layer, logits, 3, 3, -5 * rng.random(9))
    layer.close()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("vocab", [7, 1000, 20000])
def test_choose_equal_logits(vocab, dt):
    """Beams and tokens that tie: the lowest beam, then the lowest token; more of them than a workgroup lists."""
    layer, rng = make(), np.random.default_rng(vocab)
    same = torch.zeros(8, vocab, dtype=dt, device=DEV)
    run_choose(layer, same, 2, 4, [-1.0] * 8)
    same[:, ::2] = -0.0                                                   # equal to 0
    run_choose(layer, same, 2, 4, [-1.0, -1.0, -2.0, -1.0] * 2)
    few = torch.tensor(rng.integers(0, 3, (1, vocab)), dtype=dt, device=DEV).expand(8, vocab).contiguous()
    run_choose(layer, few, 2, 4, [-1.0, -3.0, -1.0, -1.0] * 2)
    run_choose(layer, few[:1], 1, 1, [0.0])
    run_choose(layer, few.repeat(8, 1), 1, 64, [-1.0] * 64)
    layer.close()


def test_choose_logits_far_from_zero():
    """Rows around the size where a part needs more care, lowest numbers beside ordinary ones."""
    layer, rng = make(), np.random.default_rng(9)
    for offset in (0.0, 4000.0, 8180.0, 8200.0, -8180.0, -8300.0, 1e6, -1e6):
        x = words(rng, 6, 20011, torch.float32) + offset
        x[1, ::3] = -1e6
        x[2, 5:9000] = -3.4028234e38
        x[3, 17] = -float("inf")
        x[4, 8000] = float("nan")
        run_choose(layer, x, 2, 3, -rng.random(6))
    layer.close()


def test_choose_masked_logits():
    """Minus infinity, NaN and plus infinity among the logits; beams that are not live; fewer continuations than beams."""
    layer, rng = make(), np.random.default_rng(0)
    inf, nan = float("inf"), float("nan")
    x = words(rng, 12, 3000, torch.float32)
    x[0] = -inf
    x[1, 5:] = -inf
    x[2] = nan
    x[3, 100] = nan
    x[4, 17], x[4, 2900] = inf, inf
    x[5, 1:] = -inf
    x[6] = -inf
    x[7] = -inf
    x[8] = -3e38
    x[9] *= 1e30
    x[10] = -inf
    x[10, 2999] = -1e20
    x[11] = inf
    run_choose(layer, x, 3, 4, -rng.random(12))
    scores = -rng.random(12)
    scores[[0, 4, 5, 9]] = -inf, inf, nan, -inf
    run_choose(layer, x, 3, 4, scores)
    run_choose(layer, x, 1, 12, scores, done=np.arange(12) % 3, eos=2999)
    run_choose(layer, x, 12, 1, scores, done=np.ones(12, dtype=int), eos=0)
    only = torch.full((4, 3000), -inf, device=DEV)
    only[:, 0::1024] = 0.5                                               # a few tokens that fall to one thread
    run_choose(layer, only, 1, 4, [-1.0, -2.0, -1.5, -1.0])
    run_choose(layer, torch.full((4, 3000), -inf, device=DEV), 1, 4, [-1.0] * 4)
    run_choose(layer, x[:0], 1, 4, [-1.0] * 4)
    run_choose(layer, x, 2, 4, [-1.0] * 8, row_start=np.array([0, 1, 1, -3, 2, 40, 41, 3, 12]))  # rows outside are none
    layer.close()


@pytest.mark.parametrize("dt,patterns", [(torch.float32, (0x7f800001, 0x7fbfffff, 0x7fc00000, -0x7fffff, -0x400001)), (torch.bfloat16, (0x7f81, 0x7fbf, 0x7fc0, -0x7f, -0x41))], ids=str)
def test_choose_every_kind_of_nan(dt, patterns):
    """Signalling and quiet ones of either sign count as minus infinity, in the middle of a row and at its end, and where they are all that there is."""
    layer, rng = make(), np.random.default_rng(4)
    x = words(rng, 2 * len(patterns), 4099, dt)
    bits = x.view(torch.int32 if dt is torch.float32 else torch.int16)
    for i, p in enumerate(patterns):
        bits[i, [0, 77, 2048, 4096, 4098]] = p
        bits[len(patterns) + i, :] = p
    assert torch.isnan(x[:5, 77]).all() and torch.isnan(x[5:]).all()
    run_choose(layer, x, 2, len(patterns), -rng.random(len(x)))
    run_choose(layer, x, len(x), 1, -rng.random(len(x)))
    layer.close()


def test_choose_without_a_row():
    """An array of no rows, whatever its strides are."""
    layer = make()
    for logits in (torch.zeros(0, 9, device=DEV), torch.zeros(9, 0, device=DEV).t(), torch.tensor(np.zeros((0, 9)), dtype=torch.bfloat16).to(DEV)):
        run_choose(layer, logits, 2, 2, [-1.0] * 4)
        run_choose(layer, logits, 2, 2, [-1.0] * 4, row_start=np.zeros(5, dtype=int))
    layer.close()


def last_rows(logits, row_start, scores, done):
    """What a choice among beams of which some have no row is, as one among beams that all have one: a finished beam needs none, another one without is not live."""
    rows = [ref.beam_row(row_start, s, len(logits)) for s in range(len(scores))]
    x = np.stack([logits[r] if r >= 0 else np.zeros(logits.shape[1]) for r in rows])
    return x, np.array([v if r >= 0 or d else -math.inf for v, r, d in zip(scores, rows, done)], dtype=np.float32)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("groups,width,vocab", [(1, 1, 9), (3, 4, 3001), (2, 20, 20011)])
def test_choose_finished_beams_without_rows(groups, width, vocab, dt):
    """A finished beam is its own continuation whether it has a row of logits or not, and where its row lies outside; a live one without a row has none."""
    print("case:", groups, width, vocab, dt, flush=True)
    layer, rng = make(), np.random.default_rng(width)
    S = groups * width
    done = (np.arange(S) % 3 == 0).astype(int)
    for start in (np.concatenate([[0], np.cumsum(np.where(done, 0, rng.integers(0, 3, S)))]), np.zeros(S + 1, dtype=int), np.concatenate([[0], np.where(done, 10 ** 6, np.arange(S)) + 1])):
        scores = (-20 * rng.random(S)).astype(np.float32)
        if S > 6:
            scores[6] = -math.inf                                          # finished, and not live all the same
        logits = words(rng, int(start[start < 10 ** 6].max()), vocab, dt)
        x, live = last_rows(host(logits), start, scores, done)
        p, t, v, d, gaps = ref.choose(x, None, live, done, 2, groups, width)
        assert all(g == 0.0 or g > 2.0 ** -30 for g in gaps)
        beams = binding.BeamMap(groups, width, DEV)
        layer.beam_select(logits, torch.tensor(scores, device=DEV), beams, row_start=i32(start), done=i32(done), eos=2)
        for got, want in zip((beams.parents, beams.tokens, beams.done), (p, t, d)):
            assert np.array_equal(got.cpu().numpy(), want), (got, want)
        assert (p >= 0).sum() >= (S > 1) and np.allclose(host(beams.scores)[p >= 0], v[p >= 0], rtol=2.0 ** -23, atol=2.0 ** -34)
    layer.close()


# ---- children -------------------------------------------------------------------------------------------------------------

def run_fork(layer, parents, kv, table, shared, free, used, width):
    c, (S, max_blocks) = layer.cfg, table.shape
    want = ref.fork(parents, kv, table, shared, free, used, c.block_size, c.num_blocks, width, np.full(table.shape, -77))
    m = binding.ForkMap(S // width, width, max_blocks, DEV)
    for t in (m.kv_lens, m.copy_src, m.copy_dst, m.counts, m.block_tables):
        t.fill_(-77)
    f = i32(free)
    layer.fork_sequences(i32(parents), i32(kv), i32(table).reshape(table.shape), m, f, i32([used]), None if shared is None else i32(shared))
    torch.cuda.synchronize()
    for name in ("kv_lens", "counts", "copy_src", "copy_dst", "block_tables"):
        got = getattr(m, name).cpu().numpy()
        assert np.array_equal(got, want[name]), (name, np.argwhere(got != want[name])[:5], got.ravel()[:30], want[name].ravel()[:30])
    assert np.array_equal(f.cpu().numpy(), want["free"]), (f.cpu().numpy()[:40], want["free"][:40])
    return want


def family(rng, groups, width, max_blocks, bk, shared):
    """Tables of sequences that came apart somewhere, the number of blocks in use, and their lengths."""
    S, at = groups * width, 0
    table, kv = np.full((S, max_blocks), -1), np.zeros(S, dtype=int)
    for g in range(groups):
        trunk = np.arange(at, at + max_blocks)
        at += max_blocks
        for i in range(width):
            n = int(rng.integers(0, max_blocks * bk + 1))
            nb, apart = blocks_of(n, bk), int(rng.integers(0, max_blocks + 1))
            s = g * width + i
            kv[s] = n
            table[s, :nb] = trunk[:nb]
            apart = max(apart, shared)
            if apart < nb:
                table[s, apart:nb] = np.arange(at, at + nb - apart)
                at += nb - apart
    ids = rng.permutation(at)
    return np.where(table >= 0, ids[table], -1), kv, at


@pytest.mark.parametrize("bk", [1, 16, 7])
@pytest.mark.parametrize("groups,width,max_blocks,shared", [(1, 1, 1, 0), (3, 4, 5, 2), (1, 64, 130, 60), (7, 8, 129, 0), (40, 3, 20, 19), (2, 5, 600, 300), (300, 2, 3, 1), (5, 9, 140, 30), (3, 16, 260, 100), (2, 17, 129, 64), (64, 8, 140, 100), (3, 24, 300, 50), (2, 32, 140, 0), (2, 33, 200, 0), (4, 64, 150, 10), (1100, 2, 3, 0)])
def test_fork(groups, width, max_blocks, shared, bk):
    print("case:", groups, width, max_blocks, shared, bk, flush=True)
    rng = np.random.default_rng(groups + bk)
    table, kv, used = family(rng, groups, width, max_blocks, bk, shared)
    S = groups * width
    layer = make(bk=bk, num_blocks=used + S + 3)
    free = rng.permutation(used + S)
    for parents in (rng.integers(0, width, S), rng.integers(-1, width + 1, S), np.zeros(S, dtype=int), np.full(S, -1), np.arange(S) % width):
        run_fork(layer, parents, kv, table, np.full(groups, shared), free, used, width)
        run_fork(layer, parents, kv, table, None, free, used, width)
    layer.close()


def test_fork_where_blocks_run_out():
    """Children that find no block are refused, in the order of the sequences; freed ids are there for them; ids that the list has no room for are left out."""
    rng = np.random.default_rng(1)
    table, kv, used = family(rng, 9, 6, 30, 16, 4)
    layer = make(num_blocks=used + 5)
    parents = rng.integers(0, 3, 54)
    for n_free, head in ((used, used), (used + 4, used), (used + 4, used + 4), (10, 3), (10, 10), (0, 0), (used, -7), (used, used + 1000), (40, 40), (400, 0)):
        print("case:", n_free, head, flush=True)
        run_fork(layer, parents, kv, table, rng.integers(-2, 8, 9), rng.integers(0, used + 5, n_free), head, 6)
        run_fork(layer, np.zeros(54, dtype=int), kv, table, None, rng.integers(0, used + 5, n_free), head, 6)
    layer.close()


def test_fork_of_what_is_out_of_range():
    """Lengths below 0 and beyond the table, parents and ids outside, shared columns beyond the table."""
    rng = np.random.default_rng(2)
    table, kv, used = family(rng, 6, 5, 40, 16, 0)
    kv[[0, 7, 12]] = -5, 10 ** 9, 40 * 16 + 1
    table[7] = rng.integers(0, used, 40)
    table[rng.random(table.shape) < 0.1] = -3
    table[rng.random(table.shape) < 0.1] = used + 99
    layer = make(num_blocks=used)
    free = rng.integers(-2, used + 4, used + 50)
    for seed in range(4):
        parents = rng.integers(-2, 7, 30)
        parents[seed] = 2 ** 31 - 1
        run_fork(layer, parents, kv, table, rng.integers(-1, 45, 6), free, used, 5)
    run_fork(layer, rng.integers(0, 5, 30), kv, np.zeros((30, 0), dtype=int), None, free, 20, 5)
    layer.close()


# ---- copies ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(fp8=True), dict(D=64, Hq=4, Hkv=4, bf16=False), dict(D=20, Hkv=1, bk=3)], ids=str)
@pytest.mark.parametrize("n", [1, 9, 700])
def test_copy(kw, n):
    print("case:", kw, n, flush=True)
    layer, rng = make(num_blocks=2 * n + 5, **kw), np.random.default_rng(n)
    c = layer.cfg
    perm = rng.permutation(2 * n + 5)
    src, dst = perm[:n].copy(), perm[n:2 * n].copy()
    if n > 5:
        src[1], dst[2], src[3], dst[4] = -1, -1, 2 * n + 5, 2 ** 31 - 1
        dst[5] = src[5]
    spare = torch.randint(0, 256, (4 * (2 * n + 5) * 12 + 4,), dtype=torch.uint8, device=DEV)
    arrays = [random_pool(layer, rng) for _ in range(3)] + [torch.randint(-127, 127, (2 * n + 5, 2, 2, c.head_dim), dtype=torch.int8, device=DEV), torch.rand(2 * n + 5, 2, device=DEV),
                                                            torch.rand(2 * n + 5, device=DEV), spare[4:].view(2 * n + 5, 48), torch.rand(2 * n + 9, 4099, device=DEV)]
    want = [t.clone() for t in arrays]
    for t in want:
        for s, d in zip(src, dst):
            if 0 <= s < 2 * n + 5 and 0 <= d < 2 * n + 5:
                t[d] = t[s].clone()
    layer.copy_blocks(arrays, i32(src), i32(dst))
    torch.cuda.synchronize()
    for a, b in zip(arrays, want):
        assert torch.equal(a.reshape(-1).view(torch.uint8), b.reshape(-1).view(torch.uint8))
    layer.copy_blocks([], i32(src), i32(dst))
    layer.copy_blocks(arrays, i32([]), i32([]))
    layer.close()


def test_copy_many_arrays_and_large_blocks():
    layer = make(num_blocks=4)
    arrays = [torch.rand(4, 5, device=DEV) for _ in range(130)] + [torch.randint(0, 100, (4, 1 << 22), dtype=torch.int32, device=DEV)]
    want = [t.clone() for t in arrays]
    for t in want:
        t[3] = t[0]
    layer.copy_blocks(arrays, i32([0, -1]), i32([3, 1]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(arrays, want))
    layer.close()


# ---- attention over a shared prefix -------------------------------------------------------------------------------------------

def bound(layer, want, weight, size, count):
    """A score is a sum of D products in float32 (D half steps of the sum of sizes, and 3 for the scale and the code's scale): off by ds, so each p by 2 ds of itself (its own and the
    sum's); exp, its argument (below 2^7 where p counts) and the sums over up to n tokens: 2^-17 + n 2^-24, all of sum p |v|.  On the matrix cores a weight is two numbers of
    bfloat16 (2^-15 of sum p |v| more), over an FP8 cache one of float16 (2^-11)."""
    c = layer.cfg
    ds = (c.head_dim + 3) * E24 * size
    return (2.0 ** -8 if c.bf16 else E24) * np.abs(want) + weight * (2 * ds + 2.0 ** -17 + count * E24 + (0.0 if not c.bf16 else 2.0 ** -11 if c.kv_fp8 else 2.0 ** -15)) + 1e-30


def both_widths(table, bk):
    """The table, and the same one with columns of no block behind it: one of at most 1024 tokens may be read in one launch, wider ones are cut into items."""
    return [table, np.concatenate([table, np.full((len(table), 1024 // bk + 1), -1)], axis=1)]


def run_attend(layer, q, pool, table, kv, row_start, group_start, prefix):
    c = layer.cfg
    want, weight, size, count = ref.attend(host(q), pool_values(layer, pool), table, kv, row_start, group_start, c.block_size, np.full(q.shape, 7.0))
    outs = []
    for t in both_widths(table, c.block_size):
        outs.append(torch.full(q.shape, 7.0, dtype=c.torch_dtype, device=DEV))
        layer.attn_prefix(q, pool, i32(t).reshape(t.shape), i32(kv), i32(row_start), i32(group_start), i32(prefix), outs[-1])
        torch.cuda.synchronize()
        got = host(outs[-1])
        ok = np.abs(got - want) <= bound(layer, want, weight, size, count)
        assert ok.all(), (t.shape, np.argwhere(~ok)[:5], np.argwhere(~ok).shape, np.nanmax(np.abs(got - want)))
    return outs


def blocks_that_may_be_read(layer, pool, table, kv):
    """Everything else becomes NaN."""
    c = layer.cfg
    seen = np.zeros((c.num_blocks, c.block_size), dtype=bool)
    for row, n in zip(table, kv):
        n = min(max(int(n), 0), len(row) * c.block_size)
        for i in range(blocks_of(n, c.block_size)):
            if 0 <= row[i] < c.num_blocks:
                seen[row[i], :n - i * c.block_size] = True
    gone = torch.tensor(~seen, device=DEV)
    nan = torch.tensor(float("nan")).to(torch.float8_e4m3fn).view(torch.uint8).item() if c.kv_fp8 else float("nan")
    pool.view(c.num_blocks, c.n_kv_heads, 2, c.block_size, c.head_dim)[:, :, 0].masked_fill_(gone[:, None, :, None], nan)
    pool.view(c.num_blocks, c.n_kv_heads, 2, c.head_dim, c.block_size)[:, :, 1].masked_fill_(gone[:, None, None, :], nan)


def crowd(layer, rng, groups, max_blocks):
    """groups: (rows of each sequence, tokens of the prefix, tails).  Tables that share the prefix's whole blocks, lengths, row_start, group_start, prefix lengths."""
    bk, at, table, kv, rows, start = layer.cfg.block_size, 0, [], [], [], [0]
    ids = rng.permutation(layer.cfg.num_blocks)
    for n_rows, pre, tails in groups:
        whole = ids[at:at + pre // bk]
        at += pre // bk
        for r, t in zip(n_rows, tails):
            nb = blocks_of(pre + t, bk) - pre // bk if t >= 0 else 0
            row = np.full(max_blocks, -1)
            row[:pre // bk] = whole
            row[pre // bk:pre // bk + nb] = ids[at:at + nb]
            at += nb
            table.append(row)
            kv.append(pre + t if t >= 0 else 0)
            rows.append(r)
        start.append(len(table))
    assert at <= layer.cfg.num_blocks
    return np.array(table), np.array(kv), np.concatenate([[0], np.cumsum(rows)]), np.array(start), np.array([g[1] for g in groups])


def queries(layer, rng, rows, size=1.0):
    c = layer.cfg
    return torch.tensor(rng.standard_normal((rows, c.n_q_heads, c.head_dim)) * size, dtype=torch.float32).to(c.torch_dtype).to(DEV)


SHAPES = [dict(), dict(Hq=4, Hkv=4), dict(Hq=32, Hkv=8), dict(fp8=True, k_scale=0.5, v_scale=0.25), dict(Hq=16, Hkv=2, fp8=True, k_scale=0.05, v_scale=0.03), dict(Hq=40, Hkv=2), dict(Hq=3, Hkv=1),
          dict(D=64), dict(Hq=4, Hkv=4, D=64, bf16=False), dict(bf16=False), dict(D=80), dict(D=256), dict(D=112, bf16=False), dict(D=64, fp8=True, k_scale=2.0), dict(bf16=False, fp8=True, v_scale=0.5),
          dict(D=256, bf16=False, fp8=True), dict(bk=32), dict(bk=48, fp8=True, k_scale=0.3), dict(bk=64, bf16=False), dict(bk=128, D=64), dict(mode=1), dict(bk=5, D=30), dict(bk=8)]


@pytest.mark.parametrize("kw", SHAPES, ids=str)
def test_attend(kw):
    """Groups of one and of many, prefixes that end inside a block, at its end and at zero, tails of nothing and of many blocks, sequences that are empty or have no rows;
    everything that must not be read holds NaN."""
    print("case:", kw, flush=True)
    layer = make(num_blocks=400, **kw)
    bk, rng = layer.cfg.block_size, np.random.default_rng(3)
    pool = random_pool(layer, rng)
    groups = [([1], 0, [1]), ([2, 1, 3], 5 * bk, [0, 1, bk]), ([1] * 17, 9 * bk + bk // 2, list(range(17))), ([4, 0, 2], 3 * bk - 1, [2 * bk, 5, 7 * bk + 1]), ([2, 2], 0, [-1, -1]),
              ([1, 5, 1, 1], 12 * bk, [3, -1, 0, 20 * bk]), ([9, 9, 9], 70 * bk + 1, [1, 9 * bk, 33]), ([0, 0], 2 * bk, [1, 1]), ([30], 6 * bk, [17])]
    table, kv, row_start, group_start, prefix = crowd(layer, rng, groups, 90)
    blocks_that_may_be_read(layer, pool, table, kv)
    q = queries(layer, rng, int(row_start[-1]) + 2, 2.0)
    run_attend(layer, q, pool, table, kv, row_start, group_start, prefix)
    run_attend(layer, q, pool, table, kv, row_start, group_start, np.zeros_like(prefix))                 # nothing is shared
    run_attend(layer, q, pool, table, kv, row_start, group_start, np.maximum(prefix - bk, -3))
    run_attend(layer, q, pool, table, kv, row_start, group_start[2:5], prefix[2:4])                      # the other sequences are in no group
    run_attend(layer, q, pool, table, kv, row_start, np.arange(len(kv) + 1), kv)                         # every sequence for itself, all of it shared
    layer.close()


@pytest.mark.parametrize("kw", [dict(Hq=32, Hkv=8), dict(Hq=8, Hkv=1, fp8=True), dict(Hq=8, Hkv=4, bf16=False), dict(Hq=8, Hkv=1, D=64)], ids=str)
@pytest.mark.parametrize("n,rows", [(1, 1), (2, 8), (5, 3), (33, 1), (40, 4), (70, 5)])
def test_attend_crowds(kw, n, rows):
    """Numbers of queries around those of a tile, a wave and a workgroup, over one long prefix."""
    print("case:", kw, n, rows, flush=True)
    layer = make(num_blocks=700, **kw)
    rng = np.random.default_rng(n)
    pool = random_pool(layer, rng)
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([rows] * n, 4000 + n, [int(t) for t in rng.integers(0, 60, n)])], 260)
    blocks_that_may_be_read(layer, pool, table, kv)
    run_attend(layer, queries(layer, rng, n * rows, 2.0), pool, table, kv, row_start, group_start, prefix)
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True), dict(D=64, bf16=False), dict(mode=1)], ids=str)
def test_attend_many_groups(kw):
    layer = make(num_blocks=3000, **kw)
    rng = np.random.default_rng(5)
    pool = random_pool(layer, rng)
    groups = [([int(r) for r in rng.integers(0, 4, n)], int(rng.integers(0, 200)), [int(t) for t in rng.integers(-1, 40, n)]) for n in rng.integers(0, 5, 180)]
    table, kv, row_start, group_start, prefix = crowd(layer, rng, groups, 20)
    run_attend(layer, queries(layer, rng, int(row_start[-1])), pool, table, kv, row_start, group_start, prefix)
    layer.close()


@pytest.mark.parametrize("kw,tokens", [(dict(), 1024), (dict(fp8=True), 1024), (dict(bf16=False), 512), (dict(D=64), 512)], ids=str)
@pytest.mark.parametrize("beyond", [0, 1])
@pytest.mark.parametrize("n,rows", [(3, 1), (1, 70), (130, 1)])
def test_attend_tables_as_wide_as_one_launch_takes(kw, tokens, beyond, n, rows):
    """And one column wider; many rows of a sequence, many sequences, tables that are full."""
    layer = make(num_blocks=1000, Hq=32, Hkv=8, **kw)
    rng = np.random.default_rng(n)
    pool = random_pool(layer, rng)
    cols, apart = tokens // 16 + beyond, min(5, 900 // n)
    tails = [int(t) for t in rng.integers(0, apart * 16 + 1, n)]
    tails[-1] = apart * 16
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([rows] * n, (cols - apart) * 16, tails)], cols)
    run_attend(layer, queries(layer, rng, n * rows, 2.0), pool, table, kv, row_start, group_start, prefix)
    layer.close()


@pytest.mark.parametrize("kw", [dict(Hq=4, Hkv=1), dict(Hq=4, Hkv=1, fp8=True), dict(Hq=2, Hkv=1, D=64)], ids=str)
@pytest.mark.parametrize("n,groups", [(256, 1), (257, 3), (512, 200), (513, 40), (1100, 1), (1500, 700)])
def test_attend_many_sequences(kw, n, groups):
    """Counts of sequences around those that a plan holds to a thread."""
    print("case:", kw, n, groups, flush=True)
    layer = make(num_blocks=6000, **kw)
    rng = np.random.default_rng(n)
    pool = random_pool(layer, rng)
    parts = np.diff(np.concatenate([[0], np.sort(rng.integers(0, n + 1, groups - 1)), [n]]))
    spec = [([int(r) for r in rng.integers(0, 3, m)], int(rng.integers(0, 40)), [int(t) for t in rng.integers(-1, 33, m)]) for m in parts]
    spec[0] = (spec[0][0], 16 * 60 + 3, spec[0][2])
    table, kv, row_start, group_start, prefix = crowd(layer, rng, spec, 66)
    run_attend(layer, queries(layer, rng, int(row_start[-1])), pool, table, kv, row_start, group_start, prefix)
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True, k_scale=0.5), dict(bf16=False)], ids=str)
def test_attend_large_scores(kw):
    """Scores in the hundreds: the running maximum moves, and one part's sums are nothing beside another's."""
    layer = make(num_blocks=200, Hq=8, Hkv=2, **kw)
    rng = np.random.default_rng(0)
    pool = random_pool(layer, rng)
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([3, 3, 3], 1500, [40, 200, 0])], 120)
    run_attend(layer, queries(layer, rng, 9, 30.0), pool, table, kv, row_start, group_start, prefix)
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(bf16=False), dict(D=64), dict(mode=1)], ids=str)
def test_attend_scores_of_minus_infinity(kw):
    """Keys whose scores are minus infinity weigh nothing; a row with no others becomes zeros; NaN and plus infinity make NaN, for the rows that see them."""
    layer = make(num_blocks=100, Hq=8, Hkv=2, **kw)
    c, rng = layer.cfg, np.random.default_rng(2)
    pool = random_pool(layer, rng)
    q = queries(layer, rng, 6)
    q[:, :, 0] = 1.0
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([2, 2, 2], 320, [0, 100, 40])], 30)
    keys = pool.view(100, 2, 2, 16, c.head_dim)[:, :, 0]
    keys[torch.tensor(table[0, :20].copy(), device=DEV), :, :, 0] = -float("inf")   # the whole prefix
    run_attend(layer, q, pool, table, kv, row_start, group_start, prefix)
    keys[int(table[1, 22]), :, :, 0] = -float("inf")
    run_attend(layer, q, pool, table, kv, row_start, group_start, prefix)
    for t in both_widths(table, 16):
        out = torch.zeros_like(q)
        keys[int(table[2, 21]), 1, 3, 5] = float("nan")
        layer.attn_prefix(q, pool, i32(t), i32(kv), i32(row_start), i32(group_start), i32(prefix), out)
        bad = torch.isnan(out.float()).any(-1).cpu().numpy()
        assert bad[4:, 4:].all() and not bad[:4].any() and not bad[4:, :4].any()
        keys[int(table[2, 21]), 1, 3, 5] = 0.0
        was = keys[int(table[0, 3]), 0, 3, 0].clone()
        keys[int(table[0, 3]), 0, 3, 0] = float("inf")
        layer.attn_prefix(q, pool, i32(t), i32(kv), i32(row_start), i32(group_start), i32(prefix), out)
        bad = torch.isnan(out.float()).any(-1).cpu().numpy()
        assert bad[:, :4].all() and not bad[:, 4:].any()
        keys[int(table[0, 3]), 0, 3, 0] = was
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(D=64, bf16=False), dict(mode=1)], ids=str)
def test_attend_ids_outside_the_pool(kw):
    layer = make(num_blocks=300, **kw)
    rng = np.random.default_rng(7)
    pool = random_pool(layer, rng)
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([2, 3], 700, [100, 50]), ([1] * 9, 200, [30] * 9)], 60)
    table[0:2, 7], table[0:2, 20], table[1, 45], table[5] = -1, 300, 2 ** 31 - 1, np.where(np.arange(60) < 12, table[5], -5)
    table[3:, 12:] = np.where(rng.random(table[3:, 12:].shape) < 0.5, table[3:, 12:], -1)  # behind the 200 // 16 columns that the group shares
    kv[10] = 10 ** 9                                                      # beyond the table
    run_attend(layer, queries(layer, rng, 14), pool, table, kv, row_start, group_start, prefix)
    run_attend(layer, queries(layer, rng, 14), pool, np.full_like(table, -1), kv, row_start, group_start, prefix)
    run_attend(layer, queries(layer, rng, 14), pool, table[:, :0], kv, row_start, group_start, prefix)
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True), dict(D=64, bf16=False)], ids=str)
@pytest.mark.parametrize("others", [0, 300, 600])
def test_attend_row_start_that_decreases(kw, others):
    """Rows that are not among those of their group have no part in its shared blocks: they attend to their sequence's own, and nothing is read where no part of theirs is.  Workspace and
    what lies around it hold NaN."""
    print("case:", kw, others, flush=True)
    layer = make(num_blocks=200, **kw)
    c, rng = layer.cfg, np.random.default_rng(6)
    pool = random_pool(layer, rng)
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([10, 60, 3], 640, [5, 130, 40])] + [([0] * others, 16, [0] * others)] * (others > 0), 100)
    row_start = np.concatenate([[50, 0, 60, 63], np.full(others, 63)])     # the group's rows are 50 .. 62, those of its second sequence 0 .. 59
    q, (S, cols) = queries(layer, rng, 63, 2.0), table.shape
    own = np.concatenate([table[:, 40:], np.full((S, 40), -1)], axis=1)
    want = [ref.attend(host(q), pool_values(layer, pool), t, n, row_start, group_start, 16, np.full(q.shape, 7.0)) for t, n in ((own, kv - 640), (table, kv))]
    need = binding._lib.icarus_attn_prefix_workspace_bytes(layer._h, S, len(prefix), 63, cols)
    around = torch.full((need + (2 << 20),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, 7.0)
    layer.attn_prefix(q, pool, i32(table), i32(kv), i32(row_start), i32(group_start), i32(prefix), out, workspace=around[1 << 20:(1 << 20) + need])
    torch.cuda.synchronize()
    for rows, (w, weight, size, count) in ((slice(0, 60), want[0]), (slice(60, 63), want[1])):
        assert (np.abs(host(out) - w) <= bound(layer, w, weight, size, count))[rows].all(), rows
    layer.close()


def attend_repeated(q, pool, table, kv, row_start, bk, num_blocks):
    """ref.attend of sequences whose tables name few blocks many times: a block counts as often as it is named."""
    out, weight, size, count = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2] + (1,)), np.zeros(q.shape[:2] + (1,))
    hkv, D = pool.shape[1], q.shape[2]
    g = q.shape[1] // hkv
    for s, n in enumerate(kv):
        rows, full = slice(row_start[s], row_start[s + 1]), table[s, :n // bk]
        ids, times = np.unique(full[(full >= 0) & (full < num_blocks)], return_counts=True)
        parts = [(b, bk, t) for b, t in zip(ids, times)] + ([(table[s, n // bk], n % bk, 1)] if n % bk and 0 <= table[s, n // bk] < num_blocks else [])
        times = np.concatenate([np.full(m, t) for _, m, t in parts])
        for c in range(hkv):
            k = np.concatenate([pool[b, c, 0].reshape(bk, D)[:m] for b, m, _ in parts])
            v = np.concatenate([pool[b, c, 1].reshape(D, bk).T[:m] for b, m, _ in parts])
            qq = q[rows, c * g:(c + 1) * g]
            sc = qq @ k.T / math.sqrt(D)
            p = times * np.exp(sc - sc.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[rows, c * g:(c + 1) * g], weight[rows, c * g:(c + 1) * g] = p @ v, p @ np.abs(v)
            size[rows, c * g:(c + 1) * g] = (np.abs(qq) @ np.abs(k).T).max(-1, keepdims=True) / math.sqrt(D)
            count[rows, c * g:(c + 1) * g] = times.sum()
    return out, weight, size, count


@pytest.mark.parametrize("kw", [dict(Hq=64, Hkv=64), dict(Hq=64, Hkv=64, fp8=True, k_scale=0.5), dict(Hq=64, Hkv=64, D=64, bf16=False), dict(Hq=64, Hkv=64, bk=32)], ids=str)
@pytest.mark.parametrize("columns,rows", [(4000, [3]), (4000, [50, 0, 60]), (9001, [40, 1, 30, 29]), (9216, [128])], ids=str)
def test_attend_items_of_many_blocks(kw, columns, rows):
    """Items of more than 256 blocks, whose ids are gathered in rounds, and of as many as an item may have; ids outside the pool all over, a last block that is not full.  Few blocks, named
    many times."""
    print("case:", kw, columns, rows, flush=True)
    layer, rng, S = make(num_blocks=50, **kw), np.random.default_rng(columns + len(rows)), len(rows)
    bk, pool = layer.cfg.block_size, random_pool(layer, rng)
    table = np.repeat(rng.integers(0, 50, (1, columns)), S, axis=0)
    if columns % 1024:
        table[:, rng.random(columns) < 0.1] = -1
        table[:, 7], table[:, columns - 90] = 50, 2 ** 31 - 1
    table[:, columns - 8:] = rng.integers(0, 50, (S, 8))                 # behind the shared columns
    table[-1, columns - 5] = -7 if columns % 1024 else 3
    kv = columns * bk - 8 * bk + rng.integers(1, 8 * bk, S)
    kv[0] = columns * bk - 3
    row_start, q = np.concatenate([[0], np.cumsum(rows)]), queries(layer, rng, sum(rows), 2.0)
    want = attend_repeated(host(q), pool_values(layer, pool), table, kv, row_start, bk, 50)
    for prefix in ((columns - 8) * bk + 5, 0):
        out = layer.attn_prefix(q, pool, i32(table), i32(kv), i32(row_start), i32([0, S]), i32([prefix]))
        assert (np.abs(host(out) - want[0]) <= bound(layer, *want)).all(), prefix
    layer.close()


@pytest.mark.parametrize("kw,first", [(kw, first) for kw in (dict(Hq=4, Hkv=1), dict(Hq=4, Hkv=1, fp8=True), dict(Hq=4, Hkv=1, D=64, bf16=False), dict(Hq=2, Hkv=1, D=256))
                                      for first in ("growing", "minus infinity", "shrinking") if not ("fp8" in kw and first == "minus infinity")], ids=str)  # no infinity among the codes
@pytest.mark.parametrize("prefix", [0, 330 * 16])
def test_attend_rows_of_many_parts(kw, first, prefix):
    """More than 64 parts to a row, which are joined in rounds: scores that grow along the sequence, so that each round outweighs the ones before, that are minus infinity in the first round, and
    that shrink."""
    print("case:", kw, first, prefix, flush=True)
    layer, rng = make(num_blocks=1300, **kw), np.random.default_rng(1)
    c, pool = layer.cfg, random_pool(layer, rng)
    ids = rng.permutation(1300)
    table = np.stack([ids[:640], np.concatenate([ids[:330], ids[640:950]])])
    if not prefix:
        table, kv, row_start, group_start = table[:1], [640 * 16 - 5], [0, 3], [0, 1]
    else:
        kv, row_start, group_start = [640 * 16 - 5, 600 * 16 + 1], [0, 3, 5], [0, 2]
    q = queries(layer, rng, row_start[-1])
    q[:, :, 0] = 4.0
    for row in table:                                                       # channel 0 of the keys: scores rise to 4 * 40 / sqrt(D) and more
        x = np.arange(640)[:, None] / 640 * 40.0
        x = {"growing": x, "shrinking": 40.0 - x, "minus infinity": np.where(np.arange(640)[:, None] < 300, -math.inf, x)}[first]
        keys = pool.view(1300, 1, 2, 16, c.head_dim)[:, :, 0]
        there = torch.tensor(row.copy(), device=DEV)
        values = torch.tensor(x, dtype=torch.float32, device=DEV).expand(640, 16)
        keys[there, 0, :, 0] = values.to(torch.float8_e4m3fn).view(torch.uint8) if c.kv_fp8 else values.to(c.torch_dtype)
    run_attend(layer, q, pool, table, np.array(kv), np.array(row_start), np.array(group_start), np.array([prefix]))
    layer.close()


def test_prefix_beyond_32_bits():
    """A pool of more than 2^32 elements, read at its end."""
    layer = make(Hq=32, Hkv=8, num_blocks=140000)
    c = layer.cfg
    pool = torch.zeros(c.pool_shape(), dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(0)
    ids = np.arange(139960, 140000)
    small = make(Hq=32, Hkv=8, num_blocks=40)
    some = random_pool(small, rng)
    pool[139960:] = some
    table = np.stack([np.concatenate([ids[:20], ids[20:30]]), np.concatenate([ids[:20], ids[30:]])])
    q = queries(layer, rng, 4)
    args = ([470, 480], np.array([0, 2, 4]), np.array([0, 2]), [320])
    want = run_attend(small, q, some, table - 139960, *args)
    for t, w in zip(both_widths(table, 16), want):
        out = torch.zeros_like(q)
        layer.attn_prefix(q, pool, i32(t), i32(args[0]), i32(args[1]), i32(args[2]), i32(args[3]), out)
        assert torch.equal(out, w)
    layer.copy_blocks([pool], i32([139990, 3]), i32([1, 139999]))
    assert torch.equal(pool[1], some[30]) and not pool[139999].any()
    layer.close()
    small.close()


def test_integer_arrays_need_only_their_own_alignment():
    layer, rng = make(num_blocks=200), np.random.default_rng(0)

    def off(a):
        t = torch.empty(int(np.size(a)) + 1, dtype=torch.int32, device=DEV)
        t[1:] = i32(a).reshape(-1)
        return t[1:].view(np.shape(a))
    pool = random_pool(layer, rng)
    table, kv, row_start, group_start, prefix = crowd(layer, rng, [([2, 1], 333, [20, 31])], 30)
    q = queries(layer, rng, 3)
    for t in both_widths(table, 16):
        a = layer.attn_prefix(q, pool, i32(t), i32(kv), i32(row_start), i32(group_start), i32(prefix))
        b = layer.attn_prefix(q, pool, off(t), off(kv), off(row_start), off(group_start), off(prefix))
        assert torch.equal(a, b)
    got = []
    for put in (i32, off):
        m = binding.ForkMap(1, 2, 30, DEV)
        m.block_tables.fill_(-1)
        free = put(np.arange(200))
        layer.fork_sequences(put([1, 1]), put(kv), put(table), m, free, put([60]), put([20]))
        got.append([m.kv_lens, m.block_tables, m.copy_src, m.copy_dst, m.counts, free])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    layer.close()


def test_workspaces_elsewhere_are_refused():
    layer = make(num_blocks=20)
    small, away = torch.zeros(16, dtype=torch.uint8, device=DEV), torch.zeros(1 << 20, dtype=torch.uint8)
    table, q = i32([[1, 2]]), torch.zeros(1, 8, 128, dtype=torch.bfloat16, device=DEV)
    pool, beams, forked = torch.zeros(layer.cfg.pool_shape(), dtype=torch.bfloat16, device=DEV), binding.BeamMap(1, 1, DEV), binding.ForkMap(1, 1, 2, DEV)
    calls = (lambda ws: layer.attn_prefix(q, pool, table, i32([20]), i32([0, 1]), i32([0, 1]), i32([16]), workspace=ws),
             lambda ws: layer.beam_select(torch.zeros(1, 50, device=DEV), torch.zeros(1, device=DEV), beams, workspace=ws),
             lambda ws: layer.fork_sequences(i32([0]), i32([20]), table, forked, i32([3, 4]), i32([0]), workspace=ws))
    for call in calls:
        with pytest.raises(ValueError):
            call(away)
        with pytest.raises(binding.IcarusError, match="CAPACITY"):
            call(small)
    layer.close()


# ---- together ------------------------------------------------------------------------------------------------------------------

def _search(layer, seed, groups=3, width=4, max_blocks=40, vocab=5003):
    """A beam search's buffers: two sets of tables that a step reads and fills, prompts of different lengths whose whole blocks are shared, two layers' pools."""
    c, rng = layer.cfg, np.random.default_rng(seed)
    S = groups * width
    kv = np.repeat(rng.integers(40, 300, groups), width)
    ids = rng.permutation(c.num_blocks)
    table, at = np.full((S, max_blocks), -1), 0
    for g in range(groups):
        nb = blocks_of(kv[g * width], 16)
        table[g * width:(g + 1) * width, :nb] = ids[at:at + nb]             # the partly filled one too: the first fork copies it
        at += nb
    b = dict(S=S, groups=groups, rng=rng, shared=i32(kv[::width] // 16), prefix=i32(kv[::width]), group_start=i32(np.arange(0, S + 1, width)), used=i32([at]), free=i32(ids),
             new=i32([1] * S), act=i32([1] * S), rows=binding.SequenceMap(S, 2 * S, DEV), vocab=vocab, step=0)
    b["tables"] = [binding.ForkMap(groups, width, max_blocks, DEV) for _ in range(2)]
    b["beams"] = [binding.BeamMap(groups, width, DEV) for _ in range(2)]
    for t in b["tables"]:
        t.block_tables.fill_(-1)
    b["tables"][0].kv_lens.copy_(i32(kv))
    b["tables"][0].block_tables.copy_(i32(table))
    first = b["beams"][0]
    first.scores.fill_(-math.inf)
    first.scores[::width] = 0.0                                            # one beam is live at first
    first.done.zero_()
    b["pools"] = [random_pool(layer, rng) for _ in range(2)]
    b["codes"], b["scales"] = layer.new_key_bounds(DEV)
    b["logits"] = torch.empty(2 * S, vocab, device=DEV)
    b["row_start"] = i32(2 * np.arange(S + 1))
    b["qkv"] = torch.empty(2 * S, (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, dtype=c.torch_dtype, device=DEV)
    b["q"] = torch.zeros(2 * S, c.n_q_heads, c.head_dim, dtype=c.torch_dtype, device=DEV)
    b["out"] = [torch.zeros_like(b["q"]) for _ in range(2)]
    return b


def _feed(b, i):
    """What a model would give the step: logits and projections, from the seed and the step alone."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000 + i)
    b["logits"].normal_(generator=gen).mul_(3)
    b["logits"][:, 7] += 4.0 * (i > 4)                                      # the end token, likely later on
    b["qkv"].copy_(torch.randn(b["qkv"].shape, generator=gen, device=DEV))


def _half(layer, b, k):
    """One step from tables and beams k into the others."""
    now, nxt, old, new = b["tables"][k], b["tables"][1 - k], b["beams"][k], b["beams"][1 - k]
    layer.beam_select(b["logits"], old.scores, new, row_start=b["row_start"], done=old.done, eos=7)
    layer.fork_sequences(new.parents, now.kv_lens, now.block_tables, nxt, b["free"], b["used"], shared=b["shared"])
    b["used"].copy_(nxt.counts[:1])
    layer.copy_blocks(b["pools"] + [b["codes"], b["scales"]], nxt.copy_src, nxt.copy_dst)
    m = layer.extend_sequences(b["rows"], nxt.kv_lens, b["new"], nxt.block_tables, b["free"], b["used"], streams=b["act"])
    b["used"].copy_(m.counts[:1])
    for pool, out in zip(b["pools"], b["out"]):
        layer.rope_append(b["qkv"], m.row_pos, m.row_slot, pool, b["q"])
        layer.attn_prefix(b["q"], pool, nxt.block_tables, m.kv_lens, m.row_start, b["group_start"], b["prefix"], out)
    nxt.kv_lens.copy_(m.kv_lens)


def _state(b):
    every = [b["used"], b["q"], *b["out"], *b["pools"], b["rows"].row_slot]
    for m in b["beams"]:
        every += [m.parents, m.tokens, m.scores, m.done]
    for m in b["tables"]:
        every += [m.kv_lens, m.block_tables, m.copy_src, m.copy_dst, m.counts]
    return [t.clone() for t in every]


def _same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True), dict(Hq=4, Hkv=4, D=64, bf16=False)], ids=str)
def test_a_search_keeps_its_histories(kw):
    """Twenty steps: every beam's attention is the one over its own history, gathered from its ancestors token by token, and no block is lost or in two hands."""
    layer = make(num_blocks=260, **kw)
    c, b = layer.cfg, _search(layer, 3)
    S, W = b["S"], 4
    first = b["tables"][0]
    pool0 = pool_values(layer, b["pools"][0]).reshape(c.num_blocks, c.n_kv_heads, 2, -1)

    def tokens(table, n, values):
        k = np.stack([values[int(table[p // 16]), :, 0].reshape(c.n_kv_heads, 16, -1)[:, p % 16] for p in range(n)])
        v = np.stack([values[int(table[p // 16]), :, 1].reshape(c.n_kv_heads, -1, 16)[:, :, p % 16] for p in range(n)])
        return np.stack([k, v], 1)
    table0, kv0 = first.block_tables.cpu().numpy(), first.kv_lens.cpu().numpy()
    history = [tokens(table0[s], int(kv0[s]), pool0) for s in range(S)]
    prefix_blocks = {int(x) for s in range(0, S, W) for x in table0[s, :kv0[s] // 16]}
    total = int(b["used"].item())
    for i in range(20):
        _feed(b, i)
        _half(layer, b, i & 1)
        torch.cuda.synchronize()
        nxt = b["tables"][1 - (i & 1)]
        parents = b["beams"][1 - (i & 1)].parents.cpu().numpy()
        table, kv = nxt.block_tables.cpu().numpy(), nxt.kv_lens.cpu().numpy()
        values = pool_values(layer, b["pools"][0]).reshape(c.num_blocks, c.n_kv_heads, 2, -1)
        grown = []
        for s in range(S):
            n = int(kv[s])
            if parents[s] < 0:
                assert n == 1                                              # a child of nobody starts anew
                grown.append(tokens(table[s], 1, values))
                continue
            mine = tokens(table[s], n, values)
            assert np.array_equal(mine[:-1], history[s // W * W + parents[s]]), (i, s)
            grown.append(mine)
        history = grown
        held = {int(x) for s in range(S) for x in table[s, :blocks_of(kv[s], 16)]}
        left = set(b["free"].cpu().numpy()[int(b["used"].item()):].tolist())
        assert not held & left and left | held | prefix_blocks | set(table0[:, :].ravel().tolist()) >= set(range(c.num_blocks)) - {-1}
        assert len(left) == c.num_blocks - int(b["used"].item())
        rows = b["rows"].row_start.cpu().numpy()
        want, weight, size, count = ref.attend(host(b["q"]), values, table, kv, rows, np.arange(0, S + 1, W), 16, host(b["out"][0]))
        assert (np.abs(host(b["out"][0]) - want) <= bound(layer, want, weight, size, count)).all(), i
    assert total > 0
    layer.close()


@pytest.mark.parametrize("samples", [False, True])
@pytest.mark.parametrize("groups,width,ends", [(1, 3, 1), (5, 8, 0), (4, 20, 15)])
def test_branches_of_one_prompt(groups, width, ends, samples):
    """Beams (children of one live sequence) and samples (each its own parent, the prompt's last block a shared column for the first fork) that grow for forty steps, some of them dropped:
    every sequence holds its own tokens, and every block is a prompt's, in a table, or free, once."""
    print("case:", groups, width, ends, samples, flush=True)
    rng, cols = np.random.default_rng(width), 8
    S = groups * width
    num = groups * cols + S * cols
    layer, kv = make(num_blocks=num), np.repeat(16 * rng.integers(1, 4, groups) + ends, width)
    ids, table, at, prompts, shared = rng.permutation(num), np.full((S, cols), -1), 0, set(), [kv[::width] // 16, -(-kv[::width] // 16) if samples else kv[::width] // 16]
    for g in range(groups):
        nb = blocks_of(kv[g * width], 16)
        table[g * width:(g + 1) * width, :nb] = ids[at:at + nb]
        prompts |= set(ids[at:at + shared[1][g]].tolist())
        at += nb
    text = torch.tensor(rng.integers(0, 10 ** 6, (num, 16)), dtype=torch.int32, device=DEV)
    words_of = lambda row, n, t: [int(t[row[p // 16], p % 16]) for p in range(n)]
    history = [words_of(table[s], kv[s], text.cpu().numpy()) for s in range(S)]
    maps, rows = [binding.ForkMap(groups, width, cols, DEV) for _ in range(2)], binding.SequenceMap(S, S, DEV)
    maps[0].kv_lens.copy_(i32(kv))
    maps[0].block_tables.copy_(i32(table))
    free, used = i32(ids), i32([at])
    parents = np.arange(S) % width if samples else np.zeros(S, dtype=int)
    for i in range(40):
        now, nxt = maps[i & 1], maps[1 - (i & 1)]
        layer.fork_sequences(i32(parents), now.kv_lens, now.block_tables, nxt, free, used, shared=i32(shared[i == 0]))
        used.copy_(nxt.counts[:1])
        layer.copy_blocks([text], nxt.copy_src, nxt.copy_dst)
        m = layer.extend_sequences(rows, nxt.kv_lens, (nxt.kv_lens > 0).int(), nxt.block_tables, free, used)
        used.copy_(m.counts[:1])
        slots = m.row_slot[:int(m.row_start[S])].long()
        text.view(-1)[slots] = i32(rng.integers(0, 10 ** 6, len(slots)))
        nxt.kv_lens.copy_(m.kv_lens)
        n, row, t = m.kv_lens.cpu().numpy(), nxt.block_tables.cpu().numpy(), text.cpu().numpy()
        grown = [words_of(row[s], n[s], t) for s in range(S)]
        for s, p in enumerate(parents):
            assert grown[s][:-1] == (history[s // width * width + p] if p >= 0 else []) and len(grown[s]) != 1, (i, s)
        history = grown
        held = {int(b) for s in range(S) for b in row[s, :blocks_of(n[s], 16)]}
        left = free.cpu().numpy()[int(used.item()):].tolist()
        assert len(left) == len(set(left)) and not (held | prompts) & set(left) and held | prompts | set(left) == set(range(num)), i
        parents = np.where(rng.random(S) < 0.9, np.arange(S) % width, rng.integers(-1, width, S))
        parents[:: width] = [next(iter(np.flatnonzero(n[g * width:(g + 1) * width])), 0) for g in range(groups)]
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True), dict(Hq=4, Hkv=4, D=64, bf16=False)], ids=str)
def test_captured_search_replays(kw):
    """Two searches, each captured once (two steps, one from each set of tables) and replayed in turn with the program's own work between; every replay is the eager
    pair of steps, bit for bit."""
    layer = make(num_blocks=400, **kw)
    eager, captured, graphs = [], [], []
    for seed in (1, 2):
        warm = _search(layer, seed)
        _feed(warm, 0)
        _half(layer, warm, 0)
        b, want = _search(layer, seed), []
        for i in range(10):
            _feed(b, i)
            _half(layer, b, 0)
            _half(layer, b, 1)
            want.append(_state(b))
        eager.append(want)
        captured.append(_search(layer, seed))
    torch.cuda.synchronize()
    for b in captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _half(layer, b, 0)
            _half(layer, b, 1)
        graphs.append(g)
    for i in range(10):
        for want, b, g in zip(eager, captured, graphs):
            _feed(b, i)
            g.replay()
            if i % 3 == 0:
                torch.cuda.synchronize()
            assert _same(_state(b), want[i]), i
            (b["out"][0].float() * 2).sum().item()
    layer.close()


def test_two_searches_on_two_streams():
    layer = make(num_blocks=400)
    want, loops = [], []
    for seed in (3, 4):
        b = _search(layer, seed)
        _feed(b, seed)
        for i in range(6):
            _half(layer, b, i & 1)
        want.append(_state(b))
        loops.append(_search(layer, seed))
        _feed(loops[-1], seed)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in loops]
    for i in range(6):
        for b, st in zip(loops, streams):
            with torch.cuda.stream(st):
                _half(layer, b, i & 1)
    torch.cuda.synchronize()
    for b, w in zip(loops, want):
        assert _same(_state(b), w)
    layer.close()


def test_finished_beams_that_are_fed_no_more():
    """A search that gives finished beams no new token, so no row, keeps them, their lengths and their scores until better ones push them out."""
    layer, rng = make(num_blocks=300), np.random.default_rng(8)
    groups, width, vocab, eos, cols = 3, 4, 601, 7, 12
    S = groups * width
    kv = np.repeat(rng.integers(20, 90, groups), width)
    table = np.full((S, cols), -1)
    for s in range(S):
        table[s, :blocks_of(kv[s], 16)] = s // width * cols + np.arange(blocks_of(kv[s], 16))
    used, free = i32([groups * cols]), i32(np.arange(300))
    maps, beams = [binding.ForkMap(groups, width, cols, DEV) for _ in range(2)], [binding.BeamMap(groups, width, DEV) for _ in range(2)]
    maps[0].kv_lens.copy_(i32(kv))
    maps[0].block_tables.copy_(i32(table))
    beams[0].scores.fill_(-math.inf)
    beams[0].scores[::width] = 0.0
    beams[0].done.zero_()
    rows, start, shared = binding.SequenceMap(S, S, DEV), i32(np.arange(S + 1)), i32(kv[::width] // 16)
    kept = 0
    for i in range(12):
        now, nxt, old, new = maps[i & 1], maps[1 - (i & 1)], beams[i & 1], beams[1 - (i & 1)]
        logits = words(rng, S, vocab, torch.float32)
        logits[:, eos] += 9.0 * (i in (2, 5))
        x, live = last_rows(host(logits), start.cpu().numpy(), old.scores.cpu().numpy(), old.done.cpu().numpy())
        p, t, v, d, _ = ref.choose(x, None, live, old.done.cpu().numpy(), eos, groups, width)
        layer.beam_select(logits, old.scores, new, row_start=start, done=old.done, eos=eos)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((new.parents, new.tokens, new.done), (p, t, d))), i
        layer.fork_sequences(new.parents, now.kv_lens, now.block_tables, nxt, free, used, shared=shared)
        used.copy_(nxt.counts[:1])
        m = layer.extend_sequences(rows, nxt.kv_lens, ((new.parents >= 0) & (new.done == 0)).int(), nxt.block_tables, free, used)
        used.copy_(m.counts[:1])
        start = m.row_start.clone()
        for s in range(S):
            q = s // width * width + p[s]
            was = p[s] >= 0 and old.done[q].item()
            kept += bool(was)
            assert m.kv_lens[s] == (0 if p[s] < 0 else now.kv_lens[q] + (0 if d[s] else 1))
            assert not was or (new.scores[s] == old.scores[q] and t[s] == eos and start[s] == start[s + 1])
        nxt.kv_lens.copy_(m.kv_lens)
    assert kept > 5
    layer.close()
