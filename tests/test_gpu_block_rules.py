"""What include/icarus_blocks.h promises beyond each operator's values: results that do not go by hints, cache entries that do not go by the call that
wrote them, NaN that is not hidden."""
import math

import numpy as np
import pytest
import torch

import block_reference as ref
from paper_2603_13281_amd import binding
from test_gpu_block_ops import DEV, E24, _loop, _state, _step, host, i32, make, pool_values, random_pool

pytestmark = pytest.mark.gpu


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- hints ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(Hq=32, Hkv=8), dict(Hq=64, Hkv=8, fp8=True, k_scale=0.5), dict(Hq=40, Hkv=2), dict(Hq=4, Hkv=4, D=64, bf16=False), dict(Hq=16, Hkv=2, D=64),
                                dict(Hq=32, Hkv=8, bk=32), dict(Hq=8, Hkv=2, mode=1)], ids=str)
@pytest.mark.parametrize("rows,top", [([9], 128), ([9] * 16, 256), ([1, 9, 0, 3, 25], 40), ([70, 2], 64)], ids=str)
@pytest.mark.parametrize("unit", [1.0, 30.0])
def test_attention_does_not_go_by_the_hint(kw, rows, top, unit):
    """unit 30: scores in the hundreds, so that the softmax references of the tiles move at different times."""
    print("case:", kw, rows, top, unit, flush=True)
    layer = make(num_blocks=300, **kw)
    c, rng = layer.cfg, np.random.default_rng(top)
    S, start = len(rows), np.concatenate([[0], np.cumsum(rows)])
    pool = random_pool(layer, rng)
    table, kv = i32(rng.integers(0, 300, (S, 300))), i32(rng.integers(200, 300 * c.block_size, S))
    blocks, counts = i32(rng.integers(0, 300, (S, c.n_kv_heads, top))), i32(rng.integers(top // 2, top + 1, S))
    q = torch.tensor(rng.standard_normal((start[-1] + 5, c.n_q_heads, c.head_dim)) * unit, dtype=torch.float32).to(c.torch_dtype).to(DEV)
    want = layer.attn_blocks(q, pool, table, kv, i32(start), blocks, counts)
    for hint in (1, 2, 4, 9, 25, 1000):
        assert same_bits(layer.attn_blocks(q, pool, table, kv, i32(start), blocks, counts, seq_rows=hint), want), hint
    layer.close()


# ---- one cache ------------------------------------------------------------------------------------------------------------

def _projecting(seed, Hq, Hkv, D, bk, num_blocks, bf16, fp8=False, qk_norm=False, scale=1.0, mode=0):
    """A layer whose keys and values are known before the cache: each row of W_k and W_v has one element, and hidden states of 1 and -1 stay what they
    are under the norm, so that every projection is an element or its negative, exactly."""
    dt = torch.bfloat16 if bf16 else torch.float32
    gen = torch.Generator().manual_seed(seed)
    d = 256
    column = {p: torch.randint(0, d, (Hkv * D,), generator=gen) for p in "kv"}
    element = {p: torch.randn(Hkv * D, generator=gen).to(dt) for p in "kv"}
    w = {p: torch.zeros(n, m, dtype=dt) for p, n, m in (("q", Hq * D, d), ("k", Hkv * D, d), ("v", Hkv * D, d), ("o", d, Hq * D), ("gate", d, d), ("up", d, d), ("down", d, d))}
    for p in "kv":
        w[p][torch.arange(Hkv * D), column[p]] = element[p]
    w["norm_attn"], w["norm_ffn"] = torch.ones(d, dtype=dt), torch.ones(d, dtype=dt)
    if qk_norm:
        w["q_norm"], w["k_norm"] = ((1 + 0.2 * torch.randn(D, generator=gen)).to(dt) for _ in range(2))
    cfg = binding.LayerConfig(d_model=d, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, d_ffn=d, block_size=bk, num_blocks=num_blocks, bf16=bf16, qk_norm=qk_norm, max_position=1 << 20,
                              rope_theta=5e5, rms_eps=0.0, kv_fp8=fp8, k_scale=scale, v_scale=scale)
    layer = binding.IcarusLayer(cfg, {n: t.to(DEV) for n, t in w.items()})
    layer.set_kernel_mode(mode)
    return layer, column, element


@pytest.mark.parametrize("kw", [dict(Hq=8, Hkv=8, D=128, bk=16, bf16=True), dict(Hq=8, Hkv=8, D=128, bk=16, bf16=True, qk_norm=True),
                                dict(Hq=64, Hkv=8, D=128, bk=16, bf16=True, qk_norm=True),
                                dict(Hq=8, Hkv=4, D=128, bk=16, bf16=True, qk_norm=True, fp8=True, scale=0.02), dict(Hq=4, Hkv=4, D=128, bk=16, bf16=False, qk_norm=True),
                                dict(Hq=4, Hkv=4, D=64, bk=16, bf16=False), dict(Hq=4, Hkv=4, D=64, bk=16, bf16=False, qk_norm=True), dict(Hq=4, Hkv=4, D=64, bk=16, bf16=True, qk_norm=True),
                                dict(Hq=4, Hkv=2, D=256, bk=16, bf16=True, qk_norm=True), dict(Hq=4, Hkv=2, D=256, bk=16, bf16=False, qk_norm=True),
                                dict(Hq=4, Hkv=2, D=192, bk=16, bf16=False, qk_norm=True), dict(Hq=6, Hkv=2, D=36, bk=5, bf16=False, qk_norm=True),
                                dict(Hq=8, Hkv=8, D=128, bk=16, bf16=False, qk_norm=True, mode=1), dict(Hq=4, Hkv=4, D=64, bk=16, bf16=False, fp8=True, qk_norm=True)], ids=str)
def test_appended_entries_are_prefills(kw):
    """The same projections at the same positions, appended here and by icarus_prefill_kv and icarus_decode_step: the same cache, bit for bit."""
    print("case:", kw, flush=True)
    ctx, new = [0, 99990, 131, 5000], [40, 300, 17, 1]
    bk = kw["bk"]
    used = [ref.blocks_of(c + n + 1, bk) - c // bk for c, n in zip(ctx, new)]
    layer, column, element = _projecting(3, num_blocks=1 + sum(used), **kw)
    c, rng = layer.cfg, np.random.default_rng(4)
    table = np.zeros((4, max(ref.blocks_of(a + n + 1, bk) for a, n in zip(ctx, new))), dtype=np.int64)  # earlier positions: block 0, which holds zeros
    ids, at = 1 + rng.permutation(sum(used)), 0
    for s in range(4):
        table[s, ctx[s] // bk: ctx[s] // bk + used[s]] = ids[at:at + used[s]]
        at += used[s]
    pools = [torch.zeros(c.pool_shape(), dtype=c.pool_dtype, device=DEV) for _ in range(2)]

    def both(starts, counts, decode):
        x = torch.tensor(rng.integers(0, 2, (sum(counts), c.d_model)) * 2 - 1, dtype=torch.float32).to(c.torch_dtype)
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(starts, counts)])
        seq = np.repeat(np.arange(4), counts)
        if decode:
            layer.decode_step(pools[0], i32(table), starts, seq, [-1] * len(seq), x.to(DEV))
        else:
            layer.prefill_kv(pools[0], i32(table), starts, counts, x.to(DEV), want_out=False)
        kv = [x[:, column[p]] * element[p] for p in "kv"]
        qkv = torch.cat([torch.zeros(len(pos), c.n_q_heads * c.head_dim, dtype=c.torch_dtype), *kv], 1).to(DEV)
        slot = table[seq, pos // bk] * bk + pos % bk
        layer.rope_append(qkv, i32(pos), torch.tensor(slot, dtype=torch.int64, device=DEV), pools[1])

    both(ctx, new, False)
    both([a + n for a, n in zip(ctx, new)], [1] * 4, True)
    torch.cuda.synchronize()
    a, b = (host(p.view(torch.float8_e4m3fn) if c.kv_fp8 else p) for p in pools)
    assert np.abs(a[1:]).max() > 0 and np.array_equal(a[:, :, 1], b[:, :, 1])      # values: the projections are what they were made to be
    assert np.array_equal(a[:, :, 0], b[:, :, 0]), ((a != b).mean(), np.abs(a - b).max())
    assert same_bits(*pools)
    layer.close()


@pytest.mark.parametrize("kw", [dict(Hq=8, Hkv=2, qk_norm=True), dict(Hq=8, Hkv=2, fp8=True, qk_norm=True), dict(Hq=4, Hkv=4, D=64, bf16=False), dict(Hq=4, Hkv=2, D=36, bk=5, qk_norm=True),
                                dict(Hq=4, Hkv=2, D=256), dict(Hq=8, Hkv=2, qk_norm=True, mode=1)], ids=str)
def test_append_does_not_go_by_what_it_leaves_out(kw):
    """K and V of rows whose slot is outside the pool, and whole rows with a negative position, hold NaN: the same bits as with anything else there."""
    print("case:", kw, flush=True)
    layer = make(num_blocks=64, **kw)
    c, rng = layer.cfg, np.random.default_rng(6)
    rows, n_slots, first_k = 75, c.num_blocks * c.block_size, c.n_q_heads * c.head_dim
    pos, slot = rng.integers(0, 9999, rows), 7 + np.arange(rows)             # runs through several blocks, with these between
    slot[3::5], slot[11], slot[40] = -1, n_slots, 2 ** 62
    pos[20:23], pos[50] = -1, -(2 ** 31)
    qkv = torch.tensor(rng.standard_normal((rows, first_k + 2 * c.n_kv_heads * c.head_dim)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
    nan = qkv.clone()
    nan[torch.tensor((slot < 0) | (slot >= n_slots), device=DEV), first_k:] = float("nan")
    nan[torch.tensor(pos < 0, device=DEV)] = float("nan")
    results = []
    for x in (qkv, nan):
        pool, q = random_pool(layer, np.random.default_rng(7)), torch.full((rows, c.n_q_heads, c.head_dim), 7.0, dtype=c.torch_dtype, device=DEV)
        layer.rope_append(x, i32(pos), torch.tensor(slot, dtype=torch.int64, device=DEV), pool, q)
        results.append((pool, q))
    assert all(same_bits(a, b) for a, b in zip(*results)) and not bool(torch.isnan(results[1][1]).any()) and bool((results[1][1][20:23] == 7).all())
    layer.close()


# ---- bits -------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(fp8=True, k_scale=0.5, v_scale=0.3), dict(Hq=40, Hkv=2), dict(Hq=40, Hkv=2, fp8=True), dict(D=64), dict(D=64, fp8=True), dict(mode=1), dict(bk=32)],
                         ids=str)
@pytest.mark.parametrize("top,unit", [(1, 0.1), (2, 1.0), (38, 1.0), (38, 4.0)])
def test_attention_keeps_its_weights(kw, top, unit):
    """Error beyond the rounding of the result: weights have more bits than the result's type, so that they do not add to it."""
    print("case:", kw, top, unit, flush=True)
    layer = make(num_blocks=160, **kw)
    c, rng = layer.cfg, np.random.default_rng(top)
    pool = random_pool(layer, rng)
    S, bk = 4, c.block_size
    table, kv, start = rng.permutation(156).reshape(S, 39), np.array([39 * bk, 39 * bk - 3, 39 * bk, 37 * bk + 1]), np.array([0, 1, 3, 8, 12])
    blocks = np.stack([[rng.permutation(39)[:top] for _ in range(c.n_kv_heads)] for _ in range(S)])
    q = torch.tensor(rng.standard_normal((12, c.n_q_heads, c.head_dim)) * unit, dtype=torch.float32).to(c.torch_dtype).to(DEV)
    got = host(layer.attn_blocks(q, pool, i32(table), i32(kv), i32(start), i32(blocks), i32([top] * S)))
    want, weight, size = ref.attend(host(q), pool_values(layer, pool), table, kv, start, blocks, [top] * S, bk, np.zeros(q.shape))
    # run_attend's bound, with the weights' own rounding (half a step of float16, 2^-11) where it has half a step of bfloat16
    tol = 2.0 ** -8 * np.abs(want) + weight * (2 * (c.head_dim + 3) * E24 * size + 2.0 ** -17 + top * bk * E24 + 2.0 ** -11)
    assert (np.abs(got - want) <= tol).all(), ((np.abs(got - want) > tol).sum(), (np.abs(got - want) / tol).max())
    # Roundings have no common direction, so their squares add: the result's own is what the oracle's values lose in bfloat16; weights of float16 add a 64th of it (1.01 in
    # all), of bfloat16 as much again (1.4)
    if unit <= 1:
        own = host(torch.tensor(want).to(c.torch_dtype)) - want
        assert ((got - want) ** 2).sum() < 1.1 ** 2 * (own ** 2).sum()
    layer.close()


@pytest.mark.parametrize("fp8", [True, False])
def test_attention_keeps_small_weights(fp8):
    """In every block one key of weight 1 and value 0, and 15 of weight 2^-13 to 2^-22 which alone make the result: in float16 the smallest are below its least normal."""
    layer = make(num_blocks=256, Hq=4, Hkv=1, fp8=fp8)
    rng = np.random.default_rng(0)
    pool = random_pool(layer, rng)
    k, v = pool.view(256, 1, 2, 16, 128)[:, 0, 0], pool.view(256, 1, 2, 128, 16)[:, 0, 1]
    k.zero_()
    k[:, 0, 0] = torch.tensor(1.0).to(torch.float8_e4m3fn).view(torch.uint8).item() if fp8 else 1.0
    v[:, :, 0] = 0
    table, kv, start = np.arange(256).reshape(1, 256), [4096], np.array([0, 10])
    q, r = torch.zeros(10, 4, 128, dtype=torch.bfloat16, device=DEV), np.arange(10)[:, None, None]
    q[:, :, 0] = (torch.arange(13, 23, device=DEV) * (math.log(2.0) * math.sqrt(128)))[:, None].to(torch.bfloat16)
    for blocks in (np.arange(256), np.arange(256)[::-1], np.arange(1)):
        blocks = np.ascontiguousarray(blocks).reshape(1, 1, -1)
        n = blocks.size
        got = host(layer.attn_blocks(q, pool, i32(table), i32(kv), i32(start), i32(blocks), i32([n])))
        want, weight, size = ref.attend(host(q), pool_values(layer, pool), table, kv, start, blocks, [n], 16, np.zeros(q.shape))
        # run_attend's bound with the weights' own rounding: bfloat16 cuts off less than 2^-7 and rounds that by at most 2^-8 of it; float16 holds 2^6 times the weight, 2^-(7 + r), to half of 2^-24 or of 2^-10 of
        # itself (q is rounded, so the exponent is off by up to 23 x 2^-8)
        own = np.maximum(2.0 ** -11, 2.0 ** (r + 0.1 - 18)) if fp8 else 2.0 ** -15
        tol = 2.0 ** -8 * np.abs(want) + weight * (2 * 131 * E24 * size + 2.0 ** -17 + 16 * n * E24 + own)
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    layer.close()


# ---- NaN and infinities in what is read -----------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(fp8=True), dict(Hq=40, Hkv=2), dict(D=64), dict(D=64, bf16=False), dict(bf16=False), dict(bk=32), dict(bk=8), dict(D=36, bk=5),
                                dict(D=36, bk=5, fp8=True), dict(mode=1), dict(mode=1, bf16=False)], ids=str)
@pytest.mark.parametrize("top", [7, 120])
def test_attention_does_not_hide_nan(kw, top):
    """A NaN or an infinite score where it counts gives NaN, as the formula does, in these rows and heads alone; 120 entries of few sequences: in parts that are joined."""
    print("case:", kw, top, flush=True)
    layer = make(num_blocks=200, **kw)
    c, rng = layer.cfg, np.random.default_rng(top)
    bk, D, Hkv, g = c.block_size, c.head_dim, c.n_kv_heads, c.n_q_heads // c.n_kv_heads
    pool = random_pool(layer, rng)
    nan = torch.tensor(float("nan")).to(torch.float8_e4m3fn).view(torch.uint8).item() if c.kv_fp8 else float("nan")
    table = rng.permutation(195).reshape(5, 39)
    kv, rows = np.full(5, 39 * bk), [3, 2, 2, 1, 2]
    start = np.concatenate([[0], np.cumsum(rows)])
    blocks = rng.integers(0, 38, (5, Hkv, top))
    blocks[1, :, top // 2] = 38                                          # listed, with a NaN key for one kv-head
    pool.view(200, Hkv, 2, bk, D)[table[1, 38], Hkv - 1, 0, 1, 2] = nan
    for b in table[2]:                                                   # nothing but NaN keys for one kv-head
        pool.view(200, Hkv, 2, bk, D)[b, 0, 0, :, 0] = nan
    pool.view(200, Hkv, 2, D, bk)[table[3, blocks[3, 0, 0]], 0, 1, 3, bk - 1] = nan  # a NaN value: of one channel
    q = torch.tensor(rng.standard_normal((start[-1], c.n_q_heads, D)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
    q[0, 1, 5] = float("nan")                                            # a query
    q[1, c.n_q_heads - 1, 0] = float("inf")                              # scores of both infinities
    q[2, 0] = float("nan")
    out = torch.full(q.shape, 7.0, dtype=c.torch_dtype, device=DEV)
    layer.attn_blocks(q, pool, i32(table), i32(kv), i32(start), i32(blocks), i32([top] * 5), out)
    got = host(out)
    with np.errstate(invalid="ignore"):
        want, weight, size = ref.attend(host(q), pool_values(layer, pool), table, kv, start, blocks, [top] * 5, bk, np.zeros(q.shape))
    bad = np.isnan(want)
    heads = bad.any(-1)                                                  # what the above says, of the oracle
    assert heads[0, 1] and heads[1, -1] and heads[2, 0] and heads[3:5, -g:].all() and heads[5:7, :g].all() and heads[7, :g].all() and not heads[8:].any()
    assert bad[7, :g].sum() == g and heads.sum() == 3 + 2 * g + 2 * g + g
    assert np.array_equal(np.isnan(got), bad)
    ds = (D + 3) * E24 * size                                            # run_attend's bound
    tol = (2.0 ** -8 if c.bf16 else E24) * np.abs(want) + weight * (2 * ds + 2.0 ** -17 + top * bk * E24 + (2.0 ** -8 if c.bf16 else 0.0))
    assert (np.abs(got - want) <= tol)[~bad].all()
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(Hq=40, Hkv=2), dict(D=64), dict(D=64, bf16=False), dict(bk=32), dict(bk=8), dict(mode=1)], ids=str)
@pytest.mark.parametrize("top", [1, 7, 120])
def test_infinite_values_stay_infinite(kw, top):
    """Values of plus or minus infinity under positive weights make their channels infinite, and no other."""
    print("case:", kw, top, flush=True)
    layer = make(num_blocks=200, **kw)
    c, rng = layer.cfg, np.random.default_rng(top)
    bk, D, Hkv = c.block_size, c.head_dim, c.n_kv_heads
    pool = random_pool(layer, rng)
    table, kv, start = rng.permutation(195).reshape(5, 39), np.full(5, 39 * bk), np.array([0, 3, 5, 7, 8, 10])
    blocks = rng.integers(0, 39, (5, Hkv, top))
    v = pool.view(200, Hkv, 2, D, bk)[:, :, 1]
    for s in range(4):
        v[table[s, blocks[s, 0, top // 2]], 0, s, rng.integers(0, bk)] = float("inf")
        v[table[s, blocks[s, 0, top // 2]], 0, D - 1 - s, :] = -float("inf")
    q = torch.tensor(rng.standard_normal((10, c.n_q_heads, D)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
    q[0] = 0                                                             # weights of 1: nothing is left for a second product
    got = host(layer.attn_blocks(q, pool, i32(table), i32(kv), i32(start), i32(blocks), i32([top] * 5)))
    want, _, _ = ref.attend(host(q), pool_values(layer, pool), table, kv, start, blocks, [top] * 5, bk, np.zeros(q.shape))
    inf = np.isinf(want)
    assert inf.sum() == 8 * (c.n_q_heads // Hkv) * 2 and not np.isnan(want).any()
    assert np.array_equal(np.where(inf, got, 0), np.where(inf, want, 0)) and np.isfinite(got[~inf]).all()
    layer.close()


# ---- sizes ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,rows", [(dict(Hq=1, Hkv=1, D=64), (1 << 23) + 237), (dict(Hq=1, Hkv=1, D=2, bk=5, bf16=False), (1 << 24) + 37)], ids=str)
def test_append_of_more_rows_than_a_launch_holds(kw, rows):
    """Every row is there, and those around the borders, with blocks that go on across one, are the rows of a small call."""
    print("case:", kw, rows, flush=True)
    layer = make(num_blocks=100, **kw)
    c, edge = layer.cfg, 1 << 23
    gen = torch.Generator(device=DEV).manual_seed(1)
    qkv = torch.randn(rows, 3 * c.head_dim, generator=gen, device=DEV).to(c.torch_dtype)
    pos = (torch.arange(rows, device=DEV) % 100000).int()
    slot = torch.full((rows,), -1, dtype=torch.int64, device=DEV)
    parts = [slice(0, 64), slice(edge - 40, edge + 40), slice(rows - 150, rows)]
    for part, at in zip(parts, (3, 101, 250)):
        slot[part] = at + torch.arange(part.stop - part.start, device=DEV)
    q = torch.full((rows, 1, c.head_dim), float("nan"), dtype=c.torch_dtype, device=DEV)
    pools = [torch.zeros(c.pool_shape(), dtype=c.pool_dtype, device=DEV) for _ in range(2)]
    layer.rope_append(qkv, pos, slot, pools[0], q)
    assert not bool(torch.isnan(q).any())
    for part in parts:
        assert same_bits(layer.rope_append(qkv[part].clone(), pos[part].clone(), slot[part].clone(), pools[1]), q[part])
    assert same_bits(*pools) and int((pools[1] != 0).sum()) >= 280 * 2 * c.head_dim
    layer.close()


# ---- a graph that outlives its lengths --------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(Hq=8, Hkv=2), dict(Hq=8, Hkv=2, fp8=True, qk_norm=True), dict(Hq=4, Hkv=4, D=64, bf16=False), dict(Hq=6, Hkv=2, D=96)], ids=str)
@pytest.mark.parametrize("columns", [300, 1500, 40000])
def test_captured_step_over_a_wide_table(kw, columns):
    """A table as wide as its sequences may become: scores and choice are launches of their own.  Every replay is the eager step, and the step over a
    table that is as wide as its sequences are, bit for bit."""
    print("case:", kw, columns, flush=True)
    layer = make(num_blocks=400, **kw)
    loops = [_loop(layer, 5) for _ in range(3)]                              # narrow, wide, wide and captured
    for b in loops[1:]:
        b["table"] = torch.cat([b["table"], torch.full((b["table"].shape[0], columns - 40), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    _step(layer, _loop(layer, 5))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(layer, loops[2])
    for i in range(18):
        for b in loops:
            b["qkv"].mul_(-1)
        _step(layer, loops[0])
        _step(layer, loops[1])
        graph.replay()
        if i % 4 == 0:
            torch.cuda.synchronize()
        narrow, eager, replayed = ([x[:, :40] if n == 2 else x for n, x in enumerate(_state(b))] for b in loops)
        assert all(same_bits(a, b) and same_bits(a, d) for a, b, d in zip(narrow, eager, replayed)), i
        (loops[2]["out"].float() * 2).sum().item()
    layer.close()
