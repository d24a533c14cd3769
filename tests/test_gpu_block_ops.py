"""The operators of include/icarus_blocks.h on the GPU against plain float64 (block_reference.py), at the sizes and contents where they can go
wrong.  Whole numbers, codes, scales and selections are equal; floats are within bounds that are derived beside them."""
import numpy as np
import pytest
import torch

import block_reference as ref
from paper_2603_13281_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E24 = 2.0 ** -24  # half a step of float32


def make(Hq=8, Hkv=2, D=128, bk=16, num_blocks=64, bf16=True, fp8=False, qk_norm=False, k_scale=1.0, v_scale=1.0, mode=0, theta=5e5, seed=0, max_position=1 << 20):
    dt = torch.bfloat16 if bf16 else torch.float32
    one = torch.zeros(512, dtype=dt, device=DEV)  # no projection is read
    w = {p: one for p in binding.PROJ + ("norm_attn", "norm_ffn")}
    if qk_norm:
        gen = torch.Generator().manual_seed(seed)
        w["q_norm"], w["k_norm"] = ((1 + 0.2 * torch.randn(D, generator=gen)).to(dt).to(DEV) for _ in range(2))
    cfg = binding.LayerConfig(d_model=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, d_ffn=256, block_size=bk, num_blocks=num_blocks, bf16=bf16, qk_norm=qk_norm,
                              max_position=max_position, rope_theta=theta, rms_eps=1e-6, kv_fp8=fp8, k_scale=k_scale, v_scale=v_scale)
    layer = binding.IcarusLayer(cfg, w)
    layer.set_kernel_mode(mode)
    layer.norms = (w.get("q_norm"), w.get("k_norm"))
    return layer


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def host(t):
    return t.detach().cpu().double().numpy()


def pool_values(layer, pool):
    c = layer.cfg
    if not c.kv_fp8:
        return host(pool)
    v = host(pool.view(torch.float8_e4m3fn))
    return v * np.array([np.float32(c.k_scale), np.float32(c.v_scale)], dtype=np.float64)[:, None]


def random_pool(layer, rng, unit=1.0):
    c = layer.cfg
    x = torch.tensor(rng.standard_normal(c.pool_shape(), dtype=np.float32) * unit)
    if c.kv_fp8:
        x[:, :, 0] /= c.k_scale
        x[:, :, 1] /= c.v_scale
        return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
    return x.to(c.torch_dtype).to(DEV)


# ---- growth of the sequences --------------------------------------------------------------------------------------------

def run_extend(ctx, new, streams, free, used, max_rows, bk=16, num_blocks=1000, max_blocks=None, max_position=1 << 20, table=None, seed=0):
    rng = np.random.default_rng(seed)
    ctx, new = np.asarray(ctx, dtype=np.int64), np.asarray(new, dtype=np.int64)
    S = len(ctx)
    if max_blocks is None:
        max_blocks = max([1] + [ref.blocks_of(max(0, int(c)) + max(0, int(n)), bk) for c, n in zip(ctx, new)])
    if table is None:
        table = np.full((S, max_blocks), -7)
        for s in range(S):
            n = min(max_blocks, ref.blocks_of(max(0, ctx[s]), bk))
            table[s, :n] = rng.integers(0, num_blocks, n)
    want = ref.extend(ctx, new, streams, table, free, used, max_rows, bk, num_blocks, max_position)
    layer = make(bk=bk, num_blocks=num_blocks, max_position=max_position)
    m = binding.SequenceMap(S, max_rows, DEV)
    for t in (m.kv_lens, m.row_start, m.counts, m.row_seq, m.row_pos, m.row_slot):
        t.fill_(-99)
    dt = i32(table).reshape(S, max_blocks)
    layer.extend_sequences(m, i32(ctx), i32(new), dt, i32(free), i32([used]), None if streams is None else i32(streams))
    torch.cuda.synchronize()
    for name in ("kv_lens", "row_start", "row_seq", "row_pos", "row_slot", "counts"):
        got = getattr(m, name).cpu().numpy()
        assert np.array_equal(got, want[name]), (name, got[:40], want[name][:40])
    assert np.array_equal(dt.cpu().numpy(), want["block_tables"])
    layer.close()
    return want


@pytest.mark.parametrize("ctx,new,streams,n_free,used,max_rows", [
    ([0], [1], None, 4, 0, 1),                                   # the first token of all
    ([15, 16, 17, 0], [1, 1, 1, 0], [0, 3, 8, 5], 9, 2, 20),     # last place of a block, first of the next; no token: no streams
    ([100, 0, 33], [40, 16, 0], None, 20, 0, 56),                # rows used up to the last
    ([100, 0, 33], [40, 16, 1], None, 20, 0, 56),                # one row too few: the last sequence is refused
    ([0, 0, 0, 5], [64, 33, 16, 2], None, 6, 0, 200),            # blocks run out at the second; the third is refused too, the fourth needs none
    ([0, 7], [5, 5], [2, 2], 0, 0, 20),                          # no free list
    ([3], [2], None, 5, 9, 4),                                   # the list was overdrawn before
    ([3], [20], None, 5, -4, 40),
    ([], [], None, 5, 3, 7),                                     # no sequence: only rows without one
    ([4, 4], [0, 0], [1, 1], 5, 0, 3),
    ([1, 2], [3, 4], [1, 1], 5, 0, 0),                           # no room for a row
])
def test_extend(ctx, new, streams, n_free, used, max_rows):
    print("case:", ctx, new, flush=True)
    run_extend(ctx, new, streams, np.random.default_rng(1).permutation(1000)[:n_free], used, max_rows)


def test_extend_refuses_what_is_out_of_range():
    free = np.arange(50)
    run_extend([-1, 5, 5, 90, 5], [3, -2, 3, 20, 1], [0, 0, -1, 0, 1], free, 0, 64, max_position=100)       # negative lengths, streams, max_position
    run_extend([2 ** 31 - 1, 5], [2 ** 31 - 1, 2 ** 31 - 1], [2 ** 31 - 1, 0], free, 0, 33, max_blocks=4)      # sums beyond 32 bits
    run_extend([0, 60, 0], [10, 10, 10], None, free, 0, 64, max_blocks=4)                                    # passes the row of the table
    run_extend([8, 8, 0], [20, 1, 3], None, np.array([5, 1000, -3, 7]), 0, 64,
               table=np.array([[-1, -7], [1000, -7], [-7, -7]]), max_blocks=2)                               # ids outside the pool


@pytest.mark.parametrize("bk", [1, 5, 16, 128])
@pytest.mark.parametrize("S,top,streams", [(64, 1, True), (1023, 40, False), (1025, 7, True), (3000, 3, True)])
def test_extend_many(S, top, streams, bk):
    print("case:", S, top, bk, flush=True)
    rng = np.random.default_rng(S + bk)
    ctx, new = rng.integers(0, 300, S), rng.integers(0, top + 1, S)
    st = rng.integers(0, 9, S) if streams else None
    rows = int((new + (st if streams else 0) * (new > 0)).sum())
    need = int(sum(ref.blocks_of(c + n, bk) - ref.blocks_of(c, bk) for c, n in zip(ctx, new)))
    for n_free, room in ((need + 3, rows + 600), (need * 2 // 3 + 3, rows), (need + 3, rows * 3 // 4)):
        run_extend(ctx, new, st, rng.integers(0, 5000, n_free), 3, room, bk=bk, num_blocks=5000, seed=S)


def test_extend_long_prompts():
    run_extend([0, 31, 70000], [20000, 9999, 1], [0, 0, 8], np.random.default_rng(0).permutation(4000), 17, 40000, num_blocks=5000)


# ---- rotation and append --------------------------------------------------------------------------------------------------

def run_append(layer, rows, seed, ld=None, slots=None, pos=None):
    """Random rows at random places; returns nothing, asserts everything."""
    c = layer.cfg
    rng = np.random.default_rng(seed)
    width = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim
    n_slots = c.num_blocks * c.block_size
    whole = torch.tensor(rng.standard_normal((rows, ld or width), dtype=np.float32)).to(c.torch_dtype).to(DEV)
    qkv = whole[:, :width]
    if slots is None:
        slots = rng.permutation(n_slots)[:rows]
    if pos is None:
        pos = rng.integers(0, 100000, rows)
    slots, pos = np.asarray(slots, dtype=np.int64), np.asarray(pos, dtype=np.int64)
    pool = random_pool(layer, rng)
    before = pool.clone()
    out = torch.full((rows, c.n_q_heads, c.head_dim), 7.0, dtype=c.torch_dtype, device=DEV)
    layer.rope_append(qkv, i32(pos), torch.tensor(slots, device=DEV), pool, out)
    torch.cuda.synchronize()
    x = host(qkv).reshape(rows, -1, c.head_dim)
    Hq, Hkv, D, bk = c.n_q_heads, c.n_kv_heads, c.head_dim, c.block_size
    qn, kn = (None if w is None else host(w) for w in layer.norms)
    eps = float(np.float32(c.rms_eps))
    at = np.maximum(pos, 0)
    q, q_size = ref.rotated(x[:, :Hq], at, c.rope_theta, qn, eps)
    k, k_size = ref.rotated(x[:, Hq:Hq + Hkv], at, c.rope_theta, kn, eps)
    # float32 before the last rounding: the norm's sum of D squares, D / 64 in a row and 6 in a tree, its root (2 steps) and two products: under
    # (4 + 6 + 4 + 2) 2^-24 = 2^-20; the angle in half turns rounds by 2^-25, pi times that and 2 steps of cosine: under 2^-21; two products and a sum: 3 x 2^-24
    slack = 2.0 ** -19
    half = 2.0 ** -8 if c.bf16 else E24
    live = pos >= 0
    got = host(out)
    assert (got[~live] == 7.0).all()
    assert (np.abs(got - q) <= half * np.abs(q) + (1 + half) * slack * q_size)[live].all()
    want_k, want_v = (host(before.view(torch.float8_e4m3fn) if c.kv_fp8 else before).reshape(-1, Hkv, 2, bk, D) if p == 0 else None for p in (0, 1))
    gp = host(pool.view(torch.float8_e4m3fn) if c.kv_fp8 else pool)
    gk, gv = gp[:, :, 0].reshape(-1, Hkv, bk, D), gp[:, :, 1].reshape(-1, Hkv, D, bk).transpose(0, 1, 3, 2)
    bp = host(before.view(torch.float8_e4m3fn) if c.kv_fp8 else before)
    bk_, bv_ = bp[:, :, 0].reshape(-1, Hkv, bk, D), bp[:, :, 1].reshape(-1, Hkv, D, bk).transpose(0, 1, 3, 2)
    touched = np.zeros((len(gp), bk), dtype=bool)
    write = live & (slots >= 0) & (slots < n_slots)
    touched[slots[write] // bk, slots[write] % bk] = True
    keep = ~touched[:, None, :, None]
    same = lambda a, b: (a == b) | (np.isnan(a) & np.isnan(b))  # noqa: E731
    assert (same(gk, bk_) | ~keep).all() and (same(gv, bv_) | ~keep).all()
    for r in np.flatnonzero(write):
        b, o = slots[r] // bk, slots[r] % bk
        for got_, want, size, scale in ((gk[b, :, o], k[r], k_size[r], c.k_scale), (gv[b, :, o], x[r, Hq + Hkv:], 0.0, c.v_scale)):
            if c.kv_fp8:  # the quotient rounds once more; half a step of E4M3 is 2^-4 of the value, 2^-10 below the smallest normal
                want = np.clip(want / scale, -448, 448)
                ok = np.abs(got_ - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -10 + 2 * (slack * size / scale + E24 * np.abs(want))
            else:
                ok = np.abs(got_ - want) <= (half if np.ndim(size) else 0.0) * np.abs(want) + (1 + half) * slack * size
            assert ok.all(), (r, np.abs(got_ - want).max())


SHAPES = [dict(), dict(qk_norm=True), dict(Hq=4, Hkv=4, D=64, bf16=False, theta=1e4), dict(Hq=64, Hkv=8, qk_norm=True, fp8=True, k_scale=0.02, v_scale=0.013),
          dict(Hq=6, Hkv=1, D=256, bk=8), dict(Hq=3, Hkv=3, D=36, bk=5, qk_norm=True), dict(Hq=2, Hkv=1, D=2, bk=1, bf16=False), dict(Hq=4, Hkv=2, D=96, bk=32, fp8=True),
          dict(Hq=4, Hkv=2, D=64, bk=16, fp8=True, bf16=False, qk_norm=True), dict(Hq=5, Hkv=5, D=254, bk=3), dict(mode=1, qk_norm=True), dict(Hq=6, Hkv=2, D=192),
          dict(Hq=2, Hkv=2, D=256, bf16=False, qk_norm=True), dict(Hq=4, Hkv=2, D=64, qk_norm=True), dict(Hq=6, Hkv=3, D=16, bf16=False), dict(Hq=4, Hkv=4, D=128, bf16=False)]


@pytest.mark.parametrize("kw", SHAPES, ids=str)
@pytest.mark.parametrize("rows", [1, 17, 130])
def test_append(kw, rows):
    print("case:", kw, rows, flush=True)
    layer = make(num_blocks=200 if kw.get("bk", 16) < 4 else 64, **kw)
    run_append(layer, rows, seed=rows)
    layer.close()


@pytest.mark.parametrize("kw", SHAPES[:6], ids=str)
@pytest.mark.parametrize("off", [0, 1, 13])
def test_append_prompts(kw, off):
    """Consecutive positions from a place inside a block on, several sequences, blocks in any order: runs that begin and end inside a block."""
    print("case:", kw, off, flush=True)
    layer = make(num_blocks=96, **kw)
    bk = layer.cfg.block_size
    rng = np.random.default_rng(off)
    ids, pos, slots, at = rng.permutation(96), [], [], 0
    for n in (40, 1, bk, 2 * bk + 3, 5):
        nb = ref.blocks_of(off + n, bk)
        p = np.arange(off, off + n)
        pos += p.tolist()
        slots += (ids[at + p // bk] * bk + p % bk).tolist()
        at += nb
        off = (off + 3) % (2 * bk)
    slots[3], pos[5] = -1, -1                          # a row that writes nothing and a row that is none, inside a run
    slots[7] = layer.cfg.num_blocks * bk               # outside the pool
    run_append(layer, len(pos), seed=off, slots=slots, pos=pos)
    layer.close()


@pytest.mark.parametrize("ld", [1536 + 8, 1536 + 3, 2048])
def test_append_strided_rows(ld):
    layer = make(Hq=8, Hkv=2)
    run_append(layer, 33, seed=ld, ld=ld)
    layer.close()


def test_append_far_positions_and_none():
    layer = make(qk_norm=True, max_position=(1 << 31) - 1)
    run_append(layer, 5, seed=1, pos=[0, 1, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 2])
    out = layer.rope_append(torch.empty(0, 1536, dtype=torch.bfloat16, device=DEV), i32([]), torch.empty(0, dtype=torch.int64, device=DEV),
                            random_pool(layer, np.random.default_rng(0)))
    assert out.shape == (0, 8, 128)
    layer.close()


def test_append_streams_of_a_step():
    """A token step as extend_sequences lays it out: an encoder row that appends and rows of streams at its position, whose K and V may hold anything."""
    layer = make(Hq=32, Hkv=8, num_blocks=64)
    rows, rng = 60, np.random.default_rng(3)
    slots = np.where(np.arange(rows) % 5 == 0, rng.permutation(64 * 16)[:rows], -1)
    run_append(layer, rows, seed=3, slots=slots, pos=np.repeat(rng.integers(0, 9999, 12), 5))
    layer.close()


# ---- bounds of the keys -----------------------------------------------------------------------------------------------------

def run_bounds(layer, pool, table, a, z, max_new, seed=0):
    c = layer.cfg
    rng = np.random.default_rng(seed)
    codes = torch.tensor(rng.integers(-128, 128, (c.num_blocks, c.n_kv_heads, 2, c.head_dim)), dtype=torch.int8, device=DEV)
    scales = torch.tensor(rng.random((c.num_blocks, c.n_kv_heads)), dtype=torch.float32, device=DEV)
    values = host(pool.view(torch.float8_e4m3fn)) if c.kv_fp8 else host(pool)
    want = ref.bounds(values, table, a, z, c.block_size, c.head_dim, host(codes), host(scales))
    layer.key_bounds(pool, i32(table), i32(a), i32(z), codes, scales, max_new=max_new)
    torch.cuda.synchronize()
    assert np.array_equal(host(scales), want[1])
    assert np.array_equal(host(codes), want[0])


@pytest.mark.parametrize("kw", SHAPES, ids=str)
@pytest.mark.parametrize("max_new", [0, 1, 1000])
def test_bounds(kw, max_new):
    print("case:", kw, max_new, flush=True)
    kw = {k: v for k, v in kw.items() if k != "qk_norm"}
    layer = make(num_blocks=60, **kw)
    bk = layer.cfg.block_size
    rng = np.random.default_rng(max_new)
    pool = random_pool(layer, rng)
    table = rng.permutation(60)[:54].reshape(6, 9)
    table[4, 2], table[5, 0] = 60, -1                                     # ids outside the pool
    a = [0, 0, bk, 2 * bk + 1, 0, 0]
    z = [9 * bk, 1, 3 * bk - 1, 2 * bk + 1, 5 * bk, bk]                    # whole row, one token, part of a block, nothing
    run_bounds(layer, pool, table, a, z, max_new)
    run_bounds(layer, pool, table, [-5, 8 * bk, 3, 0, 7, 2 ** 31 - 1], [2, 2 ** 31 - 1, -4, 0, 6, 2 ** 31 - 1], max_new)   # negative, beyond the row
    layer.close()


@pytest.mark.parametrize("bf16", [True, False])
def test_bounds_of_extreme_keys(bf16):
    """Zeros, values at a step's border, the smallest and largest numbers, infinities and NaN; what is behind the last token is not read."""
    layer = make(num_blocks=12, bf16=bf16)
    k = torch.zeros(layer.cfg.pool_shape())
    kb = k[:, :, 0].view(12, 2, 16, 128)
    rng = np.random.default_rng(0)
    kb[1] = torch.tensor(rng.standard_normal((2, 16, 128))) * 1e-30
    kb[2] = torch.tensor(rng.standard_normal((2, 16, 128))) * 1e30
    kb[3, :, 4, 7] = 127 / 32                                             # exactly 127 steps
    kb[4, :, 4, 7] = -127.5 / 32
    kb[5, 0, 2, 3], kb[5, 1, 2, 3] = float("inf"), float("-inf")
    kb[6] = float("nan")
    kb[7, :, 5, 9] = float("nan")
    kb[7, :, 6, 9] = -2.5
    kb[8] = -1.0
    kb[9] = torch.tensor(rng.standard_normal((2, 16, 128)))
    kb[9, :, 6:] = float("nan")
    kb[10, :, 3, 1] = 2.0 ** -126
    kb[11] = torch.tensor(rng.standard_normal((2, 16, 128))) * 3e11       # around the largest step
    run_bounds(layer, k.to(layer.cfg.torch_dtype).to(DEV), np.arange(12).reshape(12, 1), [0] * 12, [16] * 9 + [6] + [16] * 2, 0)
    layer.close()


# ---- choice of the blocks -----------------------------------------------------------------------------------------------------

def run_select(layer, q, codes, scales, table, kv, row_start, top, first, last, hint=0):
    c = layer.cfg
    S = table.shape[0]
    blocks = torch.full((S, c.n_kv_heads, top), 99, dtype=torch.int32, device=DEV)
    counts = torch.full((S,), 99, dtype=torch.int32, device=DEV)
    layer.select_blocks(q, codes, scales, i32(table).reshape(table.shape), i32(kv), i32(row_start), blocks, counts, first=first, last=last, seq_rows=hint)
    torch.cuda.synchronize()
    want = ref.select(host(q), host(codes).astype(np.int64), host(scales), table, kv, row_start, top, first, last, c.block_size)
    assert np.array_equal(counts.cpu().numpy(), want[1])
    assert np.array_equal(blocks.cpu().numpy(), want[0]), np.argwhere(blocks.cpu().numpy() != want[0])[:5]
    return blocks, counts


def random_bounds(layer, rng, few=False):
    c = layer.cfg
    shape = (c.num_blocks, c.n_kv_heads, 2, c.head_dim)
    codes = rng.integers(-1, 2, shape) if few else rng.integers(-127, 128, shape)
    scales = 2.0 ** rng.integers(0 if few else -40, 1 if few else 41, shape[:2])
    return torch.tensor(codes, dtype=torch.int8, device=DEV), torch.tensor(scales, dtype=torch.float32, device=DEV)


@pytest.mark.parametrize("kw", SHAPES, ids=str)
@pytest.mark.parametrize("few", [False, True])
def test_select(kw, few):
    """few: codes and queries of few values, so that many blocks score alike."""
    print("case:", kw, few, flush=True)
    kw = {k: v for k, v in kw.items() if k != "qk_norm"}
    layer = make(num_blocks=300, **kw)
    c, rng = layer.cfg, np.random.default_rng(7)
    codes, scales = random_bounds(layer, rng, few)
    lens = [0, 1, 2, 17, 40, 100, 140]                                   # blocks of the sequences, none to many
    rows = [1, 2, 0, 9, 1, 5, 3]
    start = np.concatenate([[0], np.cumsum(rows)])
    q = rng.standard_normal((start[-1] + 2, c.n_q_heads, c.head_dim))
    if few:
        q = rng.integers(0, 2, q.shape) * (np.arange(c.head_dim) < 3)
    q = torch.tensor(q, dtype=torch.float32).to(c.torch_dtype).to(DEV)
    table = rng.integers(0, 300, (7, 140))
    table[5, 50], table[5, 60], table[6, :100] = 300, -1, -1            # ids outside the pool
    kv = [max(0, n * c.block_size - int(rng.integers(0, c.block_size))) for n in lens]
    for top, first, last in ((1, 0, 0), (3, 1, 2), (16, 0, 1), (64, 5, 7), (140, 1, 1), (200, 0, 0)):
        run_select(layer, q, codes, scales, table, kv, start, top, first, last, hint=int(rng.integers(0, 12)))
    layer.close()


def test_select_extremes():
    layer = make(num_blocks=40, bf16=False)
    rng = np.random.default_rng(2)
    codes, scales = random_bounds(layer, rng)
    q = torch.tensor(rng.standard_normal((6, 8, 128)), dtype=torch.float32, device=DEV)
    q[0] = 0
    q[1] = float("nan")
    q[2, :, ::2] = float("nan")
    q[3, :, 5] = float("inf")
    q[4] *= 1e30
    q[5] *= 1e-38
    table = rng.integers(0, 40, (6, 40))
    kv = [640] * 4 + [-3, 2 ** 31 - 1]                                    # negative: none; beyond the row: the row
    for start in ([0, 1, 2, 3, 4, 5, 6], [0, 6, 6, 6, 6, 6, 6], [0, 0, 0, 0, 0, 0, 0]):
        run_select(layer, q, codes, scales, table, kv, np.array(start), 7, 1, 1)
    codes.zero_()                                                         # every block scores alike
    run_select(layer, q, codes, scales, table, kv, np.arange(7), 7, 2, 0)
    layer.close()


@pytest.mark.parametrize("kw", [dict(Hq=16), dict(Hq=8, D=64), dict(Hq=8, D=192), dict(Hq=16, D=256), dict(bf16=False), dict(D=64, bf16=False), dict(D=192, bf16=False),
                                dict(D=256, bf16=False), dict(D=128, mode=1)], ids=str)
@pytest.mark.parametrize("max_blocks", [140, 500, 600])
def test_select_many_sequences(kw, max_blocks):
    print("case:", kw, max_blocks, flush=True)
    layer = make(num_blocks=300, **{"Hq": 8, "Hkv": 8, **kw})
    c, rng = layer.cfg, np.random.default_rng(5)
    S = 33
    codes, scales = random_bounds(layer, rng, True)
    rows = rng.integers(0, 5, S)
    rows[5] = 90                                                          # more queries than are held at a time
    start = np.concatenate([[0], np.cumsum(rows)])
    q = torch.tensor(rng.standard_normal((start[-1], c.n_q_heads, c.head_dim)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
    table, kv = rng.integers(0, 300, (S, max_blocks)), rng.integers(0, max_blocks * 16 + 1, S)
    kv[:3] = max_blocks * 16, 0, 1
    run_select(layer, q, codes, scales, table, kv, start, 9, 1, 2)
    layer.close()


@pytest.mark.parametrize("max_blocks", [257, 1100, 4100, 9000])
def test_select_long(max_blocks):
    print("case:", max_blocks, flush=True)
    layer = make(num_blocks=512, Hq=4, Hkv=2, D=64)
    rng = np.random.default_rng(max_blocks)
    for few in (False, True):
        codes, scales = random_bounds(layer, rng, few)
        q = torch.tensor(rng.standard_normal((2, 4, 64)), dtype=torch.float32).to(torch.bfloat16).to(DEV)
        table = rng.integers(0, 512, (2, max_blocks))                     # a block may stand in a table often: equal scores
        for top in (3, 100, max_blocks - 1):
            run_select(layer, q, codes, scales, table, [max_blocks * 16, (max_blocks - 5) * 16 - 3], np.array([0, 1, 2]), top, 1, 2)
    layer.close()


# ---- attention over the blocks ------------------------------------------------------------------------------------------------

def run_attend(layer, q, pool, table, kv, row_start, blocks, counts, hint=0):
    c = layer.cfg
    out = torch.full(q.shape, 7.0, dtype=c.torch_dtype, device=DEV)
    layer.attn_blocks(q, pool, i32(table).reshape(table.shape), i32(kv), i32(row_start), i32(blocks).reshape(blocks.shape), i32(counts), out, seq_rows=hint)
    torch.cuda.synchronize()
    want, weight, size = ref.attend(host(q), pool_values(layer, pool), table, kv, row_start, blocks, counts, c.block_size, np.full(q.shape, 7.0))
    got = host(out)
    # A score is a sum of D products in float32 (D half steps of the sum of sizes, and 3 for the scale and the code's scale): off by ds, so each p by
    # 2 ds of itself (its own and the sum's); exp, its argument (below 2^7 where p counts) and the sums over up to n tokens: 2^-17 + n 2^-24, all of sum p |v|.  On the
    # matrix cores p is rounded to bfloat16: 2^-8 of sum p |v| more.
    ds = (c.head_dim + 3) * E24 * size
    n = blocks.shape[2] * c.block_size
    tol = (2.0 ** -8 if c.bf16 else E24) * np.abs(want) + weight * (2 * ds + 2.0 ** -17 + n * E24 + (2.0 ** -8 if c.bf16 else 0.0))
    ok = np.abs(got - want) <= tol
    assert ok.all(), (np.argwhere(~ok)[:5], np.abs(got - want).max())
    return out


ATTN = SHAPES + [dict(Hq=32, Hkv=8), dict(Hq=8, Hkv=8), dict(Hq=16, Hkv=2, fp8=True, k_scale=0.05, v_scale=0.03), dict(mode=1), dict(Hq=40, Hkv=2),
               dict(D=80), dict(D=128, bf16=False, fp8=True, v_scale=0.5), dict(D=112, bf16=False), dict(Hq=24, Hkv=1, D=96, fp8=True), dict(D=64, fp8=True, k_scale=2.0),
               dict(D=240, fp8=True), dict(D=256), dict(D=256, bf16=False, fp8=True), dict(D=208, bf16=False), dict(Hq=34, Hkv=2, D=48, bf16=False, fp8=True),
               dict(bk=32), dict(bk=48, fp8=True, k_scale=0.3), dict(bk=64, bf16=False), dict(bk=128, D=64), dict(bk=80, D=48, fp8=True, bf16=False)]


@pytest.mark.parametrize("kw", ATTN, ids=str)
@pytest.mark.parametrize("top", [1, 7, 70])
def test_attend(kw, top):
    """Rows 0 to 9 and more to a sequence, lengths that end inside a block, at its end and at zero, lists in any order with gaps, repeats and entries
    outside; everything that must not be read holds NaN."""
    print("case:", kw, top, flush=True)
    kw = {k: v for k, v in kw.items() if k != "qk_norm"}
    layer = make(num_blocks=220, **kw)
    c, rng = layer.cfg, np.random.default_rng(top)
    bk = c.block_size
    pool = random_pool(layer, rng)
    S, max_blocks = 7, 30
    table = rng.permutation(210).reshape(S, max_blocks)
    table[2, 3], table[2, 4] = 220, -1
    kv = np.array([30 * bk, 30 * bk - 1, 29 * bk + 1, 12 * bk, 1, 0, 21 * bk + bk // 2])
    rows = np.array([1, 9, 2, 13, 3, 4, 0])
    start = np.concatenate([[0], np.cumsum(rows)])
    q = torch.tensor(rng.standard_normal((start[-1] + 3, c.n_q_heads, c.head_dim)) * 2, dtype=torch.float32).to(c.torch_dtype).to(DEV)
    blocks = rng.integers(0, max_blocks, (S, c.n_kv_heads, top))          # repeats, and blocks behind the length
    blocks[0, :, 0], blocks[3, :, -1] = -1, max_blocks
    blocks[2, :, top // 2] = 3
    counts = np.array([top, top, max(1, top - 3), top, top, top, top])
    blocks[4, :, -1] = 0
    listed = np.zeros((221, bk), dtype=bool)                              # what may be read
    for s in range(S):
        for b in set(blocks[s, :, : counts[s]].ravel().tolist()):
            if 0 <= b < max_blocks and 0 <= table[s, b] < 220:
                listed[table[s, b], : max(0, min(bk, kv[s] - b * bk))] = True
    gone = torch.tensor(~listed[:220], device=DEV)
    nan = torch.tensor(float("nan")).to(torch.float8_e4m3fn).view(torch.uint8).item() if c.kv_fp8 else float("nan")
    pool.view(220, c.n_kv_heads, 2, bk, c.head_dim)[:, :, 0].masked_fill_(gone[:, None, :, None], nan)
    pool.view(220, c.n_kv_heads, 2, c.head_dim, bk)[:, :, 1].masked_fill_(gone[:, None, None, :], nan)
    for hint in (0, 1, 9):
        run_attend(layer, q, pool, table, kv, start, blocks, counts, hint)
    run_attend(layer, q, pool, table, kv, start, blocks, np.zeros(S, dtype=int))        # nothing is listed: zeros
    run_attend(layer, q, pool, table, kv, start, blocks, np.array([-5, 1, counts[2], 10 ** 9, 0, 1, 1]))  # within what may be read
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True, k_scale=0.5), dict(bf16=False)], ids=str)
def test_attend_large_scores(kw):
    """Scores in the hundreds, rising and falling along the list: the running maximum moves."""
    layer = make(num_blocks=40, Hq=4, Hkv=1, **kw)
    c, rng = layer.cfg, np.random.default_rng(0)
    pool = random_pool(layer, rng)
    table = np.arange(40).reshape(1, 40)
    q = torch.tensor(rng.standard_normal((3, 4, 128)) * 30, dtype=torch.float32).to(c.torch_dtype).to(DEV)
    for order in (np.arange(40), np.arange(40)[::-1], rng.permutation(40)):
        run_attend(layer, q, pool, table, [640], np.array([0, 3]), order.reshape(1, 1, 40).copy(), [40])
    layer.close()


@pytest.mark.parametrize("kw", [dict(), dict(bf16=False), dict(D=64), dict(mode=1)], ids=str)
def test_attend_scores_of_minus_infinity(kw):
    """Keys whose scores are minus infinity weigh nothing, wherever in the list they stand and whoever sees them first."""
    layer = make(num_blocks=40, Hq=8, Hkv=2, **kw)
    c, rng = layer.cfg, np.random.default_rng(2)
    pool = random_pool(layer, rng)
    pool.view(40, 2, 2, 16, c.head_dim)[:24, :, 0, :, 0] = -float("inf")
    q = torch.tensor(rng.standard_normal((3, 8, c.head_dim)), dtype=torch.float32)
    q[:, :, 0] = 1.0
    q = q.to(c.torch_dtype).to(DEV)
    table, start, kv = np.arange(40).reshape(1, 40), np.array([0, 3]), [640]
    rest = np.broadcast_to(np.arange(24, 40), (1, 2, 16)).copy()
    alone = run_attend(layer, q, pool, table, kv, start, rest, [16])
    want, weight, size = ref.attend(host(q), pool_values(layer, pool), table, kv, start, rest, [16], 16, np.zeros(q.shape))
    for order in (np.arange(40), np.arange(40)[::-1], rng.permutation(40)):
        out = torch.empty_like(q)
        blocks = np.broadcast_to(order, (1, 2, 40)).copy()
        layer.attn_blocks(q, pool, i32(table).reshape(table.shape), i32(kv), i32(start), i32(blocks).reshape(blocks.shape), i32([40]), out)
        # both within run_attend's bound of the same values
        tol = (2.0 ** -8 if c.bf16 else E24) * np.abs(want) + weight * (2 * (c.head_dim + 3) * E24 * size + 2.0 ** -17 + 640 * E24 + (2.0 ** -8 if c.bf16 else 0.0))
        assert (np.abs(host(out) - host(alone)) <= 2 * tol).all()
    layer.close()


def test_attend_lists_in_many_parts():
    """Lists longer than a workgroup holds, of few sequences among many without rows; and of no entry at all."""
    for kw, S, top in ((dict(), 300, 700), (dict(Hq=4, Hkv=4, D=64, bf16=False), 300, 600), (dict(), 2, 2600), (dict(Hq=4, Hkv=2, D=64, bf16=False), 1, 2600), (dict(), 3, 0)):
        print("case:", kw, S, top, flush=True)
        layer = make(num_blocks=64, **kw)
        c, rng = layer.cfg, np.random.default_rng(top)
        pool = random_pool(layer, rng)
        table = rng.integers(0, 64, (S, 64))
        kv = rng.integers(900, 1025, S)
        rows = np.zeros(S, dtype=int)
        rows[[0, S // 2, S - 1]] = (2, 5, 1) if S > 2 else (3, 3, 3)
        start = np.concatenate([[0], np.cumsum(rows)])
        q = torch.tensor(rng.standard_normal((start[-1], c.n_q_heads, c.head_dim)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
        blocks = rng.integers(0, 64, (S, c.n_kv_heads, top))
        for counts in (np.full(S, top), rng.integers(0, top + 1, S)):
            run_attend(layer, q, pool, table, kv, start, blocks, counts)
        layer.close()


def test_blocks_beyond_32_bits():
    """A pool of 9.2 GB, elements beyond 2^32: the same bits as from a small pool that holds the same blocks."""
    n_big, n_small = 140000, 48
    rng = np.random.default_rng(0)
    high = np.sort(rng.choice(np.arange(n_big - 8000, n_big), n_small, replace=False))
    high[-1] = n_big - 1
    results = []
    qkv = torch.tensor(rng.standard_normal((40, 48 * 128)), dtype=torch.float32).to(torch.bfloat16).to(DEV)
    small_pool = None
    for n, ids in ((n_small, np.arange(n_small)), (n_big, high)):
        layer = make(Hq=32, Hkv=8, num_blocks=n, qk_norm=True)
        pool = torch.empty(layer.cfg.pool_shape(), dtype=torch.bfloat16, device=DEV)
        where = torch.tensor(ids, device=DEV)
        if small_pool is None:
            small_pool = random_pool(layer, np.random.default_rng(1)).clone()
        pool[where] = small_pool
        table = ids[np.random.default_rng(2).permutation(n_small)].reshape(3, 16)
        kv = np.array([256, 255, 130])
        slots = np.concatenate([table[0, 15] * 16 + np.arange(3), table[1, 14] * 16 + np.arange(16), table[2, 8] * 16 + np.arange(2), np.full(19, -1)])
        q = torch.zeros(40, 32, 128, dtype=torch.bfloat16, device=DEV)
        layer.rope_append(qkv, i32(np.arange(40) * 7), torch.tensor(slots, dtype=torch.int64, device=DEV), pool, q)
        codes, scales = layer.new_key_bounds(DEV)
        layer.key_bounds(pool, i32(table), i32([0, 0, 0]), i32(kv), codes, scales)
        blocks, counts = torch.zeros(3, 8, 6, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
        start = i32([0, 9, 30, 40])
        layer.select_blocks(q, codes, scales, i32(table), i32(kv), start, blocks, counts)
        out = layer.attn_blocks(q, pool, i32(table), i32(kv), start, blocks, counts)
        fresh = i32(ids[:6] if n == n_small else high[:6])
        m = binding.SequenceMap(1, 70, DEV)
        grown = torch.full((1, 5), -1, dtype=torch.int32, device=DEV)
        layer.extend_sequences(m, i32([0]), i32([70]), grown, fresh, i32([0]))
        slot = m.row_slot.clone()
        at = torch.searchsorted(where, slot // 16) * 16 + slot % 16  # as the small pool counts
        results.append([q, pool[where], codes[where], scales[where], blocks, counts, out, at])
        assert int(slot.max()) // 16 == int(ids[:5].max())
        torch.cuda.synchronize()
        layer.close()
        del pool
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*results))


def test_integer_arrays_need_only_their_own_alignment():
    layer = make(num_blocks=64)
    c, rng = layer.cfg, np.random.default_rng(0)
    off = lambda a: torch.cat([i32([0]), i32(a).reshape(-1)])[1:].reshape(np.shape(a))  # noqa: E731: four bytes behind an aligned address
    pool = random_pool(layer, rng)
    table, kv, start = rng.permutation(64)[:60].reshape(3, 20), np.array([320, 77, 300]), np.array([0, 1, 4, 6])
    codes, scales = layer.new_key_bounds(DEV)
    scales = torch.ones(scales.numel() + 1, device=DEV)[1:].view(scales.shape)
    layer.key_bounds(pool, off(table), off([0, 0, 0]), off(kv), codes, scales)
    q = torch.tensor(rng.standard_normal((6, 8, 128)), dtype=torch.float32).to(torch.bfloat16).to(DEV)
    blocks, counts = off(np.zeros((3, 2, 7), dtype=int)), off([0, 0, 0])
    layer.select_blocks(q, codes, scales, off(table), off(kv), off(start), blocks, counts)
    want = ref.select(host(q), host(codes).astype(np.int64), host(scales), table, kv, start, 7, 1, 2, 16)
    assert np.array_equal(blocks.cpu().numpy(), want[0])
    out = layer.attn_blocks(q, pool, off(table), off(kv), off(start), blocks, counts)
    again = layer.attn_blocks(q, pool, i32(table), i32(kv), i32(start), blocks.clone(), counts.clone())
    assert torch.equal(out, again)
    new, used = off([1, 0, 17]), off([2])
    m, free = binding.SequenceMap(3, 21, DEV), off(np.arange(40))
    t2 = off(np.concatenate([table, np.full((3, 2), -1)], 1))
    wide = t2.cpu().numpy().copy()
    layer.extend_sequences(m, off(kv), new, t2, free, used, streams=off([2, 1, 1]))
    want = ref.extend(kv, [1, 0, 17], [2, 1, 1], wide, np.arange(40), 2, 21, 16, 64, 1 << 20)
    for name in ("kv_lens", "row_start", "row_seq", "row_pos", "row_slot", "counts"):
        assert np.array_equal(getattr(m, name).cpu().numpy(), want[name]), name
    assert np.array_equal(t2.cpu().numpy(), want["block_tables"])
    layer.close()


# ---- together -------------------------------------------------------------------------------------------------------------------

def test_workspaces_elsewhere_are_refused():
    layer = make(num_blocks=8)
    q, pool, table = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device=DEV), random_pool(layer, np.random.default_rng(0)), i32([[0, 1]])
    codes, scales = layer.new_key_bounds(DEV)
    blocks, counts = torch.zeros(1, 2, 3, dtype=torch.int32, device=DEV), i32([0])
    for ws in (torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 20, 2, dtype=torch.uint8, device=DEV)[:, 0], 5):
        with pytest.raises(ValueError):
            layer.select_blocks(q, codes, scales, table, i32([20]), i32([0, 1]), blocks, counts, workspace=ws)
        with pytest.raises(ValueError):
            layer.attn_blocks(q, pool, table, i32([20]), i32([0, 1]), blocks, counts, workspace=ws)
    with pytest.raises(binding.IcarusError):
        layer.attn_blocks(q, pool, table, i32([20]), i32([0, 1]), blocks, counts, workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    layer.close()


def test_a_step_is_the_layers_attention():
    """Growth, append, bounds, choice of all blocks, attention over them: what icarus_attn_shared_kv gives on the same cache."""
    for kw in (dict(Hq=8, Hkv=2), dict(Hq=8, Hkv=2, fp8=True, k_scale=0.02, v_scale=0.02), dict(Hq=4, Hkv=4, D=64, bf16=False)):
        print("case:", kw, flush=True)
        layer = make(num_blocks=256, qk_norm=True, **kw)
        c, rng = layer.cfg, np.random.default_rng(5)
        S, max_blocks = 5, 40
        width = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim
        ids = rng.permutation(256)
        table, free = torch.full((S, max_blocks), -1, dtype=torch.int32, device=DEV), i32(ids)
        pool = torch.zeros(c.pool_shape(), dtype=c.pool_dtype, device=DEV)
        codes, scales = layer.new_key_bounds(DEV)
        lens, used = i32([0] * S), i32([0])
        plans = [([300, 17, 16, 1, 120], [0] * S, 454), ([1] * S, [8, 0, 3, 1, 2], 19), ([1, 0, 1, 1, 1], [2, 1, 0, 8, 8], 30)]
        for new, act, rows in plans:
            m = binding.SequenceMap(S, rows, DEV)
            layer.extend_sequences(m, lens, i32(new), table, free, used, streams=i32(act))
            assert int(m.counts[1]) == 0
            qkv = torch.tensor(rng.standard_normal((rows, width)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
            q = layer.rope_append(qkv, m.row_pos, m.row_slot, pool)
            layer.key_bounds(pool, table, lens, m.kv_lens, codes, scales, max_new=max(new))
            lens, used = m.kv_lens, m.counts[:1].clone()
        blocks = torch.empty(S, c.n_kv_heads, max_blocks, dtype=torch.int32, device=DEV)
        counts = torch.empty(S, dtype=torch.int32, device=DEV)
        layer.select_blocks(q, codes, scales, table, lens, m.row_start, blocks, counts, seq_rows=9)
        out = layer.attn_blocks(q, pool, table, lens, m.row_start, blocks, counts, seq_rows=9)
        torch.cuda.synchronize()
        n = int(m.row_start[-1])
        assert n == 22 and counts.cpu().tolist() == [ref.blocks_of(x, 16) for x in lens.cpu().tolist()]
        dense = layer.attn_shared_kv(q[:n].contiguous(), pool, table.clamp(min=0), lens.cpu().numpy(), m.row_seq[:n].cpu().numpy())
        want, weight, size = ref.attend(host(q), pool_values(layer, pool), table.cpu().numpy(), lens.cpu().numpy(), m.row_start.cpu().numpy(), blocks.cpu().numpy(),
                                        counts.cpu().numpy(), 16, np.zeros(q.shape))
        # both are within the bound of run_attend, so they are within twice that of each other
        tol = (2.0 ** -8 if c.bf16 else E24) * np.abs(want) + weight * (2 * (c.head_dim + 3) * E24 * size + 2.0 ** -17 + 640 * E24 + (2.0 ** -8 if c.bf16 else 0.0))
        assert (np.abs(host(out) - want) <= tol)[:n].all() and (host(out)[n:] == 0).all()
        assert (np.abs(host(out)[:n] - host(dense)) <= 2 * tol[:n]).all()
        layer.close()


def _loop(layer, seed, S=6, steps=5):
    """A serving loop's buffers and its step: lengths, tables and the free list live on the GPU."""
    c, rng = layer.cfg, np.random.default_rng(seed)
    width = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim
    b = dict(lens=i32(rng.integers(1, 400, S)), new=i32([1] * S), act=i32(rng.integers(0, 5, S)), used=i32([0]), map=binding.SequenceMap(S, 40, DEV))
    need = [ref.blocks_of(x, 16) for x in b["lens"].cpu().tolist()]
    ids = rng.permutation(c.num_blocks)
    table = np.full((S, 40), -1)
    at = 0
    for s in range(S):
        table[s, :need[s]] = ids[at:at + need[s]]
        at += need[s]
    b["table"], b["free"] = i32(table), i32(ids[at:])
    b["pool"] = random_pool(layer, rng)
    b["codes"], b["scales"] = layer.new_key_bounds(DEV)
    layer.key_bounds(b["pool"], b["table"], i32([0] * S), b["lens"], b["codes"], b["scales"])
    b["qkv"] = torch.tensor(rng.standard_normal((40, width)), dtype=torch.float32).to(c.torch_dtype).to(DEV)
    b["q"] = torch.zeros(40, c.n_q_heads, c.head_dim, dtype=c.torch_dtype, device=DEV)
    b["out"] = torch.zeros_like(b["q"])
    b["blocks"] = torch.zeros(S, c.n_kv_heads, 8, dtype=torch.int32, device=DEV)
    b["counts"] = torch.zeros(S, dtype=torch.int32, device=DEV)
    return b


def _step(layer, b):
    m = layer.extend_sequences(b["map"], b["lens"], b["new"], b["table"], b["free"], b["used"], streams=b["act"])
    layer.rope_append(b["qkv"], m.row_pos, m.row_slot, b["pool"], b["q"])
    layer.key_bounds(b["pool"], b["table"], b["lens"], m.kv_lens, b["codes"], b["scales"], max_new=1)
    layer.select_blocks(b["q"], b["codes"], b["scales"], b["table"], m.kv_lens, m.row_start, b["blocks"], b["counts"], seq_rows=5)
    layer.attn_blocks(b["q"], b["pool"], b["table"], m.kv_lens, m.row_start, b["blocks"], b["counts"], b["out"], seq_rows=5)
    b["lens"].copy_(m.kv_lens)
    b["used"].copy_(m.counts[:1])


def _state(b):
    return [b[k].clone() for k in ("lens", "used", "table", "pool", "codes", "scales", "q", "out", "blocks", "counts")] + [b["map"].row_slot.clone(), b["map"].row_start.clone()]


@pytest.mark.parametrize("kw", [dict(Hq=8, Hkv=2), dict(Hq=8, Hkv=2, fp8=True, qk_norm=True), dict(Hq=4, Hkv=4, D=64, bf16=False)], ids=str)
def test_captured_step_replays_as_sequences_grow(kw):
    """Two loops, each captured once and replayed in turn with the program's own work between; every replay is the eager step, bit for bit."""
    layer = make(num_blocks=400, **kw)
    eager, captured, graphs = [], [], []
    for seed in (1, 2):
        _step(layer, _loop(layer, seed))  # warm
        b = _loop(layer, seed)
        want = []
        for _ in range(18):               # more than a block of tokens
            b["qkv"].mul_(-1)
            _step(layer, b)
            want.append(_state(b))
        eager.append(want)
        captured.append(_loop(layer, seed))
    torch.cuda.synchronize()
    for b in captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _step(layer, b)
        graphs.append(g)
    for i in range(18):
        for want, b, g in zip(eager, captured, graphs):
            b["qkv"].mul_(-1)
            g.replay()
            if i % 3 == 0:
                torch.cuda.synchronize()
            got = _state(b)
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, want[i])), i
            (b["out"].float() * 2).sum().item()
    layer.close()


def test_two_streams_at_once():
    """Two loops of one layer on two streams, launched in turn without waiting."""
    layer = make(num_blocks=400)
    want, loops = [], []
    for seed in (3, 4):
        b = _loop(layer, seed)
        for _ in range(6):
            _step(layer, b)
        want.append(_state(b))
        loops.append(_loop(layer, seed))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in loops]
    for _ in range(6):
        for b, st in zip(loops, streams):
            with torch.cuda.stream(st):
                _step(layer, b)
    torch.cuda.synchronize()
    for b, w in zip(loops, want):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(_state(b), w))
    layer.close()


def test_bounds_after_the_layers_own_prefill_and_decode():
    """Blocks that icarus_prefill_kv and icarus_decode_step wrote, bounded and attended to: their cache is the same cache."""
    from gpu_util import dev, make_layer
    from paper_2603_13281_amd import synth
    sh = synth.LLAMA_SMALL
    batch = synth.make_batch(sh, [70, 33], [2, 1], seed=1)
    layer = make_layer(sh, synth.make_base(sh, seed=1), synth.make_lora(sh, seed=1), batch.num_blocks)
    pool = torch.zeros(layer.cfg.pool_shape(), dtype=torch.bfloat16, device=DEV)
    table = torch.from_numpy(batch.block_tables).to(DEV)
    layer.prefill_kv(pool, table, [0, 0], [70, 33], dev(synth.make_hidden(sh, 103, seed=1, tag=1), True), want_out=False)
    layer.decode_step(pool, table, batch.ctx_lens, batch.row_seq, batch.row_model, dev(synth.make_hidden(sh, batch.R, seed=1), True))
    torch.cuda.synchronize()
    run_bounds(layer, pool, batch.block_tables, [0, 0], [71, 34], 71)
    rng = np.random.default_rng(0)
    q = torch.tensor(rng.standard_normal((batch.R, sh.n_q_heads, sh.head_dim)), dtype=torch.float32).to(torch.bfloat16).to(DEV)
    blocks = np.tile(np.arange(5), (2, sh.n_kv_heads, 1))
    run_attend(layer, q, pool, batch.block_tables[:, :5], [71, 34], np.array([0, 3, 5]), blocks, [5, 3])
    layer.close()
