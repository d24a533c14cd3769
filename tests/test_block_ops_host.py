"""icarus_blocks.h without a GPU: the plain references against brute force, and every refusal that the host makes."""
import numpy as np
import pytest

import block_reference as ref
from paper_2603_13281_amd import binding
from paper_2603_13281_amd.binding import IcarusError, IcarusLayer, LayerConfig

A = 0x10000  # 16-byte aligned, never read


def _layer(**kw):
    cfg = dict(d_model=256, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ffn=256, block_size=16, num_blocks=64, max_position=4096)
    cfg.update(kw)
    return IcarusLayer(LayerConfig(**cfg), {p: A for p in binding.PROJ + ("norm_attn", "norm_ffn")})


def _refused(layer, rc, status):
    assert binding.STATUS[rc] == status, (binding.STATUS[rc], binding._lib.icarus_last_error(layer._h))


def test_extend_refusals():
    layer, call = _layer(), binding._lib.icarus_extend_sequences
    good = dict(S=4, ctx=A, new=A + 64, streams=None, bt=A + 256, mb=8, free=A + 512, nf=10, used=A + 1024, rows=16, kv=A + 2048, start=A + 3136,
                seq=A + 4096, pos=A + 5120, slot=A + 6144, counts=A + 7168)

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, call(layer._h, a["S"], a["ctx"], a["new"], a["streams"], a["bt"], a["mb"], a["free"], a["nf"], a["used"], a["rows"], a["kv"], a["start"],
                             a["seq"], a["pos"], a["slot"], a["counts"], None), status)
    for name in ("S", "mb", "nf", "rows"):
        run("INVALID_ARG", **{name: -1})
    for name in ("ctx", "new", "bt", "free", "used", "kv", "start", "seq", "pos", "slot", "counts"):
        run("INVALID_ARG", **{name: None})
        run("ALIGNMENT", **{name: good[name] + 2})
    run("ALIGNMENT", slot=A + 6148)
    run("UNSUPPORTED", rows=(1 << 30) + 1)
    run("INVALID_ARG", kv=good["ctx"])            # the lengths are read while kv_lens is written
    run("INVALID_ARG", kv=good["new"] + 12)
    run("INVALID_ARG", streams=good["kv"])
    run("INVALID_ARG", used=good["counts"] + 4)
    layer.close()


def test_append_refusals():
    layer, call = _layer(), binding._lib.icarus_rope_append
    good = dict(qkv=A, ld=768, R=4, pos=A + (1 << 20), slot=A + (2 << 20), q=A + (3 << 20), pool=A + (4 << 20))

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, call(layer._h, a["qkv"], a["ld"], a["R"], a["pos"], a["slot"], a["q"], a["pool"], None), status)
    run("OK", R=0)
    run("INVALID_ARG", R=-1)
    run("SHAPE", ld=767)
    for name in ("qkv", "pos", "slot", "q", "pool"):
        run("INVALID_ARG", **{name: None})
    for name in ("qkv", "q", "pool"):
        run("ALIGNMENT", **{name: good[name] + 8})
    run("ALIGNMENT", pos=good["pos"] + 2)
    run("ALIGNMENT", slot=good["slot"] + 4)
    run("INVALID_ARG", q=good["qkv"])             # in place: rows are read while others are written
    run("INVALID_ARG", q=good["qkv"] + 2 * (3 * 768 + 752))
    layer.close()


def test_bounds_refusals():
    layer, call = _layer(), binding._lib.icarus_key_bounds
    good = dict(pool=A, bt=A, mb=8, S=2, a=A, b=A, new=16, codes=A, scales=A)

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, call(layer._h, a["pool"], a["bt"], a["mb"], a["S"], a["a"], a["b"], a["new"], a["codes"], a["scales"], None), status)
    run("OK", S=0)
    run("OK", mb=0)
    for name in ("S", "mb", "new"):
        run("INVALID_ARG", **{name: -1})
    run("UNSUPPORTED", S=65536)
    for name in ("pool", "bt", "a", "b", "codes", "scales"):
        run("INVALID_ARG", **{name: None})
        run("ALIGNMENT", **{name: A + 2})
    layer.close()


def test_select_and_attend_refusals():
    layer, lib = _layer(), binding._lib
    assert lib.icarus_select_workspace_bytes(layer._h, -1, 4) == 0 and lib.icarus_attn_blocks_workspace_bytes(layer._h, 1, -1, 4) == 0
    good = dict(q=A, codes=A, scales=A, bt=A, mb=8, S=2, kv=A, R=3, start=A, hint=0, k=4, first=1, last=2, blocks=A, counts=A, ws=A, wsb=1 << 30)

    def run(status, **kw):
        a = {**good, **kw}
        _refused(layer, lib.icarus_select_blocks(layer._h, a["q"], a["codes"], a["scales"], a["bt"], a["mb"], a["S"], a["kv"], a["R"], a["start"], a["hint"], a["k"],
                                                 a["first"], a["last"], a["blocks"], a["counts"], a["ws"], a["wsb"], None), status)
    run("OK", S=0)
    for name in ("S", "mb", "R", "hint", "first", "last"):
        run("INVALID_ARG", **{name: -1})
    run("INVALID_ARG", k=0, first=0, last=0)
    run("INVALID_ARG", k=2)
    run("INVALID_ARG", first=2 ** 31 - 1, last=2 ** 31 - 1)
    run("UNSUPPORTED", S=65536)
    for name in ("q", "codes", "scales", "bt", "kv", "start", "blocks", "counts", "ws"):
        run("INVALID_ARG", **{name: None})
        run("ALIGNMENT", **{name: A + 2})
    run("CAPACITY", wsb=lib.icarus_select_workspace_bytes(layer._h, 2, 8) - 1)
    run("UNSUPPORTED", mb=(1 << 22) + 1)
    run("UNSUPPORTED", R=1 << 29)                 # rows x heads of a kv-head beyond 2^30
    good = dict(q=A, pool=A, bt=A, mb=8, S=2, kv=A, R=3, start=A, hint=0, blocks=A, counts=A, k=4, out=A + (1 << 20), ws=A, wsb=1 << 30)

    def run(status, **kw):  # noqa: F811
        a = {**good, **kw}
        _refused(layer, lib.icarus_attn_blocks(layer._h, a["q"], a["pool"], a["bt"], a["mb"], a["S"], a["kv"], a["R"], a["start"], a["hint"], a["blocks"], a["counts"],
                                               a["k"], a["out"], a["ws"], a["wsb"], None), status)
    run("OK", S=0)
    run("OK", R=0)
    for name in ("S", "mb", "R", "hint", "k"):
        run("INVALID_ARG", **{name: -1})
    run("UNSUPPORTED", S=65536)
    for name in ("q", "pool", "bt", "kv", "start", "blocks", "counts", "out", "ws"):
        run("INVALID_ARG", **{name: None})
        run("ALIGNMENT", **{name: good[name] + 2})
    run("CAPACITY", wsb=lib.icarus_attn_blocks_workspace_bytes(layer._h, 2, 3, 4) - 1)
    run("INVALID_ARG", out=good["q"] + 2 * 3 * 8 * 64 - 16)
    run("UNSUPPORTED", S=60000, k=100000)
    run("UNSUPPORTED", R=1 << 29)
    layer.close()


def test_null_context_is_refused():
    lib = binding._lib
    assert lib.icarus_extend_sequences(None, *[0, None, None, None, None, 0, None, 0, None, 0], *[None] * 7) == 1
    assert lib.icarus_rope_append(None, None, 0, 0, None, None, None, None, None) == 1
    assert lib.icarus_key_bounds(None, None, None, 0, 0, None, None, 0, None, None, None) == 1
    assert lib.icarus_select_blocks(None, None, None, None, None, 0, 0, None, 0, None, 0, 1, 0, 0, None, None, None, 0, None) == 1
    assert lib.icarus_attn_blocks(None, None, None, None, 0, 0, None, 0, None, 0, None, None, 0, None, None, 0, None) == 1


def test_binding_refuses_tensors_the_c_signature_would_misread():
    import torch
    layer = _layer()
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):      # host tensors
        layer.key_bounds(torch.zeros(layer.cfg.pool_shape(), dtype=torch.bfloat16), table, lens, lens, None, None)
    with pytest.raises(TypeError):
        layer.attn_blocks(None, None, table.long(), lens, lens, lens, lens)
    with pytest.raises(TypeError):
        layer.rope_append(torch.zeros(2, 768), lens, lens, None)
    with pytest.raises(ValueError):      # host tensors again
        layer.rope_append(torch.zeros(2, 768, dtype=torch.bfloat16), lens, lens, None)
    layer.close()


# ---- the references ---------------------------------------------------------------------------------------------------

def test_reference_extend_by_hand():
    t = np.full((3, 4), -1)
    t[0, :2] = [7, 3]
    t[2, 0] = 5
    got = ref.extend([5, 0, 4], [2, 1, 1], [1, 0, 2], t, [8, 9, 1], 1, 9, 4, 10, 100)
    # sequence 0 fills places 5, 6 of its blocks; 1 takes block 9; 2 takes block 1
    assert got["kv_lens"].tolist() == [7, 1, 5] and got["row_start"].tolist() == [0, 3, 4, 7] and got["counts"].tolist() == [3, 0]
    assert got["row_seq"].tolist() == [0, 0, 0, 1, 2, 2, 2, -1, -1] and got["row_pos"].tolist() == [5, 6, 6, 0, 4, 4, 4, -1, -1]
    assert got["row_slot"].tolist() == [13, 14, -1, 36, 4, -1, -1, -1, -1]
    assert got["block_tables"].tolist() == [[7, 3, -1, -1], [9, -1, -1, -1], [5, 1, -1, -1]]
    short = ref.extend([5, 0, 4], [2, 1, 1], None, t, [8, 9], 2, 9, 4, 10, 100)  # the list is empty: only sequence 0 goes on
    assert short["kv_lens"].tolist() == [7, 0, 4] and short["counts"].tolist() == [2, 2] and short["row_seq"].tolist()[:4] == [0, 0, -1, -1]


def test_reference_bounds_hold_the_scores():
    """The codes bound the keys, so with the exact query instead of its code the sum bounds every q . k of the block."""
    rng = np.random.default_rng(0)
    D, bk = 10, 5
    pool = rng.standard_normal((3, 2, 2, bk * D)) * 10.0 ** rng.integers(-3, 4, (3, 2, 1, 1))
    codes, scales = ref.bounds(pool, np.array([[2, 0]]), [0], [8], bk, D, np.zeros((3, 2, 2, D)), np.ones((3, 2)))
    for i, n in ((2, 5), (0, 3)):
        k = pool[i, :, 0].reshape(2, bk, D)[:, :n]
        assert (codes[i, :, 0] * scales[i][:, None] >= k.max(1)).all() and (codes[i, :, 1] * scales[i][:, None] <= k.min(1)).all()
        assert (np.abs(codes[i]).max((1, 2)) > 63).all()  # no step is larger than it has to be
        q = rng.standard_normal(D)
        bound = (np.maximum(q, 0) * codes[i, :, 0] + np.minimum(q, 0) * codes[i, :, 1]).sum(-1) * scales[i]
        assert (bound[:, None] >= k @ q).all()
    assert (codes[1] == 0).all() and (scales[1] == 1).all()


def test_reference_attend_is_softmax():
    rng = np.random.default_rng(1)
    D, bk = 6, 4
    pool, q = rng.standard_normal((4, 1, 2, bk * D)), rng.standard_normal((1, 2, D))
    out, _, _ = ref.attend(q, pool, np.array([[3, 1]]), [6], [0, 1], np.array([[[1, 0, -1]]]), [3], bk, np.zeros((1, 2, D)))
    k = np.concatenate([pool[3, 0, 0].reshape(bk, D), pool[1, 0, 0].reshape(bk, D)[:2]])
    v = np.concatenate([pool[3, 0, 1].reshape(D, bk).T, pool[1, 0, 1].reshape(D, bk).T[:2]])
    w = np.exp(q[0] @ k.T / np.sqrt(D))
    assert np.allclose(out[0], w @ v / w.sum(-1, keepdims=True), atol=1e-14)


# ---- limits -----------------------------------------------------------------------------------------------------------

def test_limits_are_the_stated_ones():
    """Each limit of the header: one more is refused as unsupported, and at the limit the call goes on to look at its arrays (null here)."""
    lib, big = binding._lib, 1 << 29
    layer = _layer()

    def extend(S=1, free=1, rows=1):
        return lib.icarus_extend_sequences(layer._h, S, None, None, None, None, 1, None, free, None, rows, *[None] * 7)

    def append(R):
        return lib.icarus_rope_append(layer._h, None, 768, R, None, None, None, None, None)

    def bounds(S):
        return lib.icarus_key_bounds(layer._h, None, None, 1 << 30, S, None, None, 0, None, None, None)

    def select(S=1, mb=1, R=1, k=1):
        return lib.icarus_select_blocks(layer._h, None, None, None, None, mb, S, None, R, None, 0, k, 0, 0, None, None, None, 0, None)

    def attend(S=1, R=1, k=1, mb=1 << 30):
        return lib.icarus_attn_blocks(layer._h, None, None, None, mb, S, None, R, None, 0, None, None, k, None, None, 0, None)

    cases = [(extend, "S", big), (extend, "free", big), (extend, "rows", big), (append, "R", big), (bounds, "S", 65535), (select, "S", 65535), (select, "mb", 1 << 22),
             (select, "k", 1 << 22), (select, "R", 1 << 28), (attend, "S", 65535), (attend, "R", 1 << 28), (attend, "k", 1 << 22)]   # 4 heads share a kv-head: 2^30 queries
    for call, name, most in cases:
        _refused(layer, call(**{name: most}), "INVALID_ARG")
        _refused(layer, call(**{name: most + 1}), "UNSUPPORTED")
    layer.close()
    layer = _layer(n_q_heads=32, n_kv_heads=32, head_dim=2)
    for S, k in ((1 << 15, 0), (1 << 15, 256), (1 << 14, 257), (1 << 14, 512), (1, 1 << 22)):
        _refused(layer, attend(S=S, k=k), "INVALID_ARG")
        assert lib.icarus_attn_blocks_workspace_bytes(layer._h, S, 1, k) > 0
    for S, k in (((1 << 15) + 1, 0), ((1 << 15) + 1, 256), (1 << 15, 257), ((1 << 14) + 1, 512), (3, 1 << 22)):
        _refused(layer, attend(S=S, k=k), "UNSUPPORTED")
        assert lib.icarus_attn_blocks_workspace_bytes(layer._h, S, 1, k) == 0
    layer.close()
    layer = _layer(n_q_heads=65, n_kv_heads=65, head_dim=2)
    _refused(layer, select(S=((1 << 22) - 1) // 65), "INVALID_ARG")
    _refused(layer, select(S=((1 << 22) - 1) // 65 + 1), "UNSUPPORTED")
    assert lib.icarus_select_workspace_bytes(layer._h, 1, 1 << 22) > 0
    for S, mb in ((1, (1 << 22) + 1), (1, 2 ** 31 - 1), (65536, 1)):
        assert lib.icarus_select_workspace_bytes(layer._h, S, mb) == 0
    layer.close()
