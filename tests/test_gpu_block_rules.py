"""What include/icarus_blocks.h promises beyond each operator's values."""
import numpy as np
import pytest
import torch

from test_gpu_block_ops import DEV, i32, make, random_pool

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
