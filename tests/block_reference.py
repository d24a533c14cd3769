"""The operators of include/icarus_blocks.h in plain float64 numpy and whole numbers, written from their definitions: one loop
after the other, no library code.  Pools are float arrays in the library's layout [blocks, Hkv, 2, Bk * D]."""
import math

import numpy as np


def blocks_of(n, bk):
    return -(-int(n) // bk)


def extend(ctx, new, streams, table, free, used, max_rows, bk, num_blocks, max_position):
    S, max_blocks = table.shape
    table = table.copy()
    kv, start, rows = [], [], []
    head, stuck, refused, n_rows = min(max(int(used), 0), len(free)), False, 0, 0
    for s in range(S):
        c, n, m = int(ctx[s]), int(new[s]), int(streams[s]) if streams is not None else 0
        start.append(min(n_rows, max_rows))
        mine = n + max(m, 0) if n > 0 else 0
        end = c + n
        ok = c >= 0 and n >= 0 and m >= 0 and end <= max_position and blocks_of(end, bk) <= max_blocks and (mine == 0 or n_rows + mine <= max_rows)
        need = blocks_of(end, bk) - blocks_of(c, bk) if ok else 0
        if ok and need:
            stuck = stuck or head + need > len(free)
            ok = not stuck
        if ok:
            for j in range(need):
                b = int(free[head + j])
                table[s, blocks_of(c, bk) + j] = b if 0 <= b < num_blocks else -1
            head += need
            for i in range(mine):
                p = c + min(i, n - 1)
                b = int(table[s, p // bk])
                rows.append((s, p, b * bk + p % bk if i < n and 0 <= b < num_blocks else -1))
        else:
            refused += 1
            rows += [(-1, -1, -1)] * max(0, min(mine, max_rows - n_rows))
        kv.append(end if ok else c)
        n_rows += mine
    start.append(min(n_rows, max_rows))
    rows = (rows + [(-1, -1, -1)] * max_rows)[:max_rows]
    seq, pos, slot = (np.array([r[i] for r in rows], dtype=np.int64) for i in range(3))
    return dict(kv_lens=np.array(kv, dtype=np.int64), row_start=np.array(start), row_seq=seq, row_pos=pos, row_slot=slot, counts=np.array([head, refused]),
                block_tables=table)


def rotated(x, pos, theta, norm_w=None, eps=0.0):
    """x [R, heads, D] -> the same normed and rotated, and the size |a| + |b| of each pair (for a tolerance)."""
    D = x.shape[-1]
    if norm_w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * norm_w
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * theta ** (-2.0 * np.arange(D // 2) / D)
    a, b = x[..., : D // 2], x[..., D // 2:]
    size = np.abs(a) + np.abs(b)
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), a * np.sin(ang) + b * np.cos(ang)], -1), np.concatenate([size, size], -1)


def step_of(x):
    """2^e, the smallest with 127 * 2^e >= x, -40 <= e <= 40."""
    e = -40
    while e < 40 and 127.0 * 2.0 ** e < x:
        e += 1
    return 2.0 ** e


def _key(x):
    big = float(np.finfo(np.float32).max)
    return np.clip(np.nan_to_num(x, nan=0.0, posinf=big, neginf=-big), -big, big)


def bounds(pool, table, lo_lens, hi_lens, bk, D, codes, scales):
    """codes [blocks, Hkv, 2, D] and scales [blocks, Hkv], updated copies."""
    codes, scales = codes.copy(), scales.copy()
    nb, hkv = pool.shape[:2]
    for s in range(table.shape[0]):
        a, z = max(0, int(lo_lens[s])), min(max(0, int(hi_lens[s])), table.shape[1] * bk)
        for b in range(a // bk, blocks_of(z, bk) if a < z else 0):
            i = int(table[s, b])
            if not 0 <= i < nb:
                continue
            k = _key(pool[i, :, 0].reshape(hkv, bk, D)[:, : min(bk, z - b * bk)].astype(np.float64))
            hi, lo = k.max(1), k.min(1)
            for c in range(hkv):
                st = step_of(max(np.abs(hi[c]).max(), np.abs(lo[c]).max()))
                codes[i, c, 0] = np.clip(np.ceil(hi[c] / st), -127, 127)
                codes[i, c, 1] = np.clip(np.floor(lo[c] / st), -127, 127)
                scales[i, c] = st
    return codes, scales


def scores(q, codes, scales, ids):
    """q [queries, D]: the score of each block in ids, as python floats (exact)."""
    out = []
    qq = []
    for v in q:
        v = _key(v.astype(np.float64))
        st = step_of(np.abs(v).max())
        qq.append((np.clip(np.rint(v / st), -127, 127).astype(np.int64), st))
    for i in ids:
        best = 0.0 if not qq else -math.inf
        for v, st in qq:
            dot = int((np.maximum(v, 0) * codes[i][0].astype(np.int64)).sum() + (np.minimum(v, 0) * codes[i][1].astype(np.int64)).sum())
            best = max(best, dot * st * float(scales[i]))
        out.append(best)
    return out


def select(q, codes, scales, table, kv_lens, row_start, top_k, first, last, bk):
    """q [R, Hq, D] -> blocks [S, Hkv, top_k], counts [S]."""
    S, max_blocks = table.shape
    n_pool, hkv = scales.shape
    g = q.shape[1] // hkv
    out, counts = np.full((S, hkv, top_k), -1, dtype=np.int64), np.zeros(S, dtype=np.int64)
    for s in range(S):
        nb = min(blocks_of(max(0, int(kv_lens[s])), bk), max_blocks)
        k = counts[s] = min(top_k, nb)
        for c in range(hkv):
            mine = q[int(row_start[s]):int(row_start[s + 1]), c * g:(c + 1) * g].reshape(-1, q.shape[2])
            ids = [int(b) for b in table[s, :nb]]
            good = [b for b in range(nb) if 0 <= ids[b] < n_pool]
            sc = [-math.inf] * nb
            for b, v in zip(good, scores(mine, codes[:, c], scales[:, c], [ids[b] for b in good])):
                sc[b] = v
            order = sorted(range(nb), key=lambda b: (not (b < first or b >= nb - last), -sc[b], b))
            out[s, c, :k] = sorted(order[:k])
    return out, counts


def attend(q, pool, table, kv_lens, row_start, blocks, counts, bk, out):
    """out (a copy, rows of no sequence as they are), and for a tolerance the softmax-weighted |v| and the largest sum |q||k| / sqrt(D)."""
    out = out.astype(np.float64).copy()
    weight, size = np.zeros_like(out), np.zeros(out.shape[:2] + (1,))
    nb, hkv = pool.shape[:2]
    D = q.shape[2]
    g = q.shape[1] // hkv
    for s in range(table.shape[0]):
        for c in range(hkv):
            ks, vs = [], []
            for b in blocks[s, c, : max(0, int(counts[s]))]:
                b = int(b)
                if not 0 <= b < table.shape[1] or not 0 <= int(table[s, b]) < nb:
                    continue
                n = max(0, min(bk, int(kv_lens[s]) - b * bk))
                blk = pool[int(table[s, b]), c].astype(np.float64)
                ks.append(blk[0].reshape(bk, D)[:n])
                vs.append(blk[1].reshape(D, bk).T[:n])
            k, v = (np.concatenate(x) if x else np.zeros((0, D)) for x in (ks, vs))
            for r in range(int(row_start[s]), int(row_start[s + 1])):
                for h in range(c * g, (c + 1) * g):
                    if not len(k):
                        out[r, h] = 0.0
                        continue
                    sc = k @ q[r, h].astype(np.float64) / math.sqrt(D)
                    p = np.exp(sc - sc.max())
                    p /= p.sum()
                    out[r, h], weight[r, h] = p @ v, p @ np.abs(v)
                    size[r, h] = (np.abs(k) @ np.abs(q[r, h].astype(np.float64))).max() / math.sqrt(D)
    return out, weight, size
