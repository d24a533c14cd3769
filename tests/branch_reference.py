"""The operators of include/icarus_branches.h in plain float64 numpy and whole numbers, written from their definitions: one loop
after the other, no library code.  Pools are float arrays in the library's layout [blocks, Hkv, 2, Bk * D]."""
import math

import numpy as np

from block_reference import blocks_of

MOST = float(np.finfo(np.float32).max)


def beam_row(row_start, s, R):
    r = s if row_start is None else int(row_start[s + 1]) - 1 if row_start[s + 1] > row_start[s] else -1
    return r if 0 <= r < R else -1


def choose(logits, row_start, scores, done, eos, groups, width):
    """parents, tokens, scores (float64), done; and the gaps between neighbouring scores of one group's order (a choice with a gap near 0 hangs on rounding)."""
    n = groups * width
    parents, tokens, best, ended, gaps = np.full(n, -1), np.full(n, -1), np.full(n, -math.inf), np.zeros(n, dtype=int), []
    for g in range(groups):
        cand = []
        for b in range(width):
            s = g * width + b
            r = beam_row(row_start, s, len(logits))
            if r < 0 or not math.isfinite(scores[s]):
                continue
            if done is not None and done[s]:
                cand.append((-float(scores[s]), b, 0.0, eos, 1))
                continue
            x = np.asarray(logits[r], dtype=np.float64)
            x = np.where(np.isnan(x), -math.inf, np.minimum(x, MOST))
            top = x.max()
            if top == -math.inf:
                continue
            norm = math.log(math.fsum(np.exp(x - top)))
            order = np.lexsort((np.arange(len(x)), -x))[:width]
            cand += [(-(float(scores[s]) + ((float(x[t]) - top) - norm)), b, -float(x[t]), int(t), int(t) == eos) for t in order if x[t] > -math.inf]
        cand.sort()
        for i, (v, b, x, t, e) in enumerate(cand[:width]):
            parents[g * width + i], tokens[g * width + i], best[g * width + i], ended[g * width + i] = b, t, -v, e
            if i + 1 < len(cand) and (cand[i + 1][1] != b):
                gaps.append(cand[i + 1][0] - v)
    return parents, tokens, best, ended, gaps


def fork(parents, kv_lens, table, shared, free, used, bk, num_blocks, width, new_table):
    S, max_blocks = table.shape
    free, new_table = np.array(free).copy(), new_table.copy()
    head = min(max(int(used), 0), len(free))
    length = [min(max(int(n), 0), max_blocks * bk) for n in kv_lens]
    new_lens, src, dst = np.zeros(S, dtype=int), np.full(S, -1), np.full(S, -1)
    up = [int(p) if 0 <= p < width else -1 for p in parents]
    freed = []
    for g in range(S // width):
        lo = 0 if shared is None else max(0, int(shared[g]))
        kept = {g * width + up[s] for s in range(g * width, (g + 1) * width) if up[s] >= 0}
        for c in range(lo, max_blocks):
            held = {int(table[s, c]) for s in kept if c < blocks_of(length[s], bk)}
            for s in range(g * width, (g + 1) * width):
                if c < blocks_of(length[s], bk) and 0 <= table[s, c] < num_blocks and int(table[s, c]) not in held:
                    freed.append(int(table[s, c]))
                    held.add(int(table[s, c]))
    low = head - len(freed)
    for j, b in enumerate(freed):
        if low + j >= 0:
            free[low + j] = b
    at, refused = max(low, 0), 0
    for g in range(S // width):
        lo, first = 0 if shared is None else max(0, int(shared[g])), set()
        for s in range(g * width, (g + 1) * width):
            p = up[s]
            if p < 0:
                continue
            P = g * width + p
            n = length[P]
            nb = blocks_of(n, bk)
            row = table[P, :nb].copy()
            if n % bk and (p in first or n // bk < lo):
                if at >= len(free):
                    refused += 1
                    continue
                b = int(free[at])
                at += 1
                b = b if 0 <= b < num_blocks else -1
                if b >= 0 and 0 <= row[-1] < num_blocks:
                    src[s], dst[s] = row[-1], b
                row[-1] = b
            first.add(p)
            new_lens[s] = n
            new_table[s, :nb] = row
    return dict(kv_lens=new_lens, block_tables=new_table, copy_src=src, copy_dst=dst, counts=np.array([at, refused, len(freed)]), free=free)


def attend(q, pool, table, kv_lens, row_start, group_start, bk, out):
    """out (a copy, rows of no sequence or group as they are), and for a tolerance the softmax-weighted |v|, the largest sum |q||k| / sqrt(D) and the positions."""
    out = out.astype(np.float64).copy()
    weight, size, count = np.zeros_like(out), np.zeros(out.shape[:2] + (1,)), np.zeros(out.shape[:2] + (1,))
    nb, hkv = pool.shape[:2]
    D = q.shape[2]
    g = q.shape[1] // hkv
    for s in range(table.shape[0]):
        if not any(group_start[i] <= s < group_start[i + 1] for i in range(len(group_start) - 1)):
            continue
        r0, r1 = int(row_start[s]), int(row_start[s + 1])
        n = min(max(int(kv_lens[s]), 0), table.shape[1] * bk)
        ids = [(int(b), min(bk, n - i * bk)) for i, b in enumerate(table[s, :blocks_of(n, bk)]) if 0 <= b < nb]
        for c in range(hkv):
            if r0 == r1:
                continue
            if not ids:
                out[r0:r1, c * g:(c + 1) * g] = 0.0
                continue
            blk = [pool[b, c].astype(np.float64) for b, _ in ids]
            k = np.concatenate([x[0].reshape(bk, D)[:m] for x, (_, m) in zip(blk, ids)])
            v = np.concatenate([x[1].reshape(D, bk).T[:m] for x, (_, m) in zip(blk, ids)])
            qq = q[r0:r1, c * g:(c + 1) * g].astype(np.float64)
            sc = qq @ k.T / math.sqrt(D)
            with np.errstate(invalid="ignore"):
                p = np.exp(sc - sc.max(-1, keepdims=True))
            p = np.where((sc == -math.inf).all(-1, keepdims=True), 0.0, p)
            total = p.sum(-1, keepdims=True)
            p = np.where(total == 0.0, 0.0, p / np.where(total == 0.0, 1.0, total))
            out[r0:r1, c * g:(c + 1) * g], weight[r0:r1, c * g:(c + 1) * g] = p @ v, p @ np.abs(v)
            big = np.abs(qq) @ np.abs(k).T                  # a score of minus infinity weighs 0 and has no error
            size[r0:r1, c * g:(c + 1) * g] = np.where(np.isfinite(big), big, 0.0).max(-1, keepdims=True) / math.sqrt(D)
            count[r0:r1, c * g:(c + 1) * g] = len(k)
    return out, weight, size, count
