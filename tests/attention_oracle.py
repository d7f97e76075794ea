"""Plain float64 forms of the attention calls (numpy, one row at a time), written from
the definitions in include/spconv_attention.h, with the bounds that the GPU tests
hold the kernels to. Test infrastructure."""
import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half a step, relative
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}  # half a step of the smallest, and less
U32 = 2.0 ** -24


def rope(x, positions, freq, interleaved=False, inverse=False, amplitude=1.0):
    """x [T, H, D] float64."""
    rot = 2 * len(freq)
    angle = positions.astype(np.float64)[:, None] * freq[None, :] * (-1.0 if inverse else 1.0)
    c, s = np.cos(angle)[:, None, :] * amplitude, np.sin(angle)[:, None, :] * amplitude
    y = x.copy()
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def rope_bound(x, freq, interleaved, amplitude, dtype, y):
    """The fp32 angle is within pi * 2^-25 of exact (a rounded fraction of a turn) and sine and cosine
    within two steps of that, so each is within 2^-21 of exact with the products' own roundings; then one rounding to the type."""
    rot = 2 * len(freq)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    size = np.zeros_like(x)
    size[..., i] = size[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return size * abs(amplitude) * 2.0 ** -21 + HALF[dtype] * np.abs(y) * (1 + 2.0 ** -8) + TINY[dtype]


class Rows:
    """Rows and sequences of a batch, from the header's rules: each row's sequence, tokens and positions."""

    def __init__(self, q_start, kv_len, tokens, q_block):
        B = len(kv_len)
        self.tokens = tokens
        if q_start is None:
            q_start = np.arange(B + 1)
        self.rows = tokens if q_block == 1 else tokens // q_block + B
        self.of = {}
        self.seq = {}
        for b in range(B):
            n = int(q_start[b + 1] - q_start[b])
            for i0 in range(0, n, q_block):
                r = int(q_start[b]) + i0 if q_block == 1 else int(q_start[b]) // q_block + b + i0 // q_block
                t = [int(q_start[b]) + i for i in range(i0, min(i0 + q_block, n))]
                assert r not in self.of and r < self.rows
                self.of[r] = (b, t, [int(kv_len[b]) - n + i for i in range(i0, i0 + len(t))])


def scores(rows, q, sums, table, kv_len, block, heads):
    """(scores, bounds) [R, heads, blocks]."""
    nb, G = table.shape[1], q.shape[1] // heads
    D = q.shape[2]
    out = np.full((rows.rows, heads, nb), -np.inf)
    bound = np.zeros_like(out)
    for r, (b, toks, pos) in rows.of.items():
        for j in range(nb):
            page = table[b, j]
            if not 0 <= page < sums.shape[0] or pos[-1] < j * block:
                continue
            n = min(block, int(kv_len[b]) - j * block)
            see = [t for t, p in zip(toks, pos) if p >= j * block]
            for h in range(heads):
                x = q[see, h * G:(h + 1) * G].reshape(-1, D)
                with np.errstate(invalid="ignore"):
                    d = x @ sums[page, h] / n
                    a = np.abs(x) @ np.abs(sums[page, h]) / n
                d = np.where(np.isnan(d), -np.inf, d)
                out[r, h, j] = d.max()
                # A maximum is off by no more than the products it is taken over; infinite ones are exact.
                bound[r, h, j] = np.max(a[np.isfinite(d)], initial=0.0) * (D + 8) * U32
    return out, bound


def select(rows, scores, block, keep, sink, local):
    R, H, nb = scores.shape
    blocks, counts = np.full((R, H, keep), -1, np.int32), np.zeros((R, H), np.int32)
    for r, (b, toks, pos) in rows.of.items():
        if pos[-1] < 0:
            continue
        n = min(pos[-1] // block + 1, nb)
        for h in range(H):
            if n <= keep:
                chosen = list(range(n))
            else:
                low = max(pos[0], 0) // block - local + 1 if local else n
                always = [j for j in range(n) if j < sink or j >= low]
                value = [-np.inf if np.isnan(v) else float(v) for v in scores[r, h, :n]]
                rest = sorted((j for j in range(n) if j not in set(always)), key=lambda j: (-value[j], j))
                chosen = sorted(always + rest[:keep - len(always)])
            blocks[r, h, :len(chosen)] = chosen
            counts[r, h] = len(chosen)
    return blocks, counts


def attention(rows, q, k_cache, v_cache, table, block, scale, blocks=None, counts=None, dtype=torch.float32):
    """(out, lse, bound of out, bound of lse): out [T, HQ, D]; tokens of no sequence are NaN."""
    T, HQ, D = q.shape
    pages, H = k_cache.shape[:2]
    G, nb = HQ // H, table.shape[1]
    out, lse = np.full((T, HQ, D), np.nan), np.full((T, HQ), np.nan)
    bo, bl = np.zeros_like(out), np.zeros_like(lse)
    half = HALF[dtype]
    for r, (b, toks, pos) in rows.of.items():
        for h in range(H):
            if blocks is None:
                names = range(nb)
            else:
                names = blocks[r, h, :blocks.shape[2] if counts is None else min(max(int(counts[r, h]), 0), blocks.shape[2])]
            names = [int(j) for j in names if 0 <= j < nb and 0 <= table[b, j] < pages and j * block <= pos[-1]]
            if names:
                K = np.concatenate([k_cache[table[b, j], h] for j in names])
                V = np.concatenate([v_cache[table[b, j], h] for j in names])
                at = np.concatenate([np.arange(j * block, (j + 1) * block) for j in names])
            for t, p in zip(toks, pos):
                see = at <= p if names else np.zeros(0, bool)
                for g in range(h * G, (h + 1) * G):
                    if not see.any():
                        out[t, g], lse[t, g] = 0.0, -np.inf
                        continue
                    with np.errstate(all="ignore"):
                        x = K[see] @ q[t, g] * scale
                        top = x.max()
                        if top == -np.inf:
                            out[t, g], lse[t, g] = 0.0, -np.inf
                            continue
                        w = np.exp(x - top)
                        total = w.sum()
                        out[t, g] = (w @ V[see]) / total
                        lse[t, g] = top + np.log(total)
                        # An fp32 product of D terms, its scaling and the difference to the maximum: x is off by dx.
                        dx = (np.abs(K[see]) @ np.abs(q[t, g])).max() * abs(scale) * (D + 16) * U32
                        size = (w @ np.abs(V[see])) / total
                        # Each weight is off by dx (as is the sum), by its exponential, by its rounding to the type, and
                        # the sums run over all keys; then the output's own rounding.
                        weight = 2 * dx + (half if dtype is not torch.float32 else U32) + (see.sum() + 32) * U32
                        bo[t, g] = size * weight * 1.05 + half * np.abs(out[t, g]) * 1.01 + TINY[dtype]
                        bl[t, g] = dx + (see.sum() + 32) * U32 + np.abs(lse[t, g]) * 4 * U32 + 4 * U32
    return out, lse, bo, bl
