"""The paged 8-bit K/V cache in numpy, 64 bits, from the definitions: bookkeeping, quantization by blocks of 64 tokens,
attention of new tokens over a row's tokens.  Nothing is shared with the HIP path."""
import math

import numpy as np

PAGE = 64


class Book:
    """Block table, lengths and free stack of a cache."""

    def __init__(self, rows, n_pages, max_blocks, free=None):
        self.length = [0] * rows
        self.table = np.full((rows, max_blocks), -1, dtype=np.int32)
        self.free = list(range(n_pages - 1, -1, -1)) if free is None else [int(x) for x in free]
        self.n_pages, self.max_blocks = n_pages, max_blocks

    def plan(self, new, release, n_slots):
        """-> cu, slots, req, status; changes the book unless status[0]"""
        R = len(self.length)
        release = [0] * R if release is None else release
        held = [0 if x else n for n, x in zip(self.length, release)]
        blocks = lambda n: (n + PAGE - 1) // PAGE
        back = sum(blocks(n) for n, x in zip(self.length, release) if x)
        need = sum(blocks(h + n) - blocks(h) for h, n in zip(held, new) if n > 0)
        flags = 0
        if any(n < 0 for n in new):
            flags = 8
        else:
            flags |= 1 * (len(self.free) + back < need)
            flags |= 2 * any(h + n > self.max_blocks * PAGE for h, n in zip(held, new))
            flags |= 4 * (sum(new) > n_slots)
        slots, req = np.full(n_slots, -1, np.int32), np.full(n_slots, -1, np.int32)
        if flags:
            return np.zeros(R + 1, np.int32), slots, req, [flags, len(self.free)]
        for r in range(R):
            if release[r]:
                self.free += [int(p) for p in self.table[r, :blocks(self.length[r])]]
        cu, i = [0], 0
        for r in range(R):
            for b in range(blocks(held[r]), blocks(held[r] + new[r])):
                self.table[r, b] = self.free.pop()
            for t in range(held[r], held[r] + new[r]):
                slots[i], req[i] = PAGE * self.table[r, t // PAGE] + t % PAGE, r
                i += 1
            self.length[r] = held[r] + new[r]
            cu.append(i)
        return np.array(cu, np.int32), slots, req, [0, len(self.free)]


def quantize_tokens(x, shift=None):
    """x [n, H, d] of one row from its first token on (fp32 values) -> codes int64, amax fp32 [blocks, H]; codes of a block
    with a NaN or an infinity are 0."""
    y = x.astype(np.float32)
    if shift is not None:
        y = y - shift.astype(np.float32)
    n = y.shape[0]
    codes = np.zeros(y.shape, np.int64)
    amax = np.zeros(((n + PAGE - 1) // PAGE, y.shape[1]), np.float32)
    for b in range(amax.shape[0]):
        blk = y[b * PAGE:(b + 1) * PAGE]
        for h in range(y.shape[1]):
            a = np.abs(blk[:, h])
            top = np.float32(np.nan) if np.isnan(a).any() else a.max()
            amax[b, h] = top
            if np.isfinite(top) and top > 0:
                # 127 x has 31 bits and the quotient is at least 2^-32 from a half that it does not hit: one rounding to
                # 53 bits decides it
                codes[b * PAGE:(b + 1) * PAGE, h] = np.rint(127.0 * blk[:, h].astype(np.float64) / np.float64(top)).astype(np.int64)
    return codes, amax


def values(codes, amax, shift=None):
    """what the codes stand for, fp64 [n, H, d]"""
    step = np.repeat(amax.astype(np.float64) / 127.0, PAGE, axis=0)[:codes.shape[0]]
    with np.errstate(invalid="ignore"):
        v = codes * step[:, :, None]
    return v if shift is None else v + shift.astype(np.float64)


def attend(q, k, v, first, causal, mask=None, scale=None):
    """q [n, H, d] the new tokens, k, v [len, H_kv, d] all of the row's; token t sees keys up to first + t (causal) in the blocks
    that mask [H_kv, blocks] keeps.  -> O [n, H, d], sum p |v| / sum p, max over the seen keys of sum |q k| scale [n, H]."""
    n, H, d = q.shape
    L, Hkv = k.shape[:2]
    G = H // Hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    O, A, S = np.zeros((n, H, d)), np.zeros((n, H, d)), np.zeros((n, H))
    key = np.arange(L)
    for h in range(H):
        kv = h // G
        s = (q[:, h] @ k[:, kv].T) * scale
        see = key[None] <= first + np.arange(n)[:, None] if causal else np.ones((n, L), bool)
        if mask is not None:
            see = see & (mask[kv][key // PAGE] != 0)[None]
        big = (np.abs(q[:, h]) @ np.abs(k[:, kv]).T) * scale
        for t in range(n):
            j = np.nonzero(see[t])[0]
            if len(j) == 0:
                continue
            with np.errstate(invalid="ignore"):
                p = np.exp(s[t, j] - s[t, j].max())
                O[t, h] = p @ v[j, kv] / p.sum()
                A[t, h] = p @ np.abs(v[j, kv]) / p.sum()
            S[t, h] = big[t, j].max()
    return O, A, S
