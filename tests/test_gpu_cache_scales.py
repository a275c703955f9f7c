"""Attention over the paged 8-bit cache where the size of V differs between a row's blocks and the largest are not the ones that count:
blocks of large V whose keys score far below the others, that only other queries of the same tile attend to, or that only later tokens
see.  What a result may be off by is taken from its own weights times its own values, never from the largest V of the row."""
import math

import numpy as np
import pytest

from cache_cases import Model, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2502_18137_amd as sp
    return sp


def contributions(q, k, v, amax, first, causal=True):
    """-> O, sum p |v|, max over the keys of p amax (amax of the key's block), max over the seen keys of sum |q k| scale"""
    n, H, d = q.shape
    L, Hkv = k.shape[:2]
    O, A, M, S = np.zeros((n, H, d)), np.zeros((n, H, d)), np.zeros((n, H, 1)), np.zeros((n, H, 1))
    for t in range(n):
        seen = slice(0, min(L, first + t + 1) if causal else L)
        for h in range(H):
            g = h // (H // Hkv)
            s = k[seen, g] @ q[t, h] / math.sqrt(d)
            p = np.exp(s - s.max())
            p /= p.sum()
            O[t, h], A[t, h] = p @ v[seen, g], p @ np.abs(v[seen, g])
            M[t, h] = (p * np.repeat(amax[:, g].astype(np.float64), 64)[seen]).max()
            S[t, h] = (np.abs(k[seen, g]) @ np.abs(q[t, h])).max() / math.sqrt(d)
    return O, A, M, S


def check(m, plan, H, q, causal=True):
    """As Model.check_attn, with what fp16's weights lose below its normal range taken from the largest of a query's own weights times V's
    size: a weight below 2^-14 is off by 2^-25 at most, and the largest is 2^9 or more, so a key adds at most 2^-34 of the
    largest p amax; an output below the normal range is off by half its step."""
    got = m.sp.sparge_cache_attn(m.cache, m.gpu(q), plan, causal=causal).double().cpu().numpy()
    least = 2.0 ** -25 if m.dtype == "fp16" else 2.0 ** -134
    at = 0
    for r, n in enumerate(m.new):
        if n == 0:
            continue
        k, v, _, av = m.stored(r)
        O, A, M, S = contributions(q[at:at + n], k, v, av, len(k) - n, causal)
        tol = U[m.dtype] * np.abs(O) + 1.02 * (2.0 ** -11 + 64 * 2.0 ** -24 + 2.0 ** -23 * (m.d + 8) * S) * A + len(k) * 2.0 ** -34 * M + least
        ratio = np.abs(got[at:at + n] - O) / tol
        assert ratio.max() <= 1.0, (r, ratio.max(), np.unravel_index(ratio.argmax(), ratio.shape))
        at += n


def tokens(m, n, loud, large, small, away):
    """K, V of a row's n tokens: those of the blocks in `loud` have values of size `large` and keys that point away from the
    direction (1, .., 1) by `away`, the others values of size `small`"""
    K, V = m.tokens(n)
    V = np.clip(np.rint(V * 2), -7, 7) / 7
    for b in range(-(-n // 64)):
        t = slice(64 * b, 64 * b + 64)
        V[t] *= large if b in loud else small
        if b in loud:
            K[t] = 0.1 * K[t] - away
    return m.round16(K), m.round16(V)


# sizes of V, how far the loud keys point away, the size of the queries: scores 60 powers of two below (d = 64: 8 away size nats), or 277
SIZES = [("bf16", 2.0 ** 33, 1.0, 2.6, 2.0), ("bf16", 2.0 ** 30, 1.0, 2.6, 2.0), ("bf16", 2.0 ** 20, 1.0, 2.6, 2.0), ("bf16", 2.0 ** 120, 2.0 ** -120, 6.0, 4.0),
         ("fp16", 60000.0, 1e-4, 2.6, 2.0), ("fp16", 60000.0, 0.02, 2.6, 2.0)]


@pytest.mark.parametrize("G,new", [(4, 1), (2, 8), (4, 30), (20, 3), (1, 100)])
@pytest.mark.parametrize("dtype,large,small,away,size", SIZES)
def test_large_values_that_no_query_attends_to(sp, dtype, large, small, away, size, G, new):
    """in front of the ordinary blocks, between them, behind them, everywhere but in the last two blocks; beside queries of the same tile that
    attend to nothing else"""
    where = [(0,), (1, 2), (3,), (0, 1, 2)]
    held = [256, 300, 256, 256, 256]
    m = Model(sp, len(held), 2, 64, 60, 8, dtype=dtype, seed=50 + G)
    parts = [tokens(m, h + new, loud, large, small, away) for h, loud in zip(held, where + [(0,)])]
    m.step(held, tokens=tuple(np.concatenate([p[i][:h] for p, h in zip(parts, held)]) for i in range(2)))
    plan = m.step([new] * len(held), tokens=tuple(np.concatenate([p[i][h:] for p, h in zip(parts, held)]) for i in range(2)))
    q = m.queries(2 * G, 0.1 * size) + size
    q[4 * new:, 1::2] *= -1                   # the last row: every other head attends to the loud block alone
    check(m, plan, 2 * G, m.round16(q))


@pytest.mark.parametrize("G,new", [(1, 9), (4, 40), (1, 200)])
@pytest.mark.parametrize("causal", [True, False])
def test_large_values_that_only_later_tokens_see(sp, causal, G, new):
    """a step's last page holds values 2^240 times as large as all before; the step's tokens before that page do not see it"""
    held = 256 - new // 2 - 1
    m = Model(sp, 2, 1, 64, 20, 8, dtype="bf16", seed=60 + G)
    parts = []
    for row in range(2):
        K, V = m.tokens(held + new)
        V = np.clip(np.rint(V * 2), -7, 7) * 2.0 ** -120
        V[(held + new - 1) // 64 * 64:] *= 2.0 ** (240 if row == 0 else 40)
        parts.append((K, V))
    m.step([held] * 2, tokens=tuple(np.concatenate([p[i][:held] for p in parts]) for i in range(2)))
    plan = m.step([new] * 2, tokens=tuple(np.concatenate([p[i][held:] for p in parts]) for i in range(2)))
    check(m, plan, G, m.queries(G), causal)


@pytest.mark.parametrize("dtype,large,small", [("bf16", 2.0 ** 33, 1.0), ("fp16", 60000.0, 1e-4)])
@pytest.mark.parametrize("G,new", [(4, 1), (4, 20)])
def test_large_values_in_long_rows(sp, dtype, large, small, G, new):
    """rows that several waves and workgroups share, a loud block in some of their parts, or a part of nothing else"""
    n = 9000
    m = Model(sp, 2, 1, 64, 300, 160, dtype=dtype, seed=70)
    parts = [tokens(m, n + new, loud, large, small, 2.6) for loud in ((0, 40, 41, 139), tuple(range(1, 100)))]
    m.step([n] * 2, tokens=tuple(np.concatenate([p[i][:n] for p in parts]) for i in range(2)))
    plan = m.step([new] * 2, tokens=tuple(np.concatenate([p[i][n:] for p in parts]) for i in range(2)))
    check(m, plan, G, m.round16(m.queries(G, 0.2) + 2.0))


def test_blocks_of_zeros_that_the_queries_attend_to(sp):
    """the largest weights' values are zero: what is left are the small weights' ordinary ones"""
    m = Model(sp, 3, 1, 64, 30, 8, dtype="bf16", seed=80)
    K, V = m.tokens(3 * 250)
    K[:100] = 0.1 * K[:100] + 2.0             # row 0: in front
    V[:128] = 0
    K[250 + 128:250 + 192] = 0.1 * K[250 + 128:250 + 192] + 2.0
    V[250 + 128:250 + 192] = 0                # row 1: in the middle
    V[500:] = 0                               # row 2: nothing but zeros
    K, V = m.round16(K), m.round16(V)
    m.step([250] * 3, tokens=(K, V))
    K2, V2 = m.tokens(3 * 3)
    V2[6:] = 0
    plan = m.step([3] * 3, tokens=(K2, V2))
    check(m, plan, 8, m.round16(m.queries(8, 0.2) + 0.5))
