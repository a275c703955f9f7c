"""The paged 8-bit K/V cache at the ends of its ranges, and in the orders that a program may call it in."""
import numpy as np
import pytest

from cache_cases import Model, U
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2502_18137_amd as sp
    return sp


def relative_check(m, plan, H, q):
    """as Model.check_attn, without its absolute term: 2^-11 and the sums' 2^-18 of sum p |v|, 2^-33 of the largest |v| per key, half a
    step of the output, half of bf16's least subnormal"""
    got = m.sp.sparge_cache_attn(m.cache, m.gpu(q), plan).double().cpu().numpy()
    at = 0
    for r, n in enumerate(m.new):
        if n == 0:
            continue
        k, v, _, _ = m.stored(r)
        O, A, S = co.attend(q[at:at + n], k, v, len(k) - n, True, None, None)
        exp = 2.0 ** -23 * (m.d + 8) * S
        tol = U["bf16"] * np.abs(O) + 1.02 * (2.0 ** -11 + 64 * 2.0 ** -24 + exp[:, :, None]) * A
        tol += len(k) * 2.0 ** -33 * np.abs(v).max(initial=0) + 2.0 ** -134
        ratio = np.abs(got[at:at + n] - O) / tol
        assert ratio.max() <= 1.0, (r, ratio.max())
        at += n


@pytest.mark.parametrize("G,new", [(2, 1), (2, 30), (5, 64), (20, 3)])
def test_values_over_bf16s_range(sp, G, new):
    """V's amax from the least subnormal to nearly the largest value, the same for a row's blocks and different ones, items in one part and
    in several"""
    powers = [(-133,) * 4, (-126,) * 4, (-100,) * 4, (100,) * 4, (124,) * 4, (-130, 0, -130, 0), (0, -120, 60, -133), (-133, -126, -110, -90),
              (124, 0, -124, 124)]
    held = 256 - new
    m = Model(sp, len(powers), 2, 64, 60, 6, dtype="bf16", seed=G)
    for first in (True, False):
        n = [held] * len(powers) if first else [new] * len(powers)
        K, V = m.tokens(sum(n))
        V = np.clip(np.rint(V * 2), -7, 7)
        at = 0
        for p in powers:
            for t in range(n[0]):
                V[at + t] *= 2.0 ** p[((0 if first else held) + t) // 64]
            at += n[0]
        plan = m.step(n, tokens=(K, V))
    m.check_stored()
    relative_check(m, plan, 2 * G, m.queries(2 * G))


@pytest.mark.parametrize("G", [1, 4, 17])
def test_all_rows_there_can_be(sp, G):
    """4096 rows of few keys, some of them empty: more rows than parts, parts that hold several rows"""
    m = Model(sp, 4096, 1, 64, 4200, 2, dtype="bf16", seed=30 + G)
    m.step(m.rng.integers(0, 4, size=4096).tolist())
    plan = m.step((m.rng.random(4096) < 0.9).astype(int).tolist())
    m.check_attn(plan, G)
    plan = m.step((m.rng.integers(0, 40, size=4096) == 0).astype(int).tolist(), pad=5)
    m.check_attn(plan, G, pad=5)


@pytest.mark.parametrize("G,new", [(1, 1), (3, 40)])
def test_as_many_heads_as_there_can_be(sp, G, new):
    Hkv = 128 // G
    m = Model(sp, 2, Hkv, 64, 20, 8, dtype="fp16", seed=33, shift=True)
    m.step([130, 5])
    m.check_stored()
    m.check_attn(m.step([new, new]), Hkv * G)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("G,new", [(2, [1, 1, 1]), (2, [30, 1, 0]), (40, [2, 1, 3])])
def test_everything_at_once(sp, G, new, causal):
    """a block mask, tokens inside a projection's output, rows behind the last token, a shift, a softmax scale"""
    m = Model(sp, 3, 2, 128, 40, 12, dtype="bf16", seed=34, shift=True)
    m.step([500, 63, 1], pad=9, fused=3)
    plan = m.step(new, pad=21, fused=2)
    m.check_stored()
    mask = (m.rng.random((3, 2, 12)) < 0.5).astype(np.uint8)
    m.check_attn(plan, 2 * G, causal=causal, mask=mask, scale=0.3, pad=21, fused=1)


def test_two_calls_at_once(sp):
    """the same and different queries over one cache on two streams, a workspace each"""
    import torch
    m = Model(sp, 4, 2, 128, 400, 130, dtype="bf16", seed=35)
    m.step([8000, 100, 3000, 64])
    plan = m.step([1, 20, 1, 3])
    q = [m.gpu(m.queries(8)) for _ in range(2)]
    want = [sp.sparge_cache_attn(m.cache, x, plan) for x in q]
    n = sp.sparge_cache_attn_workspace_bytes(m.cache, 8)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [[torch.zeros_like(x) for _ in range(4)] for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                sp.sparge_cache_attn(m.cache, q[i], plan, ws=ws[i], out=out[i][k])
    torch.cuda.synchronize()
    for i in range(2):
        for o in out[i]:
            assert torch.equal(o, want[i])


def test_a_step_without_tokens(sp):
    """rows that are only padding, or none at all: nothing changes, nothing is written"""
    import torch
    m = Model(sp, 3, 2, 64, 20, 4, dtype="fp16", seed=36)
    m.step([70, 0, 5])
    plan = m.step([0, 0, 0], pad=6)
    m.check_stored()
    m.check_attn(plan, 4, pad=6)
    plan = m.step([0, 0, 0])
    m.check_stored()
    assert sp.sparge_cache_attn(m.cache, m.gpu(np.zeros((0, 4, 64))), plan).shape == (0, 4, 64)
    k, v = sp.sparge_cache_read(m.cache, m.i32([]))
    assert k.shape == v.shape == (0, 2, 64)
    m.step([0, 0, 0], release=[1, 0, 1])
    assert m.book.length == [0, 0, 0]


@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16")])
def test_reads_in_every_order(sp, d, dtype):
    """the same slot again and again, runs forwards and backwards, single ones, runs over a page's end, more slots than tokens"""
    import torch
    m = Model(sp, 2, 3, d, 10, 4, dtype=dtype, seed=37)
    m.step([200, 131])
    at = lambda r, t: m.book.table[r, t // 64] * 64 + t % 64
    seq = [(0, t) for t in range(200)] + [(0, t) for t in range(199, 150, -1)] + [(1, 7)] * 70 + [(1, t) for t in range(60, 70)]
    seq += [(int(r), int(t)) for r, t in zip(m.rng.integers(0, 2, 300), m.rng.integers(0, 131, 300))]
    k, v = sp.sparge_cache_read(m.cache, m.i32([int(at(r, t)) for r, t in seq]), dtype=torch.float32)
    kept = [m.stored(r)[:2] for r in range(2)]
    for i, x in enumerate((k, v)):
        want = np.stack([kept[r][i][t] for r, t in seq]).astype(np.float32)
        assert np.array_equal(x.cpu().numpy(), want)


@pytest.mark.parametrize("G,new", [(4, 1), (2, 6), (20, 1), (3, 20)])
def test_fp16_results_are_off_by_their_own_rounding(sp, G, new):
    """Up to 64 query rows a row, weights keep 22 bits: the error's norm is that of rounding the exact results to fp16 (half a step, 2^-11, at
    most; 2^-12.3 of the results in the mean) but for terms of some 2^-18 of them (scores and sums in fp32), which add 1 % in
    quadrature; 10 % is taken.  (Weights of one part, 2^-12.3 too, would add 20 to 60 %.)"""
    m = Model(sp, 4, 2, 128, 140, 40, dtype="fp16", seed=40 + G)
    m.step([2000, 130, 700, 1500])
    plan = m.step([new] * 4)
    q = m.queries(2 * G)
    got = sp.sparge_cache_attn(m.cache, m.gpu(q), plan).double().cpu().numpy()
    want = np.zeros_like(got)
    for r in range(4):
        k, v, _, _ = m.stored(r)
        rows = slice(new * r, new * (r + 1))
        want[rows] = co.attend(q[rows], k, v, len(k) - new, True, None, None)[0]
    assert np.linalg.norm(got - want) <= 1.1 * np.linalg.norm(m.round16(want) - want)
