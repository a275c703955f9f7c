"""Steps whose rows differ: which rows a workgroup takes together, and how, is decided on the device from the rows' tokens and keys.  Rows of
several tiles of 16 query rows in little work and in much, one row among idle ones, pieces beside decoding rows."""
import numpy as np
import pytest

from cache_cases import Model
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2502_18137_amd as sp
    return sp


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("G,new", [(16, [18, 0]), (5, [4, 1]), (4, [5, 30]), (3, [40, 0, 2, 6]), (1, [130, 1]), (1, [17, 17, 16]), (7, [33, 1, 2])])
def test_rows_of_several_tiles_in_little_work(sp, G, new, dtype, causal):
    """at most a few blocks a wave: waves take them tile by tile, the last one of fewer tokens"""
    m = Model(sp, len(new), 2, 128 if G < 5 else 64, 80, 30, dtype=dtype, seed=90 + G)
    m.step(([300, 70, 0, 64] * 2)[:len(new)])
    plan = m.step(new, pad=2)
    m.check_attn(plan, 2 * G, causal=causal, pad=2)
    mask = (m.rng.random((len(new), 2, 30)) < 0.5).astype(np.uint8)
    m.check_attn(plan, 2 * G, causal=causal, mask=mask, pad=2)


@pytest.mark.parametrize("new", [159, 160, 161])
def test_the_most_that_counts_as_little(sp, new):
    """tiles of one token, 64 blocks of keys each: up to 10240 blocks are waves' work, more are workgroups'"""
    m = Model(sp, 2, 1, 64, 140, 70, dtype="bf16", seed=new)
    m.step([4096 - new, 0])
    m.check_attn(m.step([new, 0]), 16)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("G,piece,others", [(4, 300, 0), (4, 300, 1), (1, 700, 0), (1, 700, 1), (2, 300, 2), (16, 40, 1)])
def test_one_row_among_many(sp, G, piece, others, dtype):
    """one row's piece of a prompt, the other 299 idle, or adding one token, or two; rows in any place"""
    m = Model(sp, 300, 2, 64, 900, 100, dtype=dtype, seed=100 + G + others)
    long = 5000 if G < 16 else 6000
    held = [int(n) for n in m.rng.integers(0, 100, 300)]
    held[131] = long
    m.step(held)
    new = [others] * 300
    new[131], new[7], new[299] = piece, 0, 3
    m.check_attn(m.step(new, pad=1), 2 * G, pad=1)


def test_the_same_step_again_and_again(sp):
    """the same bits on every call, whatever an earlier call left in the workspace"""
    import torch
    m = Model(sp, 40, 2, 128, 300, 60, dtype="bf16", seed=110)
    m.step([3000] + [50] * 39)
    mixed = m.step([200] + [1] * 39)
    q = m.gpu(m.queries(8))
    ws = torch.full((sp.sparge_cache_attn_workspace_bytes(m.cache, 8),), 255, dtype=torch.uint8, device="cuda")
    first = sp.sparge_cache_attn(m.cache, q, mixed, ws=ws).clone()
    m.check_attn(mixed, 8, q=q.double().cpu().numpy())
    small = m.step([3, 9] + [0] * 38)
    few = sp.sparge_cache_attn(m.cache, q[:12], small, ws=ws).clone()
    m.check_attn(small, 8, q=q[:12].double().cpu().numpy())
    for _ in range(2):
        assert torch.equal(sp.sparge_cache_attn(m.cache, q[:12], small, ws=ws), few)
    ws.fill_(0x7F)
    assert torch.equal(sp.sparge_cache_attn(m.cache, q[:12], small, ws=ws), few)
    assert bool(torch.isfinite(first.float()).all())


@pytest.mark.parametrize("G,few,many", [(4, 10, 200), (4, 16, 170), (1, 60, 700), (20, 3, 8), (32, 2, 3)])
def test_fp16_rows_do_not_lose_bits_to_their_neighbours(sp, G, few, many):
    """Rows of up to 64 query rows keep 22 bits of the weights whatever the other rows add: the norm of the error is that of rounding the exact
    results to fp16 (2^-12.3 of them in the mean) but for scores and sums in fp32, some 2^-20 of sum p |v|: for 700 keys attended to
    alike, whose values cancel to 1/26 of that, 2^-15.3 of the results and 1 % in quadrature; 5 % is taken.  (11 bits, 2^-12.3 of sum p |v|
    / sqrt(keys), would add 10 to 45 %.)"""
    m = Model(sp, 4, 2, 128, 500, 160, dtype="fp16", seed=120 + G)
    m.step([60, 8900, 700, 9000])
    new = [few, many, few, many]
    plan = m.step(new)
    q = m.queries(2 * G, 0.25)
    got = sp.sparge_cache_attn(m.cache, m.gpu(q), plan).double().cpu().numpy()
    at, error, rounding = 0, 0.0, 0.0
    for r, n in enumerate(new):
        if n == few:
            k, v, _, _ = m.stored(r)
            want = co.attend(q[at:at + n], k, v, len(k) - n, True, None, None)[0]
            error, rounding = error + np.square(got[at:at + n] - want).sum(), rounding + np.square(m.round16(want) - want).sum()
        at += n
    assert error <= 1.05 ** 2 * rounding, (error / rounding) ** 0.5


def test_a_captured_step_whose_rows_change(sp):
    """one graph of plan, append and attention, replayed with other rows adding other numbers of tokens every time: single tokens, rows of
    several tiles in little work, a long piece beside them, nothing at all; equal to the oracle, and to the call itself, bit by bit"""
    import torch
    m = Model(sp, 6, 2, 64, 400, 110, dtype="bf16", seed=130)
    m.step([6000, 3, 127, 200, 0, 64])
    slots = 400
    x = [torch.zeros(slots, h, 64, dtype=m.dt, device="cuda") for h in (2, 2, 8)]
    new = m.i32([0] * 6)
    plan = sp.CachePlan(*[torch.zeros(n, dtype=torch.int32, device="cuda") for n in (7, slots, slots, 2)])
    ws = torch.empty(sp.sparge_cache_attn_workspace_bytes(m.cache, 8), dtype=torch.uint8, device="cuda")
    out = torch.zeros(slots, 8, 64, dtype=m.dt, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sp.sparge_cache_plan(m.cache, new, slots, out=plan)
        sp.sparge_cache_append(m.cache, x[0], x[1], plan)
        sp.sparge_cache_attn(m.cache, x[2], plan, ws=ws, out=out)
    for step in ([1] * 6, [300, 1, 1, 1, 1, 1], [0, 40, 0, 7, 1, 0], [0] * 6, [2, 0, 5, 0, 350, 1], [1, 1, 0, 1, 1, 1]):
        n = sum(step)
        (K, V), m.new = m.tokens(n), step
        q = m.queries(8)
        for t, v in zip(x, (K, V, q)):
            t[:n].copy_(m.gpu(v))
        new.copy_(m.i32(step))
        out.fill_(7.25)
        m.book.plan(step, None, slots)
        at = 0
        for r, k in enumerate(step):
            m.K[r], m.V[r] = np.concatenate([m.K[r], K[at:at + k]]), np.concatenate([m.V[r], V[at:at + k]])
            at += k
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert plan.status[0] == 0 and m.cache.length.tolist() == m.book.length
        m.check_stored()
        eager, _ = m.check_attn(plan, 8, q=q, pad=slots - n)
        assert np.array_equal(out.double().cpu().numpy(), eager)


@pytest.mark.parametrize("G", [1, 4, 20])
def test_pieces_among_all_rows_there_can_be(sp, G):
    """4096 rows, several to a thread that looks for them; two of them add long pieces, some a token or a few"""
    m = Model(sp, 4096, 2, 64, 4500, 110, dtype="fp16", seed=140 + G)
    held = m.rng.integers(0, 4, 4096)
    held[[777, 4095]] = 5000, 1500
    m.step(held.tolist())
    new = (m.rng.random(4096) < 0.02).astype(int)
    new[[3, 776, 2000]] = 9, 2, 30
    new[[777, 4095]] = 300, 260
    m.check_attn(m.step(new.tolist(), pad=2), 2 * G, pad=2)
