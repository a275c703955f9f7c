"""The paged 8-bit K/V cache through the public entry points, against the 64-bit oracle: bookkeeping (equal), stored codes and
scales (equal), attention (element by element, tests/cache_cases.py says what is allowed)."""
import numpy as np
import pytest

from tests.cache_cases import Model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2502_18137_amd as sp
    sp.load_library()
    return sp


# ---- bookkeeping and storage
def test_steps_with_releases(sp):
    m = Model(sp, 5, 2, 64, 40, 9, dtype="fp16", seed=1, free=np.random.default_rng(0).permutation(40))
    m.step([3, 0, 64, 130, 65], pad=2)
    m.step([1, 1, 1, 1, 1])
    m.step([60, 0, 0, 200, 2], release=[0, 1, 1, 0, 0], pad=1)
    m.step([0, 0, 0, 0, 0])
    m.step([0, 0, 70, 0, 1], release=[1, 0, 1, 1, 1])
    m.step([0, 0, 0, 0, 0], release=[1, 1, 1, 1, 1])
    assert int(m.cache.n_free) == 40
    m.step([200, 64, 63, 1, 576])
    m.check_stored()


@pytest.mark.parametrize("rows", [1, 64, 1000, 4096])
def test_many_rows(sp, rows):
    rng = np.random.default_rng(rows)
    m = Model(sp, rows, 1, 64, 3 * rows + 8, 3, seed=rows)
    m.step(rng.integers(0, 70, rows).tolist(), pad=5)
    m.step((rng.random(rows) < 0.8).astype(int).tolist(), release=(rng.random(rows) < 0.2).astype(int).tolist())
    if rows <= 64:
        m.check_stored()


def test_long_prompt_fills_its_slots(sp):
    m = Model(sp, 3, 1, 64, 700, 400, seed=2)
    m.step([20011, 0, 9000], pad=77)       # (slots beyond what the plan's own workgroup fills)
    m.check_stored()


def test_a_step_that_does_not_fit_changes_nothing(sp):
    import torch
    m = Model(sp, 3, 1, 64, 6, 4, seed=3)
    m.step([70, 10, 0])
    before, k = m.cache.book.clone(), m.cache.k.clone()
    for new, n_slots, want in (([0, 0, 256], 300, sp.CACHE_NO_PAGES), ([200, 0, 0], 300, sp.CACHE_ROW_FULL), ([1, 1, 1], 2, sp.CACHE_NO_SLOTS),
                               ([300, 300, 300], 2, 7), ([1, -1, 0], 5, sp.CACHE_BAD_STATE), ([1, 2 ** 31 - 1, 2 ** 31 - 1], 5, 7)):
        plan = sp.sparge_cache_plan(m.cache, m.i32(new), n_slots)
        assert plan.status.tolist() == [want, 3] and torch.equal(m.cache.book, before)
        assert plan.cu.tolist() == [0] * 4 and plan.slots.tolist() == [-1] * n_slots and plan.req.tolist() == [-1] * n_slots
        x = torch.ones(n_slots, 1, 64, dtype=torch.bfloat16, device="cuda")
        sp.sparge_cache_append(m.cache, x, x, plan)
        out = torch.full((n_slots, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        sp.sparge_cache_attn(m.cache, torch.ones_like(out), plan, out=out)
        assert torch.equal(m.cache.k, k) and bool((out == 3).all())
    bad = m.cache.length.clone()
    for length in (-1, 4 * 64 + 1):
        m.cache.length[1] = length
        assert sp.sparge_cache_plan(m.cache, m.i32([0, 0, 0]), 0).status[0] == sp.CACHE_BAD_STATE
    m.cache.length.copy_(bad)
    m.step([0, 5, 0])
    m.check_stored()


@pytest.mark.parametrize("d,dtype,shift", [(64, "fp16", False), (64, "bf16", True), (128, "fp16", True), (128, "bf16", False)])
def test_codes_do_not_depend_on_the_steps(sp, d, dtype, shift):
    """The same tokens at once and in pieces (one by one through an open page, across several pages, ends on a page's end)."""
    pieces = [[1, 130], [1, 1], [62, 0], [1, 61], [70, 1], [3, 64], [200, 200], [1, 1]]
    m = Model(sp, 2, 3, d, 40, 12, dtype=dtype, seed=4, shift=shift)
    for p in pieces:
        m.step(p, pad=3, fused=2)
        m.check_stored()
    one = Model(sp, 2, 3, d, 40, 12, dtype=dtype, seed=4, shift=shift)
    one.step(np.sum(pieces, axis=0).tolist(), tokens=(np.concatenate(m.K), np.concatenate(m.V)))
    one.check_stored()


def test_blocks_of_extreme_size(sp):
    """amax from the smallest subnormal to the largest finite value, zero blocks, a NaN and an infinity (codes 0)."""
    import torch
    m = Model(sp, 6, 1, 64, 12, 2, dtype="bf16", seed=5)
    K, V = m.tokens(6 * 64)
    for r, s in enumerate((2.0 ** -133, 2.0 ** -126, 0.0, 2.0 ** 126, 1.0, 1.0)):
        K[r * 64:(r + 1) * 64] = np.clip(np.rint(K[r * 64:(r + 1) * 64] * 2), -3, 3) * s if s != 1.0 else K[r * 64:(r + 1) * 64]
    K[4 * 64 + 7, 0, 3], K[5 * 64 + 8, 0, 4] = np.inf, np.nan
    V[5 * 64 + 1, 0, 1] = -np.inf
    m.step([64] * 6, tokens=(K, V))
    m.check_stored()


def test_halves_round_to_even(sp):
    """quotients 127 x / amax that are a half exactly: amax 127 2^a, x odd multiples of 2^(a-1)"""
    m = Model(sp, 1, 1, 64, 2, 2, dtype="fp16", seed=6)
    x = (np.arange(64 * 64).reshape(64, 1, 64) % 507 - 253) / 2.0
    x[0, 0, 0] = 127.0
    m.step([64], tokens=(x / 4, x * 2))
    m.check_stored()


def test_read_any_slots(sp):
    import torch
    m = Model(sp, 3, 2, 128, 20, 4, dtype="bf16", seed=7, shift=True)
    m.step([100, 64, 3])
    rows = np.array([0, 2, 1, 0, 0, 1, 2, 0])
    pos = np.array([99, 2, 63, 0, 64, 1, 0, 99])
    slots = m.book.table[rows, pos // 64] * 64 + pos % 64
    slots = np.concatenate([slots, [-1, 20 * 64, 2 ** 31 - 1]])
    req = np.concatenate([rows, [0, 0, 0]])
    for dt in (torch.float32, torch.bfloat16):
        out = tuple(torch.full((11, 2, 128), 5.0, dtype=dt, device="cuda") for _ in range(2))
        k, v = sp.sparge_cache_read(m.cache, m.i32(slots), m.i32(req), dtype=dt, out=out)
        assert bool((k[8:] == 5).all()) and bool((v[8:] == 5).all())
        for i, (r, t) in enumerate(zip(rows, pos)):
            wk, wv, _, _ = m.stored(r)
            want = [torch.from_numpy((w[t] + s).astype(np.float32)).to(dt) for w, s in ((wk, m.shift[r]), (wv, 0))]
            assert torch.equal(k[i].cpu(), want[0]) and torch.equal(v[i].cpu(), want[1])


# ---- attention
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hkv,G", [(1, 1), (2, 3), (3, 16), (1, 20), (2, 64), (1, 128)])
def test_decode(sp, Hkv, G, d, dtype):
    """one token a row, rows of one key to several pages"""
    held = [0, 1, 62, 63, 64, 127, 300, 1000]
    m = Model(sp, len(held), Hkv, d, 60, 20, dtype=dtype, seed=G)
    m.step(held)
    plan = m.step([1] * len(held))
    m.check_attn(plan, Hkv * G)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("G,new", [(1, [5, 0, 33, 200, 1]), (4, [70, 3, 0, 64, 17]), (7, [20, 1, 100, 9, 0]), (80, [3, 0, 2, 5, 1]), (2, [700, 1, 0, 2, 90])])
def test_pieces(sp, G, new, causal):
    m = Model(sp, 5, 1 if G > 7 else 2, 128 if G != 2 else 64, 80, 30, dtype="bf16" if G != 4 else "fp16", seed=G, shift=G == 7)
    m.step([0, 130, 64, 1, 500])
    plan = m.step(new, pad=3, fused=1)
    m.check_attn(plan, m.Hkv * G, causal=causal, pad=3, fused=2)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kept", [0.0, 0.3, 0.8])
def test_masks(sp, kept, causal):
    """blocks left out, rows that see nothing (output 0), the last block left out"""
    m = Model(sp, 4, 2, 64, 120, 40, dtype="fp16", seed=int(kept * 10))
    m.step([0, 100, 640, 1900])
    plan = m.step([40, 3, 1, 130])
    mask = (np.random.default_rng(1).random((4, 2, 40)) < kept).astype(np.uint8) * 255
    mask[2, 1] = 0
    mask[1, 0, 1] = 0
    got, _ = m.check_attn(plan, 6, causal=causal, mask=mask)
    assert (got[43, 3:] == 0).all()


def test_split_over_workgroups(sp):
    """one long row: its keys are shared by many workgroups; long rows among short ones"""
    m = Model(sp, 1, 1, 128, 700, 650, dtype="bf16", seed=11)
    m.step([40000])
    plan = m.step([1])
    m.check_attn(plan, 4)
    plan = m.step([9])
    m.check_attn(plan, 4)
    m = Model(sp, 12, 2, 64, 700, 400, dtype="fp16", seed=12)
    m.step([20000] + [17] * 10 + [5000])
    plan = m.step([1, 0, 30] + [1] * 8 + [40])
    m.check_attn(plan, 10)


def test_scales_that_differ_between_blocks(sp):
    """V of very different size from block to block (rising, falling, zero blocks), keys that win late"""
    m = Model(sp, 3, 1, 64, 40, 12, dtype="fp16", seed=13)
    K, V = m.tokens(3 * 640)
    up = np.repeat(2.0 ** np.array([0, 3, -4, 5, -8, 7, 0, -12, 2, 6]), 64)[:, None, None]
    V[:640] = m.round16(V[:640] * up)
    V[640:1280] = m.round16(V[640:1280] * up[::-1])
    V[1280:1280 + 128] = 0
    V[1500:1570] = 0
    K[1280:] = m.round16(K[1280:] * np.linspace(0.01, 4, 640)[:, None, None])
    m.step([640] * 3, tokens=(K, V))
    plan = m.step([1, 2, 30])
    m.check_attn(plan, 4, scale=0.3)
    m.check_attn(plan, 4, causal=False, scale=1e-4)


def test_zero_queries_and_tiny_ones(sp):
    m = Model(sp, 1, 2, 64, 10, 5, dtype="bf16", seed=14)
    m.step([200])
    plan = m.step([4])
    q = m.queries(4)
    q[0], q[1], q[2] = 0, m.round16(q[1] * 2.0 ** -130), m.round16(q[2] * 2.0 ** 20)
    m.check_attn(plan, 4, q=q, scale=2.0 ** -19)


def test_not_finite_stays_where_it_is_seen(sp):
    """a NaN key block, an infinite V block, a NaN query: NaN exactly in the rows that see them; a block behind the mask or in
    the future of a query does nothing to it"""
    import torch
    m = Model(sp, 3, 1, 64, 20, 6, dtype="bf16", seed=15)
    K, V = m.tokens(3 * 256)
    K[70, 0, 5], V[256 + 200, 0, 5], K[512 + 255] = np.nan, np.inf, np.nan
    m.step([250, 256, 192], tokens=(np.concatenate([K[:250], K[256:512], K[512:704]]), np.concatenate([V[:250], V[256:512], V[512:704]])))
    K2, V2 = m.tokens(74)
    K2[-1] = np.nan                      # row 2: its last token's page
    plan = m.step([2, 8, 64], tokens=(K2, V2))
    q = m.queries(2)
    q[5, 1, 3] = np.inf
    out = sp.sparge_cache_attn(m.cache, m.gpu(q), plan).float().cpu().numpy()
    nan = np.isnan(out).all(axis=2)
    assert nan[:2].all() and nan[2:10].all()          # rows 0 and 1 see their bad blocks
    assert nan[10:].all()                             # the page of row 2's last token is the page of all its new tokens
    mask = np.ones((3, 1, 6), np.uint8)
    mask[0, 0, 1], mask[1, 0, 3], mask[2, 0, 3] = 0, 0, 0
    got = sp.sparge_cache_attn(m.cache, m.gpu(q), plan, mask=torch.from_numpy(mask).cuda()).float().cpu().numpy()
    want = np.zeros(got.shape[:2], bool)
    want[5, 1] = True
    assert (np.isnan(got).any(axis=2) == want).all()
    # a piece whose last token's page is bad: earlier pages' tokens are untouched by it
    m = Model(sp, 1, 1, 64, 20, 6, dtype="fp16", seed=16)
    K, V = m.tokens(200)
    K[199, 0, 0], V[199, 0, 1] = np.inf, np.nan
    plan = m.step([200], tokens=(K, V))
    got = sp.sparge_cache_attn(m.cache, m.gpu(m.queries(3)), plan).float().cpu().numpy()
    assert np.isfinite(got[:192]).all() and np.isnan(got[192:]).all()


def test_workspace_and_outputs_need_no_clearing(sp):
    """the same bits whatever the workspace, stale pages and the output held, and on every call"""
    import torch
    m = Model(sp, 9, 2, 128, 200, 60, dtype="fp16", seed=17)
    m.step([3000, 1, 70, 500, 64, 0, 2, 1500, 9])
    plan = m.step([1, 1, 40, 1, 3, 2, 1, 1, 100])
    q = m.gpu(m.queries(8))
    n = sp.sparge_cache_attn_workspace_bytes(m.cache, 8)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    first = sp.sparge_cache_attn(m.cache, q, plan, ws=ws).clone()
    for fill in (255, 0x7F):
        ws.fill_(fill)
        assert torch.equal(sp.sparge_cache_attn(m.cache, q, plan, ws=ws, out=torch.full_like(first, float("nan"))), first)


def test_strides(sp):
    """tokens and heads in other orders: heads outermost, one projection's output, an output inside a wider tensor"""
    import torch
    m = Model(sp, 4, 4, 64, 40, 10, dtype="bf16", seed=18)
    m.step([100, 5, 64, 300])
    plan = m.step([3, 1, 20, 2])
    q = m.gpu(m.queries(8))
    want = sp.sparge_cache_attn(m.cache, q, plan)
    heads_first = q.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((26, 11, 72), 9.0, dtype=q.dtype, device="cuda")
    got = sp.sparge_cache_attn(m.cache, heads_first, plan, out=wide[:, 2:10, :64])
    assert torch.equal(got, want) and bool((wide[:, :2] == 9).all()) and bool((wide[:, 10:] == 9).all()) and bool((wide[:, :, 64:] == 9).all())


def test_pages_outside_the_pool_are_not_seen(sp):
    import torch
    m = Model(sp, 2, 1, 64, 12, 6, dtype="fp16", seed=19)
    m.step([200, 130])
    plan = m.step([1, 1])
    mask = np.ones((2, 1, 6), np.uint8)
    mask[0, 0, 1] = mask[1, 0, 0] = 0
    q = m.gpu(m.queries(2))
    want = sp.sparge_cache_attn(m.cache, q, plan, mask=torch.from_numpy(mask).cuda())
    m.cache.table[0, 1], m.cache.table[1, 0] = 12, -5
    assert torch.equal(sp.sparge_cache_attn(m.cache, q, plan), want)


# ---- as a program uses them
def test_a_program_of_steps(sp):
    """prompts, decoding, a row that ends and is used again, a piece of a prompt beside decoding rows"""
    m = Model(sp, 6, 2, 128, 80, 16, dtype="bf16", seed=20, shift=True)
    for new, release in (([100, 0, 64, 7, 0, 0], None), ([1, 300, 1, 1, 0, 0], None), ([1, 1, 1, 1, 0, 65], None),
                         ([1, 1, 50, 1, 0, 1], [0, 0, 1, 0, 0, 0]), ([0, 128, 1, 0, 3, 1], [1, 0, 0, 1, 0, 0])):
        plan = m.step(new, release, pad=2)
        m.check_attn(plan, 8, pad=2)
    m.check_stored()


def test_layers_share_a_plan(sp):
    import torch
    a = sp.SpargeCache(2, 1, 64, 10, 4, dtype=torch.float16)
    b = sp.SpargeCache(2, 2, 64, 10, 4, dtype=torch.float16, share=a)
    x = torch.randn(70, 3, 64, device="cuda").half()
    plan = sp.sparge_cache_plan(a, torch.tensor([66, 4], dtype=torch.int32, device="cuda"), 70)
    sp.sparge_cache_append(a, x[:, :1], x[:, 1:2], plan)
    sp.sparge_cache_append(b, x[:, 1:], x[:, :2], plan)
    assert torch.equal(sp.sparge_cache_read(a, plan.slots)[1], sp.sparge_cache_read(b, plan.slots)[0][:, :1])


def test_other_stream(sp):
    import torch
    m = Model(sp, 3, 2, 64, 30, 8, dtype="fp16", seed=21)
    m.step([100, 200, 3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan = m.step([1, 1, 1])
        m.check_attn(plan, 4)


def test_graph_of_a_step(sp):
    """plan, append and attention captured once, replayed as the steps of a program; two graphs at once on two streams"""
    import torch
    models, graphs, ins, outs, plans = [], [], [], [], []   # (a graph's tensors, its workspace too, live as long as the graph)
    for s in range(2):
        m = Model(sp, 4, 2, 64, 60, 8, dtype="bf16", seed=22 + s)
        m.step([60, 3, 127, 200])
        x = [torch.zeros(4, h, 64, dtype=m.dt, device="cuda") for h in (2, 2, 4)]
        new = m.i32([1] * 4)
        plan = sp.CachePlan(*[torch.zeros(n, dtype=torch.int32, device="cuda") for n in (5, 4, 4, 2)])
        ws = torch.empty(sp.sparge_cache_attn_workspace_bytes(m.cache, 4), dtype=torch.uint8, device="cuda")
        out = torch.zeros(4, 4, 64, dtype=m.dt, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sp.sparge_cache_plan(m.cache, new, 4, out=plan)
            sp.sparge_cache_append(m.cache, x[0], x[1], plan)
            sp.sparge_cache_attn(m.cache, x[2], plan, ws=ws, out=out)
        models.append(m), graphs.append(g), ins.append(x), outs.append(out), plans.append((plan, new, ws))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step in range(6):
        qs = []
        for m, x in zip(models, ins):
            K, V = m.tokens(4)
            m.new = [1] * 4
            q = m.queries(4)
            for t, v in zip(x, (K, V, q)):
                t.copy_(m.gpu(v))
            for r in range(4):
                m.K[r], m.V[r] = np.concatenate([m.K[r], K[r:r + 1]]), np.concatenate([m.V[r], V[r:r + 1]])
            m.book.plan([1] * 4, None, 4)
            qs.append(q)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for m, q, out, (plan, _, _) in zip(models, qs, outs, plans):
            assert plan.status[0] == 0 and m.cache.length.tolist() == m.book.length
            m.check_stored()
            eager, _ = m.check_attn(plan, 4, q=q)
            assert np.array_equal(out.double().cpu().numpy(), eager)


def test_offsets_beyond_32_bits(sp):
    """a pool whose K alone is beyond 2^32 bytes, rows at its end"""
    import torch
    pages = (1 << 32) // (8 * 64 * 128) + 40
    m = Model(sp, 2, 8, 128, pages, 8, dtype="bf16", seed=30, free=None)
    m.cache.free_pages.copy_(torch.arange(pages, dtype=torch.int32))
    m.book.free = list(range(pages))
    m.step([200, 3])
    m.check_stored()
    plan = m.step([1, 70], check=False)
    m.check_attn(plan, 16)


def test_a_cached_prefix_for_the_sparse_attention(sp):
    """tokens read back feed the attention over whole tensors: it gives what the cache's attention gives, up to the
    quantization of Q and K on either side (3e-2, the bound of the INT8 path against exact attention)"""
    import torch
    n, H, d = 512, 2, 128
    m = Model(sp, 1, H, d, 10, 9, dtype="bf16", seed=31)
    plan = m.step([n])
    slots = plan.slots
    k, v = sp.sparge_cache_read(m.cache, slots)
    q = m.gpu(m.queries(H, 1.0))
    whole = lambda t: t.transpose(0, 1).unsqueeze(0).contiguous()
    O = sp.sparge_attn(whole(q), whole(k), whole(v), None, -float("inf"), causal=True)
    got = sp.sparge_cache_attn(m.cache, q, plan)
    a, b = whole(got).float(), O.float()
    assert float((a - b).abs().sum() / b.abs().sum()) <= 3e-2


def test_the_binding_refuses(sp):
    import torch
    m = Model(sp, 2, 2, 64, 10, 4, dtype="bf16", seed=40)
    plan = m.step([3, 2])
    c, new = m.cache, m.i32([1, 1])
    x = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    cpu = sp.CachePlan(plan.cu.cpu(), plan.slots.cpu(), plan.req.cpu(), plan.status.cpu())
    other = sp.CachePlan(torch.cat([plan.cu, plan.cu[-1:]]), plan.slots, plan.req, plan.status)     # of three rows
    calls = [lambda: sp.CachePlan(plan.cu.cpu(), plan.slots, plan.req, plan.status), lambda: sp.CachePlan(plan.cu, plan.slots, plan.req[1:], plan.status),
             lambda: sp.CachePlan(plan.cu.long(), plan.slots, plan.req, plan.status), lambda: sp.sparge_cache_append(c, x, x, other),
             lambda: sp.sparge_cache_attn(c, q, other), lambda: sp.sparge_cache_plan(c, new, 5, out=other), lambda: sp.sparge_cache_plan(c, new.long(), 5), lambda: sp.sparge_cache_plan(c, new[:1], 5), lambda: sp.sparge_cache_plan(c, new.cpu(), 5),
             lambda: sp.sparge_cache_plan(c, new, 5, release=new), lambda: sp.sparge_cache_plan(c, new, 4, out=plan),
             lambda: sp.sparge_cache_plan(c, new, -1),
             lambda: sp.sparge_cache_append(c, x[:4], x, plan), lambda: sp.sparge_cache_append(c, x, x.half(), plan),
             lambda: sp.sparge_cache_append(c, x.cpu(), x, plan), lambda: sp.sparge_cache_append(c, q, x, plan), lambda: sp.sparge_cache_append(c, x, x, cpu),
             lambda: sp.sparge_cache_append(c, x.transpose(1, 2).contiguous().transpose(1, 2), x, plan),
             lambda: sp.sparge_cache_read(c, plan.slots.long()), lambda: sp.sparge_cache_read(c, plan.slots, dtype=torch.float16),
             lambda: sp.sparge_cache_read(c, plan.slots, plan.req[:2]), lambda: sp.sparge_cache_read(c, plan.slots, out=(x, x[:, :1])),
             lambda: sp.sparge_cache_attn(c, q[:, :3], plan), lambda: sp.sparge_cache_attn(c, q[:3], plan), lambda: sp.sparge_cache_attn(c, q.half(), plan),
             lambda: sp.sparge_cache_attn(c, q, plan, mask=torch.ones(2, 2, 3, dtype=torch.uint8, device="cuda")),
             lambda: sp.sparge_cache_attn(c, q, plan, ws=torch.empty(256, dtype=torch.uint8, device="cuda")),
             lambda: sp.sparge_cache_attn(c, q, plan, out=q[:, :1].expand(5, 4, 64)), lambda: sp.sparge_cache_attn(c, q, cpu),
             lambda: sp.SpargeCache(2, 2, 64, 10, 4, k_shift=torch.zeros(2, 2, 64, device="cuda").half()),
             lambda: sp.SpargeCache(2, 2, 64, 11, 4, share=c)]
    before = c.book.clone()
    for i, f in enumerate(calls):
        with pytest.raises((sp.SpargeError, RuntimeError)):
            f()
    assert torch.equal(before, c.book)
