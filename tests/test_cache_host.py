"""The paged 8-bit cache without a GPU: the oracle against independent evaluations, and what the entry points refuse (before
anything is enqueued: the device pointers are made up)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from oracle import cache_oracle as co


# ---- the oracle
def test_codes_are_the_exact_quotients_rounded():
    rng = np.random.default_rng(0)
    x = np.float32(rng.normal(size=(64, 1, 8))).astype(np.float16).astype(np.float32)
    x[:8, 0, 0] = [1.0, 0.5, -0.5, 0.25, 63.5 / 127, 2.5 / 127, 0.0, -1.0]
    for shift in (None, np.float32(rng.normal(size=(1, 8)))):
        codes, amax = co.quantize_tokens(x, shift)
        y = x if shift is None else x - shift
        top = Fraction(float(np.abs(y).max()))
        assert Fraction(float(amax[0, 0])) == top
        for c, v in zip(codes.reshape(-1), y.reshape(-1)):
            q = 127 * Fraction(float(v)) / top
            n = round(q)                     # (python rounds a fraction's halves to even)
            assert c == n
    assert np.abs(co.values(*co.quantize_tokens(x))- x).max() <= float(np.abs(x).max()) / 254 * (1 + 1e-12)


def test_zero_and_not_finite_blocks():
    x = np.ones((130, 2, 4), np.float32)
    x[:64, 0], x[70, 1, 2], x[128, 0, 0] = 0, np.nan, -np.inf
    codes, amax = co.quantize_tokens(x)
    assert (codes[:64, 0] == 0).all() and amax[0, 0] == 0 and (codes[:64, 1] == 127).all()
    assert (codes[64:128, 1] == 0).all() and np.isnan(amax[1, 1]) and (codes[64:128, 0] == 127).all()
    assert (codes[128:, 0] == 0).all() and np.isinf(amax[2, 0])


def test_attend_is_softmax_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(70, 2, 8)), rng.normal(size=(70, 2, 8))
    mask = np.array([[1, 1], [0, 1]])
    O, A, _ = co.attend(q, k, v, 65, True, mask)
    for t in range(3):
        for h in range(4):
            keys = [j for j in range(70) if j <= 65 + t and mask[h // 2][j // 64]]
            w = {j: np.exp(sum(q[t, h, c] * k[j, h // 2, c] for c in range(8)) / np.sqrt(8)) for j in keys}
            want = sum(w[j] * v[j, h // 2] for j in keys) / sum(w.values())
            assert np.abs(O[t, h] - want).max() < 1e-13 and (A[t, h] >= np.abs(want) - 1e-13).all()
    assert (co.attend(q, k, v, 65, False, np.zeros((2, 2)))[0] == 0).all()


def test_book():
    b = co.Book(3, 6, 4)
    cu, slots, req, status = b.plan([65, 0, 2], None, 70)
    assert cu.tolist() == [0, 65, 65, 67] and status == [0, 3] and b.free == [5, 4, 3]
    assert slots.tolist() == list(range(64)) + [64, 128, 129] + [-1] * 3 and req.tolist() == [0] * 65 + [2, 2] + [-1] * 3
    cu, slots, req, status = b.plan([1, 130, 0], [1, 0, 0], 131)     # row 0 gives 0, 1 back and takes 1 again
    assert b.table[0, 0] == 1 and b.table[1, :3].tolist() == [0, 3, 4] and status == [0, 1] and b.free == [5]
    before = (list(b.free), b.table.copy(), list(b.length))
    assert b.plan([0, 0, 127], None, 127)[3] == [1, 1] and b.plan([256, 0, 0], None, 255)[3] == [7, 1]
    assert b.plan([0, -1, 0], None, 0)[3] == [8, 1]
    assert before[0] == b.free and (before[1] == b.table).all() and before[2] == b.length


# ---- refusals
P = 4096   # a made-up device pointer


@pytest.fixture(scope="module")
def lib():
    import paper_2502_18137_amd as sp
    return sp.load_library()


def cache(**kw):
    from paper_2502_18137_amd.binding import _Cache
    f = dict(R=2, H_kv=2, d=64, dtype=1, n_pages=10, max_blocks=4, k=P, v=P, k_amax=P, v_amax=P, k_tail=P, v_tail=P, k_tail_amax=P, v_tail_amax=P, table=P, length=P,
             free_pages=P, n_free=P, k_shift=0)
    f.update(kw)
    return ctypes.byref(_Cache(**f))


BAD_SHAPES = [(dict(R=0), -1), (dict(H_kv=0), -1), (dict(n_pages=0), -1), (dict(max_blocks=0), -1), (dict(d=96), -2), (dict(dtype=2), -2),
              (dict(R=4097), -2), (dict(H_kv=129), -2), (dict(n_pages=(1 << 24) + 1), -2), (dict(max_blocks=(1 << 24) + 1), -2)]
BAD_PAGES = [(dict(k=0), -1), (dict(v=0), -1), (dict(k=P + 8), -1), (dict(v=P + 8), -1), (dict(k_amax=0), -1), (dict(v_amax=P + 2), -1),
             (dict(k_shift=P + 4), -1)]


def plan(lib, c=None, new=P, n=3, cu=P, slots=P, req=P, status=P):
    return lib.sparge_cache_plan(cache() if c is None else c, new, None, n, cu, slots, req, status, None)


def append(lib, c=None, K=P, V=P, n=3, s=(128, 64, 128, 64), cu=P, slots=P, req=P):
    return lib.sparge_cache_append(cache() if c is None else c, K, V, n, *s, cu, slots, req, None)


def read(lib, c=None, slots=P, req=P, n=3, dt=2, K=P, V=P):
    return lib.sparge_cache_read(cache() if c is None else c, slots, req, n, dt, K, V, None)


def attn(lib, c=None, Q=P, n=3, H=4, s=(256, 64), cu=P, scale=0.0, O=P, o=(256, 64), ws=P, size=1 << 40):
    return lib.sparge_cache_attn(cache() if c is None else c, Q, n, H, *s, cu, None, scale, 1, O, *o, ws, size, None)


def refused(rc, want, lib):
    assert rc == want and len(lib.sparge_last_error()) > 0, (rc, want, lib.sparge_last_error())


@pytest.mark.parametrize("f", [plan, append, read, attn])
def test_shapes_that_are_refused(lib, f):
    for kw, want in BAD_SHAPES:
        refused(f(lib, cache(**kw)), want, lib)
    refused(f(lib, n=-1), -1, lib)
    refused(f(lib, n=(1 << 30) + 1), -2, lib)


def test_pointers_that_are_refused(lib):
    for kw in (dict(new=0), dict(cu=0), dict(slots=0), dict(req=0), dict(status=0), dict(new=P + 2), dict(cu=P + 1), dict(slots=P + 2),
               dict(req=P + 3), dict(status=P + 2)):
        refused(plan(lib, **kw), -1, lib)
    for kw in (dict(table=0), dict(length=0), dict(free_pages=0), dict(n_free=0), dict(table=P + 2), dict(length=P + 1),
               dict(free_pages=P + 2), dict(n_free=P + 2)):
        refused(plan(lib, cache(**kw)), -1, lib)
    for f in (append, read, attn):
        for kw, want in BAD_PAGES:
            refused(f(lib, cache(**kw)), want, lib)
    for kw in (dict(k_tail=0), dict(v_tail=0), dict(k_tail=P + 8), dict(v_tail=P + 4), dict(k_tail_amax=0), dict(v_tail_amax=0), dict(k_tail_amax=P + 2)):
        refused(append(lib, cache(**kw)), -1, lib)
    for kw in (dict(K=0), dict(V=0), dict(K=P + 8), dict(V=P + 2), dict(cu=0), dict(slots=0), dict(req=0), dict(slots=P + 2),
               dict(s=(-8, 64, 128, 64)), dict(s=(128, 64, 128, 60)), dict(s=(128, 64, 100, 64))):
        refused(append(lib, **kw), -1, lib)
    for kw in (dict(K=0), dict(V=0), dict(K=P + 8), dict(V=P + 4), dict(slots=0), dict(slots=P + 1), dict(req=P + 1)):
        refused(read(lib, **kw), -1, lib)
    refused(read(lib, dt=0), -2, lib)            # fp16 from a bf16 cache
    refused(read(lib, dt=3), -2, lib)
    refused(read(lib, cache(k_shift=P), req=None), -1, lib)
    for kw in (dict(Q=0), dict(O=0), dict(cu=0), dict(Q=P + 8), dict(O=P + 8), dict(cu=P + 2), dict(ws=0), dict(ws=P + 128), dict(H=3), dict(H=0),
               dict(s=(252, 64)), dict(s=(256, -8)), dict(o=(256, 0)), dict(o=(0, 64)), dict(o=(256, 4)), dict(scale=float("inf")),
               dict(scale=float("nan"))):
        refused(attn(lib, **kw), -1, lib)
    refused(attn(lib, H=130), -2, lib)
    refused(attn(lib, cache(length=0)), -1, lib)
    refused(attn(lib, cache(table=0)), -1, lib)
    refused(attn(lib, size=1 << 10), -3, lib)


def test_null_cache(lib):
    for f in (plan, append, read, attn):
        refused(f(lib, ctypes.POINTER(__import__("paper_2502_18137_amd.binding", fromlist=["_Cache"])._Cache)()), -1, lib)
    refused(lib.sparge_cache_attn_workspace_bytes(cache(), 4, None), -1, lib)


def test_workspace_size(lib):
    n = ctypes.c_size_t(0)
    for d in (64, 128):
        assert lib.sparge_cache_attn_workspace_bytes(cache(d=d), 4, ctypes.byref(n)) == 0
        refused(attn(lib, cache(d=d), s=(1024, 128), o=(1024, 128), size=n.value - 1), -3, lib)
        assert n.value <= 100 << 20
    refused(lib.sparge_cache_attn_workspace_bytes(cache(), 5, ctypes.byref(n)), -1, lib)
    refused(lib.sparge_cache_attn_workspace_bytes(cache(), 130, ctypes.byref(n)), -2, lib)


def test_nothing_to_do_is_no_error(lib):
    """no slots: nothing is enqueued, so no GPU is needed"""
    assert append(lib, n=0) == 0 and read(lib, n=0) == 0 and attn(lib, n=0) == 0


def test_the_binding_refuses_a_cache_elsewhere():
    import torch
    import paper_2502_18137_amd as sp
    for kw in (dict(device="cpu"), dict(dtype=torch.float32), dict(head_dim=80), dict(rows=0), dict(n_pages=0), dict(rows=5000)):
        a = dict(rows=1, kv_heads=1, head_dim=64, n_pages=1, max_blocks=1, device="cpu")
        a.update(kw)
        with pytest.raises(sp.SpargeError):
            sp.SpargeCache(**a)
