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
