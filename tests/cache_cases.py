"""Shared by the tests of the paged 8-bit cache: a cache under test with the tokens and the book that the oracle keeps."""
import numpy as np

from oracle import cache_oracle as co

U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a step, relative


class Model:
    """A cache on the GPU, the same steps in the oracle, all tokens of all rows."""

    def __init__(self, sp, rows, Hkv, d, n_pages, max_blocks, dtype="bf16", seed=0, shift=False, free=None):
        import torch
        self.sp, self.torch, self.dt = sp, torch, torch.float16 if dtype == "fp16" else torch.bfloat16
        self.rng = np.random.default_rng(seed)
        self.R, self.Hkv, self.d, self.dtype = rows, Hkv, d, dtype
        self.shift = self.rng.normal(size=(rows, Hkv, d)).astype(np.float32) if shift else None
        self.cache = sp.SpargeCache(rows, Hkv, d, n_pages, max_blocks, dtype=self.dt,
                                    k_shift=None if self.shift is None else torch.from_numpy(self.shift).cuda())
        self.book = co.Book(rows, n_pages, max_blocks, free)
        if free is not None:
            self.cache.free_pages.copy_(torch.tensor(free, dtype=torch.int32))
        self.K = [np.zeros((0, Hkv, d)) for _ in range(rows)]
        self.V = [np.zeros((0, Hkv, d)) for _ in range(rows)]

    def i32(self, x):
        return self.torch.tensor(x, dtype=self.torch.int32, device="cuda")

    def tokens(self, n):
        """K, V [n, Hkv, d], fp64 arrays of 16-bit values"""
        x = self.torch.from_numpy(self.rng.normal(size=(2, n, self.Hkv, self.d)) * np.exp(0.5 * self.rng.normal(size=(2, n, 1, 1))))
        return self.round16(x[0].numpy()), self.round16(x[1].numpy())

    def round16(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).to(self.dt).double().numpy()

    def gpu(self, x, pad=0, fused=0):
        """pad rows of NaN behind, `fused` columns of other data in front of every token's heads"""
        t = self.torch.from_numpy(np.ascontiguousarray(x)).to("cuda", self.dt)
        big = self.torch.full((t.shape[0] + pad, t.shape[1] + fused, t.shape[2]), float("nan"), dtype=self.dt, device="cuda")
        big[:t.shape[0], fused:] = t
        return big[:, fused:]

    def step(self, new, release=None, pad=0, fused=0, tokens=None, check=True):
        """plan and append of new[r] tokens per row -> the plan"""
        n = sum(new)
        plan = self.sp.sparge_cache_plan(self.cache, self.i32(new), n + pad, None if release is None else
                                         self.torch.tensor(release, dtype=self.torch.uint8, device="cuda"))
        cu, slots, req, status = self.book.plan(list(new), release, n + pad)
        if check:
            for name, want in (("cu", cu), ("slots", slots), ("req", req), ("status", np.array(status))):
                assert np.array_equal(getattr(plan, name).cpu().numpy(), want), (name, getattr(plan, name), want)
            assert self.cache.length.tolist() == self.book.length
            free = self.cache.free_pages.tolist()[:int(self.cache.n_free)]
            assert free == self.book.free
            for r, length in enumerate(self.book.length):
                nb = -(-length // 64)
                assert self.cache.table[r, :nb].tolist() == self.book.table[r, :nb].tolist()
        assert status[0] == 0
        K, V = self.tokens(n) if tokens is None else tokens
        self.sp.sparge_cache_append(self.cache, self.gpu(K, pad, fused), self.gpu(V, pad, fused), plan)
        at = 0
        for r in range(self.R):
            if release is not None and release[r]:
                self.K[r], self.V[r] = self.K[r][:0], self.V[r][:0]
            self.K[r] = np.concatenate([self.K[r], K[at:at + new[r]]])
            self.V[r] = np.concatenate([self.V[r], V[at:at + new[r]]])
            at += new[r]
        self.new = list(new)
        return plan

    def stored(self, r):
        """the values that the oracle's codes of row r stand for, K (without the shift), V, amax of both"""
        ck, ak = co.quantize_tokens(self.K[r], None if self.shift is None else self.shift[r])
        cv, av = co.quantize_tokens(self.V[r])
        return co.values(ck, ak), co.values(cv, av), ak, av

    def check_stored(self):
        """every code and scale of every row"""
        for r in range(self.R):
            n = len(self.K[r])
            if n == 0:
                continue
            t = np.arange(n)
            slots = self.book.table[r, t // 64] * 64 + t % 64
            k, v = self.sp.sparge_cache_read(self.cache, self.i32(slots), self.i32([r] * n), dtype=self.torch.float32)
            wk, wv, ak, av = self.stored(r)
            if self.shift is not None:
                wk = wk + self.shift[r]
            assert np.array_equal(k.cpu().numpy(), wk.astype(np.float32), equal_nan=True), r
            assert np.array_equal(v.cpu().numpy(), wv.astype(np.float32), equal_nan=True), r
            pages = self.book.table[r, :len(ak)]
            assert np.array_equal(self.cache.k_amax.cpu().numpy()[pages], ak, equal_nan=True)
            assert np.array_equal(self.cache.v_amax.cpu().numpy()[pages], av, equal_nan=True)

    def queries(self, H, size=1.5):
        return self.round16(self.rng.normal(size=(sum(self.new), H, self.d)) * size)

    def check_attn(self, plan, H, causal=True, mask=None, scale=0.0, q=None, pad=0, fused=0):
        """O against the oracle on the stored values, element by element.

        What the kernel may add: the weights' rounding to fp16 (half a step, 2^-11 of each; below fp16's normal range 2^-33 of
        the largest, per key), products and sums in fp32 (a dot product of d terms is off by at most d 2^-24 of its absolute
        sum, exp2's argument by a few 2^-24 of it; the sums over n keys by n 2^-24 in the worst case, which no row comes
        near, sqrt(n) 2^-24 being typical: 64 2^-24 is taken), Q's power of two (2^-24 of the row's largest per
        element: inside the doubled constant), and the output's rounding, half a step."""
        q = self.queries(H) if q is None else q
        u = U[self.dtype]
        sentinel = 7.25
        out = self.torch.full((sum(self.new) + pad, H, self.d), sentinel, dtype=self.dt, device="cuda")
        m = None if mask is None else self.torch.from_numpy(mask).cuda()
        got = self.sp.sparge_cache_attn(self.cache, self.gpu(q, pad, fused), plan, causal=causal, mask=m, sm_scale=scale, out=out)
        got = got.double().cpu().numpy()
        assert (got[sum(self.new):] == sentinel).all(), "rows behind the last token were written"
        at, worst = 0, 0.0
        for r in range(self.R):
            n = self.new[r]
            if n == 0:
                continue
            k, v, _, _ = self.stored(r)
            O, A, S = co.attend(q[at:at + n], k, v, len(k) - n, causal, None if mask is None else mask[r], scale or None)
            exp = 2.0 ** -23 * (self.d + 8) * S
            tol = u * np.abs(O) + 1.02 * (2.0 ** -11 + 64 * 2.0 ** -24 + exp[:, :, None]) * A + len(k) * 2.0 ** -33 * np.abs(v).max(initial=0)
            tol = tol + 2.0 ** -25        # fp16 outputs below the normal range
            ratio = np.abs(got[at:at + n] - O) / tol
            assert ratio.max() <= 1.0, (r, ratio.max(), np.unravel_index(ratio.argmax(), ratio.shape))
            worst = max(worst, ratio.max())
            at += n
        return got, worst
