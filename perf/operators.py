"""The operators of a paged 8-bit K/V cache as timed cases: the step's plan (block table, slot map), the append of new
tokens, the read-back of cached ones, and the attention of new tokens over the cache.

The cache, as all four see it.  R rows (requests); pages of 64 tokens from a pool; row r's block b lies in page
table[r, b].  A page holds, per kv head, the 64 tokens' K and V as 8-bit codes with one scale each:
    amax = max |x| over the block's tokens so far, code = 127 x / amax rounded to nearest, ties to even,
    the value it stands for = code amax / 127 (x = K - shift for K, with the row's shift where there is one).
Plan: rows marked for release push their pages onto the free stack (rows, then blocks ascending) and become empty;
then every row takes the pages that its new tokens need from the top of the stack (the same order).  cu is the prefix
sum of the new tokens, slot = 64 page + offset and req = row for every one of them.
Attention: new token t of a row that holds p tokens sees the keys up to position p + t (all of the row's keys where
the call is not causal), but only in blocks that the mask keeps; G query heads share a kv head; a row of the output
that sees nothing is 0.

Sizes of a case are plain numbers; the rows' lengths follow from them without the seed (`rows`).
"""
import math

import torch

own = False

P = 64  # tokens of a page
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}

# held, new: smallest and largest number of tokens that rows hold and add (spread over the logarithm).  start: "any", or
# "page": held tokens are whole pages, or "inside": the new tokens stay inside the open page (the last two leave a cache
# on which the same append can be repeated).  release: every so many rows, one is given up and used again (0: none).
# shift: K is stored less a per-row shift.  fused: K and V (and Q) lie in one projection's output.  kept: share of the
# blocks that the mask keeps (1: no mask).  out: type that a read gives.  pad: slots behind the last new token.
BASE = dict(op="attn", R=1, Hkv=8, G=4, d=128, dtype="bf16", held=(0, 0), new=(1, 1), start="any", release=0, shift=False,
            fused=False, kept=1.0, causal=True, out="fp32", pad=0)


def _case(**kw):
    c = dict(BASE, **kw)
    for k in ("held", "new"):
        lo, hi = c.pop(k)
        c[k + "_lo"], c[k + "_hi"] = lo, hi
    return c


def listed():
    return [
        # One decoding step's bookkeeping of a small batch: latency alone.
        _case(name="plan_step", op="plan", R=48, held=(100, 9000)),
        # A big server's step: most rows add a token, some are given up and start again with a prompt.
        _case(name="plan_mixed", op="plan", R=1000, held=(64, 16000), new=(1, 512), release=5, pad=100),
        # The append of one decoding step (one token a row), and what was stored.
        _case(name="append_step", op="append", R=128, held=(100, 2000), start="inside"),
        # Ragged prompts of a language model, K less its mean.
        _case(name="append_prompts", op="append", R=5, new=(2500, 16000), start="page", shift=True, fused=True),
        # A later piece of a small model's prompt, head dimension 64.
        _case(name="append_piece", op="append", R=3, Hkv=12, G=1, d=64, dtype="fp16", held=(512, 2048), new=(300, 1100),
              start="page"),
        # A cached prefix for attention over whole tensors; a short fp16 one.
        _case(name="read_prefix", op="read", R=4, held=(9000, 32768), out="16"),
        _case(name="read_short", op="read", R=2, Hkv=4, G=2, d=64, dtype="fp16", held=(70, 1100), shift=True),
        # A lone short request answering token by token: the smallest call.
        _case(name="decode_one", R=1, held=(500, 500)),
        # A decoding batch of ragged lengths, the ordinary serving step, and a large one.
        _case(name="decode_batch", R=64, held=(300, 9000), fused=True),
        _case(name="decode_large", R=160, held=(5000, 32768), pad=3),
        # Four long requests, fp16, under a block mask that keeps 35 % of the blocks.
        _case(name="decode_masked", R=4, Hkv=4, G=8, dtype="fp16", held=(60000, 131072), kept=0.35),
        # Pieces of prompts over what their rows hold already: products count here.
        _case(name="prefill_piece", R=3, held=(4000, 30000), new=(700, 2048), fused=True),
    ]


def _spread(lo, hi, i):
    f = (i * 0.6180339887498949 + 0.5) % 1.0
    return int(round(lo * (hi / lo) ** f)) if lo > 0 else int(round(hi * f))


def rows(c):
    """-> held, new, release: lists of R numbers"""
    held = [_spread(c["held_lo"], c["held_hi"], i) for i in range(c["R"])]
    new = [_spread(c["new_lo"], c["new_hi"], i * 7 + 3) for i in range(c["R"])]
    release = [int(c["release"] > 0 and i % c["release"] == 1) for i in range(c["R"])]
    if c["op"] == "plan" and c["release"]:
        new = [n if x else int(i % 9 != 4) for i, (n, x) in enumerate(zip(new, release))]
    if c["op"] == "read":
        new = [0] * c["R"]
    if c["start"] == "page":
        held = [h // P * P for h in held]
    if c["start"] == "inside":
        held = [h - max(0, h % P + n - P) if h % P else h for h, n in zip(held, new)]
    return held, new, release


def _blocks(n):
    return -(-n // P)


def _loguniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _pair(rng, lo, hi):
    a, b = _loguniform(rng, lo, hi), _loguniform(rng, lo, hi)
    return min(a, b), max(a, b)


def draw(rng):
    """One more case: any operator, type and head layout, up to the largest listed one's cost."""
    op = rng.choice(["plan", "append", "append", "read"] + ["attn"] * 5)
    kw = dict(op=op, R=_loguniform(rng, 1, 256), Hkv=rng.choice([1, 2, 3, 4, 8, 8, 16, 32]), G=rng.choice([1, 2, 4, 4, 5, 7, 8, 16]),
              d=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "fp16"]), shift=rng.random() < 0.4,
              fused=rng.random() < 0.5, held=_pair(rng, 1, 32768))
    while kw["Hkv"] * kw["G"] > 128:
        kw["G"] //= 2
    if op == "plan":
        kw.update(R=_loguniform(rng, 1, 2000), release=rng.choice([0, 3, 10]), new=_pair(rng, 1, 600), pad=rng.choice([0, 37]))
    elif op == "append":
        kw.update(start=rng.choice(["page", "inside"]))
        kw.update(new=_pair(rng, 1, 8000) if kw["start"] == "page" else (1, rng.choice([1, 1, 6])))
    elif op == "read":
        kw.update(out=rng.choice(["fp32", "16"]))
    else:
        kind = rng.choice(["decode", "decode", "few", "piece"])
        kw.update(new={"decode": (1, 1), "few": (1, rng.randint(2, 12)), "piece": _pair(rng, 16, 2048)}[kind], causal=rng.random() < 0.85,
                  kept=rng.choice([1.0, 1.0, 0.3, 0.6]), pad=rng.choice([0, 0, 5]))
        if kind == "decode" and rng.random() < 0.3:
            kw.update(R=rng.randint(1, 4), held=_pair(rng, 4000, 131072))
    c = _case(**kw)
    most = {k: max(work(x)[k] for x in listed()) for k in ("bytes", "flops")}
    tokens = lambda: sum(map(sum, rows(c)[:2])) * c["Hkv"] * c["d"]
    while c["R"] > 1 and (any(work(c)[k] > most[k] for k in most) or tokens() > 2.5e9):
        c["R"] = max(1, c["R"] * 2 // 3)
    if any(work(c)[k] > most[k] for k in most):
        c["new_hi"] = c["new_lo"]
    return c


def _kept(c, row, n_blocks):
    """blocks of a row that the mask keeps, per kv head"""
    return n_blocks if c["kept"] >= 1 else int(round(c["kept"] * n_blocks))


def work(c):
    held, new, release = rows(c)
    T, R, per = sum(new), c["R"], c["Hkv"] * c["d"]
    if c["op"] == "plan":
        start = [0 if x else h for h, x in zip(held, release)]
        popped = sum(_blocks(h + n) - _blocks(h) for h, n in zip(start, new))
        pushed = sum(_blocks(h) for h, x in zip(held, release) if x)
        # lengths, new tokens and marks in, lengths, prefix sums, slots, rows, the pages that change hands
        return {"bytes": 9 * R + 8 * R + 8 * (T + c["pad"]) + 8 * (popped + pushed), "flops": 3 * (R + T)}
    if c["op"] == "append":
        old = sum(h % P for h in held)                       # tokens of the open pages that share their scales with new ones
        return {"bytes": per * (2 * 2 * (T + old) + 2 * (T + old) + 2 * 4 * T), "flops": 2 * per * 4 * (T + old)}
    if c["op"] == "read":
        T = sum(held)
        return {"bytes": 2 * per * T * (1 + (2 if c["out"] == "16" else 4)), "flops": 2 * per * 2 * T}
    keys = pairs = 0
    for h, n in zip(held, new):
        share = _kept(c, 0, _blocks(h + n)) / _blocks(h + n)
        keys += share * (h + n)
        pairs += share * ((h + n) * n - (n * (n - 1) / 2 if c["causal"] else 0))
    return {"bytes": int(2 * per * keys + 2 * 2 * T * c["G"] * per), "flops": int(4 * c["d"] * c["Hkv"] * c["G"] * pairs)}


# ---- inputs --------------------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt * 7919 + 29) % (1 << 62))
    return g


def _tokens(c, seed):
    """K, V of all tokens (a row's held ones, then its new ones; row after row) [n, Hkv, d], the rows' shifts [R, Hkv, d]"""
    held, new, _ = rows(c)
    n, g = sum(held) + sum(new), _gen(seed, 1)
    Hkv, d, dt = c["Hkv"], c["d"], DTYPES[c["dtype"]]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    # keys: channels of different size around a common offset, the first token of a row larger; values: tokens of
    # different size
    offset, size = 0.8 * rnd(Hkv, d), torch.exp(0.3 * rnd(Hkv, d))
    K = torch.empty(n, Hkv, d, dtype=dt, device="cuda")
    V = torch.empty_like(K)
    for a in range(0, n, 1 << 17):
        b = min(n, a + (1 << 17))
        K[a:b] = rnd(b - a, Hkv, d) * size + offset
        V[a:b] = rnd(b - a, Hkv, d) * torch.exp(0.3 * rnd(b - a, 1, 1))
    first = 0
    for h, m in zip(held, new):
        if h + m:
            K[first] *= 3
            V[first] *= 0.1
        first += h + m
    shift = offset + 0.05 * rnd(c["R"], Hkv, d) if c["shift"] else None
    return K, V, shift


def _queries(c, seed):
    T = sum(rows(c)[1]) + c["pad"]
    g = _gen(seed, 2)
    x = torch.randn(T, c["Hkv"] * c["G"], c["d"], generator=g, device="cuda")
    return (1.6 * x).to(DTYPES[c["dtype"]])


def _mask(c, seed):
    """uint8 [R, Hkv, blocks]: the kept blocks of every row and kv head; None: all"""
    if c["kept"] >= 1:
        return None
    held, new, _ = rows(c)
    most, g = _max_blocks(c), _gen(seed, 3)
    mask = torch.zeros(c["R"], c["Hkv"], most, dtype=torch.uint8, device="cuda")
    for r, (h, m) in enumerate(zip(held, new)):
        nb = _blocks(h + m)
        order = torch.rand(c["Hkv"], nb, generator=g, device="cuda").argsort(dim=1)[:, :_kept(c, r, nb)]
        mask[r].scatter_(1, order, 1)
    return mask


def _max_blocks(c):
    held, new, _ = rows(c)
    return max(1, max(_blocks(h + n) for h, n in zip(held, new))) + 1


def _pages(c):
    held, new, _ = rows(c)
    return sum(_blocks(h + n) for h, n in zip(held, new)) + sum(_blocks(n) for n in new) + 7


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _new_rows(c):
    """indices of the new tokens among all tokens"""
    held, new, _ = rows(c)
    at, out = 0, []
    for h, n in zip(held, new):
        out.append(torch.arange(at + h, at + h + n))
        at += h + n
    return torch.cat(out).cuda()


def _held_rows(c):
    held, new, _ = rows(c)
    at, out = 0, []
    for h, n in zip(held, new):
        out.append(torch.arange(at, at + h))
        at += h + n
    return torch.cat(out).cuda()


def _fused(c, x, heads):
    """x [n, heads, d] as a projection leaves it: one part of a wider row"""
    if not c["fused"]:
        return x
    whole = torch.empty(x.shape[0], heads + x.shape[1], x.shape[2], dtype=x.dtype, device="cuda")
    whole[:, heads:] = x
    return whole[:, heads:]


# ---- plain forms: elementary torch operations ------------------------------------------------------------------
class PlainCache:
    def __init__(self, c, shift):
        R, Hkv, d, n = c["R"], c["Hkv"], c["d"], _pages(c)
        dt = DTYPES[c["dtype"]]
        self.length = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.table = torch.full((R, _max_blocks(c)), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
        self.n_free = torch.full((1,), n, dtype=torch.int32, device="cuda")
        if c["op"] != "plan":
            self.codes = torch.zeros(2, n, Hkv, P, d, dtype=torch.int8, device="cuda")
            self.amax = torch.zeros(2, n, Hkv, device="cuda")
            self.tail = torch.zeros(2, R, P, Hkv, d, dtype=dt, device="cuda")
        self.shift = shift


def plain_plan(length, table, free, n_free, new, release, n_slots):
    R, MB = table.shape
    free = torch.cat([free, free.new_zeros(1)])
    n_pages = free.numel() - 1
    before = lambda x: torch.cumsum(x, 0, dtype=torch.int64) - x
    held = torch.where(release != 0, 0, length)
    push = torch.where(release != 0, (length + P - 1) // P, 0)
    b0, b1 = (held + P - 1) // P, (held + new + P - 1) // P
    need, col = b1 - b0, torch.arange(MB, device="cuda")[None]
    short = n_free + push.sum() < need.sum()
    flags = short.int() + 2 * (b1 > MB).any() + 4 * (new.sum() > n_slots)
    ok = flags == 0
    to = torch.where((col < push[:, None]) & ok, n_free + before(push)[:, None] + col, n_pages)
    free2 = free.scatter(0, to.reshape(-1), table.reshape(-1))
    src = (n_free + push.sum() - 1 - before(need)[:, None] - (col - b0[:, None])).clamp(0, n_pages)
    taken = (col >= b0[:, None]) & (col < b1[:, None]) & ok
    table2 = torch.where(taken, free2[src], table)
    left = torch.where(ok, n_free + push.sum() - need.sum(), n_free).int()
    cu = torch.cat([new.new_zeros(1), torch.cumsum(new, 0, dtype=torch.int32)]) * ok.int()
    i = torch.arange(n_slots, dtype=torch.int32, device="cuda")
    r = torch.searchsorted(cu[1:].contiguous(), i, right=True)
    there, r = r < R, r.clamp(max=R - 1)
    pos = (held[r] + i - cu[r]).clamp(min=0)
    slots = torch.where(there, table2[r, (pos // P).clamp(max=MB - 1).long()] * P + pos % P, -1)
    length2 = torch.where(ok, held + new, length)
    return (length2, table2, free2[:-1], left, cu, slots.int(), torch.where(there, r, -1).int(),
            torch.cat([flags.int().reshape(1), left]))


def _touched(held, new):
    """row and number of every page that gets new tokens"""
    pairs = [(r, b) for r, (h, n) in enumerate(zip(held, new)) if n for b in range(h // P, _blocks(h + n))]
    return torch.tensor(pairs, dtype=torch.int64, device="cuda").reshape(-1, 2)


def plain_append(cache, K, V, touched, start, cu, new, update_tail=False):
    """The pages that get new tokens are quantized whole, from the open page's tokens and the new ones."""
    R, n = start.numel(), K.shape[0]
    r, b = touched[:, 0], touched[:, 1]
    pos = b[:, None] * P + torch.arange(P, device="cuda")[None]
    old = pos < start[r][:, None]
    there = pos < (start + new)[r][:, None]
    src = torch.where(old, r[:, None] * P + pos % P, R * P + cu[:-1][r][:, None].long() + pos - start[r][:, None])
    src = torch.where(there, src, R * P + n)
    page = cache.table[r, b].long()
    for which, x in enumerate((K, V)):
        for a in range(0, r.numel(), 1024):
            s = slice(a, a + 1024)
            pool = torch.cat([cache.tail[which].reshape(R * P, *x.shape[1:]), x, x.new_zeros(1, *x.shape[1:])])
            block = pool[src[s]].float()                                        # [pages, 64, Hkv, d]
            if which == 0 and cache.shift is not None:
                block = block - cache.shift[r[s]][:, None]
            block = torch.where(there[s][:, :, None, None], block, 0.0)
            amax = block.abs().amax(dim=(1, 3))
            # 64 bits: 127 x / amax lies on or next to a half often, and its rounding has to be the exact quotient's
            q = 127.0 * block.double() / torch.where(amax > 0, amax, 1.0)[:, None, :, None].double()
            cache.codes[which].index_copy_(0, page[s], torch.round(q).to(torch.int8).transpose(1, 2))
            cache.amax[which].index_copy_(0, page[s], amax)
    if update_tail:
        for row in range(R):
            end = int(start[row] + new[row])
            k = min(end % P, int(new[row]))
            last = int(cu[row + 1])
            for which, x in enumerate((K, V)):
                cache.tail[which, row, end % P - k:end % P] = x[last - k:last]


def plain_read(cache, slots, req, dtype):
    page, at = (slots // P).long(), (slots % P).long()
    out = []
    for which in range(2):
        x = cache.codes[which][page, :, at].float() * cache.amax[which][page][:, :, None] / 127.0
        if which == 0 and cache.shift is not None:
            x = x + cache.shift[req.long()]
        out.append(x.to(dtype))
    return out


def plain_attn(cache, Q, O, held, new, causal, mask):
    Hkv, d = cache.codes.shape[2], cache.codes.shape[4]
    G = Q.shape[1] // Hkv
    at = 0
    for r, (h, n) in enumerate(zip(held, new)):
        page = cache.table[r, :_blocks(h + n)].long()
        q = Q[at:at + n].float().reshape(n, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, n * G, d)
        see = torch.arange(h + n, device="cuda")[None] <= torch.arange(n, device="cuda")[:, None] + (h if causal else h + n)
        see = see[:, None].expand(n, G, h + n).reshape(1, n * G, h + n)
        step = max(1, int(1.5e9) // max(1, (h + n) * max(n * G, d)))           # kv heads at a time
        for a in range(0, Hkv, step):
            heads = slice(a, min(Hkv, a + step))
            k, v = ((cache.codes[w][page][:, heads].float() * (cache.amax[w][page][:, heads] / 127.0)[:, :, None, None])
                    .transpose(0, 1).reshape(-1, page.numel() * P, d)[:, :h + n] for w in range(2))
            s = torch.matmul(q[heads], k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
            seen = see if mask is None else see & (mask[r, heads].repeat_interleave(P, 1)[:, None, :h + n] != 0)
            s = torch.where(seen, s, -math.inf)
            m = s.amax(dim=2, keepdim=True)
            p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
            l = p.sum(dim=2, keepdim=True)
            o = torch.matmul(p, v) / torch.where(l > 0, l, 1.0)
            o = o.reshape(-1, n, G, d).permute(1, 0, 2, 3)
            O[at:at + n].reshape(n, Hkv, G, d)[:, heads] = o.to(O.dtype)
        at += n
    return O


# ---- the cases -------------------------------------------------------------------------------------------------
def prepare(c, seed):
    held, new, release = rows(c)
    R, dt = c["R"], DTYPES[c["dtype"]]
    s = dict(case=c, held=held, new=new, new_len=_i32(new), start=_i32(held), zero=_i32([0] * R), T=sum(new),
             release=torch.tensor(release, dtype=torch.uint8, device="cuda"))
    K = V = shift = None
    if c["op"] != "plan":
        K, V, shift = _tokens(c, seed)
    plain = PlainCache(c, shift)
    # a pool in use: the free pages in no order
    n = _pages(c)
    plain.free = torch.randperm(n, generator=_gen(seed, 4), device="cuda").int()
    fill = _i32(held)
    if own:
        import paper_2502_18137_amd as sp
        cache = sp.SpargeCache(R, c["Hkv"], c["d"], n, _max_blocks(c), dtype=dt, device="cuda", k_shift=shift)
        cache.free_pages.copy_(plain.free)
        s["cache"], s["sp"] = cache, sp
        first = sp.sparge_cache_plan(cache, fill, sum(held))
        if c["op"] != "plan" and sum(held):
            i = _held_rows(c)
            sp.sparge_cache_append(cache, K[i], V[i], first)
        if c["op"] in ("append", "attn"):
            s["plan"] = sp.sparge_cache_plan(cache, s["new_len"], s["T"] + c["pad"])
        if c["op"] == "plan":
            s["book"] = cache.book.clone()
    else:
        (plain.length, plain.table, plain.free, plain.n_free, cu, slots, req, _) = plain_plan(
            plain.length, plain.table, plain.free, plain.n_free, fill, torch.zeros_like(s["release"]), sum(held))
        if c["op"] != "plan" and sum(held):
            i = _held_rows(c)
            plain_append(plain, K[i], V[i], _touched([0] * R, held), s["zero"], cu, fill, update_tail=True)
        if c["op"] in ("append", "attn"):
            (plain.length, plain.table, plain.free, plain.n_free, s["cu"], s["slots"], s["req"], _) = plain_plan(
                plain.length, plain.table, plain.free, plain.n_free, s["new_len"], torch.zeros_like(s["release"]), s["T"])
        s["cache"] = plain
    cache = s["cache"]
    if c["op"] == "append":
        i = _new_rows(c)
        heads = c["Hkv"] * c["G"]
        s["K"], s["V"] = _fused(c, K[i], heads), _fused(c, V[i], heads + c["Hkv"])
    if c["op"] == "read":
        row = torch.repeat_interleave(torch.arange(R), torch.tensor(held)).cuda()
        pos = torch.cat([torch.arange(h) for h in held]).cuda()
        s["slots"], s["req"] = (cache.table[row, pos // P] * P + pos % P).int(), row.int()
        s["out"] = torch.float32 if c["out"] == "fp32" else dt
    if c["op"] == "attn":
        if s["T"]:
            i = _new_rows(c)
            if own:
                sp.sparge_cache_append(cache, torch.cat([K[i], K[:c["pad"]]]), torch.cat([V[i], V[:c["pad"]]]), s["plan"])
            else:
                plain_append(plain, K[i], V[i], _touched(held, new), s["start"], s["cu"], s["new_len"])
        s["Q"], s["mask"] = _fused(c, _queries(c, seed), 2 * c["Hkv"]), _mask(c, seed)
        s["O"] = torch.zeros(s["Q"].shape, dtype=dt, device="cuda")
        if own:
            s["ws"] = torch.empty(sp.sparge_cache_attn_workspace_bytes(cache, s["Q"].shape[1]), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    c, cache = s["case"], s["cache"]
    if own:
        sp = s["sp"]
        if c["op"] == "plan":
            cache.book.copy_(s["book"])          # the bookkeeping of before the step, so that the pass can be repeated
            p = sp.sparge_cache_plan(cache, s["new_len"], s["T"] + c["pad"], release=s["release"])
            return cache.length, cache.table, cache.free_pages, cache.n_free, p.cu, p.slots, p.req, p.status
        if c["op"] == "append":
            sp.sparge_cache_append(cache, s["K"], s["V"], s["plan"])
            return sp.sparge_cache_read(cache, s["plan"].slots, s["plan"].req, dtype=torch.float32) + (cache.k_amax, cache.v_amax)
        if c["op"] == "read":
            return sp.sparge_cache_read(cache, s["slots"], s["req"], dtype=s["out"])
        return sp.sparge_cache_attn(cache, s["Q"], s["plan"], causal=c["causal"], mask=s["mask"], ws=s["ws"], out=s["O"])
    if c["op"] == "plan":
        return plain_plan(cache.length, cache.table, cache.free, cache.n_free, s["new_len"], s["release"], s["T"] + c["pad"])
    if c["op"] == "append":
        plain_append(cache, s["K"], s["V"], _touched(s["held"], s["new"]), s["start"], s["cu"], s["new_len"])
        return tuple(plain_read(cache, s["slots"], s["req"], torch.float32)) + (cache.amax[0], cache.amax[1])
    if c["op"] == "read":
        return tuple(plain_read(cache, s["slots"], s["req"], s["out"]))
    return plain_attn(cache, s["Q"], s["O"], s["held"], s["new"], c["causal"], s["mask"])


# ---- 64 bits, from the definitions, page by page of each row's tokens ------------------------------------------
def _stored(x, shift):
    """[n, Hkv, d] of one row from its first token on -> the values its codes stand for (fp64, without the shift), the
    pages' amax"""
    y = x.float() if shift is None else x.float() - shift
    n = y.shape[0]
    y = torch.cat([y.double(), torch.zeros(-n % P, *y.shape[1:], dtype=torch.float64, device=y.device)])
    y = y.reshape(-1, P, *y.shape[1:])
    top = y.abs().flatten(3).amax(dim=(1, 3), keepdim=True)
    step = top / 127
    # the quotient as 127 y / top: two roundings fewer than y / step, exact on halves
    code = torch.where(top > 0, 127 * y / torch.where(top > 0, top, 1.0), 0.0).round()
    return (code * step).reshape(-1, *y.shape[2:])[:n], top.reshape(top.shape[0], -1)


def exact(c, seed):
    held, new, _ = rows(c)
    if c["op"] == "plan":
        return None
    K, V, shift = _tokens(c, seed)
    starts = [0]
    for h, n in zip(held, new):
        starts.append(starts[-1] + h + n)
    if c["op"] != "attn":
        ks, vs, tops = [], [], torch.zeros(2, _pages(c), c["Hkv"], dtype=torch.float64, device="cuda")
        # pages in the order in which they are taken: the held blocks of all rows, then the new ones
        pages = torch.randperm(_pages(c), generator=_gen(seed, 4), device="cuda").flip(0).split(
            [_blocks(h) for h in held] + [_blocks(h + n) - _blocks(h) for h, n in zip(held, new)] + [_pages(c) - sum(
                _blocks(h + n) for h, n in zip(held, new))])
        for r, (h, n) in enumerate(zip(held, new)):
            sh = None if shift is None else shift[r]
            rows_ = slice(starts[r], starts[r] + h + n)
            first = h if c["op"] == "append" else 0
            (k, top_k), (v, top_v) = _stored(K[rows_], sh), _stored(V[rows_], None)
            at = torch.cat([pages[r], pages[c["R"] + r]])
            tops[0, at], tops[1, at] = top_k, top_v
            if sh is not None:
                k = k + sh.double()
            ks.append(k[first:])
            vs.append(v[first:])
        return [torch.cat(ks), torch.cat(vs)] + list(tops) * (c["op"] == "append")
    Q, mask = _queries(c, seed), _mask(c, seed)
    out = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    at = 0
    for r, (h, n) in enumerate(zip(held, new)):
        rows_ = slice(starts[r], starts[r] + h + n)
        k = _stored(K[rows_], None if shift is None else shift[r])[0]
        v = _stored(V[rows_], None)[0]
        key = torch.arange(h + n, device="cuda")
        for x in range(c["Hkv"] * c["G"]):
            kv = x // c["G"]
            for a in range(0, n, 512):
                b = min(n, a + 512)
                z = (Q[at + a:at + b, x].double() @ k[:, kv].T.contiguous()) / math.sqrt(c["d"])
                hidden = torch.zeros(b - a, h + n, dtype=torch.bool, device="cuda")
                if c["causal"]:
                    hidden |= key[None] > torch.arange(h + a, h + b, device="cuda")[:, None]
                if mask is not None:
                    hidden |= (mask[r, kv][key // P] == 0)[None]
                z = z.masked_fill(hidden, -math.inf)
                w = torch.exp(z - z.amax(dim=1, keepdim=True).clamp(min=-1e300))
                out[at + a:at + b, x] = (w @ v[:, kv].contiguous()) / w.sum(dim=1, keepdim=True).clamp(min=1e-300)
        at += n
    return out
