// Paged 8-bit K/V cache: the step's plan (pages, block table, slot map), the append of new tokens and the read-back.
#include "cache.hpp"

namespace sparge {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int FILL_IN_PLAN = 8 * PLAN_THREADS;   // slots that the plan's one workgroup fills itself

__device__ __forceinline__ int blocks_of(int tokens) { return (tokens + PAGE - 1) / PAGE; }

// the last index r < n with prefix[r] <= a (prefix ascending from 0; entries of equal value: the last of them, which is the
// one that holds something)
__device__ __forceinline__ int row_of(const int* prefix, int n, int a) {
    int lo = 0, hi = n;   // prefix[lo] <= a, hi: beyond
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= a) lo = mid; else hi = mid;
    }
    return lo;
}

struct Sums {
    long long push, need, tok;
};

// exclusive prefix of v over the workgroup's threads, and the total; lds: a Sums per wave
__device__ Sums scan(Sums v, Sums* lds, Sums& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums x = v;
    for (int s = 1; s < 64; s <<= 1) {
        const long long a = __shfl_up(x.push, s), b = __shfl_up(x.need, s), c = __shfl_up(x.tok, s);
        if (lane >= s) x.push += a, x.need += b, x.tok += c;
    }
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    Sums before = {0, 0, 0};
    total = {0, 0, 0};
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        if (w == wave) before = total;
        total.push += lds[w].push, total.need += lds[w].need, total.tok += lds[w].tok;
    }
    return {before.push + x.push - v.push, before.need + x.need - v.need, before.tok + x.tok - v.tok};
}

__device__ __forceinline__ void fill_slot(const sparge_cache& c, const int* cu, int total, int i, const int* held, int32_t* slots,
                                          int32_t* req) {
    int slot = -1, r = -1;
    if (i < total) {
        r = row_of(cu, c.R, i);
        const int pos = held[r] + i - cu[r];
        slot = c.table[static_cast<long long>(r) * c.max_blocks + pos / PAGE] * PAGE + pos % PAGE;
    }
    slots[i] = slot;
    req[i] = r;
}

// One workgroup.  Lengths and new tokens are summed over the rows, everything is checked, and only then is anything changed.
// What bounds it is a chain of four round trips to memory (lengths; the pages that rows give up; the pages that rows take;
// the table entries that slots are made of), so rows, pages and slots are spread over the threads through the prefix sums.
__global__ __launch_bounds__(PLAN_THREADS) void cache_plan_kernel(sparge_cache c, const int32_t* __restrict__ new_len,
                                                                  const uint8_t* __restrict__ release, int n_slots, int32_t* cu,
                                                                  int32_t* slots, int32_t* req, int32_t* status) {
    extern __shared__ int lds[];
    int* push_at = lds;                 // prefix sums over the rows; then the rows' held tokens
    int* need_at = lds + c.R;
    int* tok_at = lds + 2 * c.R;
    __shared__ Sums wave_sums[PLAN_THREADS / 64];
    __shared__ int wave_flags[PLAN_THREADS / 64];
    const int tid = threadIdx.x;
    const int per = (c.R + PLAN_THREADS - 1) / PLAN_THREADS;
    const int r0 = tid * per, r1 = min(r0 + per, c.R);
    const long long most = static_cast<long long>(c.max_blocks) * PAGE;
    Sums mine = {0, 0, 0};
    int flags = 0;
    const int n_free = c.n_free[0];
    if (n_free < 0 || n_free > c.n_pages) flags = SPARGE_CACHE_BAD_STATE;
    for (int r = r0; r < r1; ++r) {
        const int len = c.length[r], n = new_len[r];
        const bool rel = release && release[r];
        if (len < 0 || len > most || n < 0) flags |= SPARGE_CACHE_BAD_STATE;
        const long long held = rel ? 0 : len;
        if (held + n > most) flags |= SPARGE_CACHE_ROW_FULL;
        mine.push += rel ? blocks_of(len) : 0;
        mine.need += (held + n + PAGE - 1) / PAGE - (held + PAGE - 1) / PAGE;
        mine.tok += n;
    }
    Sums total;
    Sums at = scan(mine, wave_sums, total);
    for (int s = 1; s < 64; s <<= 1) flags |= __shfl_xor(flags, s);
    if ((tid & 63) == 0) wave_flags[tid >> 6] = flags;
    __syncthreads();
    for (int w = 0; w < PLAN_THREADS / 64; ++w) flags |= wave_flags[w];
    if (n_free + total.push > c.n_pages) flags |= SPARGE_CACHE_BAD_STATE;
    if (n_free + total.push < total.need) flags |= SPARGE_CACHE_NO_PAGES;
    if (total.tok > n_slots) flags |= SPARGE_CACHE_NO_SLOTS;
    if (flags & SPARGE_CACHE_BAD_STATE) flags = SPARGE_CACHE_BAD_STATE;   // the other sums mean nothing then
    if (flags) {
        for (int r = tid; r <= c.R; r += PLAN_THREADS) cu[r] = 0;
        if (n_slots <= FILL_IN_PLAN)
            for (int i = tid; i < n_slots; i += PLAN_THREADS) slots[i] = req[i] = -1;
        if (tid == 0) status[0] = flags, status[1] = n_free;
        return;
    }
    for (int r = r0; r < r1; ++r) {
        push_at[r] = static_cast<int>(at.push), need_at[r] = static_cast<int>(at.need), tok_at[r] = static_cast<int>(at.tok);
        cu[r] = static_cast<int>(at.tok);
        const int len = c.length[r], n = new_len[r];
        const bool rel = release && release[r];
        const int held = rel ? 0 : len;
        at.push += rel ? blocks_of(len) : 0;
        at.need += blocks_of(held + n) - blocks_of(held);
        at.tok += n;
    }
    __syncthreads();
    const int pushed = static_cast<int>(total.push), needed = static_cast<int>(total.need), tokens = static_cast<int>(total.tok);
    for (int a = tid; a < pushed; a += PLAN_THREADS) {
        const int r = row_of(push_at, c.R, a);
        c.free_pages[n_free + a] = c.table[static_cast<long long>(r) * c.max_blocks + a - push_at[r]];
    }
    __syncthreads();
    for (int r = r0; r < r1; ++r) {
        const int held = release && release[r] ? 0 : c.length[r];
        push_at[r] = held;
        c.length[r] = held + new_len[r];
    }
    __syncthreads();
    for (int a = tid; a < needed; a += PLAN_THREADS) {
        const int r = row_of(need_at, c.R, a);
        c.table[static_cast<long long>(r) * c.max_blocks + blocks_of(push_at[r]) + a - need_at[r]] =
            c.free_pages[n_free + pushed - 1 - a];
    }
    if (tid == 0) {
        cu[c.R] = tokens;
        c.n_free[0] = n_free + pushed - needed;
        status[0] = 0, status[1] = n_free + pushed - needed;
    }
    if (n_slots > FILL_IN_PLAN) return;
    __syncthreads();
    for (int i = tid; i < n_slots; i += PLAN_THREADS) fill_slot(c, tok_at, tokens, i, push_at, slots, req);
}

// The slot map of a long step, from what the plan has written; a workgroup per 2048 slots.
constexpr int FILL_SLOTS = 2048;
__global__ __launch_bounds__(256) void cache_slots_kernel(sparge_cache c, int n_slots, const int32_t* __restrict__ cu,
                                                          int32_t* slots, int32_t* req) {
    extern __shared__ int lds[];
    int* held = lds + c.R;
    const int total = min(cu[c.R], n_slots);
    for (int r = threadIdx.x; r < c.R; r += 256) {
        lds[r] = cu[r];
        held[r] = c.length[r] - (cu[r + 1] - cu[r]);
    }
    __syncthreads();
    for (int i = blockIdx.x * FILL_SLOTS + threadIdx.x; i < min(n_slots, (static_cast<int>(blockIdx.x) + 1) * FILL_SLOTS); i += 256)
        fill_slot(c, lds, total, i, held, slots, req);
}

// ---- append ------------------------------------------------------------------------------------------------------

// 127 x / amax rounded to the nearest integer, halves to even, of the exact quotient: amax scaled to [1, 2) and x with it
// (exact; what underflows is far below a half), the quotient's floor f from an approximation, and the sign of
// 127 x - (f + 1/2) amax, whose product is split into its rounded value and the rest.  Where the approximation puts f on
// the wrong side of an integer the sign still gives that integer.
__device__ __forceinline__ int code_of(float x, int up, float amax1, float r) {
    const float y = __builtin_ldexpf(x, up);
    const float f = floorf(y * r);
    const float h = f + 0.5f, p = h * amax1, rest = __builtin_fmaf(h, amax1, -p);
    const float over = __builtin_fmaf(127.0f, y, -p) - rest;
    const int i = static_cast<int>(f);
    return i + ((over > 0.f || (over == 0.f && (i & 1))) ? 1 : 0);
}

// A workgroup quantizes one kv head's K or V of every page that begins to get tokens inside its window of `window` (a power of two up to
// 64) slots: the open page's older tokens from the tail, the new ones from the call's tensor.  The amax is taken over the
// bit patterns, so that a NaN or an infinity is the largest.  The row's first page also stores the tokens of the row's last
// page if that stays open (after it has read the older ones, which lie in the same place).
template <int D, int DT>
__global__ __launch_bounds__(256) void cache_append_kernel(sparge_cache c, const uint16_t* __restrict__ K,
                                                           const uint16_t* __restrict__ V, int n_slots, int window, long long k_sn,
                                                           long long k_sh, long long v_sn, long long v_sh,
                                                           const int32_t* __restrict__ cu, const int32_t* __restrict__ slots,
                                                           const int32_t* __restrict__ req) {
    constexpr int LPR = D / 8, RPS = 256 / LPR, NL = PAGE / RPS;   // lanes per row, rows a step, steps
    __shared__ __align__(16) uint8_t codes[PAGE * D];
    __shared__ uint32_t wave_amax[4];
    const int tid = threadIdx.x, lane = tid & 63, hk = blockIdx.y;
    const bool is_v = blockIdx.z != 0;
    const uint16_t* x = is_v ? V + hk * v_sh : K + hk * k_sh;
    const long long sn = is_v ? v_sn : k_sn;
    uint16_t* tails = static_cast<uint16_t*>(is_v ? c.v_tail : c.k_tail);
    uint8_t* pages = static_cast<uint8_t*>(is_v ? c.v : c.k);
    float* amaxes = is_v ? c.v_amax : c.k_amax;
    const float* shifts = is_v ? nullptr : c.k_shift;

    const int i0 = blockIdx.x * window;
    int my_slot = -1, my_row = -1, my_prev = -1;
    if (lane < window && i0 + lane < n_slots) {
        my_slot = slots[i0 + lane];
        my_row = req[i0 + lane];
        my_prev = i0 + lane ? req[i0 + lane - 1] : -1;
    }
    const bool there = my_slot >= 0 && my_slot / PAGE < c.n_pages && my_row >= 0 && my_row < c.R;
    unsigned long long starts = __ballot(there && (my_slot % PAGE == 0 || my_prev != my_row));
    const int col = (tid % LPR) * 8, row0 = tid / LPR;
    while (starts) {
        const int first = __builtin_ctzll(starts);
        starts &= starts - 1;
        const int i = i0 + first;
        const int slot = __builtin_amdgcn_readlane(my_slot, first), r = __builtin_amdgcn_readlane(my_row, first);
        const int page = slot / PAGE, off = slot % PAGE;
        const int row_begin = max(0, min(cu[r], n_slots)), row_end = max(0, min(cu[r + 1], n_slots));
        const int n = max(1, min(PAGE - off, row_end - i));
        uint16_t* tail = tails + (static_cast<long long>(r) * c.H_kv + hk) * PAGE * D;
        float y[NL][8];
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < NL; ++s) {
            const int t = s * RPS + row0;
            uint4 raw = make_uint4(0u, 0u, 0u, 0u);
            if (t < off) raw = *reinterpret_cast<const uint4*>(tail + t * D + col);
            else if (t < off + n) raw = *reinterpret_cast<const uint4*>(x + (i + t - off) * sn + col);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[s][2 * e] = cvt16<DT>(static_cast<uint16_t>(w[e] & 0xFFFFu));
                y[s][2 * e + 1] = cvt16<DT>(static_cast<uint16_t>(w[e] >> 16));
            }
        }
        if (shifts) {
            const float* sh = shifts + (static_cast<long long>(r) * c.H_kv + hk) * D + col;
#pragma unroll
            for (int s = 0; s < NL; ++s)
                if (s * RPS + row0 < off + n)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[s][e] -= sh[e];
        }
#pragma unroll
        for (int s = 0; s < NL; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[s][e]) & 0x7FFFFFFFu);
        for (int s = 1; s < 64; s <<= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), s)));
        if (lane == 0) wave_amax[tid >> 6] = top;
        __syncthreads();   // (the tail's older tokens are read, too)
        top = max(max(wave_amax[0], wave_amax[1]), max(wave_amax[2], wave_amax[3]));
        const bool plain = top > 0 && top < 0x7F800000u;   // a block with an infinity or a NaN has codes 0
        int up = 1;
        const float amax = __uint_as_float(top);
        if (plain) up = 1 - __builtin_amdgcn_frexp_expf(amax);
        const float amax1 = plain ? __builtin_ldexpf(amax, up) : 1.0f, inv = 127.0f / amax1;
#pragma unroll
        for (int s = 0; s < NL; ++s) {
            const int t = s * RPS + row0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int code = plain ? code_of(y[s][e], up, amax1, inv) : 0;
                codes[is_v ? v_byte(t, col + e) : k_byte(t, col + e, D)] = static_cast<uint8_t>(code + 128);
            }
        }
        if (i == row_begin) {   // the tokens of the row's last page, if it stays open
            const int last = row_end > 0 ? slots[row_end - 1] : -1;
            const int open = last >= 0 ? (last % PAGE + 1) % PAGE : 0;
            const int keep = min(open, row_end - row_begin);
            for (int t = open - keep + row0; t < open; t += RPS)
                *reinterpret_cast<uint4*>(tail + t * D + col) = *reinterpret_cast<const uint4*>(x + (row_end - open + t) * sn + col);
        }
        __syncthreads();
        const long long at = static_cast<long long>(page) * c.H_kv + hk;
        for (int b = tid; b < PAGE * D / 16; b += 256)
            reinterpret_cast<uint4*>(pages + at * PAGE * D)[b] = reinterpret_cast<const uint4*>(codes)[b];
        if (tid == 0) amaxes[at] = amax;
        __syncthreads();   // the next page uses the LDS again
    }
}

// ---- read-back ---------------------------------------------------------------------------------------------------

// value = code amax / 127 (+ shift), in 64 bits and rounded once to fp32, then to 16 bits where asked for.  A thread gives 16
// channels of one token of one kv head, K (blockIdx.z 0) or V.
template <int D, int OUT>
__global__ __launch_bounds__(256) void cache_read_kernel(sparge_cache c, const int32_t* __restrict__ slots,
                                                         const int32_t* __restrict__ req, int n_slots, void* K, void* V) {
    constexpr int TPT = D / 16, TOK = 256 / TPT;   // threads per token, tokens per workgroup
    const int hk = blockIdx.y, i = blockIdx.x * TOK + threadIdx.x / TPT, ch = (threadIdx.x % TPT) * 16;
    const bool is_v = blockIdx.z != 0;
    if (i >= n_slots) return;
    const int slot = slots[i], r = req ? req[i] : 0;
    if (slot < 0 || slot / PAGE >= c.n_pages || r < 0 || r >= c.R) return;
    const int page = slot / PAGE, key = slot % PAGE;
    const long long at = static_cast<long long>(page) * c.H_kv + hk;
    const uint8_t* p = static_cast<const uint8_t*>(is_v ? c.v : c.k) + at * PAGE * D;
    uint8_t b[16];
    if (is_v) {
#pragma unroll
        for (int e = 0; e < 16; ++e) b[e] = p[v_byte(key, ch + e)];
    } else {
        const uint4 w = *reinterpret_cast<const uint4*>(p + k_byte(key, ch, D));
        __builtin_memcpy(b, &w, 16);
    }
    const double step = static_cast<double>((is_v ? c.v_amax : c.k_amax)[at]) / 127.0;
    const float* sh = !is_v && c.k_shift ? c.k_shift + (static_cast<long long>(r) * c.H_kv + hk) * D + ch : nullptr;
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        double v = static_cast<double>(static_cast<int>(b[e]) - 128) * step;
        if (sh) v += static_cast<double>(sh[e]);
        y[e] = static_cast<float>(v);
    }
    const long long o = (static_cast<long long>(i) * c.H_kv + hk) * D + ch;
    void* out = is_v ? V : K;
    if constexpr (OUT == SPARGE_F32) {
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(static_cast<float*>(out) + o + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
    } else {
        uint16_t h[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) h[e] = cvt_to16<OUT>(y[e]);
        uint4 w[2];
        __builtin_memcpy(w, h, 32);
        reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + o)[0] = w[0];
        reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + o)[1] = w[1];
    }
}

}  // namespace

hipError_t launch_cache_plan(const sparge_cache& c, const int32_t* new_len, const uint8_t* release, int n_slots, int32_t* cu,
                             int32_t* slots, int32_t* req, int32_t* status, hipStream_t st) {
    hipLaunchKernelGGL(cache_plan_kernel, dim3(1), dim3(PLAN_THREADS), 3 * c.R * sizeof(int), st, c, new_len, release, n_slots, cu,
                       slots, req, status);
    if (n_slots > FILL_IN_PLAN)
        hipLaunchKernelGGL(cache_slots_kernel, dim3((n_slots + FILL_SLOTS - 1) / FILL_SLOTS), dim3(256), 2 * c.R * sizeof(int), st, c,
                           n_slots, cu, slots, req);
    return hipGetLastError();
}

hipError_t launch_cache_append(const sparge_cache& c, const void* K, const void* V, int n_slots, long long k_sn, long long k_sh,
                               long long v_sn, long long v_sh, const int32_t* cu, const int32_t* slots, const int32_t* req,
                               hipStream_t st) {
    // a window per page where a step has that many, down to one per slot (each of which may be a page of its own) where there
    // are few: a workgroup quantizes its window's pages one after the other
    int window = 64;
    while (window > 1 && static_cast<long long>(n_slots / window) * c.H_kv < 4096) window /= 2;
    const dim3 grid((n_slots + window - 1) / window, c.H_kv, 2);
    const uint16_t *k = static_cast<const uint16_t*>(K), *v = static_cast<const uint16_t*>(V);
#define APPEND(D, DT) \
    hipLaunchKernelGGL((cache_append_kernel<D, DT>), grid, dim3(256), 0, st, c, k, v, n_slots, window, k_sn, k_sh, v_sn, v_sh, cu, slots, req)
    if (c.d == 64) {
        if (c.dtype == SPARGE_F16) APPEND(64, SPARGE_F16); else APPEND(64, SPARGE_BF16);
    } else {
        if (c.dtype == SPARGE_F16) APPEND(128, SPARGE_F16); else APPEND(128, SPARGE_BF16);
    }
#undef APPEND
    return hipGetLastError();
}

hipError_t launch_cache_read(const sparge_cache& c, const int32_t* slots, const int32_t* req, int n_slots, int out_dtype, void* K,
                             void* V, hipStream_t st) {
    const int tok = 256 / (c.d / 16);
    const dim3 grid((n_slots + tok - 1) / tok, c.H_kv, 2);
#define READ(D, OUT) hipLaunchKernelGGL((cache_read_kernel<D, OUT>), grid, dim3(256), 0, st, c, slots, req, n_slots, K, V)
    if (c.d == 64) {
        if (out_dtype == SPARGE_F32) READ(64, SPARGE_F32); else if (out_dtype == SPARGE_F16) READ(64, SPARGE_F16); else READ(64, SPARGE_BF16);
    } else {
        if (out_dtype == SPARGE_F32) READ(128, SPARGE_F32); else if (out_dtype == SPARGE_F16) READ(128, SPARGE_F16); else READ(128, SPARGE_BF16);
    }
#undef READ
    return hipGetLastError();
}

}  // namespace sparge
