// Paged 8-bit K/V cache: the step's plan (pages, block table, slot map), the append of new tokens and the read-back.
#include "cache.hpp"

namespace sparge {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int DEAL = 8 * PLAN_THREADS;           // pages that change hands at a time
constexpr int FILL_IN_PLAN = 4 * PLAN_THREADS;   // slots that the plan's one workgroup fills itself

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
__device__ Sums scan(const Sums& v, Sums* lds, Sums& total) {
    constexpr int WAVES = PLAN_THREADS / 64;
    static_assert(WAVES == 16, "a row of lanes holds the waves' sums");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    Sums x = {scan_lanes(v.push), scan_lanes(v.need), scan_lanes(v.tok)};
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    const Sums w = lds[lane % WAVES], upto = {scan_lanes<16>(w.push), scan_lanes<16>(w.need), scan_lanes<16>(w.tok)};
    total = {lane_value(upto.push, WAVES - 1), lane_value(upto.need, WAVES - 1), lane_value(upto.tok, WAVES - 1)};
    x.push += lane_value(upto.push, wave) - lane_value(w.push, wave) - v.push;
    x.need += lane_value(upto.need, wave) - lane_value(w.need, wave) - v.need;
    x.tok += lane_value(upto.tok, wave) - lane_value(w.tok, wave) - v.tok;
    return x;
}

// the largest of a wave's values up to each lane (values >= 0), through DPP row moves
__device__ __forceinline__ int max_lanes(int v) {
    auto step = [&](auto ctrl, auto rows) {
        v = max(v, __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
    };
    using all = std::integral_constant<int, 0xF>;
    step(std::integral_constant<int, 0x111>{}, all{});
    step(std::integral_constant<int, 0x112>{}, all{});
    step(std::integral_constant<int, 0x114>{}, all{});
    step(std::integral_constant<int, 0x118>{}, all{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});
    return v;
}
// the largest value of the threads before (0 for the first, values >= 0); lds: an int per wave
__device__ __forceinline__ int max_before(int v, int* lds) {
    v = max_lanes(v);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 63) lds[wave] = v;
    lds_barrier();
    int before = __shfl_up(v, 1);
    if (lane == 0) before = 0;
    for (int w = 0; w < PLAN_THREADS / 64; ++w)
        if (w < wave) before = max(before, lds[w]);
    return before;
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
// the table entries that slots are made of), so rows, pages and slots are spread over the threads through the prefix sums,
// and the instructions that it runs once: loops that are short anyway stay rolled up (unrolled, with the rows kept in
// registers, 11 us in the place of 6 for 48 rows; it is 4.7 us now, and 16 for 1000 rows of which 200 give up 9200 pages and
// 410 are taken; 15 where 1000 rows take 10000, 22 where they give up as many, too).
__global__ __launch_bounds__(PLAN_THREADS) void cache_plan_kernel(sparge_cache c, const int32_t* __restrict__ new_len,
                                                                  const uint8_t* __restrict__ release, int n_slots, int32_t* cu,
                                                                  int32_t* slots, int32_t* req, int32_t* status) {
    extern __shared__ __align__(16) int lds[];   // over the rows: prefix sums of pages given up, pages taken, new tokens; held tokens
    int* push_at = lds;
    int* need_at = lds + c.R;
    int* tok_at = lds + 2 * c.R;
    int* held_of = lds + 3 * c.R;
    int* top = lds + (c.R + 1) / 2 * 2 * 4;   // the stack's upper end after the pushes: page `pushed - 1 - a` in top[a], a < cached
    int* map = top + DEAL;              // where rows begin
    __shared__ int wave_max[PLAN_THREADS / 64];
    __shared__ Sums wave_sums[PLAN_THREADS / 64];
    __shared__ int all_flags;
    const int tid = threadIdx.x;
    const int per = (c.R + PLAN_THREADS - 1) / PLAN_THREADS;
    const int r0 = tid * per, r1 = min(r0 + per, c.R);
    const long long most = static_cast<long long>(c.max_blocks) * PAGE;
    if (tid == 0) all_flags = 0;
    Sums mine = {0, 0, 0};
    int flags = 0;
    const int n_free = c.n_free[0];
    if (n_free < 0 || n_free > c.n_pages) flags = SPARGE_CACHE_BAD_STATE;
#pragma unroll 1
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
    Sums at = scan(mine, wave_sums, total);   // (its barrier: all_flags is 0)
    if (flags) atomicOr(&all_flags, flags);
    __syncthreads();
    flags = all_flags;
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
    const int pushed = static_cast<int>(total.push), needed = static_cast<int>(total.need), tokens = static_cast<int>(total.tok);
    const int cached = min(min(pushed, needed), DEAL);
#pragma unroll 1
    for (int r = r0; r < r1; ++r) {
        const int len = c.length[r], n = new_len[r], held = release && release[r] ? 0 : len;
        push_at[r] = static_cast<int>(at.push), need_at[r] = static_cast<int>(at.need), tok_at[r] = static_cast<int>(at.tok), held_of[r] = held;
        cu[r] = static_cast<int>(at.tok);
        c.length[r] = held + n;
        at.push += blocks_of(len) * (held != len);
        at.need += blocks_of(held + n) - blocks_of(held);
        at.tok += n;
    }
    lds_barrier();
    int32_t* stack = c.free_pages + n_free;
#pragma unroll 1
    for (int pop = 0; pop < 2; ++pop) {
        // Pages are dealt out eight a thread, in the rows' order: every row writes its number where its pages begin, and the
        // largest number up to a place is the place's row.  (The one workgroup's issue is what bounds this: for the 9000 pages that 200
        // of 1000 rows give up, the kernel takes 25 us with a search per page through the prefix sums, 21 to 23 with pieces of
        // rows dealt to waves, 16 like this.)
        const int* prefix = pop ? need_at : push_at;
        const int n = pop ? needed : pushed;
#pragma unroll 1
        for (int c0 = 0; c0 < n; c0 += DEAL) {
            int4* mine4 = reinterpret_cast<int4*>(map + 8 * tid);
            mine4[0] = mine4[1] = make_int4(0, 0, 0, 0);
            lds_barrier();
#pragma unroll 1
            for (int r = r0; r < r1; ++r) {
                const int begin = prefix[r], end = r + 1 < c.R ? prefix[r + 1] : n;
                if (begin < end && begin < c0 + DEAL && end > c0) map[max(begin - c0, 0)] = r + 1;
            }
            lds_barrier();
            int row[8];
            *reinterpret_cast<int4*>(row) = mine4[0], *reinterpret_cast<int4*>(row + 4) = mine4[1];
#pragma unroll
            for (int e = 1; e < 8; ++e) row[e] = max(row[e], row[e - 1]);
            const int before = max_before(row[7], wave_max);
#pragma unroll
            for (int e = 0; e < 8; ++e) row[e] = max(row[e], before);
            // back to LDS: the wave's 512 pages again with neighbours in neighbouring lanes, for whole lines to and from memory
            mine4[0] = *reinterpret_cast<int4*>(row), mine4[1] = *reinterpret_cast<int4*>(row + 4);
            const int a0 = 512 * (tid >> 6) + (tid & 63);
            int page[8], *entry[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int a = c0 + a0 + 64 * e, r = map[a0 + 64 * e] - 1;
                entry[e] = nullptr;
                if (a >= n) continue;
                entry[e] = c.table + static_cast<long long>(r) * c.max_blocks + (a - prefix[r] + (pop ? blocks_of(held_of[r]) : 0));
                if (!pop) page[e] = *entry[e];
                else if (a < cached) page[e] = top[a];
                else page[e] = stack[pushed - 1 - a];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int a = c0 + a0 + 64 * e;
                if (!entry[e]) continue;
                if (pop) {
                    *entry[e] = page[e];
                } else {
                    stack[a] = page[e];
                    if (pushed - 1 - a < cached) top[pushed - 1 - a] = page[e];
                }
            }
        }
        if (pop) break;
        // What is taken now may be what was given up just now: it is passed on through LDS, so that nobody waits for the stack's
        // stores, unless there are too many.  (Entries are written only after all that are given up have been read.)
        if (min(pushed, needed) > cached) __syncthreads();
        else lds_barrier();
    }
    if (tid == 0) {
        cu[c.R] = tokens;
        c.n_free[0] = n_free + pushed - needed;
        status[0] = 0, status[1] = n_free + pushed - needed;
    }
    if (n_slots > FILL_IN_PLAN) return;
    __syncthreads();
    for (int i = tid; i < n_slots; i += PLAN_THREADS) fill_slot(c, tok_at, tokens, i, held_of, slots, req);
}

// The slot map of a long step, from what the plan has written; a workgroup per 512 slots.
constexpr int FILL_SLOTS = 512;
__global__ __launch_bounds__(256) void cache_slots_kernel(sparge_cache c, int n_slots, const int32_t* __restrict__ cu,
                                                          int32_t* slots, int32_t* req) {
    extern __shared__ __align__(16) int lds[];
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

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }   // a NaN or an infinity is the largest

// What the codes of a block with this amax are made with; codes are 0 in a block of zeros or with an infinity or a NaN.
// x (127 / amax) with 127 / amax in two parts, rounded once to fp32, is off by at most 2^-18.  For 16-bit x (no shift) that
// decides every rounding: a quotient that is a half (k + 1/2 has 8 bits) comes out exact, and another is at least 2^-20 of
// itself away from one (127 X / A, X and A of 11 bits), so it stays on its side: adding 1.5 2^23 + 128 rounds it as asked and
// leaves code + 128 in the low byte.  Shifted x has 24 bits: where four quotients of a wave's lanes come near a half
// (one time in a hundred) code_of decides, as it does where amax's reciprocal leaves the normal range.
struct Quantizer {
    bool plain, fast;
    int up;
    float amax1, inv, hi, lo;

    __device__ explicit Quantizer(uint32_t top) {
        const float amax = __uint_as_float(top);
        plain = top > 0 && top < 0x7F800000u;
        fast = amax > 0x1p-60f && amax < 0x1p60f;
        up = plain ? 1 - __builtin_amdgcn_frexp_expf(amax) : 1;
        amax1 = plain ? __builtin_ldexpf(amax, up) : 1.0f, inv = 127.0f / amax1;
        hi = __builtin_ldexpf(inv, up), lo = __builtin_ldexpf(__builtin_fmaf(-inv, amax1, 127.0f) * (inv * (1.0f / 127.0f)), up);
    }
    // code + 128 in the low byte
    __device__ __forceinline__ uint32_t quick(float x) const { return __float_as_uint(__builtin_fmaf(x, hi, x * lo) + UP); }
    // how near the quotient is to a half: the distance from its rounding
    __device__ __forceinline__ float far(float x) const {
        const float q = __builtin_fmaf(x, hi, x * lo);
        return fabsf(q - ((q + UP) - UP));
    }
    static constexpr float UP = 12583040.0f, NEAR_HALF = 0.5f - 0x1p-16f;
    __device__ __forceinline__ uint32_t slow(float x) const { return static_cast<uint32_t>((plain ? code_of(x, up, amax1, inv) : 0) + 128); }
};
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
    return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
}

// the largest of 256 threads' values below 2^31, N of them at once; lds: 4 N
template <int N>
__device__ __forceinline__ void workgroup_max(uint32_t (&v)[N], uint32_t* lds) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = max_lanes(v[k]);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) {
#pragma unroll
        for (int k = 0; k < N; ++k) lds[4 * k + (threadIdx.x >> 6)] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k)
        v[k] = __builtin_amdgcn_readfirstlane(max(max(lds[4 * k], lds[4 * k + 1]), max(lds[4 * k + 2], lds[4 * k + 3])));
}

// The kv head and the first slot of a workgroup of a grid (windows, kv heads, ..): the heads of a window run together, as their tokens and
// pages lie together.  (Windows first, all workgroups that run at one time want the same 256 bytes of every 4 KB of 16 heads'
// tokens: 65k of them took 234 us to append in the place of 190 and 306 to read to fp32 in the place of 247.)
__device__ __forceinline__ void heads_first(int window, int& hk, int& i0) {
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
    hk = id % gridDim.y;
    i0 = id / gridDim.y * window;
}

// A workgroup quantizes one kv head's K or V of every page that begins to get tokens inside its window of `window` (a power of two
// up to 64) slots: the open page's older tokens from the tail, the new ones from the call's tensor.  Bound by its bytes: a
// thread holds what makes whole 16-byte pieces of the page (K: 16 channels of a token; V: a channel of 16 tokens), loads and
// stores are coalesced and nothing goes through LDS but the maxima: 65k tokens of 16 heads of 128 channels, 805 MB that no cache holds,
// in 151 us, 5.3 TB/s, with a shift 155, where a large copy reaches 5; 29k tokens of 8 heads 39 and 42 us.  Behind a
// read-back to fp32, whose stores are 1.07 and 0.24 GB, these take 190 and 57 us.  (K and V of a page in one workgroup, their loads
// together: 69 us in the place of those 57.)  Where a page gets few tokens that do not raise its amax
// (decoding: all but one of t + 1 at the t-th token of a page), the older codes are what they were and only the new ones are
// written; the tail's amax per token tells without reading the tail.
// The row's first page also stores the tokens of the row's last page if that stays open (after it has read the older
// ones, which lie in the same place).
// FEW: tokens of a page up to which their codes are written by themselves (200 rows of 32 heads, all by themselves against none: 34 us
// against 45 for one token a row, 42 against 47 for 2, 46 against 61 for 8).
constexpr int FEW = 8;
template <int D, int DT>
__global__ __launch_bounds__(256, 6) void cache_append_kernel(sparge_cache c, const uint16_t* __restrict__ K,
                                                           const uint16_t* __restrict__ V, int n_slots, int window, long long k_sn,
                                                           long long k_sh, long long v_sn, long long v_sh,
                                                           const int32_t* __restrict__ cu, const int32_t* __restrict__ slots,
                                                           const int32_t* __restrict__ req) {
    constexpr int LPR = D / 8, RPS = 256 / LPR;   // threads per token of 8 channels each, tokens at a time
    constexpr int CV = D / 64;                    // V: channels per thread; K: pieces per thread
    __shared__ uint32_t lds_max[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int hk, i0;
    heads_first(window, hk, i0);
    const bool is_v = blockIdx.z != 0;
    const uint16_t* x = is_v ? V + hk * v_sh : K + hk * k_sh;
    const long long sn = is_v ? v_sn : k_sn;

    int my_slot = -1, my_row = -1, my_prev = -1;
    if (lane < window && i0 + lane < n_slots) {
        my_slot = slots[i0 + lane];
        my_row = req[i0 + lane];
        my_prev = i0 + lane ? req[i0 + lane - 1] : -1;
    }
    const bool there = my_slot >= 0 && my_slot / PAGE < c.n_pages && my_row >= 0 && my_row < c.R;
    unsigned long long starts = __ballot(there && (my_slot % PAGE == 0 || my_prev != my_row));
    const int col = (tid % LPR) * 8, tok = tid / LPR;   // where 8 channels of a token are taken
    while (starts) {
        const int first = __builtin_ctzll(starts);
        starts &= starts - 1;
        const int i = i0 + first;
        const int slot = __builtin_amdgcn_readlane(my_slot, first), r = __builtin_amdgcn_readlane(my_row, first);
        const int page = slot / PAGE, off = slot % PAGE;
        const int row_begin = max(0, min(cu[r], n_slots)), row_end = max(0, min(cu[r + 1], n_slots));
        const int n = max(1, min(PAGE - off, row_end - i));
        const long long at = static_cast<long long>(page) * c.H_kv + hk, row_at = static_cast<long long>(r) * c.H_kv + hk;
        uint16_t* tail = static_cast<uint16_t*>(is_v ? c.v_tail : c.k_tail) + row_at * PAGE * D;
        float* tail_amax = (is_v ? c.v_tail_amax : c.k_tail_amax) + row_at * PAGE;
        const float* shift = is_v || !c.k_shift ? nullptr : c.k_shift + row_at * D;
        uint8_t* codes = static_cast<uint8_t*>(is_v ? c.v : c.k) + at * PAGE * D;
        auto load8 = [&](const uint16_t* p, float (&y)[8]) {
            const uint4 raw = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = cvt16<DT>(static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)))) - (shift ? shift[col + e] : 0.f);
            return raw;
        };
        bool done = false;
        if (n <= FEW) {
            float y[8] = {};
            uint32_t top = 0;
            const uint32_t before = tid < off ? __float_as_uint(tail_amax[tid]) : 0u;
            if (tok < n) {
                load8(x + (i + tok) * sn + col, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, abs_bits(y[e]));
            }
            uint32_t tops[2] = {before, top};
            workgroup_max(tops, lds_max);
            const uint32_t old = tops[0], now = tops[1];
            if (off == 0 || old >= now) {
                done = true;
                const uint32_t amax = max(old, now);
                const Quantizer q(amax);
                if (tok < n) {
                    uint32_t b[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) b[e] = q.fast && !shift ? q.quick(y[e]) : q.slow(y[e]);
                    if (is_v) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) codes[v_byte(off + tok, col + e)] = static_cast<uint8_t>(b[e]);
                    } else {
                        *reinterpret_cast<uint2*>(codes + k_byte(off + tok, col, D)) =
                            make_uint2(low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7]));
                    }
                }
                if (tid == 0) (is_v ? c.v_amax : c.k_amax)[at] = __uint_as_float(amax);
            }
        }
        if (!done) {
            // K: pieces wave + 4 p: token 16 (piece / CV) + lane % 16, channels 64 (piece % CV) + 16 (lane / 16) + 0..15
            // V: tokens 16 t + 4 wave + 0..3, channels CV lane + 0..CV-1
            // (kept as they come, 16 bits each: twice the workgroups fit a compute unit)
            uint32_t raw[CV][8];
            auto k_token = [&](int p) { return 16 * ((wave + 4 * p) / CV) + (lane & 15); };
            auto k_channel = [&](int p) { return 64 * ((wave + 4 * p) % CV) + 16 * (lane >> 4); };
            if (is_v) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = 16 * (e >> 2) + 4 * wave + (e & 3);
                    const uint16_t* from = (t < off ? tail + t * D : x + (i + t - off) * sn) + CV * lane;
                    w[e] = 0;
                    if (t < off + n) {
                        if constexpr (CV == 2) w[e] = *reinterpret_cast<const uint32_t*>(from); else w[e] = *from;
                    }
                }
#pragma unroll
                for (int p = 0; p < CV; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e)   // the 16-bit halves p of two words side by side
                        raw[p][e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], p ? 0x07060302u : 0x05040100u);
            } else {
#pragma unroll
                for (int p = 0; p < CV; ++p) {
                    const int t = k_token(p);
                    uint4 two[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
                    const uint4* from = reinterpret_cast<const uint4*>((t < off ? tail + t * D : x + (i + t - off) * sn) + k_channel(p));
                    if (t < off + n) two[0] = from[0], two[1] = from[1];
                    __builtin_memcpy(raw[p], two, 32);
                }
            }
            float sh[16] = {};   // (the same channels for all p)
            if (shift) {
#pragma unroll
                for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(sh + e) = *reinterpret_cast<const float4*>(shift + k_channel(0) + e);
            }
            auto plain_value = [&](int p, int e) { return cvt16<DT>(static_cast<uint16_t>(raw[p][e >> 1] >> (16 * (e & 1)))); };
            auto shifted_value = [&](int p, int e) { return k_token(p) < off + n ? plain_value(p, e) - sh[e] : 0.f; };
            uint32_t top = 0;
            if (shift) {
#pragma unroll
                for (int p = 0; p < CV; ++p)
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = max(top, abs_bits(shifted_value(p, e)));
            } else {   // two 16-bit values at a time: their bits are ordered as their sizes
                typedef unsigned short v2u __attribute__((ext_vector_type(2)));
                v2u two = {0, 0};
#pragma unroll
                for (int p = 0; p < CV; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t bits = raw[p][e] & 0x7FFF7FFFu;
                        v2u w;
                        __builtin_memcpy(&w, &bits, 4);
                        two = __builtin_elementwise_max(two, w);
                    }
                top = abs_bits(cvt16<DT>(max(two[0], two[1])));
            }
            uint32_t tops[1] = {top};
            workgroup_max(tops, lds_max);
            top = tops[0];
            const Quantizer q(top);
#pragma unroll
            for (int p = 0; p < CV; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(raw[p][e]));   // unpacked again, not kept as fp32 from the maximum on
            auto write = [&](auto four) {
#pragma unroll
                for (int p = 0; p < CV; ++p) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = four(p, 4 * e);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    const int ch = CV * lane + p;
                    const int piece = is_v ? (ch >> 4) * 64 + (ch & 15) + 16 * wave : (wave + 4 * p) * 64 + lane;
                    reinterpret_cast<uint4*>(codes)[piece] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            };
            if (q.fast && !shift) {
                write([&](int p, int e) {
                    return low_bytes(q.quick(plain_value(p, e)), q.quick(plain_value(p, e + 1)), q.quick(plain_value(p, e + 2)), q.quick(plain_value(p, e + 3)));
                });
            } else {
                write([&](int p, int e) {
                    float y[4], far = 1.0f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = shift ? shifted_value(p, e + k) : plain_value(p, e + k);
                    if (q.fast) far = fmaxf(fmaxf(q.far(y[0]), q.far(y[1])), fmaxf(q.far(y[2]), q.far(y[3])));
                    if (__any(far > Quantizer::NEAR_HALF)) return low_bytes(q.slow(y[0]), q.slow(y[1]), q.slow(y[2]), q.slow(y[3]));
                    return low_bytes(q.quick(y[0]), q.quick(y[1]), q.quick(y[2]), q.quick(y[3]));
                });
            }
            if (tid == 0) (is_v ? c.v_amax : c.k_amax)[at] = __uint_as_float(top);
        }
        if (i == row_begin) {   // the tokens of the row's last page, if it stays open (the older ones have been read: the maxima's barriers)
            const int last = row_end > 0 ? slots[row_end - 1] : -1;
            const int open = last >= 0 ? (last % PAGE + 1) % PAGE : 0;
            const int keep = min(open, row_end - row_begin);
            for (int t = open - keep + tok; t < open; t += RPS) {
                float y[8];
                const uint4 raw = load8(x + (row_end - open + t) * sn + col, y);
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, abs_bits(y[e]));
#pragma unroll
                for (int s = 1; s < LPR; s <<= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), s)));
                *reinterpret_cast<uint4*>(tail + t * D + col) = raw;
                if (col == 0) tail_amax[t] = __uint_as_float(top);
            }
        }
    }
}

// ---- read-back ---------------------------------------------------------------------------------------------------

// value = code amax / 127 (+ shift) rounded once to fp32, then to 16 bits where asked for.  With a shift, and where amax is next to
// the ends of fp32's range, it is formed in 64 bits.  Otherwise step = amax / 127 is split into its upper 17 bits, whose
// products with a code are exact, and the rest: value = code upper + code rest in one fma, off by 2^-41 of itself before its rounding.
// That is the exact quotient's rounding: N / 127 (N = code times amax's 24 bits) is no nearer than 2^-32 of itself to what lies half
// way between two floats, unless it is just there, and then 127 divides amax's bits and both parts are exact.
template <int OUT, int N>
__device__ __forceinline__ void put(void* out, const float (&y)[N]) {   // 4, 8 or 16 bytes
    if constexpr (OUT == SPARGE_F32) {
        __builtin_memcpy(__builtin_assume_aligned(out, 4 * N), y, 4 * N);
    } else {
        uint16_t w[N];
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = cvt_to16<OUT>(y[e]);
        __builtin_memcpy(__builtin_assume_aligned(out, 2 * N), w, 2 * N);
    }
}
// A workgroup takes the runs of consecutive slots of one page inside its window of `window` (a power of two up to 64) slots, K
// (blockIdx.z 0) or V of one kv head.  Bound by its bytes; what counts is that a store instruction covers whole lines: a thread takes
// 16 bytes' worth of a token's channels of K (4 or 8 codes; with 16 codes a thread as the pieces lie the stores are 64 bytes
// apart: 294 us in the place of 231 for 50k tokens of 16 heads of 128 channels to fp32, now 195, 5.2 TB/s) and 1 or 2 channels of V's
// 16 tokens.
template <int D, int OUT>
__global__ __launch_bounds__(256, 6) void cache_read_kernel(sparge_cache c, const int32_t* __restrict__ slots,
                                                         const int32_t* __restrict__ req, int n_slots, int window, void* K, void* V) {
    constexpr int EL = OUT == SPARGE_F32 ? 4 : 2, CV = D / 64, KCH = 16 / EL;   // bytes of an output; channels of a thread, V and K
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    int hk, i0;
    heads_first(window, hk, i0);
    const bool is_v = blockIdx.z != 0;
    int my_slot = -1, my_row = 0;
    if (lane < window && i0 + lane < n_slots) {
        my_slot = slots[i0 + lane];
        if (req) my_row = req[i0 + lane];
    }
    const bool there = my_slot >= 0 && my_slot / PAGE < c.n_pages && my_row >= 0 && my_row < c.R;
    const int prev_slot = __shfl_up(my_slot, 1), prev_row = __shfl_up(my_row, 1);
    const bool goes_on = there && lane > 0 && my_slot == prev_slot + 1 && my_slot % PAGE != 0 && my_row == prev_row;
    unsigned long long starts = __ballot(there && !goes_on);
    const unsigned long long breaks = __ballot(!goes_on);
    while (starts) {
        const int first = __builtin_ctzll(starts);
        starts &= starts - 1;
        const unsigned long long behind = first == 63 ? 0ull : breaks >> (first + 1);
        const int n = behind ? __builtin_ctzll(behind) + 1 : 64 - first;   // lanes beyond the window break the run
        const int slot = __builtin_amdgcn_readlane(my_slot, first), r = __builtin_amdgcn_readlane(my_row, first);
        const int page = slot / PAGE, off = slot % PAGE;
        const long long at = static_cast<long long>(page) * c.H_kv + hk;
        const uint8_t* codes = static_cast<const uint8_t*>(is_v ? c.v : c.k) + at * PAGE * D;
        const float amax = (is_v ? c.v_amax : c.k_amax)[at];
        const double step = static_cast<double>(amax) / 127.0;
        const float* shift = c.k_shift && !is_v ? c.k_shift + (static_cast<long long>(r) * c.H_kv + hk) * D : nullptr;
        // outputs: a uniform address for the page's token t, and the thread's own bytes from there (4 MiB at most)
        const uint32_t row_bytes = c.H_kv * D * EL;
        char* out0 = static_cast<char*>(is_v ? V : K) + (static_cast<long long>(i0 + first - off) * c.H_kv + hk) * (D * EL);
        auto in_run = [&](int t) { return t >= off && t < off + n; };
        constexpr int LPT = D / KCH, STEP = 256 / LPT;   // K: threads per token, tokens of the workgroup at a time
        const int k_tok = threadIdx.x / LPT, k_ch = (threadIdx.x % LPT) * KCH;
        uint32_t w[D / 16];   // K: KCH codes of each of its tokens; V: 16 codes of each of its channels
        if (is_v) {
#pragma unroll
            for (int p = 0; p < CV; ++p) {
                const int ch = CV * lane + p;
                const uint4 raw = reinterpret_cast<const uint4*>(codes)[(ch >> 4) * 64 + (ch & 15) + 16 * wave];
                w[4 * p] = raw.x, w[4 * p + 1] = raw.y, w[4 * p + 2] = raw.z, w[4 * p + 3] = raw.w;
            }
        } else {
#pragma unroll
            for (int p = 0; p < PAGE / STEP; ++p)
                if (in_run(p * STEP + k_tok))
                    __builtin_memcpy(w + KCH / 4 * p, __builtin_assume_aligned(codes + k_byte(p * STEP + k_tok, k_ch, D), KCH), KCH);
        }
        auto write = [&](auto value) {   // value(code, the channel's index of the thread)
#pragma unroll
            for (int k = 0; k < D / 16; ++k) asm volatile("" : "+v"(w[k]));   // unpacked here, not ahead of the branch
            auto code = [](uint32_t word, int e) { return static_cast<int>((word >> (8 * e)) & 0xFFu) - 128; };
            if (is_v) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = 16 * (e >> 2) + 4 * wave + (e & 3);
                    if (!in_run(t)) continue;
                    float y[CV];
#pragma unroll
                    for (int p = 0; p < CV; ++p) y[p] = value(code(w[4 * p + (e >> 2)], e & 3), p);
                    put<OUT>(out0 + static_cast<long long>(t) * row_bytes + static_cast<uint32_t>(CV * EL * lane), y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int p = 0; p < PAGE / STEP; ++p) {
                    const int t = p * STEP + k_tok;
                    if (!in_run(t)) continue;
                    float y[KCH];
#pragma unroll
                    for (int e = 0; e < KCH; ++e) y[e] = value(code(w[KCH / 4 * p + e / 4], e & 3), e);
                    put<OUT>(out0 + static_cast<long long>(p * STEP) * row_bytes + (k_tok * row_bytes + static_cast<uint32_t>(k_ch * EL)), y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        if (!shift && amax >= 0x1p-90f && amax <= 0x1p127f) {
            const float upper = __uint_as_float(__float_as_uint(static_cast<float>(step)) & ~0x7Fu);
            const float rest = static_cast<float>(step - static_cast<double>(upper));
            write([&](int q, int) { return __builtin_fmaf(static_cast<float>(q), rest, static_cast<float>(q) * upper); });
        } else {
            float sh[KCH] = {};
            if (shift)
#pragma unroll
                for (int e = 0; e < KCH; e += 4) *reinterpret_cast<float4*>(sh + e) = *reinterpret_cast<const float4*>(shift + k_ch + e);
            write([&](int q, int e) { return static_cast<float>(static_cast<double>(q) * step + static_cast<double>(sh[e])); });
        }
    }
}

}  // namespace

hipError_t launch_cache_plan(const sparge_cache& c, const int32_t* new_len, const uint8_t* release, int n_slots, int32_t* cu,
                             int32_t* slots, int32_t* req, int32_t* status, hipStream_t st) {
    const int lds = (c.R + 1) / 2 * 2 * 4 + 2 * DEAL;   // ints: the rows (16-byte aligned for what follows), the stack's end, the map
    hipLaunchKernelGGL(cache_plan_kernel, dim3(1), dim3(PLAN_THREADS), lds * sizeof(int), st, c, new_len, release, n_slots, cu, slots, req,
                       status);
    if (n_slots > FILL_IN_PLAN)
        hipLaunchKernelGGL(cache_slots_kernel, dim3((n_slots + FILL_SLOTS - 1) / FILL_SLOTS), dim3(256), 2 * c.R * sizeof(int), st, c,
                           n_slots, cu, slots, req);
    return hipGetLastError();
}

// Slots per workgroup of the append and the read-back: a page's worth where that makes enough workgroups, down to one (which may be a
// page of its own) where it does not: a workgroup takes its window's pages one after the other.  Enough is 1024 for the
// append (with 512, 200 rows of one token and 32 heads take 46 us in the place of 33, 128 rows and 8 heads 10.1 in the place of 8.8; with 4096, a
// piece of a prompt 13 in the place of 7.7: most workgroups have nothing to do) and 512 for the read-back, whose runs end
// at windows (with 1024, 374 tokens of 4 heads take 7.8 us in the place of 5.6).
static int window_of(int n_slots, int heads, int groups) {
    int window = 64;
    while (window > 1 && static_cast<long long>(n_slots / window) * heads < groups) window /= 2;
    return window;
}

hipError_t launch_cache_append(const sparge_cache& c, const void* K, const void* V, int n_slots, long long k_sn, long long k_sh,
                               long long v_sn, long long v_sh, const int32_t* cu, const int32_t* slots, const int32_t* req,
                               hipStream_t st) {
    const int window = window_of(n_slots, c.H_kv, 1024);
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
    if (!c.k_shift) req = nullptr;   // the rows are asked for the shift alone
    const int window = window_of(n_slots, c.H_kv, 512);
    const dim3 grid((n_slots + window - 1) / window, c.H_kv, 2);
#define READ(D, OUT) hipLaunchKernelGGL((cache_read_kernel<D, OUT>), grid, dim3(256), 0, st, c, slots, req, n_slots, window, K, V)
    if (c.d == 64) {
        if (out_dtype == SPARGE_F32) READ(64, SPARGE_F32); else if (out_dtype == SPARGE_F16) READ(64, SPARGE_F16); else READ(64, SPARGE_BF16);
    } else {
        if (out_dtype == SPARGE_F32) READ(128, SPARGE_F32); else if (out_dtype == SPARGE_F16) READ(128, SPARGE_F16); else READ(128, SPARGE_BF16);
    }
#undef READ
    return hipGetLastError();
}

}  // namespace sparge
