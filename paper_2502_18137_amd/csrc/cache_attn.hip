// Attention of new tokens over the paged 8-bit K/V cache.
//
// O_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i . k_j - m_i), in one pass over the keys.  With codes a, b (integers) and a
// block's scales sk, sv: q_i . k_j = sk (q_i . a_j) and v_j = sv b_j.  Both products run on the 16-bit MFMA with the codes as
// fp16 integers (exact), S^T = A Q^T and O^T = B^T P^T, so that a lane owns one query (lane % 16) and four keys of every
// sixteen, and P goes from the accumulators of the first product to the operand of the second without leaving the lane:
// the pages' byte order is made for that.  Both scales enter the exponent.  A query keeps two references: m, the largest score
// so far, for the sum of the weights, and mo, the largest score + log2 sv, for O: the weights that meet V's codes are
// exp2(score + log2 sv - mo), so that what fp16 rounds away is small beside what counts for this query most, whatever the sizes of V
// in blocks that it gives no weight.
//
// The query rows of one row of the cache are its new tokens times the G heads that share a kv head.  Two kernels:
//   rows of at most 16 query rows (decoding), and of more where all is little: the work is reading pages.  A wave takes blocks by itself, operands come
//   from memory into registers, 1 KB of consecutive bytes a load, without LDS and without barriers.
//   others: the work is products.  Four waves take 32 query rows each and share the blocks, which they convert to
//   fp16 into LDS once, a quarter each.
// In both, items (a kv head's tile of query rows) lie one behind the other on a line, each as long as the keys it sees; the
// line is cut into equal parts, one per wave or workgroup.  A long item is split over several parts, whose results a
// further launch joins in a fixed order; short ones share a part.  The host knows the step's tokens but not which rows have them: where
// rows of both kinds are possible, one launch's workgroups take their parts of the first line, then, if there are any, of the second.
#include "cache.hpp"

namespace sparge {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr float FAR = -1e30f;          // reference of a row that has seen no key
constexpr float SLACK = 6.0f;          // log2: how far a row's maxima may run ahead of their references inside exp2
constexpr float W_UP = 9.0f;           // log2: weights are at most 2^(6 + 9) in fp16; the largest is 2^9 or more, and one of 2^-34 of it is
                                       // not lost
constexpr float W_LEAST = 60.0f;       // log2: a block whose largest weight would be less than 2^-60 (small V, zeros) is taken as if it were
                                       // that: 0 in fp16, and the sum of the weights keeps it

constexpr int NARROW_ROWS = 16, NARROW_WGS = 512, NARROW_LOG2 = 11;   // two workgroups per compute unit, a part per wave
constexpr int WIDE_ROWS = 128, WIDE_WGS = 512, WIDE_LOG2 = 9;         // a part per workgroup
// Rows of several tiles are the narrow kernel's too where the whole line is at most 5 blocks a wave: the wide kernel's workgroups would
// have few blocks each, one after the other (4 rows of 9000 keys, 16 heads a kv head, 8 tokens: 30 us in the place of 46; of 4 heads and
// 8 tokens: 33.0, 36.9; 8.8 blocks a wave, 4 heads and 16 tokens: 53.7, 46.4).
constexpr u64 NARROW_BLOCKS = 5;
static_assert(4 * NARROW_WGS == 1 << NARROW_LOG2 && WIDE_WGS == 1 << WIDE_LOG2, "the line is cut into up to 2^LOG2 parts");

template <int X>
__device__ __forceinline__ float other(float v) {   // of lane ^ X, X = 16 or 32
    const uint32_t u = __float_as_uint(v);
    if constexpr (X == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return __uint_as_float(threadIdx.x & 16 ? r[0] : r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
    }
}
__device__ __forceinline__ float max_groups(float v) {
    v = fmaxf(v, other<16>(v));
    return fmaxf(v, other<32>(v));
}
__device__ __forceinline__ float sum_groups(float v) {
    v += other<16>(v);
    return v + other<32>(v);
}
// What the narrow and the wide half of a kernel make of a value is not kept in registers from the one to the other.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ u64 uniform(u64 v) {
    return static_cast<u64>(uniform(static_cast<int>(v >> 32))) << 32 | static_cast<uint32_t>(uniform(static_cast<int>(v)));
}

// 8 bytes (code + 128) -> 8 fp16 codes: the byte under 0x64 is the fp16 1024 + byte, less 1152 the code, all exact
__device__ __forceinline__ v8h codes8(uint32_t a, uint32_t b) {
    uint32_t w[4] = {__builtin_amdgcn_perm(0x64646464u, a, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u),
                     __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)};
    v2h h[4];
    const v2h bias = {(_Float16)1152.0f, (_Float16)1152.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        __builtin_memcpy(&h[e], &w[e], 4);
        h[e] -= bias;
    }
    v8h r;
    __builtin_memcpy(&r, h, 16);
    return r;
}

// How a row's query rows are cut into tiles of up to `rows`: TT whole tokens of G heads.  (The narrow kernel gets groups of up to its
// 16 rows, the wide one all there are.)
struct Cut {
    int G, TT;
};
static_assert(SPARGE_MAX_HEADS <= WIDE_ROWS, "a token's group fits a tile");
__device__ __forceinline__ Cut cut_of(int G, int rows) { return {G, rows / G}; }

// Which rows a line holds: those of more than `above` and at most `upto` query rows of a kv head.
struct Rows {
    long long above, upto;

    __device__ __forceinline__ bool hold(int n, int G) const { return static_cast<long long>(n) * G > above && static_cast<long long>(n) * G <= upto; }
};
constexpr Rows ALL_ROWS = {0, 1ll << 62};

struct RowInfo {
    int first, n, len, p0;     // new tokens [first, first + n) (0: not this line's), keys, keys before the first new token
    int tiles;                 // tiles of TT tokens
};
__device__ __forceinline__ RowInfo row_info(const sparge_cache& c, const CacheAttn& a, const Cut& t, const Rows& which, int r) {
    RowInfo x;
    x.first = max(0, min(a.cu[r], a.n_slots));
    x.n = max(0, min(a.cu[r + 1], a.n_slots) - x.first);
    x.len = max(0, min(c.length[r], static_cast<int>(min(static_cast<long long>(c.max_blocks) * PAGE, 0x7FFFFFC0ll))));
    x.p0 = max(0, x.len - x.n);
    if (!which.hold(x.n, t.G)) x.n = 0;
    x.tiles = (x.n + t.TT - 1) / t.TT;
    return x;
}
__device__ __forceinline__ RowInfo uniform(RowInfo x) {
    x.first = uniform(x.first), x.n = uniform(x.n), x.len = uniform(x.len), x.p0 = uniform(x.p0), x.tiles = uniform(x.tiles);
    return x;
}

struct Joint {                          // workspace
    JoinDesc* desc;                     // [parts]
    float* ml;                          // [2 parts][rows of a tile][2] reference and sum of a row's part
    float* o;                           // [2 parts][rows of a tile][d] mean of the values over the part's keys
};

// exclusive prefixes of v over the 256 threads and the totals; lds: 4 per value
template <int N>
__device__ __forceinline__ void prefix(u64 (&v)[N], u64 (*lds)[4], u64 (&total)[N]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 upto[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        upto[k] = scan_lanes(static_cast<long long>(v[k]));
        if (lane == 63) lds[k][wave] = upto[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        total[k] = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) upto[k] += lds[k][w];
            total[k] += lds[k][w];
        }
        v[k] = upto[k] - v[k];
    }
}

// a / b, both below 2^52.  (Kernels that run for a few microseconds wait for their own instructions: the 64-bit division that the
// compiler would put in its place has 130 of them.)
__device__ __forceinline__ u64 quotient(u64 a, u64 b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    u64 q = static_cast<u64>(static_cast<double>(a) / static_cast<double>(b));
    while (q * b > a) --q;
    while ((q + 1) * b <= a) ++q;
    return q;
}

// A line of `total` places in 2^log2 equal parts.
struct Line {
    u64 total;
    int log2;

    __device__ __forceinline__ u64 begin(int part) const { return (total * part) >> log2; }
    __device__ __forceinline__ int part_of(u64 place) const {   // the last part that begins at or before a place
        int p = static_cast<int>(static_cast<float>(place) / static_cast<float>(total) * static_cast<float>(1 << log2));
        while (begin(p) > place) --p;
        while (begin(p + 1) <= place) ++p;
        return p;
    }
};
// A part that begins inside an item: what the join needs.  start, end: the item on the line; token, head: its first.
__device__ __forceinline__ JoinDesc boundary(const Line& line, int part, u64 start, u64 end, int token, int n_tok, int head) {
    const int first = line.part_of(start) + 1;                   // the first part that begins inside it
    return {line.part_of(end - 1) - first + 2, first, part, token, n_tok, head, {0, 0}};
}

// The blocks of an item's range, 64 table entries at a time, one a lane, the next 64 on their way.
struct Blocks {
    int base, end, next_page, l_page;
    float l_ka, l_va;
    u64 bits;
    const int32_t* table;
    const uint8_t* mask;

    __device__ __forceinline__ void ahead(int j) {   // a page, or -1: not there or not kept
        next_page = -1;
        if (j < end && (!mask || mask[j])) next_page = table[j];
    }
    __device__ __forceinline__ void open(const sparge_cache& c, const CacheAttn& a, int r, int kh, int b0, int b1) {
        base = b0 - 64, end = b1, bits = 0;
        table = c.table + static_cast<long long>(r) * c.max_blocks;
        mask = a.mask ? a.mask + (static_cast<long long>(r) * c.H_kv + kh) * c.max_blocks : nullptr;
        ahead(b0 + static_cast<int>(threadIdx.x & 63));
    }
    // at: the lane that holds the block's page and scales
    __device__ __forceinline__ bool next(const sparge_cache& c, int kh, int& block, int& page, int& at) {
        while (bits == 0) {
            base += 64;
            if (base >= end) return false;
            l_page = next_page;
            const bool keep = l_page >= 0 && l_page < c.n_pages;
            if (keep) {
                l_ka = c.k_amax[static_cast<long long>(l_page) * c.H_kv + kh];
                l_va = c.v_amax[static_cast<long long>(l_page) * c.H_kv + kh];
            }
            ahead(base + 64 + static_cast<int>(threadIdx.x & 63));
            bits = __ballot(keep);
        }
        at = __builtin_ctzll(bits);
        bits &= bits - 1;
        block = base + at;
        page = __builtin_amdgcn_readlane(l_page, at);
        return true;
    }
    __device__ __forceinline__ float ka(int at) const { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l_ka), at)); }
    __device__ __forceinline__ float va(int at) const { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l_va), at)); }
};

// A tile of 16 query rows as an MFMA operand: fp16 as it is; bf16 times the power of two that brings the row's largest to [1, 2)
// (exact but for what is below 2^-24 of it).  Operand s holds channels 64 (s / 2) + 16 (lane / 16) + 8 (s % 2) + 0..7.
template <int D>
__device__ __forceinline__ void load_q(uint4 (&raw)[D / 32], const uint16_t* row, bool valid) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        raw[s] = make_uint4(0u, 0u, 0u, 0u);
        if (valid) raw[s] = *reinterpret_cast<const uint4*>(row + 64 * (s >> 1) + 8 * (s & 1));
    }
}
__device__ __forceinline__ uint32_t top16(const uint4& raw) {   // the largest |x| of 8 bf16, as its bits
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7FFFu, (w[e] >> 16) & 0x7FFFu));
    return top;
}
__device__ __forceinline__ int exponent16(uint32_t top) {       // of bf16 bits; 0 for zero, infinity and NaN, which stay what they are
    const int ex = static_cast<int>(top >> 7) - 127;
    return ex > 127 || top == 0 ? 0 : ex;
}
template <int DT>
__device__ __forceinline__ v8h scaled8(const uint4& raw, float by) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    v8h r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r[2 * e] = static_cast<_Float16>(cvt16<DT>(static_cast<uint16_t>(w[e] & 0xFFFFu)) * by);
        r[2 * e + 1] = static_cast<_Float16>(cvt16<DT>(static_cast<uint16_t>(w[e] >> 16)) * by);
    }
    return r;
}
template <int D, int DT>
__device__ __forceinline__ float convert_q(const uint4 (&raw)[D / 32], v8h (&qf)[D / 32]) {
    if constexpr (DT == SPARGE_F16) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) __builtin_memcpy(&qf[s], &raw[s], 16);
        return 1.0f;
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) top = max(top, top16(raw[s]));
        top = max(top, __float_as_uint(other<16>(__uint_as_float(top))));
        top = max(top, __float_as_uint(other<32>(__uint_as_float(top))));
        const int ex = exponent16(top);
        const float down = __builtin_ldexpf(1.0f, -ex);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) qf[s] = scaled8<DT>(raw[s], down);
        return __builtin_ldexpf(1.0f, ex);
    }
}

// A block with a NaN or an infinity in K or V: its codes are 0; the queries that see one of its keys get NaN, through their
// sums, and the others nothing.
__device__ __forceinline__ bool not_finite(float ka, float va) { return !(ka < INFINITY && va < INFINITY); }
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7FC00000u); }

// log2 of a block's V amax (-inf for zeros), subnormal ones too, which v_log_f32 takes for 0
__device__ __forceinline__ float log2_of(float va) {
    return __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(va)) + static_cast<float>(__builtin_amdgcn_frexp_expf(va));
}
// What is added to a row's scores of a block to make the exponents of its weights; top: the largest score.
__device__ __forceinline__ float weight_log2(float v_log2, float mo, float top) {
    return fmaxf(v_log2 - mo + W_UP, -W_LEAST - fmaxf(top, FAR));
}
// The block's sum of weights back in the units of l.
__device__ __forceinline__ float weight_back(float add, float m) { return __builtin_amdgcn_exp2f(-add - m); }

// One tile's softmax step on a block's scores s (keys 16 t + 4 (lane / 16) + e): the weights with V's scale as operand pf, the row's
// references m and mo and sum l, O and l scaled where the references move.  last: the last key of the block that the row sees,
// less 4 (lane / 16); looked at only if `masked`.  pf[2], pf[3], where asked for: what the weights' rounding left.
template <int NV, int NP>
__device__ __forceinline__ void softmax(v4f (&s)[4], float cq, float v_log2, bool masked, int last, float& m, float& mo, float& l,
                                        v4f (&o)[NV], v8h (&pf)[NP]) {
    if (cq == 0.f) cq = 1e-37f;   // a block of zeros: -inf stays what it is and becomes a weight of 0
    if (masked) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * t + e > last) s[t][e] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, s[t][e]);
    top = max_groups(top) * cq;
    if (__any(top > m + SLACK || top + v_log2 > mo + SLACK)) {
        const float to = fmaxf(m, top), o_to = fmaxf(mo, top + v_log2), down = __builtin_amdgcn_exp2f(mo - o_to);
        l *= __builtin_amdgcn_exp2f(m - to);
        m = to, mo = o_to;
#pragma unroll
        for (int n = 0; n < NV; ++n) o[n] *= down;
    }
    float w[16];
    const float add = weight_log2(v_log2, mo, top);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * t + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], cq, add));
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum += w[e];
    l += sum * weight_back(add, m);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        pf[e >> 3][e & 7] = static_cast<_Float16>(w[e]);
        if constexpr (NP == 4) pf[2 + (e >> 3)][e & 7] = static_cast<_Float16>(w[e] - static_cast<float>(pf[e >> 3][e & 7]));
    }
}

// A row's O over its sum: times `by`, then 2^up.  (One after the other: neither leaves fp32's range where the result does not.)
struct Mean {
    float by;
    int up;

    __device__ __forceinline__ Mean(float l, float m, float mo) {
        const float e = fminf(fmaxf(mo - m - W_UP, -400.0f), 400.0f), whole = floorf(e);   // (-400: a result of 0)
        by = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(e - whole) * (1.0f / 127.0f) / l;
        up = static_cast<int>(whole);
    }
    __device__ __forceinline__ float operator()(float o) const { return __builtin_ldexpf(o * by, up); }
};
// A tile's rows, divided by their sums, as results or as a part's.
template <int NV, int DT>
__device__ __forceinline__ void store_whole(const v4f (&o)[NV], const Mean& mean, uint16_t* out) {
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        uint16_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = cvt_to16<DT>(mean(o[n][e]));
        uint2 w;
        __builtin_memcpy(&w, h, 8);
        *reinterpret_cast<uint2*>(out + 16 * n) = w;
    }
}
template <int NV>
__device__ __forceinline__ void store_part(const v4f (&o)[NV], const Mean& mean, float m, float l, const Joint& ws, long long at) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        v4f y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = mean(o[n][e]);
        *reinterpret_cast<v4f*>(ws.o + at * (16 * NV) + 16 * n + 4 * (lane >> 4)) = y;
    }
    if (lane < 16) ws.ml[2 * at] = m, ws.ml[2 * at + 1] = l;
}

// ---- few query rows: a wave by itself ------------------------------------------------------------------------------

// Bound by the pages' bytes: a wave keeps the next block's K and V on their way while it works on one, 16 KB (d = 128), eight
// waves on a compute unit; and it looks ahead over the end of an item, so that the next one's table, queries and first block
// come while the last block of this one is worked on.  160 rows of 5000 to 33000 keys, 8 kv heads of 128 channels, 4.9 GB: 832 us, 5.8 TB/s,
// where a large copy reaches 5.0; 64 rows of 300 to 9000 keys, 0.33 GB: 65 us.  (Three waves a SIMD, whose registers spill: 116 us
// in the place of 100.)  A lone row of 500 keys takes 7.6 us, a chain of latencies: the rows' sums, the table, the
// queries, the page.
struct NarrowShared {
    u64 sums[2][4], before[256];        // per thread: places on the line before its rows, the first of these
    RowInfo info[256];
};
// The line of blocks.  (All tiles of a row count with all its blocks: they are few here.)
struct NarrowLine {
    Cut cut;
    int heads, per;                     // kv heads; rows per thread
    Line line;
    Rows which;                         // its rows
    bool others;                        // whether there are others

    __device__ __forceinline__ int blocks_in(const RowInfo& x) const { return x.n ? (x.len + PAGE - 1) / PAGE : 0; }
    __device__ __forceinline__ u64 length_of(const RowInfo& x) const { return static_cast<u64>(x.tiles) * heads * blocks_in(x); }
};
// MIXED: there may be rows of more than one tile.
template <bool MIXED>
__device__ __forceinline__ NarrowLine narrow_line(const sparge_cache& c, const CacheAttn& a, NarrowShared& sh) {
    NarrowLine x;
    x.cut = cut_of(a.H / c.H_kv, NARROW_ROWS);
    x.heads = c.H_kv, x.per = (c.R + 255) / 256, x.which = ALL_ROWS, x.others = false;
    const int tid = threadIdx.x, r0 = tid * x.per, r1 = min(r0 + x.per, c.R);
    constexpr int N = MIXED ? 2 : 1;    // rows of one tile; of several
    u64 mine[N] = {}, total[N];
    auto add = [&](const RowInfo& row) {
        const u64 length = x.length_of(row);
        const bool one = !MIXED || row.n <= x.cut.TT;
        mine[0] += one ? length : 0;
        if constexpr (MIXED) mine[1] += one ? 0 : length;
    };
    RowInfo row0 = {0, 0, 0, 0, 0};
    if (r0 < r1) row0 = row_info(c, a, x.cut, ALL_ROWS, r0);
    add(row0);
#pragma unroll 1
    for (int r = r0 + 1; r < r1; ++r) add(row_info(c, a, x.cut, ALL_ROWS, r));
    prefix(mine, sh.sums, total);
    x.line.total = uniform(total[0]);
    if constexpr (MIXED) {
        const u64 more = uniform(total[1]);
        x.others = more && x.line.total + more > NARROW_BLOCKS << NARROW_LOG2;
        if (x.others) {
            x.which.upto = NARROW_ROWS;
            if (!x.which.hold(row0.n, x.cut.G)) row0.n = row0.tiles = 0;
        } else {
            x.line.total += more, mine[0] += mine[1];
        }
    }
    x.line.log2 = x.line.total >> NARROW_LOG2 ? NARROW_LOG2 : x.line.total ? 63 - __builtin_clzll(x.line.total) : 0;
    sh.before[tid] = mine[0], sh.info[tid] = row0;
    __syncthreads();
    return x;
}
template <int D, int DT>
__device__ __forceinline__ void narrow(const sparge_cache& c, const CacheAttn& a, const NarrowLine& rows, const uint16_t* __restrict__ Q,
                                       uint16_t* __restrict__ O, const Joint& ws, int bid, const NarrowShared& sh) {
    constexpr int NK = 4 * D / 64, NV = D / 16, KS = D / 32;
    const int tid = opaque(threadIdx.x), lane = tid & 63, wave = uniform(tid >> 6), heads = rows.heads;
    const Cut& cut = rows.cut;
    const Line& line = rows.line;
    const int parts = line.total ? 1 << line.log2 : 0, part = bid * 4 + wave;
    if (part >= parts) {
        if (lane == 0) ws.desc[part] = NO_JOIN;
        return;
    }
    // the next item's first block to take: row, of all heads' tiles the tile's number, block.  The row is one of the last thread's that
    // has no more than the part's beginning before it.
    const u64 lo = line.begin(part);
    int t = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) t += __builtin_popcountll(__ballot(sh.before[4 * lane + e] <= lo));
    int r = t * rows.per;
    u64 rem = lo - uniform(sh.before[t]);
    RowInfo info = uniform(sh.info[t]);
#pragma unroll 1
    while (rem >= rows.length_of(info) && r < c.R - 1) {
        rem -= rows.length_of(info);
        info = uniform(row_info(c, a, cut, rows.which, ++r));
    }
    int row_blocks = rows.blocks_in(info);
    u64 left = line.begin(part + 1) - lo;                     // blocks that this wave still has to take
    const u64 in_row = row_blocks ? quotient(rem, row_blocks) : 0;
    int b_next = static_cast<int>(rem - in_row * row_blocks);
    int head = info.tiles ? static_cast<int>(quotient(in_row, info.tiles)) : 0;
    int tile = static_cast<int>(in_row) - head * info.tiles;

    struct Item {
        RowInfo x;
        int row, kh, tile, ntok, b0, b1, blocks;
    };
    auto next_item = [&](Item& it) -> bool {
        if (left == 0) return false;
        if (b_next == row_blocks) {     // on to the next tile, head, row
            b_next = 0;
            if (++tile >= info.tiles) tile = 0, ++head;
            if (head >= heads) {
                head = 0;
                do {
                    if (++r >= c.R) return false;
                    info = uniform(row_info(c, a, cut, rows.which, r));
                    row_blocks = rows.blocks_in(info);
                } while (row_blocks == 0);
            }
        }
        it.x = info, it.row = r, it.tile = tile, it.blocks = row_blocks, it.b0 = b_next;
        it.kh = head;
        it.ntok = min(cut.TT, info.n - tile * cut.TT);
        const int take = static_cast<int>(min(static_cast<u64>(row_blocks - b_next), left));
        it.b1 = b_next += take;
        left -= take;
        return true;
    };

    Blocks blocks;
    uint4 q_raw[KS], kraw[NK], vraw[NV];
    int limit = -1, lim_lo = -1;        // of the item whose queries are in q_raw: the lane's row; the least of all rows
    int out_token = 0, out_head = 0;    // the lane's row of Q and O
    bool valid = false;
    auto open = [&](const Item& it) {
        const int row = lane & 15, tok = row / cut.G, g = row - tok * cut.G;
        valid = tok < it.ntok;
        const int t = it.tile * cut.TT;
        limit = !valid ? -1 : a.causal ? min(it.x.p0 + t + tok, it.x.len - 1) : it.x.len - 1;
        lim_lo = a.causal ? min(it.x.p0 + t, it.x.len - 1) : it.x.len - 1;
        const int lim_hi = a.causal ? min(it.x.p0 + t + it.ntok - 1, it.x.len - 1) : it.x.len - 1;
        blocks.open(c, a, it.row, it.kh, it.b0, min(it.b1, lim_hi / PAGE + 1));
        out_token = it.x.first + t + tok, out_head = it.kh * cut.G + g;
        load_q<D>(q_raw, Q + out_token * a.q_sn + out_head * a.q_sh + 16 * (lane >> 4), valid);
    };
    auto load_k = [&](int page, int kh) {
        const uint8_t* p = static_cast<const uint8_t*>(c.k) + (static_cast<long long>(page) * c.H_kv + kh) * (PAGE * D) + lane * 16;
#pragma unroll
        for (int n = 0; n < NK; ++n) kraw[n] = *reinterpret_cast<const uint4*>(p + n * 1024);
    };
    auto load_v = [&](int page, int kh) {
        const uint8_t* p = static_cast<const uint8_t*>(c.v) + (static_cast<long long>(page) * c.H_kv + kh) * (PAGE * D) + lane * 16;
#pragma unroll
        for (int n = 0; n < NV; ++n) vraw[n] = *reinterpret_cast<const uint4*>(p + n * 1024);
    };

    Item it;
    bool have = next_item(it), more = false;
    int block = 0, page = 0, at = 0;
    JoinDesc join = NO_JOIN;
    if (have) {
        open(it);
        if (it.b0 > 0)   // (worked out while the table is on its way)
            join = boundary(line, part, lo - it.b0, lo - it.b0 + it.blocks, it.x.first + it.tile * cut.TT, it.ntok, it.kh * cut.G);
        more = blocks.next(c, it.kh, block, page, at);
        if (more) {
            load_k(page, it.kh);
            load_v(page, it.kh);
        }
    }
    if (lane == 0) ws.desc[part] = join;
    while (have) {
        v8h qf[KS];
        const float qs = a.scale_log2 * convert_q<D, DT>(q_raw, qf);
        const int my_limit = limit - 4 * (lane >> 4), all_limit = lim_lo;
        const int my_token = out_token, my_head = out_head;
        const bool mine_valid = valid;
        v4f o[NV];
        float m = FAR, mo = FAR, l = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) o[n] = {0.f, 0.f, 0.f, 0.f};
        Item nx;
        bool n_have = false, asked = false, n_more = false;
        int n_block = 0, n_page = 0, n_at = 0;
        while (true) {
            v4f s[4];
            float ka = 0.f, va = 0.f;
            if (more) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    s[t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < D / 64; ++e) {
                        const uint4 w = kraw[t * (D / 64) + e];
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(w.x, w.y), qf[2 * e], s[t], 0, 0, 0);
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(w.z, w.w), qf[2 * e + 1], s[t], 0, 0, 0);
                    }
                }
                ka = blocks.ka(at), va = blocks.va(at);
            }
            // the next block: of this item, else of the next one
            n_more = blocks.next(c, it.kh, n_block, n_page, n_at);
            int n_kh = it.kh;
            if (!n_more) {
                asked = true;
                n_have = next_item(nx);
                if (n_have) {
                    n_kh = nx.kh;
                    open(nx);
                    n_more = blocks.next(c, n_kh, n_block, n_page, n_at);
                }
            }
            if (n_more) load_k(n_page, n_kh);
            if (more) {
                const bool bad = not_finite(ka, va);
                if (bad) ka = va = 0.f;
                // fp16 tokens: weights in two parts, as their rounding would show beside that of the results (relative error of four
                // masked rows of 100k keys 3.3e-4 in the place of 2.1e-4, which the results' rounding alone makes; bf16's is eight times
                // that).  It costs 2 us of 38 there.
                constexpr int NP = DT == SPARGE_F16 ? 4 : 2;
                v8h pf[NP];
                softmax<NV>(s, qs * (ka * (1.0f / 127.0f)), log2_of(va), block * PAGE + PAGE - 1 > all_limit, my_limit - block * PAGE, m, mo, l, o, pf);
                if (bad && my_limit + 4 * (lane >> 4) >= block * PAGE) l = nan_f();
#pragma unroll
                for (int n = 0; n < NV; ++n) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const v8h v = k ? codes8(vraw[n].z, vraw[n].w) : codes8(vraw[n].x, vraw[n].y);
                        o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pf[k], o[n], 0, 0, 0);
                        if constexpr (NP == 4) o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pf[2 + k], o[n], 0, 0, 0);
                    }
                }
            }
            if (n_more) load_v(n_page, n_kh);
            more = n_more, block = n_block, page = n_page, at = n_at;
            if (asked) break;
        }
        l = sum_groups(l);
        if (mine_valid) {
            const Mean mean(l, m, mo);
            if (it.b0 == 0 && it.b1 == it.blocks) {
                store_whole<NV, DT>(o, mean, O + my_token * a.o_sn + my_head * a.o_sh + 4 * (lane >> 4));
            } else {
                store_part<NV>(o, mean, m, l, ws, static_cast<long long>(2 * part + (it.b0 > 0 ? 0 : 1)) * NARROW_ROWS + (lane & 15));
            }
        }
        it = nx;
        have = n_have;
    }
}

// ---- many query rows: four waves share the blocks --------------------------------------------------------------------

__device__ __forceinline__ u64 sum_vis(const RowInfo& x, const Cut& t, bool causal, int i) {   // keys that the tiles before i see
    if (!causal) return static_cast<u64>(i) * x.len;
    u64 s = static_cast<u64>(i) * x.p0 + static_cast<u64>(t.TT) * i * (i + 1) / 2;
    if (i == x.tiles) s -= static_cast<u64>(x.tiles) * t.TT - x.n;   // the last tile may hold fewer tokens
    return s;
}

// A wave's 32 query rows as operands of the 32x32x16 MFMA: operand s holds channels 16 s + 8 (lane / 32) + 0..7 of row lane % 32.
template <int D, int DT>
__device__ __forceinline__ float convert_q32(const uint4 (&raw)[D / 16], v8h (&qf)[D / 16]) {
    if constexpr (DT == SPARGE_F16) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) __builtin_memcpy(&qf[s], &raw[s], 16);
        return 1.0f;
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) top = max(top, top16(raw[s]));
        top = max(top, __float_as_uint(other<32>(__uint_as_float(top))));
        const int ex = exponent16(top);
        const float down = __builtin_ldexpf(1.0f, -ex);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[s] = scaled8<DT>(raw[s], down);
        return __builtin_ldexpf(1.0f, ex);
    }
}

// No unit is full, at the clock that the power limit leaves: of a compute unit's cycles the vector ALU issues in 62 % (conversions,
// exponentials), the matrix pipe works in 43 %, LDS in 38 %, a seventh of that for bank conflicts; of their own cycles the two waves a
// SIMD issue in 48 %, wait to issue in 29 % and for memory, LDS or the others in 23 %.  3 rows of 700 to 2048 tokens over 4000 to 30000
// keys, 32 heads over 8: 540 GFLOP in 640 us with the join, 0.84 PFLOP/s, where a large bf16 product reaches 1.14.  (64 query rows a wave,
// one workgroup a compute unit, before the loop's order was laid down: 1147 us in the place of 917.)
// Four waves share the blocks: their codes are converted once per workgroup into LDS, in the operand order of the 32x32x16 MFMA
// (two buffers, one barrier a block; the raw bytes of the block after the next are on their way meanwhile), and every wave
// reads them for its own 32 query rows.  In that MFMA's accumulators a lane owns one query (lane % 32) and, of every 16 keys,
// 4 (lane / 32) + 0..3 and those + 8; V's operands are laid out for that order.
template <int D>
struct WideShared {
    u64 sums[1][4], rem;
    int row;
    RowInfo info;
    __align__(16) v8h k[2][2 * D / 16 * 64], v[2][D / 32 * 4 * 64];
};
// fp16: the weights of rows of up to TWO_ROWS query rows are in two parts, as in the narrow kernel: there reading pages counts for more than
// products (32 rows of one token, 32 heads a kv head: 47.1 us in the place of 45; prompts of 1000 tokens would take 840 us in the
// place of 650, and theirs are many rows: 1.25 times the error of the results' own rounding).  By the row, so that its bits and its
// cost do not depend on the other rows; the branches cost the prompts 1 %.  (The second part behind all products of the first, which read
// V's operands once more: 50.7 us.  Two copies of the loop: registers spill, twice the time.)
constexpr int TWO_ROWS = WIDE_ROWS / 2;
template <int D, int DT>
__device__ __forceinline__ void wide(const sparge_cache& c, const CacheAttn& a, const Rows& which, const uint16_t* __restrict__ Q, uint16_t* __restrict__ O,
                                     const Joint& ws, int bid, WideShared<D>& sh) {
    constexpr int KS = D / 16, NC = D / 32, RAW = D / 64;   // steps of K Q^T, channel tiles, 16-byte pieces of K (of V) per thread
    auto& lds_k = sh.k;
    auto& lds_v = sh.v;
    const int tid = opaque(threadIdx.x), lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
    const Cut cut = cut_of(a.H / c.H_kv, WIDE_ROWS);
    const int heads = c.H_kv;

    // ---- this workgroup's part of the line, in keys
    const int per = (c.R + 255) / 256;
    auto length_of = [&](const RowInfo& x) { return sum_vis(x, cut, a.causal, x.tiles); };
    Line line;
    const int r0 = tid * per, r1 = min(r0 + per, c.R);
    RowInfo row0 = {0, 0, 0, 0, 0};
    if (r0 < r1) row0 = row_info(c, a, cut, which, r0);
    u64 mine = length_of(row0) * heads;
#pragma unroll 1
    for (int r = r0 + 1; r < r1; ++r) mine += length_of(row_info(c, a, cut, which, r)) * heads;
    u64 upto[1] = {mine}, total[1];
    prefix(upto, sh.sums, total);
    const u64 before = upto[0];
    line.total = uniform(total[0]);
    // parts of at least two blocks; neighbours on the line, which share pages, are neighbours on an XCD
    const u64 wanted = line.total / (2 * PAGE);
    line.log2 = wanted >> WIDE_LOG2 ? WIDE_LOG2 : wanted ? 63 - __builtin_clzll(wanted) : 0;
    const int parts = line.total ? 1 << line.log2 : 0;
    if (bid >= parts) {
        if (tid == 0) ws.desc[bid] = NO_JOIN;
        return;
    }
    const int part = parts >= 8 ? (bid & 7) * (parts >> 3) + (bid >> 3) : bid;
    const u64 lo = line.begin(part);
    if (before <= lo && lo < before + mine) {
        u64 rem = lo - before;
        int r = r0;
        RowInfo x = row0;
#pragma unroll 1
        while (rem >= length_of(x) * heads && r < c.R - 1) {
            rem -= length_of(x) * heads;
            x = row_info(c, a, cut, which, ++r);
        }
        sh.row = r, sh.rem = rem, sh.info = x;
    }
    __syncthreads();
    int r = uniform(sh.row);
    RowInfo x = uniform(sh.info);
    u64 left = line.begin(part + 1) - lo;                     // keys that this workgroup still has to take
    JoinDesc join = NO_JOIN;
    // where it begins: head, tile, key
    const u64 rem = uniform(sh.rem), chunk = max(length_of(x), static_cast<u64>(1));
    int head = static_cast<int>(quotient(rem, chunk)), i = 0;
    const u64 in = rem - head * chunk;
#pragma unroll 1
    for (int up = x.tiles; up - i > 1;) {
        const int mid = (i + up) >> 1;
        if (sum_vis(x, cut, a.causal, mid) <= in) i = mid; else up = mid;
    }
    int x0 = static_cast<int>(in - sum_vis(x, cut, a.causal, i));

    while (left > 0) {
        const int ntok = min(cut.TT, x.n - i * cut.TT), token0 = x.first + i * cut.TT;
        const int kh = head;
        const int vis = a.causal ? x.p0 + i * cut.TT + ntok : x.len;
        const int take = static_cast<int>(min(static_cast<u64>(vis - x0), left)), x1 = x0 + take;
        const int b0 = x0 / PAGE, b1 = x1 == vis ? (vis + PAGE - 1) / PAGE : x1 / PAGE;
        const bool whole = x0 == 0 && x1 == vis, is_first = left == line.begin(part + 1) - lo;
        if (is_first && x0 > 0) join = boundary(line, part, lo - x0, lo - x0 + vis, token0, ntok, kh * cut.G);

        // this wave's rows, the lane's one of them, and the least and the largest key that a row sees last
        const int n_rows = ntok * cut.G, w0 = wave * 32, w1 = min(w0 + 32, n_rows) - 1;
        const int row = w0 + (lane & 31), tok = row / cut.G, g = row - tok * cut.G;
        const bool valid = row < n_rows;
        const int first_limit = a.causal ? x.p0 + i * cut.TT : x.len - 1;
        const int limit = !valid ? -1 : min(first_limit + (a.causal ? tok : 0), x.len - 1);
        const int lim_lo = min(first_limit + (a.causal ? w0 / cut.G : 0), x.len - 1);
        const int lim_hi = w1 < w0 ? -1 : min(first_limit + (a.causal ? w1 / cut.G : 0), x.len - 1);
        Blocks blocks;
        blocks.open(c, a, r, kh, b0, min(b1, (x.len + PAGE - 1) / PAGE));
        const long long token = token0 + tok, hd = kh * cut.G + g;
        uint4 q_raw[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q_raw[s] = make_uint4(0u, 0u, 0u, 0u);
            if (valid) q_raw[s] = *reinterpret_cast<const uint4*>(Q + token * a.q_sn + hd * a.q_sh + 16 * s + 8 * half);
        }

        uint4 kraw[RAW] = {}, vraw[RAW] = {};
        auto load_raw = [&](int page) {
            const long long at = (static_cast<long long>(page) * c.H_kv + kh) * (PAGE * D) + tid * 16;
#pragma unroll
            for (int n = 0; n < RAW; ++n) {
                kraw[n] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(c.k) + at + n * 4096);
                vraw[n] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(c.v) + at + n * 4096);
            }
        };
        // a quarter of a thread's pieces n (K's first and second half, V's first and second) into LDS
        constexpr int CHUNKS = 4 * RAW;
        auto convert_chunk = [&](int buf, int chunk) {
            const int l16 = lane & 15, gr = lane >> 4, n = chunk >> 2, which = chunk & 3, piece = wave + 4 * n;
            if (which < 2) {
                // K: keys 16 t + l16, channels 64 e + 16 gr + 0..15: step 4 e + gr of key tile t / 2, eight channels a half
                const int t = piece / (D / 64), e = piece - t * (D / 64);
                lds_k[buf][((t >> 1) * KS + 4 * e + gr) * 64 + 16 * (t & 1) + l16 + 32 * which] =
                    which ? codes8(kraw[n].z, kraw[n].w) : codes8(kraw[n].x, kraw[n].y);
            } else {
                // V: channel 16 piece + l16, keys 16 t + 4 gr + 0..3 in word t: step t, half gr % 2, place 4 (gr / 2)
                uint2* v = reinterpret_cast<uint2*>(&lds_v[buf][(piece >> 1) * 4 * 64 + 16 * (piece & 1) + l16 + 32 * (gr & 1)]) + (gr >> 1);
                const v8h two = which == 2 ? codes8(vraw[n].x, vraw[n].y) : codes8(vraw[n].z, vraw[n].w);
                uint4 w;
                __builtin_memcpy(&w, &two, 16);
                v[256 * (which - 2)] = make_uint2(w.x, w.y);
                v[256 * (which - 2) + 128] = make_uint2(w.z, w.w);
            }
        };
        auto convert = [&](int buf) {
#pragma unroll
            for (int x = 0; x < CHUNKS; ++x) convert_chunk(buf, x);
        };
        int block = 0, page = 0, at = 0, n_block = 0, n_at = 0;
        float ka = 0.f, va = 0.f, n_ka = 0.f, n_va = 0.f;
        bool more = blocks.next(c, kh, block, page, at), n_more = false;
        if (more) {
            load_raw(page);
            ka = blocks.ka(at), va = blocks.va(at);
        }
        v8h qf[KS];
        const float qs = a.scale_log2 * (1.0f / 127.0f) * convert_q32<D, DT>(q_raw, qf);
        float m = FAR, mo = FAR, l = 0.f;
        v16f o[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[n][e] = 0.f;
        if (more) {
            convert(0);
            n_more = blocks.next(c, kh, n_block, page, n_at);
            if (n_more) {
                load_raw(page);
                n_ka = blocks.ka(n_at), n_va = blocks.va(n_at);
            }
        }
        __syncthreads();
        // Scores of a block beside the conversion of the next one, and, in weigh, O beside the weights.  The order is laid down
        // (nothing crosses the sched_barriers): operands are read four products ahead; left to itself the compiler reads
        // one, waits for it and issues its product.
        v16f s[2];
        auto scores = [&](int buf) {
            v8h k[4];
            auto operand = [&](int x) { return lds_k[buf][((x & 1) * KS + (x >> 1)) * 64 + lane]; };
#pragma unroll
            for (int x = 0; x < 4; ++x) k[x] = operand(x);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < 2 * KS; ++x) {
                s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[x & 3], qf[x >> 1], s[x & 1], 0, 0, 0);
                if (x + 4 < 2 * KS) k[x & 3] = operand(x + 4);
                if (x & 1) convert_chunk(buf ^ 1, x >> 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            static_assert(CHUNKS == KS, "a chunk for every other product");
        };
        const bool two = DT == SPARGE_F16 && static_cast<long long>(x.n) * cut.G <= TWO_ROWS;
        auto weigh = [&](bool masked, int buf) {
            float cq = qs * ka;
            if (cq == 0.f) cq = 1e-37f;   // a block of zeros: -inf stays what it is and becomes a weight of 0
            const int last = limit - block * PAGE - 4 * half;   // key 32 t + 8 (e / 4) + e % 4 of the lane's
            if (masked) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * t + 8 * (e >> 2) + (e & 3) > last) s[t][e] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
            top = fmaxf(top, other<32>(top)) * cq;
            const float v_log2 = log2_of(va);
            if (__any(top > m + SLACK || top + v_log2 > mo + SLACK)) {
                const float to = fmaxf(m, top), o_to = fmaxf(mo, top + v_log2), down = __builtin_amdgcn_exp2f(mo - o_to);
                l *= __builtin_amdgcn_exp2f(m - to);
                m = to, mo = o_to;
#pragma unroll
                for (int n = 0; n < NC; ++n) o[n] *= down;
            }
            const float add = weight_log2(v_log2, mo, top);
            float sum = 0.f;
            v8h pf[4], v[4], rest;
            auto weights = [&](int u, int e) {   // two of the eight of step u
#pragma unroll
                for (int k = e; k < e + 2; ++k) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][8 * (u & 1) + k], cq, add));
                    s[u >> 1][8 * (u & 1) + k] = w;
                    sum += w;   // before its rounding: w carries V's scale, which may be small
                    pf[u][k] = static_cast<_Float16>(w);
                }
                asm volatile("" : "+v"(sum));   // here, not all of them behind the last product
            };
            auto operand = [&](int x) { return lds_v[buf][((x % NC) * 4 + x / NC) * 64 + lane]; };
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = operand(x);
#pragma unroll
            for (int e = 0; e < 8; e += 2) weights(0, e);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < 4 * NC; ++x) {
                const int u = x / NC, n = x % NC;
                o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[x & 3], pf[u], o[n], 0, 0, 0);
                if (two) {   // what the weights' rounding left
                    if (n == 0) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) rest[k] = static_cast<_Float16>(s[u >> 1][8 * (u & 1) + k] - static_cast<float>(pf[u][k]));
                    }
                    o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[x & 3], rest, o[n], 0, 0, 0);
                }
                if (x + 4 < 4 * NC) v[x & 3] = operand(x + 4);
                if (u < 3) {
#pragma unroll
                    for (int e = 8 / NC * n; e < 8 / NC * (n + 1); e += 2) weights(u + 1, e);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            l += sum * weight_back(add, m);
        };
        for (int buf = 0; more; buf ^= 1) {
            // the next block's bytes into the other buffer (nobody reads it; behind the last block whatever is there), the one
            // after it on its way
            const bool mine = block * PAGE <= lim_hi;
            if (mine) {
                scores(buf);
            } else {
#pragma unroll
                for (int n = 0; n < RAW; ++n)   // (that the two conversions have nothing to be drawn together from)
                    asm volatile("" : "+v"(kraw[n].x), "+v"(kraw[n].y), "+v"(kraw[n].z), "+v"(kraw[n].w), "+v"(vraw[n].x), "+v"(vraw[n].y),
                                 "+v"(vraw[n].z), "+v"(vraw[n].w));
                convert(buf ^ 1);
            }
            int nn_block = 0, nn_at = 0;
            float nn_ka = 0.f, nn_va = 0.f;
            const bool nn_more = n_more && blocks.next(c, kh, nn_block, page, nn_at);
            if (nn_more) {
                load_raw(page);
                nn_ka = blocks.ka(nn_at), nn_va = blocks.va(nn_at);
            }
            if (mine) {
                const bool bad = not_finite(ka, va);
                if (bad) ka = va = 0.f;
                weigh(block * PAGE + PAGE - 1 > lim_lo, buf);
                if (bad && limit >= block * PAGE) l = nan_f();
            }
            lds_barrier();
            more = n_more, block = n_block, ka = n_ka, va = n_va;
            n_more = nn_more, n_block = nn_block, n_ka = nn_ka, n_va = nn_va;
        }

        l += other<32>(l);
        if (valid) {
            const Mean mean(l, m, mo);
            uint16_t* out = O + token * a.o_sn + hd * a.o_sh + 4 * half;
            const long long row_at = static_cast<long long>(2 * part + (x0 > 0 ? 0 : 1)) * WIDE_ROWS + row;
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // channels 32 n + 8 e + 4 half + 0..3
                    v4f y;
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = mean(o[n][4 * e + k]);
                    if (whole) {
                        uint16_t h[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) h[k] = cvt_to16<DT>(y[k]);
                        uint2 w;
                        __builtin_memcpy(&w, h, 8);
                        *reinterpret_cast<uint2*>(out + 32 * n + 8 * e) = w;
                    } else {
                        *reinterpret_cast<v4f*>(ws.o + row_at * D + 32 * n + 8 * e + 4 * half) = y;
                    }
                }
            if (!whole && half == 0) ws.ml[2 * row_at] = m, ws.ml[2 * row_at + 1] = l;
        }
        // on to the next tile, head, row
        left -= take;
        x0 = 0;
        if (++i >= x.tiles) i = 0, ++head;
        if (head >= heads && left > 0) {
            head = 0;
            do {
                if (++r >= c.R) left = 0;     // (cannot be: the line ends with the rows)
                else x = uniform(row_info(c, a, cut, which, r));
            } while (left > 0 && x.n == 0);
        }
    }
    if (tid == 0) ws.desc[bid] = join;
}

// ---- the launches: rows of the one kind, of the other, or of both
template <int D, int DT>
__global__ __launch_bounds__(256, 2) void cache_attn_narrow_kernel(sparge_cache c, CacheAttn a, const uint16_t* __restrict__ Q, uint16_t* __restrict__ O, Joint ws) {
    __shared__ NarrowShared sh;
    const NarrowLine rows = narrow_line<false>(c, a, sh);
    narrow<D, DT>(c, a, rows, Q, O, ws, blockIdx.x, sh);
}
template <int D, int DT>
__global__ __launch_bounds__(256, 2) void cache_attn_wide_kernel(sparge_cache c, CacheAttn a, const uint16_t* __restrict__ Q, uint16_t* __restrict__ O, Joint ws) {
    __shared__ WideShared<D> sh;
    wide<D, DT>(c, a, ALL_ROWS, Q, O, ws, blockIdx.x, sh);
}
template <int D, int DT>
__global__ __launch_bounds__(256, 2) void cache_attn_both_kernel(sparge_cache c, CacheAttn a, const uint16_t* __restrict__ Q, uint16_t* __restrict__ O,
                                                                 Joint ws_wide, Joint ws_narrow) {
    __shared__ NarrowShared sh;
    __shared__ WideShared<D> sh_wide;
    static_assert(WIDE_WGS == NARROW_WGS, "a workgroup has a part of either line");
    // the wide part first: where it has ended, the narrow one's four waves end each by itself
    const NarrowLine rows = narrow_line<true>(c, a, sh);
    if (rows.others) wide<D, DT>(c, a, Rows{NARROW_ROWS, ALL_ROWS.upto}, Q, O, ws_wide, blockIdx.x, sh_wide);
    else if (threadIdx.x == 0) ws_wide.desc[blockIdx.x] = NO_JOIN;
    narrow<D, DT>(c, a, rows, Q, O, ws_narrow, blockIdx.x, sh);
}

// ---- join ----------------------------------------------------------------------------------------------------------

// Joins items that several parts hold, each in its parts' order.  An item's rows are cut into chunks of channels, which the waves
// of the parts that begin inside the item deal out among them.  A wave's lanes take 4 channels each of 256 / PG, and the
// PG groups of lanes every PG-th part, up to eight of them in one round trip to memory.  What is joined are means of the values, with
// weights that add up to 1: no sum leaves fp32's range where the result does not.
template <int D, int DT, int ROWS, int PG>
__device__ __forceinline__ void join_item(const JoinDesc& d, int me, int workers, int G, const CacheAttn& a, uint16_t* O, const Joint& ws) {
    constexpr int LANES = 64 / PG;
    const int lane = threadIdx.x & 63, grp = lane / LANES, n_chunks = (d.n_tok * G * D * PG + 255) / 256;
    for (int chunk = me; chunk < n_chunks; chunk += workers) {
        const int flat = chunk * (256 / PG) + (lane % LANES) * 4, row = flat / D, ch = flat % D;
        const int tok = row / G, g = row - tok * G;
        const bool there = tok < d.n_tok;
        float m = FAR, l = 0.f;
        v4f o = {0.f, 0.f, 0.f, 0.f};
        for (int k0 = grp; k0 < d.n_parts; k0 += 8 * PG) {
            float pm[8], pl[8];
            v4f po[8];
            float top = m;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = k0 + e * PG;
                pm[e] = FAR, pl[e] = 0.f, po[e] = {0.f, 0.f, 0.f, 0.f};
                if (there && k < d.n_parts) {
                    // the item's start is the second result of the part before the first boundary, the rest are first results
                    const long long at = static_cast<long long>(k == 0 ? 2 * (d.first - 1) + 1 : 2 * (d.first + k - 1)) * ROWS + row;
                    pm[e] = ws.ml[2 * at], pl[e] = ws.ml[2 * at + 1];
                    po[e] = *reinterpret_cast<const v4f*>(ws.o + at * D + ch);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, pm[e]);
            const float before = l * __builtin_amdgcn_exp2f(m - top);
            l = before, m = top;
#pragma unroll
            for (int e = 0; e < 8; ++e) pl[e] *= __builtin_amdgcn_exp2f(pm[e] - top), l += pl[e];
            const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);
            o *= before * inv;
#pragma unroll
            for (int e = 0; e < 8; ++e) o += po[e] * (pl[e] * inv);
        }
#pragma unroll
        for (int x = LANES; x < 64; x <<= 1) {
            const float om = __shfl_xor(m, x), ol = __shfl_xor(l, x), top = fmaxf(m, om);
            const float la = l * __builtin_amdgcn_exp2f(m - top), lb = ol * __builtin_amdgcn_exp2f(om - top);
            l = la + lb, m = top;
            const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = o[e] * (la * inv) + __shfl_xor(o[e], x) * (lb * inv);
        }
        if (there && grp == 0) {
            uint16_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = cvt_to16<DT>(o[e]);
            uint2 w;
            __builtin_memcpy(&w, h, 8);
            *reinterpret_cast<uint2*>(O + static_cast<long long>(d.token + tok) * a.o_sn + static_cast<long long>(d.head + g) * a.o_sh + ch) = w;
        }
    }
}
// WAVES: of a workgroup, for one description
template <int D, int DT, int ROWS, int WAVES>
__device__ __forceinline__ void join(const sparge_cache& c, const CacheAttn& a, uint16_t* O, const Joint& ws, int bid) {
    const int wave = uniform(static_cast<int>(threadIdx.x) >> 6);
    const JoinDesc d = ws.desc[(bid * 4 + wave) / WAVES];
    if (d.n_parts == 0) return;
    const int G = a.H / c.H_kv, me = (d.part - d.first) * WAVES + wave % WAVES, workers = (d.n_parts - 1) * WAVES;
    // as many groups of lanes as bring an item's parts in with one round trip, while its waves have chunks enough
    if (d.n_parts <= 4) join_item<D, DT, ROWS, 1>(d, me, workers, G, a, O, ws);
    else if (d.n_parts <= 64) join_item<D, DT, ROWS, 8>(d, me, workers, G, a, O, ws);
    else join_item<D, DT, ROWS, 32>(d, me, workers, G, a, O, ws);
}
// the first n_narrow workgroups take the narrow kernel's parts, the others the wide one's
template <int D, int DT>
__global__ __launch_bounds__(256) void cache_join_kernel(sparge_cache c, CacheAttn a, int n_narrow, uint16_t* __restrict__ O, Joint ws_wide, Joint ws_narrow) {
    const int bid = blockIdx.x;
    if (bid < n_narrow) join<D, DT, NARROW_ROWS, 1>(c, a, O, ws_narrow, bid);
    else join<D, DT, WIDE_ROWS, 4>(c, a, O, ws_wide, bid - n_narrow);
}

// ---- host ------------------------------------------------------------------------------------------------------------

// The workspace, once per kernel: descriptions, references and sums, partial rows.
struct Layout {
    size_t desc[2], ml[2], o[2], total;   // wide, narrow
};
Layout layout_of(int d) {
    const size_t parts[2] = {1u << WIDE_LOG2, 1u << NARROW_LOG2}, rows[2] = {2 * parts[0] * WIDE_ROWS, 2 * parts[1] * NARROW_ROWS};
    Layout x;
    size_t at = 0;
    for (int k = 0; k < 2; ++k) {
        x.desc[k] = at, at += parts[k] * sizeof(JoinDesc);
        x.ml[k] = at, at += rows[k] * 2 * sizeof(float);
        x.o[k] = at, at += rows[k] * d * sizeof(float);
    }
    x.total = at;
    return x;
}

template <int D, int DT>
void launch(const sparge_cache& c, const CacheAttn& a, bool narrow, bool wide, const void* Qp, void* Op, const Joint (&j)[2], hipStream_t st) {
    const uint16_t* Q = static_cast<const uint16_t*>(Qp);
    uint16_t* O = static_cast<uint16_t*>(Op);
    if (narrow && wide) hipLaunchKernelGGL((cache_attn_both_kernel<D, DT>), dim3(WIDE_WGS), dim3(256), 0, st, c, a, Q, O, j[0], j[1]);
    else if (wide) hipLaunchKernelGGL((cache_attn_wide_kernel<D, DT>), dim3(WIDE_WGS), dim3(256), 0, st, c, a, Q, O, j[0]);
    else hipLaunchKernelGGL((cache_attn_narrow_kernel<D, DT>), dim3(NARROW_WGS), dim3(256), 0, st, c, a, Q, O, j[1]);
    const int n_wide = wide ? WIDE_WGS : 0, n_narrow = narrow ? NARROW_WGS : 0;
    hipLaunchKernelGGL((cache_join_kernel<D, DT>), dim3(n_wide + n_narrow), dim3(256), 0, st, c, a, n_narrow, O, j[0], j[1]);
}

}  // namespace

size_t cache_attn_workspace(int d) { return layout_of(d).total; }

hipError_t launch_cache_attn(const sparge_cache& c, const CacheAttn& a, const void* Q, void* O, void* ws, hipStream_t st) {
    const Layout x = layout_of(c.d);
    char* p = static_cast<char*>(ws);
    Joint j[2];
    for (int k = 0; k < 2; ++k)
        j[k] = {reinterpret_cast<JoinDesc*>(p + x.desc[k]), reinterpret_cast<float*>(p + x.ml[k]), reinterpret_cast<float*>(p + x.o[k])};
    // How many tokens each row adds is not known here.  Groups beyond a wave's 16 rows are the wide kernel's (16 rows, 8 queries a head: narrow
    // 26 us, wide 36; 16 queries: 30 and 38).  The narrow kernel alone runs where no row can have more than a tile; a single row's
    // tokens are the wide kernel's from half a tile on (9000 keys, 4 queries a head: 2 tokens narrow 17.8 us, wide 18.1; 4 tokens 22.3
    // and 18.6; 8 tokens 27.2 and 18.9).  Else one kernel holds both, which costs a step of single tokens 0.1 to 0.9 us, and shares
    // the rows out on the device (255 rows of one token beside one of 1500 over 30000 keys, 1 query a head: 549 us, the narrow kernel
    // alone 1059; one row of 500 tokens over 9000 keys among 511 idle ones: 141 and 267).
    const long long G = a.H / c.H_kv, most = a.n_slots * G;
    const bool few = c.R > 1 ? most <= NARROW_ROWS : a.n_slots == 1 || most <= NARROW_ROWS / 2;
    const bool narrow = G <= NARROW_ROWS && (few || c.R > 1), wide = G > NARROW_ROWS || !few;
#define RUN(D, DT) launch<D, DT>(c, a, narrow, wide, Q, O, j, st)
    if (c.d == 64) {
        if (c.dtype == SPARGE_F16) RUN(64, SPARGE_F16); else RUN(64, SPARGE_BF16);
    } else {
        if (c.dtype == SPARGE_F16) RUN(128, SPARGE_F16); else RUN(128, SPARGE_BF16);
    }
#undef RUN
    return hipGetLastError();
}

}  // namespace sparge
