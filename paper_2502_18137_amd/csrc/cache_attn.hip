// Attention of new tokens over the paged 8-bit K/V cache.
//
// O_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i . k_j - m_i), in one pass over the keys.  With codes a, b (integers) and a
// block's scales sk, sv: q_i . k_j = sk (q_i . a_j) and v_j = sv b_j.  Both products run on the 16-bit MFMA with the codes as
// fp16 integers (exact), S^T = A Q^T and O^T = B^T P^T, so that a lane owns one query (lane % 16) and four keys of every
// sixteen, and P goes from the accumulators of the first product to the operand of the second without leaving the lane:
// the pages' byte order is made for that, and operands are loaded from memory into registers, 1 KB per wave and load,
// without LDS.  sk enters the exponent; sv enters p before it is rounded, relative to the largest sv so far, to which O
// is kept relative.
//
// Work: an item is a kv head's group of up to 64 QT query rows (tokens x grouped heads) of one row of the cache, weighed by the keys
// it sees and the waves it needs.  The items lie one behind the other on a line that is cut into equal parts, one per
// workgroup: a long item is split over several, whose partial results a second launch joins in a fixed order, and a
// short one shares a workgroup with others.  Where the rows of an item fit 16 QT (32 QT), its four (two) waves take
// every fourth (second) kept block instead of rows.
#include "cache.hpp"

namespace sparge {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr float FAR = -1e30f;          // reference of a row that has seen no key
constexpr float SLACK = 4.0f;          // log2: how far a row's maximum may run ahead of the reference inside exp2
constexpr float SV_SLACK = 4.0f;       // how far a block's V scale may exceed the one that O is relative to
constexpr float P_UP = 256.0f;         // p is at most 2^4, its factor sv ratio at most 4: p x ratio x 2^8 <= 2^14 in fp16, and
                                       // weights down to 2^-33 of the largest are not lost

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

// How a row of the cache is cut: Gp grouped heads a tile holds (the group, or a part of it where it exceeds a workgroup), TT tokens.
struct Cut {
    int G, Gp, parts, TT;
};
__host__ __device__ inline Cut cut_of(int G, int rows) {
    if (G <= rows) return {G, G, 1, rows / G};
    return {G, rows, (G + rows - 1) / rows, 1};
}

struct RowInfo {
    int first, n, len, p0;     // new tokens [first, first + n), keys, keys before the first new token
    int tiles, rg;             // tiles of TT tokens; waves over rows
    u64 chunk;                 // weight of one kv head's part
};
__device__ __forceinline__ u64 sum_vis(const RowInfo& x, const Cut& t, bool causal, int i) {   // keys that the tiles before i see
    if (!causal) return static_cast<u64>(i) * x.len;
    u64 s = static_cast<u64>(i) * x.p0 + static_cast<u64>(t.TT) * i * (i + 1) / 2;
    if (i == x.tiles) s -= static_cast<u64>(x.tiles) * t.TT - x.n;   // the last tile may hold fewer tokens
    return s;
}
template <int QT>
__device__ __forceinline__ RowInfo row_info(const sparge_cache& c, const CacheAttn& a, const Cut& t, int r) {
    RowInfo x;
    x.first = max(0, min(a.cu[r], a.n_slots));
    x.n = max(0, min(a.cu[r + 1], a.n_slots) - x.first);
    x.len = max(0, min(c.length[r], static_cast<int>(min(static_cast<long long>(c.max_blocks) * PAGE, 0x7FFFFFC0ll))));
    x.p0 = max(0, x.len - x.n);
    x.tiles = (x.n + t.TT - 1) / t.TT;
    const int rows = min(x.n, t.TT) * t.Gp;
    x.rg = rows <= 16 * QT ? 1 : rows <= 32 * QT ? 2 : 4;
    x.chunk = x.rg * sum_vis(x, t, a.causal, x.tiles);
    return x;
}

__device__ __forceinline__ u64 uniform(u64 v) {
    return static_cast<u64>(__builtin_amdgcn_readfirstlane(static_cast<int>(v >> 32))) << 32 |
           static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
}

struct Joint {                          // workspace
    JoinDesc* desc;                     // [CACHE_WGS]
    float* ml;                          // [2 CACHE_WGS][CACHE_WG_ROWS][2] reference and sum of a row's part
    float* o;                           // [2 CACHE_WGS][CACHE_WG_ROWS][d]
};

template <int D, int DT, int QT>
__global__ __launch_bounds__(256, 2) void cache_attn_kernel(sparge_cache c, CacheAttn a, const uint16_t* __restrict__ Q,
                                                            uint16_t* __restrict__ O, Joint ws) {
    constexpr int NK = 4 * D / 64, NV = D / 16, KS = D / 32, ROWS = 64 * QT;
    static_assert(ROWS <= CACHE_WG_ROWS, "a part has room for that many rows");
    __shared__ u64 sums[4];
    __shared__ u64 found[2];
    __shared__ __align__(16) float merge[3][QT][D * 16 + 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.H / c.H_kv;
    const Cut cut = cut_of(G, ROWS);

    // ---- this workgroup's part of the line
    const int per = (c.R + 255) / 256;
    u64 mine = 0;
    for (int r = tid * per; r < min((tid + 1) * per, c.R); ++r) mine += row_info<QT>(c, a, cut, r).chunk;
    mine *= static_cast<u64>(c.H_kv) * cut.parts;
    u64 upto = mine;
    for (int s = 1; s < 64; s <<= 1) {
        const u64 x = __shfl_up(upto, s);
        if (lane >= s) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    u64 total = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) upto += sums[w];
        total += sums[w];
    }
    // equal parts of at least 256 weights (a block for each wave); a multiple of 8, so that neighbours on the line, which share
    // pages, are neighbours on an XCD
    const u64 wanted = total / 256;
    int parts = wanted >= CACHE_WGS ? CACHE_WGS : wanted >= 8 ? static_cast<int>(wanted) & ~7 : wanted >= 1 ? static_cast<int>(wanted) : total > 0;
    const int bid = blockIdx.x;
    if (bid >= parts) {
        if (tid == 0) ws.desc[bid].n_parts = 0;
        return;
    }
    const int part = parts >= 8 ? (bid & 7) * (parts / 8) + (bid >> 3) : bid;
    const u64 lo = uniform(total * part / parts), hi = uniform(total * (part + 1) / parts);
    if (upto - mine <= lo && lo < upto) {
        u64 rem = lo - (upto - mine);
        int r = tid * per;
        for (; r < c.R - 1; ++r) {
            const u64 all = row_info<QT>(c, a, cut, r).chunk * c.H_kv * cut.parts;
            if (rem < all) break;
            rem -= all;
        }
        found[0] = r;
        found[1] = rem;
    }
    __syncthreads();
    int r = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
    u64 rem = uniform(found[1]), pos = uniform(lo);
    bool joins = false;

    while (pos < hi && r < c.R) {
        RowInfo x = row_info<QT>(c, a, cut, r);
        x.first = __builtin_amdgcn_readfirstlane(x.first), x.n = __builtin_amdgcn_readfirstlane(x.n);
        x.len = __builtin_amdgcn_readfirstlane(x.len), x.p0 = __builtin_amdgcn_readfirstlane(x.p0);
        x.tiles = __builtin_amdgcn_readfirstlane(x.tiles), x.rg = __builtin_amdgcn_readfirstlane(x.rg);
        x.chunk = uniform(x.chunk);
        if (rem >= x.chunk * c.H_kv * cut.parts) {
            rem -= x.chunk * c.H_kv * cut.parts;
            ++r;
            continue;
        }
        const int head = static_cast<int>(rem / x.chunk);   // kv head and part of its group
        const u64 in = rem - head * x.chunk;
        int i = 0;
        for (int up = x.tiles; up - i > 1;) {
            const int mid = (i + up) >> 1;
            if (x.rg * sum_vis(x, cut, a.causal, mid) <= in) i = mid; else up = mid;
        }
        const u64 x0 = in - x.rg * sum_vis(x, cut, a.causal, i);
        const int ntok = min(cut.TT, x.n - i * cut.TT);
        const int vis = a.causal ? x.p0 + i * cut.TT + ntok : x.len;
        const u64 item = static_cast<u64>(x.rg) * vis;
        const u64 take = min(item - x0, hi - pos), x1 = x0 + take;
        const int b0 = static_cast<int>(x0 / x.rg) / PAGE;
        const int b1 = x1 == item ? (vis + PAGE - 1) / PAGE : static_cast<int>(x1 / x.rg) / PAGE;
        const bool whole = x0 == 0 && x1 == item;
        if (pos == lo && x0 > 0) {
            // a boundary inside an item; the item's first one has it joined
            const u64 start = lo - x0, end = start + item;
            const bool is_first = total * (part - 1) / parts <= start;
            joins = is_first;
            if (tid == 0 && is_first) {
                const u64 last = (end * parts + total - 1) / total - 1;   // the last boundary before the item's end
                ws.desc[bid] = {static_cast<int>(last) - part + 2, part, r, head, i};
            }
        }

        // ---- one item's blocks [b0, b1)
        const int kh = head / cut.parts, gpart = head - kh * cut.parts;
        const int rg = x.rg, kg = 4 / rg, my_rg = wave & (rg - 1), my_kg = wave / rg;
        const int n_rows = ntok * cut.Gp;
        const int row0 = my_rg * 16 * QT + (lane & 15);
        int limit[QT];
        long long q_at[QT];
        bool valid[QT];
        int lim_lo = 0x7FFFFFFF, lim_hi = -1;
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int row = row0 + 16 * q, tok = row / cut.Gp, g = gpart * ROWS + row - tok * cut.Gp;
            valid[q] = row < n_rows && g < G;
            limit[q] = !valid[q] ? -1 : a.causal ? min(x.p0 + i * cut.TT + tok, x.len - 1) : x.len - 1;
            q_at[q] = static_cast<long long>(x.first + i * cut.TT + tok);
            if (valid[q]) lim_lo = min(lim_lo, limit[q]);
            lim_hi = max(lim_hi, limit[q]);
        }
        for (int s = 1; s < 16; s <<= 1) {
            lim_lo = min(lim_lo, __shfl_xor(lim_lo, s));
            lim_hi = max(lim_hi, __shfl_xor(lim_hi, s));
        }
        lim_lo = __builtin_amdgcn_readfirstlane(lim_lo);
        lim_hi = __builtin_amdgcn_readfirstlane(lim_hi);

        // Q: fp16 as it is; bf16 times the power of two that brings the row's largest to [1, 2) (exact but for what is below
        // 2^-24 of it).  An operand holds, of channels 64 s + 16 (lane / 16) + 8 u + 0..7, the one of step 2 s + u.
        v8h qf[QT][KS];
        float qs[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int row = row0 + 16 * q, tok = row / cut.Gp, g = gpart * ROWS + row - tok * cut.Gp;
            uint4 raw[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                raw[s] = make_uint4(0u, 0u, 0u, 0u);
                if (valid[q])
                    raw[s] = *reinterpret_cast<const uint4*>(Q + q_at[q] * a.q_sn + static_cast<long long>(kh * G + g) * a.q_sh +
                                                             64 * (s >> 1) + 16 * (lane >> 4) + 8 * (s & 1));
            }
            qs[q] = a.scale_log2;
            if constexpr (DT == SPARGE_F16) {
#pragma unroll
                for (int s = 0; s < KS; ++s) __builtin_memcpy(&qf[q][s], &raw[s], 16);
            } else {
                uint32_t top = 0;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const uint32_t w[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7FFFu, (w[e] >> 16) & 0x7FFFu));
                }
                top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16)));
                top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
                int ex = static_cast<int>(top >> 7) - 127;          // exponent of the largest (top: bf16 bits)
                if (ex > 127 || top == 0) ex = 0;                   // NaN and infinity stay what they are
                const float down = ldexpf(1.0f, -ex);
                qs[q] *= ldexpf(1.0f, ex);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const uint32_t w[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        qf[q][s][2 * e] = static_cast<_Float16>(cvt16<DT>(static_cast<uint16_t>(w[e] & 0xFFFFu)) * down);
                        qf[q][s][2 * e + 1] = static_cast<_Float16>(cvt16<DT>(static_cast<uint16_t>(w[e] >> 16)) * down);
                    }
                }
            }
        }

        v4f o[QT][NV];
        float m[QT], l[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            m[q] = FAR, l[q] = 0.f;
#pragma unroll
            for (int n = 0; n < NV; ++n) o[q][n] = {0.f, 0.f, 0.f, 0.f};
        }
        float sv_ref = 0.f;

        // blocks: 64 table entries at a time, one a lane; of the kept ones a wave takes those of its rank
        int base = b0 - 64, seen_blocks = 0;
        const int end = lim_hi < 0 ? 0 : min(b1, lim_hi / PAGE + 1);
        u64 bits = 0;
        int l_page = 0;
        float l_ka = 0.f, l_va = 0.f;
        const long long table_at = static_cast<long long>(r) * c.max_blocks;
        const long long mask_at = (static_cast<long long>(r) * c.H_kv + kh) * c.max_blocks;
        auto next = [&](int& block, int& page, float& ka, float& va) -> bool {
            while (bits == 0) {
                base += 64;
                if (base >= end) return false;
                const int j = base + lane;
                bool keep = j < end;
                l_page = -1;
                if (keep) {
                    l_page = c.table[table_at + j];
                    keep = l_page >= 0 && l_page < c.n_pages && (!a.mask || a.mask[mask_at + j]);
                }
                if (keep) {
                    l_ka = c.k_amax[static_cast<long long>(l_page) * c.H_kv + kh];
                    l_va = c.v_amax[static_cast<long long>(l_page) * c.H_kv + kh];
                }
                const u64 kept = __ballot(keep);
                const int rank = seen_blocks + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(kept >> 32),
                                                                          __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(kept), 0));
                bits = __ballot(keep && (rank & (kg - 1)) == my_kg);
                seen_blocks += __builtin_popcountll(kept);
            }
            const int b = __builtin_ctzll(bits);
            bits &= bits - 1;
            block = base + b;
            page = __builtin_amdgcn_readlane(l_page, b);
            ka = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l_ka), b));
            va = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l_va), b));
            return true;
        };
        uint4 kraw[NK], vraw[NV];
        auto load_k = [&](int page) {
            const uint8_t* p = static_cast<const uint8_t*>(c.k) + (static_cast<long long>(page) * c.H_kv + kh) * (PAGE * D) + lane * 16;
#pragma unroll
            for (int n = 0; n < NK; ++n) kraw[n] = *reinterpret_cast<const uint4*>(p + n * 1024);
        };
        auto load_v = [&](int page) {
            const uint8_t* p = static_cast<const uint8_t*>(c.v) + (static_cast<long long>(page) * c.H_kv + kh) * (PAGE * D) + lane * 16;
#pragma unroll
            for (int n = 0; n < NV; ++n) vraw[n] = *reinterpret_cast<const uint4*>(p + n * 1024);
        };
        int block, page;
        float ka, va;
        bool more = next(block, page, ka, va);
        if (more) {
            load_k(page);
            load_v(page);
        }
        while (more) {
            v4f s[QT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int q = 0; q < QT; ++q) s[q][t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < D / 64; ++e) {
                    const uint4 w = kraw[t * (D / 64) + e];
                    const v8h k0 = codes8(w.x, w.y), k1 = codes8(w.z, w.w);
#pragma unroll
                    for (int q = 0; q < QT; ++q) {
                        s[q][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[q][2 * e], s[q][t], 0, 0, 0);
                        s[q][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[q][2 * e + 1], s[q][t], 0, 0, 0);
                    }
                }
            }
            int n_block = 0, n_page = 0;
            float n_ka = 0.f, n_va = 0.f;
            const bool n_more = next(n_block, n_page, n_ka, n_va);
            if (n_more) load_k(n_page);

            const bool masked = block * PAGE + PAGE - 1 > lim_lo;
            const float sk = ka * (1.0f / 127.0f);
            if (va > SV_SLACK * sv_ref && va < INFINITY) {
                const float down = sv_ref / va;
#pragma unroll
                for (int q = 0; q < QT; ++q)
#pragma unroll
                    for (int n = 0; n < NV; ++n) o[q][n] *= down;
                sv_ref = va;
            }
            const float f = P_UP * (sv_ref > 0.f ? va / sv_ref : va);
            v8h pf[QT][2];
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                float cq = qs[q] * sk;
                if (cq == 0.f) cq = 1e-37f;   // a block of zeros: -inf below stays what it is
                float top = -INFINITY;
                if (masked) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (block * PAGE + 16 * t + 4 * (lane >> 4) + e > limit[q]) s[q][t][e] = -INFINITY;
                }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, s[q][t][e]);
                top = max_groups(top) * cq;
                if (__any(top > m[q] + SLACK)) {
                    const float to = fmaxf(m[q], top), down = __builtin_amdgcn_exp2f(m[q] - to);
                    m[q] = to;
                    l[q] *= down;
#pragma unroll
                    for (int n = 0; n < NV; ++n) o[q][n] *= down;
                }
                float p[16];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[4 * t + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][t][e], cq, -m[q]));
                float w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = p[e] * f;
                if (masked) {   // a key that is not seen has no weight even where the block's scales are NaN or infinite
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (block * PAGE + 16 * t + 4 * (lane >> 4) + e > limit[q]) p[4 * t + e] = w[4 * t + e] = 0.f;
                }
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += p[e];
                l[q] += sum;
#pragma unroll
                for (int e = 0; e < 16; ++e) pf[q][e >> 3][e & 7] = static_cast<_Float16>(w[e]);
            }
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const v8h v0 = codes8(vraw[n].x, vraw[n].y), v1 = codes8(vraw[n].z, vraw[n].w);
#pragma unroll
                for (int q = 0; q < QT; ++q) {
                    o[q][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[q][0], o[q][n], 0, 0, 0);
                    o[q][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[q][1], o[q][n], 0, 0, 0);
                }
            }
            if (n_more) load_v(n_page);
            more = n_more, block = n_block, page = n_page, ka = n_ka, va = n_va;
        }

        // ---- the waves that shared rows are joined, then the rows are written, whole or as a part
        const float o_scale = sv_ref * (1.0f / (127.0f * P_UP));
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            l[q] = sum_groups(l[q]);
#pragma unroll
            for (int n = 0; n < NV; ++n) o[q][n] *= o_scale;
        }
        if (kg > 1) {
            if (my_kg > 0) {
#pragma unroll
                for (int q = 0; q < QT; ++q) {
                    float* at = merge[wave - rg][q];
#pragma unroll
                    for (int n = 0; n < NV; ++n) reinterpret_cast<v4f*>(at)[n * 64 + lane] = o[q][n];
                    if (lane < 16) at[D * 16 + lane] = m[q], at[D * 16 + 16 + lane] = l[q];
                }
            }
            __syncthreads();
            if (my_kg == 0) {
#pragma unroll
                for (int q = 0; q < QT; ++q)
                    for (int k = 1; k < kg; ++k) {
                        const float* at = merge[k * rg + my_rg - rg][q];
                        const float om = at[D * 16 + (lane & 15)], ol = at[D * 16 + 16 + (lane & 15)];
                        const float to = fmaxf(m[q], om);
                        const float wa = __builtin_amdgcn_exp2f(m[q] - to), wb = __builtin_amdgcn_exp2f(om - to);
                        m[q] = to;
                        l[q] = l[q] * wa + ol * wb;
#pragma unroll
                        for (int n = 0; n < NV; ++n) o[q][n] = o[q][n] * wa + reinterpret_cast<const v4f*>(at)[n * 64 + lane] * wb;
                    }
            }
            __syncthreads();
        }
        if (my_kg == 0) {
            const int slot = 2 * part + (x0 > 0 ? 0 : 1);
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                if (!valid[q]) continue;
                const int row = row0 + 16 * q, tok = row / cut.Gp, g = gpart * ROWS + row - tok * cut.Gp;
                if (whole) {
                    const float inv = l[q] == 0.f ? 0.f : 1.0f / l[q];
                    uint16_t* out = O + q_at[q] * a.o_sn + static_cast<long long>(kh * G + g) * a.o_sh + 4 * (lane >> 4);
#pragma unroll
                    for (int n = 0; n < NV; ++n) {
                        uint2 w;
                        uint16_t h[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) h[e] = l[q] == 0.f ? 0 : cvt_to16<DT>(o[q][n][e] * inv);
                        __builtin_memcpy(&w, h, 8);
                        *reinterpret_cast<uint2*>(out + 16 * n) = w;
                    }
                } else {
                    const long long at = static_cast<long long>(slot) * CACHE_WG_ROWS + row;
#pragma unroll
                    for (int n = 0; n < NV; ++n)
                        *reinterpret_cast<v4f*>(ws.o + at * D + 16 * n + 4 * (lane >> 4)) = o[q][n];
                    if (lane < 16) ws.ml[2 * at] = m[q], ws.ml[2 * at + 1] = l[q];
                }
            }
        }
        pos += take;
        rem += take;
    }
    if (tid == 0 && !joins) ws.desc[bid].n_parts = 0;
}

// Joins an item that several workgroups have parts of, in their order.
template <int D, int DT, int QT>
__global__ __launch_bounds__(256) void cache_join_kernel(sparge_cache c, CacheAttn a, uint16_t* __restrict__ O, Joint ws) {
    constexpr int ROWS = 64 * QT, TPR = D / 4;   // threads per row, 4 channels each
    const JoinDesc d = ws.desc[blockIdx.x];
    if (d.n_parts == 0) return;
    const int G = a.H / c.H_kv;
    const Cut cut = cut_of(G, ROWS);
    const RowInfo x = row_info<QT>(c, a, cut, d.row);
    const int kh = d.head / cut.parts, gpart = d.head - kh * cut.parts;
    const int n_rows = min(cut.TT, x.n - d.tile * cut.TT) * cut.Gp, ch = (threadIdx.x % TPR) * 4;
    // the item's start is the second part of the workgroup before the first boundary, the rest first parts
    auto slot = [&](int k) { return static_cast<long long>(k == 0 ? 2 * (d.part - 1) + 1 : 2 * (d.part + k - 1)) * CACHE_WG_ROWS; };
    for (int row = threadIdx.x / TPR; row < n_rows; row += 256 / TPR) {
        const int tok = row / cut.Gp, g = gpart * ROWS + row - tok * cut.Gp;
        if (g >= G) continue;
        float m = FAR, l = 0.f;
        for (int k = 0; k < d.n_parts; ++k) m = fmaxf(m, ws.ml[2 * (slot(k) + row)]);
        v4f o = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < d.n_parts; ++k) {
            const long long at = slot(k) + row;
            const float w = __builtin_amdgcn_exp2f(ws.ml[2 * at] - m);
            l += ws.ml[2 * at + 1] * w;
            o += *reinterpret_cast<const v4f*>(ws.o + at * D + ch) * w;
        }
        uint16_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = l == 0.f ? 0 : cvt_to16<DT>(o[e] / l);
        uint2 w;
        __builtin_memcpy(&w, h, 8);
        *reinterpret_cast<uint2*>(O + static_cast<long long>(x.first + d.tile * cut.TT + tok) * a.o_sn +
                                  static_cast<long long>(kh * G + g) * a.o_sh + ch) = w;
    }
}

struct Layout {
    size_t ml, o, total;
};
Layout layout_of(int d) {
    const size_t up = 255, rows = 2ull * CACHE_WGS * CACHE_WG_ROWS;
    Layout x;
    x.ml = (CACHE_WGS * sizeof(JoinDesc) + up) & ~up;
    x.o = x.ml + rows * 2 * sizeof(float);
    x.total = x.o + rows * d * sizeof(float);
    return x;
}

template <int D, int DT, int QT>
void launch(const sparge_cache& c, const CacheAttn& a, const void* Q, void* O, const Joint& j, hipStream_t st) {
    hipLaunchKernelGGL((cache_attn_kernel<D, DT, QT>), dim3(CACHE_WGS), dim3(256), 0, st, c, a, static_cast<const uint16_t*>(Q),
                       static_cast<uint16_t*>(O), j);
    hipLaunchKernelGGL((cache_join_kernel<D, DT, QT>), dim3(CACHE_WGS), dim3(256), 0, st, c, a, static_cast<uint16_t*>(O), j);
}

}  // namespace

size_t cache_attn_workspace(int d) { return layout_of(d).total; }

hipError_t launch_cache_attn(const sparge_cache& c, const CacheAttn& a, const void* Q, void* O, void* ws, hipStream_t st) {
    const Layout x = layout_of(c.d);
    char* p = static_cast<char*>(ws);
    const Joint j = {reinterpret_cast<JoinDesc*>(p), reinterpret_cast<float*>(p + x.ml), reinterpret_cast<float*>(p + x.o)};
    // two tiles of 16 rows a wave where the rows of the cache have more query rows on average than four waves' single ones
    const bool wide = static_cast<long long>(a.n_slots) * (a.H / c.H_kv) > 64ll * c.R;
#define RUN(D, DT) wide ? launch<D, DT, 2>(c, a, Q, O, j, st) : launch<D, DT, 1>(c, a, Q, O, j, st)
    if (c.d == 64) {
        if (c.dtype == SPARGE_F16) RUN(64, SPARGE_F16); else RUN(64, SPARGE_BF16);
    } else {
        if (c.dtype == SPARGE_F16) RUN(128, SPARGE_F16); else RUN(128, SPARGE_BF16);
    }
#undef RUN
    return hipGetLastError();
}

}  // namespace sparge
