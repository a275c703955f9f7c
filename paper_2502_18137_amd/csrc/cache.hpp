// Internal declarations of the paged 8-bit K/V cache: plan, append, read-back, attention over it.
#pragma once
#include <type_traits>

#include "common.hpp"

namespace sparge {

// A page holds 64 tokens per kv head, K and V each as 64 d bytes in the operand order of the 16x16x32 MFMA, so that the
// attention loads its operands straight into registers, 1 KB of consecutive bytes per wave and load.  A byte is code + 128.
//   K: [key / 16][channel / 64][key % 16 + 16 (channel % 64 / 16)][channel % 16]
//   V: [channel / 16][channel % 16 + 16 (key % 16 / 4)][4 (key / 16) + key % 4]
// (the V order is the one in which the accumulators of K Q^T hand a lane its keys).
constexpr int PAGE = SPARGE_CACHE_PAGE;
static_assert(PAGE == 64, "the layouts, a ballot per page of a window and the attention's tiles are made for 64");

__host__ __device__ inline int k_byte(int key, int ch, int d) {
    return (((key >> 4) * (d >> 6) + (ch >> 6)) * 64 + (key & 15) + 16 * ((ch >> 4) & 3)) * 16 + (ch & 15);
}
__host__ __device__ inline int v_byte(int key, int ch) {
    return ((ch >> 4) * 64 + (ch & 15) + 16 * ((key >> 2) & 3)) * 16 + 4 * (key >> 4) + (key & 3);
}

// Inclusive prefix sum over a wave's lanes, through DPP row moves: the vector ALU alone (a loop of __shfl_up of 64-bit sums takes
// 2.4 us where this takes 0.2).  WIDTH 16: over each row of 16 lanes.
template <int WIDTH = 64>
__device__ __forceinline__ long long scan_lanes(long long v) {
    auto add = [&](auto ctrl, auto rows) {
        const unsigned lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
        const unsigned hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
        v += static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo);
    };
    using all = std::integral_constant<int, 0xF>;
    add(std::integral_constant<int, 0x111>{}, all{});   // row_shr:1, 2, 4, 8: the lane that far below in a row of 16, or 0
    add(std::integral_constant<int, 0x112>{}, all{});
    add(std::integral_constant<int, 0x114>{}, all{});
    add(std::integral_constant<int, 0x118>{}, all{});
    if constexpr (WIDTH == 64) {
        add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});   // row_bcast:15 into rows 1 and 3
        add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});   // row_bcast:31 into rows 2 and 3
    }
    return v;
}
__device__ __forceinline__ long long lane_value(long long v, int lane) {
    return static_cast<long long>(static_cast<unsigned long long>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane))) << 32 |
                                  static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), lane)));
}

// A barrier for what goes through LDS: loads from memory that are on their way stay on it (__syncthreads waits for them).
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One attention call: what the host knows of it.
struct CacheAttn {
    int n_slots, H, causal;
    long long q_sn, q_sh, o_sn, o_sh;   // element strides
    const int32_t* cu;
    const uint8_t* mask;                // [R, H_kv, max_blocks] or null
    float scale_log2;                   // softmax scale times log2 e
};

// What the joining launch has to know of a part of the attention's work.
struct JoinDesc {
    int n_parts;                        // that the item has; 0: nothing to join here
    int first, part;                    // the first part that begins inside the item; this one
    int token, n_tok, head;             // the item's rows of Q and O: tokens, their first head
    int pad[2];                         // (two 16-byte loads)
};
constexpr JoinDesc NO_JOIN = {0, 0, 0, 0, 0, 0, {0, 0}};
size_t cache_attn_workspace(int d);

hipError_t launch_cache_plan(const sparge_cache& c, const int32_t* new_len, const uint8_t* release, int n_slots, int32_t* cu,
                             int32_t* slots, int32_t* req, int32_t* status, hipStream_t st);
hipError_t launch_cache_append(const sparge_cache& c, const void* K, const void* V, int n_slots, long long k_sn, long long k_sh,
                               long long v_sn, long long v_sh, const int32_t* cu, const int32_t* slots, const int32_t* req,
                               hipStream_t st);
hipError_t launch_cache_read(const sparge_cache& c, const int32_t* slots, const int32_t* req, int n_slots, int out_dtype, void* K,
                             void* V, hipStream_t st);
hipError_t launch_cache_attn(const sparge_cache& c, const CacheAttn& a, const void* Q, void* O, void* ws, hipStream_t st);

}  // namespace sparge
