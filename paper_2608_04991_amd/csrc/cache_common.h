// What the kernels of the paged cache and of the tree attention share.
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "rac_cache.h"

namespace {

inline bool cache_valid(const rac_cache_config* c) {
    if (!c || c->layers < 1 || c->layers > 1024 || c->kv_heads < 1 || c->kv_heads > 1024) return false;
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16) return false;
    if (c->page_tokens < 8 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return false;
    if (c->pages < 1 || c->pages > (1 << 24) || c->seqs < 1 || c->seqs > 4096 || c->max_pages < 1) return false;
    if ((int64_t)c->max_pages * c->page_tokens > (1 << 30)) return false;
    if (c->type != RAC_CACHE_BF16 && c->type != RAC_CACHE_FP16 && c->type != RAC_CACHE_FP8) return false;
    return c->type != RAC_CACHE_FP8 || (c->k_scale > 0.0f && c->k_scale < __builtin_inff() && c->v_scale > 0.0f &&
                                        c->v_scale < __builtin_inff());
}

inline int cache_elem_bytes(const rac_cache_config* c) { return c->type == RAC_CACHE_FP8 ? 1 : 2; }

// Bytes of one page: all layers, keys and values.
inline uint64_t cache_page_bytes(const rac_cache_config* c) {
    return (uint64_t)c->layers * 2u * (uint64_t)c->kv_heads * (uint64_t)c->page_tokens * (uint64_t)c->head_dim *
           (uint64_t)cache_elem_bytes(c);
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int log2_of(int v) { return __builtin_ctz((unsigned)v); }

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Sums over the lanes up to this one, by moves between neighbouring lanes.
template <class T>
__device__ __forceinline__ T scan_wave(T v) {
    const auto from = [](T x, auto ctrl, auto rows) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value,
                                                                 decltype(rows)::value, 0xF, false));
    };
    using std::integral_constant;
    using all = integral_constant<int, 0xF>;
    v = v + from(v, integral_constant<int, 0x111>{}, all{});                          // row_shr:1
    v = v + from(v, integral_constant<int, 0x112>{}, all{});
    v = v + from(v, integral_constant<int, 0x114>{}, all{});
    v = v + from(v, integral_constant<int, 0x118>{}, all{});
    v = v + from(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});  // row_bcast:15
    return v + from(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});  // row_bcast:31
}

constexpr int kMostSum = 1 << 30;

// Sum over the threads of a workgroup of WAVES wavefronts before this one, and
// over all of them (sums: LDS).  With up to 2^24 a thread no sum of a wavefront
// wraps; the whole one stays at kMostSum where it is more, and then the sums before
// a thread mean nothing.
template <int WAVES>
__device__ __forceinline__ int scan_workgroup(int v, int* sums, int* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x / 64;
    int x = v;
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        x += lane >= o ? y : 0;
    }
    __syncthreads();
    if (lane == 63) sums[w] = x;
    __syncthreads();
    uint32_t before = 0;
    int all = 0;
    for (int i = 0; i < WAVES; ++i) {
        before += i < w ? sums[i] : 0;
        all = sums[i] < kMostSum - all ? all + sums[i] : kMostSum;
    }
    *total = all;
    return (int)(before + (uint32_t)x - (uint32_t)v);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

}  // namespace
