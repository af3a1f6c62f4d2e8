// What the attention of drafted trees and the weights it gives to cached tokens
// share: which keys a row sees, and the products on the matrix cores.
#pragma once

#include "cache_common.h"

namespace {

// What a sequence brings to the call, whatever the device arrays hold.
struct Seq {
    int q0, m;    // first query row, rows
    int d0, n;    // first drafted row, drafted tokens
    int length;   // committed tokens
};

template <class Args>
__device__ __forceinline__ Seq seq_of(const Args& a, int s) {
    Seq r;
    r.q0 = clamp_int(a.q_start[s], 0, a.rows);
    r.m = clamp_int(a.q_start[s + 1], r.q0, a.rows) - r.q0;
    r.m = r.m < a.max_rows ? r.m : a.max_rows;
    r.d0 = r.n = 0;
    if (a.k) {
        r.d0 = clamp_int(a.draft_start[s], 0, a.draft_rows);
        r.n = clamp_int(a.draft_start[s + 1], r.d0, a.draft_rows) - r.d0;
        r.n = r.n < a.max_draft ? r.n : a.max_draft;
    }
    r.length = clamp_int(a.lengths[s], 0, a.max_pages << a.log_page);
    return r;
}

// What a query row sees: committed positions from `from` on, and the drafted
// tokens of [first, end) that its mask names (all of them without a mask).
struct Sight {
    int from, first, end;
};

template <class Args>
__device__ __forceinline__ Sight sight_of(const Args& a, const Seq& s, int i) {
    Sight r{0, 0, s.n};
    int c;  // drafted tokens it sees
    const uint64_t* words = a.mask ? a.mask + (size_t)(s.q0 + i) * a.mask_words : nullptr;
    if (words) {
        const int most = a.mask_words * 64;
        r.end = s.n < most ? s.n : most;
        c = 0;
        for (int w = 0; 64 * w < r.end; ++w) {
            const int left = r.end - 64 * w;
            c += __popcll(left >= 64 ? words[w] : words[w] & ((uint64_t(1) << left) - 1));
        }
    } else {
        r.end = clamp_int(s.n - s.m + i + 1, 0, s.n);
        c = r.end;
    }
    if (a.window > 0) {
        if (c < a.window) {
            r.from = s.length - (a.window - c);
            r.from = r.from < 0 ? 0 : r.from;
        } else {
            r.from = s.length;
            int drop = c - a.window;  // the first ones that fall out of the window
            if (!words) {
                r.first = drop;
            } else {
                int w = 0;
                for (; drop > 0; ++w) {
                    const int in = __popcll(words[w]);
                    if (in > drop) break;
                    drop -= in;
                }
                if (drop > 0) {
                    uint64_t bits = words[w];
                    for (; drop > 0; --drop) bits &= bits - 1;
                    r.first = 64 * w + __builtin_ctzll(bits);
                } else {
                    r.first = 64 * w;
                }
            }
        }
    }
    return r;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int TYPE>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (TYPE == RAC_CACHE_FP16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight e4m3 as bf16 (exact).
__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
    return r;
}

// LDS: a tile of 16-bit queries, keys or values is rows of DP / 8 pieces of 16
// bytes; piece c of a row sits at c ^ swizzle(row), so that 16 lanes that read
// the same piece of 16 rows, or write the pieces of one row, touch every bank
// once.
template <int DP>
__device__ __forceinline__ uint32_t piece_at(uint32_t row, uint32_t c) {
    if constexpr (DP == 64)
        return row * 8u + (c ^ ((row >> 1) & 7u));
    else
        return row * (DP / 8) + (c ^ (row & 15u));
}

}  // namespace
