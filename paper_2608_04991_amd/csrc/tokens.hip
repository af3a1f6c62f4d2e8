// tokens.hip - gfx950 kernels and C ABI of rotary positions and of the log
// probabilities of drafted tokens.  The contract is in include/rac_tokens.h.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "rac_tokens.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// 16 bytes of a type: kN elements, as floats and back (one rounding, to nearest even).
template <int TYPE>
struct Block {
    static constexpr int kBytes = TYPE == RAC_TYPE_FP32 ? 4 : 2, kN = 16 / kBytes;

    static __device__ __forceinline__ void widen(u32x4 v, float (&x)[kN]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == RAC_TYPE_FP32) {
                x[i] = __uint_as_float(v[i]);
            } else if constexpr (TYPE == RAC_TYPE_FP16) {
                const uint32_t u = v[i];  // (of a vector's element itself, the cast would take the first)
                const f16x2 h = __builtin_bit_cast(f16x2, u);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            } else {
                x[2 * i] = __uint_as_float(v[i] << 16);
                x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
            }
        }
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&x)[kN]) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == RAC_TYPE_FP32)
                v[i] = __float_as_uint(x[i]);
            else if constexpr (TYPE == RAC_TYPE_FP16)
                v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, f16x2));
            else
                v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
        }
        return v;
    }
    static __device__ __forceinline__ float top(const float (&x)[kN]) {
        float m = x[0];
#pragma unroll
        for (int i = 1; i < kN; ++i) m = __builtin_fmaxf(m, x[i]);
        return m;
    }
    static __device__ __forceinline__ float one(const uint8_t* p) {
        if constexpr (TYPE == RAC_TYPE_FP32) return *reinterpret_cast<const float*>(p);
        if constexpr (TYPE == RAC_TYPE_FP16) return (float)*reinterpret_cast<const _Float16*>(p);
        return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
    }
    static __device__ __forceinline__ void put(uint8_t* p, float x) {
        if constexpr (TYPE == RAC_TYPE_FP32)
            *reinterpret_cast<float*>(p) = x;
        else if constexpr (TYPE == RAC_TYPE_FP16)
            *reinterpret_cast<_Float16*>(p) = (_Float16)x;
        else
            *reinterpret_cast<__bf16*>(p) = (__bf16)x;
    }
};

// ---------------------------------------------------------------------------
// Rotary positions.  A workgroup takes a few rows: first a sine and cosine for
// every pair of a row, which all heads share, then 16 bytes of a head a thread and
// step (of both halves where the pairs lie apart).  The fraction of a turn is that
// of a binary64 product, off by 2^-53 of the turns at most.
//
// Bound by the bytes of queries and keys, read and written once: 4099 rows of 28 + 4 heads
// of 128 channels, 64 of them turned, 67 MB, in 16.7 us, 4.0 TB/s (a large copy reaches 4.9).
// A level of 8 rows of 8 + 8 heads takes 3 us, the time of a launch.
struct RotaryArgs {
    const int32_t* pos;
    const double* freq;
    const uint8_t* in[2];   // queries, keys
    uint8_t* out[2];
    int64_t in_stride[2], out_stride[2];  // bytes
    int64_t rows;
    float amplitude, sign;
    int32_t q_heads, heads;  // of queries, of both
    int32_t head_bytes, pairs, each;  // rows a workgroup
    int32_t turned, pieces;  // pieces of a head that turn, and all
    uint32_t by_pieces;      // 2^32 / pieces, rounded up
    uint32_t by_row;         // 2^32 / (heads * pieces), rounded up
};

constexpr int kRotaryThreads = 256, kRotaryRows = 8, kMostPairs = 128;

template <int TYPE, bool HALF>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
    using B = Block<TYPE>;
    constexpr int kAtOnce = 2;
    __shared__ f32x2 turn[kRotaryRows * kMostPairs];
    const int t = (int)threadIdx.x, per = a.heads * a.pieces;
    for (int64_t row0 = (int64_t)blockIdx.x * a.each; row0 < a.rows; row0 += (int64_t)gridDim.x * a.each) {
        const int rows = a.rows - row0 < a.each ? (int)(a.rows - row0) : a.each, all = rows * per;
        for (int i0 = 0; i0 < all || i0 == 0; i0 += kRotaryThreads * kAtOnce) {
            u32x4 x[kAtOnce], y[kAtOnce];
            uint8_t* to[kAtOnce];
            int at[kAtOnce];  // the first pair, -1: channels that are kept, -2: nothing to do
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int i = i0 + k * kRotaryThreads + t;
                at[k] = -2;
                if (i >= all) continue;
                const int r = a.each == 1 ? 0 : per == 1 ? i : (int)__umulhi((uint32_t)i, a.by_row), in = i - r * per;
                if (a.pos[row0 + r] < 0) continue;
                const int h = a.pieces == 1 ? in : (int)__umulhi((uint32_t)in, a.by_pieces), p = in - h * a.pieces;
                const int side = h >= a.q_heads, head = side ? h - a.q_heads : h;
                // (where pairs lie apart, the pieces of the second half come with those of the first)
                const int o = p < a.turned ? 16 * p : 16 * (p + (HALF ? a.turned : 0));
                const uint8_t* from = a.in[side] + (row0 + r) * a.in_stride[side] + (int64_t)head * a.head_bytes + o;
                to[k] = a.out[side] + (row0 + r) * a.out_stride[side] + (int64_t)head * a.head_bytes + o;
                x[k] = *reinterpret_cast<const u32x4*>(from);
                at[k] = p < a.turned ? r * a.pairs + p * (HALF ? B::kN : B::kN / 2) : -1;
                if (HALF && at[k] >= 0) y[k] = *reinterpret_cast<const u32x4*>(from + 16 * a.turned);
            }
            if (i0 == 0) {
                for (int i = t; i < rows * a.pairs; i += kRotaryThreads) {
                    const int r = a.each == 1 ? 0 : i / a.pairs;
                    const double turns = (double)a.pos[row0 + r] * a.freq[i - r * a.pairs];
                    float s, c;
                    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
                    turn[i] = f32x2{c * a.amplitude, s * a.sign};
                }
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (at[k] == -2) continue;
                if (at[k] < 0) {
                    *reinterpret_cast<u32x4*>(to[k]) = x[k];
                    continue;
                }
                float u[B::kN], v[B::kN];
                B::widen(x[k], u);
                if constexpr (HALF) {
                    B::widen(y[k], v);
#pragma unroll
                    for (int j = 0; j < B::kN; ++j) {
                        const f32x2 w = turn[at[k] + j];
                        const float p = u[j] * w[0] - v[j] * w[1];
                        v[j] = v[j] * w[0] + u[j] * w[1];
                        u[j] = p;
                    }
                    *reinterpret_cast<u32x4*>(to[k] + 16 * a.turned) = B::narrow(v);
                } else {
#pragma unroll
                    for (int j = 0; j < B::kN; j += 2) {
                        const f32x2 w = turn[at[k] + j / 2];
                        const float p = u[j] * w[0] - u[j + 1] * w[1];
                        u[j + 1] = u[j + 1] * w[0] + u[j] * w[1];
                        u[j] = p;
                    }
                }
                *reinterpret_cast<u32x4*>(to[k]) = B::narrow(u);
            }
        }
        __syncthreads();  // (the next rows' sines take the same place)
    }
}

// ---------------------------------------------------------------------------
// Log probabilities.  A row's logits are blocks of 16 aligned bytes, the first and
// last of them perhaps partly outside the row.
template <int TYPE>
struct Row {
    using B = Block<TYPE>;
    const uint8_t* first;  // block 0
    int phase, vocab, blocks;

    __device__ __forceinline__ Row(const uint8_t* p, int v) {
        const uint32_t in = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
        first = p - in;
        phase = (int)in / B::kBytes;
        vocab = v;
        blocks = (phase + v + B::kN - 1) / B::kN;
    }
    __device__ __forceinline__ int word(int b, int i) const { return b * B::kN + i - phase; }
    __device__ __forceinline__ bool whole(int b) const { return (b > 0 || phase == 0) && word(b, B::kN) <= vocab; }
    __device__ __forceinline__ u32x4 raw(int b) const {
        return *reinterpret_cast<const u32x4*>(first + (int64_t)b * 16);
    }
    // A block that is not whole; what is outside the row is -infinity.
    __device__ __forceinline__ void some(int b, float (&x)[B::kN]) const {
#pragma unroll
        for (int i = 0; i < B::kN; ++i) {
            const int v = word(b, i);
            x[i] = -INFINITY;
            if (v >= 0 && v < vocab) x[i] = B::one(first + ((int64_t)b * B::kN + i) * B::kBytes);
        }
    }
    __device__ __forceinline__ void get(int b, float (&x)[B::kN]) const {
        if (whole(b))
            B::widen(raw(b), x);
        else
            some(b, x);
    }
};

// Over the lanes of a wavefront, by moves between neighbouring lanes, for all lanes.
template <class F>
__device__ __forceinline__ float over_wave(float v, bool zero, F f) {
    const auto from = [&](auto ctrl, auto rows) {
        const float x = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
            zero ? 0 : __builtin_bit_cast(int, v), __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
        v = f(v, x);
    };
    using std::integral_constant;
    using all = integral_constant<int, 0xF>;
    from(integral_constant<int, 0x111>{}, all{});  // row_shr:1, 2, 4, 8
    from(integral_constant<int, 0x112>{}, all{});
    from(integral_constant<int, 0x114>{}, all{});
    from(integral_constant<int, 0x118>{}, all{});
    from(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});  // row_bcast:15, 31
    from(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float sum_wave(float v) { return over_wave(v, true, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float max_wave(float v) { return over_wave(v, false, [](float a, float b) { return __builtin_fmaxf(a, b); }); }
__device__ __forceinline__ float min_wave(float v) { return over_wave(v, false, [](float a, float b) { return __builtin_fminf(a, b); }); }

// Partial sums of a softmax, in powers of two: sum of e = 2^(c (x - m)) and of
// c (x - m) e.  m need not be the largest logit, only no more than kSlack / c below it.
// (The difference comes before the factor: a mask of the type's lowest value stays in
// range, and equal logits give equal weights.)
struct Sums {
    float m, s, t;
    static constexpr float kSlack = 8.0f;

    // Ready for logits of up to `top`; slack: kSlack / c.
    template <bool ENTROPY>
    __device__ __forceinline__ void grow(float top, float c, float slack) {
        if (__any(top > m + slack)) {
            const float now = top > m + slack ? top : m, by = (m - now) * c;
            const float keep = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(by);
            if constexpr (ENTROPY) t = m == -INFINITY ? 0.0f : (t + __builtin_fmaxf(by, -200.0f) * s) * keep;
            s = s * keep;
            m = now;
        }
    }
    template <int N, bool ENTROPY>
    __device__ __forceinline__ void add(const float (&x)[N], float c) {
        const float ref = m == -INFINITY ? 0.0f : m;
        float e[N], u[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            u[i] = (x[i] - ref) * c;
            e[i] = __builtin_amdgcn_exp2f(u[i]);
        }
        if constexpr (ENTROPY)
#pragma unroll
            for (int i = 0; i < N; ++i) t = __builtin_fmaf(__builtin_fmaxf(u[i], -200.0f), e[i], t);  // (0 where e is)
#pragma unroll
        for (int o = N / 2; o > 0; o /= 2)
#pragma unroll
            for (int i = 0; i < o; ++i) e[i] = e[i] + e[i + o];
        s = s + e[0];
    }
    // As sums against the reference `to`.
    __device__ __forceinline__ void rebase(float to, float c) {
        const float ref = to == -INFINITY ? 0.0f : to, by = m == ref ? 0.0f : (m - ref) * c;
        const float keep = __builtin_amdgcn_exp2f(by);
        t = m == -INFINITY ? 0.0f : (t + __builtin_fmaxf(by, -200.0f) * s) * keep;
        s = m == -INFINITY ? s : s * keep;  // (a NaN alone leaves m at -infinity)
        m = to;
    }
    __device__ __forceinline__ void join_wave(float c) {
        rebase(max_wave(m), c);
        s = sum_wave(s);
        t = sum_wave(t);
    }
    // (an infinity above the range would make every word's log probability one below it)
    __device__ __forceinline__ float lse(float scale) const {
        const float x = (float)((double)m * (double)scale + (double)log2f(s) * 0.6931471805599453);
        return s == 0.0f ? -INFINITY : x == INFINITY ? NAN : x;
    }
    __device__ __forceinline__ float entropy() const {
        if (s == 0.0f) return 0.0f;
        const float h = (log2f(s) - t / s) * 0.6931472f;
        return h < 0.0f ? 0.0f : h;
    }
};

// Logits in the order of alternatives: the larger first, ties to the lower word.
// 0 is none.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);  // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float float_of(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u); }
__device__ __forceinline__ uint64_t key_of(float x, int word) { return (uint64_t)order_of(x) << 32 | (uint32_t)~word; }
__device__ __forceinline__ int word_of(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float logit_of(uint64_t key) { return float_of((uint32_t)(key >> 32)); }

struct LogprobArgs {
    const uint8_t* logits;
    int64_t stride;  // bytes
    const int32_t* tokens;
    const int32_t* token_rows;
    float* logprob;
    float* lse;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    float* part_sums;     // [rows][parts][4]
    uint64_t* part_top;   // [rows][parts][top]
    int64_t rows;
    int32_t vocab, count, top, parts;
    int32_t part_blocks;  // blocks of a part
    int32_t each;  // alternatives of a part that make up the row's with as many of others
    float scale, scale2, slack;  // scale2: times log2(e); slack: Sums::kSlack over that
};

__device__ __forceinline__ float logprob_of(float x, float scale, float lse) {
    return (x == -INFINITY || lse == -INFINITY) && lse == lse ? -INFINITY : __builtin_fmaf(x, scale, -lse);
}

constexpr int kLogThreads = 256, kMostTop = 64, kMostParts = 64, kCandidates = 1024;

// The blocks of a thread: every T-th of [b0, b1).  Held in registers, kHeld at most
// (what is outside is -infinity), or read anew each time.  (One more than 8: a row of 8 T
// blocks that does not begin at one has a part of another.)  Where there is one for a thread at
// most, the wavefronts take them in turn, so that each has as many as another: the bar of
// the alternatives rests on that (395 rows of 697 words, 64 alternatives: 14 us, else 43).
constexpr int kHeld = 9;

template <int TYPE, int T>
struct Held {
    using B = Block<TYPE>;
    u32x4 raw[kHeld];
    float tops[kHeld];  // the largest logit of each
    int first, size;

    __device__ __forceinline__ Held(const Row<TYPE>& row, int b0, int b1) {
        const int t = (int)threadIdx.x, me = b1 - b0 <= T ? (t & 63) * (T / 64) + t / 64 : t;
        constexpr uint32_t kNone = TYPE == RAC_TYPE_FP32 ? 0xFF800000u : TYPE == RAC_TYPE_FP16 ? 0xFC00FC00u : 0xFF80FF80u;
        first = b0 + me;
        size = b1 - b0;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int b = first + k * T;
            raw[k] = u32x4{kNone, kNone, kNone, kNone};
            if (b < b1 && row.whole(b)) raw[k] = row.raw(b);
        }
        // (the first and the last of the row)
        if (b0 == 0 && row.phase > 0 && me == 0) raw[0] = part_of(row, 0);
        if (b1 == row.blocks && !row.whole(b1 - 1) && (size - 1) % T == me) {
            const u32x4 last = part_of(row, b1 - 1);
#pragma unroll
            for (int k = 0; k < kHeld; ++k) raw[k] = k == (size - 1) / T ? last : raw[k];
        }
    }
    static __device__ __forceinline__ u32x4 part_of(const Row<TYPE>& row, int b) {
        float x[B::kN];
        row.some(b, x);
        return B::narrow(x);
    }
    // f(logits, the largest of them).
    template <class F>
    __device__ __forceinline__ void each(const Row<TYPE>&, F f) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) tops[k] = -INFINITY;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            if (k * T >= size) break;
            float x[B::kN];
            B::widen(raw[k], x);
            tops[k] = B::top(x);
            f(x, tops[k]);
        }
    }
    // f(logit, word) of those of at least bar, -infinity not.  (Few: their blocks are marked
    // and picked out one by one, so that there is one copy of what is done with them.)
    template <class F>
    __device__ __forceinline__ void reach(const Row<TYPE>& row, float bar, F f) const {
        uint32_t marks = 0;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) marks |= tops[k] >= bar ? 1u << k : 0u;
        while (__any(marks)) {
            const int k = marks ? __builtin_ctz(marks) : kHeld;
            u32x4 v = raw[0];
#pragma unroll
            for (int j = 1; j < kHeld; ++j) {
                const bool is = k == j;
                v = u32x4{is ? raw[j][0] : v[0], is ? raw[j][1] : v[1], is ? raw[j][2] : v[2], is ? raw[j][3] : v[3]};
            }
            float x[B::kN];
            B::widen(v, x);
            uint32_t hits = 0;
#pragma unroll
            for (int i = 0; i < B::kN; ++i) hits |= marks && x[i] >= bar && x[i] > -INFINITY ? 1u << i : 0u;
            while (__any(hits)) {
                const int i = hits ? __builtin_ctz(hits) : 0;
                float y = x[0];
#pragma unroll
                for (int j = 1; j < B::kN; ++j) y = i == j ? x[j] : y;
                if (hits) f(y, row.word(first + k * T, i));
                hits &= hits - 1u;
            }
            marks &= marks - 1u;
        }
    }
};

template <int TYPE, int T, int AT_ONCE>
struct Streamed {
    using B = Block<TYPE>;
    int b0, b1;

    __device__ __forceinline__ Streamed(const Row<TYPE>&, int from, int to) : b0(from), b1(to) {}
    // f(logits, their first word).
    template <class F>
    __device__ __forceinline__ void blocks(const Row<TYPE>& row, F f) const {
        for (int b = b0 + (int)threadIdx.x; b < b1; b += AT_ONCE * T) {
            u32x4 v[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                if (b + k * T < b1 && row.whole(b + k * T)) v[k] = row.raw(b + k * T);
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int at = b + k * T;
                if (at >= b1) break;
                float x[B::kN];
                if (row.whole(at))
                    B::widen(v[k], x);
                else
                    row.some(at, x);
                f(x, row.word(at, 0));
            }
        }
    }
    template <class F>
    __device__ __forceinline__ void each(const Row<TYPE>& row, F f) const {
        blocks(row, [&](const float (&x)[B::kN], int) { f(x, B::top(x)); });
    }
    template <class F>
    __device__ __forceinline__ void reach(const Row<TYPE>& row, float bar, F f) const {
        blocks(row, [&](const float (&x)[B::kN], int word) {
            if (!(B::top(x) >= bar)) return;  // (most blocks)
#pragma unroll
            for (int i = 0; i < B::kN; ++i)
                if (x[i] >= bar && x[i] > -INFINITY) f(x[i], word + i);
        });
    }
    // f(logits, their first word), by all threads at once, in the order of words; f that returns
    // false ends it.
    template <class F>
    __device__ __forceinline__ void in_order(const Row<TYPE>& row, F f) const {
        for (int b = b0; b < b1; b += T) {
            float x[B::kN];
#pragma unroll
            for (int i = 0; i < B::kN; ++i) x[i] = -INFINITY;
            if (b + (int)threadIdx.x < b1) row.get(b + (int)threadIdx.x, x);
            if (!f(x, row.word(b + (int)threadIdx.x, 0))) return;
        }
    }
};

// The `top` largest logits into best[], descending, 0 where there are fewer.  Every
// thread knows its own largest.  With the d-th largest of these in each of g wavefronts,
// d g >= top, there are enough: the g-th largest of the wavefronts' d-th ones is a bar
// that few logits reach as a rule, and they are ranked by counting.
template <int TYPE, int T>
struct Top {
    using B = Block<TYPE>;
    static constexpr int kWaves = T / 64;
    uint64_t buffer[kCandidates];
    uint64_t best[kMostTop];
    uint64_t wave_key[kWaves];
    float wave_bar[kWaves];
    int count, wave_count[kWaves];

    __device__ __forceinline__ void push(float x, int word) {
        const int at = atomicAdd(&count, 1);  // (any order: the keys are ranked)
        if (at < kCandidates) buffer[at] = key_of(x, word);
    }
    template <class Blocks>
    __device__ __forceinline__ void find(const Row<TYPE>& row, const Blocks& blocks, int b0, int b1, int top, float mine) {
        const int t = (int)threadIdx.x, lane = t & 63;
        const int d = (top + kWaves - 1) / kWaves, g = (top + d - 1) / d;
        float bar = max_wave(mine), rest = mine;
        for (int have = __popcll(__ballot(rest == bar)); have < d; have += __popcll(__ballot(rest == bar))) {
            if (rest == bar) rest = -INFINITY;
            bar = max_wave(rest);
            if (bar == -INFINITY) break;
        }
        if (lane == 0) wave_bar[t / 64] = bar;
        if (t < kMostTop) best[t] = 0;
        if (t == 0) count = 0;
        __syncthreads();
        const float own = lane < kWaves ? wave_bar[lane] : -INFINITY;
        int above = 0;  // wavefronts with a bar of at least this one
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            above += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, own), w)) >= own;
        bar = max_wave(lane < kWaves && above >= g ? own : -INFINITY);
        if (mine >= bar && mine > -INFINITY) blocks.reach(row, bar, [&](float x, int word) { push(x, word); });
        __syncthreads();
        // (whose largest `mine` is differs where the wavefronts took blocks in turn)
        if (count > kCandidates) many(row, Streamed<TYPE, T, 1>(row, b0, b1), top, b1 - b0 <= T ? INFINITY : mine, bar);
        const int n = count;
        for (int c = t; c < n; c += T) {
            const uint64_t key = buffer[c];
            int rank = 0;
#pragma unroll 8
            for (int i = 0; i < n; ++i) rank += buffer[i] > key;
            if (rank < top) best[rank] = key;
        }
        __syncthreads();
    }
    // More reach the bar than there is room for: as a rule words that tie with it, of
    // which the first will do.
    __device__ __forceinline__ void many(const Row<TYPE>& row, const Streamed<TYPE, T, 1>& blocks, int top, float mine, float bar) {
        const int t = (int)threadIdx.x;
        __syncthreads();
        if (t == 0) count = 0;
        __syncthreads();
        if (mine > bar) blocks.reach(row, bar, [&](float x, int word) { if (x > bar) push(x, word); });
        __syncthreads();
        int n = count;
        __syncthreads();
        if (n <= kCandidates - kMostTop) {
            if (n < top)
                blocks.in_order(row, [&](const float (&x)[B::kN], int word) {
                    int own = 0;
#pragma unroll
                    for (int i = 0; i < B::kN; ++i) own += x[i] == bar;
                    int before = own;
                    for (int o = 1; o < 64; o <<= 1) {
                        const int y = __shfl_up(before, o);
                        before += (t & 63) >= o ? y : 0;
                    }
                    if ((t & 63) == 63) wave_count[t / 64] = before;
                    __syncthreads();
                    int at = n + before - own;
                    for (int w = 0; w < kWaves; ++w) {
                        at += w < t / 64 ? wave_count[w] : 0;
                        n += wave_count[w];
                    }
#pragma unroll
                    for (int i = 0; i < B::kN; ++i)
                        if (x[i] == bar) {
                            if (at < top) buffer[at] = key_of(bar, word + i);
                            ++at;
                        }
                    __syncthreads();
                    return n < top;
                });
            if (t == 0 && count < top) count = n < top ? n : top;
        } else {
            // A few threads have most of the large ones, as of a mask that allows one range of words:
            // one alternative after the other, a look at all blocks each.  Rows of 131072 in bf16 of
            // which 2000 words in a row are allowed, 64 alternatives: 393 us a row and 2.9 ms for 681
            // of them, with every word allowed 16 and 76; 8 alternatives 67 and 462 us.
            uint64_t last = ~uint64_t(0);
            n = 0;
            for (; n < top; ++n) {
                uint64_t next = 0;
                blocks.blocks(row, [&](const float (&x)[B::kN], int word) {
#pragma unroll
                    for (int i = 0; i < B::kN; ++i) {
                        const uint64_t key = x[i] > -INFINITY ? key_of(x[i], word + i) : 0;
                        if (key < last && key > next) next = key;
                    }
                });
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const uint64_t y = __shfl_xor((unsigned long long)next, o);
                    next = y > next ? y : next;
                }
                __syncthreads();
                if ((t & 63) == 0) wave_key[t / 64] = next;
                __syncthreads();
                for (int w = 0; w < kWaves; ++w) next = wave_key[w] > next ? wave_key[w] : next;
                if (next == 0) break;
                last = next;
                if (t == 0) buffer[n] = next;
            }
            if (t == 0) count = n;
        }
        __syncthreads();
    }
};

// Nothing, where no alternatives are wanted.
struct NoTop {};

// The scored token of a row and its logit, read ahead of the sums.
template <int TYPE>
struct Scored {
    bool there;
    float logit;

    __device__ __forceinline__ Scored(const LogprobArgs& a, int64_t row) {
        const int token = a.token_rows || a.count == 0 ? -1 : a.tokens[row];
        there = token >= 0 && token < a.vocab;
        logit = there ? Block<TYPE>::one(a.logits + row * a.stride + (int64_t)token * Block<TYPE>::kBytes) : 0.0f;
    }
};

template <int TYPE>
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int64_t row, const Sums& x, const Scored<TYPE>& y) {
    const float lse = x.lse(a.scale);
    a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = x.entropy();
    if (!a.token_rows && a.count > 0) a.logprob[row] = y.there ? logprob_of(y.logit, a.scale, lse) : 0.0f;
}

__device__ __forceinline__ void finish_top(const LogprobArgs& a, int64_t row, int i, uint64_t key, float lse) {
    a.top_ids[row * a.top + i] = key ? word_of(key) : -1;
    a.top_logprobs[row * a.top + i] = key ? logprob_of(logit_of(key), a.scale, lse) : -INFINITY;
}

// A workgroup a row, or a part of one: one pass with a running reference and sums.  With
// alternatives the blocks stay in registers for the second look where they fit (HELD).
//
// Bound by the logits' bytes, 4099 rows of 100003 in bf16: 820 MB in 151 us, 5.4 TB/s (call
// after call; under a profiler, with gaps between them, 162 in the median).  With alternatives
// of short rows by what follows the loads, the bar, the look and the ranking of candidates, for
// which a workgroup waits on itself: 681 rows of 32768, 45 MB, in 20 us.
template <int TYPE, bool ENTROPY, bool TOP, int T, bool HELD>
__global__ __launch_bounds__(T) void logprob_kernel(LogprobArgs a) {
    using B = Block<TYPE>;
    using Blocks = typename std::conditional<HELD, Held<TYPE, T>, Streamed<TYPE, T, 4>>::type;
    constexpr int kWaves = T / 64;
    __shared__ Sums waves[kWaves];
    __shared__ typename std::conditional<TOP, Top<TYPE, T>, NoTop>::type alternatives;
    const int t = (int)threadIdx.x, part = (int)blockIdx.x;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const int64_t item = r * a.parts + part;
        const Row<TYPE> row(a.logits + r * a.stride, a.vocab);
        const int b0 = part * a.part_blocks < row.blocks ? part * a.part_blocks : row.blocks;
        const int b1 = b0 + a.part_blocks < row.blocks ? b0 + a.part_blocks : row.blocks;
        Blocks blocks(row, b0, b1);
        const Scored<TYPE> scored(a, r);
        Sums x{-INFINITY, 0.0f, 0.0f};
        float most = -INFINITY;
        blocks.each(row, [&](const float (&v)[B::kN], float top) {
            if constexpr (TOP) most = __builtin_fmaxf(most, top);
            x.grow<ENTROPY>(top, a.scale2, a.slack);
            x.add<B::kN, ENTROPY>(v, a.scale2);
        });
        x.join_wave(a.scale2);
        if ((t & 63) == 0) waves[t / 64] = x;
        if constexpr (TOP) alternatives.find(row, blocks, b0, b1, a.top, most + 0.0f);
        __syncthreads();
        x = waves[t % kWaves];
        float top = x.m;
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
        x.rebase(top, a.scale2);
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) {
            x.s = x.s + __shfl_xor(x.s, o);
            x.t = x.t + __shfl_xor(x.t, o);
        }
        if (a.parts == 1) {
            if (t == 0) finish_row<TYPE>(a, r, x, scored);
            if constexpr (TOP)
                if (t < a.top) finish_top(a, r, t, alternatives.best[t], x.lse(a.scale));
        } else {
            if (t == 0) *reinterpret_cast<float4*>(a.part_sums + 4 * item) = float4{x.m, x.s, x.t, 0.0f};
            if constexpr (TOP)
                if (t < a.top) a.part_top[item * a.top + t] = alternatives.best[t];
        }
        __syncthreads();
    }
}

// Joins the parts of a row: a wavefront has the sums.  With d alternatives of each of
// top / d parts there are enough: so the top / d-th largest of the parts' d-th ones bounds
// the row's from below, and the few keys that reach it are ranked by counting.  Bound by
// the loads' latency and its own barriers: 4 to 5 us for 8 parts and 20 alternatives.
template <int TYPE>
__global__ __launch_bounds__(kLogThreads) void logprob_join_kernel(LogprobArgs a) {
    __shared__ uint64_t keys[kMostParts * kMostTop];
    __shared__ uint64_t best[kMostTop];
    __shared__ int count;
    const int t = (int)threadIdx.x, all = a.parts * a.top;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Scored<TYPE> scored(a, r);
        constexpr int kAtOnce = kMostParts * kMostTop / kLogThreads;
        uint64_t key[kAtOnce], bar = 0;
        if (a.top > 0) {
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                key[i] = 0;
                if (i * kLogThreads < all && t + i * kLogThreads < all) key[i] = a.part_top[r * all + t + i * kLogThreads];
            }
            if ((t & 63) < a.parts) bar = a.part_top[r * all + (t & 63) * a.top + a.each - 1];
        }
        Sums x{-INFINITY, 0.0f, 0.0f};
        if ((t & 63) < a.parts) {
            const float4 v = *reinterpret_cast<const float4*>(a.part_sums + 4 * (r * a.parts + (t & 63)));
            x = Sums{v.x, v.y, v.z};
        }
        x.join_wave(a.scale2);
        if (t == kLogThreads - 64) finish_row<TYPE>(a, r, x, scored);
        if (a.top == 0) continue;
        int above = 0;
        for (int p = 0; p < a.parts; ++p) {
            const uint64_t y = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(bar >> 32), p) << 32 |
                               (uint32_t)__builtin_amdgcn_readlane((int)bar, p);
            above += y > bar || (y == bar && p < (t & 63));
        }
        const int at = __builtin_ctzll(__ballot((t & 63) < a.parts && above == (a.top + a.each - 1) / a.each - 1));
        bar = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(bar >> 32), at) << 32 |
              (uint32_t)__builtin_amdgcn_readlane((int)bar, at);
        if (t < kMostTop) best[t] = 0;
        if (t == 0) count = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (key[i] && key[i] >= bar) keys[atomicAdd(&count, 1)] = key[i];  // (any order: they are ranked)
        __syncthreads();
        const int n = count;
        for (int i = t; i < n; i += kLogThreads) {
            const uint64_t k = keys[i];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += keys[j] > k;
            if (rank < a.top) best[rank] = k;
        }
        __syncthreads();
        if (t < a.top) finish_top(a, r, t, best[t], x.lse(a.scale));
        __syncthreads();
    }
}

// The log probabilities of tokens that name their rows, from the rows' lse: a thread each.
// Bound by the latency of its loads, one after the other: 4 us.
template <int TYPE>
__global__ __launch_bounds__(kLogThreads) void logprob_pick_kernel(LogprobArgs a) {
    const int64_t j = (int64_t)blockIdx.x * kLogThreads + threadIdx.x;
    if (j >= a.count) return;
    const int token = a.tokens[j], row = a.token_rows[j];
    a.logprob[j] = token < 0 || token >= a.vocab || row < 0 || row >= a.rows ? 0.0f :
        logprob_of(Block<TYPE>::one(a.logits + row * a.stride + (int64_t)token * Block<TYPE>::kBytes), a.scale, a.lse[row]);
}

// Gradients: every logit read and every gradient written once, at the same place.  With u
// = c x - lse and p = e^u the gradient of a logit is c (g_l ([it is the token] - p) - g_h p (u + H)).
//
// Bound by those bytes: 4096 rows of 131072 in bf16, 2.15 GB, in 358 us, 6.0 TB/s; 64 rows
// of 32003 in fp32, 16 MB, in 6.2 us.  Without ALIKE the elements are stored one by one, for
// what a thread has read are parts of two of the gradient's 16 bytes: 786 us.
struct GradientArgs {
    const uint8_t* logits;
    uint8_t* grad;
    int64_t stride, grad_stride;  // bytes
    const int32_t* tokens;
    const float* lse;
    const float* entropy;
    const float* grad_logprob;
    const float* grad_entropy;
    int64_t rows;
    int32_t vocab, parts;
    float scale;
};

constexpr int kGradAtOnce = 4, kGradBlocks = kLogThreads * kGradAtOnce;

template <int TYPE, bool ENTROPY, bool ALIKE>
__global__ __launch_bounds__(kLogThreads) void logprob_backward_kernel(GradientArgs a) {
    using B = Block<TYPE>;
    const int t = (int)threadIdx.x;
    const int part = (int)blockIdx.x;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const Row<TYPE> row(a.logits + r * a.stride, a.vocab);
        uint8_t* const out = a.grad + r * a.grad_stride - row.phase * B::kBytes;
        const float lse = a.lse[r];
        const int token = a.tokens[r];
        const bool none = lse == -INFINITY;
        float gl = a.grad_logprob ? a.grad_logprob[r] : 0.0f, ge = 0.0f, h = 0.0f;
        if (token < 0 || token >= a.vocab || none) gl = 0.0f;
        if constexpr (ENTROPY) {
            ge = none ? 0.0f : a.grad_entropy[r];
            h = a.entropy[r];
        }
        const auto of = [&](float x, int word) {
            const float u = none ? -INFINITY : __builtin_fmaf(x, a.scale, -lse);
            const float p = __builtin_amdgcn_exp2f(u * 1.44269504f);
            float g = -gl * p;
            if constexpr (ENTROPY) g = __builtin_fmaf(-ge * p, __builtin_fmaxf(u, -1000.0f) + h, g);
            if (word == token) g = g + gl;
            return g * a.scale;
        };
        for (int b0 = part * kGradBlocks + t; b0 < row.blocks; b0 += a.parts * kGradBlocks) {
            u32x4 v[kGradAtOnce];
#pragma unroll
            for (int k = 0; k < kGradAtOnce; ++k) {
                const int b = b0 + k * kLogThreads;
                if (b < row.blocks && row.whole(b)) v[k] = row.raw(b);
            }
#pragma unroll
            for (int k = 0; k < kGradAtOnce; ++k) {
                const int b = b0 + k * kLogThreads;
                if (b >= row.blocks) break;
                const bool whole = row.whole(b);
                float x[B::kN];
                if (whole)
                    B::widen(v[k], x);
                else
                    row.some(b, x);
#pragma unroll
                for (int i = 0; i < B::kN; ++i) x[i] = of(x[i], row.word(b, i));
                if (ALIKE && whole) {
                    *reinterpret_cast<u32x4*>(out + (int64_t)b * 16) = B::narrow(x);
                } else {
#pragma unroll
                    for (int i = 0; i < B::kN; ++i)
                        if (row.word(b, i) >= 0 && row.word(b, i) < a.vocab)
                            B::put(out + ((int64_t)b * B::kN + i) * B::kBytes, x[i]);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Host side

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
uint64_t up256(uint64_t v) { return (v + 255u) & ~uint64_t(255); }
int type_bytes(int type) { return type == RAC_TYPE_FP32 ? 4 : 2; }
constexpr int64_t kMostGroups = 1 << 20;  // workgroups of a launch: a kernel of a call's rows goes on with further ones

template <class A>
rac_status launch(void (*kernel)(A), int64_t x, int64_t y, int threads, const A& args, hipStream_t st) {
    A a = args;
    void* p[] = {&a};
    x = x < kMostGroups ? x : kMostGroups;
    const int64_t most = kMostGroups / x < 65535 ? kMostGroups / x : 65535;
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)x, (unsigned)(y < most ? y : most)),
                           dim3((unsigned)threads), p, 0, st) == hipSuccess ? RAC_OK : RAC_ERR_HIP;
}

bool rotary_dim_valid(int32_t d) { return d >= 16 && d <= 256 && d % 16 == 0; }

bool rotary_valid(const rac_rotary_config* c) {
    return c && c->rows >= 0 && c->rows <= (1 << 24) && c->q_heads >= 1 && c->q_heads <= 4096 && c->k_heads >= 0 &&
           c->k_heads <= 4096 && rotary_dim_valid(c->head_dim) && rotary_dim_valid(c->rotary_dim) &&
           c->rotary_dim <= c->head_dim && c->type >= RAC_TYPE_BF16 && c->type <= RAC_TYPE_FP32 &&
           (c->layout == RAC_ROTARY_INTERLEAVED || c->layout == RAC_ROTARY_HALF) &&
           (c->transpose == 0 || c->transpose == 1) && isfinite(c->amplitude);
}

template <int TYPE>
void (*rotary_of(bool half))(RotaryArgs) { return half ? rotary_kernel<TYPE, true> : rotary_kernel<TYPE, false>; }

bool logprob_valid(const rac_logprob_config* c) {
    return c && c->rows >= 0 && c->rows <= (1 << 24) && c->vocab >= 1 && c->vocab <= (1 << 24) && c->tokens >= 0 &&
           c->tokens <= (1 << 24) && c->top >= 0 && c->top <= kMostTop && c->type >= RAC_TYPE_BF16 &&
           c->type <= RAC_TYPE_FP32 && (c->scale == 0.0f || (c->scale >= 0x1p-40f && c->scale <= 0x1p40f));
}

// How rows are cut.  Without alternatives: few rows so that every compute unit has work,
// into parts of at least two blocks a thread (4 rows of 32000 in bf16 6.3 us, with four
// blocks 7.1; 256 rows of 131072 19.4 us in four parts, 27.8 in two).  With them: into as few
// parts as workgroups of 512 threads hold in registers, for an own look at alternatives and a
// join cost more than the bytes (a row of 32000, 8 alternatives: 9.0 us, in seven parts 11.1;
// 128 rows 10.0 and 14.6).  256 threads do if the part fits (128 rows of 32000 in eight parts
// 14.6 us, with 512 threads 19.7).  Longer rows are read twice, as if none were wanted (held
// in registers 600 rows of 131072 take 56 us, read twice 75).
struct LogprobCut {
    int parts, part_blocks, threads;
    bool held;
};

LogprobCut cut_of(const rac_logprob_config* c) {
    const int64_t blocks = ((int64_t)c->vocab * type_bytes(c->type) + 15) / 16 + 1, rows = c->rows > 0 ? c->rows : 1;
    int64_t parts = rows >= 512 ? 1 : 1024 / rows;
    const int64_t most = blocks / (2 * kLogThreads);
    parts = parts < most ? parts : most;
    parts = parts < 1 ? 1 : parts > kMostParts ? kMostParts : parts;
    const int64_t hold = (blocks + kHeld * 512 - 1) / (kHeld * 512);
    LogprobCut r{};
    r.held = c->top > 0 && hold <= kMostParts;
    if (r.held) parts = hold;
    r.parts = (int)parts;
    r.part_blocks = (int)((blocks + parts - 1) / parts);
    r.threads = r.held && r.part_blocks > kHeld * 256 ? 512 : 256;
    return r;
}

template <int TYPE, bool ENTROPY>
void (*logprob_of_form(const LogprobCut& cut, bool top))(LogprobArgs) {
    if (!top) return logprob_kernel<TYPE, ENTROPY, false, 256, false>;
    if (!cut.held) return logprob_kernel<TYPE, ENTROPY, true, 256, false>;
    return cut.threads == 512 ? logprob_kernel<TYPE, ENTROPY, true, 512, true> : logprob_kernel<TYPE, ENTROPY, true, 256, true>;
}
template <int TYPE>
void (*logprob_of_type(const LogprobCut& cut, bool entropy, bool top))(LogprobArgs) {
    return entropy ? logprob_of_form<TYPE, true>(cut, top) : logprob_of_form<TYPE, false>(cut, top);
}

template <int TYPE>
void (*backward_of(bool entropy, bool alike))(GradientArgs) {
    return entropy ? alike ? logprob_backward_kernel<TYPE, true, true> : logprob_backward_kernel<TYPE, true, false>
                   : alike ? logprob_backward_kernel<TYPE, false, true> : logprob_backward_kernel<TYPE, false, false>;
}

// Rows of `vocab` elements that do not reach into each other.
bool rows_apart(int64_t stride, const rac_logprob_config* c) {
    return stride >= c->vocab && stride <= (int64_t(1) << 40);
}

}  // namespace

extern "C" {

rac_status rac_rotary_frequencies(int32_t rotary_dim, double base, double factor, int32_t trained, double slow,
                                  double fast, double* turns) {
    if (!rotary_dim_valid(rotary_dim) || !turns || !(base > 1.0) || !isfinite(base) || !(factor > 0.0) ||
        !isfinite(factor) || trained < 0 || !(slow >= 0.0) || !(fast > slow) || !isfinite(fast))
        return RAC_ERR_INVALID;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / rotary_dim) / 6.283185307179586476925;
        double keep = (trained * f - slow) / (fast - slow);
        keep = keep < 0.0 || trained == 0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        turns[i] = f * (keep + (1.0 - keep) / factor);
    }
    return RAC_OK;
}

rac_status rac_rotary(const rac_rotary_config* cfg, const int32_t* pos, const double* freq,
                      const rac_rotary_tensors* t, rac_stream_t stream) {
    if (!rotary_valid(cfg) || !t) return RAC_ERR_INVALID;
    if (cfg->rows == 0) return RAC_OK;
    const int bytes = type_bytes(cfg->type), keys = cfg->k_heads > 0;
    const int64_t q_row = (int64_t)cfg->q_heads * cfg->head_dim, k_row = (int64_t)cfg->k_heads * cfg->head_dim;
    if (!pos || !freq || !t->q || !t->q_out || (keys && (!t->k || !t->k_out))) return RAC_ERR_INVALID;
    const int64_t far = int64_t(1) << 36;
    if (t->q_stride < q_row || t->q_out_stride < q_row || t->q_stride % 8 || t->q_out_stride % 8 || t->q_stride > far ||
        t->q_out_stride > far)
        return RAC_ERR_INVALID;
    if (keys && (t->k_stride < k_row || t->k_out_stride < k_row || t->k_stride % 8 || t->k_out_stride % 8 ||
                 t->k_stride > far || t->k_out_stride > far))
        return RAC_ERR_INVALID;
    // (in place means the same rows)
    if ((t->q == t->q_out && t->q_stride != t->q_out_stride && cfg->rows > 1) ||
        (keys && t->k == t->k_out && t->k_stride != t->k_out_stride && cfg->rows > 1))
        return RAC_ERR_INVALID;
    if (!aligned(pos, 4) || !aligned(freq, 8) || !aligned(t->q, 16) || !aligned(t->q_out, 16) ||
        (keys && (!aligned(t->k, 16) || !aligned(t->k_out, 16))))
        return RAC_ERR_ALIGN;
    RotaryArgs a{};
    a.pos = pos;
    a.freq = freq;
    a.in[0] = static_cast<const uint8_t*>(t->q);
    a.in[1] = static_cast<const uint8_t*>(t->k);
    a.out[0] = static_cast<uint8_t*>(t->q_out);
    a.out[1] = static_cast<uint8_t*>(t->k_out);
    a.in_stride[0] = t->q_stride * bytes;
    a.in_stride[1] = t->k_stride * bytes;
    a.out_stride[0] = t->q_out_stride * bytes;
    a.out_stride[1] = t->k_out_stride * bytes;
    a.rows = cfg->rows;
    a.amplitude = cfg->amplitude;
    a.sign = cfg->transpose ? -cfg->amplitude : cfg->amplitude;
    a.q_heads = cfg->q_heads;
    a.heads = cfg->q_heads + cfg->k_heads;
    a.head_bytes = cfg->head_dim * bytes;
    a.pairs = cfg->rotary_dim / 2;
    const bool half = cfg->layout == RAC_ROTARY_HALF, in_place = t->q == t->q_out && (!keys || t->k == t->k_out);
    const int turned = cfg->rotary_dim * bytes / 16, kept = in_place ? 0 : (cfg->head_dim - cfg->rotary_dim) * bytes / 16;
    a.turned = half ? turned / 2 : turned;
    a.pieces = a.turned + kept;
    const int per = a.heads * a.pieces;
    // (as many rows as give every thread a piece: 100000 rows of 8 + 8 heads of 64 channels
    // 109 us, with a row a workgroup 170; of 1 + 1 head 20 and 96)
    a.each = per >= kRotaryThreads ? 1 : kRotaryThreads / per < kRotaryRows ? kRotaryThreads / per : kRotaryRows;
    a.by_pieces = (uint32_t)(((uint64_t(1) << 32) + a.pieces - 1) / a.pieces);
    a.by_row = (uint32_t)(((uint64_t(1) << 32) + per - 1) / per);
    const auto kernel = cfg->type == RAC_TYPE_FP32 ? rotary_of<RAC_TYPE_FP32>(half)
                      : cfg->type == RAC_TYPE_FP16 ? rotary_of<RAC_TYPE_FP16>(half) : rotary_of<RAC_TYPE_BF16>(half);
    return launch(kernel, (a.rows + a.each - 1) / a.each, 1, kRotaryThreads, a, stream);
}

size_t rac_logprobs_workspace(const rac_logprob_config* cfg) {
    if (!logprob_valid(cfg)) return 0;
    const int parts = cut_of(cfg).parts;
    const uint64_t items = parts > 1 ? (uint64_t)cfg->rows * parts : 0;
    return (size_t)(256 + up256(items * 16) + up256(items * cfg->top * 8));
}

rac_status rac_logprobs(const rac_logprob_config* cfg, const rac_logprob_tensors* t, void* workspace,
                        size_t workspace_bytes, rac_stream_t stream) {
    if (!logprob_valid(cfg) || !t) return RAC_ERR_INVALID;
    if (!t->token_rows && cfg->tokens != 0 && cfg->tokens != cfg->rows) return RAC_ERR_INVALID;
    if (cfg->tokens > 0 && (!t->tokens || !t->logprob)) return RAC_ERR_INVALID;
    if (cfg->rows > 0 && (!t->logits || !t->lse || !workspace || !rows_apart(t->stride, cfg))) return RAC_ERR_INVALID;
    if (cfg->rows > 0 && cfg->top > 0 && (!t->top_ids || !t->top_logprobs)) return RAC_ERR_INVALID;
    const int bytes = type_bytes(cfg->type);
    if (!aligned(t->logits, bytes) || !aligned(t->tokens, 4) || !aligned(t->token_rows, 4) || !aligned(t->logprob, 4) ||
        !aligned(t->lse, 4) || !aligned(t->entropy, 4) || !aligned(t->top_ids, 4) || !aligned(t->top_logprobs, 4) ||
        !aligned(workspace, 256))
        return RAC_ERR_ALIGN;
    if (cfg->rows > 0 && workspace_bytes < rac_logprobs_workspace(cfg)) return RAC_ERR_CAPACITY;
    const float scale = cfg->scale == 0.0f ? 1.0f : cfg->scale;
    const LogprobCut cut = cut_of(cfg);
    const int parts = cut.parts;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    LogprobArgs a{static_cast<const uint8_t*>(t->logits), t->stride * bytes, t->tokens, t->token_rows, t->logprob, t->lse,
                  t->entropy, t->top_ids, t->top_logprobs, reinterpret_cast<float*>(ws),
                  reinterpret_cast<uint64_t*>(ws + up256((uint64_t)cfg->rows * parts * 16)), cfg->rows, cfg->vocab,
                  cfg->tokens, cfg->top, parts, cut.part_blocks, (cfg->top + parts - 1) / parts, scale, scale * 1.44269504f, Sums::kSlack / (scale * 1.44269504f)};
    const int type = cfg->type;
    rac_status st = RAC_OK;
    if (cfg->rows > 0) {
        const bool e = t->entropy != nullptr, top = cfg->top > 0;
        const auto kernel = type == RAC_TYPE_FP32 ? logprob_of_type<RAC_TYPE_FP32>(cut, e, top)
                          : type == RAC_TYPE_FP16 ? logprob_of_type<RAC_TYPE_FP16>(cut, e, top)
                                                  : logprob_of_type<RAC_TYPE_BF16>(cut, e, top);
        st = launch(kernel, parts, a.rows, cut.threads, a, stream);
        if (st == RAC_OK && parts > 1)
            st = launch(type == RAC_TYPE_FP32 ? logprob_join_kernel<RAC_TYPE_FP32>
                      : type == RAC_TYPE_FP16 ? logprob_join_kernel<RAC_TYPE_FP16> : logprob_join_kernel<RAC_TYPE_BF16>,
                        a.rows, 1, kLogThreads, a, stream);
    }
    if (st == RAC_OK && t->token_rows && cfg->tokens > 0)
        st = launch(type == RAC_TYPE_FP32 ? logprob_pick_kernel<RAC_TYPE_FP32>
                  : type == RAC_TYPE_FP16 ? logprob_pick_kernel<RAC_TYPE_FP16> : logprob_pick_kernel<RAC_TYPE_BF16>,
                    ((int64_t)cfg->tokens + kLogThreads - 1) / kLogThreads, 1, kLogThreads, a, stream);
    return st;
}

rac_status rac_logprobs_backward(const rac_logprob_config* cfg, const rac_logprob_gradients* g, rac_stream_t stream) {
    if (!logprob_valid(cfg) || !g || cfg->tokens != cfg->rows) return RAC_ERR_INVALID;
    if (cfg->rows == 0) return RAC_OK;
    if (!g->logits || !g->tokens || !g->lse || !g->grad_logits || (!g->grad_logprob && !g->grad_entropy) ||
        (g->grad_entropy && !g->entropy) || !rows_apart(g->stride, cfg) || !rows_apart(g->grad_stride, cfg))
        return RAC_ERR_INVALID;
    if (g->logits == g->grad_logits && g->stride != g->grad_stride && cfg->rows > 1) return RAC_ERR_INVALID;
    const int bytes = type_bytes(cfg->type);
    if (!aligned(g->logits, bytes) || !aligned(g->grad_logits, bytes) || !aligned(g->tokens, 4) || !aligned(g->lse, 4) ||
        !aligned(g->entropy, 4) || !aligned(g->grad_logprob, 4) || !aligned(g->grad_entropy, 4))
        return RAC_ERR_ALIGN;
    const int64_t blocks = ((int64_t)cfg->vocab * bytes + 15) / 16 + 1;
    const int64_t parts = (blocks + kGradBlocks - 1) / kGradBlocks;
    GradientArgs a{static_cast<const uint8_t*>(g->logits), static_cast<uint8_t*>(g->grad_logits), g->stride * bytes,
                   g->grad_stride * bytes, g->tokens, g->lse, g->entropy, g->grad_logprob, g->grad_entropy, cfg->rows,
                   cfg->vocab, (int32_t)parts, cfg->scale == 0.0f ? 1.0f : cfg->scale};
    // (logits and gradients lie alike in every row if they do in the first and their rows are as far apart, modulo 16)
    const bool alike = ((reinterpret_cast<uintptr_t>(a.logits) ^ reinterpret_cast<uintptr_t>(a.grad)) & 15) == 0 &&
                       ((a.stride ^ a.grad_stride) & 15) == 0;
    const bool entropy = g->grad_entropy != nullptr;
    const auto kernel = cfg->type == RAC_TYPE_FP32 ? backward_of<RAC_TYPE_FP32>(entropy, alike)
                      : cfg->type == RAC_TYPE_FP16 ? backward_of<RAC_TYPE_FP16>(entropy, alike)
                                                   : backward_of<RAC_TYPE_BF16>(entropy, alike);
    return launch(kernel, parts, a.rows, kLogThreads, a, stream);
}

}  // extern "C"
