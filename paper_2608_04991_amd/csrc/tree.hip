// tree.hip - gfx950 kernels and C ABI of the attention of drafted trees over
// the paged cache.  The contract is in include/rac_cache.h.
#include <math.h>

#include "cache_common.h"

namespace {

// Where the workgroups of a sequence, and its partial results, begin, and what it brings.
struct alignas(16) SeqPlan {
    int32_t base, slot, chunks, q0, m, d0, n, length;
};

struct TreeArgs {
    const uint8_t* pool;
    const int32_t* table;
    const int32_t* lengths;
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* q_start;
    const int32_t* draft_start;
    const uint64_t* mask;
    uint16_t* out;
    float* lse;
    int64_t q_stride, kv_stride, out_stride;
    int32_t layers, layer, heads, group, dim, log_page, pages, seqs, max_pages;
    int32_t rows, max_rows, draft_rows, max_draft, window, mask_words;
    float scale2;   // of the scores, times log2(e)
    float k_scale, v_scale;
    int32_t target;     // parts wanted (0: sequences are not split)
    int32_t min_chunk;  // fewest key tiles of a part
    float* parts;       // [slots] partial results
    int32_t slots;
    SeqPlan* plan;      // [seqs + 1], or null: every workgroup finds its work by itself
    int32_t m;          // query rows a workgroup
};

// What a sequence brings to the call, whatever the device arrays hold.
struct Seq {
    int q0, m;    // first query row, rows
    int d0, n;    // first drafted row, drafted tokens
    int length;   // committed tokens
};

__device__ __forceinline__ Seq seq_of(const TreeArgs& a, int s) {
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

__device__ __forceinline__ Sight sight_of(const TreeArgs& a, const Seq& s, int i) {
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

// Two floats in the 16-bit type, round to nearest even.
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (TYPE == RAC_CACHE_FP16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, f16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// One of them as a float.
template <int TYPE>
__device__ __forceinline__ float widen2(uint32_t u, int i) {
    if constexpr (TYPE == RAC_CACHE_FP16)
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(i ? u >> 16 : u));
    else
        return __uint_as_float(i ? u & 0xFFFF0000u : u << 16);
}

// Orders a wavefront's LDS writes before its later reads by other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The largest of three; a NaN among them is passed over.  (__builtin_fmaxf adds
// an instruction to each operand that might be a signalling NaN.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The four lanes l, l ^ 16, l ^ 32, l ^ 48 of a query row.
__device__ __forceinline__ float max_row(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __builtin_fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_row(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ---------------------------------------------------------------------------
// The work.  Query rows of one key-value head are the (node, query head) pairs
// of a sequence, node by node; a workgroup takes M of them and a run of key
// tiles.  Keys come in tiles of kTile: the committed ones from the first that
// the window reaches, then the drafted ones.
constexpr int kTile = 32;
constexpr int kWaves = 4;

struct Work {
    int seq, head, row_tile;
    int chunk, chunks;  // the part of the key tiles, and how many parts there are
    int slot;           // where its partial result goes
    Seq q;
};

__device__ __forceinline__ int committed_tile0(const TreeArgs& a, const Seq& q) {
    const int from = a.window > 0 && q.length > a.window ? q.length - a.window : 0;
    return from / kTile;
}

// Key tiles of a sequence.
__device__ __forceinline__ int key_tiles(const TreeArgs& a, const Seq& q) {
    return (q.length + kTile - 1) / kTile - committed_tile0(a, q) + (q.n + kTile - 1) / kTile;
}

// How a sequence is cut: tiles of M query rows, and parts of its key tiles.
struct Cut {
    int tiles, chunks;
};

__device__ __forceinline__ Cut cut_of(const TreeArgs& a, const Seq& q, int most) {
    const int keys = key_tiles(a, q);
    return Cut{(q.m * a.group + a.m - 1) / a.m, keys > most ? (keys + most - 1) / most : 1};
}

// Parts of at most this many key tiles: all parts of all sequences together just
// fill the workgroups that the device holds at once (a.target), or twice that
// where the sequences alone take nearly half of them and rounding their parts up
// would leave many idle, and are of like size whatever the lengths.  sum(f): the
// sum over all sequences of f(tiles of rows, tiles of keys).  The first size would
// give as many parts if none were rounded up; a second round of a few workgroups
// costs more than parts a little longer (us, with the first size alone and now:
// 32 x 16k tokens 236, 216; 32 rows each 174, 143; trees of 64 nodes 110, 94;
// 64 x 4k tokens 69, 66).
template <class Sum>
__device__ __forceinline__ int chunk_tiles(const TreeArgs& a, Sum sum) {
    if (a.target == 0) return 1 << 30;
    const float heads = (float)a.heads;
    const float units = heads * sum([](float t, float) { return t; });
    const float work = heads * sum([](float t, float k) { return t * k; });
    const float full = (float)a.target, want = a.m <= 32 && units > 0.4f * full && units < full ? 2.0f * full : full;
    // (the margin keeps sums in fp32 from asking for more than a.slots)
    float most = __builtin_fminf(work / want * 1.0001f + 1.0f, 1e9f);
    for (int i = 0; i < 3 && units < want; ++i) {
        const float whole = __builtin_floorf(most);
        const float parts = heads * sum([whole](float t, float k) { return t * __builtin_ceilf(k / whole); });
        if (parts <= want) break;
        most = __builtin_fminf(most * (parts / want) + 0.5f, 1e9f);
    }
    return (int)most < a.min_chunk ? a.min_chunk : (int)most;
}

// Up to 64 sequences need no launch ahead: a lane a sequence, each wavefront
// finds the cuts by itself.  That is the faster side up to the last size that a
// wavefront's lanes can hold (us, so and with tree_plan_kernel ahead: 8 drafted
// trees of up to 12 tokens 10.9, 13.3; one token of 8k 16.2, 19.3; 32 x 16k tokens
// 217, 221; 64 x 4k tokens 72, 75).
struct LaneSeq {
    Seq q;
    Cut c;
    int base, slot;
};

__device__ __forceinline__ LaneSeq lane_seq(const TreeArgs& a) {
    const int lane = (int)threadIdx.x & 63;
    LaneSeq r{Seq{0, 0, 0, 0, 0}, Cut{0, 1}, 0, 0};
    float t = 0.0f, k = 0.0f;
    if (lane < a.seqs) {
        r.q = seq_of(a, lane);
        t = (float)cut_of(a, r.q, 1 << 30).tiles;
        k = (float)key_tiles(a, r.q);
    }
    const int most = chunk_tiles(a, [&](auto f) {
        const float all = scan_wave(f(t, k));
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, all), 63));
    });
    if (lane < a.seqs) r.c = cut_of(a, r.q, most);
    const int units = r.c.tiles * r.c.chunks * a.heads;
    if (a.m <= 32) {
        const int split = r.c.chunks > 1 ? units : 0;
        r.base = scan_wave(units) - units;
        r.slot = scan_wave(split) - split;
        return r;
    }
    // (many rows) the sequences with the longest parts first: what starts last ends last
    const int keys = lane < a.seqs ? (key_tiles(a, r.q) + r.c.chunks - 1) / r.c.chunks : -1;
    for (int j = 0; j < a.seqs; ++j) {
        const int k = __builtin_amdgcn_readlane(keys, j), u = __builtin_amdgcn_readlane(units, j);
        const bool ahead = k > keys || (k == keys && j < lane);
        r.base += ahead ? u : 0;
        r.slot += ahead && __builtin_amdgcn_readlane(r.c.chunks, j) > 1 ? u : 0;
    }
    return r;
}

// The last of n ascending values that is at most x; a wavefront looks at 64
// at a time (at(0) <= x).
template <class At>
__device__ __forceinline__ int last_at_most(int n, int x, At at) {
    const int lane = (int)threadIdx.x & 63;
    int lo = 0;
    while (n > 64) {
        const int step = (n + 63) / 64;
        const int k = __popcll(__ballot(lane * step < n && at(lo + lane * step) <= x)) - 1;
        lo += k * step;
        n = n - k * step < step ? n - k * step : step;
    }
    return lo + __popcll(__ballot(lane < n && at(lo + lane) <= x)) - 1;
}

// Which work workgroup `block` has; false: none.
__device__ __forceinline__ bool find_work(const TreeArgs& a, int block, Work& w) {
    int i, tiles;
    if (a.plan) {
        // 64 records at a time, the last step with all that a record holds
        const int lane = (int)threadIdx.x & 63, all = a.plan[a.seqs].base;
        int lo = 0, n = a.seqs;
        while (n > 64) {
            const int step = (n + 63) / 64;
            const int k = __popcll(__ballot(lane * step < n && a.plan[lo + lane * step].base <= block)) - 1;
            lo += k * step;
            n = n - k * step < step ? n - k * step : step;
        }
        SeqPlan p{};
        if (lane < n) p = a.plan[lo + lane];
        const int at = __popcll(__ballot(lane < n && p.base <= block)) - 1;
        if (block >= all || at < 0) return false;
        const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        w.seq = __builtin_amdgcn_readfirstlane(lo + at);
        w.q = Seq{of(p.q0), of(p.m), of(p.d0), of(p.n), of(p.length)};
        tiles = cut_of(a, w.q, 1 << 30).tiles;
        w.chunks = of(p.chunks);
        i = block - of(p.base);
        w.slot = of(p.slot) + i;
    } else {
        const LaneSeq l = lane_seq(a);
        const uint64_t mine = __ballot(block >= l.base && block < l.base + l.c.tiles * l.c.chunks * a.heads);
        if (!mine) return false;
        const int at = __builtin_ctzll(mine);
        const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        w.seq = at;
        w.q = Seq{of(l.q.q0), of(l.q.m), of(l.q.d0), of(l.q.n), of(l.q.length)};
        tiles = of(l.c.tiles);
        w.chunks = of(l.c.chunks);
        i = block - of(l.base);
        w.slot = of(l.slot) + i;
    }
    if (i < 0) return false;
    w.head = i % a.heads;
    i /= a.heads;
    w.chunk = i % w.chunks;
    w.row_tile = tiles - 1 - i / w.chunks;  // (the last rows of a causal sequence see most)
    // (ranges that overlap, as a broken q_start has them, may ask for more parts than there is room for)
    return w.row_tile >= 0 && (w.chunks == 1 || (uint32_t)w.slot < (uint32_t)a.slots);
}

// The plan of more sequences: one workgroup, four sequences a thread.  Bound by
// the latency of its few dependent reads and sums: 5.0 us for 200 sequences.
constexpr int kPlanThreads = 1024;

__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(TreeArgs a) {
    constexpr int kPer = 4;  // sequences a thread (4096 / 1024)
    __shared__ int sums[kPlanThreads / 64];
    __shared__ float totals[kPlanThreads / 64];
    const int t = (int)threadIdx.x;
    Seq q[kPer];
    float tiles[kPer], keys[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = t + i * kPlanThreads;
        q[i] = Seq{0, 0, 0, 0, 0};
        tiles[i] = keys[i] = 0.0f;
        if (s < a.seqs) {
            q[i] = seq_of(a, s);
            tiles[i] = (float)cut_of(a, q[i], 1 << 30).tiles;
            keys[i] = (float)key_tiles(a, q[i]);
        }
    }
    const int most = chunk_tiles(a, [&](auto f) {
        const float all = scan_wave((f(tiles[0], keys[0]) + f(tiles[1], keys[1])) + (f(tiles[2], keys[2]) + f(tiles[3], keys[3])));
        __syncthreads();
        if ((t & 63) == 63) totals[t / 64] = all;
        __syncthreads();
        float total = 0.0f;
        for (int i = 0; i < kPlanThreads / 64; ++i) total = total + totals[i];
        return total;
    });
    int base = 0, slot = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = t + i * kPlanThreads;
        if (i * kPlanThreads > a.seqs) break;
        const Cut c = s < a.seqs ? cut_of(a, q[i], most) : Cut{0, 1};
        const int units = c.tiles * c.chunks * a.heads, split = c.chunks > 1 ? units : 0;
        int all_units, all_split;
        const int b = base + scan_workgroup<kPlanThreads / 64>(units, sums, &all_units);
        const int l = slot + scan_workgroup<kPlanThreads / 64>(split, sums, &all_split);
        if (s <= a.seqs) a.plan[s] = SeqPlan{b, l, c.chunks, q[i].q0, q[i].m, q[i].d0, q[i].n, q[i].length};
        base += all_units;
        slot += all_split;
    }
    if (t == 0 && a.seqs == kPer * kPlanThreads) a.plan[a.seqs] = SeqPlan{base, slot, 1, 0, 0, 0, 0, 0};
}

// ---------------------------------------------------------------------------
// LDS: a tile of 16-bit keys or values is kTile rows of DP / 8 pieces of 16
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

// Four of eight keys of channel 16 dt + lane % 16: the transposing read takes
// from the 16 lanes of a group the four 8-byte parts of four rows.
template <int DP>
__device__ __forceinline__ u32x2 read_column(const u32x4* tile, uint32_t lane, uint32_t dt, uint32_t half) {
    const uint32_t row = 16u * half + 4u * (lane >> 4) + ((lane >> 2) & 3u), c = 2u * dt + ((lane >> 1) & 1u);
    const u32x2* at = reinterpret_cast<const u32x2*>(tile + piece_at<DP>(row, c)) + (lane & 1u);
    typedef __attribute__((address_space(3))) s16x4* lds;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)at));
}

// What a wavefront keeps of its TM x 16 query rows.  With keys (values) as the
// first operand of the matrix cores, lane l holds everything of row l % 16:
// scores of keys 16 t + 4 (l / 16) + i, outputs of channels 16 t + 4 (l / 16) +
// i; the weights of the former are the second operand of the latter as they
// lie, if the values' keys are taken in the same order.
//
// KP = 2: a weight goes to the matrix cores as two 16-bit numbers, its rounding
// and the rest, so that only the output's rounding is left: with one, the two
// roundings together are 1.4 times the output's.  Where few rows wait for memory
// the second product costs nothing (32 x 16k tokens 217 us with it and without,
// one sequence of 8k 16), but with 256 channels, where one wavefront has all of it
// to do, 3 to 6% (32 x 8k tokens 330 us with it, 316 without).
//
// The largest weight of a row so far lies between 2^kUp and 2^(kUp + kSlack).  bf16
// has the exponents of the sums, so kUp = 0 does.  fp16 weights end below 2^16 and
// lose bits below 2^-14: as far up as they go, a weight keeps its 11 bits down to 2^-25
// of the largest (17 nats below it), and what is smaller is off by 2^-36 of it at most.
template <int TYPE, int DP, int TM>
struct Rows {
    static constexpr float kUp = TYPE == RAC_CACHE_FP16 ? 11.0f : 0.0f, kSlack = TYPE == RAC_CACHE_FP16 ? 4.0f : 8.0f;
    u32x4 q[TM][DP / 32];
    f32x4 o[TM][DP / 16];
    float m[TM];  // reference of the exponentials, log2: kUp to kUp + kSlack below the largest score so far
    float l[TM];  // sum of the weights over this lane's keys
    bool alone;   // a value that some row must not see is an infinity or NaN: the rows are redone one by one

    __device__ __forceinline__ void start() {
        alone = false;
#pragma unroll
        for (int r = 0; r < TM; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.0f;
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) o[r][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // Scores of the tile of keys in LDS.
    __device__ __forceinline__ void scores(const u32x4* kl, f32x4 (&s)[TM][2]) const {
        const uint32_t lane = threadIdx.x & 63u;
        constexpr int kAtOnce = TM > 1 ? 2 : DP / 32 < 4 ? DP / 32 : 4;
#pragma unroll
        for (int r = 0; r < TM; ++r) s[r][0] = s[r][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t0 = 0; t0 < DP / 32; t0 += kAtOnce) {
            u32x4 k[kAtOnce][2];
#pragma unroll
            for (int t = 0; t < kAtOnce; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) k[t][h] = kl[piece_at<DP>(16u * h + (lane & 15u), 4u * (t0 + t) + (lane >> 4))];
#pragma unroll
            for (int t = 0; t < kAtOnce; ++t)
#pragma unroll
                for (int r = 0; r < TM; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[r][h] = mma<TYPE>(k[t][h], q[r][t0 + t], s[r][h]);
        }
    }

    // The same of a tile that not every row sees all of: bits[r] has the keys
    // that this lane's row of r sees, `there` the keys whose values are loaded
    // (the others are zeros).  Returns whether some row must not see a loaded value.
    __device__ __forceinline__ bool hide(f32x4 (&s)[TM][2], const uint32_t (&bits)[TM], uint32_t there) const {
        const uint32_t first = 4u * ((threadIdx.x & 63u) >> 4);
        bool mixed = false;
#pragma unroll
        for (int r = 0; r < TM; ++r) {
            mixed |= bits[r] != there;
            const uint32_t b = bits[r] >> first;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][h][i] = b & (1u << (16 * h + i)) ? s[r][h][i] : -INFINITY;
        }
        return __any(mixed);
    }

    // Scores of NT tiles to weights, in the type and order that the values'
    // product takes.  c: factors of the scores, with log2(e) in them; vs: factors
    // of the values (8-bit pages).
    template <int NT, int KP>
    __device__ __forceinline__ void weights(const f32x4 (&s)[NT][TM][2], const float (&c)[NT], const float (&vs)[NT],
                                            u32x4 (&p)[NT][TM][KP]) {
        float top[TM];
        bool grow = false;
#pragma unroll
        for (int r = 0; r < TM; ++r) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f32x4 u = s[n][r][0], v = s[n][r][1];
                const float x = max3(max3(max3(u[0], u[1], u[2]), u[3], v[0]), v[1], v[2]);
                top[r] = n ? max3(top[r], x * c[n], v[3] * c[n]) : max3(x, v[3], v[3]) * c[n];
            }
            grow |= top[r] > m[r] + (kUp + kSlack);
        }
        if (__any(grow)) {  // (seldom: the reference need not be the maximum, only near it)
#pragma unroll
            for (int r = 0; r < TM; ++r) {
                const float now = __builtin_fmaxf(m[r], max_row(top[r]) - kUp);
                const float keep = now == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[r] - now);
                m[r] = now;
                l[r] = l[r] * keep;
#pragma unroll
                for (int t = 0; t < DP / 16; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[r][t][i] = o[r][t][i] * keep;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < TM; ++r) {
                const float ref = m[r] == -INFINITY ? 0.0f : m[r];
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r][i / 4][i % 4], c[n], -ref));
                l[r] = l[r] + (((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = e[2 * i], y = e[2 * i + 1];
                    if constexpr (TYPE == RAC_CACHE_FP8) {
                        x = x * vs[n];
                        y = y * vs[n];
                    }
                    const uint32_t u = pack2<TYPE>(x, y);
                    p[n][r][0][i] = u;
                    if constexpr (KP == 2) p[n][r][1][i] = pack2<TYPE>(x - widen2<TYPE>(u, 0), y - widen2<TYPE>(u, 1));
                }
            }
    }

    // Adds the values of the tile in LDS by their weights.
    template <int KP>
    __device__ __forceinline__ void values(const u32x4* vl, const u32x4 (&p)[TM][KP]) {
        const uint32_t lane = threadIdx.x & 63u;
        constexpr int kAtOnce = TM > 1 || DP == 64 ? 4 : 8;
#pragma unroll
        for (int t0 = 0; t0 < DP / 16; t0 += kAtOnce) {
            u32x4 v[kAtOnce];
#pragma unroll
            for (int t = 0; t < kAtOnce; ++t) {
                const u32x2 lo = read_column<DP>(vl, lane, t0 + t, 0), hi = read_column<DP>(vl, lane, t0 + t, 1);
                v[t] = u32x4{lo[0], lo[1], hi[0], hi[1]};
            }
#pragma unroll
            for (int t = 0; t < kAtOnce; ++t)
#pragma unroll
                for (int r = 0; r < TM; ++r)
#pragma unroll
                    for (int x = 0; x < KP; ++x) o[r][t0 + t] = mma<TYPE>(v[t], p[r][x], o[r][t0 + t]);
        }
    }

    // Two tiles, for many rows: the fragments of a step are read while the step
    // before is multiplied, and the first of the values while the weights are
    // formed (a read takes longer than its products). Chunks of a prompt of 2048
    // take 369 us with this and 377 without, 256 channels a head 61 and 64.
    struct KeyStep {
        u32x4 k[2][2];
    };
    struct ValueStep {
        u32x4 v[4];
    };
    static __device__ __forceinline__ KeyStep read_keys(const u32x4* kl, int t0) {
        const uint32_t lane = threadIdx.x & 63u;
        KeyStep x;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) x.k[t][h] = kl[piece_at<DP>(16u * h + (lane & 15u), 4u * (t0 + t) + (lane >> 4))];
        return x;
    }
    template <bool AHEAD>
    __device__ __forceinline__ void scores_of(const u32x4* k0, const u32x4* k1, f32x4 (&s)[2][TM][2]) const {
        if constexpr (!AHEAD) {
            scores(k0, s[0]);
            scores(k1, s[1]);
            return;
        }
        constexpr int kEach = DP / 64;  // steps a tile
        KeyStep now = read_keys(k0, 0);
#pragma unroll
        for (int i = 0; i < 2 * kEach; ++i) {
            const int n = i / kEach, t0 = i % kEach * 2;
            KeyStep next = now;
            if (i + 1 < 2 * kEach) next = read_keys((i + 1) / kEach ? k1 : k0, (i + 1) % kEach * 2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < TM; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        s[n][r][h] = mma<TYPE>(now.k[t][h], q[r][t0 + t], t0 + t ? s[n][r][h] : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
            now = next;
        }
    }
    static __device__ __forceinline__ ValueStep read_values(const u32x4* vl, int t0) {
        const uint32_t lane = threadIdx.x & 63u;
        ValueStep x;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const u32x2 lo = read_column<DP>(vl, lane, t0 + t, 0), hi = read_column<DP>(vl, lane, t0 + t, 1);
            x.v[t] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
        return x;
    }
    template <int KP>
    __device__ __forceinline__ void values_of(ValueStep now, const u32x4* v0, const u32x4* v1, const u32x4 (&p)[2][TM][KP]) {
        constexpr int kEach = DP / 64;
#pragma unroll
        for (int i = 0; i < 2 * kEach; ++i) {
            const int n = i / kEach, t0 = i % kEach * 4;
            ValueStep next = now;
            if (i + 1 < 2 * kEach) next = read_values((i + 1) / kEach ? v1 : v0, (i + 1) % kEach * 4);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < TM; ++r)
#pragma unroll
                    for (int x = 0; x < KP; ++x) o[r][t0 + t] = mma<TYPE>(now.v[t], p[n][r][x], o[r][t0 + t]);
            now = next;
        }
    }

    // Some row must not see some value of the tile: a weight of 0 hides it
    // unless it is an infinity or NaN (all exponent bits set).
    __device__ __forceinline__ void look(const u32x4* vl) {
        constexpr uint32_t kExp = TYPE == RAC_CACHE_FP16 ? 0x7C00u : 0x7F80u;
        bool odd = false;
#pragma unroll 2
        for (uint32_t i = threadIdx.x & 63u; i < kTile * DP / 8; i += 64u) {
            const u32x4 v = vl[i];
#pragma unroll
            for (int y = 0; y < 4; ++y) odd |= (v[y] & kExp) == kExp || (v[y] & (kExp << 16)) == (kExp << 16);
        }
        alone |= __any(odd);
    }
};

// Where a row lives (its node and query head), and what it sees.
struct RowAt {
    int node, head;
    Sight see;
};

__device__ __forceinline__ RowAt row_at(const TreeArgs& a, const Work& w, int row) {
    const int last = w.q.m * a.group - 1;
    row = row < last ? row : last;  // (rows past the last repeat it and are not stored)
    RowAt r;
    r.node = row / a.group;
    r.head = w.head * a.group + row % a.group;
    r.see = sight_of(a, w.q, r.node);
    return r;
}

// The arguments once more.  What only the start, the end or a rare path needs is
// read when it is needed: a kernel that keeps all of it in scalar registers over
// its loop has too few of them.
__device__ __forceinline__ TreeArgs args_again() {
    TreeArgs a;
#ifdef __HIP_DEVICE_COMPILE__
    uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    __builtin_memcpy(&a, (const void*)(const __attribute__((address_space(4))) void*)p, sizeof a);
#endif
    return a;
}

// The key axis of a workgroup, as its loop needs it.
struct Axis {
    const uint8_t* pool;   // keys of this layer and head in page 0
    uint32_t page_stride;  // in 256 bytes, which divide every page (2^38 bytes are the largest)
    uint32_t side;         // bytes from a page's keys to its values
    const int32_t* row;    // the sequence's table entries
    const uint16_t* k;     // drafted keys and values of this sequence and head
    const uint16_t* v;
    int64_t kv_stride;
    const uint64_t* mask;
    int mask_words;
    int max_pages, log_page, pages, dim, length, n;
    // the tiles that the rows see at all: committed ones [ca, ca + committed), then drafted ones from da on
    int ca, committed, da, count;
};

template <int TYPE>
__device__ __forceinline__ Axis axis_of(const TreeArgs& a, const Work& w, int from, int first, int end) {
    constexpr int kB = TYPE == RAC_CACHE_FP8 ? 1 : 2;
    const uint64_t plane = ((uint64_t)a.dim << a.log_page) * kB;
    Axis x;
    x.pool = a.pool + ((uint64_t)a.layer * 2 * a.heads + w.head) * plane;
    x.page_stride = (uint32_t)(plane / 128 * a.heads * a.layers);
    x.side = (uint32_t)(plane * a.heads);
    x.row = a.table + (size_t)w.seq * a.max_pages;
    const int64_t o = w.q.d0 * a.kv_stride + (int64_t)w.head * a.dim;
    x.k = a.k + o;
    x.v = a.v + o;
    x.kv_stride = a.kv_stride;
    x.mask = a.mask;
    x.mask_words = a.mask_words;
    x.max_pages = a.max_pages;
    x.log_page = a.log_page;
    x.pages = a.pages;
    x.dim = a.dim;
    x.length = w.q.length;
    x.n = w.q.n;
    const int c0 = committed_tile0(a, w.q), all = key_tiles(a, w.q), n = (w.q.length + kTile - 1) / kTile - c0;
    const int each = all / w.chunks, more = all % w.chunks;
    const int lo = w.chunk * each + (w.chunk < more ? w.chunk : more), hi = lo + each + (w.chunk < more);
    x.ca = c0 + (lo < n ? lo : n);
    x.da = lo > n ? lo - n : 0;
    int cb = c0 + (hi < n ? hi : n), db = hi > n ? hi - n : 0;
    if (x.ca < from / kTile) x.ca = from / kTile;
    if (x.da < first / kTile) x.da = first / kTile;
    const int e = (end + kTile - 1) / kTile;
    if (db > e) db = e;
    x.committed = cb > x.ca ? cb - x.ca : 0;
    x.count = x.committed + (db > x.da ? db - x.da : 0);
    return x;
}

// The table entries of ROWS keys from key row0 of a tile on, eight keys each.
template <int ROWS>
struct Pages {
    int p[ROWS / 8];
};

template <int ROWS>
__device__ __forceinline__ Pages<ROWS> pages_of(const Axis& x, int tile, int row0) {
    using cptr = const __attribute__((address_space(4))) int32_t*;  // read-only in this launch: scalar loads
    Pages<ROWS> r;
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i) {
        const int at = (tile * kTile + row0 + 8 * i) >> x.log_page;
        r.p[i] = ((cptr)x.row)[at < x.max_pages ? at : x.max_pages - 1];
    }
    return r;
}

// A tile's keys or values (or the rows [row0, row0 + ROWS) of it) on their way
// from memory to LDS, through registers: neighbouring lanes take the 16-byte
// pieces of a row.
template <int TYPE, int DP, int ROWS>
struct Load {
    static constexpr int kPieces = DP / 8, kRowsAtOnce = 64 / kPieces, kLoads = ROWS / kRowsAtOnce;       // 16 bits
    static constexpr int kPieces8 = DP / 16, kRowsAtOnce8 = 64 / kPieces8, kLoads8 = ROWS / kRowsAtOnce8;  // 8 bits
    static constexpr int kN = TYPE == RAC_CACHE_FP8 ? kLoads8 : kLoads;
    u32x4 x[kN];

    // Tile i of the axis, keys or values.  Every address lies in the pool or the
    // drafted rows whatever the tile lacks: what does not exist becomes zeros when
    // it is put.  (One sequence of loads: with one each for committed and drafted
    // tiles the registers of both are live, 37 more.)
    __device__ __forceinline__ void tile(const Axis& ax, int i, const Pages<ROWS>& pg, int row0, bool values) {
        const uint32_t lane = threadIdx.x & 63u;
        constexpr int kB = TYPE == RAC_CACHE_FP8 ? 1 : 2, kR = TYPE == RAC_CACHE_FP8 ? kRowsAtOnce8 : kRowsAtOnce;
        constexpr uint32_t kP = TYPE == RAC_CACHE_FP8 ? kPieces8 : kPieces;
        const uint32_t in = lane / kP, row_bytes = (uint32_t)(ax.dim * kB);
        const uint32_t c = (lane % kP * 16u < row_bytes ? lane % kP : 0u) * 16u;
        const bool past = i < ax.committed;
        const int tile = past ? ax.ca + i : ax.da + i - ax.committed;
        // (eight aligned rows lie in one page: its address is the same in all
        // lanes, but for the second eight of sixteen)
        const uint32_t inner = (kR > 8 ? in & 7u : in) * row_bytes + c;
        const uint8_t* const pool = ax.pool + (values ? ax.side : 0u);
        const uint8_t* eight[ROWS / 8];
#pragma unroll
        for (int g = 0; g < ROWS / 8; ++g) {
            const uint32_t p = (uint32_t)pg.p[g] < (uint32_t)ax.pages ? (uint32_t)pg.p[g] : 0u;
            eight[g] = pool + (((uint64_t)p * ax.page_stride << 8) +
                               ((uint32_t)(tile * kTile + row0 + 8 * g) & ((1u << ax.log_page) - 1u)) * row_bytes);
        }
        // (a drafted row past the last reads the last; offsets from the first row of
        // the tile, so that ROWS - 1 rows of up to 2^26 bytes are the most)
        const uint32_t stride = (uint32_t)(2 * ax.kv_stride);
        const int first = tile * kTile + row0, left = ax.n - 1 - first;
        const uint32_t rows = left <= 0 ? 0u : left < ROWS ? (uint32_t)left : (uint32_t)(ROWS - 1);
        const uint8_t* const draft = reinterpret_cast<const uint8_t*>((values ? ax.v : ax.k) + (int64_t)(first < ax.n ? first : ax.n - 1) * ax.kv_stride);
        const uint32_t own = past ? inner : in * stride + c, last = past ? ~0u : rows * stride + c;
#pragma unroll
        for (int y = 0; y < kN; ++y) {
            const uint8_t* at = eight[y * kR / 8];
            if constexpr (kR > 8) at = in >= 8u ? eight[(y * kR / 8 + 1) % (ROWS / 8)] : at;
            if constexpr (TYPE == RAC_CACHE_FP8) {
                at += (uint32_t)(y * kR % 8) * row_bytes + inner;
            } else {
                const uint32_t off = own + (past ? (uint32_t)(y * kR % 8) * row_bytes : (uint32_t)(y * kR) * stride);
                at = (past ? at : draft) + (off < last ? off : last);
            }
            x[y] = *reinterpret_cast<const u32x4*>(at);
        }
    }
    // Half a tile of drafted keys or values: with 8-bit pages the registers hold
    // no more, and these few last tiles come when they are put.
    __device__ __forceinline__ void drafted(const Axis& ax, const uint16_t* base, int tile, int row0) {
        const uint32_t lane = threadIdx.x & 63u, in = lane / kPieces;
        const uint32_t c = lane % kPieces * 8u < (uint32_t)ax.dim ? lane % kPieces : 0u;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            int row = tile * kTile + row0 + i * kRowsAtOnce + (int)in;
            row = row < ax.n ? row : ax.n - 1;
            x[i] = *reinterpret_cast<const u32x4*>(base + (int64_t)row * ax.kv_stride + 8u * c);
        }
    }
    // valid: the keys of the tile that exist.  clean: infinities and NaNs become zeros.
    __device__ __forceinline__ void put_drafted(u32x4* lds, const Axis& ax, const uint16_t* base, int tile, uint32_t valid, int row0,
                                                bool clean) {
        if constexpr (TYPE != RAC_CACHE_FP8) {
            put_wide(lds, ax, valid, row0, clean);
        } else {
            constexpr int kRows = kLoads8 * kRowsAtOnce;
#pragma unroll 1
            for (int r = 0; r < ROWS; r += kRows) {
                drafted(ax, base, tile, row0 + r);
                put_wide(lds, ax, valid, row0 + r, clean);
            }
        }
    }
    __device__ __forceinline__ void put_committed(u32x4* lds, const Axis& ax, uint32_t valid, int row0, bool clean) {
        if constexpr (TYPE != RAC_CACHE_FP8) {
            put_wide(lds, ax, valid, row0, clean);
        } else {
            const uint32_t lane = threadIdx.x & 63u, c = lane % kPieces8, in = lane / kPieces8;
            if (valid != ~0u || ax.dim != DP)
#pragma unroll
                for (int i = 0; i < kLoads8; ++i)
                    x[i] &= (c * 16u < (uint32_t)ax.dim && (valid >> (row0 + i * kRowsAtOnce8 + in)) & 1u) ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < kLoads8; ++i)
#pragma unroll
                for (uint32_t y = 0; y < 2; ++y) {
                    u32x4 w = widen8(x[i][2 * y], x[i][2 * y + 1]);
                    if (clean) w = finite(w);
                    lds[piece_at<DP>(row0 + i * kRowsAtOnce8 + in, 2u * c + y)] = w;
                }
        }
    }
    __device__ __forceinline__ void put_zeros(u32x4* lds, int row0) {
        if constexpr (TYPE == RAC_CACHE_FP8) {
            for (uint32_t y = threadIdx.x & 63u; y < ROWS * DP / 8; y += 64u) lds[row0 * (DP / 8) + y] = u32x4{0u, 0u, 0u, 0u};
        }
    }
    __device__ __forceinline__ void put_wide(u32x4* lds, const Axis& ax, uint32_t valid, int row0, bool clean) {
        const uint32_t lane = threadIdx.x & 63u, c = lane % kPieces, in = lane / kPieces;
        if (valid != ~0u || ax.dim != DP)
#pragma unroll
            for (int i = 0; i < kN; ++i)
                x[i] &= (c * 8u < (uint32_t)ax.dim && (valid >> (row0 + i * kRowsAtOnce + in)) & 1u) ? ~0u : 0u;
        if (clean)
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = finite(x[i]);
#pragma unroll
        for (int i = 0; i < kN; ++i) lds[piece_at<DP>(row0 + i * kRowsAtOnce + in, c)] = x[i];
    }

    static __device__ __forceinline__ u32x4 finite(u32x4 v) {
        constexpr uint32_t kExp = TYPE == RAC_CACHE_FP16 ? 0x7C00u : 0x7F80u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] &= (v[i] & kExp) == kExp ? 0xFFFF0000u : ~0u;
            v[i] &= (v[i] & (kExp << 16)) == (kExp << 16) ? 0xFFFFu : ~0u;
        }
        return v;
    }

    // Eight e4m3 as bf16 (exact).
    static __device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b) {
        u32x4 r;
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
        return r;
    }
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// The keys of a tile that exist, of those from row0 on (bits as in the tile).
template <int ROWS>
__device__ __forceinline__ uint32_t exist_of(const Axis& x, int i, const Pages<ROWS>& pg, int row0) {
    if (i >= x.committed) return i < x.count ? low_bits(x.n - (x.da + i - x.committed) * kTile) : 0u;
    uint32_t r = low_bits(x.length - (x.ca + i) * kTile);
#pragma unroll
    for (int g = 0; g < ROWS / 8; ++g)
        if ((uint32_t)pg.p[g] >= (uint32_t)x.pages) r &= ~(0xFFu << (row0 + 8 * g));
    return r;
}

// What the rows of a workgroup see, in LDS: it is read for few tiles.
struct Seen {
    int from, first, end, mask_row;
};

__device__ __forceinline__ uint32_t bits_of(const Axis& x, const Seen& r, bool past, int tile) {
    if (past) return ~low_bits(r.from - tile * kTile);
    uint32_t b = low_bits(r.end - tile * kTile) & ~low_bits(r.first - tile * kTile);
    if (x.mask && b)  // (a mask reaches r.end)
        b &= reinterpret_cast<const uint32_t*>(x.mask + (size_t)r.mask_row * x.mask_words)[tile];
    return b;
}

__device__ __forceinline__ int min_wave(int v) {
    for (int o = 1; o < 16; o <<= 1) { const int x = __shfl_xor(v, o); v = x < v ? x : v; }
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int max_wave(int v) {
    for (int o = 1; o < 16; o <<= 1) { const int x = __shfl_xor(v, o); v = x > v ? x : v; }
    return __builtin_amdgcn_readfirstlane(v);
}

// A partial result: [M][DP] outputs, M references, M sums.
__device__ __forceinline__ float* partial(const TreeArgs& a, int slot, int M, int DP) {
    return a.parts + (size_t)slot * (M * (DP + 2));
}

__device__ __forceinline__ uint16_t* out_at(const TreeArgs& a, const Work& w, int node, int head) {
    return a.out + (int64_t)(w.q.q0 + node) * a.out_stride + (int64_t)head * a.dim;
}

// Of a reference (log2) and a sum of weights.
__device__ __forceinline__ float lse_of(float m, float l) {
    return l == 0.0f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
}

// A row by itself, over the same keys: a lane per key for the scores, a lane per
// channel for the values, of which only those that the row sees are read.  Where
// a tile holds infinities or NaNs that some row must not see, the tiles are
// taken again with zeros in their place, and a row that does see one gets its
// result from here.
template <int TYPE>
__device__ __forceinline__ float widen(const uint8_t* p, int i, bool page) {
    if (TYPE == RAC_CACHE_FP8 && page) return __builtin_amdgcn_cvt_f32_fp8((int)p[i], 0);
    const uint16_t b = reinterpret_cast<const uint16_t*>(p)[i];
    if (TYPE == RAC_CACHE_FP16) return (float)__builtin_bit_cast(_Float16, b);
    return __uint_as_float((uint32_t)b << 16);
}

template <int TYPE>
__device__ __forceinline__ void row_alone(const TreeArgs& a, const Work& w, const Axis& ax, int row, float* part, int in,
                                          int M, int DP) {
    const int lane = (int)threadIdx.x & 63;
    const RowAt at = row_at(a, w, row);
    const uint8_t* q = reinterpret_cast<const uint8_t*>(a.q + (int64_t)(w.q.q0 + at.node) * a.q_stride + (int64_t)at.head * a.dim);
    const int kb = TYPE == RAC_CACHE_FP8 ? 1 : 2;
    const uint64_t plane = ((uint64_t)a.dim << a.log_page) * kb;
    float top = -INFINITY, total = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int side = 0; side < 2; ++side) {  // committed, then drafted
        int j0 = (side ? ax.da : ax.ca) * kTile, j1 = j0 + (side ? ax.count - ax.committed : ax.committed) * kTile;
        const int from = side ? at.see.first : at.see.from, end = side ? at.see.end : w.q.length;
        j0 = j0 < from ? from : j0;
        j1 = j1 < end ? j1 : end;
        for (; j0 < j1; j0 += 64) {
            const int j = j0 + lane;
            bool seen = j < j1;
            const uint8_t *kp = nullptr, *vp = nullptr;
            if (seen && side == 0) {
                const int p = a.table[(size_t)w.seq * a.max_pages + (j >> a.log_page)];
                seen = p >= 0 && p < a.pages;
                if (seen) {
                    kp = a.pool + (((uint64_t)p * a.layers + a.layer) * 2 * a.heads + w.head) * plane +
                         (uint64_t)((j & ((1 << a.log_page) - 1)) * a.dim * kb);
                    vp = kp + a.heads * plane;
                }
            } else if (seen) {
                seen = !a.mask || ((a.mask[(size_t)(w.q.q0 + at.node) * a.mask_words + (j >> 6)] >> (j & 63)) & 1);
                const int64_t o = (int64_t)(w.q.d0 + j) * a.kv_stride + (int64_t)w.head * a.dim;
                kp = reinterpret_cast<const uint8_t*>(a.k + o);
                vp = reinterpret_cast<const uint8_t*>(a.v + o);
            }
            float sc = 0.0f;
            if (seen)
                for (int c = 0; c < a.dim; ++c)
                    sc = __builtin_fmaf(widen<TYPE>(q, c, false), widen<TYPE>(kp, c, side == 0), sc);
            sc = sc * (TYPE == RAC_CACHE_FP8 && side == 0 ? a.scale2 * a.k_scale : a.scale2);
            const uint64_t live = __ballot(seen);
            float m = seen ? sc : -INFINITY;
            for (int o = 1; o < 64; o <<= 1) m = __builtin_fmaxf(m, __shfl_xor(m, o));
            m = __builtin_fmaxf(m, top);
            const float ref = m == -INFINITY ? 0.0f : m, keep = __builtin_amdgcn_exp2f(top - ref);
            float p = seen ? __builtin_amdgcn_exp2f(sc - ref) : 0.0f, sum = p;
            for (int o = 1; o < 64; o <<= 1) sum = sum + __shfl_xor(sum, o);
            total = __builtin_fmaf(total, keep, sum);
            top = m;
            if (TYPE == RAC_CACHE_FP8 && side == 0) p = p * a.v_scale;
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[x] = acc[x] * keep;
            for (uint64_t rest = live; rest; rest &= rest - 1) {
                const int y = __builtin_ctzll(rest);
                const float py = __shfl(p, y);
                const uint8_t* vy = reinterpret_cast<const uint8_t*>(__shfl((unsigned long long)vp, y));
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (lane + 64 * x < a.dim) acc[x] = __builtin_fmaf(py, widen<TYPE>(vy, lane + 64 * x, side == 0), acc[x]);
            }
        }
    }
    bool odd = !(__builtin_fabsf(total) < INFINITY);
#pragma unroll
    for (int x = 0; x < 4; ++x) odd |= !(__builtin_fabsf(acc[x]) < INFINITY);
    if (!__any(odd)) return;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int c = lane + 64 * x;
        if (part) {
            if (c < DP) part[in * DP + c] = acc[x];
        } else if (c < a.dim) {
            out_at(a, w, at.node, at.head)[c] = (uint16_t)pack2<TYPE>(acc[x] / total, 0.0f);
        }
    }
    if (part && lane == 0) {
        part[M * DP + in] = top;
        part[M * DP + M + in] = total;
    }
}

__device__ __forceinline__ Work uniform(const Work& w) {
    const auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return Work{u(w.seq), u(w.head), u(w.row_tile), u(w.chunk), u(w.chunks), u(w.slot),
                Seq{u(w.q.q0), u(w.q.m), u(w.q.d0), u(w.q.n), u(w.q.length)}};
}

// The queries of a wavefront's rows, and what they see: into registers and LDS.
// Returns the extremes.
struct Reach {
    int from_lo, from_hi;    // least and greatest first committed position
    int first, first_hi;     // of the first drafted token
    int end, end_lo;         // greatest and least end of the drafted ones

    // Whether every row sees all of a tile.
    __device__ __forceinline__ bool all_see(const Axis& ax, bool past, int tile) const {
        return past ? tile * kTile >= from_hi : !ax.mask && tile * kTile >= first_hi && (tile + 1) * kTile <= end_lo;
    }
    // Whether no row sees any of it.
    __device__ __forceinline__ bool none_sees(bool past, int tile) const {
        return past ? (tile + 1) * kTile <= from_lo : tile * kTile >= end || (tile + 1) * kTile <= first;
    }
};

template <int TYPE, int DP, int TM>
__device__ __forceinline__ Reach take_rows(const TreeArgs& a, const Work& w, int row0, Rows<TYPE, DP, TM>& rows, Seen* seen) {
    const uint32_t lane = threadIdx.x & 63u;
    Reach x{1 << 30, 0, 1 << 30, 0, 0, 1 << 30};
#pragma unroll
    for (int r = 0; r < TM; ++r) {
        const RowAt at = row_at(a, w, row0 + 16 * r + (int)(lane & 15u));
        if (lane < 16u) seen[16 * r + lane] = Seen{at.see.from, at.see.first, at.see.end, w.q.q0 + at.node};
        x.from_lo = at.see.from < x.from_lo ? at.see.from : x.from_lo;
        x.from_hi = at.see.from > x.from_hi ? at.see.from : x.from_hi;
        x.first = at.see.first < x.first ? at.see.first : x.first;
        x.first_hi = at.see.first > x.first_hi ? at.see.first : x.first_hi;
        x.end = at.see.end > x.end ? at.see.end : x.end;
        x.end_lo = at.see.end < x.end_lo ? at.see.end : x.end_lo;
        const uint16_t* q = a.q + (int64_t)(w.q.q0 + at.node) * a.q_stride + (int64_t)at.head * a.dim;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) {
            const int c = 32 * t + 8 * (int)(lane >> 4);
            rows.q[r][t] = u32x4{0u, 0u, 0u, 0u};
            if (c < a.dim) rows.q[r][t] = *reinterpret_cast<const u32x4*>(q + c);
        }
    }
    return Reach{min_wave(x.from_lo), max_wave(x.from_hi), min_wave(x.first), max_wave(x.first_hi), max_wave(x.end),
                 min_wave(x.end_lo)};
}

// Few rows: all wavefronts hold the same 16 TM rows and take key tiles in
// turn, each through LDS of its own (first the keys, then, in the same place,
// the values), without a barrier until they join.
//
// Bound by the bytes of the committed keys and values, which each (sequence,
// key-value head) reads once: a query row brings 2 flop a byte (4 in 8 bits) and the
// matrix cores would take 250.  So every wavefront keeps the keys and
// values of its next tile on their way while it works on one, and one tile of LDS a
// wavefront, not two, lets more of them run on a compute unit.  32 sequences of up to 16k tokens, 8 heads of 128 channels
// (1.18 GB): 211 us, 5.6 TB/s; one of 131k in 8 bits (268 MB): 48 us, 5.6 TB/s; a
// copy that reads and writes reaches 4.9.  8 trees over up to 64 tokens: 7.7 us, latency.
// 200 sequences of up to 1000 tokens in a window (44 MB): 42 us; 1100 workgroups have
// work where 768 fit at once, in no order of length, and 75 sequences of more than 16
// rows read every key twice.
template <int TYPE, int DP, int TM>
__global__ __launch_bounds__(64 * kWaves, TM == 1 && DP == 64 ? 4 : TM == 1 && TYPE == RAC_CACHE_FP8 ? 3 : 2) void tree_few_kernel(TreeArgs a) {
    constexpr int M = 16 * TM, kTileP = kTile * DP / 8, kPad = DP + 4;
    constexpr int kStage = kTileP * 16 * kWaves, kJoin = kWaves * 16 * kPad * 4;
    __shared__ alignas(16) uint8_t mem[kStage > kJoin ? kStage : kJoin];
    __shared__ float wm[kWaves][M], wl[kWaves][M];
    __shared__ Seen seen[kWaves][M];
    __shared__ Work work;
    const uint32_t lane = threadIdx.x & 63u;
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    Rows<TYPE, DP, TM> rows;
    Axis ax;
    Reach x;
    {
        Work w;
        if (!find_work(a, (int)blockIdx.x, w)) return;
        if (threadIdx.x == 0u) work = w;
        x = take_rows(a, w, w.row_tile * M, rows, seen[wv]);
        ax = axis_of<TYPE>(a, w, x.from_lo, x.first, x.end);
    }
    u32x4* const tile_lds = reinterpret_cast<u32x4*>(mem) + wv * kTileP;
    Load<TYPE, DP, kTile> lk, lv;
    const float c16 = a.scale2, c8 = a.scale2 * a.k_scale, v8 = a.v_scale;
    auto pass = [&](bool clean) {
        rows.start();
        uint32_t there = 0;
        Pages<kTile> pg{};
        auto fetch = [&](int i) { if (i < ax.committed) pg = pages_of<kTile>(ax, ax.ca + i, 0); };
        fetch(wv);
        if (wv < ax.count) {
            there = exist_of(ax, wv, pg, 0);
            if (TYPE != RAC_CACHE_FP8 || wv < ax.committed) {
                lk.tile(ax, wv, pg, 0, false);
                lv.tile(ax, wv, pg, 0, true);
            }
        }
        fetch(wv + kWaves);
        for (int i = wv; i < ax.count; i += kWaves) {
            const bool past = i < ax.committed, narrow = TYPE == RAC_CACHE_FP8 && past;
            const int tile = past ? ax.ca + i : ax.da + i - ax.committed;
            const uint32_t now = there;
            if (past)
                lk.put_committed(tile_lds, ax, now, 0, false);
            else
                lk.put_drafted(tile_lds, ax, ax.k, tile, now, 0, false);
            if (i + kWaves < ax.count) {
                there = exist_of(ax, i + kWaves, pg, 0);
                if (TYPE != RAC_CACHE_FP8 || i + kWaves < ax.committed) lk.tile(ax, i + kWaves, pg, 0, false);
            }
            wave_sync();
            f32x4 s[1][TM][2];
            rows.scores(tile_lds, s[0]);
            wave_sync();
            if (past)
                lv.put_committed(tile_lds, ax, now, 0, clean);
            else
                lv.put_drafted(tile_lds, ax, ax.v, tile, now, 0, clean);
            if (i + kWaves < (TYPE == RAC_CACHE_FP8 ? ax.committed : ax.count)) lv.tile(ax, i + kWaves, pg, 0, true);
            fetch(i + 2 * kWaves);
            bool mixed = false;
            if (!(now == ~0u && x.all_see(ax, past, tile))) {
                uint32_t bits[TM];
#pragma unroll
                for (int r = 0; r < TM; ++r) bits[r] = now & bits_of(ax, seen[wv][16 * r + (lane & 15u)], past, tile);
                mixed = rows.hide(s[0], bits, now);
            }
            u32x4 p[1][TM][2];
            const float c[1] = {narrow ? c8 : c16}, vs[1] = {narrow ? v8 : 1.0f};
            rows.weights(s, c, vs, p);
            wave_sync();
            if (mixed) rows.look(tile_lds);
            rows.values(tile_lds, p[0]);
            wave_sync();
        }
    };
    pass(false);
    const bool clean = __syncthreads_or(rows.alone);
    if (clean) pass(true);
    // join the wavefronts
#pragma unroll
    for (int r = 0; r < TM; ++r) {
        const float l = sum_row(rows.l[r]);
        if (lane < 16u) {
            wm[wv][16 * r + lane] = rows.m[r];
            wl[wv][16 * r + lane] = l;
        }
    }
    __syncthreads();
    const TreeArgs b = args_again();
    const Work w = uniform(work);
    float* const sums = reinterpret_cast<float*>(mem);
    float* const part = w.chunks > 1 ? partial(b, w.slot, M, DP) : nullptr;
#pragma unroll
    for (int r = 0; r < TM; ++r) {
        const int in = 16 * r + (int)(lane & 15u);
        float top = wm[0][in];
#pragma unroll
        for (int x = 1; x < kWaves; ++x) top = __builtin_fmaxf(top, wm[x][in]);
        const float f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(rows.m[r] - top);
        if (r) __syncthreads();
#pragma unroll
        for (int t = 0; t < DP / 16; ++t)
            *reinterpret_cast<f32x4*>(sums + (wv * 16 + (lane & 15u)) * kPad + 16 * t + 4 * (lane >> 4)) =
                f32x4{rows.o[r][t][0] * f, rows.o[r][t][1] * f, rows.o[r][t][2] * f, rows.o[r][t][3] * f};
        __syncthreads();
        for (int e = (int)threadIdx.x; e < 16 * DP / 4; e += 64 * kWaves) {
            const int row = e / (DP / 4), c = 4 * (e % (DP / 4)), ir = 16 * r + row;
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
            float best = wm[0][ir], l = 0.0f;
#pragma unroll
            for (int x = 1; x < kWaves; ++x) best = __builtin_fmaxf(best, wm[x][ir]);
#pragma unroll
            for (int x = 0; x < kWaves; ++x) {
                const f32x4 y = *reinterpret_cast<const f32x4*>(sums + (x * 16 + row) * kPad + c);
                v = f32x4{v[0] + y[0], v[1] + y[1], v[2] + y[2], v[3] + y[3]};
                l = l + wl[x][ir] * (best == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(wm[x][ir] - best));
            }
            const int all = w.row_tile * M + ir;
            if (all >= w.q.m * b.group) continue;
            if (part) {
                *reinterpret_cast<f32x4*>(part + ir * DP + c) = v;
                if (c == 0) {
                    part[M * DP + ir] = best;
                    part[M * DP + M + ir] = l;
                }
                continue;
            }
            const int node = all / b.group, head = w.head * b.group + all % b.group;
            const bool none = l == 0.0f;
            if (c < b.dim)
                *reinterpret_cast<u32x2*>(out_at(b, w, node, head) + c) =
                    none ? u32x2{0u, 0u} : u32x2{pack2<TYPE>(v[0] / l, v[1] / l), pack2<TYPE>(v[2] / l, v[3] / l)};
            if (c == 0 && b.lse) b.lse[(size_t)(w.q.q0 + node) * b.heads * b.group + head] = lse_of(best, l);
        }
    }
    if (clean) {
        __syncthreads();
        for (int in = wv; in < M && w.row_tile * M + in < w.q.m * b.group; in += kWaves)
            row_alone<TYPE>(b, w, ax, w.row_tile * M + in, part, in, M, DP);
    }
}

// Many rows: each wavefront holds 16 TM rows of its own, and all share the
// keys and values of two tiles at a time in LDS, two such pairs in turn: the next
// pair's loads are under way during the products of this one, and one barrier a
// pair is enough.
//
// Bound by no unit alone: of the prompt's cycles the matrix cores are busy for 35%,
// vector instructions are issued in 42% and LDS is read in 33%.  Products, exponentials
// and LDS reads mostly follow each other, with two wavefronts a SIMD and a barrier a
// pair.  Without its exponentials the prompt's case would take 339 us instead of 363; four
// tiles of rows a wavefront would halve the LDS reads, but do not fit in the registers
// (755 us).  Chunks of prompts of up to 2048 tokens, 28 query heads of 128 channels
// (310 GF): 363 us, 855 TF/s, where a product of two 8192 x 8192 matrices reaches
// 1210.  16 trees of up to 64 nodes over up to 8k tokens, four query heads a key-value
// head (34 GF, 211 MB): 79 us and a join of 13; matrix cores 22%, vector 37%, LDS 25%,
// its tiles of 128 rows are 77% full, and 12 sequences read their keys for two of them.
//
// KP: 16-bit numbers of a weight.
template <int TYPE, int DP, int TM, int W, int KP>
__device__ __forceinline__ void many_rows(const TreeArgs& a) {
    // Fragments read ahead need registers: four wavefronts of 32 rows have none left.
    constexpr bool kAhead = W == 8 || TM == 1;
    constexpr int M = 16 * TM * W, kBring = 2 * kTile / W, kParts = kTile / kBring, kTileP = kTile * DP / 8;
    __shared__ u32x4 mem[2][2][2][kTileP];  // pair, tile, keys or values
    __shared__ uint32_t exist[2][2][kParts];  // the keys of a tile that exist, by parts
    __shared__ Seen seen[W][16 * TM];
    __shared__ Reach reach[W];
    __shared__ Work work;
    const uint32_t lane = threadIdx.x & 63u;
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    Rows<TYPE, DP, TM> rows;
    Axis ax;
    Reach x;
    bool busy;  // whether this wavefront has rows
    {
        Work w;
        if (!find_work(a, (int)blockIdx.x, w)) return;
        if (threadIdx.x == 0u) work = w;
        const int row0 = w.row_tile * M + 16 * TM * wv;
        busy = row0 < w.q.m * a.group;
        x = take_rows(a, w, row0, rows, seen[wv]);
        if (lane == 0u) reach[wv] = x;
        __syncthreads();
        Reach all = reach[0];
#pragma unroll
        for (int y = 1; y < W; ++y) {
            const Reach z = reach[y];
            all.from_lo = z.from_lo < all.from_lo ? z.from_lo : all.from_lo;
            all.first = z.first < all.first ? z.first : all.first;
            all.end = z.end > all.end ? z.end : all.end;
        }
        const auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
        ax = axis_of<TYPE>(a, w, u(all.from_lo), u(all.first), u(all.end));
    }
    // the tiles that this wavefront's rows see all of, if all their keys exist, as runs of indices
    const int plain0 = (x.from_hi + kTile - 1) / kTile - ax.ca, draft0 = ax.committed - ax.da;
    const int plain2 = ax.mask ? 1 << 30 : draft0 + (x.first_hi + kTile - 1) / kTile, plain3 = draft0 + x.end_lo / kTile;
    const auto plain = [&](int i) { return i < ax.committed ? i >= plain0 : i >= plain2 && i < plain3; };
    // (this wavefront brings kBring rows of every pair)
    const int half = kBring * (wv % kParts), which = wv / kParts;
    Load<TYPE, DP, kBring> lk, lv;
    const float c16 = a.scale2, c8 = a.scale2 * a.k_scale, v8 = a.v_scale;
    bool clean = false;
again:
    rows.start();
    Pages<kBring> pg{};
    uint32_t there = 0;
    auto load = [&](int i) {
        there = exist_of(ax, i, pg, half);
        if (i >= (TYPE == RAC_CACHE_FP8 ? ax.committed : ax.count)) return;
        lk.tile(ax, i, pg, half, false);
        lv.tile(ax, i, pg, half, true);
    };
    auto fetch = [&](int i) { if (i < ax.committed) pg = pages_of<kBring>(ax, ax.ca + i, half); };
    auto pair = [&](int i, u32x4 (&buf)[2][2][kTileP], uint32_t (&ex)[2][kParts]) {
        const int mine = i + which;
        if (TYPE != RAC_CACHE_FP8 || mine < ax.committed) {
            lk.put_committed(buf[which][0], ax, there, half, false);
            lv.put_committed(buf[which][1], ax, there, half, clean);
        } else if (mine < ax.count) {
            const int tile = ax.da + mine - ax.committed;
            lk.put_drafted(buf[which][0], ax, ax.k, tile, there, half, false);
            lv.put_drafted(buf[which][1], ax, ax.v, tile, there, half, clean);
        } else {
            lk.put_zeros(buf[which][0], half);
            lv.put_zeros(buf[which][1], half);
        }
        if (lane == 0u) ex[which][wv % kParts] = there & (low_bits(kBring) << half);
        load(mine + 2);
        fetch(mine + 4);
        __syncthreads();
        if (!busy) return;
        // two tiles at a time: their products and weights overlap
        f32x4 s[2][TM][2];
        uint32_t now0 = ex[0][0], now1 = ex[1][0];
#pragma unroll
        for (int y = 1; y < kParts; ++y) {
            now0 |= ex[0][y];
            now1 |= ex[1][y];
        }
        now0 = __builtin_amdgcn_readfirstlane(now0);
        now1 = __builtin_amdgcn_readfirstlane(now1);
        if ((now0 & now1) == ~0u && plain(i) && plain(i + 1)) {
            rows.template scores_of<kAhead>(buf[0][0], buf[1][0], s);
        } else {
            const auto tile_of = [&](int j) { return j < ax.committed ? ax.ca + j : ax.da + j - ax.committed; };
            // what no row of this wavefront sees is passed over
            if (x.none_sees(i < ax.committed, tile_of(i)) &&
                (i + 1 >= ax.count || x.none_sees(i + 1 < ax.committed, tile_of(i + 1))))
                return;
            rows.template scores_of<kAhead>(buf[0][0], buf[1][0], s);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint32_t now = y ? now1 : now0;
                uint32_t bits[TM];
#pragma unroll
                for (int r = 0; r < TM; ++r)
                    bits[r] = now ? now & bits_of(ax, seen[wv][16 * r + (lane & 15u)], i + y < ax.committed, tile_of(i + y)) : 0u;
                if (rows.hide(s[y], bits, now)) rows.look(buf[y][1]);
            }
        }
        const bool n0 = TYPE == RAC_CACHE_FP8 && i < ax.committed, n1 = TYPE == RAC_CACHE_FP8 && i + 1 < ax.committed;
        const float c[2] = {n0 ? c8 : c16, n1 ? c8 : c16}, vs[2] = {n0 ? v8 : 1.0f, n1 ? v8 : 1.0f};
        u32x4 p[2][TM][KP];
        if constexpr (kAhead) {
            const auto first = rows.read_values(buf[0][1], 0);
            __builtin_amdgcn_sched_barrier(0);
            rows.weights(s, c, vs, p);
            rows.values_of(first, buf[0][1], buf[1][1], p);
        } else {
            rows.weights(s, c, vs, p);
            rows.values(buf[0][1], p[0]);
            rows.values(buf[1][1], p[1]);
        }
    };
    fetch(which);
    load(which);
    fetch(which + 2);
    for (int i = 0; i < ax.count; i += 4) {
        pair(i, mem[0], exist[0]);
        if (i + 2 < ax.count) pair(i + 2, mem[1], exist[1]);
    }
    if (!clean && __syncthreads_or(rows.alone)) {
        clean = true;
        goto again;
    }
    const TreeArgs b = args_again();
    const Work w = uniform(work);
    float* const part = w.chunks > 1 ? partial(b, w.slot, M, DP) : nullptr;
#pragma unroll
    for (int r = 0; r < TM; ++r) {
        const float l = sum_row(rows.l[r]);
        const int in = 16 * (TM * wv + r) + (int)(lane & 15u), all = w.row_tile * M + in;
        if (all >= w.q.m * b.group) continue;
        const int node = all / b.group, head = w.head * b.group + all % b.group;
        const bool none = l == 0.0f;
        uint16_t* const out = out_at(b, w, node, head);
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
            const int c = 16 * t + 4 * (int)(lane >> 4);
            const f32x4 v = rows.o[r][t];
            if (part)
                *reinterpret_cast<f32x4*>(part + in * DP + c) = v;
            else if (c < b.dim)
                *reinterpret_cast<u32x2*>(out + c) =
                    none ? u32x2{0u, 0u} : u32x2{pack2<TYPE>(v[0] / l, v[1] / l), pack2<TYPE>(v[2] / l, v[3] / l)};
        }
        if (lane < 16u) {
            if (part) {
                part[M * DP + in] = rows.m[r];
                part[M * DP + M + in] = l;
            } else if (b.lse) {
                b.lse[(size_t)(w.q.q0 + node) * b.heads * b.group + head] = lse_of(rows.m[r], l);
            }
        }
    }
    if (clean) {
        __syncthreads();
        const int r0 = 16 * TM * wv;
        for (int in = r0; in < r0 + 16 * TM && w.row_tile * M + in < w.q.m * b.group; ++in)
            row_alone<TYPE>(b, w, ax, w.row_tile * M + in, part, in, M, DP);
    }
}

// (with 256 channels for up to 16 rows: tree_few_kernel has no registers for their
// outputs and its tiles)
template <int TYPE, int DP, int TM, int W>
__global__ __launch_bounds__(64 * W, TM * DP <= 256 && DP < 256 ? 2 : 1) void tree_many_kernel(TreeArgs a) {
    many_rows<TYPE, DP, TM, W, DP == 256 ? 2 : 1>(a);
}

// More than 16 rows of 144 to 256 channels: a weight rounded once (chunks of prompts of
// 2048 tokens, 8 query heads of 256 channels, 115 GF: 301 us, 380 TF/s).
template <int TYPE>
__global__ __launch_bounds__(64 * kWaves, 1) void tree_wide_kernel(TreeArgs a) {
    many_rows<TYPE, 256, 1, kWaves, 1>(a);
}

// Joins the parts of the sequences that were split:
//   max = max_c m_c,  l = sum_c l_c 2^(m_c - max),  out = sum_c o_c 2^(m_c - max) / l.
// DP / 4 lanes take a (row, query head) pair, four channels each.  A workgroup takes
// a row; with SPLIT (few pairs, so many parts) a few pairs, and its wavefronts share
// their parts.  Bound by latency where parts are many and pairs few (one sequence of
// 131k tokens, 64 pairs: 7.1 us; 32 of 16k: 5.9) and by the parts' bytes where pairs
// are many (694 rows of 32 heads, 13 us).
template <int TYPE, int DP, bool SPLIT>
__global__ __launch_bounds__(64 * kWaves) void tree_join_kernel(TreeArgs a) {
    constexpr int kLanes = DP / 4, kPairs = 64 / kLanes, kAtOnce = 8;
    __shared__ f32x4 sums[SPLIT ? kWaves : 1][64];
    __shared__ float wm[SPLIT ? kWaves : 1][kPairs], wl[SPLIT ? kWaves : 1][kPairs];
    const int lane = (int)threadIdx.x & 63, wv = (int)threadIdx.x / 64, hq = a.heads * a.group;
    const int groups = (hq + kPairs - 1) / kPairs;  // of the heads of a row
    const int row = SPLIT ? (int)blockIdx.x / groups : (int)blockIdx.x;
    if (row >= a.rows) return;
    Seq q;
    int chunks, slot;
    if (a.plan) {
        const int s = __builtin_amdgcn_readfirstlane(last_at_most(a.seqs, row, [&](int i) { return i ? a.q_start[i] : -1; }));
        const SeqPlan p = a.plan[s];
        chunks = p.chunks;
        if (chunks == 1) return;
        q = Seq{p.q0, p.m, p.d0, p.n, p.length};
        slot = p.slot;
    } else {
        const LaneSeq l = lane_seq(a);
        const uint64_t has = __ballot(row >= l.q.q0 && row < l.q.q0 + l.q.m);
        if (!has) return;
        const int at = __builtin_ctzll(has);
        const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        chunks = of(l.c.chunks);
        if (chunks == 1) return;
        q = Seq{of(l.q.q0), of(l.q.m), of(l.q.d0), of(l.q.n), of(l.q.length)};
        slot = of(l.slot);
    }
    const int tiles = cut_of(a, q, 1 << 30).tiles;
    if (row < q.q0 || row >= q.q0 + q.m || (uint32_t)(slot + tiles * chunks * a.heads) > (uint32_t)a.slots) return;
    const int pair = lane / kLanes, c4 = lane % kLanes;
    // parts of a row tile are a.heads slots apart
    const size_t stride = (size_t)a.m * (DP + 2), step = stride * a.heads;
    for (int g = SPLIT ? (int)blockIdx.x % groups : wv; g < groups; g += SPLIT ? groups : kWaves) {
        const int h = g * kPairs + pair;
        const int hc = h < hq ? h : hq - 1, r = (row - q.q0) * a.group + hc % a.group;
        const int in = r % a.m;
        const float* const base = a.parts + ((size_t)slot + (size_t)((tiles - 1 - r / a.m) * chunks) * a.heads + hc / a.group) * stride;
        float top = -INFINITY, l = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        const int first = SPLIT ? wv : 0, by = SPLIT ? kWaves : 1;
        for (int c = first; c < chunks; c += by * kAtOnce) {
            f32x4 x[kAtOnce];
            float m[kAtOnce], s[kAtOnce], now = top;
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const bool is = c + i * by < chunks;
                const float* p = base + (size_t)(is ? c + i * by : c) * step;
                x[i] = *reinterpret_cast<const f32x4*>(p + (size_t)in * DP + 4 * c4);
                m[i] = is ? p[a.m * DP + in] : -INFINITY;
                s[i] = p[a.m * DP + a.m + in];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) now = __builtin_fmaxf(now, m[i]);
            const float ref = now == -INFINITY ? 0.0f : now, keep = __builtin_amdgcn_exp2f(top - ref);
            l = l * keep;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] * keep;
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (c + i * by >= chunks) break;
                const float f = __builtin_amdgcn_exp2f(m[i] - ref);
                l = __builtin_fmaf(s[i], f, l);
#pragma unroll
                for (int y = 0; y < 4; ++y) v[y] = __builtin_fmaf(x[i][y], f, v[y]);
            }
            top = now;
        }
        if constexpr (SPLIT) {
            sums[wv][lane] = v;
            if (c4 == 0) {
                wm[wv][pair] = top;
                wl[wv][pair] = l;
            }
            __syncthreads();
            if (wv != 0) return;
            top = wm[0][pair];
#pragma unroll
            for (int x = 1; x < kWaves; ++x) top = __builtin_fmaxf(top, wm[x][pair]);
            v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            l = 0.0f;
#pragma unroll
            for (int x = 0; x < kWaves; ++x) {
                const float f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(wm[x][pair] - top);
                l = __builtin_fmaf(wl[x][pair], f, l);
#pragma unroll
                for (int y = 0; y < 4; ++y) v[y] = __builtin_fmaf(sums[x][lane][y], f, v[y]);
            }
        }
        if (h >= hq) continue;
        const bool none = l == 0.0f;
        if (4 * c4 < a.dim)
            *reinterpret_cast<u32x2*>(a.out + (int64_t)row * a.out_stride + (int64_t)h * a.dim + 4 * c4) =
                none ? u32x2{0u, 0u} : u32x2{pack2<TYPE>(v[0] / l, v[1] / l), pack2<TYPE>(v[2] / l, v[3] / l)};
        if (c4 == 0 && a.lse) a.lse[(size_t)row * hq + h] = lse_of(top, l);
    }
}

// ---------------------------------------------------------------------------
// Host side

bool tree_valid(const rac_cache_config* c, const rac_tree_config* t) {
    return cache_valid(c) && t && t->q_heads >= 1 && t->q_heads % c->kv_heads == 0 && t->q_heads / c->kv_heads <= 64 &&
           t->rows >= 0 && t->rows <= (1 << 20) && t->max_rows >= 0 && t->max_draft >= 0 && t->window >= 0 &&
           t->scale >= 0.0f && t->scale < __builtin_inff();
}

// (row, query head) pairs that the kernels' 32-bit counts of workgroups and slots hold.
bool tree_counted(const rac_tree_config* t) { return (int64_t)t->rows * t->q_heads < (int64_t(1) << 26); }

// Which kernel a call takes, how its work is split, and what that needs.
struct Choice {
    const void* kernel;
    int threads;        // a workgroup
    int m, dp;          // query rows a workgroup, channels (padded)
    int target, slots;  // parts wanted, room for partial results
    int64_t grid;
    uint64_t bytes, plan;  // of the scratch; where the plan lies in it
};

// Key tiles that a part has at least, two a wavefront: shorter ones cost more in
// the join than they save, longer ones leave compute units without work (one
// sequence of 8k tokens 16.2 us; 18.6 with 4, 18.2 with 16).
constexpr int kMinChunk = 8;

// rows: the most of a sequence and a key-value head; mean: of all sequences.
template <int TYPE, int DP>
void choose_form(int rows, int mean, Choice& c) {
    c.dp = DP;
    c.threads = 64 * kWaves;
    // (workgroups of the form that the 256 compute units hold at once)
    c.target = DP == 256 ? 256 : 512;
    // (TM = 2 with 16-bit pages of 128 channels would need more than 256 registers)
    constexpr bool kTwo = DP == 64 || (DP == 128 && TYPE == RAC_CACHE_FP8);
    // (most sequences with 16 rows or fewer: two tiles of 16 for the others are
    // faster, 64 sequences of 12 to 20 rows, 64 channels, 58 us, 64 with one of 32; where
    // all have 32 it is the other way round, 135 and 126, in 8 bits 174 and 145)
    if ((rows <= 16 || (rows <= 32 && mean <= 17)) && DP < 256) {
        c.m = 16;
        c.target = DP == 64 ? 1024 : TYPE == RAC_CACHE_FP8 ? 768 : 512;
        c.kernel = reinterpret_cast<const void*>(tree_few_kernel<TYPE, DP < 256 ? DP : 128, 1>);
    } else if (rows <= 32 && kTwo) {
        c.m = 32;
        c.kernel = reinterpret_cast<const void*>(tree_few_kernel<TYPE, kTwo ? DP : 64, 2>);
    } else if (rows <= 64 || DP == 256) {
        // (64 rows on up to 8k tokens 142 us, 151 with 128 rows a workgroup; 24 rows 240 and 252;
        // 256 channels leave registers for 16 rows a wavefront)
        c.m = 64;
        c.kernel = DP == 256 && rows > 16 ? reinterpret_cast<const void*>(tree_wide_kernel<TYPE>)
                                          : reinterpret_cast<const void*>(tree_many_kernel<TYPE, DP, 1, 4>);
    } else if (rows < 512 || DP == 64) {
        // (trees of 64 nodes, 256 rows: 93 us, 108 with 256 rows a workgroup, which leaves too few;
        // prompts, 4900 to 14000 rows: 386 and 369)
        c.m = 128;
        c.kernel = reinterpret_cast<const void*>(tree_many_kernel<TYPE, DP < 256 ? DP : 128, 2, 4>);
    } else {
        c.m = 256;
        c.threads = 512;
        c.kernel = reinterpret_cast<const void*>(tree_many_kernel<TYPE, 128, 2, 8>);
    }
}

// Workgroups from which the join takes a row each instead of sharing the parts of
// a few pairs (us, rows and shared: one of 32 heads, 8k tokens, 29.8, 16.2; 694 of 32
// heads 92, 129).
constexpr int kSplitJoin = 1024;

template <int TYPE>
const void* join_of(int dp, bool split) {
    if (dp == 64)
        return split ? reinterpret_cast<const void*>(tree_join_kernel<TYPE, 64, true>)
                     : reinterpret_cast<const void*>(tree_join_kernel<TYPE, 64, false>);
    if (dp == 128)
        return split ? reinterpret_cast<const void*>(tree_join_kernel<TYPE, 128, true>)
                     : reinterpret_cast<const void*>(tree_join_kernel<TYPE, 128, false>);
    return split ? reinterpret_cast<const void*>(tree_join_kernel<TYPE, 256, true>)
                 : reinterpret_cast<const void*>(tree_join_kernel<TYPE, 256, false>);
}

template <int TYPE>
void choose_type(int dim, int rows, int mean, Choice& c) {
    if (dim <= 64)
        choose_form<TYPE, 64>(rows, mean, c);
    else if (dim <= 128)
        choose_form<TYPE, 128>(rows, mean, c);
    else
        choose_form<TYPE, 256>(rows, mean, c);
}

Choice choose(const rac_cache_config* cfg, const rac_tree_config* tree) {
    Choice c{};
    const int group = tree->q_heads / cfg->kv_heads;
    const int64_t of_seq = tree->max_rows < tree->rows ? tree->max_rows : tree->rows;
    const int rows = (int)(of_seq * group);
    const int64_t seqs = cfg->seqs < tree->rows ? cfg->seqs : tree->rows > 0 ? tree->rows : 1;
    const int mean = (int)((int64_t)tree->rows * group / seqs);
    if (cfg->type == RAC_CACHE_BF16)
        choose_type<RAC_CACHE_BF16>(cfg->head_dim, rows, mean, c);
    else if (cfg->type == RAC_CACHE_FP16)
        choose_type<RAC_CACHE_FP16>(cfg->head_dim, rows, mean, c);
    else
        choose_type<RAC_CACHE_FP8>(cfg->head_dim, rows, mean, c);
    // the longest key axis there can be
    int64_t keys = (int64_t)cfg->max_pages * cfg->page_tokens;
    if (tree->window > 0 && tree->window < keys) keys = tree->window + kTile;
    const int64_t most = (keys + kTile - 1) / kTile + ((int64_t)tree->max_draft + kTile - 1) / kTile;
    const int64_t row_tiles = ((int64_t)tree->rows * group + c.m - 1) / c.m;
    // (no parts, and no join, where there is nothing to cut, where the sequences
    // fill the device by themselves, or nearly do and none is long)
    const int64_t units = row_tiles * cfg->kv_heads;
    if (most <= kMinChunk || units >= c.target || (2 * units >= c.target && most <= 8 * kMinChunk)) c.target = 0;
    // (a sequence that is split has fewer than twice its keys over the part's size parts)
    c.slots = 2 * c.target * (c.m <= 32 ? 2 : 1);
    c.plan = ((uint64_t)c.slots * (uint64_t)c.m * (uint64_t)(c.dp + 2) * 4u + 255u) & ~uint64_t(255);
    c.bytes = c.plan + (uint64_t)(cfg->seqs + 1) * sizeof(SeqPlan);
    // (see chunk_tiles: at most the workgroups it wants, and one more a sequence, head and tile of rows)
    const int64_t most_units = (row_tiles + seqs) * cfg->kv_heads, t = c.target;
    c.grid = t + most_units;
    if (c.m <= 32) {
        const int64_t twice = 2 * t + (most_units < t ? most_units : t);
        c.grid = twice > c.grid ? twice : c.grid;
    }
    return c;
}

}  // namespace

extern "C" {

size_t rac_tree_attention_workspace(const rac_cache_config* cfg, const rac_tree_config* tree) {
    return tree_valid(cfg, tree) && tree_counted(tree) ? (size_t)choose(cfg, tree).bytes : 0;
}

rac_status rac_tree_attention(const rac_cache_config* cfg, const rac_tree_config* tree, int32_t layer,
                              const void* pool, const int32_t* table, const int32_t* lengths,
                              const rac_tree_tensors* t, void* workspace, size_t workspace_bytes,
                              rac_stream_t stream) {
    if (!tree_valid(cfg, tree) || layer < 0 || layer >= cfg->layers || !t) return RAC_ERR_INVALID;
    if (tree->rows == 0) return RAC_OK;
    const int64_t kv_row = (int64_t)cfg->kv_heads * cfg->head_dim, q_row = (int64_t)tree->q_heads * cfg->head_dim;
    if (!pool || !table || !lengths || !t->q || !t->q_start || !t->out || !workspace) return RAC_ERR_INVALID;
    if (t->q_stride < q_row || t->out_stride < q_row || t->q_stride % 8 || t->out_stride % 8) return RAC_ERR_INVALID;
    if ((t->k != nullptr) != (t->v != nullptr) || t->draft_rows < 0 || t->mask_words < 0) return RAC_ERR_INVALID;
    if (t->k && (t->kv_stride < kv_row || t->kv_stride % 8 || t->kv_stride > (1 << 25))) return RAC_ERR_INVALID;
    if ((t->mask != nullptr) != (t->mask_words > 0)) return RAC_ERR_INVALID;
    if (!aligned(pool, 16) || !aligned(t->q, 16) || !aligned(t->k, 16) || !aligned(t->v, 16) || !aligned(t->out, 16) ||
        !aligned(table, 4) || !aligned(lengths, 4) || !aligned(t->q_start, 4) || !aligned(t->draft_start, 4) ||
        !aligned(t->lse, 4) || !aligned(t->mask, 8) || !aligned(workspace, 256))
        return RAC_ERR_ALIGN;
    if (!tree_counted(tree)) return RAC_ERR_UNSUPPORTED;
    if (workspace_bytes < rac_tree_attention_workspace(cfg, tree)) return RAC_ERR_CAPACITY;
    const bool drafted = t->k && t->draft_rows > 0;
    TreeArgs a{};
    a.pool = static_cast<const uint8_t*>(pool);
    a.table = table;
    a.lengths = lengths;
    a.q = static_cast<const uint16_t*>(t->q);
    a.k = drafted ? static_cast<const uint16_t*>(t->k) : nullptr;
    a.v = drafted ? static_cast<const uint16_t*>(t->v) : nullptr;
    a.q_start = t->q_start;
    a.draft_start = t->draft_start ? t->draft_start : t->q_start;
    a.mask = t->mask;
    a.out = static_cast<uint16_t*>(t->out);
    a.lse = t->lse;
    a.q_stride = t->q_stride;
    a.kv_stride = t->kv_stride;
    a.out_stride = t->out_stride;
    a.layers = cfg->layers;
    a.layer = layer;
    a.heads = cfg->kv_heads;
    a.group = tree->q_heads / cfg->kv_heads;
    a.dim = cfg->head_dim;
    a.log_page = log2_of(cfg->page_tokens);
    a.pages = cfg->pages;
    a.seqs = cfg->seqs;
    a.max_pages = cfg->max_pages;
    a.rows = tree->rows;
    a.max_rows = tree->max_rows;
    a.draft_rows = t->draft_rows;
    a.max_draft = tree->max_draft;
    a.window = tree->window;
    a.mask_words = t->mask_words;
    a.scale2 = (tree->scale > 0.0f ? tree->scale : 1.0f / sqrtf((float)cfg->head_dim)) * 1.4426950408889634f;
    a.k_scale = cfg->k_scale;
    a.v_scale = cfg->v_scale;
    const Choice c = choose(cfg, tree);
    a.target = c.target;
    a.min_chunk = kMinChunk;
    a.parts = static_cast<float*>(workspace);
    a.slots = c.slots;
    a.plan = cfg->seqs > 64 ? reinterpret_cast<SeqPlan*>(static_cast<uint8_t*>(workspace) + c.plan) : nullptr;
    a.m = c.m;
    void* p[] = {&a};
    const auto launch = [&](const void* kernel, int64_t grid, int threads) {
        return hipLaunchKernel(kernel, dim3((unsigned)grid), dim3((unsigned)threads), p, 0, stream) == hipSuccess
                   ? RAC_OK
                   : RAC_ERR_HIP;
    };
    rac_status st = RAC_OK;
    if (a.plan) st = launch(reinterpret_cast<const void*>(tree_plan_kernel), 1, kPlanThreads);
    if (st == RAC_OK) st = launch(c.kernel, c.grid, c.threads);
    if (st != RAC_OK || c.target == 0) return st;
    const int pairs = 256 / c.dp;  // (row, head) pairs a wavefront
    const int64_t units = (int64_t)tree->rows * ((tree->q_heads + pairs - 1) / pairs);
    const bool split = units < kSplitJoin;
    const void* join = cfg->type == RAC_CACHE_FP16 ? join_of<RAC_CACHE_FP16>(c.dp, split) : join_of<RAC_CACHE_BF16>(c.dp, split);
    return launch(join, split ? units : tree->rows, 64 * kWaves);
}

}  // extern "C"
