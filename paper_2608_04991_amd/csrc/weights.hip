// weights.hip - gfx950 kernels and C ABI of the attention weight that cached
// tokens receive.  The contract is in include/rac_cache.h.
#include <math.h>

#include "tree_common.h"

namespace {

struct WeightsArgs {
    const uint8_t* pool;
    const int32_t* table;
    const int32_t* lengths;
    const uint16_t* q;
    const uint16_t* k;
    const int32_t* q_start;
    const int32_t* draft_start;
    const uint64_t* mask;
    const float* lse;
    float* weight;
    float* draft_weight;
    float* parts;  // [slots][64]
    int64_t q_stride, kv_stride, positions;
    int32_t layers, layer, heads, group, dim, log_page, pages, seqs, max_pages;
    int32_t rows, max_rows, draft_rows, max_draft, window, mask_words;
    int32_t sets, first_set, unit_heads;  // heads with units of their own (1: a unit has all)
    int32_t item_heads;                   // heads of a unit
    uint32_t by_group;  // 2^32 / group, rounded up
    float scale2;       // of the scores, times log2(e)
    float k_scale;
};

// ---------------------------------------------------------------------------
// The work.  A unit is a tile of keys of a sequence, for one key-value head or all of
// them; its items are blocks of query rows (rows of a key-value head are the (node, query
// head) pairs of a sequence, node by node) of its heads, one head after the other.
constexpr int kThreads = 256, kWavesEach = kThreads / 64;

struct Units {
    int tile0, committed, drafted;  // first tile that the window reaches, tiles
    int rows;                       // blocks of rows of a head
};

template <int KEYS, int ROWS>
__device__ __forceinline__ Units units_of(const WeightsArgs& a, const Seq& q) {
    Units u;
    u.tile0 = a.window > 0 && q.length > a.window ? (q.length - a.window) / KEYS : 0;
    u.committed = (q.length + KEYS - 1) / KEYS - u.tile0;
    u.drafted = a.draft_weight ? (q.n + KEYS - 1) / KEYS : 0;
    u.rows = (q.m * a.group + ROWS - 1) / ROWS;
    if (u.rows == 0) u.committed = u.drafted = 0;
    return u;
}

__device__ __forceinline__ int64_t sum_before(int64_t v, int64_t* sums, int64_t* total) {
    const int lane = (int)threadIdx.x & 63, w = (int)threadIdx.x / 64;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up((long long)x, o);
        x += lane >= o ? y : 0;
    }
    __syncthreads();
    if (lane == 63) sums[w] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kWavesEach; ++i) {
        before += i < w ? sums[i] : 0;
        all += sums[i];
    }
    *total = all;
    return before + x - v;
}

constexpr int kNoMore = 0x7FFFFFFF;
__device__ __forceinline__ int held_int(int64_t v) { return v < kNoMore ? (int)v : kNoMore; }

// Where the units of every sequence begin, in LDS, as every workgroup finds it by itself;
// base[seqs] is the end.
template <int KEYS, int ROWS>
__device__ __forceinline__ void lay_out(const WeightsArgs& a, int32_t* base) {
    __shared__ int64_t sums[kWavesEach];
    const int each = (a.seqs + kThreads - 1) / kThreads, s0 = (int)threadIdx.x * each;
    const int s1 = s0 + each < a.seqs ? s0 + each : a.seqs;
    const auto units = [&](int s) {
        const Units u = units_of<KEYS, ROWS>(a, seq_of(a, s));
        return (int64_t)(u.committed + u.drafted) * a.unit_heads;
    };
    int64_t mine = 0, all;
    for (int s = s0; s < s1; ++s) mine += units(s);
    int64_t at = sum_before(mine, sums, &all);
    for (int s = s0; s < s1; ++s) {
        base[s] = held_int(at);
        at += each > 1 ? units(s) : 0;  // (with one sequence a thread it is not needed)
    }
    if (threadIdx.x == 0) base[a.seqs] = held_int(all);
    __syncthreads();
}

// The last sequence whose work begins at or before x.
__device__ __forceinline__ int seq_at(const int32_t* base, int n, int x) {
    const int lane = (int)threadIdx.x & 63;
    int lo = 0;
    while (n > 64) {
        const int step = (n + 63) / 64;
        const int k = __popcll(__ballot(lane * step < n && base[lo + lane * step] <= x)) - 1;
        lo += k * step;
        n = n - k * step < step ? n - k * step : step;
    }
    return lo + __popcll(__ballot(lane < n && base[lo + lane] <= x)) - 1;
}

__device__ __forceinline__ uint64_t low64(int n) { return n >= 64 ? ~uint64_t(0) : n <= 0 ? 0 : (uint64_t(1) << n) - 1; }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A unit's keys and where their sums go.
struct Unit {
    int seq, key0, head;  // first key (of the committed or the drafted); -1: all heads
    bool past;
};

template <int KEYS>
__device__ __forceinline__ Unit unit_at(const WeightsArgs& a, int s, const Units& u, int i) {
    Unit r;
    r.seq = s;
    const int t = a.unit_heads > 1 ? uniform(i / a.unit_heads) : i;
    r.head = a.unit_heads > 1 ? i - t * a.unit_heads : a.heads > 1 ? -1 : 0;
    r.past = t < u.committed;
    r.key0 = (r.past ? u.tile0 + t : t - u.committed) * KEYS;
    return r;
}

// Of the 16 NT keys from u.key0 on, those that exist, and the pages of the committed ones.
// (Lanes of a column of 16 ask for the same.)
template <int NT>
__device__ __forceinline__ uint64_t exist_in(const WeightsArgs& a, const Unit& u, const Seq& q, int (&page)[NT]) {
    if (!u.past) return low64(q.n - u.key0) & low64(16 * NT);
    const int lane = (int)threadIdx.x & 63;
    uint64_t r = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int j = u.key0 + 16 * t + (lane & 15);
        page[t] = -1;
        if (j < q.length) page[t] = a.table[(size_t)u.seq * a.max_pages + (j >> a.log_page)];
        if ((uint32_t)page[t] >= (uint32_t)a.pages) page[t] = -1;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) r |= (uint64_t)(__ballot(page[t] >= 0) & 0xFFFFu) << (16 * t);
    return r;
}

// Where the sum of key u.key0 + key is.
__device__ __forceinline__ float* sum_of(const WeightsArgs& a, const Unit& u, const Seq& q, int key) {
    const int64_t set = a.first_set + (u.head > 0 && a.sets > 1 ? u.head : 0), j = (int64_t)u.key0 + key;
    return u.past ? a.weight + ((int64_t)u.seq * a.sets + set) * a.positions + j : a.draft_weight + set * a.draft_rows + q.d0 + j;
}

// Adds to it, if there is such a key.
__device__ __forceinline__ void add_to(const WeightsArgs& a, const Unit& u, const Seq& q, uint64_t exist, int key, float v) {
    if (!((exist >> key) & 1)) return;
    float* const to = sum_of(a, u, q, key);
    *to = *to + v;
}

// Which of the keys from k0 on a row sees (those that exist aside).
__device__ __forceinline__ uint64_t sees(const WeightsArgs& a, const Seq& q, const Unit& u, int node, const Sight& see) {
    if (u.past) return ~low64(see.from - u.key0);
    uint64_t bits = low64(see.end - u.key0) & ~low64(see.first - u.key0);
    if (a.mask && bits)  // (a mask reaches see.end)
        bits &= a.mask[(int64_t)(q.q0 + node) * a.mask_words + u.key0 / 64] >> (u.key0 % 64);
    return bits;
}

// First channel of lane group g in step u: the order of channels is free, and with 8 bits
// the 16 bytes of a load serve two steps.
template <int TYPE>
__device__ __forceinline__ int channel(int u, int g) {
    return TYPE == RAC_CACHE_FP8 ? 64 * (u / 2) + 16 * g + 8 * (u % 2) : 32 * u + 8 * g;
}

// A wavefront keeps 16 NT keys in registers, as the first operand of the matrix cores, and
// takes the rows 16 at a time as the second: lane l then holds the scores of row l % 16
// with keys 16 t + 4 (l / 16) + i, so a row's lse is one number a lane, and the sums over
// rows are additions in place; the 16 lanes of a key are added at the end.
template <int TYPE, int DP, int NT>
struct Keys {
    static constexpr int kSteps = DP / 32;
    u32x4 k[NT][kSteps];

    __device__ __forceinline__ void take(const WeightsArgs& a, const Unit& u, const Seq& q, int head, const int (&page)[NT]) {
        if (u.past)
            committed(a, u, head, page);
        else
            drafted(a, u, q, head);
    }
    __device__ __forceinline__ void committed(const WeightsArgs& a, const Unit& u, int head, const int (&page)[NT]) {
        constexpr int kB = TYPE == RAC_CACHE_FP8 ? 1 : 2;
        const int lane = (int)threadIdx.x & 63, g = lane >> 4;
        const uint64_t plane = ((uint64_t)a.dim << a.log_page) * kB;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int j = u.key0 + 16 * t + (lane & 15);
            const uint8_t* const at = a.pool + (((uint64_t)(page[t] < 0 ? 0 : page[t]) * a.layers + a.layer) * 2 * a.heads + head) * plane +
                                      (uint64_t)((j & ((1 << a.log_page) - 1)) * a.dim * kB);
            if constexpr (TYPE == RAC_CACHE_FP8) {
#pragma unroll
                for (int s = 0; s < kSteps; s += 2) {
                    const int c = channel<TYPE>(s, g);
                    u32x4 x = {0u, 0u, 0u, 0u};
                    if (c < a.dim && page[t] >= 0) x = *reinterpret_cast<const u32x4*>(at + c);
                    k[t][s] = widen8(x[0], x[1]);
                    k[t][s + 1] = widen8(x[2], x[3]);
                }
            } else {
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int c = channel<TYPE>(s, g);
                    k[t][s] = u32x4{0u, 0u, 0u, 0u};
                    if (c < a.dim && page[t] >= 0) k[t][s] = *reinterpret_cast<const u32x4*>(at + 2 * c);
                }
            }
        }
    }
    __device__ __forceinline__ void drafted(const WeightsArgs& a, const Unit& u, const Seq& q, int head) {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int j = u.key0 + 16 * t + (lane & 15);
            const uint16_t* const at = a.k + (int64_t)(q.d0 + j) * a.kv_stride + (int64_t)head * a.dim;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int c = channel<TYPE>(s, g);
                k[t][s] = u32x4{0u, 0u, 0u, 0u};
                if (c < a.dim && j < q.n) k[t][s] = *reinterpret_cast<const u32x4*>(at + c);
            }
        }
    }
};

template <int NT>
struct KeySums {
    f32x4 s[NT];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // Of 16 rows that see every key (what does not exist is not stored).
    __device__ __forceinline__ void add(const f32x4 (&x)[NT], float c2, float lse2) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int y = 0; y < 4; ++y) s[t][y] = s[t][y] + __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][y], c2, -lse2));
    }
    // bits: the keys that this lane's row sees.
    __device__ __forceinline__ void add_some(const f32x4 (&x)[NT], float c2, float lse2, uint64_t bits) {
        const int g = ((int)threadIdx.x & 63) >> 4;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t b = (uint32_t)(bits >> (16 * t)) >> (4 * g);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][y], c2, -lse2));
                s[t][y] = s[t][y] + ((b >> y) & 1u ? e : 0.0f);
            }
        }
    }
    // Over the 16 lanes of a key: halves of the sums change places, until every lane has
    // one, that of key key_of_lane().
    template <int O>
    static __device__ __forceinline__ void halve(float (&v)[4 * NT]) {
        if constexpr (O >= 4 * NT) {
#pragma unroll
            for (int i = 0; i < 4 * NT; ++i) v[i] = v[i] + __shfl_xor(v[i], O);
        } else {
            const bool high = threadIdx.x & O;
#pragma unroll
            for (int i = 0; i < O; ++i) {
                const float keep = high ? v[i + O] : v[i], give = high ? v[i] : v[i + O];
                v[i] = keep + __shfl_xor(give, O);
            }
        }
        if constexpr (O > 1) halve<O / 2>(v);
    }
    __device__ __forceinline__ float join() const {
        float v[4 * NT];
#pragma unroll
        for (int i = 0; i < 4 * NT; ++i) v[i] = s[i / 4][i % 4];
        halve<8>(v);
        return v[0];
    }
    static __device__ __forceinline__ int key_of_lane() {
        const int lane = (int)threadIdx.x & 63, i = lane & (4 * NT - 1) & 15;
        return 16 * (i >> 2) + 4 * (lane >> 4) + (i & 3);
    }
    // (with fewer than 16 sums several lanes have the same)
    static __device__ __forceinline__ bool first_lane() { return ((int)threadIdx.x & 15) < 4 * NT; }
};

// ---------------------------------------------------------------------------
// Few rows a head.  A wavefront takes 32 keys and goes through heads and tiles of 16 rows.
// With SHARE (sums of all heads) the wavefronts of a workgroup have the same keys and
// divide heads and rows; else each has a unit of its own.
//
// Bound by the bytes of the committed keys: one token of 32 sequences of 4001 to 16383 in
// bf16, 8 heads of 128 channels, 591 MB in 114 us, 5.2 TB/s (a large copy reaches 4.9).  200
// short drafts in a window of 1000, 24 MB in 8 bits, take 17 us: three units or less for a
// wavefront, and the latency of their pages, keys and rows one after the other.
constexpr int kFewKeys = 32, kFewRows = 16;

template <int TYPE, int DP, bool SHARE>
__global__ __launch_bounds__(kThreads, DP == 256 ? 2 : 4) void weights_few_kernel(WeightsArgs a) {
    constexpr int NT = kFewKeys / 16, kSteps = DP / 32;
    extern __shared__ int32_t base[];  // [seqs + 1]
    __shared__ float shared_sums[2][kWavesEach][kFewKeys];
    lay_out<kFewKeys, kFewRows>(a, base);
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x / 64);
    const int total = base[a.seqs];
    int turn = 0;
    for (int64_t w = SHARE ? blockIdx.x : (int64_t)blockIdx.x * kWavesEach + wave; w < total;
         w += SHARE ? gridDim.x : gridDim.x * kWavesEach) {
        const int s = uniform(seq_at(base, a.seqs, (int)w));
        const Seq q = seq_of(a, s);
        const Units us = units_of<kFewKeys, kFewRows>(a, q);
        const Unit u = unit_at<kFewKeys>(a, s, us, uniform((int)w - base[s]));
        int page[NT];
        const uint64_t exist = exist_in(a, u, q, page);
        const float c2 = TYPE == RAC_CACHE_FP8 && u.past ? a.scale2 * a.k_scale : a.scale2;
        const bool look = !u.past || a.window > 0;  // whether rows differ in what they see
        // (what is to be added to, ahead of the work)
        const int key = SHARE ? (int)threadIdx.x % kFewKeys : KeySums<NT>::key_of_lane();
        const bool adds = (SHARE ? threadIdx.x < kFewKeys : KeySums<NT>::first_lane()) && ((exist >> key) & 1);
        float* to = nullptr;
        float before = 0.0f;
        if (adds) {
            to = sum_of(a, u, q, key);
            before = *to;
        }
        KeySums<NT> sums;
        sums.clear();
        const int items = us.rows * a.item_heads;
        int at = SHARE ? items * wave / kWavesEach : 0;
        const int end = SHARE ? items * (wave + 1) / kWavesEach : items;
        while (at < end) {
            const int head = u.head >= 0 ? u.head : us.rows == 1 ? at : uniform(at / us.rows), h0 = u.head >= 0 ? 0 : head * us.rows;
            const int stop = h0 + us.rows < end ? h0 + us.rows : end;
            Keys<TYPE, DP, NT> keys;
            keys.take(a, u, q, head, page);
            for (; at < stop; ++at) {
                const int r = (at - h0) * kFewRows + (lane & 15);
                const int n = a.group == 1 ? r : (int)__umulhi((uint32_t)r, a.by_group), h = head * a.group + r - n * a.group;
                const bool is = r < q.m * a.group;
                const int64_t row = q.q0 + n;
                float lse2 = -INFINITY;  // (a row that gives nothing)
                if (is) lse2 = a.lse[row * (a.heads * a.group) + h] * 1.44269504f;
                u32x4 qs[kSteps];
#pragma unroll
                for (int y = 0; y < kSteps; ++y) {
                    const int c = channel<TYPE>(y, lane >> 4);
                    qs[y] = u32x4{0u, 0u, 0u, 0u};
                    if (is && c < a.dim) qs[y] = *reinterpret_cast<const u32x4*>(a.q + row * a.q_stride + (int64_t)h * a.dim + c);
                }
                uint64_t bits = lse2 == -INFINITY ? 0 : exist;
                if (look && bits) bits &= sees(a, q, u, n, sight_of(a, q, n));
                if (!__any(bits != 0)) continue;
                f32x4 x[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    x[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int y = 0; y < kSteps; ++y) x[t] = mma<TYPE>(keys.k[t][y], qs[y], x[t]);
                }
                sums.add_some(x, c2, lse2, bits);
            }
        }
        float v = sums.join();
        if constexpr (SHARE) {
            if (KeySums<NT>::first_lane()) shared_sums[turn][wave][KeySums<NT>::key_of_lane()] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int y = 0; y < kWavesEach; ++y) v = v + shared_sums[turn][y][key];
            turn ^= 1;  // (what is read here is written again only after the next barrier)
        }
        if (adds) *to = before + v;
    }
}

// ---------------------------------------------------------------------------
// Many rows a head.  A workgroup takes 256 keys, 64 a wavefront, and goes through blocks
// of 64 rows, which it shares in LDS: the next block's loads are under way during the
// products of this one.  A unit is cut into parts of at most `size` blocks, which about
// kWant workgroups share out, and the parts are joined.
//
// Chunks of 701 to 2048 rows over 1003 to 6001 tokens, 28 heads on 4 of 128 channels: 170
// GFLOP in 302 us, 563 TF/s (a large matrix product reaches 1360), and 9 us for the join; under
// a profiler 323.  No unit alone is the bound.  For 16 rows by 64 keys the matrix cores are busy
// for 256 cycles, and the vector unit has 16 exponentials of 8 cycles and 32 factors and sums of
// 4; counted are 506 of its cycles, 64 of them the issue of matrix instructions, for 46 vector
// instructions more than these.  Of the 1021 cycles that a tile takes that is 25% and 50%; the
// wavefronts, two a SIMD, wait for 40% of theirs.  With a mask and a window every committed tile
// is masked key by key: 16 trees of 130 nodes, 32 heads on 8, in a window of 4096 take 222 us,
// without the mask 176.
constexpr int kManyKeys = 256, kManyRows = 64, kWant = 3000;
constexpr int kSlots = 2 * kWant;  // (a unit that is cut has fewer than twice its blocks over the size parts)

// base[s]: where the parts of a sequence (with JOIN: its units that were cut) begin, slot[s]
// its partial results.  Returns the size of a part.
template <bool JOIN>
__device__ __forceinline__ int lay_out_parts(const WeightsArgs& a, int32_t* base, int32_t* slot) {
    __shared__ int64_t sums[kWavesEach];
    const int each = (a.seqs + kThreads - 1) / kThreads, s0 = (int)threadIdx.x * each;
    const int s1 = s0 + each < a.seqs ? s0 + each : a.seqs;
    struct Share {
        int64_t units;
        int items;
    };
    const auto share = [&](int s) {
        const Units u = units_of<kManyKeys, kManyRows>(a, seq_of(a, s));
        return Share{(int64_t)(u.committed + u.drafted) * a.unit_heads, u.rows * a.item_heads};
    };
    int64_t work = 0, all;
    Share one{0, 0};  // (with one sequence a thread it is kept)
    for (int s = s0; s < s1; ++s) {
        one = share(s);
        work += one.units * one.items;
    }
    sum_before(work, sums, &all);
    const int64_t even = all / kWant + 1;
    const int size = even < (1 << 30) ? (int)even : 1 << 30;
    const auto parts = [&](int items) { return items > size ? (items + size - 1) / size : 1; };
    int64_t mine = 0, split = 0;
    for (int s = s0; s < s1; ++s) {
        if (each > 1) one = share(s);
        const int p = parts(one.items);
        mine += JOIN ? p > 1 ? one.units : 0 : one.units * p;
        split += p > 1 ? one.units * p : 0;
    }
    int64_t b = sum_before(mine, sums, &all), ignored, at = sum_before(split, sums, &ignored);
    for (int s = s0; s < s1; ++s) {
        if (each > 1) one = share(s);
        const int p = parts(one.items);
        base[s] = held_int(b);
        slot[s] = held_int(at);
        b += JOIN ? p > 1 ? one.units : 0 : one.units * p;
        at += p > 1 ? one.units * p : 0;
    }
    if (threadIdx.x == 0) base[a.seqs] = held_int(all);
    __syncthreads();
    return size;
}

template <int TYPE, int DP>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void weights_many_kernel(WeightsArgs a) {
    constexpr int NT = 4, kSteps = DP / 32, kPieces = DP / 8, kLoads = kManyRows * kPieces / kThreads;
    extern __shared__ int32_t starts[];  // base [seqs + 1], slot [seqs]
    __shared__ u32x4 block[2][kManyRows * kPieces];
    __shared__ float lses[2][kManyRows];
    __shared__ Sight sights[2][kManyRows];
    __shared__ alignas(4) uint8_t whole[2][kWavesEach];  // whether all rows that a wavefront brought give something
    int32_t* const base = starts;
    int32_t* const slot = starts + a.seqs + 1;
    const int size = lay_out_parts<false>(a, base, slot);
    const int t = (int)threadIdx.x, lane = t & 63, wave = uniform(t / 64);
    const int total = base[a.seqs];
    for (int w = (int)blockIdx.x; w < total; w += (int)gridDim.x) {
        const int s = uniform(seq_at(base, a.seqs, w));
        const Seq q = seq_of(a, s);
        const Units us = units_of<kManyKeys, kManyRows>(a, q);
        const int rows = q.m * a.group, all_items = us.rows * a.item_heads;
        const int parts = all_items > size ? uniform((all_items + size - 1) / size) : 1;
        const int i = uniform(w - base[s]), of = uniform(i / parts), part = i - of * parts;
        Unit u = unit_at<kManyKeys>(a, s, us, of);
        // (without a mask no row ahead of the first drafted key sees any)
        int skip = 0;
        if (!u.past && !a.mask) {
            const int64_t first = (int64_t)(u.key0 - (q.n - q.m)) * a.group / kManyRows;
            skip = first <= 0 ? 0 : first < us.rows ? (int)first : us.rows;
        }
        const int blocks = us.rows - skip, items = blocks * a.item_heads;
        const int even = uniform(items / parts), more = items - even * parts;
        const int i0 = part * even + (part < more ? part : more), i1 = i0 + even + (part < more);
        u.key0 += 64 * wave;
        int page[NT];
        const uint64_t exist = exist_in(a, u, q, page);
        const float c2 = TYPE == RAC_CACHE_FP8 && u.past ? a.scale2 * a.k_scale : a.scale2;
        const bool look = !u.past || a.window > 0;  // whether rows differ in what they see
        KeySums<NT> sums;
        sums.clear();
        // Four threads bring a row: of the next block, on its way.  (Where that is: its head, and
        // its first row.)
        u32x4 ahead[kLoads];
        float lse_ahead = 0.0f;
        Sight sight_ahead{0, 0, 0};
        int next_head = u.head >= 0 ? u.head : blocks > 0 ? uniform(i0 / blocks) : 0;
        int next_row = (skip + i0 - (u.head >= 0 ? 0 : next_head * blocks)) * kManyRows;
        const auto node_of = [&](int r) { return a.group == 1 ? r : (int)__umulhi((uint32_t)r, a.by_group); };
        const auto fetch = [&] {
            const int r = next_row + t / 4, node = node_of(r), h = next_head * a.group + r - node * a.group;
            const uint16_t* const from = a.q + (int64_t)(q.q0 + node) * a.q_stride + (int64_t)h * a.dim;
            const bool is = r < rows;
#pragma unroll
            for (int y = 0; y < kLoads; ++y) {
                const int c = 8 * (t % 4 + 4 * y);
                ahead[y] = u32x4{0u, 0u, 0u, 0u};
                if (is && c < a.dim) ahead[y] = *reinterpret_cast<const u32x4*>(from + c);
            }
            lse_ahead = -INFINITY;  // (a row that gives nothing)
            if (is) lse_ahead = a.lse[(int64_t)(q.q0 + node) * (a.heads * a.group) + h] * 1.44269504f;
            if (look && is) sight_ahead = sight_of(a, q, node);
        };
        const auto put = [&](int to) {
#pragma unroll
            for (int y = 0; y < kLoads; ++y) block[to][piece_at<DP>((uint32_t)t / 4, (uint32_t)(t % 4 + 4 * y))] = ahead[y];
            if (t % 4 == 0) {
                lses[to][t / 4] = lse_ahead;
                if (look) sights[to][t / 4] = sight_ahead;
            }
            const bool all = __all(lse_ahead != -INFINITY);
            if (lane == 0) whole[to][wave] = all;
        };
        if (i0 < i1) {
            fetch();
            put(0);
        }
        uint32_t piece[kSteps];  // of this lane's row in a tile of 16
#pragma unroll
        for (int y = 0; y < kSteps; ++y) piece[y] = piece_at<DP>((uint32_t)lane & 15u, (uint32_t)(channel<TYPE>(y, lane >> 4) / 8));
        Keys<TYPE, DP, NT> keys;
        int of_head = -1, now = 0;
        for (int at = i0; at < i1; ++at, now ^= 1) {
            __syncthreads();
            const int head = next_head, r0 = next_row;
            next_row += kManyRows;
            if (next_row >= us.rows * kManyRows) {
                next_row = skip * kManyRows;
                ++next_head;
            }
            if (at + 1 < i1) fetch();
            if (head != of_head) {
                keys.take(a, u, q, head, page);
                of_head = head;
            }
            const uint32_t given = *reinterpret_cast<const uint32_t*>(whole[now]);
            const u32x4* const tile = block[now];
            const auto products = [&](int rt, f32x4 (&x)[NT]) {
#pragma unroll
                for (int y = 0; y < kSteps; ++y) {
                    const u32x4 qs = tile[rt * 16 * kPieces + piece[y]];
#pragma unroll
                    for (int k = 0; k < NT; ++k) x[k] = mma<TYPE>(keys.k[k][y], qs, y ? x[k] : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
                }
            };
            // (without a mask what a row sees moves on with the rows: the first and the last of the
            // block tell whether all see every key, or none any)
            bool plain = !look, none = exist == 0;
            if (look && !a.mask && !none) {
                const int last_row = r0 + kManyRows < rows ? r0 + kManyRows - 1 : rows - 1;
                const Sight first = sight_of(a, q, uniform(node_of(r0))), last = sight_of(a, q, uniform(node_of(last_row)));
                if (u.past) {
                    plain = last.from <= u.key0;
                    none = first.from >= u.key0 + 64;
                } else {
                    plain = last.first <= u.key0 && first.end >= (u.key0 + 64 < q.n ? u.key0 + 64 : q.n);
                    none = last.end <= u.key0 || first.first >= u.key0 + 64;
                }
            }
            if (none) {
            } else if (plain && given == 0x01010101u) {
#pragma unroll
                for (int rt = 0; rt < kManyRows / 16; ++rt) {
                    f32x4 x[NT];
                    products(rt, x);
                    sums.add(x, c2, lses[now][16 * rt + (lane & 15)]);
                }
            } else {
#pragma unroll 1
                for (int rt = 0; rt < kManyRows / 16; ++rt) {
                    const int in = 16 * rt + (lane & 15);
                    const float lse2 = lses[now][in];
                    uint64_t bits = lse2 == -INFINITY ? 0 : exist;
                    if (look && bits) bits &= sees(a, q, u, node_of(r0 + in), sights[now][in]);
                    if (!__any(bits != 0)) continue;
                    f32x4 x[NT];
                    products(rt, x);
                    sums.add_some(x, c2, lse2, bits);
                }
            }
            if (at + 1 < i1) put(now ^ 1);
        }
        __syncthreads();  // (the next unit's first block takes the place of one that is read)
        const float v = sums.join();
        const int key = KeySums<NT>::key_of_lane();
        if (parts == 1) {
            add_to(a, u, q, exist, key, v);
        } else {
            const int64_t to = (int64_t)slot[s] + i;
            if (to < kSlots) a.parts[to * kManyKeys + 64 * wave + key] = v;
        }
    }
}

// Adds the parts of the units that were cut, in order: a workgroup a unit, a thread a key.
__global__ __launch_bounds__(kThreads) void weights_join_kernel(WeightsArgs a) {
    extern __shared__ int32_t starts[];
    int32_t* const base = starts;
    int32_t* const slot = starts + a.seqs + 1;
    const int size = lay_out_parts<true>(a, base, slot);
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x / 64);
    const int total = base[a.seqs];
    for (int w = (int)blockIdx.x; w < total; w += (int)gridDim.x) {
        const int s = uniform(seq_at(base, a.seqs, w));
        const Seq q = seq_of(a, s);
        const Units us = units_of<kManyKeys, kManyRows>(a, q);
        const int items = us.rows * a.item_heads, parts = uniform((items + size - 1) / size), i = uniform(w - base[s]);
        Unit u = unit_at<kManyKeys>(a, s, us, i);
        u.key0 += 64 * wave;
        int page[4];
        const uint64_t exist = exist_in(a, u, q, page);
        const int64_t from = (int64_t)slot[s] + (int64_t)i * parts;
        if (from + parts > kSlots) continue;
        float v = 0.0f;
        constexpr int kAtOnce = 8;
        for (int p = 0; p < parts; p += kAtOnce) {
            float x[kAtOnce];
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) x[y] = p + y < parts ? a.parts[(from + p + y) * kManyKeys + threadIdx.x] : 0.0f;
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) v = v + x[y];
        }
        add_to(a, u, q, exist, lane, v);
    }
}

// ---------------------------------------------------------------------------
// The sums of appended tokens: a lane a token, a wavefront a set.  The time of a launch, 2 us.
struct AppendArgs {
    const int32_t* lengths;
    const int32_t* committed;
    const int32_t* start;
    const int32_t* path;
    const float* draft_weight;
    float* weight;
    int64_t positions;
    int32_t seqs, sets, draft_rows, max_path;
};

__global__ __launch_bounds__(kThreads) void weights_append_kernel(AppendArgs a) {
    const int s = (int)blockIdx.x, len = a.lengths[s], lane = (int)threadIdx.x & 63;
    const int n = a.committed[s] < len ? a.committed[s] : len;
    if (len > a.positions) return;
    const int lo = clamp_int(a.start[s], 0, a.draft_rows), rows = clamp_int(a.start[s + 1], lo, a.draft_rows) - lo;
    // (a wavefront a set)
    for (int set = (int)blockIdx.y * kWavesEach + (int)threadIdx.x / 64; set < a.sets; set += (int)gridDim.y * kWavesEach) {
        float* const to = a.weight + ((int64_t)s * a.sets + set) * a.positions + len - n;
        for (int t = lane; t < n; t += 64) {
            const int node = a.path ? t < a.max_path ? a.path[(int64_t)s * a.max_path + t] : -1 : t;
            float v = 0.0f;
            if (a.draft_weight && node >= 0 && node < rows) v = a.draft_weight[(int64_t)set * a.draft_rows + lo + node];
            to[t] = v;
        }
    }
}

// ---------------------------------------------------------------------------
// Host side

bool weights_valid(const rac_cache_config* c, const rac_tree_config* t) {
    return cache_valid(c) && t && t->q_heads >= 1 && t->q_heads % c->kv_heads == 0 && t->q_heads / c->kv_heads <= 64 &&
           t->rows >= 0 && t->rows <= (1 << 20) && t->max_rows >= 0 && t->max_draft >= 0 && t->window >= 0 &&
           t->scale >= 0.0f && t->scale < __builtin_inff();
}

// The kernel of a call: from 64 rows a key-value head on that of many rows; below it the
// wavefronts share a unit's heads and rows where there are enough of them.  16 sequences of
// 1000 to 8000, 8 heads of 128 channels: the few and the many rows' kernel take 32 and 46 us
// with 16 rows a head, 41 and 47 with 32, 48 and 49 with 48, 55 and 47 with 64, 84 and 58 with
// 128.  Shared and alone: sums of all heads, 4 sequences 13 and 21 us, 16 with 16 rows a head
// 32 and 34; sums for every head 58 and 32.
enum Form { kMany, kShare, kAlone };

template <int TYPE, int DP>
const void* kernel_of(Form form) {
    return form == kMany    ? reinterpret_cast<const void*>(weights_many_kernel<TYPE, DP>)
           : form == kShare ? reinterpret_cast<const void*>(weights_few_kernel<TYPE, DP, true>)
                            : reinterpret_cast<const void*>(weights_few_kernel<TYPE, DP, false>);
}
template <int TYPE>
const void* kernel_of(Form form, int dim) {
    return dim <= 64 ? kernel_of<TYPE, 64>(form) : dim <= 128 ? kernel_of<TYPE, 128>(form) : kernel_of<TYPE, 256>(form);
}

rac_status start(const void* kernel, dim3 grid, void* args, size_t lds, hipStream_t st) {
    void* p[] = {args};
    return hipLaunchKernel(kernel, grid, dim3(kThreads), p, lds, st) == hipSuccess ? RAC_OK : RAC_ERR_HIP;
}

}  // namespace

extern "C" {

size_t rac_tree_weights_workspace(const rac_cache_config* cfg, const rac_tree_config* tree) {
    return weights_valid(cfg, tree) && (int64_t)tree->rows * tree->q_heads < (int64_t(1) << 26) ? (size_t)kSlots * kManyKeys * 4 : 0;
}

rac_status rac_tree_weights(const rac_cache_config* cfg, const rac_tree_config* tree, int32_t layer, int32_t sets,
                            const void* pool, const int32_t* table, const int32_t* lengths, const rac_tree_tensors* t,
                            float* weight, float* draft_weight, void* workspace, size_t workspace_bytes,
                            rac_stream_t stream) {
    if (!weights_valid(cfg, tree) || layer < 0 || layer >= cfg->layers || !t || !sets_valid(cfg, sets)) return RAC_ERR_INVALID;
    if (tree->rows == 0) return RAC_OK;
    const int64_t kv_row = (int64_t)cfg->kv_heads * cfg->head_dim, q_row = (int64_t)tree->q_heads * cfg->head_dim;
    if (!pool || !table || !lengths || !t->q || !t->q_start || !t->lse || !weight || !workspace) return RAC_ERR_INVALID;
    if (t->q_stride < q_row || t->q_stride % 8 || t->draft_rows < 0 || t->mask_words < 0) return RAC_ERR_INVALID;
    if (t->k && (t->kv_stride < kv_row || t->kv_stride % 8 || t->kv_stride > (1 << 25))) return RAC_ERR_INVALID;
    if ((t->mask != nullptr) != (t->mask_words > 0)) return RAC_ERR_INVALID;
    if (!aligned(pool, 16) || !aligned(t->q, 16) || !aligned(t->k, 16) || !aligned(table, 4) || !aligned(lengths, 4) ||
        !aligned(t->q_start, 4) || !aligned(t->draft_start, 4) || !aligned(t->lse, 4) || !aligned(t->mask, 8) ||
        !aligned(weight, 4) || !aligned(draft_weight, 4) || !aligned(workspace, 256))
        return RAC_ERR_ALIGN;
    if ((int64_t)tree->rows * tree->q_heads >= (int64_t(1) << 26) || !sums_counted(cfg, sets)) return RAC_ERR_UNSUPPORTED;
    if (workspace_bytes < rac_tree_weights_workspace(cfg, tree)) return RAC_ERR_CAPACITY;
    const bool drafted = t->k && t->draft_rows > 0;
    WeightsArgs a{};
    a.pool = static_cast<const uint8_t*>(pool);
    a.table = table;
    a.lengths = lengths;
    a.q = static_cast<const uint16_t*>(t->q);
    a.k = drafted ? static_cast<const uint16_t*>(t->k) : nullptr;
    a.q_start = t->q_start;
    a.draft_start = t->draft_start ? t->draft_start : t->q_start;
    a.mask = t->mask;
    a.lse = t->lse;
    a.weight = weight;
    a.draft_weight = drafted ? draft_weight : nullptr;
    a.parts = static_cast<float*>(workspace);
    a.q_stride = t->q_stride;
    a.kv_stride = t->kv_stride;
    a.positions = (int64_t)cfg->max_pages * cfg->page_tokens;
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
    a.sets = sets;
    a.first_set = sets > 1 ? layer * cfg->kv_heads : 0;
    a.unit_heads = sets > 1 ? cfg->kv_heads : 1;
    a.item_heads = cfg->kv_heads / a.unit_heads;
    a.by_group = (uint32_t)(((uint64_t(1) << 32) + a.group - 1) / a.group);
    a.scale2 = (tree->scale > 0.0f ? tree->scale : 1.0f / sqrtf((float)cfg->head_dim)) * 1.4426950408889634f;
    a.k_scale = cfg->k_scale;
    const int64_t most = (int64_t)(tree->max_rows < tree->rows ? tree->max_rows : tree->rows) * a.group;
    const Form form = most >= kManyRows ? kMany : (most + kFewRows - 1) / kFewRows * a.item_heads >= kWavesEach ? kShare : kAlone;
    const void* kernel = cfg->type == RAC_CACHE_BF16   ? kernel_of<RAC_CACHE_BF16>(form, cfg->head_dim)
                         : cfg->type == RAC_CACHE_FP16 ? kernel_of<RAC_CACHE_FP16>(form, cfg->head_dim)
                                                       : kernel_of<RAC_CACHE_FP8>(form, cfg->head_dim);
    const size_t lds = (size_t)(2 * cfg->seqs + 1) * 4;
    if (form != kMany) return start(kernel, dim3(cfg->head_dim > 128 ? 512 : 1024), &a, lds, stream);
    const rac_status st = start(kernel, dim3(cfg->head_dim > 128 ? 256 : 512), &a, lds, stream);
    return st != RAC_OK ? st : start(reinterpret_cast<const void*>(weights_join_kernel), dim3(512), &a, lds, stream);
}

rac_status rac_cache_weights_commit(const rac_cache_config* cfg, int32_t sets, const int32_t* lengths,
                                    const int32_t* committed, const int32_t* draft_start, const int32_t* path,
                                    int32_t max_path, const float* draft_weight, int32_t draft_rows, float* weight,
                                    rac_stream_t stream) {
    if (!cache_valid(cfg) || !sets_valid(cfg, sets) || max_path < 0 || draft_rows < 0 || !lengths || !committed ||
        !draft_start || !weight)
        return RAC_ERR_INVALID;
    if (!aligned(lengths, 4) || !aligned(committed, 4) || !aligned(draft_start, 4) || !aligned(path, 4) ||
        !aligned(draft_weight, 4) || !aligned(weight, 4))
        return RAC_ERR_ALIGN;
    if (!sums_counted(cfg, sets)) return RAC_ERR_UNSUPPORTED;
    AppendArgs a{lengths, committed, draft_start, path, draft_weight, weight, (int64_t)cfg->max_pages * cfg->page_tokens,
                 cfg->seqs, sets, draft_rows, max_path};
    const int y = (sets + kWavesEach - 1) / kWavesEach < 1024 ? (sets + kWavesEach - 1) / kWavesEach : 1024;
    return start(reinterpret_cast<const void*>(weights_append_kernel), dim3((unsigned)cfg->seqs, (unsigned)y), &a, 0, stream);
}

}  // extern "C"
