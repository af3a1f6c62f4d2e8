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
    int32_t slots;
    uint32_t by_group;  // 2^32 / group, rounded up
    float scale2;       // of the scores, times log2(e)
    float k_scale;
};

// ---------------------------------------------------------------------------
// The work.  A unit is a tile of 64 keys of a sequence, for one key-value head or
// all of them; its items are tiles of 16 query rows (rows of a key-value head are the
// (node, query head) pairs of a sequence, node by node) of its heads, one head after the
// other.  A wavefront takes a unit, or a part of one where units are few and long: parts
// of at most `size` items, which about kWant wavefronts share out.
constexpr int kWant = 16384;  // parts of the work wanted: a few for every wavefront that runs at once
constexpr int kKeys = 64, kRowTile = 16, kThreads = 256, kWavesEach = kThreads / 64;

struct Units {
    int tile0, committed, drafted;  // first tile that the window reaches, tiles
    int rows;                       // tiles of rows of a head
};

__device__ __forceinline__ Units units_of(const WeightsArgs& a, const Seq& q) {
    Units u;
    u.tile0 = a.window > 0 && q.length > a.window ? (q.length - a.window) / kKeys : 0;
    u.committed = (q.length + kKeys - 1) / kKeys - u.tile0;
    u.drafted = a.draft_weight ? (q.n + kKeys - 1) / kKeys : 0;
    u.rows = (q.m * a.group + kRowTile - 1) / kRowTile;
    if (u.rows == 0) u.committed = u.drafted = 0;
    return u;
}

// What a sequence has: units, and parts of each.
struct Share {
    int64_t units;
    int items;
};
__device__ __forceinline__ Share share_of(const WeightsArgs& a, int s) {
    const Units u = units_of(a, seq_of(a, s));
    return Share{(int64_t)(u.committed + u.drafted) * a.unit_heads, u.rows * a.item_heads};
}
__device__ __forceinline__ int parts_of(int items, int size) { return items > size ? (items + size - 1) / size : 1; }

constexpr int kNoMore = 0x7FFFFFFF;

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

// Where the work of every sequence begins, in LDS, as every workgroup finds it by itself:
// base[s] of parts (with JOIN: of units that were cut), slot[s] of partial results.
// Returns the size of a part; base[seqs] is the end.
template <bool JOIN>
__device__ __forceinline__ int lay_out(const WeightsArgs& a, int32_t* base, int32_t* slot) {
    __shared__ int64_t sums[kWavesEach];
    const int each = (a.seqs + kThreads - 1) / kThreads, s0 = (int)threadIdx.x * each;
    const int s1 = s0 + each < a.seqs ? s0 + each : a.seqs;
    int64_t work = 0, all;
    Share one{0, 0};  // (with one sequence a thread it is kept)
    for (int s = s0; s < s1; ++s) {
        one = share_of(a, s);
        work += one.units * one.items;
    }
    sum_before(work, sums, &all);
    const int64_t even = all / kWant + 1;
    const int size = even < (1 << 30) ? (int)even : 1 << 30;
    int64_t mine = 0, split = 0;
    for (int s = s0; s < s1; ++s) {
        if (each > 1) one = share_of(a, s);
        const int p = parts_of(one.items, size);
        mine += JOIN ? p > 1 ? one.units : 0 : one.units * p;
        split += p > 1 ? one.units * p : 0;
    }
    int64_t b = sum_before(mine, sums, &all), ignored, at = sum_before(split, sums, &ignored);
    for (int s = s0; s < s1; ++s) {
        if (each > 1) one = share_of(a, s);
        const int p = parts_of(one.items, size);
        base[s] = b < kNoMore ? (int)b : kNoMore;
        slot[s] = at < kNoMore ? (int)at : kNoMore;
        b += JOIN ? p > 1 ? one.units : 0 : one.units * p;
        at += p > 1 ? one.units * p : 0;
    }
    if (threadIdx.x == 0) base[a.seqs] = all < kNoMore ? (int)all : kNoMore;
    __syncthreads();
    return size;
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
    int seq, tile, head;  // the tile of 64 (of the committed or the drafted), -1: all heads
    bool past;
};

__device__ __forceinline__ Unit unit_at(const WeightsArgs& a, int s, const Units& u, int i) {
    Unit r;
    r.seq = s;
    const int t = a.unit_heads > 1 ? uniform(i / a.unit_heads) : i;
    r.head = a.unit_heads > 1 ? i - t * a.unit_heads : a.heads > 1 ? -1 : 0;
    r.past = t < u.committed;
    r.tile = r.past ? u.tile0 + t : t - u.committed;
    return r;
}

// Of the keys of a unit, those that exist.  (Lanes of a column of 16 ask for the same.)
__device__ __forceinline__ uint64_t exist_in(const WeightsArgs& a, const Unit& u, const Seq& q, int (&page)[4]) {
    if (!u.past) return low64(q.n - u.tile * kKeys);
    const int lane = (int)threadIdx.x & 63;
    uint64_t r = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int j = u.tile * kKeys + 16 * t + (lane & 15);
        page[t] = -1;
        if (j < q.length) page[t] = a.table[(size_t)u.seq * a.max_pages + (j >> a.log_page)];
        if ((uint32_t)page[t] >= (uint32_t)a.pages) page[t] = -1;
        r |= (uint64_t)(__ballot(page[t] >= 0) & 0xFFFFu) << (16 * t);
    }
    return r;
}

// Adds a lane's sum of key `key` of the unit.
__device__ __forceinline__ void add_to(const WeightsArgs& a, const Unit& u, const Seq& q, uint64_t exist, int key, float v) {
    if (!((exist >> key) & 1)) return;
    const int64_t set = a.first_set + (u.head > 0 && a.sets > 1 ? u.head : 0), j = (int64_t)u.tile * kKeys + key;
    float* const to = u.past ? a.weight + ((int64_t)u.seq * a.sets + set) * a.positions + j
                             : a.draft_weight + set * a.draft_rows + q.d0 + j;
    *to = *to + v;
}

// A wavefront keeps the keys of its tile in registers, as the first operand of the matrix
// cores, and takes the rows 16 at a time as the second: lane l then holds the scores
// of row l % 16 with keys 16 t + 4 (l / 16) + i, so a row's lse is one number a lane,
// and the sums over rows are additions in place; the 16 lanes of a key are added at the end.
template <int TYPE, int DP>
struct Keys {
    static constexpr int kSteps = DP / 32;
    u32x4 k[4][kSteps];

    // First channel of lane group g in step u: the order of channels is free, and with 8
    // bits the 16 bytes of a load serve two steps.
    static __device__ __forceinline__ int channel(int u, int g) {
        return TYPE == RAC_CACHE_FP8 ? 64 * (u / 2) + 16 * g + 8 * (u % 2) : 32 * u + 8 * g;
    }

    __device__ __forceinline__ void committed(const WeightsArgs& a, const Unit& u, int head, const int (&page)[4]) {
        constexpr int kB = TYPE == RAC_CACHE_FP8 ? 1 : 2;
        const int lane = (int)threadIdx.x & 63, g = lane >> 4;
        const uint64_t plane = ((uint64_t)a.dim << a.log_page) * kB;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int j = u.tile * kKeys + 16 * t + (lane & 15);
            const uint8_t* const at = a.pool + (((uint64_t)(page[t] < 0 ? 0 : page[t]) * a.layers + a.layer) * 2 * a.heads + head) * plane +
                                      (uint64_t)((j & ((1 << a.log_page) - 1)) * a.dim * kB);
            if constexpr (TYPE == RAC_CACHE_FP8) {
#pragma unroll
                for (int s = 0; s < kSteps; s += 2) {
                    const int c = channel(s, g);
                    u32x4 x = {0u, 0u, 0u, 0u};
                    if (c < a.dim && page[t] >= 0) x = *reinterpret_cast<const u32x4*>(at + c);
                    k[t][s] = widen8(x[0], x[1]);
                    k[t][s + 1] = widen8(x[2], x[3]);
                }
            } else {
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int c = channel(s, g);
                    k[t][s] = u32x4{0u, 0u, 0u, 0u};
                    if (c < a.dim && page[t] >= 0) k[t][s] = *reinterpret_cast<const u32x4*>(at + 2 * c);
                }
            }
        }
    }
    __device__ __forceinline__ void drafted(const WeightsArgs& a, const Unit& u, const Seq& q, int head) {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int j = u.tile * kKeys + 16 * t + (lane & 15);
            const uint16_t* const at = a.k + (int64_t)(q.d0 + j) * a.kv_stride + (int64_t)head * a.dim;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int c = channel(s, g);
                k[t][s] = u32x4{0u, 0u, 0u, 0u};
                if (c < a.dim && j < q.n) k[t][s] = *reinterpret_cast<const u32x4*>(at + c);
            }
        }
    }
};

// 16 rows: their queries, and their lse in powers of two (infinity: nothing to give).
template <int TYPE, int DP>
struct Queries {
    static constexpr int kSteps = DP / 32;
    u32x4 q[kSteps];
    float lse2;
    int node;   // -1: no row
    bool none;  // a row that gives nothing

    __device__ __forceinline__ void take(const WeightsArgs& a, const Seq& s, int head, int tile) {
        const int lane = (int)threadIdx.x & 63, r = tile * kRowTile + (lane & 15);
        const bool is = r < s.m * a.group;
        const int n = a.group == 1 ? r : (int)__umulhi((uint32_t)r, a.by_group);
        node = is ? n : -1;
        lse2 = INFINITY;
        const int h = head * a.group + r - n * a.group;
        const int64_t row = s.q0 + n;
        if (is) lse2 = a.lse[row * (a.heads * a.group) + h] * 1.44269504f;
        none = lse2 == -INFINITY;
        const uint16_t* const at = a.q + row * a.q_stride + (int64_t)h * a.dim;
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int c = Keys<TYPE, DP>::channel(u, lane >> 4);
            q[u] = u32x4{0u, 0u, 0u, 0u};
            if (is && c < a.dim) q[u] = *reinterpret_cast<const u32x4*>(at + c);
        }
    }
};

// Bound by the bytes of the committed keys where sequences have few rows, and by the
// exponentials (a quarter of the matrix cores' rate for 128 channels) where they
// have many.
template <int TYPE, int DP>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : DP == 128 ? 2 : 3) void weights_kernel(WeightsArgs a) {
    extern __shared__ int32_t starts[];  // base [seqs + 1], slot [seqs]
    int32_t* const base = starts;
    int32_t* const slot = starts + a.seqs + 1;
    const int size = lay_out<false>(a, base, slot);
    const int lane = (int)threadIdx.x & 63;
    const int total = base[a.seqs], step = (int)gridDim.x * kWavesEach;
    for (int64_t w = (int64_t)blockIdx.x * kWavesEach + __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64); w < total; w += step) {
        const int s = __builtin_amdgcn_readfirstlane(seq_at(base, a.seqs, (int)w));
        const Seq q = seq_of(a, s);
        const Units us = units_of(a, q);
        const int items = us.rows * a.item_heads, parts = uniform(parts_of(items, size));
        const int i = uniform((int)w - base[s]), of = uniform(i / parts), part = i - of * parts;
        const Unit u = unit_at(a, s, us, of);
        int page[4];
        const uint64_t exist = exist_in(a, u, q, page);
        const float c2 = TYPE == RAC_CACHE_FP8 && u.past ? a.scale2 * a.k_scale : a.scale2;
        const bool look = !u.past || a.window > 0;  // whether rows differ in what they see
        f32x4 sum[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const int even = uniform(items / parts), more = items - even * parts;
        const int i0 = part * even + (part < more ? part : more), i1 = i0 + even + (part < more);
        for (int at = i0; at < i1;) {
            const int head = u.head >= 0 ? u.head : uniform(at / us.rows), h0 = u.head >= 0 ? 0 : head * us.rows;
            const int end = h0 + us.rows < i1 ? h0 + us.rows : i1;
            Keys<TYPE, DP> keys;
            if (u.past)
                keys.committed(a, u, head, page);
            else
                keys.drafted(a, u, q, head);
            Queries<TYPE, DP> next;
            next.take(a, q, head, at - h0);
            for (; at < end; ++at) {
                const Queries<TYPE, DP> now = next;
                if (at + 1 < end) next.take(a, q, head, at + 1 - h0);
                uint64_t bits = now.none ? 0 : exist;
                if (look && now.node >= 0 && !now.none) {
                    const Sight see = sight_of(a, q, now.node);
                    const int k0 = u.tile * kKeys;
                    if (u.past) {
                        bits &= ~low64(see.from - k0);
                    } else {
                        bits &= low64(see.end - k0) & ~low64(see.first - k0);
                        if (a.mask && bits) bits &= a.mask[(int64_t)(q.q0 + now.node) * a.mask_words + u.tile];
                    }
                }
                if (!__any(now.node >= 0 && bits)) continue;
                const bool all = !__any(now.node < 0 || bits != exist);
                const float ref = now.lse2;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int y = 0; y < DP / 32; ++y) x = mma<TYPE>(keys.k[t][y], now.q[y], x);
                    if (all) {
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            sum[t][y] = sum[t][y] + __builtin_amdgcn_exp2f(__builtin_fmaf(x[y], c2, -ref));
                    } else {
                        const uint32_t b = (uint32_t)(bits >> (16 * t)) >> (4 * (lane >> 4));
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[y], c2, -ref));
                            sum[t][y] = sum[t][y] + (now.node >= 0 && (b >> y) & 1u ? e : 0.0f);
                        }
                    }
                }
            }
        }
        // over the 16 lanes of a key: halves of the sums change places, until every lane has one
        float v[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) v[t] = sum[t / 4][t % 4];
#pragma unroll
        for (int o = 8; o > 0; o /= 2) {
            const bool high = lane & o;
#pragma unroll
            for (int t = 0; t < o; ++t) {
                const float keep = high ? v[t + o] : v[t], give = high ? v[t] : v[t + o];
                v[t] = keep + __shfl_xor(give, o);
            }
        }
        const int key = 16 * ((lane & 15) >> 2) + 4 * (lane >> 4) + (lane & 3);
        if (parts == 1) {
            add_to(a, u, q, exist, key, v[0]);
        } else {
            const int64_t to = (int64_t)slot[s] + i;
            if (to < a.slots) a.parts[to * kKeys + key] = v[0];
        }
    }
}

// Adds the parts of the units that were cut, in order: a wavefront a unit, a lane a key.
__global__ __launch_bounds__(kThreads) void weights_join_kernel(WeightsArgs a) {
    extern __shared__ int32_t starts[];
    int32_t* const base = starts;
    int32_t* const slot = starts + a.seqs + 1;
    const int size = lay_out<true>(a, base, slot);
    const int lane = (int)threadIdx.x & 63;
    const int total = base[a.seqs], step = (int)gridDim.x * kWavesEach;
    for (int64_t w = (int64_t)blockIdx.x * kWavesEach + __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64); w < total; w += step) {
        const int s = __builtin_amdgcn_readfirstlane(seq_at(base, a.seqs, (int)w));
        const Seq q = seq_of(a, s);
        const Units us = units_of(a, q);
        const int parts = uniform(parts_of(us.rows * a.item_heads, size)), i = uniform((int)w - base[s]);
        const Unit u = unit_at(a, s, us, i);
        int page[4];
        const uint64_t exist = exist_in(a, u, q, page);
        const int64_t from = (int64_t)slot[s] + (int64_t)i * parts;
        if (from + parts > a.slots) continue;
        float v = 0.0f;
        constexpr int kAtOnce = 8;
        for (int p = 0; p < parts; p += kAtOnce) {
            float x[kAtOnce];
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) x[y] = p + y < parts ? a.parts[(from + p + y) * kKeys + lane] : 0.0f;
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) v = v + x[y];
        }
        add_to(a, u, q, exist, lane, v);
    }
}

// ---------------------------------------------------------------------------
// The sums of appended tokens: a lane a token, a wavefront a set.
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

constexpr int kSlots = 2 * kWant;  // (a unit that is cut has fewer than twice its items over the size parts)

bool weights_valid(const rac_cache_config* c, const rac_tree_config* t) {
    return cache_valid(c) && t && t->q_heads >= 1 && t->q_heads % c->kv_heads == 0 && t->q_heads / c->kv_heads <= 64 &&
           t->rows >= 0 && t->rows <= (1 << 20) && t->max_rows >= 0 && t->max_draft >= 0 && t->window >= 0 &&
           t->scale >= 0.0f && t->scale < __builtin_inff();
}

template <int TYPE>
const void* kernel_of(int dim) {
    return dim <= 64    ? reinterpret_cast<const void*>(weights_kernel<TYPE, 64>)
           : dim <= 128 ? reinterpret_cast<const void*>(weights_kernel<TYPE, 128>)
                        : reinterpret_cast<const void*>(weights_kernel<TYPE, 256>);
}

rac_status start(const void* kernel, dim3 grid, void* args, size_t lds, hipStream_t st) {
    void* p[] = {args};
    return hipLaunchKernel(kernel, grid, dim3(kThreads), p, lds, st) == hipSuccess ? RAC_OK : RAC_ERR_HIP;
}

}  // namespace

extern "C" {

size_t rac_tree_weights_workspace(const rac_cache_config* cfg, const rac_tree_config* tree) {
    return weights_valid(cfg, tree) && (int64_t)tree->rows * tree->q_heads < (int64_t(1) << 26) ? (size_t)kSlots * kKeys * 4 : 0;
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
    a.slots = kSlots;
    a.by_group = (uint32_t)(((uint64_t(1) << 32) + a.group - 1) / a.group);
    a.scale2 = (tree->scale > 0.0f ? tree->scale : 1.0f / sqrtf((float)cfg->head_dim)) * 1.4426950408889634f;
    a.k_scale = cfg->k_scale;
    const void* kernel = cfg->type == RAC_CACHE_BF16   ? kernel_of<RAC_CACHE_BF16>(cfg->head_dim)
                         : cfg->type == RAC_CACHE_FP16 ? kernel_of<RAC_CACHE_FP16>(cfg->head_dim)
                                                       : kernel_of<RAC_CACHE_FP8>(cfg->head_dim);
    const size_t lds = (size_t)(2 * cfg->seqs + 1) * 4;
    const rac_status st = start(kernel, dim3(1024), &a, lds, stream);
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
