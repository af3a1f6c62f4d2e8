// evict.hip - gfx950 kernels and C ABI of eviction from the paged cache by
// accumulated attention weight.  The contract is in include/rac_cache.h.
//
// A kept token moves only if it lies past the cut, into a place that an evicted one
// left: so a round that evicts a few tokens moves a few, sources and targets never
// meet, and most shared pages stay shared.  Only the last `recent` tokens shift, in order.
#include "cache_common.h"

namespace {

// What the first launch finds out about a sequence.  Places are its positions that
// have a page, in order.
struct EvictRecord {
    int32_t cut;      // whether it is to be cut
    int32_t n, m;     // tokens that stay, places before
    int32_t length;   // positions before
    int32_t border;   // n - recent: from here on the last tokens go, in order
    int32_t pages;    // that it has
    int32_t gaps;     // whether some position has no page
    int32_t demand;   // pages to be replaced
    int32_t base;     // where its pages begin in the list of free ones, -1: refused
};

// What stays of the places in [lo, hi): those above the bar, and the first `left` at it.
struct Choice {
    int32_t lo, hi, left;
    uint32_t bar;
    bool ties;  // whether not all of those at the bar stay
};

struct EvictArgs {
    uint8_t* pool;
    int32_t* table;
    int32_t* lengths;
    int32_t* refs;
    float* weight;
    const int32_t* keep;
    int32_t* evicted;
    int32_t* source;
    EvictRecord* record;  // [seqs]
    int32_t* old_page;    // [seqs][max_pages], of the places' pages: number,
    int32_t* old_at;      // where in the table,
    int32_t* fresh;       // and which of the demanded pages replaces it, or -1
    int32_t* free_list;   // [pages]
    int32_t* list;        // [seqs][sets][positions]: holes from the front, what fills them from the back
    int32_t* holes;       // [seqs][sets]
    uint64_t* hole_bits;  // [seqs][sets][words]
    int32_t* digits;      // [seqs][sets][3][2048], counts of weights' digits, and
    int32_t* tally;       // [seqs][sets][split][4], of parts, and
    Choice* chosen;       // [seqs][sets], where a sequence has several parts
    int64_t positions, words;
    int32_t split, part, digit;
    int32_t layers, heads, row_bytes, log_page, pages, seqs, max_pages, sets, first, recent, parts, end_parts;

    __device__ __forceinline__ int64_t sums(int s, int set) const { return ((int64_t)s * sets + set); }
    // The position of a place.
    __device__ __forceinline__ int position(const EvictRecord& r, int s, int place) const {
        if (!r.gaps) return place;
        return (old_at[(int64_t)s * max_pages + (place >> log_page)] << log_page) | (place & ((1 << log_page) - 1));
    }
    __device__ __forceinline__ int page_now(const EvictRecord& r, int s, int d) const {
        const int64_t at = (int64_t)s * max_pages + d;
        const int f = fresh[at];
        return *(f < 0 ? old_page + at : free_list + r.base + f);
    }
    __device__ __forceinline__ uint8_t* row_of(int page, int layer, int side, int head, int place) const {
        const uint64_t plane = ((uint64_t)page * layers + layer) * 2 * heads + (uint64_t)side * heads + head;
        return pool + (plane << log_page) * row_bytes + (uint64_t)(place & ((1 << log_page) - 1)) * row_bytes;
    }
};

// Weights in an order of whole numbers; a NaN is below all.
__device__ __forceinline__ uint32_t rank_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);  // (-0 is 0)
    return x != x ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// ---------------------------------------------------------------------------
// First: the places of a sequence; the weight that divides what stays from what goes,
// digit by digit from the top (counts of 2048 values in LDS); and, in one ordered pass, the
// holes and what fills them.  Bound by the latency of one workgroup's passes: 15 us for
// sequences of up to 4000 (kSteps 8: 17 us), and 9 us more for every 8192 places of a long one.
constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64, kDigit = 2048;
constexpr int kSteps = 4, kChunk = kPickThreads * kSteps;  // places a thread and a workgroup has at once

__device__ __forceinline__ Choice choice_of(const EvictArgs& a, const EvictRecord& r) {
    const int recent = r.n - r.border;
    Choice c{a.first < r.border ? a.first : r.border, r.m - recent, 0, 0, false};
    c.left = r.border - c.lo;
    if (c.left == 0) c.bar = ~0u;  // (no weight has this rank)
    return c;
}

// The record and the pages of a sequence, by a workgroup.
__device__ EvictRecord see(const EvictArgs& a, int s, int set, int32_t* sums) {
    const int t = (int)threadIdx.x, page = 1 << a.log_page;
    EvictRecord r{};
    r.length = clamp_int(a.lengths[s], 0, a.max_pages << a.log_page);
    const int keep = a.keep[s], used = (r.length + page - 1) >> a.log_page;
    const int32_t* const row = a.table + (int64_t)s * a.max_pages;
    __syncthreads();
    // how many positions have a page
    int mine = 0, all;
    constexpr int kEach = 8;  // entries a thread has at once
    for (int64_t d0 = 0; d0 < used; d0 += kPickThreads * kEach) {
        int p[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t d = d0 + t + i * kPickThreads;
            p[i] = row[d < used ? d : used - 1];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine += d0 + t + i * kPickThreads < used && (uint32_t)p[i] < (uint32_t)a.pages;
    }
    scan_workgroup<kPickWaves>(mine, sums, &all);
    r.pages = all;
    r.gaps = all != used;
    const int tail = r.length & (page - 1);
    const bool whole = tail == 0 || (uint32_t)row[used - 1] >= (uint32_t)a.pages;
    r.m = (all << a.log_page) - (whole ? 0 : page - tail);
    r.cut = keep >= 0 && r.m > keep;
    r.n = r.cut ? keep : r.m;
    r.border = r.n - (a.recent < r.n ? a.recent : r.n);
    if (set == 0 && t == 0) a.record[s] = r;
    if (!r.cut) return r;
    if (set == 0 || r.gaps) {  // (with gaps every set needs the places: they write the same)
        int at = 0;
        for (int64_t d0 = 0; d0 < used; d0 += kPickThreads * kEach) {
            const int lane = t & 63;
            const int64_t own = d0 + t / 64 * (64 * kEach) + lane;
            int p[kEach], count = 0;
            uint64_t is[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) p[i] = row[own + 64 * i < used ? own + 64 * i : used - 1];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                is[i] = __ballot(own + 64 * i < used && (uint32_t)p[i] < (uint32_t)a.pages);
                count += __popcll(is[i]);
            }
            __syncthreads();
            if (lane == 0) sums[t / 64] = count;
            __syncthreads();
            int64_t to = (int64_t)s * a.max_pages + at;
            for (int x = 0; x < kPickWaves; ++x) {
                to += x < t / 64 ? sums[x] : 0;
                at += sums[x];
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int64_t k = to + __popcll(is[i] & ((uint64_t(1) << lane) - 1));
                if ((is[i] >> lane) & 1) {
                    a.old_page[k] = p[i];
                    a.old_at[k] = (int)own + 64 * i;
                }
                to += __popcll(is[i]);
            }
        }
        __syncthreads();
    }
    return r;
}

// The places of a thread in the chunk at p0, 64 kSteps in a row to a wavefront.
__device__ __forceinline__ int place_of(int p0, int y) {
    return p0 + (int)threadIdx.x / 64 * 64 * kSteps + 64 * y + ((int)threadIdx.x & 63);
}

__device__ __forceinline__ void load_places(const EvictArgs& a, const EvictRecord& r, int s, const float* w, const Choice& c,
                                            int p0, uint32_t (&k)[kSteps]) {
    int at[kSteps];
    float x[kSteps];
#pragma unroll
    for (int y = 0; y < kSteps; ++y) {  // (those outside read a place inside, and are not counted)
        const int p = place_of(p0, y);
        at[y] = p < c.lo ? c.lo : p < c.hi ? p : c.hi - 1;
    }
    if (r.gaps)
#pragma unroll
        for (int y = 0; y < kSteps; ++y) at[y] = a.position(r, s, at[y]);
#pragma unroll
    for (int y = 0; y < kSteps; ++y) x[y] = w[at[y]];
#pragma unroll
    for (int y = 0; y < kSteps; ++y) k[y] = rank_of(x[y]);
}

// Counts the values of a digit, among those whose higher digits are the bar's.
__device__ __forceinline__ void count_places(const Choice& c, int digit, int p0, const uint32_t (&k)[kSteps], int32_t* count) {
    const int lane = (int)threadIdx.x & 63, shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    const uint32_t high = digit == 0 ? 0 : ~0u << (shift + bits), mask = (1u << bits) - 1;
#pragma unroll
    for (int y = 0; y < kSteps; ++y) {
        const int p = place_of(p0, y);
        const bool in = p >= c.lo && p < c.hi && ((k[y] ^ c.bar) & high) == 0;
        const uint64_t who = __ballot(in);
        if (!who) continue;
        // (weights that are alike, zeros for one, would queue up at one counter)
        const uint32_t v = (k[y] >> shift) & mask, one = __builtin_amdgcn_readlane(v, __builtin_ctzll(who));
        if (__ballot(in && v == one) == who) {
            if (lane == __builtin_ctzll(who)) atomicAdd(count + one, __popcll(who));
        } else if (in) {
            atomicAdd(count + v, 1);
        }
    }
}

// The digit at which the counts from the top reach what is left.
__device__ void take_digit(Choice& c, int digit, const int32_t* count, int32_t* sums, int32_t* found) {
    const int t = (int)threadIdx.x, shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
    int all;
    const int c1 = count[kDigit - 1 - 2 * t], c0 = count[kDigit - 2 - 2 * t];
    const int above = scan_workgroup<kPickWaves>(c0 + c1, sums, &all);
    if (above < c.left && c.left <= above + c1) {
        found[0] = kDigit - 1 - 2 * t;
        found[1] = above;
        found[2] = c1;
    } else if (above + c1 < c.left && c.left <= above + c1 + c0) {
        found[0] = kDigit - 2 - 2 * t;
        found[1] = above + c1;
        found[2] = c0;
    }
    __syncthreads();
    c.bar |= (uint32_t)found[0] << shift;
    c.left -= found[1];
    c.ties = found[2] > c.left;
    __syncthreads();
}

// Holes before the border and what stays behind it, of the places in [begin, end), in
// order, after nh, nf and (at the bar) nt of earlier ones; k has them if there is one chunk only.
__device__ void order_places(const EvictArgs& a, const EvictRecord& r, int s, int set, const Choice& c, int begin, int end,
                             bool held, uint32_t (&k)[kSteps], int& nh, int& nf, int& nt, int32_t* sums, int32_t* more) {
    const int lane = (int)threadIdx.x & 63, wv = (int)threadIdx.x / 64;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    const float* const w = a.weight + a.sums(s, set) * a.positions;
    int32_t* const list = a.list + a.sums(s, set) * a.positions;
    uint64_t* const bits = a.hole_bits + a.sums(s, set) * a.words;
    for (int p0 = begin; p0 < end; p0 += kChunk) {
        if (!held) load_places(a, r, s, w, c, p0, k);
        uint64_t hole[kSteps], fill[kSteps];
        int h = 0, f = 0, before = nt;
        if (c.ties) {
            int e = 0;
#pragma unroll
            for (int y = 0; y < kSteps; ++y) {
                const int p = place_of(p0, y);
                e += __popcll(__ballot(p >= c.lo && p < c.hi && k[y] == c.bar));
            }
            __syncthreads();
            if (lane == 0) sums[wv] = e;
            __syncthreads();
            for (int x = 0; x < kPickWaves; ++x) {
                before += x < wv ? sums[x] : 0;
                nt += sums[x];
            }
        }
#pragma unroll
        for (int y = 0; y < kSteps; ++y) {
            const int p = place_of(p0, y);
            const bool at_bar = p >= c.lo && p < c.hi && k[y] == c.bar;
            bool stays = p < c.lo || k[y] > c.bar || at_bar;
            if (c.ties) {
                const uint64_t tie = __ballot(at_bar);
                stays &= !at_bar || before + __popcll(tie & below) < c.left;
                before += __popcll(tie);
            }
            hole[y] = __ballot(p < r.border && !stays);
            fill[y] = __ballot(p >= r.border && p < c.hi && stays);
            h += __popcll(hole[y]);
            f += __popcll(fill[y]);
        }
        __syncthreads();
        if (lane == 0) {
            sums[wv] = h;
            more[wv] = f;
        }
        __syncthreads();
        int ah = nh, af = nf;
        for (int x = 0; x < kPickWaves; ++x) {
            ah += x < wv ? sums[x] : 0;
            af += x < wv ? more[x] : 0;
            nh += sums[x];
            nf += more[x];
        }
#pragma unroll
        for (int y = 0; y < kSteps; ++y) {
            const int p = place_of(p0, y), q = p - lane;
            if ((hole[y] >> lane) & 1) list[ah + __popcll(hole[y] & below)] = p;
            if ((fill[y] >> lane) & 1) list[a.positions - 1 - (af + __popcll(fill[y] & below))] = p;
            if (lane == 0 && q < r.border) bits[q / 64] = hole[y];
            ah += __popcll(hole[y]);
            af += __popcll(fill[y]);
        }
    }
}

// A workgroup a sequence and set does it all.
__global__ __launch_bounds__(kPickThreads) void evict_pick_kernel(EvictArgs a) {
    __shared__ int32_t count[kDigit], sums[kPickWaves], more[kPickWaves], found[3];
    const int t = (int)threadIdx.x, s = (int)blockIdx.y;
    for (int set = (int)blockIdx.x; set < a.sets; set += (int)gridDim.x) {
        const EvictRecord r = see(a, s, set, sums);
        if (!r.cut) continue;
        const float* const w = a.weight + a.sums(s, set) * a.positions;
        Choice c = choice_of(a, r);
        uint32_t k[kSteps];
        const bool held = c.hi <= kChunk;
        if (held) load_places(a, r, s, w, c, 0, k);
        for (int digit = 0; digit < (c.left > 0 ? 3 : 0); ++digit) {
            for (int i = t; i < kDigit; i += kPickThreads) count[i] = 0;
            __syncthreads();
            for (int p0 = 0; p0 < c.hi; p0 += kChunk) {
                if (!held) load_places(a, r, s, w, c, p0, k);
                count_places(c, digit, p0, k, count);
            }
            __syncthreads();
            take_digit(c, digit, count, sums, found);
        }
        int nh = 0, nf = 0, nt = 0;
        order_places(a, r, s, set, c, 0, c.hi, held, k, nh, nf, nt, sums, more);
        if (t == 0) a.holes[a.sums(s, set)] = nh;
    }
}

// Long sequences of few sets: `split` workgroups each, of `part` places, and a launch for
// each of these steps.  The counts are whole numbers, so that their order is no matter.
// 131k places of 8 heads: 6 us, three times 6, 11 and 9; in one workgroup each 153 us.
__global__ __launch_bounds__(kPickThreads) void evict_see_kernel(EvictArgs a) {
    __shared__ int32_t sums[kPickWaves];
    const int s = (int)blockIdx.y;
    for (int set = (int)blockIdx.x; set < a.sets; set += (int)gridDim.x) {
        see(a, s, set, sums);
        for (int i = (int)threadIdx.x; i < 3 * kDigit; i += kPickThreads) a.digits[a.sums(s, set) * 3 * kDigit + i] = 0;
    }
}

// The choice after some digits, from the counts of all parts.
__device__ Choice choice_after(const EvictArgs& a, const EvictRecord& r, int s, int set, int digits, int32_t* sums, int32_t* found) {
    Choice c = choice_of(a, r);
    for (int digit = 0; digit < (c.left > 0 ? digits : 0); ++digit)
        take_digit(c, digit, a.digits + (a.sums(s, set) * 3 + digit) * kDigit, sums, found);
    return c;
}

__global__ __launch_bounds__(kPickThreads) void evict_count_kernel(EvictArgs a) {
    __shared__ int32_t count[kDigit], sums[kPickWaves], found[3];
    const int t = (int)threadIdx.x, s = (int)blockIdx.y;
    const EvictRecord r = a.record[s];
    if (!r.cut) return;
    for (int i = (int)blockIdx.x; i < a.sets * a.split; i += (int)gridDim.x) {
        const int set = i / a.split, begin = (i - set * a.split) * a.part;
        const Choice c = choice_after(a, r, s, set, a.digit, sums, found);
        const int end = begin + a.part < c.hi ? begin + a.part : c.hi;
        if (c.left == 0 || begin >= end) continue;
        for (int x = t; x < kDigit; x += kPickThreads) count[x] = 0;
        __syncthreads();
        for (int p0 = begin; p0 < end; p0 += kChunk) {
            uint32_t k[kSteps];
            load_places(a, r, s, a.weight + a.sums(s, set) * a.positions, c, p0, k);
            count_places(c, a.digit, p0, k, count);
        }
        __syncthreads();
        for (int x = t; x < kDigit; x += kPickThreads)
            if (count[x]) atomicAdd(a.digits + (a.sums(s, set) * 3 + a.digit) * kDigit + x, count[x]);
        __syncthreads();
    }
}

// How many holes and fills a part has, and how many at the bar on either side of the border.
__global__ __launch_bounds__(kPickThreads) void evict_tally_kernel(EvictArgs a) {
    __shared__ int32_t sums[kPickWaves], found[3];
    const int t = (int)threadIdx.x, s = (int)blockIdx.y;
    const EvictRecord r = a.record[s];
    if (!r.cut) return;
    for (int i = (int)blockIdx.x; i < a.sets * a.split; i += (int)gridDim.x) {
        const int set = i / a.split, begin = (i - set * a.split) * a.part;
        const Choice c = choice_after(a, r, s, set, 3, sums, found);
        const int end = begin + a.part < c.hi ? begin + a.part : c.hi;
        if (t == 0 && begin == 0) a.chosen[a.sums(s, set)] = c;
        int of[4] = {0, 0, 0, 0};
        for (int p0 = begin; p0 < end; p0 += kChunk) {
            uint32_t k[kSteps];
            load_places(a, r, s, a.weight + a.sums(s, set) * a.positions, c, p0, k);
#pragma unroll
            for (int y = 0; y < kSteps; ++y) {
                const int p = place_of(p0, y);
                const bool in = p >= c.lo && p < c.hi, early = p < r.border, at_bar = in && k[y] == c.bar, above = k[y] > c.bar;
                of[0] += in && early && !at_bar && !above;
                of[1] += in && !early && above;
                of[2] += early && at_bar;
                of[3] += !early && at_bar;
            }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            int all;
            scan_workgroup<kPickWaves>(of[x], sums, &all);
            if (t == 0) a.tally[(a.sums(s, set) * a.split + i - set * a.split) * 4 + x] = all;
        }
    }
}

__global__ __launch_bounds__(kPickThreads) void evict_order_kernel(EvictArgs a) {
    __shared__ int32_t sums[kPickWaves], more[kPickWaves];
    const int s = (int)blockIdx.y;
    const EvictRecord r = a.record[s];
    if (!r.cut) return;
    for (int i = (int)blockIdx.x; i < a.sets * a.split; i += (int)gridDim.x) {
        const int set = i / a.split, part = i - set * a.split, begin = part * a.part;
        const Choice c = a.chosen[a.sums(s, set)];
        const int end = begin + a.part < c.hi ? begin + a.part : c.hi;
        int nh = 0, nf = 0, nt = 0;
        for (int x = 0; x < part; ++x) {
            const int32_t* const of = a.tally + (a.sums(s, set) * a.split + x) * 4;
            const int ties = of[2] + of[3], stay = clamp_int(c.left - nt, 0, ties), early = stay < of[2] ? stay : of[2];
            nh += of[0] + of[2] - early;
            nf += of[1] + stay - early;
            nt += ties;
        }
        uint32_t k[kSteps];
        if (begin < end) order_places(a, r, s, set, c, begin, end, false, k, nh, nf, nt, sums, more);
        if (threadIdx.x == 0 && part == a.split - 1) a.holes[a.sums(s, set)] = nh;
    }
}

// ---------------------------------------------------------------------------
// Then: a workgroup a sequence finds the shared pages that change in any set.  Latency:
// 4 to 5 us with few sets, 8 for 3000 pages of a sequence (with 256 threads 15).  A thread goes
// through the sets of a page until one has changed it, a load each: where no set changes any of
// 188 shared pages of three forks the whole call takes 36 us with one set, 176 with 256.
constexpr int kDemandThreads = 1024;

__global__ __launch_bounds__(kDemandThreads) void evict_demand_kernel(EvictArgs a) {
    __shared__ int32_t sums[kDemandThreads / 64];
    const int s = (int)blockIdx.y, t = (int)threadIdx.x, page = 1 << a.log_page;
    const EvictRecord r = a.record[s];
    if (!r.cut) return;
    const int used = (r.n + page - 1) >> a.log_page;
    int demand = 0;
    for (int d0 = 0; d0 < used; d0 += kDemandThreads) {
        const int d = d0 + t;
        bool change = false;
        if (d < used && a.refs[a.old_page[(int64_t)s * a.max_pages + d]] > 1) {
            change = ((d + 1) << a.log_page) > r.border && r.border < r.n;
            const int p0 = d << a.log_page, p1 = p0 + page < r.border ? p0 + page : r.border;
            for (int set = 0; set < a.sets && !change; ++set) {
                const uint64_t* const bits = a.hole_bits + a.sums(s, set) * a.words;
                for (int p = p0; p < p1; p += 64) {
                    const uint64_t b = bits[p / 64] >> (p & 63);
                    change |= (page >= 64 ? b : b & ((uint64_t(1) << page) - 1)) != 0;
                }
            }
        }
        int all;
        const int at = demand + scan_workgroup<kDemandThreads / 64>(change, sums, &all);
        if (d < used) a.fresh[(int64_t)s * a.max_pages + d] = change ? at : -1;
        demand += all;
    }
    if (t == 0) a.record[s].demand = demand;
}

// ---------------------------------------------------------------------------
// Then: one workgroup hands out the free pages, the lowest first, to the sequences in
// order.  Bound by latency: 3 us for 32 sequences, 9 where thousands of pages are looked at.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

__global__ __launch_bounds__(kPlanThreads) void evict_plan_kernel(EvictArgs a) {
    constexpr int kPer = 4;  // sequences a thread (4096 / 1024)
    __shared__ int32_t sums[kPlanWaves];
    __shared__ int32_t turn[kPer * kPlanThreads];
    const int t = (int)threadIdx.x, lane = t & 63;
    EvictRecord r[kPer];
    int need[kPer], base[kPer], demand = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = t + i * kPlanThreads;
        need[i] = base[i] = 0;
        r[i].cut = 0;
        if (i * kPlanThreads >= a.seqs) continue;
        if (s < a.seqs) {
            r[i] = a.record[s];
            if (r[i].cut) need[i] = r[i].demand;
        }
        int all;
        base[i] = (int)((uint32_t)demand + (uint32_t)scan_workgroup<kPlanWaves>(need[i], sums, &all));
        demand = all < kMostSum - demand ? demand + all : kMostSum;
    }
    int found = 0;
    constexpr int kEach = 16, kStep = kPlanThreads * kEach;
    for (int p0 = 0; p0 < a.pages && found < demand; p0 += kStep) {
        uint64_t free[kEach];
        int mine = 0;
        const int own = p0 + t / 64 * (64 * kEach) + lane;
        int ref[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) ref[i] = own + 64 * i < a.pages ? a.refs[own + 64 * i] : 1;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            free[i] = __ballot(ref[i] == 0);
            mine += __popcll(free[i]);
        }
        __syncthreads();
        if (lane == 0) sums[t / 64] = mine;
        __syncthreads();
        int at = found;
        for (int w = 0; w < kPlanWaves; ++w) {
            at += w < t / 64 ? sums[w] : 0;
            found += sums[w];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int k = at + __popcll(free[i] & ((uint64_t(1) << lane) - 1));
            if (ref[i] == 0 && k < demand) a.free_list[k] = own + 64 * i;
            at += __popcll(free[i]);
        }
    }
    if (demand > found) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (t + i * kPlanThreads < a.seqs) turn[t + i * kPlanThreads] = need[i];
        __syncthreads();
        if (t < 64) serve_in_turn(turn, a.seqs, found);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (t + i * kPlanThreads < a.seqs) base[i] = turn[t + i * kPlanThreads];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = t + i * kPlanThreads;
        if (s >= a.seqs) continue;
        a.record[s].base = base[i];
        a.evicted[s] = !r[i].cut ? 0 : base[i] < 0 ? -1 : r[i].m - r[i].n;
    }
}

// ---------------------------------------------------------------------------
// Then: keys and values that fill holes, and those of replaced pages that
// stay where they are.  `parts` workgroups a (sequence, layer, head).
//
// Bound by the bytes that move, each read and written once, and below some 20 MB by the
// chain of loads that leads to them: 10 to 11 us for 4000 rows of 8 heads or 24 of 32 sequences,
// 32 us for 20000 rows of 6 heads, 38 MB (with a quarter of the workgroups and a branch at each load 53).
constexpr int kMoveThreads = 256;

// A thread's part of the rows that move: 16 bytes of a row's keys or values, always the
// same, and every how many-th row.
struct Lane {
    int first, step;  // row, rows at once
    int side, byte;
    bool on;

    __device__ __forceinline__ explicit Lane(int row_bytes, int threads) {
        const int each = row_bytes / 8;  // pieces of keys and values
        step = threads / each;
        first = (int)threadIdx.x / each;
        const int in = (int)threadIdx.x - first * each;
        side = in >= each / 2;
        byte = (in - side * (each / 2)) * 16;
        on = first < step;
    }
};

__device__ void move_unit(const EvictArgs& a, const EvictRecord& r, int s, int lh, int part) {
    const int layer = lh / a.heads, head = lh - layer * a.heads, set = a.sets > 1 ? lh : 0, page = 1 << a.log_page;
    const Lane l(a.row_bytes, kMoveThreads);
    const int32_t* const list = a.list + a.sums(s, set) * a.positions;
    const int32_t* const old_page = a.old_page + (int64_t)s * a.max_pages;
    const int holes = a.holes[a.sums(s, set)];
    if (!r.gaps && (a.sets > 1 || lh == 0)) {  // the sums, once a set
        float* const w = a.weight + a.sums(s, set) * a.positions;
        for (int64_t e = (int64_t)part * kMoveThreads + threadIdx.x; e < holes; e += (int64_t)a.parts * kMoveThreads)
            w[list[e]] = w[list[a.positions - 1 - e]];
    }
    if (!l.on) return;
    constexpr int kAtOnce = 4;
    for (int64_t e0 = part * l.step + l.first; e0 < holes; e0 += (int64_t)a.parts * l.step * kAtOnce) {
        u32x4 x[kAtOnce];
        uint8_t* to[kAtOnce];
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            int64_t e = e0 + (int64_t)y * a.parts * l.step;
            e = e < holes ? e : holes - 1;  // (loads without branches; what is too much is not stored)
            const int from = list[a.positions - 1 - e], hole = list[e];
            x[y] = *reinterpret_cast<const u32x4*>(a.row_of(old_page[from >> a.log_page], layer, l.side, head, from) + l.byte);
            to[y] = a.row_of(a.page_now(r, s, hole >> a.log_page), layer, l.side, head, hole) + l.byte;
        }
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y)
            if (e0 + (int64_t)y * a.parts * l.step < holes) *reinterpret_cast<u32x4*>(to[y]) = x[y];
    }
    if (r.demand == 0) return;
    const uint64_t* const bits = a.hole_bits + a.sums(s, set) * a.words;
    for (int d = part; (d << a.log_page) < r.border; d += a.parts) {
        if (a.fresh[(int64_t)s * a.max_pages + d] < 0) continue;
        const int now = a.page_now(r, s, d), was = old_page[d], p0 = d << a.log_page;
        const int p1 = p0 + page < r.border ? p0 + page : r.border;
        for (int p = p0 + l.first; p < p1; p += l.step) {
            if ((bits[p / 64] >> (p & 63)) & 1) continue;
            *reinterpret_cast<u32x4*>(a.row_of(now, layer, l.side, head, p) + l.byte) =
                *reinterpret_cast<const u32x4*>(a.row_of(was, layer, l.side, head, p) + l.byte);
        }
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a) {
    const int s = (int)blockIdx.y;
    const EvictRecord r = a.record[s];
    if (!r.cut || r.base < 0) return;
    for (int i = (int)blockIdx.x; i < a.layers * a.heads * a.parts; i += (int)gridDim.x) {
        const int lh = i / a.parts;
        move_unit(a, r, s, lh, i - lh * a.parts);
    }
}

// ---------------------------------------------------------------------------
// Last launch, what the moves had to be ahead of: the last tokens shift; the sums of
// weights move; table, counts and lengths.  Where the last tokens shift by less than their
// number, one workgroup a (sequence, layer, head) reads ahead of where it writes; else
// `end_parts` of them share the rows.  The sums' tail becomes zeros, by `end_parts` workgroups
// too; so are the tokens' sources and the table.  Bound by latency as well: 14 us for 32
// sequences, 6 for 131k places of 8 heads or one sequence of 20000 pages.  Many last tokens that
// shift by few take their steps one after the other, 32 tokens of 128 channels each: whole calls
// that let 24 of 16408 tokens go, 4 layers of 8 heads, 55 us with 64 last ones, 147 with 2000 and
// 426 with 8192; of 32 such sequences 78, 478 and 1686.
constexpr int kEndThreads = 256;

__device__ void shift_recent(const EvictArgs& a, const EvictRecord& r, int s, int layer, int head, int part) {
    const int by = r.m - r.n, parts = by >= r.n - r.border ? a.end_parts : 1;
    if (part >= parts) return;
    const Lane l(a.row_bytes, kEndThreads);
    const int32_t* const old_page = a.old_page + (int64_t)s * a.max_pages;
    constexpr int kAtOnce = 4;
    for (int64_t p0 = r.border + (int64_t)part * l.step * kAtOnce; p0 < r.n; p0 += (int64_t)parts * l.step * kAtOnce) {
        u32x4 x[kAtOnce];
        uint8_t* to[kAtOnce];
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            const int64_t at = p0 + y * l.step + l.first;
            const int p = at < r.n ? (int)at : r.n - 1, from = p + by;  // (as above)
            x[y] = *reinterpret_cast<const u32x4*>(a.row_of(old_page[from >> a.log_page], layer, l.side, head, from) + l.byte);
            to[y] = a.row_of(a.page_now(r, s, p >> a.log_page), layer, l.side, head, p) + l.byte;
        }
        __syncthreads();  // (a token's place may be the source of an earlier one's)
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y)
            if (l.on && p0 + y * l.step + l.first < r.n) *reinterpret_cast<u32x4*>(to[y]) = x[y];
    }
}

// w[to + i] = w[at(i)], i < n, where no at(i) lies before to + i, or before an at of a smaller i.
template <class At>
__device__ __forceinline__ void shift_sums(float* w, int to, int n, At at) {
    constexpr int kAtOnce = 4;
    for (int i0 = 0; i0 < n; i0 += kEndThreads * kAtOnce) {
        float x[kAtOnce];
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            const int i = i0 + y * kEndThreads + (int)threadIdx.x;
            if (i < n) x[y] = w[at(i)];
        }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            const int i = i0 + y * kEndThreads + (int)threadIdx.x;
            if (i < n) w[to + i] = x[y];
        }
    }
    __syncthreads();
}

__device__ void move_sums(const EvictArgs& a, const EvictRecord& r, int s, int set) {
    const int t = (int)threadIdx.x;
    const int64_t of = a.sums(s, set) * a.positions;
    float* const w = a.weight + of;
    const int32_t* const list = a.list + of;
    const int holes = a.holes[a.sums(s, set)], by = r.m - r.n;
    if (r.gaps) {  // (else the move kernel has filled the holes)
        shift_sums(w, 0, r.m, [&](int i) { return a.position(r, s, i); });
        for (int e = t; e < holes; e += kEndThreads) w[list[e]] = w[list[a.positions - 1 - e]];
        __syncthreads();
    }
    shift_sums(w, r.border, r.n - r.border, [&](int i) { return r.border + by + i; });
    // (the last tokens' former places; with gaps, all from n on)
    for (int p = (r.gaps || r.m - (r.n - r.border) < r.n ? r.n : r.m - (r.n - r.border)) + t; p < r.length; p += kEndThreads) w[p] = 0.0f;
}

// Where the tokens were, and zeros between the cut and the last ones' former places: what was
// there has moved.
__device__ void clear_sums(const EvictArgs& a, const EvictRecord& r, int s, int set, int part) {
    if (a.source) {
        int32_t* const source = a.source + a.sums(s, set) * a.positions;
        const int32_t* const list = a.list + a.sums(s, set) * a.positions;
        const uint64_t* const bits = a.hole_bits + a.sums(s, set) * a.words;
        const int first = part * kEndThreads + (int)threadIdx.x, step = a.end_parts * kEndThreads;
        for (int64_t p = first; p < r.n; p += step)
            if (p >= r.border || !((bits[p / 64] >> (p % 64)) & 1))
                source[p] = a.position(r, s, (int)p < r.border ? (int)p : (int)p + r.m - r.n);
        for (int64_t e = first; e < a.holes[a.sums(s, set)]; e += step) source[list[e]] = a.position(r, s, list[a.positions - 1 - e]);
    }
    if (r.gaps) return;  // (the one that moves the sums clears all of it)
    float* const w = a.weight + a.sums(s, set) * a.positions;
    const int end = r.m - (r.n - r.border);
    for (int64_t p = r.n + (int64_t)part * kEndThreads + threadIdx.x; p < end; p += (int64_t)a.end_parts * kEndThreads) w[p] = 0.0f;
}

__device__ void enter_pages(const EvictArgs& a, const EvictRecord& r, int s, int part) {
    const int page = 1 << a.log_page;
    const int used = (r.n + page - 1) >> a.log_page, before = (r.length + page - 1) >> a.log_page;
    int32_t* const row = a.table + (int64_t)s * a.max_pages;
    for (int64_t d = part * kEndThreads + (int)threadIdx.x; d < before; d += a.end_parts * kEndThreads) {
        const int64_t at = (int64_t)s * a.max_pages + d;
        int now = -1;
        if (d < r.pages) {
            const int was = a.old_page[at];
            now = d < used ? a.page_now(r, s, (int)d) : -1;
            if (now != was) atomicAdd(a.refs + was, -1);
            if (now >= 0 && now != was) a.refs[now] = 1;
        }
        row[d] = now;
    }
    if (part == 0 && threadIdx.x == 0) a.lengths[s] = r.n;
}

__global__ __launch_bounds__(kEndThreads) void evict_end_kernel(EvictArgs a) {
    const int s = (int)blockIdx.y, units = a.layers * a.heads * a.end_parts, clears = a.sets * a.end_parts;
    const EvictRecord r = a.record[s];
    if (!r.cut || r.base < 0) return;
    for (int i = (int)blockIdx.x; i < units + clears + a.sets + a.end_parts; i += (int)gridDim.x) {
        if (i < units) {
            const int unit = i / a.end_parts;
            shift_recent(a, r, s, unit / a.heads, unit % a.heads, i - unit * a.end_parts);
        } else if (i < units + clears) {
            const int set = (i - units) / a.end_parts;
            clear_sums(a, r, s, set, i - units - set * a.end_parts);
        } else if (i < units + clears + a.sets) {
            move_sums(a, r, s, i - units - clears);
        } else {
            enter_pages(a, r, s, i - units - clears - a.sets);
        }
    }
}

// ---------------------------------------------------------------------------
// Host side

uint64_t up256(uint64_t v) { return (v + 255u) & ~uint64_t(255); }

bool evict_valid(const rac_cache_config* c, const rac_evict_config* e) {
    return cache_valid(c) && e && sets_valid(c, e->sets) && e->first >= 0 && e->first <= (1 << 30) && e->recent >= 0 &&
           e->recent <= (1 << 30);
}

// From this many chunks on, workgroups share a sequence, up to one for a compute unit (with
// two of them 64 sequences of 32768 places took 80 us instead of 62).  Whole calls of one
// layer and head, one workgroup a sequence and shared: 4 sequences of 16384 places 48 and 52 us,
// of 32768 67 and 54, of 131072 180 and 63; 64 of 32768 69 and 62, of 131072 193 and 111;
// 120 of 32768 71 and 76, of 131072 206 and 159.
constexpr int64_t kSplitChunks = 8;

// The scratch, in order; returns its bytes.
uint64_t lay_out(const rac_cache_config* c, EvictArgs& a, uint8_t* ws) {
    uint64_t at = 0;
    const auto take = [&](auto*& p, uint64_t count) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(ws + at);
        at += up256(count * sizeof(*p));
    };
    const uint64_t sums = (uint64_t)c->seqs * a.sets, entries = (uint64_t)c->seqs * c->max_pages;
    take(a.record, c->seqs);
    take(a.old_page, entries);
    take(a.old_at, entries);
    take(a.fresh, entries);
    take(a.free_list, c->pages);
    take(a.list, sums * a.positions);
    take(a.holes, sums);
    take(a.hole_bits, sums * a.words);
    take(a.digits, a.split > 1 ? sums * 3 * kDigit : 0);
    take(a.tally, a.split > 1 ? sums * a.split * 4 : 0);
    take(a.chosen, a.split > 1 ? sums : 0);
    return at;
}

EvictArgs args_of(const rac_cache_config* c, const rac_evict_config* e) {
    EvictArgs a{};
    a.positions = (int64_t)c->max_pages * c->page_tokens;
    a.words = (a.positions + 63) / 64;
    a.sets = e->sets;
    const int64_t units = (int64_t)c->seqs * a.sets, chunks = (a.positions + kChunk - 1) / kChunk;
    int64_t split = 256 / units;
    split = chunks < kSplitChunks || split < 2 ? 1 : split < chunks ? split : chunks;
    a.part = (int32_t)((chunks + split - 1) / split) * kChunk;
    a.split = (int32_t)((a.positions + a.part - 1) / a.part);
    return a;
}

// A row of workgroups for every sequence.
rac_status launch(void (*kernel)(EvictArgs), int64_t each, int64_t seqs, int threads, EvictArgs a, hipStream_t st) {
    void* p[] = {&a};
    const int64_t most = (1 << 20) / seqs;  // (they go on with further work)
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)(each < most ? each : most), (unsigned)seqs), dim3((unsigned)threads), p, 0, st) ==
                   hipSuccess
               ? RAC_OK
               : RAC_ERR_HIP;
}

}  // namespace

extern "C" {

size_t rac_cache_evict_workspace(const rac_cache_config* cfg, const rac_evict_config* evict) {
    if (!evict_valid(cfg, evict) || !sums_counted(cfg, evict->sets)) return 0;
    EvictArgs a = args_of(cfg, evict);
    return (size_t)lay_out(cfg, a, nullptr);
}

rac_status rac_cache_evict(const rac_cache_config* cfg, const rac_evict_config* evict, void* pool, int32_t* table,
                           int32_t* lengths, int32_t* refs, float* weight, const int32_t* keep, int32_t* evicted,
                           int32_t* source, void* workspace, size_t workspace_bytes, rac_stream_t stream) {
    if (!evict_valid(cfg, evict) || !pool || !table || !lengths || !refs || !weight || !keep || !evicted || !workspace)
        return RAC_ERR_INVALID;
    if (!aligned(pool, 16) || !aligned(table, 4) || !aligned(lengths, 4) || !aligned(refs, 4) || !aligned(weight, 4) ||
        !aligned(keep, 4) || !aligned(evicted, 4) || !aligned(source, 4) || !aligned(workspace, 256))
        return RAC_ERR_ALIGN;
    if (!sums_counted(cfg, evict->sets)) return RAC_ERR_UNSUPPORTED;
    if (workspace_bytes < rac_cache_evict_workspace(cfg, evict)) return RAC_ERR_CAPACITY;
    EvictArgs a = args_of(cfg, evict);
    lay_out(cfg, a, static_cast<uint8_t*>(workspace));
    a.pool = static_cast<uint8_t*>(pool);
    a.table = table;
    a.lengths = lengths;
    a.refs = refs;
    a.weight = weight;
    a.keep = keep;
    a.evicted = evicted;
    a.source = source;
    a.layers = cfg->layers;
    a.heads = cfg->kv_heads;
    a.row_bytes = cfg->head_dim * cache_elem_bytes(cfg);
    a.log_page = log2_of(cfg->page_tokens);
    a.pages = cfg->pages;
    a.seqs = cfg->seqs;
    a.max_pages = cfg->max_pages;
    a.first = evict->first;
    a.recent = evict->recent;
    // (a few workgroups for every compute unit where the sequences and heads are few: a round of
    // 32 sequences 73 us, with four times as many 82; the cut of 131k places 79 us, with a quarter 82)
    const int64_t units = (int64_t)cfg->layers * cfg->kv_heads, parts = 2048 / (units * cfg->seqs);
    a.parts = (int32_t)(parts < 1 ? 1 : parts > 256 ? 256 : parts);
    const int64_t ends = 256 / (units * cfg->seqs);
    a.end_parts = (int32_t)(ends < 1 ? 1 : ends > 32 ? 32 : ends);
    rac_status st;
    if (a.split == 1) {
        st = launch(evict_pick_kernel, evict->sets, cfg->seqs, kPickThreads, a, stream);
    } else {
        const int64_t each = (int64_t)evict->sets * a.split;
        st = launch(evict_see_kernel, evict->sets, cfg->seqs, kPickThreads, a, stream);
        for (; st == RAC_OK && a.digit < 3; ++a.digit) st = launch(evict_count_kernel, each, cfg->seqs, kPickThreads, a, stream);
        if (st == RAC_OK) st = launch(evict_tally_kernel, each, cfg->seqs, kPickThreads, a, stream);
        if (st == RAC_OK) st = launch(evict_order_kernel, each, cfg->seqs, kPickThreads, a, stream);
    }
    if (st == RAC_OK) st = launch(evict_demand_kernel, 1, cfg->seqs, kDemandThreads, a, stream);
    if (st == RAC_OK) st = launch(evict_plan_kernel, 1, 1, kPlanThreads, a, stream);
    if (st == RAC_OK) st = launch(evict_move_kernel, units * a.parts, cfg->seqs, kMoveThreads, a, stream);
    if (st == RAC_OK) st = launch(evict_end_kernel, (units + evict->sets + 1) * a.end_parts + evict->sets, cfg->seqs, kEndThreads, a, stream);
    return st;
}

}  // extern "C"
