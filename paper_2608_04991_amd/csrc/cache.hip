// cache.hip - gfx950 kernels and C ABI of the paged key-value cache: forking,
// committing and copying pages.  The contract is in include/rac_cache.h.
//
// All bookkeeping (page tables, lengths, reference counts) stays on the device
// and gives the same pages whatever order the workgroups run in: counts change
// by commutative integer atomics, and pages are taken lowest number first.
#include "cache_common.h"

namespace {

// ---------------------------------------------------------------------------
// Fork.  A table entry only moves within its column, so a workgroup that owns
// whole columns can read all of them before it writes any, in place and in one
// launch: COLS columns of all sequences through LDS.  Lengths move within the
// last workgroup, which does nothing else.
//
// Bound by latency: entries, parents and bounds are dependent reads.  8 sequences of
// up to 250 tokens 2.0 us; 256 of up to 32000 (6 MB of table and counts) 7.9.
struct ForkArgs {
    const int32_t* parents;
    const int32_t* from;
    const int32_t* to;
    int32_t* table;
    int32_t* lengths;
    int32_t* refs;
    int32_t seqs, max_pages, pages, log_page;
};

constexpr int kForkThreads = 256;

// Adds to the count of a page; neighbouring sequences often hold the same one,
// so a thread adds up what it has for a page before it touches the count.
struct RefSum {
    int32_t* refs;
    int32_t pages, page, sum;
    __device__ __forceinline__ void add(int p, int by) {
        if (p != page) {
            flush();
            page = p;
        }
        sum += by;
    }
    __device__ __forceinline__ void flush() {
        if (sum != 0 && page >= 0 && page < pages) atomicAdd(refs + page, sum);
        sum = 0;
    }
};

template <int COLS>
__global__ __launch_bounds__(kForkThreads) void cache_fork_kernel(ForkArgs a) {
    extern __shared__ int32_t old[];  // [seqs][COLS]
    constexpr int kRows = kForkThreads / COLS;
    if (blockIdx.x == gridDim.x - 1) {
        for (int d = (int)threadIdx.x; d < a.seqs; d += kForkThreads) old[d] = a.lengths[d];
        __syncthreads();
        for (int d = (int)threadIdx.x; d < a.seqs; d += kForkThreads) {
            const int parent = a.parents[d];
            int n = parent >= 0 && parent < a.seqs ? old[parent] : 0;
            if (a.to && a.to[d] < n) n = a.to[d];
            a.lengths[d] = n < 0 ? 0 : n;
        }
        return;
    }
    const int c = (int)threadIdx.x % COLS, j = (int)blockIdx.x * COLS + c;
    const int each = (a.seqs + kRows - 1) / kRows;  // sequences a thread, one after the other
    const int d0 = (int)threadIdx.x / COLS * each, d1 = d0 + each < a.seqs ? d0 + each : a.seqs;
    const bool in = j < a.max_pages;
    int32_t* const column = a.table + j;
    // (what the call asks of a few sequences, read ahead of the stores between them)
    constexpr int kAtOnce = 8;
    int parent[kAtOnce], from[kAtOnce], to[kAtOnce];
    const auto ask = [&](int d) {
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            if (d + y >= d1) break;
            parent[y] = a.parents[d + y];
            from[y] = a.from ? a.from[d + y] : 0;
            to[y] = a.to ? a.to[d + y] : 0x7FFFFFFF;
        }
    };
    if (in) {
        ask(d0);
#pragma unroll 8
        for (int d = d0; d < d1; ++d) old[d * COLS + c] = column[(size_t)d * a.max_pages];
    }
    __syncthreads();
    if (!in) return;
    const int first = j << a.log_page, past = (j + 1) << a.log_page;
    RefSum less{a.refs, a.pages, -1, 0}, more{a.refs, a.pages, -1, 0};
    for (int d = d0; d < d1; d += kAtOnce) {
        if (d != d0) ask(d);
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            if (d + y >= d1) break;
            const int was = old[(d + y) * COLS + c];
            int now = parent[y] >= 0 && parent[y] < a.seqs ? old[parent[y] * COLS + c] : -1;
            if (first >= to[y] || past <= from[y]) now = -1;
            if (now < 0 || now >= a.pages) now = -1;
            if (now == was) continue;
            column[(size_t)(d + y) * a.max_pages] = now;
            less.add(was, -1);
            more.add(now, 1);
        }
    }
    less.flush();
    more.flush();
}

// ---------------------------------------------------------------------------
// Commit, first launch: one workgroup decides.  How many tokens and pages each
// sequence takes, which pages are free (a scan of the counts that ends when
// the demand is met), and the new table entries, counts and lengths.  The
// second launch moves the data by the records this one leaves.
//
// Bound by the latency of dependent reads (lengths, table, count, path) and of the
// sums over the workgroup: 7 us for 8 sequences, 12 for 128 with paths of up to 4
// nodes.  One thread enters a sequence's new pages, 0.12 us each (a prompt of 131k
// tokens in pages of 16: 1 ms).  Pages and the order of the sequences are those of a
// serial loop, so one workgroup has to see all of it.  Where there are pages enough, a
// sequence's place in them is the sum of the demands before it; where there are not,
// the loop itself finds it.
struct CommitRecord {
    int32_t length;      // before the call
    int32_t tokens;      // appended
    int32_t copy_from;   // the shared last page, or -1
    int32_t copy_to;
};

struct PlanArgs {
    int32_t* table;
    int32_t* lengths;
    int32_t* refs;
    const int32_t* start;
    const int32_t* path;
    int32_t* committed;
    CommitRecord* record;  // [seqs]
    int32_t* free_list;    // [pages]
    int32_t seqs, max_pages, pages, log_page, draft_rows, max_path;
};

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kNear = 4096;

// Rows of a sequence's drafts, whatever start[] holds.
__device__ __forceinline__ int2 row_range(const int32_t* start, int s, int rows) {
    const int lo = clamp_int(start[s], 0, rows), hi = clamp_int(start[s + 1], lo, rows);
    return make_int2(lo, hi - lo);
}

// How many of the first entries of a path name one of `drafted` rows.
__device__ __forceinline__ int path_length(const int32_t* p, int most, int drafted) {
    for (int n = 0;; n += 8) {
        int e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = n + i < most ? p[n + i] : -1;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e[i] < 0 || e[i] >= drafted) return n + i;
    }
}

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(PlanArgs a) {
    __shared__ int sums[kPlanWaves];
    __shared__ int32_t near[kNear];  // the first free pages (the others through memory)
    __shared__ int32_t turn[4 * kPlanThreads];
    const int t = (int)threadIdx.x, lane = t & 63, page = 1 << a.log_page;
    // A wavefront looks at 1024 pages a step, 64 at a time, in ascending order.
    constexpr int kEach = 16, kStep = kPlanThreads * kEach;
    const int own = t / 64 * (64 * kEach) + lane;
    int ref[kEach];
    auto look = [&](int p0) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) ref[i] = p0 + own + 64 * i < a.pages ? a.refs[p0 + own + 64 * i] : 1;
    };
    look(0);  // (on its way while the demand is counted)
    constexpr int kPer = 4;  // sequences a thread (4096 / 1024)
    int tokens[kPer], need[kPer], base[kPer], length[kPer], tail[kPer];
    bool copies[kPer], fresh[kPer];
    int demand = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = t + i * kPlanThreads;
        tokens[i] = need[i] = length[i] = base[i] = 0;
        tail[i] = -1;
        copies[i] = fresh[i] = false;
        if (i * kPlanThreads >= a.seqs) continue;
        if (s < a.seqs) {
            const int most = a.max_pages << a.log_page, len = clamp_int(a.lengths[s], 0, most);
            const int32_t* const row = a.table + (size_t)s * a.max_pages;
            const int drafted = row_range(a.start, s, a.draft_rows).y;
            if (len & (page - 1)) tail[i] = row[len >> a.log_page];
            if ((uint32_t)tail[i] >= (uint32_t)a.pages) tail[i] = -1;
            const bool shared = tail[i] >= 0 && a.refs[tail[i] < 0 ? 0 : tail[i]] > 1;
            const int n = a.path ? path_length(a.path + (size_t)s * a.max_path, a.max_path, drafted)
                                 : drafted < a.max_path ? drafted : a.max_path;
            length[i] = len;
            if (n > 0 && n <= most - len) {
                tokens[i] = n;
                need[i] = ((len + n + page - 1) >> a.log_page) - ((len + page - 1) >> a.log_page);
                if (len & (page - 1)) {
                    copies[i] = shared;
                    fresh[i] = shared || tail[i] < 0;
                    need[i] += fresh[i];
                }
                if (need[i] > a.pages) tokens[i] = need[i] = 0;
            }
        }
        int all;
        base[i] = (int)((uint32_t)demand + (uint32_t)scan_workgroup<kPlanWaves>(need[i], sums, &all));
        demand = all < kMostSum - demand ? demand + all : kMostSum;  // (more than any pool has)
    }
    // the free pages, lowest first, until the demand is met
    int found = 0;
    for (int p0 = 0; p0 < a.pages && found < demand; p0 += kStep) {
        if (p0) look(p0);
        uint64_t free[kEach];
        int mine = 0;
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
            if (ref[i] == 0 && k < demand) {
                if (k < kNear)
                    near[k] = p0 + own + 64 * i;
                else
                    a.free_list[k] = p0 + own + 64 * i;
            }
            at += __popcll(free[i]);
        }
    }
    __syncthreads();  // (the list is read by other threads of this workgroup)
    if (demand > found) {
        // (seldom: 27 us with it for 4096 sequences and no free page, 14 where none is asked for)
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
    const auto free_page = [&](int k) { return k < kNear ? near[k] : a.free_list[k]; };
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = t + i * kPlanThreads;
        if (s >= a.seqs) continue;
        CommitRecord r{length[i], tokens[i], -1, -1};
        if (base[i] < 0) r.tokens = 0;
        if (r.tokens > 0) {
            int32_t* row = a.table + (size_t)s * a.max_pages;
            int at = ((length[i] + page - 1) >> a.log_page) - (fresh[i] ? 1 : 0);
            for (int k = 0; k < need[i]; ++k, ++at) {
                const int p = free_page(base[i] + k);
                row[at] = p;
                a.refs[p] = 1;
            }
            if (copies[i]) {
                r.copy_from = tail[i];
                r.copy_to = free_page(base[i]);
                atomicAdd(a.refs + tail[i], -1);
            }
            a.lengths[s] = length[i] + r.tokens;
        }
        a.record[s] = r;
        a.committed[s] = r.tokens;
    }
}

// Second launch: `parts` workgroups per (sequence, layer), which take its tokens
// in turn; the first also copies the shared page.  Bound by bytes where there are
// many: 128 sequences, 8 layers of 8 heads of 128 channels to 8 bits, 64 MB with
// the copied pages, 14 us (4.5 TB/s); 8 sequences of one layer 4.6 us.
struct MoveArgs {
    uint8_t* pool;
    const int32_t* table;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* start;
    const int32_t* path;
    const CommitRecord* record;
    int64_t kv_stride, layer_stride;
    float k_scale, v_scale;
    int32_t layers, heads, dim, log_page, max_pages, pages, draft_rows, max_path, parts;
};

constexpr int kMoveThreads = 256;

// Eight bf16 as eight e4m3 of x / scale.
__device__ __forceinline__ u32x2 to_fp8(u32x4 x, float scale) {
    u32x2 o = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo = __uint_as_float(x[i] << 16) / scale, hi = __uint_as_float(x[i] & 0xFFFF0000u) / scale;
        // (a NaN stays one: neither comparison holds)
        lo = lo > 448.0f ? 448.0f : lo < -448.0f ? -448.0f : lo;
        hi = hi > 448.0f ? 448.0f : hi < -448.0f ? -448.0f : hi;
        if (i & 1)
            o[i >> 1] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, (int)o[i >> 1], true);
        else
            o[i >> 1] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, (int)o[i >> 1], false);
    }
    return o;
}

template <bool FP8>
__global__ __launch_bounds__(kMoveThreads) void cache_move_kernel(MoveArgs a) {
    const int part = (int)blockIdx.x % a.parts, sl = (int)blockIdx.x / a.parts;
    const int s = sl / a.layers, layer = sl % a.layers, t = (int)threadIdx.x;
    const CommitRecord r = a.record[s];
    if (r.tokens <= part) return;
    constexpr int kB = FP8 ? 1 : 2;
    const int page = 1 << a.log_page;
    const size_t plane = (size_t)page * a.dim * kB;         // keys or values of one head in a page
    const size_t side = plane * a.heads, whole = 2 * side;  // of all heads; of both
    auto at = [&](int p) { return a.pool + ((size_t)p * a.layers + layer) * whole; };
    if (part == 0 && r.copy_from >= 0) {
        const int per = (r.length & (page - 1)) * a.dim * kB / 16, all = per * 2 * a.heads;  // 16-byte pieces
        const uint8_t* from = at(r.copy_from);
        uint8_t* to = at(r.copy_to);
        constexpr int kAtOnce = 4;
        for (int i0 = t; i0 < all; i0 += kMoveThreads * kAtOnce) {
            u32x4 x[kAtOnce];
            size_t o[kAtOnce];
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const int i = i0 + y * kMoveThreads;
                o[y] = (size_t)(i / per) * plane + (size_t)(i % per) * 16;
                if (i < all) x[y] = *reinterpret_cast<const u32x4*>(from + o[y]);
            }
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y)
                if (i0 + y * kMoveThreads < all) *reinterpret_cast<u32x4*>(to + o[y]) = x[y];
        }
    }
    const int row0 = row_range(a.start, s, a.draft_rows).x;
    const int per = a.dim / 8, pieces = 2 * a.heads * per;  // of a token: (keys or values, head, eight channels)
    const int32_t* const path = a.path ? a.path + (size_t)s * a.max_path : nullptr;
    const int32_t* const row = a.table + (size_t)s * a.max_pages;
    for (int i = t; i < pieces; i += kMoveThreads) {
        const int c = i % per, h = i / per % a.heads, values = i / per / a.heads;
        const uint16_t* const from = (values ? a.v : a.k) + (size_t)layer * a.layer_stride + (size_t)h * a.dim + 8 * c;
        const size_t to = values * side + h * plane + 8 * c * kB;
        constexpr int kAtOnce = 4;  // tokens
        for (int n0 = part; n0 < r.tokens; n0 += kAtOnce * a.parts) {
            u32x4 x[kAtOnce];
            int p[kAtOnce];
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const int n = n0 + y * a.parts;
                if (n >= r.tokens) continue;
                const int node = path ? path[n] : n;
                p[y] = row[(r.length + n) >> a.log_page];
                x[y] = *reinterpret_cast<const u32x4*>(from + (size_t)(row0 + node) * a.kv_stride);
            }
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const int n = n0 + y * a.parts;
                if (n >= r.tokens || (uint32_t)p[y] >= (uint32_t)a.pages) continue;
                uint8_t* out = at(p[y]) + to + (size_t)((r.length + n) & (page - 1)) * a.dim * kB;
                if constexpr (FP8)
                    *reinterpret_cast<u32x2*>(out) = to_fp8(x[y], values ? a.v_scale : a.k_scale);
                else
                    *reinterpret_cast<u32x4*>(out) = x[y];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Copy: a workgroup per kCopyBytes of a page, four loads of 16 bytes a thread on
// their way before the first store.  Bound by bytes: 900 pages of 1 MiB, read and
// written, in 368 us (5.1 TB/s; a plain copy of 4 GB reaches 4.9); five of 32 KiB 3.0 us.
constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = kCopyThreads * 16 * 4;

struct CopyArgs {
    const uint8_t* from;
    uint8_t* to;
    const int32_t* src;
    const int32_t* dst;
    uint64_t page_bytes;
    int32_t pages, parts;
};

__global__ __launch_bounds__(kCopyThreads) void cache_copy_kernel(CopyArgs a) {
    const int i = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x % (unsigned)a.parts);
    const int s = a.src[i], d = a.dst[i];
    if (s < 0 || s >= a.pages || d < 0 || d >= a.pages) return;
    const uint64_t o = (uint64_t)part * kCopyBytes + 16u * threadIdx.x;
    const uint8_t* from = a.from + (uint64_t)s * a.page_bytes;
    uint8_t* to = a.to + (uint64_t)d * a.page_bytes;
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t at = o + 16u * kCopyThreads * k;
        if (at < a.page_bytes) x[k] = *reinterpret_cast<const u32x4*>(from + at);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t at = o + 16u * kCopyThreads * k;
        if (at < a.page_bytes) *reinterpret_cast<u32x4*>(to + at) = x[k];
    }
}

// ---------------------------------------------------------------------------
// Host side

uint64_t up256(uint64_t v) { return (v + 255u) & ~uint64_t(255); }

template <class A>
rac_status launch(const void* kernel, unsigned grid, unsigned threads, const A& args, size_t lds, hipStream_t st) {
    A a = args;
    void* p[] = {&a};
    return hipLaunchKernel(kernel, dim3(grid), dim3(threads), p, lds, st) == hipSuccess ? RAC_OK : RAC_ERR_HIP;
}

}  // namespace

extern "C" {

size_t rac_cache_pool_bytes(const rac_cache_config* cfg) {
    return cache_valid(cfg) ? (size_t)(cache_page_bytes(cfg) * (uint64_t)cfg->pages) : 0;
}

rac_status rac_cache_fork(const rac_cache_config* cfg, const int32_t* parents, const int32_t* keep_from,
                          const int32_t* keep_to, int32_t* table, int32_t* lengths, int32_t* refs,
                          rac_stream_t stream) {
    if (!cache_valid(cfg) || !parents || !table || !lengths || !refs) return RAC_ERR_INVALID;
    if (!aligned(parents, 4) || !aligned(keep_from, 4) || !aligned(keep_to, 4) || !aligned(table, 4) ||
        !aligned(lengths, 4) || !aligned(refs, 4))
        return RAC_ERR_ALIGN;
    const ForkArgs a{parents, keep_from, keep_to, table, lengths, refs, cfg->seqs, cfg->max_pages, cfg->pages,
                     log2_of(cfg->page_tokens)};
    // (64-byte pieces of the table's rows where 64 KiB of LDS hold that many columns)
    const int cols = cfg->seqs <= 1024 ? 16 : 4;
    const void* kernel = cols == 16 ? reinterpret_cast<const void*>(cache_fork_kernel<16>)
                                    : reinterpret_cast<const void*>(cache_fork_kernel<4>);
    return launch(kernel, (unsigned)((cfg->max_pages + cols - 1) / cols + 1), kForkThreads, a,
                  (size_t)cfg->seqs * cols * sizeof(int32_t), stream);
}

size_t rac_cache_commit_workspace(const rac_cache_config* cfg) {
    if (!cache_valid(cfg)) return 0;
    return (size_t)(up256((uint64_t)cfg->seqs * sizeof(CommitRecord)) + up256((uint64_t)cfg->pages * 4u));
}

rac_status rac_cache_commit(const rac_cache_config* cfg, void* pool, int32_t* table, int32_t* lengths, int32_t* refs,
                            const void* k, const void* v, int64_t kv_stride, int64_t layer_stride, int32_t draft_rows,
                            const int32_t* draft_start, const int32_t* path, int32_t max_path, int32_t* committed,
                            void* workspace, size_t workspace_bytes, rac_stream_t stream) {
    if (!cache_valid(cfg) || draft_rows < 0 || max_path < 0) return RAC_ERR_INVALID;
    const int64_t row = (int64_t)cfg->kv_heads * cfg->head_dim;
    if (kv_stride < row || kv_stride % 8 || layer_stride % 8 || layer_stride < 0) return RAC_ERR_INVALID;
    if (!pool || !table || !lengths || !refs || !draft_start || !committed || !workspace) return RAC_ERR_INVALID;
    if (draft_rows > 0 && (!k || !v)) return RAC_ERR_INVALID;
    if (!aligned(pool, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(workspace, 256) || !aligned(table, 4) ||
        !aligned(lengths, 4) || !aligned(refs, 4) || !aligned(draft_start, 4) || !aligned(path, 4) ||
        !aligned(committed, 4))
        return RAC_ERR_ALIGN;
    if (workspace_bytes < rac_cache_commit_workspace(cfg)) return RAC_ERR_CAPACITY;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    CommitRecord* record = reinterpret_cast<CommitRecord*>(ws);
    int32_t* list = reinterpret_cast<int32_t*>(ws + up256((uint64_t)cfg->seqs * sizeof(CommitRecord)));
    const int lp = log2_of(cfg->page_tokens);
    const PlanArgs plan{table, lengths, refs, draft_start, path, committed, record, list, cfg->seqs, cfg->max_pages,
                        cfg->pages, lp, draft_rows, max_path};
    rac_status st = launch(reinterpret_cast<const void*>(cache_plan_kernel), 1, kPlanThreads, plan, 0, stream);
    if (st != RAC_OK) return st;
    MoveArgs move{static_cast<uint8_t*>(pool), table, static_cast<const uint16_t*>(k),
                        static_cast<const uint16_t*>(v), draft_start, path, record, kv_stride, layer_stride,
                        cfg->k_scale, cfg->v_scale, cfg->layers, cfg->kv_heads, cfg->head_dim, lp, cfg->max_pages,
                        cfg->pages, draft_rows, max_path, 0};
    // (a workgroup per 8 of the longest path's tokens; the grid stays a million at most)
    const int64_t most = max_path < draft_rows ? max_path : draft_rows, units = (int64_t)cfg->seqs * cfg->layers;
    int64_t parts = (most + 7) / 8;
    if (parts * units > (1 << 20)) parts = (1 << 20) / units;
    move.parts = (int32_t)(parts < 1 ? 1 : parts);
    const void* kernel = cfg->type == RAC_CACHE_FP8 ? reinterpret_cast<const void*>(cache_move_kernel<true>)
                                                    : reinterpret_cast<const void*>(cache_move_kernel<false>);
    return launch(kernel, (unsigned)(units * move.parts), kMoveThreads, move, 0, stream);
}

rac_status rac_cache_copy(const rac_cache_config* cfg, const void* src_pool, const int32_t* src, void* dst_pool,
                          const int32_t* dst, int32_t n, rac_stream_t stream) {
    if (!cache_valid(cfg) || n < 0 || n > cfg->pages) return RAC_ERR_INVALID;
    if (n == 0) return RAC_OK;
    if (!src_pool || !src || !dst_pool || !dst) return RAC_ERR_INVALID;
    if (!aligned(src_pool, 16) || !aligned(dst_pool, 16) || !aligned(src, 4) || !aligned(dst, 4)) return RAC_ERR_ALIGN;
    const uint64_t bytes = cache_page_bytes(cfg), parts = (bytes + kCopyBytes - 1) / kCopyBytes;
    if (parts * (uint64_t)n * kCopyThreads >= (uint64_t(1) << 32)) return RAC_ERR_UNSUPPORTED;
    const CopyArgs a{static_cast<const uint8_t*>(src_pool), static_cast<uint8_t*>(dst_pool), src, dst, bytes,
                     cfg->pages, (int32_t)parts};
    return launch(reinterpret_cast<const void*>(cache_copy_kernel), (unsigned)(parts * (uint64_t)n), kCopyThreads, a, 0,
                  stream);
}

}  // extern "C"
