// tree.hip - gfx950 kernels and C ABI of the attention of drafted trees over
// the paged cache.  The contract is in include/rac_cache.h.
#include <math.h>

#include "cache_common.h"

namespace {

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
    float scale;    // of the scores
    float k_scale, v_scale;
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

// The sequence that query row `row` belongs to, or -1.
__device__ __forceinline__ int seq_of_row(const TreeArgs& a, int row) {
    int lo = 0, hi = a.seqs;  // the last s with q_start[s] <= row
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.q_start[mid] <= row) lo = mid; else hi = mid;
    }
    return lo;
}

template <int TYPE>
__device__ __forceinline__ float widen(const uint8_t* p, int i, bool page) {
    if (TYPE == RAC_CACHE_FP8 && page) return __builtin_amdgcn_cvt_f32_fp8((int)p[i], 0);
    const uint16_t b = reinterpret_cast<const uint16_t*>(p)[i];
    if (TYPE == RAC_CACHE_FP16) return (float)__builtin_bit_cast(_Float16, b);
    return __uint_as_float((uint32_t)b << 16);
}

template <int TYPE>
__device__ __forceinline__ uint16_t narrow(float v) {
    if (TYPE == RAC_CACHE_FP16) return __builtin_bit_cast(uint16_t, (_Float16)v);
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// One wavefront per (row, query head): a lane per key for the scores, a lane
// per channel for the values.
template <int TYPE>
__global__ __launch_bounds__(64) void tree_row_kernel(TreeArgs a) {
    __shared__ float qs[256], ps[64];
    __shared__ uint64_t at[64];
    const int hq = a.heads * a.group, lane = (int)threadIdx.x;
    const int row = (int)blockIdx.x / hq, h = (int)blockIdx.x % hq, kvh = h / a.group;
    const int s = seq_of_row(a, row);
    const Seq q = seq_of(a, s);
    const int i = row - q.q0;
    if (i < 0 || i >= q.m) return;
    const Sight see = sight_of(a, q, i);
    const uint64_t* words = a.mask ? a.mask + (size_t)row * a.mask_words : nullptr;
    for (int c = lane; c < a.dim; c += 64)
        qs[c] = widen<TYPE>(reinterpret_cast<const uint8_t*>(a.q + row * a.q_stride + (int64_t)h * a.dim), c, false) * a.scale;
    const int kb = TYPE == RAC_CACHE_FP8 ? 1 : 2;
    const uint64_t plane = ((uint64_t)a.dim << a.log_page) * kb;
    float top = -INFINITY, total = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int part = 0; part < 2; ++part) {  // committed, then drafted
        const int end = part ? see.end : q.length;
        for (int j0 = part ? see.first : see.from; j0 < end; j0 += 64) {
            const int j = j0 + lane;
            bool seen = j < end;
            const uint8_t *kp = nullptr, *vp = nullptr;
            if (seen && part == 0) {
                const int p = a.table[(size_t)s * a.max_pages + (j >> a.log_page)];
                seen = p >= 0 && p < a.pages;
                if (seen) {
                    const uint64_t b = (((uint64_t)p * a.layers + a.layer) * 2 * a.heads + kvh) * plane +
                                       (uint64_t)((j & ((1 << a.log_page) - 1)) * a.dim * kb);
                    kp = a.pool + b;
                    vp = kp + a.heads * plane;
                }
            } else if (seen) {
                seen = !words || ((words[j >> 6] >> (j & 63)) & 1);
                const int64_t o = (q.d0 + j) * a.kv_stride + (int64_t)kvh * a.dim;
                kp = reinterpret_cast<const uint8_t*>(a.k + o);
                vp = reinterpret_cast<const uint8_t*>(a.v + o);
            }
            float sc = 0.0f;
            __syncthreads();
            if (seen)
                for (int c = 0; c < a.dim; ++c) sc = __builtin_fmaf(qs[c], widen<TYPE>(kp, c, part == 0), sc);
            if (TYPE == RAC_CACHE_FP8 && part == 0) sc = sc * a.k_scale;
            const uint64_t live = __ballot(seen);
            float m = seen ? sc : -INFINITY;
            for (int o = 1; o < 64; o <<= 1) m = __builtin_fmaxf(m, __shfl_xor(m, o));
            m = __builtin_fmaxf(m, top);
            const float ref = m == -INFINITY ? 0.0f : m;
            const float p = seen ? __expf(sc - ref) : 0.0f, keep = __expf(top - ref);
            float sum = p;
            for (int o = 1; o < 64; o <<= 1) sum = sum + __shfl_xor(sum, o);
            total = __builtin_fmaf(total, keep, sum);
            top = m;
            ps[lane] = TYPE == RAC_CACHE_FP8 && part == 0 ? p * a.v_scale : p;
            at[lane] = reinterpret_cast<uint64_t>(vp);
            __syncthreads();
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int c = lane + 64 * x;
                if (c >= a.dim) break;
                float f = acc[x] * keep;
                for (uint64_t rest = live; rest; rest &= rest - 1) {
                    const int y = __builtin_ctzll(rest);
                    f = __builtin_fmaf(ps[y], widen<TYPE>(reinterpret_cast<const uint8_t*>(at[y]), c, part == 0), f);
                }
                acc[x] = f;
            }
        }
    }
    const bool none = total == 0.0f;
    for (int x = 0; x < 4; ++x) {
        const int c = lane + 64 * x;
        if (c < a.dim) a.out[row * a.out_stride + (int64_t)h * a.dim + c] = narrow<TYPE>(none ? 0.0f : acc[x] / total);
    }
    if (a.lse && lane == 0) a.lse[(size_t)row * hq + h] = none ? -INFINITY : top + logf(total);
}

// ---------------------------------------------------------------------------
// Host side

bool tree_valid(const rac_cache_config* c, const rac_tree_config* t) {
    return cache_valid(c) && t && t->q_heads >= 1 && t->q_heads % c->kv_heads == 0 && t->q_heads / c->kv_heads <= 64 &&
           t->rows >= 0 && t->rows <= (1 << 20) && t->max_rows >= 0 && t->max_draft >= 0 && t->window >= 0 &&
           t->scale >= 0.0f && t->scale < __builtin_inff();
}

}  // namespace

extern "C" {

size_t rac_tree_attention_workspace(const rac_cache_config* cfg, const rac_tree_config* tree) {
    return tree_valid(cfg, tree) ? 256 : 0;
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
    if (t->k && (t->kv_stride < kv_row || t->kv_stride % 8)) return RAC_ERR_INVALID;
    if ((t->mask != nullptr) != (t->mask_words > 0)) return RAC_ERR_INVALID;
    if (!aligned(pool, 16) || !aligned(t->q, 16) || !aligned(t->k, 16) || !aligned(t->v, 16) || !aligned(t->out, 16) ||
        !aligned(table, 4) || !aligned(lengths, 4) || !aligned(t->q_start, 4) || !aligned(t->draft_start, 4) ||
        !aligned(t->lse, 4) || !aligned(t->mask, 8) || !aligned(workspace, 256))
        return RAC_ERR_ALIGN;
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
    a.scale = tree->scale > 0.0f ? tree->scale : 1.0f / sqrtf((float)cfg->head_dim);
    a.k_scale = cfg->k_scale;
    a.v_scale = cfg->v_scale;
    const void* kernel = cfg->type == RAC_CACHE_BF16   ? reinterpret_cast<const void*>(tree_row_kernel<RAC_CACHE_BF16>)
                         : cfg->type == RAC_CACHE_FP16 ? reinterpret_cast<const void*>(tree_row_kernel<RAC_CACHE_FP16>)
                                                       : reinterpret_cast<const void*>(tree_row_kernel<RAC_CACHE_FP8>);
    if ((int64_t)tree->rows * tree->q_heads >= (int64_t(1) << 26)) return RAC_ERR_UNSUPPORTED;
    void* p[] = {&a};
    return hipLaunchKernel(kernel, dim3((unsigned)(tree->rows * tree->q_heads)), dim3(64), p, 0, stream) == hipSuccess
               ? RAC_OK
               : RAC_ERR_HIP;
}

}  // extern "C"
