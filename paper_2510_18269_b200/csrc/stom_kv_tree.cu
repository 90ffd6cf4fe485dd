// Attention of several new tokens per sequence over a paged cache (stom_kv_attend_tree).
#include "stom_kv.cuh"

#include <math.h>

namespace stom {

namespace {

struct KvTreeParams {
    const char *k, *v;            // at the layer
    int64_t stride_page, stride_token, stride_head;
    const int32_t *table;
    const int32_t *len;
    int64_t table_stride;
    int32_t n_seqs, n_pages, max_tokens;
    FastDiv page;
    int32_t n_kv_heads, group;    // query heads per kv head
    int32_t n_tokens;
    const int32_t *first, *parent;
    const char *q;
    int64_t q_stride_token, q_stride_head;
    float scale, cap;
    int32_t window;
    char *out;
    int64_t out_stride_token, out_stride_head;
    float *lse;
    uint32_t *flags;
};

// Node range of a sequence; false: skipped
__device__ __forceinline__ bool nodes_of(const KvTreeParams &p, int i, int &a, int &n, int &base) {
    a = p.first[i];
    const int b = p.first[i + 1], len = max(p.len[i], 0);
    n = b - a;
    base = len - n;
    return a >= 0 && a <= b && b <= p.n_tokens && n <= len && (!p.parent || n <= STOM_KV_MAX_TREE);
}

// One warp a (node, query head): a lane has a token at a time, then channels.
template <typename T, int D>
__global__ void __launch_bounds__(128) kv_tree_kernel(const __grid_constant__ KvTreeParams p) {
    __shared__ float qs[4][D];
    __shared__ uint32_t path[4][STOM_KV_MAX_TREE / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x, h = blockIdx.y * 4 + warp;
    const int heads = p.n_kv_heads * p.group;
    grid_dependency_wait();
    int a, n, base;
    if (!nodes_of(p, i, a, n, base)) {
        if (p.flags && threadIdx.x == 0) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
        return;
    }
    if (h >= heads) return;
    if (p.flags && lane == 0 && n > 0 && p.len[i] > p.max_tokens) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
    const int hk = h / p.group;
    for (int j = 0; j < n; ++j) {
        const T *q = reinterpret_cast<const T *>(p.q) + (a + j) * p.q_stride_token + h * p.q_stride_head;
        for (int c = lane; c < D; c += 32) qs[warp][c] = static_cast<float>(q[c]);
        for (int w = lane; w < STOM_KV_MAX_TREE / 32; w += 32) path[warp][w] = 0;
        __syncwarp();
        int depth = j;
        if (p.parent) {
            depth = 0;
            if (lane == 0)
                for (int c = j; c >= 0; ++depth) {
                    if (!p.window || depth < p.window) path[warp][c >> 5] |= 1u << (c & 31);
                    int up = p.parent[a + c];
                    if (up < -1 || up >= c) {
                        if (p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
                        up = -1;
                    }
                    c = up;
                }
            depth = __shfl_sync(~0u, depth, 0) - 1;
            __syncwarp();
        }
        const int end = min(base + j + 1, p.max_tokens);
        const int begin = p.window ? (int)max(0ll, (long long)base + depth + 1 - p.window) : 0;
        float m = -INFINITY, l = 0.f, o[D / 32];
        for (int c = 0; c < D / 32; ++c) o[c] = 0.f;
        for (int t0 = min(begin, base); t0 < end; t0 += 32) {
            const int t = t0 + lane;
            bool ok = t < end && (t >= base && p.parent ? path[warp][(t - base) >> 5] >> ((t - base) & 31) & 1u : t >= begin);
            int64_t off = 0;
            if (ok) {
                const int pg = (int)div_by(p.page, (uint32_t)t), id = p.table[i * p.table_stride + pg];
                if ((uint32_t)id >= (uint32_t)p.n_pages) {
                    ok = false;
                    if (p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
                } else {
                    off = 2 * (id * p.stride_page + (t - pg * (int)p.page.d) * p.stride_token + hk * p.stride_head);
                }
            }
            float x = -INFINITY;
            if (ok) {
                const T *k = reinterpret_cast<const T *>(p.k + off);
                float s = 0.f;
                for (int c = 0; c < D; ++c) s += qs[warp][c] * static_cast<float>(k[c]);
                x = s * p.scale;
                if (p.cap > 0.f) x = p.cap * tanhf(x / p.cap);
            }
            float top = x;
            for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
            const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn, alpha = expf(m - ref);
            const float w = ok ? expf(x - ref) : 0.f;
            m = mn;
            l = l * alpha + w;
            for (int c = 0; c < D / 32; ++c) o[c] *= alpha;
            for (int s = 0; s < 32; ++s) {
                const float ws = __shfl_sync(~0u, w, s);
                const bool is = __shfl_sync(~0u, ok, s);
                const int64_t at = __shfl_sync(~0u, off, s);
                if (!is) continue;
                const T *v = reinterpret_cast<const T *>(p.v + at);
                for (int c = 0; c < D / 32; ++c) o[c] += ws * static_cast<float>(v[c * 32 + lane]);
            }
        }
        for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(~0u, l, s);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T *dst = reinterpret_cast<T *>(p.out) + (a + j) * p.out_stride_token + h * p.out_stride_head;
        for (int c = 0; c < D / 32; ++c) dst[c * 32 + lane] = from_float<T>(o[c] * inv);
        if (p.lse && lane == 0) p.lse[(int64_t)(a + j) * heads + h] = l == 0.f ? -INFINITY : m + logf(l);
        __syncwarp();
    }
}

template <typename T>
int32_t dispatch(const KvTreeParams &p, int d, cudaStream_t s) {
    const dim3 grid(p.n_seqs, (p.n_kv_heads * p.group + 3) / 4), block(128);
    cudaError_t e = d == 64    ? launch_after_producer(kv_tree_kernel<T, 64>, grid, block, 0, s, p)
                    : d == 128 ? launch_after_producer(kv_tree_kernel<T, 128>, grid, block, 0, s, p)
                               : launch_after_producer(kv_tree_kernel<T, 256>, grid, block, 0, s, p);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int64_t stom_kv_attend_tree_workspace_bytes(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t n_tokens,
                                                       int32_t n_q_heads) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, false);
    if (rc) return rc;
    if (n_tokens < 0) return STOM_ERR_INVALID_ARG;
    if (n_q_heads < 1 || n_q_heads % pool->n_kv_heads) return STOM_ERR_SHAPE;
    return 256;
}

extern "C" int32_t stom_kv_attend_tree(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t layer, int32_t n_tokens,
                                       const int32_t *first, const int32_t *parent, int32_t n_q_heads, const void *q,
                                       int64_t q_stride_token, int64_t q_stride_head, float softmax_scale, float softcap,
                                       int32_t window, void *out, int64_t out_stride_token, int64_t out_stride_head,
                                       float *lse, void *workspace, int64_t workspace_bytes, uint32_t *dev_flags,
                                       void *stream) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, false);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->n_layers || n_q_heads < 1 || window < 0 || n_tokens < 0) return STOM_ERR_INVALID_ARG;
    // the factors that the kernel multiplies scores by have to be numbers, and one below binary32's normal ones lacks bits
    const float s1 = fabsf(softcap > 0.f ? softmax_scale / softcap : softmax_scale * 1.4426950408889634f);
    if (!(softcap >= 0.f) || !(softcap <= 2.0e38f) || !(s1 <= 3.0e38f) || (softcap > 0.f && s1 != 0.f && s1 < 1.2e-38f))
        return STOM_ERR_INVALID_ARG;
    if (n_q_heads % pool->n_kv_heads || n_q_heads / pool->n_kv_heads > 64) return STOM_ERR_SHAPE;
    if (seqs->n_seqs > STOM_KV_MAX_SEQS || (int64_t)n_tokens * n_q_heads > INT32_MAX) return STOM_ERR_SHAPE;
    const int64_t most = (int64_t)seqs->max_pages * pool->page_tokens;
    if (most > INT32_MAX - 32) return STOM_ERR_SHAPE;
    if (seqs->n_seqs == 0 || n_tokens == 0) return STOM_OK;
    if (!first || !q || !out) return STOM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(first) | reinterpret_cast<uintptr_t>(parent) | reinterpret_cast<uintptr_t>(lse)) & 3u)
        return STOM_ERR_ALIGNMENT;
    if (!aligned16(q) || !aligned16(out) || !stride_ok(q_stride_token, pool->dtype) || !stride_ok(q_stride_head, pool->dtype) ||
        !stride_ok(out_stride_token, pool->dtype) || !stride_ok(out_stride_head, pool->dtype))
        return STOM_ERR_ALIGNMENT;
    const int32_t d = pool->head_dim;
    if (n_q_heads > 1 && (out_stride_head < d || q_stride_head < 0)) return STOM_ERR_INVALID_ARG;
    if (n_tokens > 1 && (out_stride_token < d || q_stride_token < 0)) return STOM_ERR_INVALID_ARG;
    const int64_t need = stom_kv_attend_tree_workspace_bytes(pool, seqs, n_tokens, n_q_heads);
    if (!workspace || !aligned16(workspace) || workspace_bytes < need) return STOM_ERR_WORKSPACE;

    KvTreeParams p = {};
    p.k = static_cast<const char *>(pool->k) + 2 * layer * pool->stride_layer;
    p.v = static_cast<const char *>(pool->v) + 2 * layer * pool->stride_layer;
    p.stride_page = pool->stride_page;
    p.stride_token = pool->stride_token;
    p.stride_head = pool->stride_head;
    p.table = seqs->table;
    p.len = seqs->len;
    p.table_stride = seqs->table_stride;
    p.n_seqs = seqs->n_seqs;
    p.n_pages = pool->n_pages;
    p.max_tokens = (int32_t)most;
    p.page = fast_div((uint32_t)pool->page_tokens);
    p.n_kv_heads = pool->n_kv_heads;
    p.group = n_q_heads / pool->n_kv_heads;
    p.n_tokens = n_tokens;
    p.first = first;
    p.parent = parent;
    p.q = static_cast<const char *>(q);
    p.q_stride_token = q_stride_token;
    p.q_stride_head = q_stride_head;
    p.scale = softmax_scale;
    p.cap = softcap;
    p.window = window;
    p.out = static_cast<char *>(out);
    p.out_stride_token = out_stride_token;
    p.out_stride_head = out_stride_head;
    p.lse = lse;
    p.flags = dev_flags;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return pool->dtype == STOM_BF16 ? dispatch<__nv_bfloat16>(p, d, s) : dispatch<__half>(p, d, s);
}
