// Rotary positions and per-head norms of new queries and keys, in place or on the way into pages (stom_kv_rotate,
// stom_kv_append).
//
//   y = x * weight / sqrt(mean x^2 + eps);   (a, b) -> (a cos - b sin, a sin + b cos),  angle = pos * freq
//
// What bounds it: every value is read and written once and takes part in a handful of operations, so memory, and for a
// decode step (a few kilobytes) the launch.  One pass, all loads and stores 16 bytes wide.  A row (one head of one token)
// belongs to d/16 adjacent threads; a thread owns the two 16-byte chunks that rotate with one another (half layout: the
// chunk and the one rot_dim/2 channels on; pairs: two adjacent chunks), so a rotation needs no exchange and a norm a few
// shuffles.  The sines and cosines of a token are worked out once per block, in shared memory, and serve all its heads.
// Angles: pos * freq is formed and reduced to [-pi, pi] in binary64 (at position 10^6 a binary32 product would be off by
// 0.03 radians); the sine and cosine of the reduced angle are taken in binary32 with a first-order correction for the
// part of the angle that its rounding to binary32 lost.
#include "stom_kv.cuh"

namespace stom {

namespace {

constexpr int kThreads = 256;

struct RowSet {
    const char *src;
    char *dst;
    int64_t src_token, src_head, dst_token, dst_head;   // elements
    const float *weight;
};

struct RotateParams {
    RowSet set[3];              // queries, keys, values (values are only copied)
    int32_t first_k, first_v;   // rows of a token: [0, first_k) queries, [first_k, first_v) keys, then values
    FastDiv rows;
    int32_t n_tokens, tokens_per_block;
    const int32_t *pos;
    const double *freq;
    int32_t half;               // rotated pairs = rot_dim / 2
    int32_t layout;
    float magnitude, eps;
    // pages: keys and values go there (table == NULL: to set[1].dst with its strides)
    const int32_t *table;
    int64_t table_stride;
    const int32_t *slot, *seq;
    int32_t n_seqs, n_pages, max_tokens;
    FastDiv page;
    int64_t stride_page, stride_token;
    uint32_t *flags;
};

// Eight adjacent values as floats, and back
template <typename T>
struct Chunk {
    uint4 v;
    __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        unpack2<T>(v.x, f[0], f[1]);
        unpack2<T>(v.y, f[2], f[3]);
        unpack2<T>(v.z, f[4], f[5]);
        unpack2<T>(v.w, f[6], f[7]);
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        v = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
    }
};
template <>
struct Chunk<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const float4 *>(p)[0];
        b = reinterpret_cast<const float4 *>(p)[1];
    }
    __device__ __forceinline__ void store(float *p) const {
        reinterpret_cast<float4 *>(p)[0] = a;
        reinterpret_cast<float4 *>(p)[1] = b;
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv_rotate_kernel(const __grid_constant__ RotateParams p) {
    constexpr int kPerRow = D / 16;                 // threads of a row
    constexpr int kRowsAtOnce = kThreads / kPerRow;
    extern __shared__ __align__(16) float2 turn[];  // [tokens of the block][half]: cosine and sine
    __shared__ int64_t place[32];                   // of a token in the pool, in elements; -1: not stored

    const int token0 = blockIdx.x * p.tokens_per_block;
    const int tokens = min(p.tokens_per_block, p.n_tokens - token0);
    const int items = tokens * (int)p.rows.d;
    const int t = threadIdx.x % kPerRow, h2 = p.half >> 3;
    const bool turns = t < h2;
    int ca, cb;                                     // this thread's chunks of a row
    if (p.layout == STOM_ROPE_PAIRS) {
        ca = 2 * t;
        cb = 2 * t + 1;
    } else if (turns) {
        ca = t;
        cb = t + h2;
    } else {
        ca = 2 * t;                                 // 2 h2 + 2 (t - h2)
        cb = 2 * t + 1;
    }

    // item -> token of the block and row; the loads of one item are on their way while the one before is worked on
    struct Item {
        int tok, row, kind;                         // kind: 0 query, 1 key, 2 value, -1 none
    };
    auto item_at = [&](int i) {
        Item it;
        it.kind = -1;
        if (i < items) {
            it.tok = (int)div_by(p.rows, (uint32_t)i);
            it.row = i - it.tok * (int)p.rows.d;
            it.kind = it.row < p.first_k ? 0 : it.row < p.first_v ? 1 : 2;
            it.row -= it.kind == 0 ? 0 : it.kind == 1 ? p.first_k : p.first_v;
        }
        return it;
    };
    auto fetch = [&](const Item &it, Chunk<T> &a, Chunk<T> &b) {
        if (it.kind < 0) return;
        const RowSet &s = p.set[it.kind];
        const T *x = reinterpret_cast<const T *>(s.src) + (token0 + it.tok) * s.src_token + it.row * s.src_head;
        a.load(x + ca * 8);
        b.load(x + cb * 8);
    };

    grid_dependency_wait();
    int i = threadIdx.x / kPerRow;
    Item it = item_at(i);
    Chunk<T> a, b;
    fetch(it, a, b);

    for (int j = threadIdx.x; j < tokens * p.half; j += kThreads) {
        const int tok = j / p.half, pair = j - tok * p.half;
        const double angle = (double)p.pos[token0 + tok] * p.freq[pair];
        const double n = rint(angle * 0.15915494309189535);
        double r = fma(-n, 6.283185307179586, angle);
        r = fma(-n, 2.4492935982947064e-16, r);     // what 2 pi has beyond its binary64 value
        const float rf = (float)r, rest = (float)(r - (double)rf);
        float s, c;
        sincosf(rf, &s, &c);
        turn[j] = make_float2(p.magnitude * fmaf(-rest, s, c), p.magnitude * fmaf(rest, c, s));
    }
    if (p.table && threadIdx.x < tokens) {
        const int tok = token0 + threadIdx.x;
        const int sl = p.slot[tok], sq = p.seq ? p.seq[tok] : tok;
        int64_t at = -1;
        if (sl != -1) {
            bool ok = (uint32_t)sl < (uint32_t)p.max_tokens && (uint32_t)sq < (uint32_t)p.n_seqs;
            if (ok) {
                const uint32_t pg = div_by(p.page, (uint32_t)sl);
                const int id = p.table[sq * p.table_stride + pg];
                ok = (uint32_t)id < (uint32_t)p.n_pages;
                if (ok) at = id * p.stride_page + (int64_t)(sl - pg * p.page.d) * p.stride_token;
            }
            if (!ok && p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
        }
        place[threadIdx.x] = at;
    }
    __syncthreads();

    for (int round = 0; round < items; round += kRowsAtOnce) {   // the same number for every thread: shuffles below
        const int ahead = i + kRowsAtOnce;
        const Item next = item_at(ahead);
        Chunk<T> na, nb;
        fetch(next, na, nb);
        const RowSet &set = p.set[it.kind < 0 ? 0 : it.kind];
        const bool works = it.kind == 0 || it.kind == 1;
        float x[8], y[8];
        if (works) {
            a.get(x);
            b.get(y);
        }
        if (p.set[0].weight || p.set[1].weight) {
            float sum = 0.f;
            if (works)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += x[e] * x[e] + y[e] * y[e];
#pragma unroll
            for (int o = 1; o < kPerRow; o <<= 1) sum += __shfl_xor_sync(~0u, sum, o);
            if (works && set.weight) {
                const float inv = 1.f / sqrtf(sum * (1.f / D) + p.eps);
                const float4 *wa = reinterpret_cast<const float4 *>(set.weight + ca * 8);
                const float4 *wb = reinterpret_cast<const float4 *>(set.weight + cb * 8);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float4 u = wa[q], v = wb[q];
                    x[4 * q] *= inv * u.x; x[4 * q + 1] *= inv * u.y; x[4 * q + 2] *= inv * u.z; x[4 * q + 3] *= inv * u.w;
                    y[4 * q] *= inv * v.x; y[4 * q + 1] *= inv * v.y; y[4 * q + 2] *= inv * v.z; y[4 * q + 3] *= inv * v.w;
                }
            }
        }
        if (works) {
            if (turns) {
                const float2 *cs = turn + it.tok * p.half;
                if (p.layout == STOM_ROPE_PAIRS) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float2 u = cs[ca * 4 + (e >> 1)], v = cs[cb * 4 + (e >> 1)];
                        const float x0 = x[e], y0 = y[e];
                        x[e] = x0 * u.x - x[e + 1] * u.y;
                        x[e + 1] = x0 * u.y + x[e + 1] * u.x;
                        y[e] = y0 * v.x - y[e + 1] * v.y;
                        y[e + 1] = y0 * v.y + y[e + 1] * v.x;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 u = cs[t * 8 + e];
                        const float x0 = x[e];
                        x[e] = x0 * u.x - y[e] * u.y;
                        y[e] = x0 * u.y + y[e] * u.x;
                    }
                }
            }
            a.set(x);
            b.set(y);
        }
        if (it.kind >= 0) {
            int64_t at = it.kind > 0 && p.table ? place[it.tok] : (token0 + it.tok) * set.dst_token;
            if (at >= 0) {
                T *o = reinterpret_cast<T *>(set.dst) + at + it.row * set.dst_head;
                a.store(o + ca * 8);
                b.store(o + cb * 8);
            }
        }
        it = next;
        a = na;
        b = nb;
        i = ahead;
    }
}

template <typename T, int D>
int32_t launch(const RotateParams &p, cudaStream_t stream) {
    const size_t smem = (size_t)p.tokens_per_block * p.half * sizeof(float2);
    const int blocks = (p.n_tokens + p.tokens_per_block - 1) / p.tokens_per_block;
    cudaError_t e = launch_after_producer(kv_rotate_kernel<T, D>, dim3(blocks), dim3(kThreads), smem, stream, p);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}

template <typename T>
int32_t by_width(const RotateParams &p, int d, cudaStream_t s) {
    return d == 64 ? launch<T, 64>(p, s) : d == 128 ? launch<T, 128>(p, s) : launch<T, 256>(p, s);
}

// Common checks of both calls; fills all but the destination of keys and values.
int32_t prepare(RotateParams &p, const stom_kv_rope *rope, int32_t dtype, int32_t d, int32_t n, const int32_t *pos,
                const void *q, int32_t n_q, int64_t q_tok, int64_t q_head, void *q_out, int64_t qo_tok, int64_t qo_head,
                const float *q_weight, const void *k, int32_t n_k, int64_t k_tok, int64_t k_head, const float *k_weight,
                float eps) {
    if (!rope || n < 0) return STOM_ERR_INVALID_ARG;
    if (dtype != STOM_BF16 && dtype != STOM_FP16 && dtype != STOM_FP32) return STOM_ERR_UNSUPPORTED;
    if (rope->layout != STOM_ROPE_HALF && rope->layout != STOM_ROPE_PAIRS) return STOM_ERR_UNSUPPORTED;
    if (d != 64 && d != 128 && d != 256) return STOM_ERR_SHAPE;
    if (rope->rot_dim < 0 || rope->rot_dim > d || rope->rot_dim % 16) return STOM_ERR_SHAPE;
    if (!(eps >= 0.f) || !(eps < 3e38f) || !(rope->magnitude >= -3e38f && rope->magnitude <= 3e38f)) return STOM_ERR_INVALID_ARG;
    if (!q && !k) return STOM_ERR_INVALID_ARG;
    if ((q && (n_q < 1 || !q_out)) || (k && n_k < 1)) return STOM_ERR_INVALID_ARG;
    if (rope->rot_dim && (!rope->freq || !pos)) return STOM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(rope->freq) & 7u) || (reinterpret_cast<uintptr_t>(pos) & 3u)) return STOM_ERR_ALIGNMENT;
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(q_weight) || !aligned16(k_weight))
        return STOM_ERR_ALIGNMENT;
    if (q && (!stride_ok(q_tok, dtype) || !stride_ok(q_head, dtype) || !stride_ok(qo_tok, dtype) || !stride_ok(qo_head, dtype)))
        return STOM_ERR_ALIGNMENT;
    if (k && (!stride_ok(k_tok, dtype) || !stride_ok(k_head, dtype))) return STOM_ERR_ALIGNMENT;
    if (q && (q_tok < 0 || q_head < 0 || (n > 1 && qo_tok < d) || (n_q > 1 && qo_head < d) || qo_tok < 0 || qo_head < 0))
        return STOM_ERR_INVALID_ARG;
    if (k && (k_tok < 0 || k_head < 0)) return STOM_ERR_INVALID_ARG;
    if (!q) n_q = 0;
    if (!k) n_k = 0;
    if (n_q > 65536 || n_k > 65536) return STOM_ERR_SHAPE;
    p = RotateParams{};
    p.set[0] = RowSet{static_cast<const char *>(q), static_cast<char *>(q_out), q_tok, q_head, qo_tok, qo_head, q ? q_weight : nullptr};
    p.set[1] = RowSet{static_cast<const char *>(k), nullptr, k_tok, k_head, 0, 0, k ? k_weight : nullptr};
    p.first_k = n_q;
    p.first_v = n_q + n_k;
    p.rows = fast_div((uint32_t)(n_q + n_k));
    p.n_tokens = n;
    p.pos = pos;
    p.freq = rope->freq;
    p.half = rope->rot_dim / 2;
    p.layout = rope->layout;
    p.magnitude = rope->magnitude;
    p.eps = eps;
    return STOM_OK;
}

int32_t run(RotateParams &p, int32_t dtype, int32_t d, void *stream) {
    // One token per block while that leaves multiprocessors with fewer than four blocks; four after that, so that the
    // set-up of a block is shared by more rows.
    const int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    p.tokens_per_block = p.n_tokens >= 16 * sms ? 4 : 1;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == STOM_BF16) return by_width<__nv_bfloat16>(p, d, s);
    if (dtype == STOM_FP16) return by_width<__half>(p, d, s);
    return by_width<float>(p, d, s);
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int32_t stom_kv_rotate(const stom_kv_rope *rope, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                                  const int32_t *pos, const void *q, int32_t n_q_heads, int64_t q_stride_token,
                                  int64_t q_stride_head, void *q_out, int64_t q_out_stride_token,
                                  int64_t q_out_stride_head, const float *q_weight, const void *k, int32_t n_k_heads,
                                  int64_t k_stride_token, int64_t k_stride_head, void *k_out, int64_t k_out_stride_token,
                                  int64_t k_out_stride_head, const float *k_weight, float eps, void *stream) {
    RotateParams p;
    int32_t rc = prepare(p, rope, dtype, head_dim, n_tokens, pos, q, n_q_heads, q_stride_token, q_stride_head, q_out,
                         q_out_stride_token, q_out_stride_head, q_weight, k, n_k_heads, k_stride_token, k_stride_head,
                         k_weight, eps);
    if (rc) return rc;
    if (k) {
        if (!k_out) return STOM_ERR_INVALID_ARG;
        if (!aligned16(k_out) || !stride_ok(k_out_stride_token, dtype) || !stride_ok(k_out_stride_head, dtype)) return STOM_ERR_ALIGNMENT;
        if ((n_tokens > 1 && k_out_stride_token < head_dim) || (n_k_heads > 1 && k_out_stride_head < head_dim) ||
            k_out_stride_token < 0 || k_out_stride_head < 0)
            return STOM_ERR_INVALID_ARG;
        p.set[1].dst = static_cast<char *>(k_out);
        p.set[1].dst_token = k_out_stride_token;
        p.set[1].dst_head = k_out_stride_head;
    }
    if (n_tokens == 0) return STOM_OK;
    return run(p, dtype, head_dim, stream);
}

extern "C" int32_t stom_kv_append(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t layer,
                                  const stom_kv_rope *rope, int32_t n_tokens, const int32_t *pos, const int32_t *slot,
                                  const int32_t *seq, const void *q, int32_t n_q_heads, int64_t q_stride_token,
                                  int64_t q_stride_head, void *q_out, int64_t q_out_stride_token,
                                  int64_t q_out_stride_head, const float *q_weight, const void *k,
                                  int64_t k_stride_token, int64_t k_stride_head, const float *k_weight, const void *v,
                                  int64_t v_stride_token, int64_t v_stride_head, float eps, uint32_t *dev_flags,
                                  void *stream) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, false);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->n_layers || !k || !v) return STOM_ERR_INVALID_ARG;
    RotateParams p;
    rc = prepare(p, rope, pool->dtype, pool->head_dim, n_tokens, pos, q, n_q_heads, q_stride_token, q_stride_head, q_out,
                 q_out_stride_token, q_out_stride_head, q_weight, k, pool->n_kv_heads, k_stride_token, k_stride_head,
                 k_weight, eps);
    if (rc) return rc;
    if (!aligned16(v) || !stride_ok(v_stride_token, pool->dtype) || !stride_ok(v_stride_head, pool->dtype) ||
        ((reinterpret_cast<uintptr_t>(slot) | reinterpret_cast<uintptr_t>(seq)) & 3u))
        return STOM_ERR_ALIGNMENT;
    if (v_stride_token < 0 || v_stride_head < 0) return STOM_ERR_INVALID_ARG;
    if (n_tokens == 0) return STOM_OK;
    if (!slot || (!seq && n_tokens > seqs->n_seqs)) return STOM_ERR_INVALID_ARG;
    char *at_k = static_cast<char *>(pool->k) + 2 * layer * pool->stride_layer;
    char *at_v = static_cast<char *>(pool->v) + 2 * layer * pool->stride_layer;
    p.set[1].dst = at_k;
    p.set[1].dst_head = pool->stride_head;
    p.set[2] = RowSet{static_cast<const char *>(v), at_v, v_stride_token, v_stride_head, 0, pool->stride_head, nullptr};
    p.rows = fast_div((uint32_t)(p.first_v + pool->n_kv_heads));
    p.table = seqs->table;
    p.table_stride = seqs->table_stride;
    p.slot = slot;
    p.seq = seq;
    p.n_seqs = seqs->n_seqs;
    p.n_pages = pool->n_pages;
    const int64_t most = (int64_t)seqs->max_pages * pool->page_tokens;
    p.max_tokens = (int32_t)(most < INT32_MAX ? most : INT32_MAX);
    p.page = fast_div((uint32_t)pool->page_tokens);
    p.stride_page = pool->stride_page;
    p.stride_token = pool->stride_token;
    p.flags = dev_flags;
    return run(p, pool->dtype, pool->head_dim, stream);
}
