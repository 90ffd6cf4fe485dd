// Rotary positions and per-head norms of new queries and keys, in place or on the way into pages (stom_kv_rotate,
// stom_kv_append).
//
//   y = x * weight / sqrt(mean x^2 + eps);   (a, b) -> (a cos - b sin, a sin + b cos),  angle = pos * freq
//
// What bounds it: every value is read and written once and takes part in a handful of operations, so memory, and for a
// decode step (a few kilobytes) the launch.  One pass, all loads and stores 16 bytes wide.  A row (one head of one token)
// belongs to d/16 adjacent threads; a thread owns the two 16-byte chunks that rotate with one another (half layout: the
// chunk and the one rot_dim/2 channels on; pairs: two adjacent chunks), so a rotation needs no exchange and a norm a few
// shuffles; with a norm, two values per instruction (f32x2).  A warp works on one token at a time, on several of its rows
// at once and on the others after them: its sines and cosines, and the norm's weights, are then the same for all its rows
// and stay in registers, and warps need no barrier.  A token with few companions is cut into parts, one warp each, down to
// one round of rows.
// Angles: pos * freq is formed and reduced to [-pi, pi] in binary64 (at position 10^6 a binary32 product would be off by
// 0.03 radians); the sine and cosine of the reduced angle are taken in binary32 with a first-order correction for the
// part of the angle that its rounding to binary32 lost.  Sine, cosine, the norm's sum and root and the turn are binary32,
// together within 2^-20 of the terms' magnitude: far below a half step of 16 bits, and of the order of binary32's own for
// binary32 rows (error against 64 bits 6.1e-8; with the angles' sines in binary64 and one rounding at the end 6.0e-8).
//
// Measured (B200, copy rate 6 458 GB/s): 12 583 tokens of 28 + 4 heads of 128, bf16: 37.2 us for 206 MB (5.5 TB/s); 4 099
// tokens of 64 + 8 heads with norms into pages, fp16: 34.5 us for 168 MB (4.9 TB/s, held back by the 16 warps that 124
// registers leave a multiprocessor); 1 771 tokens of 16 + 8 heads of 64 with norms, binary32: 7.4 us; one token: 2.9 us.
// A persistent form (equal stretches of rows per warp, loads eight steps ahead through shared memory) ran 37.6, 33.1, 8.9
// and 2.75 us: more on its way, but bound by its own instructions, and longer to start.
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
    RowSet set[3];              // queries, keys, values (values are only copied; src NULL: none)
    int32_t n_q, n_k, n_tokens;
    FastDiv parts;              // warps a token is cut into
    int32_t steps_per_part;     // of a warp's rows: first those of the keys and values, then those of the queries
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

// Two binary32 numbers in one 64-bit register: one instruction works on both
struct Pair {
    uint64_t v;
};
__device__ __forceinline__ Pair pair_of(float a, float b) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 split(Pair a) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(a.v));
    return f;
}
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Pair swapped(Pair a) {
    const float2 f = split(a);
    return pair_of(f.y, f.x);
}

// Eight adjacent values: as stored, and as pairs
template <typename T>
struct Chunk {
    uint4 v;
    __device__ __forceinline__ void load(const char *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(char *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    __device__ __forceinline__ void get(Pair (&f)[4]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float lo, hi;
            unpack2<T>(w[e], lo, hi);
            f[e] = pair_of(lo, hi);
        }
    }
    __device__ __forceinline__ void set(const Pair (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 x = split(f[e]);
            w[e] = pack2<T>(x.x, x.y);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Chunk<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const char *p) {
        a = reinterpret_cast<const float4 *>(p)[0];
        b = reinterpret_cast<const float4 *>(p)[1];
    }
    __device__ __forceinline__ void store(char *p) const {
        reinterpret_cast<float4 *>(p)[0] = a;
        reinterpret_cast<float4 *>(p)[1] = b;
    }
    __device__ __forceinline__ void get(Pair (&f)[4]) const {
        f[0] = pair_of(a.x, a.y);
        f[1] = pair_of(a.z, a.w);
        f[2] = pair_of(b.x, b.y);
        f[3] = pair_of(b.z, b.w);
    }
    __device__ __forceinline__ void set(const Pair (&f)[4]) {
        const float2 x0 = split(f[0]), x1 = split(f[1]), x2 = split(f[2]), x3 = split(f[3]);
        a = make_float4(x0.x, x0.y, x1.x, x1.y);
        b = make_float4(x2.x, x2.y, x3.x, x3.y);
    }
};

// The rows of one kind as a lane meets them, step by step
template <typename T, int D>
struct Walk {
    const char *src;
    char *dst;
    int64_t src_step, dst_step;   // bytes
    int left;                     // rows from this lane's next one on
    __device__ __forceinline__ Walk(const RowSet &s, int tok, int head, int n, int64_t dst_at, int rows) {
        const int64_t e = sizeof(T);
        src = s.src + e * (tok * s.src_token + head * s.src_head);
        dst = s.dst + e * (dst_at + head * s.dst_head);
        src_step = e * rows * s.src_head;
        dst_step = e * rows * s.dst_head;
        left = n - head;
    }
};

// PAIRS: channels 2i and 2i + 1 rotate with one another; otherwise i and i + rot_dim / 2.
template <typename T, int D, bool NORM, bool PAIRS>
__global__ void __launch_bounds__(kThreads, NORM ? 2 : 3) kv_rotate_kernel(const __grid_constant__ RotateParams p) {
    constexpr int kPerRow = D / 16;                 // threads of a row
    constexpr int kRows = 32 / kPerRow;             // rows of a warp's step
    constexpr int kE = sizeof(T);
    __shared__ float2 turn_smem[kThreads / 32][D / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float2 *turn = turn_smem[warp];                 // cosine and sine of the token's angles
    const uint32_t unit = blockIdx.x * (kThreads / 32) + warp;
    const int tok = (int)div_by(p.parts, unit), part = (int)(unit - tok * p.parts.d);
    if (tok >= p.n_tokens) return;
    const int t = lane % kPerRow, sub = lane / kPerRow, h2 = p.half >> 3;
    const bool turns = t < h2;
    const bool across = !PAIRS && turns;
    const int ca = (across ? t : 2 * t) * 8 * kE, cb = (across ? t + h2 : 2 * t + 1) * 8 * kE;

    // steps of this part: [s0, s1), those below kv_steps with keys and values
    const int kv_steps = (p.n_k + kRows - 1) / kRows, q_steps = (p.n_q + kRows - 1) / kRows;
    const int s0 = part * p.steps_per_part, s1 = min(s0 + p.steps_per_part, kv_steps + q_steps);
    const int k0 = min(s0, kv_steps), k1 = min(s1, kv_steps), q0 = max(s0, kv_steps) - kv_steps, q1 = max(s1, kv_steps) - kv_steps;

    grid_dependency_wait();

    // the token's place in the pool, in elements; -1: it is not stored
    int64_t place = tok * p.set[1].dst_token;
    if (p.table) {
        const int sl = p.slot[tok], sq = p.seq ? p.seq[tok] : tok;
        place = -1;
        if (sl != -1) {
            bool ok = (uint32_t)sl < (uint32_t)p.max_tokens && (uint32_t)sq < (uint32_t)p.n_seqs;
            if (ok) {
                const uint32_t pg = div_by(p.page, (uint32_t)sl);
                const int id = p.table[sq * p.table_stride + pg];
                ok = (uint32_t)id < (uint32_t)p.n_pages;
                if (ok) place = id * p.stride_page + (int64_t)(sl - pg * p.page.d) * p.stride_token;
            }
            if (!ok && p.flags && lane == 0) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
        }
    }
    // the first rows are on their way before the angles are worked out
    Walk<T, D> k(p.set[1], tok, k0 * kRows + sub, min(p.n_k, k1 * kRows), place, kRows);
    Walk<T, D> v(p.set[2], tok, k0 * kRows + sub, p.set[2].src ? min(p.n_k, k1 * kRows) : 0, place, kRows);
    Chunk<T> qa[2], qb[2], ka, kb, va, vb;
    auto fetch = [&](Walk<T, D> &w, Chunk<T> &a, Chunk<T> &b, int ahead) {
        if (w.left > ahead * kRows) {
            a.load(w.src + ahead * w.src_step + ca);
            b.load(w.src + ahead * w.src_step + cb);
        }
    };
    auto queries = [&]() {
        return Walk<T, D>(p.set[0], tok, q0 * kRows + sub, min(p.n_q, q1 * kRows), tok * p.set[0].dst_token, kRows);
    };
    fetch(k, ka, kb, 0);
    fetch(v, va, vb, 0);
    {
        Walk<T, D> q = queries();
        fetch(q, qa[0], qb[0], 0);
        fetch(q, qa[1], qb[1], 1);
    }

    for (int j = lane; j < p.half; j += 32) {
        const double angle = (double)p.pos[tok] * p.freq[j];
        const double n = rint(angle * 0.15915494309189535);
        double r = ::fma(-n, 6.283185307179586, angle);
        r = ::fma(-n, 2.4492935982947064e-16, r);   // what 2 pi has beyond its binary64 value
        const float rf = (float)r, rest = (float)(r - (double)rf);
        float s, c;
        sincosf(rf, &s, &c);
        turn[j] = make_float2(p.magnitude * fmaf(-rest, s, c), p.magnitude * fmaf(rest, c, s));
    }
    __syncwarp();

    // x' = x xx + (y, or x's neighbour) xy,  y' = y yy + (x, or y's neighbour) yx, four pairs each; with a norm its
    // weights are in the factors and the row's scale comes after them
    // (without a norm all of them follow from the cosines and sines, half the registers)
    Pair xx[NORM ? 4 : 1], xy[NORM ? 4 : 1], yx[NORM ? 4 : 1], yy[NORM ? 4 : 1];
    float2 cs[NORM ? 1 : 8];
    auto factors = [&](const float *weight) {
        if constexpr (!NORM) {
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = turns ? turn[t * 8 + e] : make_float2(1.f, 0.f);
        } else {
            float wx[8], wy[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) wx[e] = wy[e] = 1.f;
            if (weight) {
                const float *a = weight + ca / kE, *b = weight + cb / kE;
#pragma unroll
                for (int e = 0; e < 8; ++e) wx[e] = a[e], wy[e] = b[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (PAIRS) {
                    const float2 u = turns ? turn[t * 8 + e] : make_float2(1.f, 0.f);
                    const float2 w = turns ? turn[t * 8 + 4 + e] : make_float2(1.f, 0.f);
                    xx[e] = pair_of(wx[2 * e] * u.x, wx[2 * e + 1] * u.x);
                    xy[e] = pair_of(-wx[2 * e + 1] * u.y, wx[2 * e] * u.y);
                    yy[e] = pair_of(wy[2 * e] * w.x, wy[2 * e + 1] * w.x);
                    yx[e] = pair_of(-wy[2 * e + 1] * w.y, wy[2 * e] * w.y);
                } else {
                    const float2 u = turns ? turn[t * 8 + 2 * e] : make_float2(1.f, 0.f);
                    const float2 w = turns ? turn[t * 8 + 2 * e + 1] : make_float2(1.f, 0.f);
                    xx[e] = pair_of(wx[2 * e] * u.x, wx[2 * e + 1] * w.x);
                    xy[e] = pair_of(-wy[2 * e] * u.y, -wy[2 * e + 1] * w.y);
                    yy[e] = pair_of(wy[2 * e] * u.x, wy[2 * e + 1] * w.x);
                    yx[e] = pair_of(wx[2 * e] * u.y, wx[2 * e + 1] * w.y);
                }
            }
        }
    };
    // norm and rotation of the two chunks of a row; all lanes of the warp take part
    auto work = [&](Pair (&x)[4], Pair (&y)[4], bool norm) {
        if constexpr (!NORM) {
            if (!turns) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 a = split(x[e]), b = split(y[e]);
                if (PAIRS) {
                    const float2 u = cs[e], w = cs[4 + e];
                    x[e] = pair_of(a.x * u.x - a.y * u.y, a.x * u.y + a.y * u.x);
                    y[e] = pair_of(b.x * w.x - b.y * w.y, b.x * w.y + b.y * w.x);
                } else {
                    const float2 u = cs[2 * e], w = cs[2 * e + 1];
                    x[e] = pair_of(a.x * u.x - b.x * u.y, a.y * w.x - b.y * w.y);
                    y[e] = pair_of(a.x * u.y + b.x * u.x, a.y * w.y + b.y * w.x);
                }
            }
        } else {
            Pair scale = pair_of(1.f, 1.f);
            if (norm) {
                Pair sum = mul(x[0], x[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) sum = fma(x[e], x[e], sum);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = fma(y[e], y[e], sum);
                const float2 f = split(sum);
                float all = f.x + f.y;
#pragma unroll
                for (int o = 1; o < kPerRow; o <<= 1) all += __shfl_xor_sync(~0u, all, o);
                const float inv = rsqrtf(fmaf(all, 1.f / D, p.eps));
                scale = pair_of(inv, inv);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                Pair a = x[e], b = y[e];
                if (turns) {
                    const Pair xo = PAIRS ? swapped(a) : b, yo = PAIRS ? swapped(b) : a;
                    a = fma(xo, xy[e], mul(a, xx[e]));
                    b = fma(yo, yx[e], mul(b, yy[e]));
                } else {
                    a = mul(a, xx[e]);
                    b = mul(b, yy[e]);
                }
                x[e] = mul(a, scale);
                y[e] = mul(b, scale);
            }
        }
    };
    // one step of rows: takes the chunks, sends for the rows `ahead` steps on, works and stores
    auto step = [&](Walk<T, D> &w, Chunk<T> &a, Chunk<T> &b, int ahead, bool norm, bool stored) {
        Pair x[4], y[4];
        a.get(x);
        b.get(y);
        fetch(w, a, b, ahead);
        work(x, y, norm);
        if (w.left > 0 && stored) {
            Chunk<T> o;
            o.set(x);
            o.store(w.dst + ca);
            o.set(y);
            o.store(w.dst + cb);
        }
        w.src += w.src_step;
        w.dst += w.dst_step;
        w.left -= kRows;
    };

    const bool stored = place >= 0;
    if (k1 > k0) {
        factors(p.set[1].weight);
        for (int s = k0; s < k1; ++s) {
            const Chunk<T> ca_v = va, cb_v = vb;
            fetch(v, va, vb, 1);
            if (v.left > 0 && stored) {
                ca_v.store(v.dst + ca);
                cb_v.store(v.dst + cb);
            }
            v.src += v.src_step;
            v.dst += v.dst_step;
            v.left -= kRows;
            step(k, ka, kb, 1, p.set[1].weight != nullptr, stored);
        }
    }
    if (q1 > q0) {
        if (k1 == k0 || NORM) factors(p.set[0].weight);
        Walk<T, D> q = queries();
        for (int s = q0; s < q1; s += 2) {
            step(q, qa[0], qb[0], 2, p.set[0].weight != nullptr, true);
            if (s + 1 < q1) step(q, qa[1], qb[1], 2, p.set[0].weight != nullptr, true);
        }
    }
}

template <typename T, int D, bool NORM, bool PAIRS>
int32_t launch(RotateParams &p, int sms, cudaStream_t stream) {
    // Few tokens are cut into parts of whole steps, as long as all parts are on the device at once; a part works the
    // token's angles out again.
    constexpr int kRows = 32 / (D / 16);
    const int steps = (p.n_k + kRows - 1) / kRows + (p.n_q + kRows - 1) / kRows;
    int parts = 1;
    while (parts < steps && (int64_t)p.n_tokens * (parts + 1) <= (NORM ? 2 : 3) * (kThreads / 32) * sms) ++parts;
    p.steps_per_part = (steps + parts - 1) / parts;
    p.parts = fast_div((uint32_t)((steps + p.steps_per_part - 1) / p.steps_per_part));
    const int64_t warps = (int64_t)p.n_tokens * p.parts.d;
    const int blocks = (int)((warps + kThreads / 32 - 1) / (kThreads / 32));
    cudaError_t e = launch_after_producer(kv_rotate_kernel<T, D, NORM, PAIRS>, dim3(blocks), dim3(kThreads), 0, stream, p);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}

template <typename T, int D>
int32_t by_kind(RotateParams &p, int sms, cudaStream_t s) {
    const bool norm = p.set[0].weight || p.set[1].weight, pairs = p.layout == STOM_ROPE_PAIRS;
    if (norm) return pairs ? launch<T, D, true, true>(p, sms, s) : launch<T, D, true, false>(p, sms, s);
    return pairs ? launch<T, D, false, true>(p, sms, s) : launch<T, D, false, false>(p, sms, s);
}

template <typename T>
int32_t by_width(RotateParams &p, int d, int sms, cudaStream_t s) {
    return d == 64 ? by_kind<T, 64>(p, sms, s) : d == 128 ? by_kind<T, 128>(p, sms, s) : by_kind<T, 256>(p, sms, s);
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
    if (n > 0 && !q && !k) return STOM_ERR_INVALID_ARG;   // without a token no array needs to be there
    if ((q && (n_q < 1 || (n > 0 && !q_out))) || (k && n_k < 1)) return STOM_ERR_INVALID_ARG;
    if (rope->rot_dim && (!rope->freq || (n > 0 && !pos))) return STOM_ERR_INVALID_ARG;
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
    if (n_q > 65536 || n_k > 65536 || n > (1 << 30)) return STOM_ERR_SHAPE;
    p = RotateParams{};
    p.set[0] = RowSet{static_cast<const char *>(q), static_cast<char *>(q_out), q_tok, q_head, qo_tok, qo_head, q ? q_weight : nullptr};
    p.set[1] = RowSet{static_cast<const char *>(k), nullptr, k_tok, k_head, 0, 0, k ? k_weight : nullptr};
    p.n_q = n_q;
    p.n_k = n_k;
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
    const int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == STOM_BF16) return by_width<__nv_bfloat16>(p, d, sms, s);
    if (dtype == STOM_FP16) return by_width<__half>(p, d, sms, s);
    return by_width<float>(p, d, sms, s);
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
        if (!k_out && n_tokens > 0) return STOM_ERR_INVALID_ARG;
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
    if (layer < 0 || layer >= pool->n_layers || (n_tokens != 0 && (!k || !v))) return STOM_ERR_INVALID_ARG;
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
    if (!slot || !seqs->table || (!seq && n_tokens > seqs->n_seqs)) return STOM_ERR_INVALID_ARG;
    char *at_k = static_cast<char *>(pool->k) + 2 * layer * pool->stride_layer;
    char *at_v = static_cast<char *>(pool->v) + 2 * layer * pool->stride_layer;
    p.set[1].dst = at_k;
    p.set[1].dst_head = pool->stride_head;
    p.set[2] = RowSet{static_cast<const char *>(v), at_v, v_stride_token, v_stride_head, 0, pool->stride_head, nullptr};
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
