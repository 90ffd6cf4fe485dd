// Products of a few tokens with 4-bit weights (stom_w4_linear).
//
//   y[t][r] = sum_g ( s_rg sum_c code_rc x_tc + z_rg sum_c x_tc ) + bias_r + add_tr,   c over the columns of group g.
//
// What bounds it: the codes, half a byte a weight, are read once; at one token each takes part in one multiply-add, so
// that memory gives 46 weights a clock to a multiprocessor.  The scalar units would need as many multiply-adds and an
// unpacking for each; on the tensor cores (m16n8k16, the weights the 16 rows, the tokens the 8 columns) a warp-wide
// product takes 256 of them, and the unpacking is what is left to make short.
//
// Codes as numbers.  A code c put under the exponent of 1, at the top of the mantissa, is the 16-bit number 1 + c/16: one
// shift and one three-input logic operation turn two codes of a word into an operand register.  With D = sum (1 + c/16) x
// and X = sum x, both exact products summed in binary32, sum c x = 16 (D - X), so that a group adds 16 s D + (z - 16 s) X.
// X comes from a product of the same tokens with ones, in the very registers where D's tokens stand.  The difference
// costs at most a factor (16 + 15) / 7.5 of binary32's 2^-24, where the output has 2^-8 or 2^-11.
//
// Layout.  Codes are used as they lie in memory.  The order of columns within a product is free as long as weights and
// tokens agree, so lane (g, t) of a fragment takes group / 32 adjacent words of 8 codes of rows g and g + 8, and the
// tokens' eight values of the same columns; halves of a register hold columns 4 apart, as the nibbles of a word do.  All of
// a product's columns lie in one group.
//
// Split.  A block has 32 rows, its warps take groups in turn, and their sums are joined in shared memory.
#include "stom_internal.cuh"
#include "stom_kv.cuh"
#include "stom_w4.h"

#include <type_traits>

namespace stom {

namespace {

constexpr int kRows = 32;     // of the matrix, per block
constexpr int kWarps = 8;
constexpr int kStages = 4;
constexpr int kPitch = 80;    // bytes from row to row of a stage in shared memory: 8 rows' words of 4 lanes lie in 32 banks
constexpr int kStageBytes = kRows * kPitch;

struct W4Params {
    const uint8_t *codes;
    const void *scale, *zero;
    int32_t n, k, groups, meta_dtype;
    int64_t code_stride, meta_stride;
    const void *x;
    int64_t x_stride;
    const void *bias, *add;
    int64_t add_stride;
    void *y;
    int64_t y_stride;
    int32_t tokens;
};

// Two codes of a word (nibbles SH / 4 and SH / 4 + 4) as the numbers 1 + c/16
template <typename T, int NIB>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
    constexpr bool bf = std::is_same<T, __nv_bfloat16>::value;
    constexpr int top = bf ? 3 : 6;          // where the four highest bits of the mantissa begin
    constexpr uint32_t one = bf ? 0x3f803f80u : 0x3c003c00u, mask = 0x000f000fu << top;
    constexpr int shift = top - 4 * NIB;
    const uint32_t at = shift >= 0 ? w << (shift >= 0 ? shift : 0) : w >> (shift >= 0 ? 0 : -shift);
    return (at & mask) | one;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

// c (16x8) = a (16x16) b (16x8): the first product of a sum
template <typename T>
__device__ __forceinline__ void mma16x8x16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// GROUP columns a group; NT blocks of 8 tokens.
// A warp goes through stages of 128 columns (the block's warps take them in turn): 64 bytes of each of its 32 rows, copied
// to its own ring in shared memory kStages - 1 stages ahead; the tokens' values and the rows' scales a stage ahead in
// registers.  No barrier but the one before the warps' sums are joined.
template <typename T, typename M, int GROUP, int NT>
__global__ void __launch_bounds__(kWarps * 32, 2) w4_few_kernel(const __grid_constant__ W4Params p) {
    constexpr int kGroups = 128 / GROUP;             // of a stage
    constexpr uint32_t ones = std::is_same<T, __nv_bfloat16>::value ? 0x3f803f80u : 0x3c003c00u;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float2 meta_s[kWarps][2][kGroups][kRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int row0 = blockIdx.x * kRows, tok0 = blockIdx.y * 8 * NT;
    const int stages = (p.k + 127) / 128;
    const int mine = warp < stages ? (stages - warp + kWarps - 1) / kWarps : 0;   // stages warp, warp + kWarps, ...
    uint8_t *ring = smem + warp * kStages * kStageBytes;
    const uint32_t ring_u = smem_u32(ring);
    grid_dependency_wait();

    // copies: lane (g, t) the t-th 16 bytes of rows g, g + 8, g + 16, g + 24 (rows behind the last: the last, never written)
    const uint8_t *codes[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) codes[r] = p.codes + min(row0 + r * 8 + g, p.n - 1) * p.code_stride + t * 16 + warp * 64;
    int copied = 0;
    auto copy_stage = [&]() {
        if (copied < mine) {
            const uint32_t dst = ring_u + (copied % kStages) * kStageBytes + g * kPitch + t * 16;
            if (GROUP == 128 || (warp + copied * kWarps) * 128 + t * 32 < p.k) {
#pragma unroll
                for (int r = 0; r < 4; ++r) copy16_async(dst + r * 8 * kPitch, codes[r], 16);
            }   // (of columns behind the last any codes will do: their tokens' values are zeros)
#pragma unroll
            for (int r = 0; r < 4; ++r) codes[r] += kWarps * 64;
        }
        ++copied;
        copy_commit();
    };
    // scales: a lane has a row
    const M *scale = static_cast<const M *>(p.scale) + min(row0 + lane, p.n - 1) * p.meta_stride;
    const M *zero = p.zero ? static_cast<const M *>(p.zero) + min(row0 + lane, p.n - 1) * p.meta_stride : nullptr;
    M sc[kGroups], ze[kGroups];
    auto load_meta = [&](int i) {
        if (i >= mine) return;
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            int gr = (warp + i * kWarps) * kGroups + q;
            if (GROUP < 128) gr = min(gr, p.groups - 1);
            sc[q] = __ldg(scale + gr);
            if (zero) ze[q] = __ldg(zero + gr);
        }
    };
    // tokens: lane (g, t) the 8 values of columns 32 j + 8 t of token g, in pairs 4 columns apart as the codes of a word
    const T *x[NT];
    bool is[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int tok = tok0 + j * 8 + g;
        is[j] = tok < p.tokens;
        x[j] = static_cast<const T *>(p.x) + (is[j] ? tok : 0) * p.x_stride + t * 8 + warp * 128;
    }
    uint4 xv[4][NT];
    auto load_x = [&](int i) {
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const bool on = is[b] && i < mine;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xv[j][b] = make_uint4(0, 0, 0, 0);
                if (on && (GROUP == 128 || (warp + i * kWarps) * 128 + j * 32 < p.k))
                    xv[j][b] = __ldg(reinterpret_cast<const uint4 *>(x[b] + i * (kWarps * 128) + j * 32));
            }
        }
    };
    float acc[2][NT][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[m][j][e] = 0.f;

#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) copy_stage();
    load_meta(0);
    load_x(0);
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        float2(*meta)[kRows] = meta_s[warp][i & 1];
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            const float s = 16.f * to_float(sc[q]);
            meta[q][lane] = make_float2(s, zero ? to_float(ze[q]) - s : -1.5f * s);
        }
        load_meta(i + 1);
        uint32_t b[4][NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const uint4 v = xv[j][c];
                b[j][c][0] = __byte_perm(v.x, v.z, 0x5410), b[j][c][1] = __byte_perm(v.x, v.z, 0x7632);
                b[j][c][2] = __byte_perm(v.y, v.w, 0x5410), b[j][c][3] = __byte_perm(v.y, v.w, 0x7632);
            }
        load_x(i + 1);
        copy_wait<kStages - 2>();
        __syncwarp();
        copy_stage();   // into the slot that the stage before this one has left
        const uint8_t *at = ring + (i % kStages) * kStageBytes + g * kPitch + t * 4;
        float d[2][NT][4], sx[NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t a[2][2][4];   // [16 rows][product][register]
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t v = *reinterpret_cast<const uint32_t *>(at + (2 * m + h) * 8 * kPitch + j * 16);
                    a[m][0][h] = code_pair<T, 0>(v);
                    a[m][0][2 + h] = code_pair<T, 1>(v);
                    a[m][1][h] = code_pair<T, 2>(v);
                    a[m][1][2 + h] = code_pair<T, 3>(v);
                }
            const uint32_t one[4] = {ones, ones, ones, ones};
            const bool first = j * 32 % GROUP == 0;
#pragma unroll
            for (int c = 0; c < NT; ++c) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    if (first) mma16x8x16_first<T>(d[m][c], a[m][0], b[j][c][0], b[j][c][1]);
                    else mma16x8x16<T>(d[m][c], a[m][0], b[j][c][0], b[j][c][1]);
                    mma16x8x16<T>(d[m][c], a[m][1], b[j][c][2], b[j][c][3]);
                }
                if (first) mma16x8x16_first<T>(sx[c], one, b[j][c][0], b[j][c][1]);
                else mma16x8x16<T>(sx[c], one, b[j][c][0], b[j][c][1]);
                mma16x8x16<T>(sx[c], one, b[j][c][2], b[j][c][3]);
            }
            if ((j + 1) * 32 % GROUP == 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float2 f = meta[j * 32 / GROUP][r * 8 + g];
#pragma unroll
                    for (int c = 0; c < NT; ++c)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float &y = acc[r >> 1][c][(r & 1) * 2 + e];
                            y = fmaf(f.x, d[r >> 1][c][(r & 1) * 2 + e], y);
                            y = fmaf(f.y, sx[c][e], y);
                        }
                }
            }
        }
    }
    copy_wait<0>();
    __syncthreads();
    // the warps' sums, in the rings' place
    float(*sums)[kRows][8 * NT + 1] = reinterpret_cast<float(*)[kRows][8 * NT + 1]>(smem);
    static_assert(sizeof(float) * kWarps * kRows * (8 * NT + 1) <= kWarps * kStages * kStageBytes, "room for the sums");
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][m * 16 + (e >> 1) * 8 + g][j * 8 + t * 2 + (e & 1)] = acc[m][j][e];
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * 8 * NT; i += kWarps * 32) {
        const int r = i % kRows, c = i / kRows;
        if (row0 + r >= p.n || tok0 + c >= p.tokens) continue;
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) y += sums[w][r][c];
        if (p.bias) y += static_cast<float>(static_cast<const T *>(p.bias)[row0 + r]);
        if (p.add) y += static_cast<float>(static_cast<const T *>(p.add)[(tok0 + c) * p.add_stride + row0 + r]);
        static_cast<T *>(p.y)[(tok0 + c) * p.y_stride + row0 + r] = from_float<T>(y);
    }
}

template <typename T, typename M, int GROUP, int NT>
cudaError_t launch(const W4Params &p, cudaStream_t s) {
    const dim3 grid((p.n + kRows - 1) / kRows, (p.tokens + 8 * NT - 1) / (8 * NT));
    constexpr int smem = kWarps * kStages * kStageBytes;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(w4_few_kernel<T, M, GROUP, NT>), smem, allowed);
    return e != cudaSuccess ? e : launch_after_producer(w4_few_kernel<T, M, GROUP, NT>, grid, dim3(kWarps * 32), smem, s, p);
}

template <typename T, typename M, int GROUP>
cudaError_t by_tokens(const W4Params &p, cudaStream_t s) {
    return p.tokens <= 8 ? launch<T, M, GROUP, 1>(p, s) : launch<T, M, GROUP, 2>(p, s);
}

template <typename T, int GROUP>
cudaError_t by_meta(const W4Params &p, cudaStream_t s) {
    return p.meta_dtype == STOM_FP32   ? by_tokens<T, float, GROUP>(p, s)
           : p.meta_dtype == STOM_BF16 ? by_tokens<T, __nv_bfloat16, GROUP>(p, s)
                                       : by_tokens<T, __half, GROUP>(p, s);
}

template <typename T>
cudaError_t by_group(const W4Params &p, int group, cudaStream_t s) {
    return group == 32 ? by_meta<T, 32>(p, s) : group == 64 ? by_meta<T, 64>(p, s) : by_meta<T, 128>(p, s);
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int32_t stom_w4_linear(const stom_w4_matrix *w, int32_t dtype, int32_t rows, const void *x, int64_t x_stride,
                                  const void *bias, const void *add, int64_t add_stride, void *y, int64_t y_stride,
                                  void *stream) {
    if (!w || !w->codes || !w->scale || w->n < 1 || w->k < 1 || rows < 0) return STOM_ERR_INVALID_ARG;
    if (w->group != 32 && w->group != 64 && w->group != 128) return STOM_ERR_SHAPE;
    if (w->k % w->group || rows > 65535 * 8) return STOM_ERR_SHAPE;
    if (w->meta_dtype != STOM_BF16 && w->meta_dtype != STOM_FP16 && w->meta_dtype != STOM_FP32) return STOM_ERR_UNSUPPORTED;
    if (dtype != STOM_BF16 && dtype != STOM_FP16) return STOM_ERR_UNSUPPORTED;
    if (!aligned16(w->codes) || w->code_stride % 16) return STOM_ERR_ALIGNMENT;
    const uintptr_t meta = reinterpret_cast<uintptr_t>(w->scale) | reinterpret_cast<uintptr_t>(w->zero);
    if (meta & (elem_bytes(w->meta_dtype) - 1)) return STOM_ERR_ALIGNMENT;
    if (w->n > 1 && (w->code_stride < w->k / 2 || w->meta_stride < w->k / w->group)) return STOM_ERR_INVALID_ARG;
    if (rows == 0) return STOM_OK;
    if (!x || !y) return STOM_ERR_INVALID_ARG;
    if (!aligned16(x) || !stride_ok(x_stride, dtype)) return STOM_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(bias) | reinterpret_cast<uintptr_t>(add) | reinterpret_cast<uintptr_t>(y)) & 1u)
        return STOM_ERR_ALIGNMENT;
    if (rows > 1 && (x_stride < 0 || y_stride < w->n || (add && add_stride < 0))) return STOM_ERR_INVALID_ARG;
    W4Params p = {};
    p.codes = w->codes;
    p.scale = w->scale;
    p.zero = w->zero;
    p.n = w->n;
    p.k = w->k;
    p.groups = w->k / w->group;
    p.meta_dtype = w->meta_dtype;
    p.code_stride = w->code_stride;
    p.meta_stride = w->meta_stride;
    p.x = x;
    p.x_stride = x_stride;
    p.bias = bias;
    p.add = add;
    p.add_stride = add_stride;
    p.y = y;
    p.y_stride = y_stride;
    p.tokens = rows;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == STOM_BF16 ? by_group<__nv_bfloat16>(p, w->group, s) : by_group<__half>(p, w->group, s);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}
