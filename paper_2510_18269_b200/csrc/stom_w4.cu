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

__device__ __forceinline__ float meta_at(const void *base, int64_t i, int dtype) {
    if (dtype == STOM_FP32) return __ldg(static_cast<const float *>(base) + i);
    if (dtype == STOM_BF16) return __bfloat162float(__ldg(static_cast<const __nv_bfloat16 *>(base) + i));
    return __half2float(__ldg(static_cast<const __half *>(base) + i));
}

// GROUP columns a group; NT blocks of 8 tokens.
// A warp goes through stages of 128 columns (the block's warps take them in turn): 64 bytes of each of its 32 rows, copied
// to its own ring in shared memory kStages - 1 stages ahead; the tokens' values and the rows' scales a stage ahead in
// registers.  No barrier but the one before the warps' sums are joined.
template <typename T, int GROUP, int NT>
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
    for (int r = 0; r < 4; ++r) codes[r] = p.codes + min(row0 + r * 8 + g, p.n - 1) * p.code_stride + t * 16;
    auto copy_stage = [&](int i) {
        if (i < mine) {
            const int at = (warp + i * kWarps) * 64;
            const uint32_t bytes = 2 * at + t * 32 < p.k ? 16u : 0u;   // columns behind the last: zeros
            const uint32_t dst = ring_u + (i % kStages) * kStageBytes + g * kPitch + t * 16;
#pragma unroll
            for (int r = 0; r < 4; ++r) copy16_async(dst + r * 8 * kPitch, codes[r] + (bytes ? at : 0), bytes);
        }
        copy_commit();
    };
    // scales: a lane has a row
    const int64_t meta0 = min(row0 + lane, p.n - 1) * p.meta_stride;
    float sc[kGroups], ze[kGroups];
    auto load_meta = [&](int i) {
        if (i >= mine) return;
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            const int gr = min((warp + i * kWarps) * kGroups + q, p.groups - 1);
            sc[q] = meta_at(p.scale, meta0 + gr, p.meta_dtype);
            ze[q] = p.zero ? meta_at(p.zero, meta0 + gr, p.meta_dtype) : -8.f * sc[q];
        }
    };
    // tokens: lane (g, t) the 8 values of columns 32 j + 8 t of token g, in pairs 4 columns apart as the codes of a word
    const T *x[NT];
    bool is[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int tok = tok0 + j * 8 + g;
        is[j] = tok < p.tokens;
        x[j] = static_cast<const T *>(p.x) + (is[j] ? tok : 0) * p.x_stride + t * 8;
    }
    uint4 xv[4][NT];
    auto load_x = [&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const int col = (warp + i * kWarps) * 128 + j * 32;
                xv[j][b] = make_uint4(0, 0, 0, 0);
                if (is[b] && i < mine && col < p.k) xv[j][b] = __ldg(reinterpret_cast<const uint4 *>(x[b] + col));
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
    for (int i = 0; i < kStages - 1; ++i) copy_stage(i);
    load_meta(0);
    load_x(0);
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        float2(*meta)[kRows] = meta_s[warp][i & 1];
#pragma unroll
        for (int q = 0; q < kGroups; ++q) meta[q][lane] = make_float2(16.f * sc[q], ze[q] - 16.f * sc[q]);
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
        copy_stage(i + kStages - 1);   // into the slot that the stage before this one has left
        const uint8_t *at = ring + (i % kStages) * kStageBytes + g * kPitch + t * 4;
        float d[2][NT][4], sx[NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j * 32 % GROUP == 0)
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[0][c][e] = d[1][c][e] = sx[c][e] = 0.f;
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
#pragma unroll
            for (int c = 0; c < NT; ++c) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    mma16x8x16<T>(d[m][c], a[m][0], b[j][c][0], b[j][c][1]);
                    mma16x8x16<T>(d[m][c], a[m][1], b[j][c][2], b[j][c][3]);
                }
                mma16x8x16<T>(sx[c], one, b[j][c][0], b[j][c][1]);
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

template <typename T, int GROUP, int NT>
cudaError_t launch(const W4Params &p, cudaStream_t s) {
    const dim3 grid((p.n + kRows - 1) / kRows, (p.tokens + 8 * NT - 1) / (8 * NT));
    constexpr int smem = kWarps * kStages * kStageBytes;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(w4_few_kernel<T, GROUP, NT>), smem, allowed);
    return e != cudaSuccess ? e : launch_after_producer(w4_few_kernel<T, GROUP, NT>, grid, dim3(kWarps * 32), smem, s, p);
}

template <typename T, int GROUP>
cudaError_t by_tokens(const W4Params &p, cudaStream_t s) {
    return p.tokens <= 8 ? launch<T, GROUP, 1>(p, s) : launch<T, GROUP, 2>(p, s);
}

template <typename T>
cudaError_t by_group(const W4Params &p, int group, cudaStream_t s) {
    return group == 32 ? by_tokens<T, 32>(p, s) : group == 64 ? by_tokens<T, 64>(p, s) : by_tokens<T, 128>(p, s);
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
