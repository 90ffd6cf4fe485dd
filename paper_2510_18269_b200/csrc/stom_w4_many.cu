// Products of many tokens with 4-bit weights (stom_w4_linear).
#include "stom_w4.cuh"

namespace stom {

namespace {

constexpr int kRows = 32, kWarps = 8, kSomeStages = 4;
constexpr int kSomePitch = 80;    // bytes from row to row of a stage in shared memory: 8 rows' words of 4 lanes lie in 32 banks
constexpr int kSomeStageBytes = kRows * kSomePitch;

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


__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

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
// to its own ring in shared memory kSomeStages - 1 stages ahead; the tokens' values and the rows' scales a stage ahead in
// registers.  No barrier but the one before the warps' sums are joined.
template <typename T, typename M, int GROUP, int NT>
__global__ void __launch_bounds__(kWarps * 32, 2) w4_some_kernel(const __grid_constant__ W4Params p) {
    constexpr int kGroups = 128 / GROUP;             // of a stage
    constexpr uint32_t ones = std::is_same<T, __nv_bfloat16>::value ? 0x3f803f80u : 0x3c003c00u;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float2 meta_s[kWarps][2][kGroups][kRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int row0 = blockIdx.x * kRows, tok0 = blockIdx.y * 8 * NT;
    const int stages = (p.k + 127) / 128;
    const int mine = warp < stages ? (stages - warp + kWarps - 1) / kWarps : 0;   // stages warp, warp + kWarps, ...
    uint8_t *ring = smem + warp * kSomeStages * kSomeStageBytes;
    const uint32_t ring_u = smem_u32(ring);
    grid_dependency_wait();

    // copies: lane (g, t) the t-th 16 bytes of rows g, g + 8, g + 16, g + 24 (rows behind the last: the last, never written)
    const uint8_t *codes[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) codes[r] = p.codes + min(row0 + r * 8 + g, p.n - 1) * p.code_stride + t * 16 + warp * 64;
    int copied = 0;
    auto copy_stage = [&]() {
        if (copied < mine) {
            const uint32_t dst = ring_u + (copied % kSomeStages) * kSomeStageBytes + g * kSomePitch + t * 16;
            if (GROUP == 128 || (warp + copied * kWarps) * 128 + t * 32 < p.k) {
#pragma unroll
                for (int r = 0; r < 4; ++r) copy16_async(dst + r * 8 * kSomePitch, codes[r], 16);
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
    for (int i = 0; i < kSomeStages - 1; ++i) copy_stage();
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
        copy_wait<kSomeStages - 2>();
        __syncwarp();
        copy_stage();   // into the slot that the stage before this one has left
        const uint8_t *at = ring + (i % kSomeStages) * kSomeStageBytes + g * kSomePitch + t * 4;
        float d[2][NT][4], sx[NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t a[2][2][4];   // [16 rows][product][register]
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t v = *reinterpret_cast<const uint32_t *>(at + (2 * m + h) * 8 * kSomePitch + j * 16);
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
    static_assert(sizeof(float) * kWarps * kRows * (8 * NT + 1) <= kWarps * kSomeStages * kSomeStageBytes, "room for the sums");
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
    constexpr int smem = kWarps * kSomeStages * kSomeStageBytes;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(w4_some_kernel<T, M, GROUP, NT>), smem, allowed);
    return e != cudaSuccess ? e : launch_after_producer(w4_some_kernel<T, M, GROUP, NT>, grid, dim3(kWarps * 32), smem, s, p);
}


template <typename T, int GROUP>
cudaError_t by_meta(const W4Params &p, cudaStream_t s) {
    return p.meta_dtype == STOM_FP32   ? launch<T, float, GROUP, 2>(p, s)
           : p.meta_dtype == STOM_BF16 ? launch<T, __nv_bfloat16, GROUP, 2>(p, s)
                                       : launch<T, __half, GROUP, 2>(p, s);
}

}  // namespace

template <typename T>
cudaError_t w4_many(const W4Params &p, int group, int sms, cudaStream_t s) {
    return group == 32 ? by_meta<T, 32>(p, s) : group == 64 ? by_meta<T, 64>(p, s) : by_meta<T, 128>(p, s);
}
template cudaError_t w4_many<__nv_bfloat16>(const W4Params &, int, int, cudaStream_t);
template cudaError_t w4_many<__half>(const W4Params &, int, int, cudaStream_t);

}  // namespace stom
