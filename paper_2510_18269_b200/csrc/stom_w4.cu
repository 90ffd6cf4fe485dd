// Products of a few tokens with 4-bit weights (stom_w4_linear).
//
//   y[t][r] = sum_g ( s_rg sum_c code_rc x_tc + z_rg sum_c x_tc ) + bias_r + add_tr,   c over the columns of group g.
//
// What bounds it: the codes, half a byte a weight, are read once; at one token each takes part in one multiply-add, so
// that memory gives 46 weights a clock to a multiprocessor.  The scalar units would need as many multiply-adds and an
// unpacking for each; on the tensor cores (m16n8k16: the weights the 16 rows, the tokens the 8 columns) a warp-wide product
// takes 256 of them behind five instructions that unpack (see stom_w4.cuh).
//
// Layout.  Codes are used as they lie in memory.  The order of columns within a product is free as long as weights and
// tokens agree: lane (g, t) of a fragment takes the t-th word (8 codes) of a row's 32 columns, two products' worth.  All of
// a product's columns lie in one group.
//
// Measured on one B200, us, called from Python with a few sets of inputs in turn (perf/more_operators.py; the smallest matrices
// then come from L2): one token of 4 608 x 3 584 5.0, of 28 672 x 3 584 in groups of 64 21.5 (2.7 of 6.5 TB/s), five of
// 151 001 x 3 584 67 to 70 (4.2 TB/s).  The comparisons below are of calls queued ahead on the device, codes from memory, groups
// of 128 with offsets, bf16; there the same three take 5.7, 17.1 and 58.  What bounds it now is the issue of instructions, 120 that read, unpack and multiply for 4 096
// weights and about as many for copies, scales and folding.  A ring of its own for every warp took one token from 74 to 30 us;
// codes as subnormal numbers instead of unpacked ones, with offsets, five tokens' logits from 93 to 84; smaller teams from 84
// to 69.
#include "stom_w4.cuh"

namespace stom {

namespace {

constexpr int kRows = 16;     // of the matrix, per slab
constexpr int kTok = 8;       // most tokens of a block
constexpr int kWarps = 16, kThreads = kWarps * 32;   // of a block
constexpr int kUnitCols = 256;                // columns of a unit
constexpr int kPitch = kUnitCols / 2 + 16;    // bytes from row to row in shared memory: 8 rows' words of 4 lanes lie in 32 banks
constexpr int kUnitBytes = kRows * kPitch;
constexpr int kMostShared = 194 * 1024;       // dynamic shared memory of a block

__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// c = a b, 16x16 by 16x8: the first product of a sum
__device__ __forceinline__ void mma16x8x16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// Bytes of shared memory: the tokens' operands, a factor and a sum for each token and group, the warps' results, the rings
struct FewLayout {
    int64_t factor, sums, rings, total;
    __host__ __device__ FewLayout(int k, int groups, int tokens, int depth) {
        const int64_t units = (k + kUnitCols - 1) / kUnitCols, group = k / groups;   // (columns behind the last: zeros)
        factor = units * (kUnitCols / 32) * tokens * 64;
        sums = factor + units * (kUnitCols / group) * kTok * 8;
        rings = sums + 2 * kWarps * kRows * (kTok + 1) * 4;
        total = rings + kWarps * depth * kUnitBytes;
    }
};

// Up to 8 tokens of those from 8 * blockIdx.y on; GROUP columns a group; a ring of DEPTH units.
// A block, one a multiprocessor, has TEAMS teams of warps, sixteen together.  A team goes through slabs of 16 rows, whose UNITS of 256
// columns its warps take in turn (and go on in turn with the next slab's, so that none has more of them).  A warp is alone
// with its units: its own ring in shared memory, filled by 16-byte asynchronous copies DEPTH - 1 units ahead, the rows' scales
// a unit ahead in registers.  At a slab's end the warps' sums are joined in shared memory, with one barrier of the team.
// Tokens stay in shared memory, in the order of the fragments.
template <typename T, int GROUP, int DEPTH, int TEAMS>
__global__ void __launch_bounds__(kThreads, 1) w4_few_kernel(const __grid_constant__ W4Params p) {
    constexpr int kGroups = kUnitCols / GROUP;   // of a unit
    constexpr int kTeams = TEAMS, kTeamWarps = kWarps / TEAMS;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float2 meta_s[kWarps][2][kGroups][kRows];
    const int tok0 = blockIdx.y * kTok, tokens = min(kTok, p.tokens - tok0);   // of the block
    const FewLayout at(p.k, p.groups, tokens, DEPTH);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, team = warp / kTeamWarps, tw = warp % kTeamWarps;
    const int g = lane >> 2, t = lane & 3;
    const int units = (p.k + kUnitCols - 1) / kUnitCols, slabs = (p.n + kRows - 1) / kRows;
    // the team's slabs: slab0, slab0 + slab_step, ...; as long as there are no more than blocks, each has a block of its own
    const int slab0 = blockIdx.x + team * gridDim.x, slab_step = kTeams * gridDim.x;
    const int mine = slab0 < slabs ? (slabs - slab0 + slab_step - 1) / slab_step : 0;
    auto first_unit = [&](int sl) { return (tw - sl * units) & (kTeamWarps - 1); };
    uint8_t *ring = smem + at.rings + warp * DEPTH * kUnitBytes;
    const uint32_t ring_u = smem_u32(ring) + (lane >> 3) * kPitch + (lane & 7) * 16;
    grid_dependency_wait();

    // ---- copies: lane l the (l % 8)-th 16 bytes of rows l / 8, + 4, + 8, + 12 (rows behind the last: the last, never written)
    int csl = -1, cu = units, cslot = 0;         // the unit to copy next
    const uint8_t *cp[4];
    auto copy_unit = [&]() {
        if (cu >= units) {
            while (cu >= units && ++csl < mine) cu = first_unit(csl);
            if (cu < units)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    cp[r] = p.codes + min((slab0 + csl * slab_step) * kRows + (lane >> 3) + 4 * r, p.n - 1) * p.code_stride +
                            cu * (kUnitCols / 2) + (lane & 7) * 16;
        }
        if (cu < units) {
            // (of columns behind the last any codes will do: the tokens are zeros there)
            if ((cu + 1) * kUnitCols <= p.k || cu * kUnitCols + (lane & 7) * 32 < p.k) {
                const uint32_t dst = ring_u + cslot * kUnitBytes;
#pragma unroll
                for (int r = 0; r < 4; ++r) copy16_async(dst + 4 * r * kPitch, cp[r], 16);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) cp[r] += kTeamWarps * (kUnitCols / 2);
            cu += kTeamWarps;
        }
        copy_commit();
        cslot = cslot + 1 == DEPTH ? 0 : cslot + 1;
    };
    // ---- scales: lane l < 16 that of row l, lane 16 + l its offset (or the scale again, where there is none)
    const bool wide = p.meta_dtype == STOM_FP32, narrow_bf = p.meta_dtype == STOM_BF16;
    const int es = wide ? 4 : 2;
    const char *meta_of = static_cast<const char *>(lane >= kRows && p.zero ? p.zero : p.scale), *mp = meta_of;
    const float meta_times = lane < kRows ? kCodeUnit : p.zero ? 1.f : -8.f;
    int msl = -1, mu = units;                    // the unit whose scales come next
    uint32_t raw[kGroups];
    auto load_meta = [&]() {
        if (mu >= units) {
            while (mu >= units && ++msl < mine) mu = first_unit(msl);
            if (mu >= units) return;
            mp = meta_of + (min((slab0 + msl * slab_step) * kRows + (lane & 15), p.n - 1) * p.meta_stride + mu * kGroups) * es;
        }
        const int last = p.groups - 1 - mu * kGroups;   // (groups behind the last: the last, times zeros)
        if (wide) {
#pragma unroll
            for (int q = 0; q < kGroups; ++q) raw[q] = __ldg(reinterpret_cast<const uint32_t *>(mp) + min(q, last));
        } else {
#pragma unroll
            for (int q = 0; q < kGroups; ++q) raw[q] = __ldg(reinterpret_cast<const uint16_t *>(mp) + min(q, last));
        }
        mp += kTeamWarps * kGroups * es;
        mu += kTeamWarps;
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) copy_unit();
    load_meta();

    // ---- tokens: a warp takes 256 columns of one at a time, a lane 8 of them; the lanes of a group find its largest value and
    // its sum
    float2 *factor = reinterpret_cast<float2 *>(smem + at.factor);   // [group][kTok / 2][factors, sums]
    for (int i = warp; i < units * tokens; i += kWarps) {
        const int tok = i / units, col = (i - tok * units) * kUnitCols + lane * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (col < p.k) v = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.x) + (tok0 + tok) * p.x_stride + col);
        float a[8];
        unpack2<T>(v.x, a[0], a[1]);
        unpack2<T>(v.y, a[2], a[3]);
        unpack2<T>(v.z, a[4], a[5]);
        unpack2<T>(v.w, a[6], a[7]);
        float sum = ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
        uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
        m = max(m & 0xffffu, m >> 16);
#pragma unroll
        for (int o = 1; o < GROUP / 8; o <<= 1) {
            sum += __shfl_xor_sync(~0u, sum, o);
            m = max(m, __shfl_xor_sync(~0u, m, o));
        }
        float before, after;
        factors_of<T>(m, before, after);
        *reinterpret_cast<uint4 *>(smem + ((int64_t)(col / 32 * tokens + tok) * 4 + (lane & 3)) * 16) = token_operand<T>(v, before);
        if (lane % (GROUP / 8) == 0) {
            float *to = reinterpret_cast<float *>(factor + (col / GROUP * (kTok / 2) + (tok >> 1)) * 2) + (tok & 1);
            to[0] = after;
            to[2] = sum;
        }
    }
    __syncthreads();

    // ---- products (a lane of a token that there is not reads the last one's: its columns of the product are not used)
    const uint8_t *own_x = smem + (min(g, tokens - 1) * 4 + t) * 16;
    int slot = 0, turn = 0;
#pragma unroll 1
    for (int sl = 0; sl < mine; ++sl) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int u = first_unit(sl); u < units; u += kTeamWarps) {
            float2(*meta)[kRows] = meta_s[warp][turn & 1];
            ++turn;
            float *to = reinterpret_cast<float *>(&meta[0][lane & 15]) + (lane >> 4);
            if (wide || narrow_bf) {
                const int up = wide ? 0 : 16;
#pragma unroll
                for (int q = 0; q < kGroups; ++q) to[q * (2 * kRows)] = __uint_as_float(raw[q] << up) * meta_times;
            } else {
#pragma unroll
                for (int q = 0; q < kGroups; ++q)
                    to[q * (2 * kRows)] = __half2float(__ushort_as_half((unsigned short)raw[q])) * meta_times;
            }
            load_meta();
            copy_wait<DEPTH - 2>();
            __syncwarp();
            copy_unit();   // into the slot that the unit before this one has left
            const uint8_t *cs = ring + slot * kUnitBytes + g * kPitch + t * 4;
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
            float d[4];
            const uint32_t x_at = u * (kUnitCols / 32) * (tokens * 64);
            const float4 *fx = reinterpret_cast<const float4 *>(factor) + u * kGroups * (kTok / 2) + t;
#pragma unroll
            for (int j = 0; j < kUnitCols / 32; ++j) {
                uint32_t a[2][4];   // [product][register]
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t v = *reinterpret_cast<const uint32_t *>(cs + h * 8 * kPitch + j * 16), w = v >> 8;
                    a[0][h] = v & 0x000f000fu;
                    a[0][2 + h] = v & 0x00f000f0u;
                    a[1][h] = w & 0x000f000fu;
                    a[1][2 + h] = w & 0x00f000f0u;
                }
                const uint4 b = *reinterpret_cast<const uint4 *>(own_x + x_at + j * (tokens * 64));
                if (j * 32 % GROUP == 0) mma16x8x16_first(d, a[0], b.x, b.y);
                else mma16x8x16<__half>(d, a[0], b.x, b.y);
                mma16x8x16<__half>(d, a[1], b.z, b.w);
                if ((j + 1) * 32 % GROUP == 0) {
                    const int q = j * 32 / GROUP;
                    const float2 f0 = meta[q][g], f1 = meta[q][g + 8];
                    const float4 x = fx[q * (kTok / 2)];   // factors and sums of tokens 2 t, 2 t + 1
                    acc[0] = fmaf(f0.y, x.z, fmaf(f0.x, d[0] * x.x, acc[0]));
                    acc[1] = fmaf(f0.y, x.w, fmaf(f0.x, d[1] * x.y, acc[1]));
                    acc[2] = fmaf(f1.y, x.z, fmaf(f1.x, d[2] * x.x, acc[2]));
                    acc[3] = fmaf(f1.y, x.w, fmaf(f1.x, d[3] * x.y, acc[3]));
                }
            }
        }
        float(*part)[kRows][kTok + 1] =
            reinterpret_cast<float(*)[kRows][kTok + 1]>(smem + at.sums) + (team * 2 + (sl & 1)) * kTeamWarps;
#pragma unroll
        for (int e = 0; e < 4; ++e) part[tw][(e >> 1) * 8 + g][t * 2 + (e & 1)] = acc[e];
        named_sync(1 + team, kTeamWarps * 32);   // (the slab after the next waits here before it writes to this part again)
        const int row = (slab0 + sl * slab_step) * kRows + (lane & 15);
#pragma unroll
        for (int c0 = 0; c0 < kTok; c0 += 2 * kTeamWarps) {
            const int c = c0 + tw * 2 + (lane >> 4);
            if (row < p.n && c < tokens) {
                float y = 0.f;
#pragma unroll
                for (int w = 0; w < kTeamWarps; ++w) y += part[w][lane & 15][c];
                if (p.bias) y += to_float(static_cast<const T *>(p.bias)[row]);
                if (p.add) y += to_float(static_cast<const T *>(p.add)[(tok0 + c) * p.add_stride + row]);
                static_cast<T *>(p.y)[(tok0 + c) * p.y_stride + row] = from_float<T>(y);
            }
        }
    }
    copy_wait<0>();
}

// Units of a warp's ring with which the few-tokens kernel fits into shared memory, or 0
int depth_of(int k, int groups, int tokens) {
    for (int depth = 4; depth >= 3; --depth)
        if (FewLayout(k, groups, tokens < kTok ? tokens : kTok, depth).total <= kMostShared) return depth;
    return 0;
}
// The few-tokens kernel takes up to 8, if they fit into shared memory, and up to 16 as twice 8 where the matrix has so few rows
// that the blocks of both have a multiprocessor each, or more than 12 slabs a block (`sms` of them; 0: no device is known, and 8
// is all that is sure).  Measured in us, this kernel (9 and 16 tokens: as twice 8 everywhere) and then the one for many:
//   columns  tokens       512 rows         4 608        18 944        28 672       151 001
//     3 584       8     6.6 / 12.7    9.4 / 14.3   15.1 / 23.1   20.3 / 36.8      61 / 142
//     3 584       9     6.8 / 12.7   13.8 / 14.4   24.4 / 23.2   33.6 / 36.8     116 / 143
//     3 584      16     6.7 / 12.7   17.4 / 14.5   28.5 / 23.3   37.8 / 37.1     125 / 143
//     2 048       8     4.5 / 10.3    6.2 / 11.6   10.4 / 15.7   13.5 / 25.0       40 / 84
//     2 048       9     4.5 / 10.3    9.5 / 11.6   17.0 / 15.7   22.6 / 25.0       74 / 85
//     2 048      16     4.5 / 10.3   11.5 / 11.7   19.3 / 15.8   24.9 / 25.5       76 / 85
//     1 024       8     3.4 / 10.1    4.1 / 10.6    6.6 / 10.9    8.8 / 18.0       25 / 46
//     1 024       9     3.4 / 10.1    6.8 / 10.6   11.2 / 10.9   14.7 / 18.0       45 / 46
//     1 024      16     3.4 / 10.2    7.6 / 10.9   12.1 / 11.0   15.7 / 18.4       46 / 47
// (So with few columns twice 8 would also be ahead by up to 4 us in between.)
bool is_few(int n, int k, int groups, int tokens, int sms) {
    const int slabs = (n + kRows - 1) / kRows;
    const bool twice = sms > 0 && (slabs <= sms / 2 || slabs > 12 * sms);
    return tokens <= (twice ? 2 * kTok : kTok) && depth_of(k, groups, tokens) > 0;
}

template <typename T, int GROUP, int DEPTH, int TEAMS>
cudaError_t launch_few(const W4Params &p, int sms, cudaStream_t s) {
    const int tokens = p.tokens < kTok ? p.tokens : kTok;
    const FewLayout l(p.k, p.groups, tokens, DEPTH);
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(w4_few_kernel<T, GROUP, DEPTH, TEAMS>), kMostShared, allowed);
    if (e != cudaSuccess) return e;
    const int slabs = (p.n + kRows - 1) / kRows;
    const dim3 grid(slabs < sms ? slabs : sms, (p.tokens + tokens - 1) / tokens);
    return launch_after_producer(w4_few_kernel<T, GROUP, DEPTH, TEAMS>, grid, dim3(kThreads), (size_t)l.total, s, p);
}
// Two teams of eight warps where a block has up to three slabs, so that each is done sooner, and eight of two where it has more:
// the joins at a slab's end then come after four times as many units of a warp.  Two against eight, one and eight tokens, us:
// 3 584 x 14 336 14.1 against 17.4 (8 take the other kernel), 4 608 x 3 584 5.7 and 9.4 against 5.9 and 10.0, 9 472 x 3 584 8.8 and
// 12.2 against 7.9 and 11.5, 28 672 x 3 584 18.9 and 22.9 against 17.0 and 20.3, 151 001 x 3 584 78 and 83 against 57 and 61.
template <typename T, int GROUP, int DEPTH>
cudaError_t by_teams(const W4Params &p, int sms, cudaStream_t s) {
    return (p.n + kRows - 1) / kRows <= 3 * sms ? launch_few<T, GROUP, DEPTH, 2>(p, sms, s) : launch_few<T, GROUP, DEPTH, 8>(p, sms, s);
}

template <typename T, int GROUP>
cudaError_t by_tokens(const W4Params &p, int sms, void *workspace, cudaStream_t s) {
    if (!is_few(p.n, p.k, p.groups, p.tokens, sms)) return w4_many<T>(p, GROUP, sms, workspace, s);
    return depth_of(p.k, p.groups, p.tokens) == 4 ? by_teams<T, GROUP, 4>(p, sms, s) : by_teams<T, GROUP, 3>(p, sms, s);
}

template <typename T>
cudaError_t by_group(const W4Params &p, int group, int sms, void *ws, cudaStream_t s) {
    return group == 32 ? by_tokens<T, 32>(p, sms, ws, s) : group == 64 ? by_tokens<T, 64>(p, sms, ws, s) : by_tokens<T, 128>(p, sms, ws, s);
}

}  // namespace

}  // namespace stom

using namespace stom;

static int32_t check_matrix(const stom_w4_matrix *w, int32_t rows) {
    if (!w || !w->codes || !w->scale || w->n < 1 || w->k < 1 || rows < 0) return STOM_ERR_INVALID_ARG;
    if (w->group != 32 && w->group != 64 && w->group != 128) return STOM_ERR_SHAPE;
    if (w->k % w->group || w->k > (1 << 24) || w->n > (1 << 23) - 128 || rows > 65535 * 8) return STOM_ERR_SHAPE;
    if (w->meta_dtype != STOM_BF16 && w->meta_dtype != STOM_FP16 && w->meta_dtype != STOM_FP32) return STOM_ERR_UNSUPPORTED;
    if (!aligned16(w->codes) || w->code_stride % 16) return STOM_ERR_ALIGNMENT;
    const uintptr_t meta = reinterpret_cast<uintptr_t>(w->scale) | reinterpret_cast<uintptr_t>(w->zero);
    if (meta & (elem_bytes(w->meta_dtype) - 1)) return STOM_ERR_ALIGNMENT;
    if (w->n > 1 && (w->code_stride < w->k / 2 || w->meta_stride < w->k / w->group)) return STOM_ERR_INVALID_ARG;
    return STOM_OK;
}

extern "C" int64_t stom_w4_workspace_bytes(const stom_w4_matrix *w, int32_t rows) {
    const int32_t rc = check_matrix(w, rows);
    if (rc) return rc;
    return rows == 0 || is_few(w->n, w->k, w->k / w->group, rows, sm_count()) ? 0 : w4_many_workspace(w->k, w->group, rows);
}

extern "C" int32_t stom_w4_linear(const stom_w4_matrix *w, int32_t dtype, int32_t rows, const void *x, int64_t x_stride,
                                  const void *bias, const void *add, int64_t add_stride, void *y, int64_t y_stride,
                                  void *workspace, int64_t workspace_bytes, uint32_t *dev_flags, void *stream) {
    const int32_t rc = check_matrix(w, rows);
    if (rc) return rc;
    if (dtype != STOM_BF16 && dtype != STOM_FP16) return STOM_ERR_UNSUPPORTED;
    if (rows == 0) return STOM_OK;
    if (!x || !y) return STOM_ERR_INVALID_ARG;
    if (!aligned16(x) || !stride_ok(x_stride, dtype)) return STOM_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(bias) | reinterpret_cast<uintptr_t>(add) | reinterpret_cast<uintptr_t>(y)) & 1u)
        return STOM_ERR_ALIGNMENT;
    if (rows > 1 && (x_stride < 0 || y_stride < w->n || (add && add_stride < 0))) return STOM_ERR_INVALID_ARG;
    const int64_t need = stom_w4_workspace_bytes(w, rows);
    if (need > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 127u) || workspace_bytes < need)) return STOM_ERR_WORKSPACE;
    const int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
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
    p.flags = dev_flags;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == STOM_BF16 ? by_group<__nv_bfloat16>(p, w->group, sms, workspace, s)
                                             : by_group<__half>(p, w->group, sms, workspace, s);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}
