// Products of many tokens with 4-bit weights (stom_w4_linear): from about as many tokens on as a fragment has, the multiplying
// is done by the fifth-generation tensor cores.
//
// What bounds it: at 16 tokens the codes' bytes, as for one; at 64 the instructions that make operands of them and that
// scale the groups' sums.  A first small kernel makes operands of the tokens, once for all blocks (see stom_w4.cuh): the tiles
// of the right operand as they lie in shared memory, 128-byte-swizzled, and a factor and a sum for each token and group.
//
// A block has 128 rows of the matrix, N tokens and a part of the columns, a STAGE of 128 of them at a time.  Codes arrive by
// 16-byte asynchronous copies, 256 columns at a time, several ahead.  Eight warps unpack: a thread has one row and half of a
// stage's columns, 8 words that become 8 chunks of 16 bytes in the left operand (K-major, 128-byte swizzle; two stages of it).
// One thread issues the products, each group into accumulators of its own in tensor memory, since scales differ from group to
// group.  Eight more warps fold those of the stage before into sums while the products of this one run: a thread has a row
// again, and half of the tokens.
// Blocks that share out the columns of the same rows form a cluster (up to 8, so many that all multiprocessors have a
// block), whose sums are joined over distributed shared memory.
#include "stom_tensor.cuh"
#include "stom_w4.cuh"

namespace stom {

namespace {

constexpr int kRows = 128, kStageCols = 128;
constexpr int kUnpackWarps = 8, kFoldWarps = 8, kWorkWarps = kUnpackWarps + kFoldWarps;
constexpr int kUnpackThreads = kUnpackWarps * 32, kFoldThreads = kFoldWarps * 32, kThreads = (kWorkWarps + 4) * 32;
constexpr int kChunkCols = 256, kChunks = 4;              // columns of a copy, copies in the ring
constexpr int kPitch = kChunkCols / 2 + 16, kChunkBytes = kRows * kPitch;   // an odd number of 16 bytes: a row a thread without conflicts
constexpr int kAStage = kRows * kStageCols * 2, kBStages = 3;
constexpr unsigned long long kWaitLimitNs = 1000000000ull;   // a wait that has taken 1 s ends the block

// Bytes of a stage's operand of the tokens, factors and sums
__host__ __device__ constexpr int stage_bytes(int group, int n) { return n * kStageCols * 2 + kStageCols / group * n * 8; }

struct ManyParams {
    W4Params w;
    uint8_t *image;        // [token tile][stage]: operand [2][N][128 bytes], factors [group][N], sums [group][N]
    int32_t stages, split; // of 128 columns; blocks of a cluster
};

__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Operands of the tokens: a warp has 256 columns of one, a lane 8; tokens and columns behind the last become zeros
template <typename T, int GROUP, int N>
__global__ void __launch_bounds__(256) w4_tokens_kernel(const __grid_constant__ ManyParams p) {
    grid_dependency_wait();
    grid_launch_dependents();   // (behind the wait: what the next kernel reads before its own wait, the weights, is there)
    const int lane = threadIdx.x & 31, spans = (p.stages + 1) / 2;
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5), tok = i / spans, col = (i - tok * spans) * 256 + lane * 8;
    if (tok >= (p.w.tokens + N - 1) / N * N) return;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (tok < p.w.tokens && col < p.w.k)
        v = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.w.x) + tok * p.w.x_stride + col);
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
    const int stage = col / kStageCols;
    if (stage >= p.stages) return;
    float before, after;
    factors_of<T>(m, before, after);
    const int tile = tok / N, row = tok % N, block = col / 64 & 1, chunk = col / 8 & 7;
    constexpr int kGroups = kStageCols / GROUP;
    uint8_t *to = p.image + ((int64_t)tile * p.stages + stage) * stage_bytes(GROUP, N);
    *reinterpret_cast<uint4 *>(to + (block * N + row) * 128 + ((chunk ^ (row & 7)) << 4)) = token_operand<T>(v, before);
    if (lane % (GROUP / 8) == 0) {
        float *f = reinterpret_cast<float *>(to + N * kStageCols * 2) + (col / GROUP % kGroups) * N + row;
        f[0] = after;
        f[kGroups * N] = sum;
    }
}

template <int GROUP, int N>
struct Many {
    static constexpr int kGroups = kStageCols / GROUP;         // of a stage
    static constexpr int kBStage = (stage_bytes(GROUP, N) + 1023) / 1024 * 1024;
    static constexpr int kMeta = kChunkCols / GROUP * kRows * 8;
    static constexpr int kCols = 2 * kGroups * N < 32 ? 32 : 2 * kGroups * N;   // of tensor memory, a power of two
    static constexpr int kOffB = 2 * kAStage, kOffCodes = kOffB + kBStages * kBStage, kOffMeta = kOffCodes + kChunks * kChunkBytes;
    static constexpr int kSmem = 1024 + kOffMeta + 3 * kMeta;
    static constexpr int kPitchOut = kRows + 4;                // floats from token to token of the sums that a cluster joins
    static_assert(kSmem <= 226 * 1024 && kCols <= 512, "room");
    static_assert(N * kPitchOut * 4 <= 2 * kAStage, "the sums take the left operand's place");
};

template <typename T, int GROUP, int N>
__global__ void __launch_bounds__(kThreads, 1) w4_many_kernel(const __grid_constant__ ManyParams p) {
    using S = Many<GROUP, N>;
    constexpr int kGroups = S::kGroups, kBStage = S::kBStage, kOwn = N / 2;   // tokens of a thread that folds
    extern __shared__ uint8_t raw_smem[];
    __shared__ uint64_t c_full[kChunks], c_empty[kChunks], b_full[kBStages], b_empty[kBStages], a_full[2], done[2], folded[2], drained;
    __shared__ uint32_t tmem_word, abort_word, never_word;   // never_word stays 0
    uint8_t *smem = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);   // the swizzle goes by addresses
    const uint32_t smem_at = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x, row0 = blockIdx.y * kRows, tile = blockIdx.z;
    // the block's stages, as equal shares as they can be
    const int s0 = (int)((int64_t)p.stages * rank / p.split), n_stages = (int)((int64_t)p.stages * (rank + 1) / p.split) - s0;
    const int col0 = s0 * kStageCols, n_chunks = (n_stages + 1) / 2;
    volatile uint32_t *abort_flag = &abort_word;
    if (tid == 0) {
        for (int i = 0; i < kChunks; ++i) mbar_init(smem_u32(&c_full[i]), 64), mbar_init(smem_u32(&c_empty[i]), kUnpackWarps);
        for (int i = 0; i < kBStages; ++i) mbar_init(smem_u32(&b_full[i]), 1), mbar_init(smem_u32(&b_empty[i]), 1 + kFoldWarps);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&a_full[i]), kUnpackThreads);
            mbar_init(smem_u32(&done[i]), 1);
            mbar_init(smem_u32(&folded[i]), kFoldThreads);
        }
        mbar_init(smem_u32(&drained), 1);
        abort_word = never_word = 0;
        mbar_init_fence();
    }
    if (warp == kWorkWarps + 1) tmem_alloc(smem_u32(&tmem_word), S::kCols);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_word;
    auto wait = [&](uint64_t &b, uint32_t parity) {
        const bool ok = mbar_wait_bounded(smem_u32(&b), parity & 1u, abort_flag, kWaitLimitNs);
        if (!ok) *abort_flag = 1;
        return ok;
    };
    const int quarter = warp & 3, side = warp >> 2 & 1, row = quarter * 32 + lane;   // of a thread that unpacks or folds

    if (warp == kWorkWarps || warp == kWorkWarps + 3) {
        // ---- codes: two warps with half of the rows each, 16 bytes a lane, 4 rows at a time (rows behind the last: the last,
        // never written).  Weights are read before the tokens' kernel is waited for: it began when all before it had ended.
        // (Bulk copies of a row's 128 bytes each would take as long as 60 clocks apiece.)
        const int half = (warp - kWorkWarps) / 3 * 64, mine = row0 + half + (lane >> 3);
        const uint8_t *from = p.w.codes + col0 / 2 + (lane & 7) * 16;
        uint32_t to = smem_at + S::kOffCodes + (half + (lane >> 3)) * kPitch + (lane & 7) * 16;
        for (int c = 0; c < n_chunks; ++c) {
            const int slot = c % kChunks;
            if (c >= kChunks && !__all_sync(~0u, wait(c_empty[slot], c / kChunks - 1))) break;
            if (col0 + c * kChunkCols + (lane & 7) * 32 < p.w.k) {   // (of columns behind the last any codes will do)
                const uint8_t *src = from + c * (kChunkCols / 2);
                const uint32_t dst = to + slot * kChunkBytes;
                if (row0 + kRows <= p.w.n) {
                    src += mine * p.w.code_stride;
#pragma unroll
                    for (int r = 0; r < 16; ++r, src += 4 * p.w.code_stride) copy16_async(dst + r * 4 * kPitch, src, 16);
                } else {
#pragma unroll 4
                    for (int r = 0; r < 16; ++r)
                        copy16_async(dst + r * 4 * kPitch, src + min(mine + 4 * r, p.w.n - 1) * p.w.code_stride, 16);
                }
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(&c_full[slot])) : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp == kWorkWarps + 2) {
        // ---- operands of the tokens
        grid_dependency_wait();
        if (lane == 0)
            for (int s = 0; s < n_stages; ++s) {
                const int slot = s % kBStages;
                if (s >= kBStages && !wait(b_empty[slot], s / kBStages - 1)) break;
                constexpr int kBytes = stage_bytes(GROUP, N);
                mbar_expect_tx(smem_u32(&b_full[slot]), kBytes);
                bulk_load(smem_at + S::kOffB + slot * kBStage, p.image + ((int64_t)tile * p.stages + s0 + s) * kBytes, kBytes,
                          smem_u32(&b_full[slot]));
            }
    } else if (warp == kWorkWarps + 1) {
        // ---- products
        if (lane == 0) {
            const uint32_t idesc = umma_idesc(0, N);
            for (int s = 0; s < n_stages; ++s) {
                const int b = s & 1, slot = s % kBStages;
                if (!(wait(b_full[slot], s / kBStages) && wait(a_full[b], s >> 1) && (s < 2 || wait(folded[b], (s >> 1) - 1)))) break;
                tc_fence_after_sync();
                const uint32_t as = smem_at + b * kAStage, bs = smem_at + S::kOffB + slot * kBStage;
#pragma unroll
                for (int ks = 0; ks < kStageCols / 16; ++ks)
                    umma_ss(tmem + (b * kGroups + ks * 16 / GROUP) * N, umma_desc_k128(as + (ks >> 2) * (kRows * 128) + (ks & 3) * 32),
                            umma_desc_k128(bs + (ks >> 2) * (N * 128) + (ks & 3) * 32), idesc, ks * 16 % GROUP != 0);
                umma_commit(smem_u32(&b_empty[slot]));
                umma_commit(smem_u32(&done[b]));
            }
            umma_commit(smem_u32(&drained));   // before tensor memory is given back
            if (!mbar_wait_bounded(smem_u32(&drained), 0, &never_word, kWaitLimitNs)) *abort_flag = 1;
        }
    } else if (warp < kUnpackWarps) {
        // ---- unpacking
        uint8_t *to = smem + side * (kRows * 128) + row * 128;
        const uint8_t *from = smem + S::kOffCodes + row * kPitch + side * 32;
        int slot = 0;
        uint32_t round = 0;
        for (int s = 0; s < n_stages; ++s) {
            const int b = s & 1;
            if (!b) wait(c_full[slot], round);
            if (s > 1) wait(done[b], (s - 2) >> 1);   // its products have read the operand that was there
            __syncwarp();
            const uint4 v[2] = {*reinterpret_cast<const uint4 *>(from + slot * kChunkBytes + b * 64),
                                *reinterpret_cast<const uint4 *>(from + slot * kChunkBytes + b * 64 + 16)};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t u = w[j] >> 8;
                    *reinterpret_cast<uint4 *>(to + b * kAStage + (((i * 4 + j) ^ (row & 7)) << 4)) =
                        make_uint4(w[j] & 0x000f000fu, w[j] & 0x00f000f0u, u & 0x000f000fu, u & 0x00f000f0u);
                }
            }
            fence_proxy_async();
            mbar_arrive(smem_u32(&a_full[b]));
            if (b || s + 1 == n_stages) {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c_empty[slot]));
                if (++slot == kChunks) {
                    slot = 0;
                    round ^= 1u;
                }
            }
        }
    } else {
        // ---- folding.  Scales of a chunk's groups go to shared memory as pairs; a thread brings kPairs of them, a chunk ahead in
        // registers, into one of three buffers (the one before the last may still be read).
        constexpr int kChunkGroups = kChunkCols / GROUP, kPairs = kChunkGroups * kRows / kFoldThreads;
        const bool wide = p.w.meta_dtype == STOM_FP32, narrow_bf = p.w.meta_dtype == STOM_BF16;
        const int ft = tid - kUnpackThreads, r0 = ft / kChunkGroups, q0 = ft % kChunkGroups;   // of a thread's first pair
        uint32_t rs[kPairs], rz[kPairs];
        auto load_meta = [&](int c) {
            const int gr = (col0 + c * kChunkCols) / GROUP + q0;
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                rs[i] = rz[i] = 0;
                if (c >= n_chunks || gr >= p.w.groups) continue;
                const int64_t at = min(row0 + r0 + i * (kFoldThreads / kChunkGroups), p.w.n - 1) * p.w.meta_stride + gr;
                if (wide) {
                    rs[i] = __ldg(static_cast<const uint32_t *>(p.w.scale) + at);
                    if (p.w.zero) rz[i] = __ldg(static_cast<const uint32_t *>(p.w.zero) + at);
                } else {
                    rs[i] = __ldg(static_cast<const uint16_t *>(p.w.scale) + at);
                    if (p.w.zero) rz[i] = __ldg(static_cast<const uint16_t *>(p.w.zero) + at);
                }
            }
        };
        auto number = [&](uint32_t bits) {
            return wide ? __uint_as_float(bits) : narrow_bf ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
        };
        uint64_t acc[kOwn / 2];   // two tokens each
#pragma unroll
        for (int i = 0; i < kOwn / 2; ++i) acc[i] = 0;
        load_meta(0);
        int b_slot = 0, m_slot = 0;
        uint32_t b_round = 0;
        for (int s = 0; s < n_stages; ++s) {
            const int b = s & 1;
            if (!b) {
                float2 *meta = reinterpret_cast<float2 *>(smem + S::kOffMeta + m_slot * S::kMeta) + q0 * kRows + r0;
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float scale = number(rs[i]);
                    meta[i * (kFoldThreads / kChunkGroups)] = make_float2(kCodeUnit * scale, p.w.zero ? number(rz[i]) : -8.f * scale);
                }
                load_meta((s >> 1) + 1);
                named_sync(1, kFoldThreads);
            }
            wait(b_full[b_slot], b_round);
            wait(done[b], s >> 1);   // (a wait that has failed: what is there is used, and the call flagged)
            __syncwarp();
            tc_fence_after_sync();
            const float2 *meta = reinterpret_cast<const float2 *>(smem + S::kOffMeta + m_slot * S::kMeta) + b * kGroups * kRows + row;
            const ulonglong2 *fx = reinterpret_cast<const ulonglong2 *>(smem + S::kOffB + b_slot * kBStage + N * kStageCols * 2 + side * kOwn * 4);
#pragma unroll
            for (int q = 0; q < kGroups; ++q) {
                float d[kOwn];
                tmem_load(tmem + ((uint32_t)(32 * quarter) << 16) + (b * kGroups + q) * N + side * kOwn, d);
                if (q == kGroups - 1) {
                    tc_fence_before_sync();
                    mbar_arrive(smem_u32(&folded[b]));
                }
                const float2 f = meta[q * kRows];
                const uint64_t fs = pair_of(f.x, f.x), fz = pair_of(f.y, f.y);
#pragma unroll
                for (int i = 0; i < kOwn; i += 4) {
                    const ulonglong2 x = fx[(q * N + i) / 4], y = fx[((kGroups + q) * N + i) / 4];   // factors, sums of four tokens
                    acc[i / 2] = fma_pair(fz, y.x, fma_pair(fs, mul_pair(pair_of(d[i], d[i + 1]), x.x), acc[i / 2]));
                    acc[i / 2 + 1] = fma_pair(fz, y.y, fma_pair(fs, mul_pair(pair_of(d[i + 2], d[i + 3]), x.y), acc[i / 2 + 1]));
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_empty[b_slot]));
            if (++b_slot == kBStages) {
                b_slot = 0;
                b_round ^= 1u;
            }
            if (b && ++m_slot == 3) m_slot = 0;
        }
        // sums to where the left operand was: its products are done
        float *out = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int i = 0; i < kOwn / 2; ++i) {
            float u, v;
            parts_of(acc[i], u, v);
            out[(side * kOwn + 2 * i) * S::kPitchOut + row] = u;
            out[(side * kOwn + 2 * i + 1) * S::kPitchOut + row] = v;
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag && p.w.flags) atomicOr(p.w.flags, STOM_FLAG_TIMEOUT);
    if (warp == kWorkWarps + 1) tmem_dealloc(tmem, S::kCols);
    grid_dependency_wait();
    cluster_sync();   // every block's sums are there
    // a block of the cluster joins every split-th token
    const float *out = reinterpret_cast<const float *>(smem);
    constexpr int kSides = kWorkWarps / 4;
    if (tid < kWorkWarps * 32) {
        const int r = tid & (kRows - 1), at_row = row0 + r;
        for (int i = rank + (tid >> 7) * p.split; i < N; i += kSides * p.split) {
            const int tok = tile * N + i;
            if (tok >= p.w.tokens || at_row >= p.w.n) continue;
            float y = 0.f;
            for (int b = 0; b < p.split; ++b) y += ld_cluster_f(out + i * S::kPitchOut + r, b);
            if (p.w.bias) y += to_float(static_cast<const T *>(p.w.bias)[at_row]);
            if (p.w.add) y += to_float(static_cast<const T *>(p.w.add)[tok * p.w.add_stride + at_row]);
            static_cast<T *>(p.w.y)[tok * p.w.y_stride + at_row] = from_float<T>(y);
        }
    }
    cluster_sync();   // nobody reads this block's sums any more
}

int tokens_of_tile(int tokens) { return tokens <= 16 ? 16 : tokens <= 32 ? 32 : 64; }

// Blocks that share out the columns: the number for which the longest-working multiprocessor has the fewest stages to go
// through (a block's beginning and end count for about six).  room[i]: clusters of i + 1 blocks that the device holds at once
// (fewer than its multiprocessors would do: a cluster lies within one of its parts).
int split_of(int stages, int64_t tiles, const int (&room)[8]) {
    int best = 1;
    int64_t least = INT64_MAX;
    for (int split = 1; split <= 8 && split <= stages; ++split) {
        if (room[split - 1] < 1) continue;
        const int64_t rounds = (tiles + room[split - 1] - 1) / room[split - 1], cost = rounds * ((stages + split - 1) / split + 6);
        if (cost < least) {
            least = cost;
            best = split;
        }
    }
    return best;
}

template <typename T, int GROUP, int N>
cudaError_t launch(ManyParams &p, cudaStream_t s) {
    const int row_tiles = (p.w.n + kRows - 1) / kRows, tiles = (p.w.tokens + N - 1) / N;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(w4_many_kernel<T, GROUP, N>), Many<GROUP, N>::kSmem, allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = Many<GROUP, N>::kSmem;
    lc.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    // what a device holds does not change: asked for once
    static std::atomic<int> known[64][8];
    int dev = 0, room[8];
    e = cudaGetDevice(&dev);
    for (int i = 0; i < 8 && e == cudaSuccess; ++i) {
        room[i] = dev < 64 ? known[dev][i].load(std::memory_order_relaxed) : 0;
        if (room[i]) continue;
        at[0].val.clusterDim.x = i + 1;
        lc.gridDim = dim3(i + 1);
        lc.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&room[i], w4_many_kernel<T, GROUP, N>, &lc);
        if (room[i] < 1) room[i] = -1;
        if (dev < 64) known[dev][i].store(room[i], std::memory_order_relaxed);
    }
    if (e != cudaSuccess) return e;
    p.split = split_of(p.stages, (int64_t)row_tiles * tiles, room);
    const int warps = tiles * N * ((p.stages + 1) / 2);
    e = launch_after_producer(w4_tokens_kernel<T, GROUP, N>, dim3((warps + 7) / 8), dim3(256), 0, s, p);
    if (e != cudaSuccess) return e;
    lc.gridDim = dim3(p.split, row_tiles, tiles);
    at[0].val.clusterDim.x = p.split;
    lc.numAttrs = 2;
    return cudaLaunchKernelEx(&lc, w4_many_kernel<T, GROUP, N>, p);
}

template <typename T, int GROUP>
cudaError_t by_tokens(ManyParams &p, cudaStream_t s) {
    const int n = tokens_of_tile(p.w.tokens);
    return n == 16 ? launch<T, GROUP, 16>(p, s) : n == 32 ? launch<T, GROUP, 32>(p, s) : launch<T, GROUP, 64>(p, s);
}

}  // namespace

int64_t w4_many_workspace(int32_t k, int32_t group, int32_t tokens) {
    const int64_t n = tokens_of_tile(tokens);
    return (tokens + n - 1) / n * ((k + kStageCols - 1) / kStageCols) * stage_bytes(group, (int)n);
}

template <typename T>
cudaError_t w4_many(const W4Params &w, int group, void *workspace, cudaStream_t s) {
    ManyParams p = {};
    p.w = w;
    p.stages = (w.k + kStageCols - 1) / kStageCols;
    p.image = static_cast<uint8_t *>(workspace);
    return group == 32 ? by_tokens<T, 32>(p, s) : group == 64 ? by_tokens<T, 64>(p, s) : by_tokens<T, 128>(p, s);
}
template cudaError_t w4_many<__nv_bfloat16>(const W4Params &, int, void *, cudaStream_t);
template cudaError_t w4_many<__half>(const W4Params &, int, void *, cudaStream_t);

}  // namespace stom
