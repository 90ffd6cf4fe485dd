// Products of many tokens with 4-bit weights (stom_w4_linear): from about as many tokens on as a fragment has, the multiplying
// is done by the fifth-generation tensor cores.
//
// What bounds it: at 16 tokens the codes' bytes, as for one; at 64 the instructions that make operands of them and that
// scale the groups' sums.  A first small kernel makes operands of the tokens, once for all blocks (see stom_w4.cuh): the tiles
// of the right operand as they lie in shared memory, 128-byte-swizzled, and a factor and a sum for each token and group.
//
// A block has 128 rows of the matrix, N tokens and a part of the columns, a STAGE of 128 of them at a time.  Codes arrive by
// 16-byte asynchronous copies, 256 columns at a time, several ahead.  Eight warps unpack: a thread has one row and half of a
// stage's columns, 8 words that become 32 registers of the left operand, in tensor memory where the accumulators leave room for
// it (all but 64 tokens with groups of 32: there in shared memory, K-major, 128-byte swizzle).  Shared memory's bandwidth is
// then left to codes and tokens.  One thread issues the products, each group into accumulators of its own in tensor memory,
// since scales differ from group to group.  Eight more warps fold those of the stage before into sums while the products of this
// one run: a thread has a row again, and half of the tokens.
//
// Split.  The work is one line of stages, tile by tile (128 rows, N tokens), and every block, one a multiprocessor, takes an
// equal, contiguous stretch of it.  The sums of a tile that is cut by a stretch's end go to the workspace, and a third small
// kernel joins them.
//
// Measured on one B200, us: 64 tokens of 3 584 x 14 336 31 (0.2 PFLOP/s, 1 TB/s), 13 of 10 007 x 8 192 in groups of 32 38.  8 to 9
// of them are the small kernels and launches.  A stage takes about 1 400 cycles, which the issuing thread (1 200) and the folding
// warps (1 400: 700 of them the sums, 80 their way out of tensor memory, the rest waits and scales) share.  The left operand in
// shared memory: 33 and 43 us; sixteen folding warps: 31.6 and 38.4.  Codes as bulk copies of a row's 128 bytes: 58 cycles each,
// 7 400 a stage.
#include "stom_tensor.cuh"
#include "stom_w4.cuh"

namespace stom {

namespace {

constexpr int kRows = 128, kStageCols = 128;
constexpr int kUnpackWarps = 8, kFoldWarps = 8, kWorkWarps = kUnpackWarps + kFoldWarps;
constexpr int kUnpackThreads = kUnpackWarps * 32, kFoldThreads = kFoldWarps * 32, kThreads = (kWorkWarps + 4) * 32;
constexpr int kChunkCols = 256;                           // columns of a copy
constexpr int kPitch = kChunkCols / 2 + 16, kChunkBytes = kRows * kPitch;   // an odd number of 16 bytes: a row a thread without conflicts
constexpr int kAStage = kRows * kStageCols * 2, kLeftCols = kStageCols / 2, kMostBStages = 6;
constexpr int kMostShared = 226 * 1024;                   // dynamic shared memory of a block
constexpr int kMaxBlocks = 256;                            // blocks of the grid the workspace has room for
constexpr unsigned long long kWaitLimitNs = 1000000000ull;   // a wait that has taken 1 s fails, and with it
// all later ones of the block, which ends; sums go on to the end of their part without waiting

// Bytes of a stage's operand of the tokens, factors and sums
__host__ __device__ constexpr int stage_bytes(int group, int n) { return n * kStageCols * 2 + kStageCols / group * n * 8; }

struct ManyParams {
    W4Params w;
    uint8_t *image;        // [token tile][stage]: operand [2][N][128 bytes], factors [group][N], sums [group][N]
    float *part;           // [block][2][N][128]: sums of the tile that came in from the block before, and of the one that goes on
    int32_t stages;        // of 128 columns, of a tile
    int32_t row_tiles, blocks;
    int64_t per, total;    // stages of a block, of all
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
    // scales and offsets of a chunk's groups as pairs, a row of kRows for each group and kMetaPad more, with which the pairs that
    // half a warp stores (of adjacent groups and rows) lie in banks of their own
    static constexpr int kChunkGroups = kChunkCols / GROUP, kMetaPad = 16 / kChunkGroups, kMetaRow = kRows + kMetaPad;
    static constexpr int kMeta = kChunkGroups * kMetaRow * 8;
    // the left operand, 64 columns a stage, lies in tensor memory beside the accumulators where it has room for two stages of both
    static constexpr bool kLeftInTmem = 2 * (kGroups * N + kLeftCols) <= 512;
    static constexpr int kStageTmem = kGroups * N + (kLeftInTmem ? kLeftCols : 0);
    static constexpr int kBufs = 3 * kStageTmem <= 512 ? 3 : 2, kChunks = N == 64 && !kLeftInTmem ? 3 : 4;
    static constexpr int kCols = kBufs * kStageTmem <= 256 ? 256 : 512;   // (a power of two of them; there is one block a multiprocessor)
    static constexpr int kLeftAt = kBufs * kGroups * N, kLeftShared = kLeftInTmem ? 0 : kBufs * kAStage;
    static constexpr int kFixed = 1024 + kLeftShared + kChunks * kChunkBytes + 3 * kMeta;
    // of the right operand as many as fit: they are given back only when the sums have been folded, and come again from L2 (13 tokens,
    // 8 192 columns, groups of 32: 42.7 us instead of 43.4 with three)
    static constexpr int kFit = (kMostShared - kFixed) / kBStage, kBStages = kFit < kMostBStages ? kFit : kMostBStages;
    static constexpr int kOffB = kLeftShared, kOffCodes = kOffB + kBStages * kBStage, kOffMeta = kOffCodes + kChunks * kChunkBytes;
    static constexpr int kSmem = kFixed + kBStages * kBStage;
    static_assert(kBStages >= 3 && kSmem <= kMostShared, "room");
};

// A part of a block's stretch: stages first ... first + n - 1 of a tile
struct Part {
    int32_t tile, row0, first, n;
    bool whole;
};
__device__ __forceinline__ Part part_at(const ManyParams &p, int64_t at, int64_t end) {
    const int64_t tile = at / p.stages;
    Part r;
    r.first = (int32_t)(at - tile * p.stages);
    r.n = (int32_t)min((int64_t)(p.stages - r.first), end - at);
    r.whole = r.n == p.stages;
    r.tile = (int32_t)(tile / p.row_tiles);                       // of tokens
    r.row0 = (int32_t)(tile - (int64_t)r.tile * p.row_tiles) * kRows;
    return r;
}
// Slots of a ring and the parity of the round
struct Ring {
    int slot = 0;
    uint32_t round = 0;
    __device__ __forceinline__ void next(int slots) {
        if (++slot == slots) {
            slot = 0;
            round ^= 1u;
        }
    }
};

template <typename T>
__device__ __forceinline__ void put(const W4Params &w, int tok, int row, float y) {
    if (w.bias) y += to_float(static_cast<const T *>(w.bias)[row]);
    if (w.add) y += to_float(static_cast<const T *>(w.add)[tok * w.add_stride + row]);
    static_cast<T *>(w.y)[tok * w.y_stride + row] = from_float<T>(y);
}

template <typename T, int GROUP, int N>
__global__ void __launch_bounds__(kThreads, 1) w4_many_kernel(const __grid_constant__ ManyParams p) {
    using S = Many<GROUP, N>;
    constexpr int kGroups = S::kGroups, kBStage = S::kBStage, kOwn = N / 2;   // tokens of a thread that folds
    constexpr int kBufs = S::kBufs, kChunks = S::kChunks, kBStages = S::kBStages;
    extern __shared__ uint8_t raw_smem[];
    // ready: a stage's left operand is there, and the accumulators' sums of the stage before in that place have been read
    __shared__ uint64_t c_full[kChunks], c_empty[kChunks], b_full[kBStages], b_empty[kBStages], ready[kBufs], done[kBufs], drained;
    __shared__ uint32_t tmem_word, abort_word, never_word;   // never_word stays 0
    uint8_t *smem = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);   // the swizzle goes by addresses
    const uint32_t smem_at = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t begin = min(p.total, blockIdx.x * p.per), end = min(p.total, begin + p.per);
    volatile uint32_t *abort_flag = &abort_word;
    if (tid == 0) {
        for (int i = 0; i < kChunks; ++i) mbar_init(smem_u32(&c_full[i]), 64), mbar_init(smem_u32(&c_empty[i]), kUnpackWarps);
        for (int i = 0; i < kBStages; ++i) mbar_init(smem_u32(&b_full[i]), 1), mbar_init(smem_u32(&b_empty[i]), kFoldWarps);
        for (int i = 0; i < kBufs; ++i) {
            mbar_init(smem_u32(&ready[i]), kUnpackWarps + kFoldWarps);
            mbar_init(smem_u32(&done[i]), 1);
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
        const bool ok = mbar_wait_bounded(smem_u32(&b), parity, abort_flag, kWaitLimitNs);
        if (!ok) *abort_flag = 1;
        return ok;
    };
    const int quarter = warp & 3, side = warp >> 2 & 1, row = quarter * 32 + lane;   // of a thread that unpacks or folds

    if (warp == kWorkWarps || warp == kWorkWarps + 3) {
        // ---- codes: two warps with half of the rows each, 16 bytes a lane, 4 rows at a time (rows behind the last: the last,
        // never written).  Weights are read before the tokens' kernel is waited for: it began when all before it had ended.
        // (Bulk copies of a row's 128 bytes each take about 58 cycles apiece.)
        const int mine = (warp - kWorkWarps) / 3 * 64 + (lane >> 3);
        const uint32_t to = smem_at + S::kOffCodes + mine * kPitch + (lane & 7) * 16;
        Ring c;
        bool again = false, live = true;
        for (int64_t at = begin; at < end && live;) {
            const Part part = part_at(p, at, end);
            at += part.n;
            const bool full_rows = part.row0 + kRows <= p.w.n;
            const uint8_t *from = p.w.codes + (part.row0 + mine) * p.w.code_stride + (lane & 7) * 16;
            for (int s = 0; s < part.n; s += 2) {
                if (again && !(live = __all_sync(~0u, wait(c_empty[c.slot], c.round ^ 1u)))) break;
                const int col = (part.first + s) * kStageCols;
                if (col + (lane & 7) * 32 < p.w.k && (s + 1 < part.n || (lane & 7) < 4)) {   // (behind the last any codes will do)
                    const uint32_t dst = to + c.slot * kChunkBytes;
                    if (full_rows) {
                        const uint8_t *src = from + col / 2;
#pragma unroll
                        for (int r = 0; r < 16; ++r, src += 4 * p.w.code_stride) copy16_async(dst + r * 4 * kPitch, src, 16);
                    } else {
#pragma unroll 4
                        for (int r = 0; r < 16; ++r)
                            copy16_async(dst + r * 4 * kPitch,
                                         p.w.codes + min(part.row0 + mine + 4 * r, p.w.n - 1) * p.w.code_stride + (lane & 7) * 16 + col / 2, 16);
                    }
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(&c_full[c.slot])) : "memory");
                c.next(kChunks);
                again |= c.slot == 0;
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp == kWorkWarps + 2) {
        // ---- operands of the tokens
        grid_dependency_wait();
        if (lane == 0) {
            Ring b;
            bool again = false, live = true;
            for (int64_t at = begin; at < end && live;) {
                const Part part = part_at(p, at, end);
                at += part.n;
                constexpr int kBytes = stage_bytes(GROUP, N);
                const uint8_t *from = p.image + ((int64_t)part.tile * p.stages + part.first) * kBytes;
                for (int s = 0; s < part.n; ++s, from += kBytes) {
                    if (again && !(live = wait(b_empty[b.slot], b.round ^ 1u))) break;
                    mbar_expect_tx(smem_u32(&b_full[b.slot]), kBytes);
                    bulk_load(smem_at + S::kOffB + b.slot * kBStage, from, kBytes, smem_u32(&b_full[b.slot]));
                    b.next(kBStages);
                    again |= b.slot == 0;
                }
            }
            // copies on their way arrive before the block ends: each slot's last, of this turn of the ring or of the one before
            for (int i = 0; i < kBStages; ++i)
                if ((i < b.slot || again) &&
                    !mbar_wait_bounded(smem_u32(&b_full[i]), i < b.slot ? b.round : b.round ^ 1u, &never_word, kWaitLimitNs))
                    *abort_flag = 1;
        }
    } else if (warp == kWorkWarps + 1) {
        // ---- products
        if (lane == 0) {
            const uint32_t idesc = umma_idesc(0, N), a_low = umma_low_k128(smem_at), b_low = umma_low_k128(smem_at + S::kOffB);
            Ring a, b;
            for (int64_t s = begin; s < end; ++s) {
                if (!(wait(b_full[b.slot], b.round) && wait(ready[a.slot], a.round))) break;
                tc_fence_after_sync();
                const uint32_t al = a_low + a.slot * (kAStage / 16), bl = b_low + b.slot * (kBStage / 16), to = tmem + a.slot * (kGroups * N),
                               at = tmem + S::kLeftAt + a.slot * kLeftCols;
#pragma unroll
                for (int ks = 0; ks < kStageCols / 16; ++ks)
                    if constexpr (S::kLeftInTmem)
                        umma_ts_low(to + ks * 16 / GROUP * N, at + ks * 8, bl + (ks >> 2) * (N * 8) + (ks & 3) * 2, idesc, ks * 16 % GROUP != 0);
                    else
                        umma_ss_low(to + ks * 16 / GROUP * N, al + (ks >> 2) * (kRows * 8) + (ks & 3) * 2,
                                    bl + (ks >> 2) * (N * 8) + (ks & 3) * 2, idesc, ks * 16 % GROUP != 0);
                umma_commit(smem_u32(&done[a.slot]));
                a.next(kBufs);
                b.next(kBStages);
            }
            umma_commit(smem_u32(&drained));   // before tensor memory is given back
            if (!mbar_wait_bounded(smem_u32(&drained), 0, &never_word, kWaitLimitNs)) *abort_flag = 1;
        }
    } else if (warp < kUnpackWarps) {
        // ---- unpacking
        uint8_t *to = smem + side * (kRows * 128) + row * 128;
        const uint8_t *from = smem + S::kOffCodes + row * kPitch + side * 32;
        Ring a, c;
        bool again = false;
        bool live = true;
        for (int64_t at = begin; at < end && live;) {
            const int n = part_at(p, at, end).n;
            at += n;
            for (int s = 0; s < n; ++s) {
                const bool there = (s & 1) || wait(c_full[c.slot], c.round);
                const bool left = !again || wait(done[a.slot], a.round ^ 1u);   // its products have read the operand that was there
                if (!(live = __all_sync(~0u, there && left))) break;
                const uint8_t *src = from + c.slot * kChunkBytes + (s & 1) * 64;
                uint8_t *dst = to + a.slot * kAStage;
                uint32_t w[8], o[32];
                *reinterpret_cast<uint4 *>(w) = *reinterpret_cast<const uint4 *>(src);
                *reinterpret_cast<uint4 *>(w + 4) = *reinterpret_cast<const uint4 *>(src + 16);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t u = w[j] >> 8;
                    o[j * 4] = w[j] & 0x000f000fu;
                    o[j * 4 + 1] = w[j] & 0x00f000f0u;
                    o[j * 4 + 2] = u & 0x000f000fu;
                    o[j * 4 + 3] = u & 0x00f000f0u;
                }
                if constexpr (S::kLeftInTmem) {
                    tc_fence_after_sync();
                    tmem_store(tmem + ((uint32_t)(32 * quarter) << 16) + S::kLeftAt + a.slot * kLeftCols + side * 32, o);
                    tmem_wait_store();
                    tc_fence_before_sync();
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4 *>(dst + ((j ^ (row & 7)) << 4)) = make_uint4(o[j * 4], o[j * 4 + 1], o[j * 4 + 2], o[j * 4 + 3]);
                    fence_proxy_async();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ready[a.slot]));
                a.next(kBufs);
                again |= a.slot == 0;
                if ((s & 1) || s + 1 == n) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c_empty[c.slot]));
                    c.next(kChunks);
                }
            }
        }
    } else {
        // ---- folding.  Scales of a chunk's groups go to shared memory as pairs; a thread brings kPairs of them, a chunk ahead in
        // registers, into one of three buffers (the one before the last may still be read).
        constexpr int kChunkGroups = S::kChunkGroups, kPairs = kChunkGroups * kRows / kFoldThreads, kPairRows = kFoldThreads / kChunkGroups;
        const bool wide = p.w.meta_dtype == STOM_FP32, half = p.w.meta_dtype == STOM_FP16, offsets = p.w.zero != nullptr;
        const void *zero = offsets ? p.w.zero : p.w.scale;
        const int ft = tid - kUnpackThreads, r0 = ft / kChunkGroups, q0 = ft % kChunkGroups;   // of a thread's first pair
        uint32_t rs[kPairs], rz[kPairs];
        auto load_meta = [&](const Part &part, int s) {
            const int gr = (part.first + s) * kGroups + q0;
            const bool is = gr < p.w.groups;
            int64_t at[kPairs];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) at[i] = min(part.row0 + r0 + i * kPairRows, p.w.n - 1) * p.w.meta_stride + gr;
            if (wide) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    rs[i] = is ? __ldg(static_cast<const uint32_t *>(p.w.scale) + at[i]) : 0u;
                    rz[i] = is ? __ldg(static_cast<const uint32_t *>(zero) + at[i]) : 0u;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    rs[i] = is ? __ldg(static_cast<const uint16_t *>(p.w.scale) + at[i]) : 0u;
                    rz[i] = is ? __ldg(static_cast<const uint16_t *>(zero) + at[i]) : 0u;
                }
            }
        };
        if (lane == 0)
            for (int i = 0; i < kBufs; ++i) mbar_arrive(smem_u32(&ready[i]));   // no sums are there at first
        Ring a, b;
        int m_slot = 0;
        Part next = part_at(p, begin, end);
        if (begin < end) load_meta(next, 0);
        for (int64_t at = begin; at < end;) {
            if (any_of_some(1, kFoldThreads, *abort_flag != 0)) break;   // all leave together
            const Part part = next;
            at += part.n;
            if (at < end) next = part_at(p, at, end);
            uint64_t acc[kOwn / 2];   // two tokens each
#pragma unroll
            for (int i = 0; i < kOwn / 2; ++i) acc[i] = 0;
            for (int s = 0; s < part.n; ++s) {
                if (!(s & 1)) {
                    float2 *meta = reinterpret_cast<float2 *>(smem + S::kOffMeta + m_slot * S::kMeta) + q0 * S::kMetaRow + r0;
                    float2 v[kPairs];
                    if (half) {
#pragma unroll
                        for (int i = 0; i < kPairs; ++i)
                            v[i] = make_float2(__half2float(__ushort_as_half((unsigned short)rs[i])), __half2float(__ushort_as_half((unsigned short)rz[i])));
                    } else {
                        const int up = wide ? 0 : 16;
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) v[i] = make_float2(__uint_as_float(rs[i] << up), __uint_as_float(rz[i] << up));
                    }
#pragma unroll
                    for (int i = 0; i < kPairs; ++i)
                        meta[i * kPairRows] = make_float2(kCodeUnit * v[i].x, offsets ? v[i].y : -8.f * v[i].x);
                    if (s + 2 < part.n) load_meta(part, s + 2);
                    else if (at < end) load_meta(next, 0);
                    named_sync(1, kFoldThreads);
                }
                wait(b_full[b.slot], b.round);
                wait(done[a.slot], a.round);   // (one that has failed: what is there is used until the part's end, and the call flagged)
                __syncwarp();
                tc_fence_after_sync();
                const float2 *meta = reinterpret_cast<const float2 *>(smem + S::kOffMeta + m_slot * S::kMeta) + (s & 1) * kGroups * S::kMetaRow + row;
                const ulonglong2 *fx = reinterpret_cast<const ulonglong2 *>(smem + S::kOffB + b.slot * kBStage + N * kStageCols * 2 + side * kOwn * 4);
#pragma unroll
                for (int q = 0; q < kGroups; ++q) {
                    float d[kOwn];
                    tmem_load(tmem + ((uint32_t)(32 * quarter) << 16) + (a.slot * kGroups + q) * N + side * kOwn, d);
                    if (q == kGroups - 1) {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&ready[a.slot]));
                    }
                    const float2 f = meta[q * S::kMetaRow];
                    const uint64_t fs = pair_of(f.x, f.x), fz = pair_of(f.y, f.y);
#pragma unroll
                    for (int i = 0; i < kOwn; i += 4) {
                        const ulonglong2 x = fx[(q * N + i) / 4], y = fx[((kGroups + q) * N + i) / 4];   // factors, sums of four tokens
                        acc[i / 2] = fma_pair(fz, y.x, fma_pair(fs, mul_pair(pair_of(d[i], d[i + 1]), x.x), acc[i / 2]));
                        acc[i / 2 + 1] = fma_pair(fz, y.y, fma_pair(fs, mul_pair(pair_of(d[i + 2], d[i + 3]), x.y), acc[i / 2 + 1]));
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_empty[b.slot]));   // (its products are done, too)
                a.next(kBufs);
                b.next(kBStages);
                if (((s & 1) || s + 1 == part.n) && ++m_slot == 3) m_slot = 0;
            }
            grid_dependency_wait();   // (kernels before may read what is written here)
            if (part.whole) {
                if (part.row0 + row < p.w.n)
#pragma unroll
                    for (int i = 0; i < kOwn / 2; ++i) {
                        float u, v;
                        parts_of(acc[i], u, v);
                        const int tok = part.tile * N + side * kOwn + 2 * i;
                        if (tok < p.w.tokens) put<T>(p.w, tok, part.row0 + row, u);
                        if (tok + 1 < p.w.tokens) put<T>(p.w, tok + 1, part.row0 + row, v);
                    }
            } else {
                float *to = p.part + (((int64_t)blockIdx.x * 2 + (part.first == 0 ? 1 : 0)) * N + side * kOwn) * kRows + row;
#pragma unroll
                for (int i = 0; i < kOwn / 2; ++i) {
                    float u, v;
                    parts_of(acc[i], u, v);
                    to[2 * i * kRows] = u;
                    to[(2 * i + 1) * kRows] = v;
                }
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag && p.w.flags) atomicOr(p.w.flags, STOM_FLAG_TIMEOUT);
    if (warp == kWorkWarps + 1) tmem_dealloc(tmem, S::kCols);
}

// Joins the sums of the tiles that are cut: block (i, j) those of the tile in which stretch i + 1 begins, if it is the first to
// begin within it, for 8 tokens; a thread has a row and every second of them.
template <typename T, int N>
__global__ void __launch_bounds__(256) w4_join_kernel(const __grid_constant__ ManyParams p) {
    grid_dependency_wait();
    const int64_t cut = (blockIdx.x + 1) * p.per;
    if (cut >= p.total) return;
    const int64_t tile = cut / p.stages, begin = tile * p.stages, end = begin + p.stages;
    if (cut == begin || cut - p.per > begin) return;   // not cut there, or before as well
    const int tok0 = (int)(tile / p.row_tiles) * N, row0 = (int)(tile % p.row_tiles) * kRows;
    const int r = threadIdx.x & (kRows - 1), first = blockIdx.x, last = (int)((end - 1) / p.per);
    if (row0 + r >= p.w.n) return;
    for (int i = blockIdx.y * 8 + (threadIdx.x >> 7); i < blockIdx.y * 8 + 8 && tok0 + i < p.w.tokens; i += 2) {
        float y = 0.f;
#pragma unroll 4
        for (int b = first; b <= last; ++b) y += p.part[(((int64_t)b * 2 + (b == first ? 1 : 0)) * N + i) * kRows + r];
        put<T>(p.w, tok0 + i, row0 + r, y);
    }
}

int tokens_of_tile(int tokens) { return tokens <= 16 ? 16 : tokens <= 32 ? 32 : 64; }

template <typename T, int GROUP, int N>
cudaError_t launch(ManyParams &p, int sms, cudaStream_t s) {
    const int tiles = (p.w.tokens + N - 1) / N;
    p.row_tiles = (p.w.n + kRows - 1) / kRows;
    p.total = (int64_t)p.row_tiles * tiles * p.stages;
    // (a stretch of fewer than four stages would be all beginning and end)
    p.per = (p.total + sms - 1) / sms;
    if (p.per < 4) p.per = 4;
    p.blocks = (int32_t)((p.total + p.per - 1) / p.per);
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(w4_many_kernel<T, GROUP, N>), Many<GROUP, N>::kSmem, allowed);
    const int warps = tiles * N * ((p.stages + 1) / 2);   // (fewer than 2^31: the workspace has 512 bytes for each)
    if (e == cudaSuccess) e = launch_after_producer(w4_tokens_kernel<T, GROUP, N>, dim3((warps + 7) / 8), dim3(256), 0, s, p);
    if (e == cudaSuccess)
        e = launch_after_producer(w4_many_kernel<T, GROUP, N>, dim3(p.blocks), dim3(kThreads), Many<GROUP, N>::kSmem, s, p);
    if (e == cudaSuccess && p.per % p.stages && p.blocks > 1)
        e = launch_after_producer(w4_join_kernel<T, N>, dim3(p.blocks - 1, N / 8), dim3(256), 0, s, p);
    return e;
}

template <typename T, int GROUP>
cudaError_t by_tokens(ManyParams &p, int sms, cudaStream_t s) {
    const int n = tokens_of_tile(p.w.tokens);
    return n == 16 ? launch<T, GROUP, 16>(p, sms, s) : n == 32 ? launch<T, GROUP, 32>(p, sms, s) : launch<T, GROUP, 64>(p, sms, s);
}

}  // namespace

static int64_t image_bytes(int32_t k, int32_t group, int32_t tokens) {
    const int64_t n = tokens_of_tile(tokens), bytes = (tokens + n - 1) / n * ((k + kStageCols - 1) / kStageCols) * stage_bytes(group, (int)n);
    return (bytes + 255) / 256 * 256;
}

int64_t w4_many_workspace(int32_t k, int32_t group, int32_t tokens) {
    return image_bytes(k, group, tokens) + (int64_t)kMaxBlocks * 2 * tokens_of_tile(tokens) * kRows * 4;
}

template <typename T>
cudaError_t w4_many(const W4Params &w, int group, int sms, void *workspace, cudaStream_t s) {
    ManyParams p = {};
    p.w = w;
    p.stages = (w.k + kStageCols - 1) / kStageCols;
    p.image = static_cast<uint8_t *>(workspace);
    p.part = reinterpret_cast<float *>(p.image + image_bytes(w.k, group, w.tokens));
    if (sms > kMaxBlocks) sms = kMaxBlocks;
    return group == 32 ? by_tokens<T, 32>(p, sms, s) : group == 64 ? by_tokens<T, 64>(p, sms, s) : by_tokens<T, 128>(p, sms, s);
}
template cudaError_t w4_many<__nv_bfloat16>(const W4Params &, int, int, void *, cudaStream_t);
template cudaError_t w4_many<__half>(const W4Params &, int, int, void *, cudaStream_t);

}  // namespace stom
