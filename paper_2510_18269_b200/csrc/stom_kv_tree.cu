// Attention of several new tokens per sequence over a paged cache (stom_kv_attend_tree).
//
//   out_j = sum_t exp(x_jt) V_t / sum_t exp(x_jt),  x_jt = scale <q_j, K_t>, capped if asked for, t over what node j sees.
//
// The query heads of a kv head and the nodes of a sequence together are the ROWS of two products with the same keys and
// values: row r is node r / group, head r % group.  Rows are cut into tiles of 128, the height of a tcgen05 product, and a
// UNIT is one (sequence, row tile, kv head).  What bounds it: a tile of 128 rows does 4 * 128 flops for every pair of a
// key's and a value's elements that it reads, 128 flops a byte, half of what the device's products take for a byte from memory
// (1 640 TFLOP/s over 6.5 TB/s).  One tile of a kv head is bound by the cache's bytes; where several read the same keys (many
// heads times nodes, a question's prefill), they come from L2, and the copies from there, the products and the exponentials share
// the time.
//
// Split.  As for one new token, the work is one line of TILES of tokens (128, or 64 where head_dim is 256): sequence by
// sequence, row tile by row tile, head by head.  Each block, one a multiprocessor, takes an equal, contiguous stretch of it;
// units that a stretch's end cuts are joined by a second kernel over two partial results per block.
//
// A block.  Four warps load: 16-byte asynchronous copies, any page size, any strides, into a ring of tiles of keys and of
// values, each of them in the 128-byte-swizzled layout in which keys are a K-major operand (rows: tokens) and values an
// MN-major one (rows: the summed axis).  One thread issues the products: S = Q K^T of tile t + 3 when the values' product
// of tile t is done, O += P V from tensor memory.  Eight warps do the softmax, two groups in turn with the tiles, a thread with
// one row: while one group waits, the other's exponentials run.  P takes the place of S in tensor memory, as two 16-bit parts.
//
// The running maximum moves only when a row's scores rise by more than 2^8 above it: the weights then are at most 2^8 (no
// loss: they are floating-point numbers, and bf16 has binary32's exponents; in fp16 the reference weight is 2^7, so that
// they end at 2^15 and begin at 2^-24, 2^-31 of it), and the accumulators in tensor memory are rescaled once or twice a unit
// instead of once a tile.  In fp16 it follows falls of more than 2^8, too (down to 2^-48 of the row's largest, so that nothing
// overflows): relative to the largest, weights would vanish where thousands of tokens count only in sum, beside one that stands
// 15 nats above them.  So a weight's error is 2^-32 of the row's largest and 2^-24 of its own tile's at most.
//
// Weights enter the second product as a high and a low part of the pool's type (2^-16 of themselves off in bf16, 2^-22 in fp16
// as long as the low part is above 2^-24): one part alone adds an error of the size of the output's own rounding (0.0023 of the
// output's norm off instead of 0.0017 in bf16, 0.00026 instead of 0.00021 in fp16), and a step of several tokens would answer
// less exactly than one of a single token over the same cache.  The parts of 32 tokens take their scores' 32 columns.  It costs
// the second product again: one tree of 64 nodes 38.4 -> 40.2 us, 48 streams 188 -> 193 to 215, questions 317 to 350 -> 385 to 470.
//
// Masks.  Only tiles that reach the nodes, or a window's edge, are masked: 32 bits a row and 32 columns, from the range of
// the context that the row sees and the bits of its path, which a row walks once per unit.  A product multiplies what a row
// does not see by zero, which is not enough where it is no number: in such tiles the values are looked through, what is no
// number is taken out, and put back afterwards in the rows that see it.
//
// Measured on one B200.  28 + 4 heads of 128, bf16, 12 583 tokens: five nodes 19.6 us, 64 nodes 40 us; 48 streams of 17 to 8 011
// tokens with up to 33 nodes, 64 + 8 heads, fp16: 193 us, 205 to 215 when the device nears its power limit (2.6 to 2.9 of 6.5
// TB/s); questions of 201 to 1 201 tokens over three caches: 385 to 470 us, likewise (0.5 to 0.6 PFLOP/s; the copies of keys and
// values, which every row tile reads again from L2, alone take 306).  Of the 40 us, 3 go to finding the place, 2.5 to page ids,
// tree and rows of q, 2 to the first keys' way, 1.45 to each of 11 tiles, 3 to the partial result, and the rest to launches and
// the second kernel.  With weights of one part a softmax group took 2.6 us for a tile of its own (0.4 until the scores are there,
// 0.6 for the maximum, 1.3 for the exponentials, 0.3 until the product before is done), of which the exponentials' units are busy
// for 0.54; the second part adds 0.3.  With one group instead of two the call took 48 us instead of 42, then.
#include "stom_kv.cuh"
#include "stom_tensor.cuh"

#include <math.h>

#include <type_traits>

namespace stom {

namespace {

constexpr int kRows = 128;            // rows of a tile
constexpr int kMaxBlocks = 256;       // blocks of the grid the workspace has room for
constexpr int kSoftWarps = 8, kLoadWarps = 4, kWarps = kSoftWarps + kLoadWarps + 1;
constexpr int kSoftThreads = kSoftWarps * 32, kLoadThreads = kLoadWarps * 32, kThreads = kWarps * 32;
constexpr int kPathWords = STOM_KV_MAX_TREE / 32;
constexpr int kSBufs = 3;            // buffers of scores: one is multiplied, one or two are in the softmax
constexpr int kUnits = 8;            // descriptions of units that are kept
constexpr int kUnitCost = 2;          // what a unit's beginning and end take, in tiles
constexpr float kSlack = 8.f;         // log2 of what weights may exceed 1 by
constexpr float kFall = 8.f;          // fp16: log2 of what a tile's largest may be below the reference
constexpr float kReach = 48.f;        // and of what the reference may be below the row's largest so far
constexpr unsigned long long kWaitLimitNs = 1000000000ull;   // a wait that has taken 1 s fails, and with
// it all later ones of the block: loads and products end there, the softmax goes on to its unit's end without waiting

// Of a unit that crosses a block's end, for the joining kernel
struct Open {
    int32_t row0, rows, node0, head;  // first row of the tile, rows it has, row of q of the sequence's first node, kv head
};

struct KvTreeParams {
    const char *k, *v;                // at the layer
    int64_t stride_page, stride_token, stride_head;
    const int32_t *table;
    const int32_t *len;
    int64_t table_stride;
    int32_t n_seqs, n_pages, max_tokens;
    FastDiv page;
    int32_t n_kv_heads, group;        // query heads per kv head
    FastDiv by_group;
    int32_t n_tokens;
    const int32_t *first, *parent;
    const char *q;
    int64_t q_stride_token, q_stride_head;
    float scale, cap;
    int32_t window;
    char *out;
    int64_t out_stride_token, out_stride_head;
    float *lse;
    int32_t blocks;                   // of the grid
    int32_t part_rows;                // rows a partial result has room for
    float *part_o;                    // [blocks][2][part_rows][d]
    float2 *part_ml;                  // [blocks][2][part_rows]: maximum and sum
    Open *open;                       // [blocks]: unit that begins in the block and goes on behind it (rows 0: none)
    int32_t *goes_on;                 // [blocks]: the unit that came in from the block before goes on behind this one too
    uint32_t *flags;
};

template <int D>
struct Shape {
    static constexpr int kTok = D == 256 ? 64 : 128;      // tokens of a tile
    static constexpr int kHalf = kTok * D * 2;            // bytes of a tile's keys or values
    static constexpr int kBlock = kTok * 128;             // bytes of 64 channels of them
    static constexpr int kSlots = D == 64 ? 8 : 4;        // tiles of keys or values in the ring
    static constexpr int kSAt = D;                        // column of tensor memory behind the accumulators, where the scores begin
    static constexpr int kQ = kRows * D * 2;
    static constexpr int kQBufs = D == 256 ? 1 : 2;
    static constexpr int kSmem = 1024 + kSlots * kHalf + kQBufs * kQ;
    static_assert(kSmem <= 212 * 1024, "shared memory");
    static_assert(kSAt + kSBufs * kTok <= 512, "tensor memory");
};

// What a unit is, and the part of it that a block has
struct Unit {
    int32_t node0, n, base;           // row of q of the sequence's first node, its nodes, tokens before them
    int32_t seq, head, row0, rows;    // rows: of this tile
    int32_t first, end;               // tokens that some row looks at
    int32_t tile0, tiles;             // the block's part
    int32_t ends;                     // bit 0: it has the unit's first tile, bit 1: its last
};

struct Shared {                       // beside the operands
    uint64_t full[8], empty[8], q_full[2], q_empty[2], unit_full[kUnits], s_full[kSBufs], p_full[kSBufs];
    uint64_t pv_done[2], drained;     // pv_done: of even and odd tiles
    uint32_t tmem, abort, never;      // never: stays 0
    int32_t start_seq, start_tile_row, start_head, start_tile;
    uint64_t warp_sum[kWarps], tiles_before[2];
    uint32_t warp_units[kWarps];
    Unit unit[kUnits];
    uint32_t tokens[8][4];            // per tile: which rows are tokens
    uint32_t dirty[2][4];             // per group: tokens of the tile with values that are no numbers
    float ref[2][kRows];              // per group: its last tile's reference
    float most[2][kRows];             // and (fp16) the row's largest score up to there
    float sum[2][kRows];
    uint32_t path[kRows][kPathWords];
    int16_t parent[kUnits][STOM_KV_MAX_TREE];
};

struct Seq {
    int node0, n, base;
};
// A sequence's nodes; n = 0 if there are none or it does not fit
__device__ __forceinline__ Seq seq_of(const KvTreeParams &p, int i, bool tell = false) {
    const int a = p.first[i], b = p.first[i + 1], raw = p.len[i], len = max(raw, 0), n = b - a;
    const bool good = a >= 0 && a <= b && b <= p.n_tokens && n <= len && (!p.parent || n <= STOM_KV_MAX_TREE);
    if (tell && p.flags && (!good || (n > 0 && raw > p.max_tokens))) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
    return Seq{a, good ? n : 0, len - n};
}
__device__ __forceinline__ int row_tiles(const KvTreeParams &p, int n) {
    return (int)(((int64_t)n * p.group + kRows - 1) / kRows);
}
// Tokens that the rows of a tile look at, and tiles of them (at least one: a unit without any still has an output)
template <int TOK>
__device__ __forceinline__ int span_of(const KvTreeParams &p, const Seq &s, int tile_row, int &first, int &end) {
    const int jf = (int)div_by(p.by_group, (uint32_t)tile_row * kRows);
    const int jl = min(s.n - 1, (int)div_by(p.by_group, (uint32_t)tile_row * kRows + kRows - 1));
    end = min(s.base + jl + 1, p.max_tokens);
    first = p.window > 0 ? min(end, max(0, s.base + (p.parent ? 0 : jf) + 1 - p.window)) : 0;
    return max(1, (end - first + TOK - 1) / TOK);
}

__device__ __forceinline__ void arrive_when_copied(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void sync_some(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void arrive_some(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Which of two 16-bit numbers are no finite ones: bits 15 and 31
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    return ((w & 0x7fff7fffu) + (std::is_same<T, __nv_bfloat16>::value ? 0x00800080u : 0x04000400u)) & 0x80008000u;
}

template <typename T, int D, bool CAP>
__global__ void __launch_bounds__(kThreads, 1) kv_tree_kernel(const __grid_constant__ KvTreeParams p) {
    using S = Shape<D>;
    constexpr int kTok = S::kTok, kHalf = S::kHalf, kBlock = S::kBlock, kSlots = S::kSlots, kQBufs = S::kQBufs;
    constexpr bool kHalfType = std::is_same<T, __half>::value;
    constexpr float kLift = kHalfType ? 7.f : 0.f;   // log2 of the weight of a score at the reference
    constexpr uint32_t kFmt = kHalfType ? 0u : 1u;
    extern __shared__ uint8_t raw_smem[];
    __shared__ Shared sh;
    uint8_t *smem = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);   // the swizzle goes by addresses
    const uint32_t ring_u = smem_u32(smem), q_u = ring_u + kSlots * kHalf;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile uint32_t *abort_flag = &sh.abort;
    auto bar = [&](const uint64_t &b) { return smem_u32(&b); };

    if (tid == 0) {
        for (int i = 0; i < 8; ++i) mbar_init(bar(sh.full[i]), kLoadThreads + kLoadWarps), mbar_init(bar(sh.empty[i]), 1);
        for (int i = 0; i < 2; ++i) mbar_init(bar(sh.q_full[i]), kLoadThreads), mbar_init(bar(sh.q_empty[i]), 1);
        for (int i = 0; i < kUnits; ++i) mbar_init(bar(sh.unit_full[i]), kLoadThreads);
        for (int i = 0; i < kSBufs; ++i) mbar_init(bar(sh.s_full[i]), 1), mbar_init(bar(sh.p_full[i]), kSoftThreads / 2);
        for (int i = 0; i < 2; ++i) mbar_init(bar(sh.pv_done[i]), 1);
        mbar_init(bar(sh.drained), 1);
        sh.abort = sh.never = 0;
        mbar_init_fence();
    }
    if (warp == kWarps - 1) tmem_alloc(smem_u32(&sh.tmem), 512);
    grid_dependency_wait();
    grid_launch_dependents();   // the joining kernel may take its places now; it waits for this grid's end

    // ---- the stretch of this block: where it begins on the line, and how many tiles it has.  On the line, a unit's tiles come
    // behind kUnitCost places for its beginning and end.
    {
        uint64_t *before = reinterpret_cast<uint64_t *>(smem);                          // places before each sequence
        uint32_t *units_before = reinterpret_cast<uint32_t *>(before + STOM_KV_MAX_SEQS);   // and units
        static_assert(kSlots * kHalf >= STOM_KV_MAX_SEQS * 12, "two numbers for each sequence");
        const int seg = (p.n_seqs + kThreads - 1) / kThreads, b0 = tid * seg;   // sequences a thread adds up
        auto places_of = [&](const Seq &s, int tr) {
            int f, e;
            return (uint64_t)span_of<kTok>(p, s, tr, f, e) + kUnitCost;
        };
        uint64_t mine = 0;
        uint32_t mine_units = 0;
        for (int j = 0; j < seg; ++j) {
            const int b = b0 + j;
            Seq s = {0, 0, 0};
            if (b < p.n_seqs) s = seq_of(p, b, blockIdx.x == 0);
            const int trs = row_tiles(p, s.n);
            uint64_t sum = 0;
            if (trs <= 8)
                for (int tr = 0; tr < trs; ++tr) sum += places_of(s, tr);
            // long ones: the warp together
            for (uint32_t many = __ballot_sync(~0u, trs > 8); many; many &= many - 1) {
                const int of = __ffs(many) - 1;
                const Seq o = {0, __shfl_sync(~0u, s.n, of), __shfl_sync(~0u, s.base, of)};
                const int n = __shfl_sync(~0u, trs, of);
                uint64_t part = 0;
                for (int tr = lane; tr < n; tr += 32) part += places_of(o, tr);
#pragma unroll
                for (int x = 16; x; x >>= 1) part += __shfl_xor_sync(~0u, part, x);
                if (lane == of) sum = part;
            }
            if (b < p.n_seqs) {
                before[b] = mine;
                units_before[b] = mine_units;
            }
            mine += sum * p.n_kv_heads;
            mine_units += (uint32_t)trs * p.n_kv_heads;
        }
        uint64_t upto = mine;
        uint32_t upto_units = mine_units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t v = __shfl_up_sync(~0u, upto, o);
            const uint32_t w = __shfl_up_sync(~0u, upto_units, o);
            if (lane >= o) {
                upto += v;
                upto_units += w;
            }
        }
        if (lane == 31) {
            sh.warp_sum[warp] = upto;
            sh.warp_units[warp] = upto_units;
        }
        __syncthreads();
        uint64_t total = 0, ahead = upto - mine;
        uint32_t all_units = 0, ahead_units = upto_units - mine_units;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) {
                ahead += sh.warp_sum[w];
                ahead_units += sh.warp_units[w];
            }
            total += sh.warp_sum[w];
            all_units += sh.warp_units[w];
        }
        for (int j = 0; j < seg && b0 + j < p.n_seqs; ++j) {
            before[b0 + j] += ahead;
            units_before[b0 + j] += ahead_units;
        }
        __syncthreads();
        // (divisions of 64 bits are slow, and the line is rarely that long)
        const uint64_t up = total + gridDim.x - 1;
        const uint64_t per = max((uint64_t)1, up >> 32 ? up / gridDim.x : (uint64_t)((uint32_t)up / gridDim.x));
        if (warp < 2) {
            // warp 0 looks for the stretch's first place, warp 1 for the first behind it: tiles before it, and where it is
            const uint64_t f = min(total, ((uint64_t)blockIdx.x + warp) * per);
            if (f == total) {
                if (lane == 0) sh.tiles_before[warp] = total - (uint64_t)all_units * kUnitCost;
            } else {
                // its sequence: the last that begins there or before (of several, the others are empty)
                int low = 0, high = p.n_seqs;
                while (high - low > 1) {
                    const int step = (high - low + 31) / 32, at = low + step * lane;
                    const uint32_t yes = __ballot_sync(~0u, at < high && before[at] <= f);
                    low += step * (31 - __clz(yes));
                    high = min(high, low + step);
                }
                const Seq s = seq_of(p, low);
                uint64_t in = f - before[low];
                const int trs = row_tiles(p, s.n);
                for (int t0 = 0; t0 < trs; t0 += 32) {
                    const uint64_t n = t0 + lane < trs ? places_of(s, t0 + lane) * p.n_kv_heads : 0;
                    uint64_t sum = n;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const uint64_t v = __shfl_up_sync(~0u, sum, o);
                        if (lane >= o) sum += v;
                    }
                    const uint32_t here = __ballot_sync(~0u, in < sum);
                    if (here) {
                        if (lane == __ffs(here) - 1) {
                            const uint64_t rest = in - (sum - n), each = places_of(s, t0 + lane);
                            const uint64_t head = rest >> 32 ? rest / each : (uint64_t)((uint32_t)rest / (uint32_t)each);
                            const int place = (int)(rest - head * each), tile = max(0, place - kUnitCost);
                            if (warp == 0) {
                                sh.start_seq = low;
                                sh.start_tile_row = t0 + lane;
                                sh.start_head = (int)head;
                                sh.start_tile = tile;
                            }
                            const uint64_t units = units_before[low] + (uint64_t)(t0 + lane) * p.n_kv_heads + head;
                            sh.tiles_before[warp] = f - place - units * kUnitCost + tile;
                        }
                        break;
                    }
                    in -= __shfl_sync(~0u, sum, 31);
                }
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();   // the numbers have been read: operands may take their place
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem;
    const uint32_t n_tiles = (uint32_t)(sh.tiles_before[1] - sh.tiles_before[0]);
    auto wait = [&](const uint64_t &b, uint32_t parity) {
        if (mbar_wait_bounded(bar(b), parity & 1u, abort_flag, kWaitLimitNs)) return true;
        *abort_flag = 1;
        return false;
    };
    // places of a tile's keys and values in the order of loads: K0 K1 K2 V0 K3 V1 ... V(n-1)
    auto half_of_k = [&](uint32_t c) { return c < kSBufs ? c : 2 * c - (kSBufs - 1); };
    auto half_of_v = [&](uint32_t c) { return c + min(c + kSBufs, n_tiles); };
    int open_rows = 0, goes_on = 0;

    if (warp >= kSoftWarps && warp < kSoftWarps + kLoadWarps && n_tiles > 0) {
        // ================================================================ loads
        const int lt = tid - kSoftThreads, lw = warp - kSoftWarps;
        constexpr int kChunks = D / 8;                    // 16-byte chunks of a row
        constexpr int kOwn = kTok / kLoadWarps;           // rows of a tile that a warp copies
        // where the page look-ups are: a tile ahead of the copies
        int seq = sh.start_seq, tr = sh.start_tile_row, head = sh.start_head, tile = sh.start_tile;
        Seq s = seq_of(p, seq);
        int trs = row_tiles(p, s.n), first, end, tiles = span_of<kTok>(p, s, tr, first, end);
        uint32_t to_look = n_tiles;
        constexpr int kNone = INT32_MIN;
        int page = kNone;
        int64_t rest = 0;
        auto look_up = [&]() {
            page = kNone;
            const int t = first + tile * kTok + lw * kOwn + lane % kOwn;
            if (t < end) {
                const uint32_t pg = div_by(p.page, (uint32_t)t);
                rest = (int64_t)(t - (int)(pg * p.page.d)) * p.stride_token + (int64_t)head * p.stride_head;
                page = p.table[seq * p.table_stride + pg];
                if (page == kNone) page = -1;
            }
        };
        auto advance = [&]() {   // to the next tile of the line
            if (++tile < tiles) return;
            tile = 0;
            if (++head < p.n_kv_heads) return;
            head = 0;
            if (++tr >= trs) {
                tr = 0;
                do {                                      // there is one: tiles are left
                    s = seq_of(p, min(++seq, p.n_seqs - 1));
                    trs = row_tiles(p, s.n);
                } while (trs == 0 && seq < p.n_seqs);
            }
            tiles = span_of<kTok>(p, s, tr, first, end);
        };
        uint32_t half = 0, unit = 0;
        bool live = true;
        auto wait_all = [&](const uint64_t &b, uint32_t parity) { return __all_sync(~0u, wait(b, parity)) != 0; };
        // Eight lanes copy 128 bytes of a row, four rows at a time; a lane keeps the offsets of its rows, of this tile for the
        // keys and of the one two before for the values.
        constexpr int kGo = kOwn / 4;                     // rounds of four rows
        int64_t offs[kGo], before1[kGo], before2[kGo];   // (kSBufs - 1 tiles behind)
        const int sub = lane >> 3, piece = lane & 7;
        const uint32_t lane_dst = ring_u + (lw * kOwn + sub) * 128;
        auto copy_half = [&](const char *from, const int64_t (&of)[kGo]) {
            const uint32_t slot = half % kSlots, round = half / kSlots;
            ++half;
            if (round > 0 && !wait_all(sh.empty[slot], round - 1)) return false;
            const uint32_t dst = lane_dst + slot * kHalf;
            const char *src = from + piece * 16;
#pragma unroll
            for (int i = 0; i < kGo; ++i) {
                const uint32_t bytes = of[i] < 0 ? 0u : 16u;
                const char *row = src + (of[i] < 0 ? 0 : of[i]);
                const uint32_t to = dst + i * 512 + ((piece ^ ((i * 4 + sub) & 7)) << 4);   // (a warp's first row is a multiple of 8)
#pragma unroll
                for (int b = 0; b < D / 64; ++b) copy16_async(to + b * kBlock, row + b * 128, bytes);
            }
            arrive_when_copied(bar(sh.full[slot]));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.full[slot]));
            return true;
        };
        look_up();
        for (uint32_t c = 0; c < n_tiles && live; ++c) {
            if (c == 0 || tile == 0) {
                // a unit begins: its description, its parents, its rows of q
                const uint32_t buf = unit % kQBufs, round = unit / kQBufs;
                if (round > 0 && !wait_all(sh.q_empty[buf], round - 1)) {
                    live = false;
                    break;
                }
                const int rows = min(kRows, s.n * p.group - tr * kRows);
                if (lt == 0) {
                    const int part = (int)min((uint32_t)(tiles - tile), to_look);
                    sh.unit[unit % kUnits] = Unit{s.node0, s.n, s.base, seq, head, tr * kRows, rows, first, end, tile, part,
                                             (tile == 0 ? 1 : 0) | (tile + part == tiles ? 2 : 0)};
                }
                if (p.parent)
                    for (int j = lt; j < s.n; j += kLoadThreads) {
                        int up = p.parent[s.node0 + j];
                        if (up < -1 || up >= j) {
                            if (p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
                            up = -1;
                        }
                        sh.parent[unit % kUnits][j] = (int16_t)up;
                    }
                mbar_arrive(bar(sh.unit_full[unit % kUnits]));
                const int sub = lt / kChunks, chunk = lt % kChunks;
#pragma unroll 4
                for (int i = 0; i < kRows * kChunks / kLoadThreads; ++i) {
                    const int r = i * (kLoadThreads / kChunks) + sub, row = tr * kRows + r;
                    const int node = (int)div_by(p.by_group, (uint32_t)row), g = row - node * p.group;
                    const char *src = p.q;
                    if (r < rows)
                        src += 2 * ((s.node0 + node) * p.q_stride_token + (head * p.group + g) * p.q_stride_head) + chunk * 16;
                    copy16_async(q_u + buf * S::kQ + (chunk >> 3) * (kRows * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4), src,
                                 r < rows ? 16u : 0u);
                }
                arrive_when_copied(bar(sh.q_full[buf]));
                ++unit;
            }
            const bool ok = (uint32_t)page < (uint32_t)p.n_pages;
            if (page != kNone && !ok && p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
            const int64_t off = ok ? 2 * (page * p.stride_page + rest) : -1;
#pragma unroll
            for (int i = 0; i < kGo; ++i) {
                before2[i] = before1[i];
                before1[i] = offs[i];
                offs[i] = __shfl_sync(~0u, off, i * 4 + sub);
            }
            const uint32_t is = __ballot_sync(~0u, ok);
            if (lane == 0) {
                if (kOwn == 32) sh.tokens[c & 7][lw] = is;
                else reinterpret_cast<uint16_t *>(sh.tokens[c & 7])[lw] = (uint16_t)is;
            }
            if (--to_look > 0) {
                advance();
                look_up();
            }
            live = copy_half(p.k, offs) && (c < kSBufs - 1 || copy_half(p.v, before2));
        }
        static_assert(kSBufs == 3, "the values' offsets are kept for two tiles");
        if (live && n_tiles > 1) live = copy_half(p.v, before1);
        if (live) copy_half(p.v, offs);
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp == kWarps - 1 && n_tiles > 0) {
        // ================================================================ products
        if (lane == 0) {
            const uint32_t idesc_s = umma_idesc(kFmt, kTok), idesc_o = umma_idesc(kFmt, D) | kUmmaRightMn;
            const uint32_t q_low = umma_low_k128(q_u), k_low = umma_low_k128(ring_u), v_low = umma_low_mn128(ring_u, kBlock);
            uint32_t unit = 0, in_unit = 0, unit_tiles = 0, fresh = 0;   // of the first products; fresh: bit c & 31, a unit begins
            bool live = true;
            auto scores = [&](uint32_t c) {
                const uint32_t k = half_of_k(c), slot = k % kSlots;
                const bool begins = in_unit == unit_tiles;
                if (begins) {
                    if (!wait(sh.unit_full[unit % kUnits], unit / kUnits)) return false;
                    unit_tiles = sh.unit[unit % kUnits].tiles;
                    in_unit = 0;
                    if (!wait(sh.q_full[unit % kQBufs], unit / kQBufs)) return false;
                    ++unit;
                }
                fresh = (fresh & ~(1u << (c & 31))) | ((begins ? 1u : 0u) << (c & 31));
                ++in_unit;
                if (!wait(sh.full[slot], k / kSlots)) return false;
                fence_proxy_async();
                tc_fence_after_sync();
                const uint32_t ql = q_low + ((unit - 1) % kQBufs) * (S::kQ / 16), kl = k_low + slot * (kHalf / 16);
                const uint32_t to = tmem + S::kSAt + c % kSBufs * kTok;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_ss_low(to, ql + (ks >> 2) * (kRows * 8) + (ks & 3) * 2, kl + (ks >> 2) * (kBlock / 16) + (ks & 3) * 2, idesc_s,
                                ks != 0);
                umma_commit(bar(sh.empty[slot]));
                umma_commit(bar(sh.s_full[c % kSBufs]));
                if (in_unit == unit_tiles) umma_commit(bar(sh.q_empty[(unit - 1) % kQBufs]));
                return true;
            };
            for (uint32_t c = 0; c < kSBufs && c < n_tiles && live; ++c) live = scores(c);
            for (uint32_t c = 0; c < n_tiles && live; ++c) {
                const uint32_t v = half_of_v(c), slot = v % kSlots;
                live = wait(sh.full[slot], v / kSlots) && wait(sh.p_full[c % kSBufs], c / kSBufs);
                if (!live) break;
                fence_proxy_async();
                tc_fence_after_sync();
                const uint32_t vl = v_low + slot * (kHalf / 16), pl = tmem + S::kSAt + c % kSBufs * kTok;
                const uint32_t more = !(fresh >> (c & 31) & 1u);
#pragma unroll
                for (int ks = 0; ks < kTok / 16; ++ks) {   // (high parts of 32 tokens' weights lie before their low ones)
                    const uint32_t w = pl + (ks >> 1) * 32 + (ks & 1) * 8;
                    umma_ts_low(tmem, w, vl + ks * 128, idesc_o, more | (ks != 0));
                    umma_ts_low(tmem, w + 16, vl + ks * 128, idesc_o, 1);
                }
                umma_commit(bar(sh.empty[slot]));
                umma_commit(bar(sh.pv_done[c & 1]));
                if (c + kSBufs < n_tiles) live = wait(sh.pv_done[c & 1], c >> 1) && scores(c + kSBufs);   // its S takes P's place
            }
            umma_commit(bar(sh.drained));   // before tensor memory is given back
            if (!mbar_wait_bounded(bar(sh.drained), 0, &sh.never, kWaitLimitNs)) *abort_flag = 1;
        }
    } else if (warp < kSoftWarps && n_tiles > 0) {
        // ================================================================ softmax
        // Two groups of four warps take the tiles in turn, a thread a row.  A tile's reference comes from the group before,
        // which passes it on as soon as it has its own tile's maximum.
        const int quarter = warp & 3, group = warp >> 2, row = quarter * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(32 * quarter) << 16), o_at = lane_base;
        const float log2e = 1.4426950408889634f;
        const float s1 = CAP ? p.scale / p.cap : p.scale * log2e, s2 = p.cap * log2e;
        // A wait that fails (the block has given up) is not a reason to leave the others alone at a barrier: the unit goes on
        // with what is there, and all leave together where the next one begins.
        auto wait_on = [&](const uint64_t &b, uint32_t parity) {
            const bool ok = wait(b, parity);
            __syncwarp();
            return ok;
        };
        // Without a cap and with a positive scale the scores stay unscaled until the exponent, where scaling and the step to
        // the reference are one multiply-add.
        const bool plain = !CAP && s1 > 0.f, falls = s1 < 0.f;   // falls: load_scores gives them with the other sign
        const float s1_abs = fabsf(s1);
        uint32_t c = 0;
        int paths_of_seq = -1, paths_of_row = -1, depth = 0;   // whose paths are in shared memory
        for (uint32_t unit = 0; c < n_tiles; ++unit) {
            // (this barrier also ends the unit before: its accumulators, sums and paths have been read)
            if (any_of_some(5, kSoftThreads, !wait_on(sh.unit_full[unit % kUnits], unit / kUnits))) break;
            const Unit u = sh.unit[unit % kUnits];
            const int at = u.row0 + row, node = (int)div_by(p.by_group, (uint32_t)at);
            const bool is = row < u.rows, some = quarter * 32 < u.rows;
            // the context that the row sees: [begin, until), and with a tree the bits of its path from u.base on
            if (!p.parent) depth = node;
            else if (u.seq != paths_of_seq || u.row0 != paths_of_row) {   // (heads of the same rows have the same)
                paths_of_seq = u.seq;
                paths_of_row = u.row0;
                if (group == 0) {
#pragma unroll
                    for (int w = 0; w < kPathWords; ++w) sh.path[row][w] = 0;
                    depth = 0;
                    if (is)
                        for (int j = node; j >= 0; j = sh.parent[unit % kUnits][j], ++depth)
                            if (!p.window || depth < p.window) sh.path[row][j >> 5] |= 1u << (j & 31);
                    sh.sum[0][row] = __int_as_float(depth - 1);
                }
                sync_some(1 + quarter, 64);
                depth = __float_as_int(sh.sum[0][row]);
            }
            const int begin = !is ? INT32_MAX : p.window > 0 ? max(0, u.base + depth + 1 - p.window) : 0;
            const int until = p.parent ? u.base : u.base + node + 1;
            // tiles before this token (and, with a window, from that one on) are not masked
            const int clean_end = u.n == 1 ? u.end : p.parent ? u.base : u.base + (int)div_by(p.by_group, (uint32_t)u.row0) + 1;
            const int clean_begin = p.window > 0 ? u.base + u.n - p.window : 0;
            float m_own = -INFINITY, l = 0.f;    // the reference that this group's sum is relative to
            for (int t = 0; t < u.tiles; ++t, ++c) {
                if ((int)(c & 1) != group) continue;
                const int t0 = u.first + (u.tile0 + t) * kTok;
                wait_on(sh.s_full[c % kSBufs], c / kSBufs);
                tc_fence_after_sync();
                const uint32_t s_at = lane_base + S::kSAt + c % kSBufs * kTok;
                bool masked = !(t0 >= clean_begin && t0 + kTok <= clean_end);
                const bool inside = !masked;
#pragma unroll
                for (int w = 0; w < kTok / 32; ++w) masked |= sh.tokens[c & 7][w] != ~0u;
                uint32_t there[kTok / 32];
#pragma unroll
                for (int w = 0; w < kTok / 32; ++w) there[w] = ~0u;
                if (masked && some) {
#pragma unroll
                    for (int w = 0; w < kTok / 32; ++w) {
                        const int from = t0 + 32 * w;
                        // bits of tokens from + 0 .. 31 in [begin, until)
                        const int lo = begin - from, hi = until - from;
                        uint32_t mask = hi <= 0 ? 0u : hi >= 32 ? ~0u : (1u << hi) - 1u;
                        mask &= lo <= 0 ? ~0u : lo >= 32 ? 0u : ~0u << lo;
                        if (p.parent && from + 31 >= u.base) {
                            const int bit = from - u.base;                   // of the path, -31 .. 255 (or beyond: none)
                            const int wd = bit >> 5;                         // floor
                            const uint32_t a = wd >= 0 && wd < kPathWords ? sh.path[row][wd] : 0u;
                            const uint32_t b = wd + 1 >= 0 && wd + 1 < kPathWords ? sh.path[row][wd + 1] : 0u;
                            mask |= __funnelshift_r(a, b, bit & 31);
                        }
                        there[w] = mask & sh.tokens[c & 7][w];
                    }
                }
                // 64 columns of S, or 32, what is not seen as what never is the largest
                auto load_scores = [&](int ch, auto &x) {
                    constexpr int n = sizeof(x) / 4;
                    tmem_load(s_at + ch * n, x);
                    if (falls)
#pragma unroll
                        for (int i = 0; i < n; ++i) x[i] = -x[i];
                    if (masked) {
                        uint32_t see[2];
                        if constexpr (n == 64) {
                            see[0] = ch ? there[kTok / 32 - 2] : there[0];
                            see[1] = ch ? there[kTok / 32 - 1] : there[1];
                        } else {
                            see[0] = there[0];
#pragma unroll
                            for (int w = 1; w < kTok / 32; ++w) see[0] = ch == w ? there[w] : see[0];
                        }
#pragma unroll
                        for (int i = 0; i < n; ++i) x[i] = see[i / 32] >> (i & 31) & 1u ? x[i] : -INFINITY;
                    }
                };
                float top = -INFINITY;
                if (some) {
#pragma unroll 1
                    for (int ch = 0; ch < kTok / 64; ++ch) {
                        float x[64];
                        load_scores(ch, x);
                        float tops[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                        for (int i = 4; i < 64; ++i) tops[i & 3] = fmaxf(tops[i & 3], x[i]);
                        top = fmaxf(top, fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
                    }
                    if (top > -INFINITY) top = CAP ? s2 * tanhf(top * s1_abs) : top * s1_abs;
                }
                // values that are no numbers, in tiles where rows differ in what they see
                bool dirty = false;
                if (!inside && u.n > 1) {
                    const uint32_t vh = half_of_v(c), slot = vh % kSlots;
                    if (c > 1) wait_on(sh.pv_done[c & 1], (c - 2) >> 1);   // what was in that slot before is used, so loaded
                    wait_on(sh.full[slot], vh / kSlots);
                    uint4 *words = reinterpret_cast<uint4 *>(smem + slot * kHalf);
                    uint32_t found = 0;
                    for (int i = row; i < kHalf / 16; i += kRows) {
                        const uint4 v = words[i];
                        found |= not_finite<T>(v.x) | not_finite<T>(v.y) | not_finite<T>(v.z) | not_finite<T>(v.w);
                    }
                    dirty = any_of_some(6 + group, kRows, found != 0);
                    if (dirty) {
                        if (row < 4) sh.dirty[group][row] = 0;
                        sync_some(6 + group, kRows);
                        for (int i = row; i < kHalf / 16; i += kRows) {
                            uint4 v = words[i];
                            uint32_t *w = reinterpret_cast<uint32_t *>(&v);
                            bool any = false;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t f = not_finite<T>(w[j]);
                                any |= f != 0;
                                w[j] &= ~((f >> 15 & 0x10001u) * 0xffffu);
                            }
                            if (any) {
                                words[i] = v;
                                const int tok = (i % (kBlock / 16)) / 8;
                                atomicOr(&sh.dirty[group][tok >> 5], 1u << (tok & 31));
                            }
                        }
                        fence_proxy_async();
                        sync_some(6 + group, kRows);
                    }
                }
                // the reference so far, from the group of the tile before; this tile's, to the group of the next
                if (c > 0) sync_some(8 + group, kSoftThreads);
                const float m_before = t > 0 ? sh.ref[group ^ 1][row] : -INFINITY;
                bool moves = top > m_before + kSlack || (m_before == -INFINITY && top > -INFINITY);
                float m_ref = moves ? top : m_before;
                if constexpr (kHalfType) {
                    const float most = t > 0 ? fmaxf(top, sh.most[group ^ 1][row]) : top, low = fmaxf(top, most - kReach);
                    sh.most[group][row] = most;
                    if (top > -INFINITY && low < m_before - kFall) {
                        moves = true;
                        m_ref = low;
                    }
                }
                sh.ref[group][row] = m_ref;
                if (!dirty && c + 1 < n_tiles) arrive_some(8 + (group ^ 1), kSoftThreads);
                if (m_own != m_ref) l *= exp2_of(m_own - m_ref);
                m_own = m_ref;
                if (some) {
                    const float one = (m_ref == -INFINITY ? 0.f : m_ref) - kLift;   // score of the weight 1
                    // (a product that has not been rounded may exceed the reference, which has: by little, unless that is
                    // huge; each row decides by itself, so that what others see changes no bit of it)
                    const bool fused = plain && fabsf(m_ref) < 65536.f;
                    const float by_one = fused ? s1 : 1.f;
                    const bool all_fused = __all_sync(~0u, fused || m_ref == -INFINITY) && plain;
                    const uint64_t by = pair_of(by_one, by_one), less = pair_of(-one, -one), minus_one = pair_of(-1.f, -1.f);
                    uint64_t sum = 0, sum1 = 0;   // two numbers each
                    // (32 columns at a time: for 64 there are too few registers, one tree of 64 nodes took 43.8 us instead of 40.2)
#pragma unroll 1
                    for (int ch = 0; ch < kTok / 32; ++ch) {
                        float x[32];
                        load_scores(ch, x);
                        // (without branches of their own: 64 of those took 5.5 us a tile)
                        if constexpr (CAP) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float y = s2 * tanhf(x[i] * s1_abs);
                                x[i] = x[i] > -INFINITY ? y : x[i];
                            }
                        } else if (!all_fused) {   // (with a cap in a kernel of its own, whose code the others' would have to pass)
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = !fused && x[i] > -INFINITY ? x[i] * s1_abs : x[i];
                        }
                        uint32_t w[16], rest[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float a, b, ha, hb;
                            parts_of(fma_pair(pair_of(x[2 * i], x[2 * i + 1]), by, less), a, b);
                            a = exp2_of(a);
                            b = exp2_of(b);
                            uint64_t &to = i & 1 ? sum1 : sum;
                            to = add_pair(to, pair_of(a, b));
                            w[i] = pack2<T>(a, b);
                            unpack2<T>(w[i], ha, hb);
                            parts_of(fma_pair(pair_of(ha, hb), minus_one, pair_of(a, b)), a, b);   // (exact)
                            rest[i] = pack2<T>(a, b);
                        }
                        tmem_store(s_at + ch * 32, w);   // over columns that have been read
                        tmem_store(s_at + ch * 32 + 16, rest);
                    }
                    float la, lb;
                    parts_of(add_pair(sum, sum1), la, lb);
                    l += la + lb;
                    tmem_wait_store();
                }
                // The product of the tile before is done: the accumulators may be rescaled.  (Every thread waits for it every time:
                // a barrier's parity tells only neighbouring phases apart.)
                if (c > 0) wait_on(sh.pv_done[(c - 1) & 1], (c - 1) >> 1);
                if (some && t > 0 && __any_sync(~0u, moves)) {
                    tc_fence_after_sync();
                    const float alpha = moves ? exp2_of(m_before - m_ref) : 1.f;
#pragma unroll 1
                    for (int o = 0; o < D; o += 32) {
                        float v[32];
                        uint32_t w[32];
                        tmem_load(o_at + o, v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(v[i] * alpha);
                        tmem_store(o_at + o, w);
                    }
                    tmem_wait_store();
                }
                tc_fence_before_sync();
                mbar_arrive(bar(sh.p_full[c % kSBufs]));
                if (dirty) {
                    // put back what was taken out, in the rows that see it (its weight is positive); the next tile's product
                    // waits for it, because its group waits for the reference
                    wait_on(sh.pv_done[c & 1], c >> 1);
                    tc_fence_after_sync();
                    if (some)
#pragma unroll 1
                        for (int o = 0; o < D; o += 32) {
                            float v[32];
                            uint32_t w[32];
                            tmem_load(o_at + o, v);
#pragma unroll
                            for (int g = 0; g < kTok / 32; ++g) {
                                for (uint32_t bits = sh.dirty[group][g] & sh.tokens[c & 7][g]; bits; bits &= bits - 1) {
                                    const int b = __ffs(bits) - 1, tok = t0 + g * 32 + b;
                                    const uint32_t pg = div_by(p.page, (uint32_t)tok);
                                    // (behind the unit's end, or none: a block that has given up, whose bits are another tile's)
                                    const int id = tok < u.end ? p.table[u.seq * p.table_stride + pg] : -1;
                                    if ((uint32_t)id >= (uint32_t)p.n_pages) continue;
                                    const T *src = reinterpret_cast<const T *>(p.v) + id * p.stride_page +
                                                   (int64_t)(tok - (int)(pg * p.page.d)) * p.stride_token + u.head * p.stride_head + o;
#pragma unroll
                                    for (int i = 0; i < 32; ++i) {
                                        const float y = static_cast<float>(src[i]);
                                        if ((there[g] >> b & 1u) && !isfinite(y)) v[i] += y;
                                    }
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(v[i]);
                            tmem_store(o_at + o, w);
                        }
                    tmem_wait_store();
                    tc_fence_before_sync();
                    if (c + 1 < n_tiles) arrive_some(8 + (group ^ 1), kSoftThreads);
                }
            }
            // ---- the unit's end, or the stretch's
            const uint32_t last = c - 1;
            if ((int)(last & 1) == group) wait_on(sh.pv_done[last & 1], last >> 1);
            sync_some(5, kSoftThreads);          // the last reference is there, and the accumulators
            tc_fence_after_sync();
            const float m_ref = sh.ref[last & 1][row];
            sh.sum[group][row] = m_own == m_ref ? l : l * exp2_of(m_own - m_ref);
            sync_some(1 + quarter, 64);
            l = sh.sum[0][row] + sh.sum[1][row];
            const bool whole = u.ends == 3;
            if (some) {
                const int g = at - node * p.group, h = u.head * p.group + g;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const int64_t slot = (int64_t)blockIdx.x * 2 + (u.ends & 1);
                char *dst = p.out + 2 * ((int64_t)(u.node0 + node) * p.out_stride_token + h * p.out_stride_head);
                float *part = p.part_o + (slot * p.part_rows + row) * D;
#pragma unroll 1
                for (int o = 0; o < D / 2; o += 32) {
                    float v[32];
                    const int ch = group * (D / 2) + o;
                    tmem_load(o_at + ch, v);
                    if (is && whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4 *>(dst + 2 * (ch + i)) =
                                make_uint4(pack2<T>(v[i] * inv, v[i + 1] * inv), pack2<T>(v[i + 2] * inv, v[i + 3] * inv),
                                           pack2<T>(v[i + 4] * inv, v[i + 5] * inv), pack2<T>(v[i + 6] * inv, v[i + 7] * inv));
                    } else if (is) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4 *>(part + ch + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                }
                if (is && group == 0) {
                    if (!whole) p.part_ml[slot * p.part_rows + row] = make_float2(m_ref, l);
                    else if (p.lse)
                        p.lse[(int64_t)(u.node0 + node) * (p.n_kv_heads * p.group) + h] =
                            l == 0.f ? -INFINITY : 0.6931471805599453f * (m_ref - kLift) + logf(l);
                }
            }
            tc_fence_before_sync();
            if (!whole && !(u.ends & 2)) {
                if (u.ends & 1) {
                    open_rows = u.rows;
                    if (tid == 0) p.open[blockIdx.x] = Open{u.row0, u.rows, u.node0, u.head};
                } else {
                    goes_on = 1;
                }
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        if (!open_rows) p.open[blockIdx.x].rows = 0;
        p.goes_on[blockIdx.x] = goes_on;
        if (*abort_flag && p.flags) atomicOr(p.flags, STOM_FLAG_TIMEOUT);
    }
    if (warp == kWarps - 1) tmem_dealloc(tmem, 512);
}

// Joins the partial results of the units that cross a block's end.  Every block reads what units those are (they begin in one
// block of the kernel above each and go on behind it).  Their rows are taken by a warp each, or, where there are so few that
// every one can have a block, by its eight warps, with every eighth partial result each.
template <typename T, int D>
__global__ void __launch_bounds__(256) kv_tree_join_kernel(const __grid_constant__ KvTreeParams p) {
    constexpr int kVec = D / 32 < 4 ? D / 32 : 4, kVecs = D / 32 / kVec;   // channels of a lane: kVecs times kVec adjacent ones
    constexpr float kLift = std::is_same<T, __half>::value ? 7.f : 0.f;
    static_assert(kMaxBlocks == 256, "a thread for each block of the kernel above");
    __shared__ float sums[8][D];
    __shared__ float2 warp_ml[8];
    __shared__ int before[kMaxBlocks + 1], warp_rows[8];   // rows before each block's unit
    __shared__ uint32_t on[kMaxBlocks / 32];               // blocks behind which the unit that came in goes on
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_wait();
    {
        const int rows = tid < p.blocks ? p.open[tid].rows : 0;
        const uint32_t goes = __ballot_sync(~0u, tid < p.blocks && p.goes_on[tid]);
        int upto = rows;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(~0u, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warp_rows[warp] = upto;
        if (lane == 0) on[warp] = goes;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) upto += w < warp ? warp_rows[w] : 0;
        before[tid + 1] = upto;
        if (tid == 0) before[0] = 0;
        __syncthreads();
    }
    const int total = before[kMaxBlocks];
    const bool together = total <= (int)gridDim.x;
    const int step = together ? 8 : 1, items = gridDim.x * (together ? 1 : 8);
    for (int item = together ? blockIdx.x : blockIdx.x * 8 + warp; item < total; item += items) {
        // its unit: the last block whose rows begin there or before
        int x = 0;
#pragma unroll
        for (int s = kMaxBlocks / 2; s; s >>= 1)
            if (before[x + s] <= item) x += s;
        const int row = item - before[x];
        const Open u = p.open[x];
        // the blocks it goes through: x, x + 1, ..., x + n - 1, the last of them the first behind x that it does not go on behind
        const uint32_t rest = lane < kMaxBlocks / 32 ? ~on[lane] & (lane == (x + 1) >> 5 ? ~0u << ((x + 1) & 31) : lane > (x + 1) >> 5 ? ~0u : 0u) : 0u;
        const uint32_t words = __ballot_sync(~0u, rest != 0);
        const int word = words ? __ffs(words) - 1 : 0, bit = __ffs(__shfl_sync(~0u, rest, word)) - 1;
        const int n = (words ? min(word * 32 + bit + 1, p.blocks) : p.blocks) - x;
        auto at = [&](int j) { return ((int64_t)(x + j) * 2 + (j == 0 ? 1 : 0)) * p.part_rows + row; };
        // this warp's partial results, four at a time, relative to the largest maximum so far
        float m = -INFINITY, l = 0.f;
        float o[kVecs][kVec];
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) o[v][i] = 0.f;
        constexpr int kBatch = 4;
        for (int j0 = together ? warp : 0; j0 < n; j0 += kBatch * step) {
            float2 ml[kBatch];
            float y[kBatch][kVecs][kVec];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int j = j0 + b * step;
                ml[b] = make_float2(-INFINITY, 0.f);
                if (j < n) {
                    ml[b] = p.part_ml[at(j)];
                    const float *src = p.part_o + at(j) * D + lane * kVec;
#pragma unroll
                    for (int v = 0; v < kVecs; ++v) {
                        if constexpr (kVec == 4) *reinterpret_cast<float4 *>(y[b][v]) = *reinterpret_cast<const float4 *>(src + v * 128);
                        else *reinterpret_cast<float2 *>(y[b][v]) = *reinterpret_cast<const float2 *>(src);
                    }
                }
            }
            float top = m;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) top = fmaxf(top, ml[b].x);
            const float base = top == -INFINITY ? 0.f : top, f = exp2_of(m - base);
            m = top;
            l *= f;
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
#pragma unroll
                for (int i = 0; i < kVec; ++i) o[v][i] *= f;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (j0 + b * step >= n) continue;
                const float g = exp2_of(ml[b].x - base);
                l = fmaf(g, ml[b].y, l);
#pragma unroll
                for (int v = 0; v < kVecs; ++v)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) o[v][i] = fmaf(g, y[b][v][i], o[v][i]);
            }
        }
        if (together) {   // (one row a block: this is its only one)
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
#pragma unroll
                for (int i = 0; i < kVec; ++i) sums[warp][v * 128 + lane * kVec + i] = o[v][i];
            if (lane == 0) warp_ml[warp] = make_float2(m, l);
            __syncthreads();
            if (warp) return;
            m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = fmaxf(m, warp_ml[w].x);
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
#pragma unroll
                for (int i = 0; i < kVec; ++i) o[v][i] = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const float f = exp2_of(warp_ml[w].x - base);
                l = fmaf(f, warp_ml[w].y, l);
#pragma unroll
                for (int v = 0; v < kVecs; ++v)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) o[v][i] = fmaf(f, sums[w][v * 128 + lane * kVec + i], o[v][i]);
            }
        }
        const int at_row = u.row0 + row, node = (int)div_by(p.by_group, (uint32_t)at_row);
        const int h = u.head * p.group + at_row - node * p.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T *dst = reinterpret_cast<T *>(p.out) + (int64_t)(u.node0 + node) * p.out_stride_token + h * p.out_stride_head + lane * kVec;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            if constexpr (kVec == 4)
                *reinterpret_cast<uint2 *>(dst + v * 128) =
                    make_uint2(pack2<T>(o[v][0] * inv, o[v][1] * inv), pack2<T>(o[v][2] * inv, o[v][3] * inv));
            else *reinterpret_cast<uint32_t *>(dst) = pack2<T>(o[v][0] * inv, o[v][1] * inv);
        }
        if (p.lse && lane == 0)
            p.lse[(int64_t)(u.node0 + node) * (p.n_kv_heads * p.group) + h] =
                l == 0.f ? -INFINITY : 0.6931471805599453f * (m - kLift) + logf(l);
    }
}

int64_t round256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// Rows of a partial result: those of a tile, or as many as there are
int64_t part_rows(int32_t n_tokens, int32_t group) {
    const int64_t rows = (int64_t)n_tokens * group;
    return rows < kRows ? rows : kRows;
}

template <typename T, int D, bool CAP>
int32_t launch_kernels(const KvTreeParams &p, int sms, cudaStream_t stream) {
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(kv_tree_kernel<T, D, CAP>), Shape<D>::kSmem, allowed);
    if (e == cudaSuccess)
        e = launch_after_producer(kv_tree_kernel<T, D, CAP>, dim3(sms), dim3(kThreads), Shape<D>::kSmem, stream, p);
    if (e == cudaSuccess)
        e = launch_after_producer(kv_tree_join_kernel<T, D>, dim3(sms * 4), dim3(256), 0, stream, p);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}

template <typename T, int D>
int32_t launch(const KvTreeParams &p, int sms, cudaStream_t s) {
    return p.cap > 0.f ? launch_kernels<T, D, true>(p, sms, s) : launch_kernels<T, D, false>(p, sms, s);
}

template <typename T>
int32_t dispatch(const KvTreeParams &p, int d, int sms, cudaStream_t s) {
    return d == 64 ? launch<T, 64>(p, sms, s) : d == 128 ? launch<T, 128>(p, sms, s) : launch<T, 256>(p, sms, s);
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
    const int64_t rows = (int64_t)kMaxBlocks * 2 * part_rows(n_tokens, n_q_heads / pool->n_kv_heads);
    return round256(rows * pool->head_dim * 4) + round256(rows * 8) + kMaxBlocks * (int64_t)(sizeof(Open) + 4);
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
    if (seqs->n_seqs > STOM_KV_MAX_SEQS || (int64_t)n_tokens * n_q_heads > INT32_MAX - kRows) return STOM_ERR_SHAPE;
    const int64_t most = (int64_t)seqs->max_pages * pool->page_tokens;
    if (most > INT32_MAX - 256) return STOM_ERR_SHAPE;   // (tokens of a row's last tile are counted in 32 bits)
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
    int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    if (sms > kMaxBlocks) sms = kMaxBlocks;

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
    p.by_group = fast_div((uint32_t)p.group);
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
    p.blocks = sms;
    p.part_rows = (int32_t)part_rows(n_tokens, p.group);
    const int64_t rows = (int64_t)kMaxBlocks * 2 * p.part_rows;
    char *ws = static_cast<char *>(workspace);
    p.part_o = reinterpret_cast<float *>(ws);
    p.part_ml = reinterpret_cast<float2 *>(ws + round256(rows * d * 4));
    p.open = reinterpret_cast<Open *>(ws + round256(rows * d * 4) + round256(rows * 8));
    p.goes_on = reinterpret_cast<int32_t *>(p.open + kMaxBlocks);
    p.flags = dev_flags;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return pool->dtype == STOM_BF16 ? dispatch<__nv_bfloat16>(p, d, sms, s) : dispatch<__half>(p, d, sms, s);
}
