// Attention of one new token per sequence over a paged cache (stom_kv_attend).
//
//   out = sum_t exp(x_t) V_t / sum_t exp(x_t),  x_t = scale <q, K_t>, capped if asked for, t over the sequence's tokens.
//
// What bounds it: every key and value row is read once and takes part in 4 * (query heads per kv head) flops per
// element, 14 flops per byte at 7 heads: memory, by a wide margin, as long as the products run on the tensor cores
// (the scalar units would need 45 of their 75 TFLOP/s).  The kernel is therefore built around keeping loads in flight.
//
// Split.  The work is one line of TILES of 16 tokens: sequence by sequence, within one head by head (a UNIT is one
// (sequence, kv head)), within one along the tokens.  Every warp of a grid of one block per multiprocessor takes an
// equal, contiguous stretch of that line, so unequal lengths need no planning on the host and a single long stream uses
// the whole device.  A warp is alone with its stretch: its own ring of tiles in shared memory, filled by 16-byte
// asynchronous copies (any page size, any strides; a tile's rows may lie in 16 pages), its own running maximum and sum,
// no barrier between warps.  A unit that a warp holds whole goes straight to the output.  Pieces of a unit are joined
// first within the block (shared memory), then, for the at most one unit that crosses each block's end, by a second
// small kernel over a workspace of two partial results per block.
//
// Products.  Transposed, so that the up to 8 query heads of a kv head are the 8 columns of an m16n8k16 product and
// the 16 tokens, respectively 16 channels, its rows: S^T = K q^T with K as stored, O^T = V^T P^T with V transposed on
// the way out of shared memory (ldmatrix.trans).  Scores and accumulators then have their head in the same thread, so
// that rescaling needs no exchange.  The softmax weights go into the second product as a high and a low 16-bit part
// (2^-16 relative at bf16): one part alone would add an error of the size of the output's own rounding, and the
// second costs nothing in a kernel that waits for memory.  fp16 has no numbers below 2^-24, so that weights relative to
// the running maximum would vanish where thousands of tokens count only in sum, beside one that stands 15 nats above
// them; there a tile's weights are relative to its own largest score, which gets 2^15, and its product has accumulators
// of its own that are scaled into the running ones: a weight is off by 2^-22 of itself or 2^-40 of its tile's largest,
// whichever is more.  bf16 has the exponents of binary32 and needs none of it.
//
// Measured (B200, copy rate 6 458 GB/s): 64 sequences of 17 to 16 411 tokens, 64 + 8 heads of 128, pages of 16: 230 to 240
// us for 1.47 GB, 6.1 to 6.4 TB/s.  One sequence of 12 583 tokens, 28 + 4 heads, pages of 50: 12.2 us, of which 4 are its
// 26 MB at the copy rate, 2.5 the way to the first load (lengths, then pages, then rows: three memory round trips), 1.5 the
// block's join, 3 the second kernel.  233 sequences of 0 to 300 tokens, 16 + 2 heads of 64, fp16: 14.1 us, all of it such latencies
// (and the same as with weights relative to the running maximum).
#include "stom_kv.cuh"

#include <math.h>

#include <type_traits>

namespace stom {

namespace {

constexpr int kTile = 16;         // tokens per tile
constexpr float kLift = 15.f;     // fp16: the largest weight of a tile is 2^kLift
constexpr int kMaxBlocks = 256;   // blocks of the grid the workspace has room for

struct KvAttendParams {
    const char *k, *v;            // at the layer
    int64_t stride_page, stride_token, stride_head;
    const int32_t *table;
    const int32_t *len;
    int64_t table_stride;
    int32_t n_seqs, n_pages, max_tokens;
    FastDiv page;
    int32_t n_kv_heads, group;    // query heads per kv head
    int32_t blocks_per_head;      // blocks of 8 * NT query heads a kv head's group is cut into
    FastDiv by_blocks, by_units;  // division by that, and by n_kv_heads * blocks_per_head
    FastDiv by_warps;             // and by the grid's warps
    const char *q;
    int64_t q_stride_seq, q_stride_head;
    float scale, cap;             // softmax scale; cap <= 0: none
    int32_t window;
    char *out;
    int64_t out_stride_seq, out_stride_head;
    float *lse;
    float *part_o;                // [blocks][2][8 NT][d]
    float2 *part_ml;              // [blocks][2][8 NT]: maximum and sum
    int32_t *open_unit;           // [blocks]: unit that begins in the block and goes on behind it, or -1
    int32_t *goes_on;             // [blocks]: the unit that came in from the block before goes on behind this one too
    uint32_t *flags;
};

template <int D, int NT>
struct Shape {
    static constexpr int kHeads = 8 * NT;
    static constexpr int kWarps = D == 64 ? (NT == 1 ? 16 : 12) : D == 128 ? (NT == 1 ? 8 : 6) : 4;
    static constexpr int kStages = 3;
    static constexpr int kRow = D * 2;                       // bytes of a row
    static constexpr int kTileBytes = kTile * kRow;          // of keys or of values
    static constexpr int kRing = kStages * 2 * kTileBytes;   // per warp
    static constexpr int kPiece = kHeads * D * 4;            // a partial result
    static constexpr int kPieces = 2 * kWarps;
    static constexpr int kSmem = kWarps * (kRing + kPiece) + kPieces * (kHeads * 8 + 8);
    static_assert(kPiece + kPieces * kHeads * 4 <= kRing, "the units' maxima lie behind the first warp's last piece");
    static_assert(kPieces * kHeads <= 32 * kWarps, "a thread for each head of each piece");
    static_assert(kPiece <= kRing, "a warp's last piece lies in its ring");
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// The tokens of a sequence that are looked at: the window ends at its length, also where that lies beyond its pages.
__device__ __forceinline__ void span_of(const KvAttendParams &p, int b, int &first, int &end) {
    const int len = max(p.len[b], 0);
    end = min(len, p.max_tokens);
    first = p.window > 0 ? min(end, max(0, len - p.window)) : 0;
}
__device__ __forceinline__ int tiles_of(const KvAttendParams &p, int b) {
    int first, end;
    span_of(p, b, first, end);
    return (end - first + kTile - 1) / kTile;
}

// A place on the line of tiles.
struct Cursor {
    int b, hu;          // sequence, head block
    int tile, tiles;    // within the unit
    int first, end;     // token range of the sequence
};

__device__ __forceinline__ void next_seq(const KvAttendParams &p, Cursor &c) {
    c.tiles = 0;
    while (c.tiles == 0 && ++c.b < p.n_seqs) {
        span_of(p, c.b, c.first, c.end);
        c.tiles = (c.end - c.first + kTile - 1) / kTile;
    }
}
__device__ __forceinline__ void advance(const KvAttendParams &p, int units, Cursor &c) {
    if (++c.tile < c.tiles) return;
    c.tile = 0;
    if (++c.hu < units) return;
    c.hu = 0;
    next_seq(p, c);
}

// Output rows of unit (b, hu): query head and count of heads.
__device__ __forceinline__ int heads_of(const KvAttendParams &p, int hu, int per, int &head0) {
    const int h = (int)div_by(p.by_blocks, (uint32_t)hu), j = hu - h * p.blocks_per_head;
    head0 = h * p.group + j * per;
    return min(per, p.group - j * per);
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(Shape<D, NT>::kWarps * 32, 1) kv_attend_kernel(const __grid_constant__ KvAttendParams p) {
    using S = Shape<D, NT>;
    constexpr int kWarps = S::kWarps, kHeads = S::kHeads, kStages = S::kStages;
    constexpr int kKs = D / 16;                      // steps of the first product, row blocks of the second
    constexpr bool kOwnScale = std::is_same<T, __half>::value;   // weights relative to the tile's largest score
    constexpr int kChunks = D / 8;                   // 16-byte chunks of a row
    constexpr int kRowsPerCopy = 32 / kChunks;       // rows one warp-wide copy covers
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint8_t *ring = smem + warp * S::kRing;
    float *first_piece = reinterpret_cast<float *>(smem + kWarps * S::kRing + warp * S::kPiece);
    float2 *piece_ml = reinterpret_cast<float2 *>(smem + kWarps * (S::kRing + S::kPiece));  // [2 kWarps][kHeads]
    int *piece_unit = reinterpret_cast<int *>(piece_ml + S::kPieces * kHeads);              // [2 kWarps], -1: none
    int *piece_ends = piece_unit + S::kPieces;  // bit 0: holds the unit's first tile, bit 1: its last

    if (lane < 2) piece_unit[2 * warp + lane] = -1;
    grid_dependency_wait();
    grid_launch_dependents();   // the joining kernel may take its places now; it waits for this grid's end

    // ---- the stretch of this warp.  The block adds up the sequences' tiles, in the memory of the first pieces.
    const int units = p.n_kv_heads * p.blocks_per_head;   // per sequence
    uint32_t *tiles_before = reinterpret_cast<uint32_t *>(smem + kWarps * S::kRing);
    uint32_t *warp_tiles = reinterpret_cast<uint32_t *>(piece_ml);
    static_assert(kWarps * S::kPiece >= STOM_KV_MAX_SEQS * 4, "a number for each sequence");
    uint32_t all_tiles;
    {
        const int seg = (p.n_seqs + kWarps * 32 - 1) / (kWarps * 32);   // sequences a thread adds up
        const int b0 = threadIdx.x * seg, b1 = min(p.n_seqs, b0 + seg);
        uint32_t mine = 0;
        for (int b = b0; b < b1; ++b) {
            tiles_before[b] = mine;
            mine += tiles_of(p, b);
        }
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(~0u, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warp_tiles[warp] = upto;
        __syncthreads();
        const uint32_t of = lane < kWarps ? warp_tiles[lane] : 0u;
        all_tiles = __reduce_add_sync(~0u, of);
        const uint32_t before = __reduce_add_sync(~0u, lane < warp ? of : 0u) + upto - mine;
        for (int b = b0; b < b1; ++b) tiles_before[b] += before;
        __syncthreads();
    }
    const uint32_t total = all_tiles * units, per = max(1u, div_by(p.by_warps, total + p.by_warps.d - 1));
    const uint32_t f0 = min(total, (blockIdx.x * kWarps + warp) * per);
    int left = (int)(min(total, f0 + per) - f0);
    // its first tile's sequence: the last that begins at f0 or before (of several, the others are empty)
    Cursor cur = {};
    if (left > 0) {
        int low = 0, high = p.n_seqs;                     // low begins there or before, high does not
        while (high - low > 1) {
            const int step = (high - low + 31) / 32, at = low + step * lane;
            const uint32_t yes = __ballot_sync(~0u, at < high && tiles_before[at] * units <= f0);
            low += step * (31 - __clz(yes));              // lane 0 stands at low
            high = min(high, low + step);
        }
        cur.b = low;
        span_of(p, cur.b, cur.first, cur.end);
        cur.tiles = (cur.end - cur.first + kTile - 1) / kTile;
        const uint32_t in = f0 - tiles_before[low] * units;
        cur.hu = (int)(in / (uint32_t)cur.tiles);
        cur.tile = (int)in - cur.hu * cur.tiles;
    }
    __syncthreads();   // the numbers have been read: pieces may take their place

    int pieces = 0;   // partial results this warp leaves in shared memory
    if (left > 0) {
        // ---- loads.  Lane r (and r + 16) looks up the page of row r two tiles ahead of the copies.
        Cursor ld = cur;
        int to_look = left;          // tiles not looked up yet
        struct Row {
            int page;                // id; kNone: not a token
            int64_t rest;            // offset within a page, in elements
        };
        constexpr int kNone = INT32_MIN;
        Row ahead[2] = {{kNone, 0}, {kNone, 0}};
        auto look_up = [&](Row &r) {
            r.page = kNone;
            if (to_look > 0) {
                const int t = ld.first + ld.tile * kTile + (lane & 15);
                if (t < ld.end) {
                    const uint32_t pg = div_by(p.page, (uint32_t)t);
                    r.rest = (int64_t)(t - (int)(pg * p.page.d)) * p.stride_token + (int64_t)div_by(p.by_blocks, (uint32_t)ld.hu) * p.stride_head;
                    r.page = p.table[ld.b * p.table_stride + pg];
                    if (r.page == kNone) r.page = -1;
                }
                if (--to_look > 0) advance(p, units, ld);
            }
        };
        uint64_t seen = 0;       // 16 bits per tile in flight, oldest lowest: which rows are tokens
        int in_flight = 0, to_issue = left;
        const uint32_t ring_u = smem_u32(ring);
        auto issue = [&](int stage) {
            if (to_issue > 0) {
                --to_issue;
                const Row r = ahead[0];
                const bool ok = (uint32_t)r.page < (uint32_t)p.n_pages;
                if (r.page != kNone && !ok && p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
                const uint32_t m = __ballot_sync(~0u, ok) & 0xffffu;
                seen |= (uint64_t)m << (16 * in_flight);
                ++in_flight;
                const int64_t off = ok ? 2 * (r.page * p.stride_page + r.rest) : -1;
                const uint32_t dst = ring_u + stage * (2 * S::kTileBytes);
                const int sub = lane / kChunks, chunk = lane % kChunks;
#pragma unroll
                for (int i = 0; i < kTile / kRowsPerCopy; ++i) {
                    const int row = i * kRowsPerCopy + sub;
                    const int64_t o = __shfl_sync(~0u, off, row);
                    const uint32_t d = dst + row * S::kRow + ((chunk ^ (row & 7)) << 4);
                    const int64_t at = (o < 0 ? 0 : o) + chunk * 16;
                    copy16_async(d, p.k + at, o < 0 ? 0u : 16u);
                    copy16_async(d + S::kTileBytes, p.v + at, o < 0 ? 0u : 16u);
                }
                ahead[0] = ahead[1];
                look_up(ahead[1]);
            }
            copy_commit();
        };
        look_up(ahead[0]);
        look_up(ahead[1]);
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) issue(i);

        // ---- per-unit state
        uint32_t qf[kKs][NT][2];
        float o_acc[kKs][NT][4];
        float m_run[NT][2], l_run[NT][2];
        bool fresh = true, whole_from = false;
        const float log2e = 1.4426950408889634f;
        const float s1 = p.cap > 0.f ? p.scale / p.cap : p.scale * log2e;
        const float s2 = p.cap * log2e;
        int stage = 0;

        while (left > 0) {
            if (fresh) {
                int head0;
                const int nh = heads_of(p, cur.hu, kHeads, head0);
                const T *q = reinterpret_cast<const T *>(p.q) + cur.b * p.q_stride_seq;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int h = n * 8 + (lane >> 2);
                    const T *row = q + (head0 + (h < nh ? h : 0)) * p.q_stride_head + (lane & 3) * 2;
#pragma unroll
                    for (int ks = 0; ks < kKs; ++ks) {
                        qf[ks][n][0] = h < nh ? *reinterpret_cast<const uint32_t *>(row + ks * 16) : 0u;
                        qf[ks][n][1] = h < nh ? *reinterpret_cast<const uint32_t *>(row + ks * 16 + 8) : 0u;
                    }
#pragma unroll
                    for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o_acc[ks][n][e] = 0.f;
                    m_run[n][0] = m_run[n][1] = -INFINITY;
                    l_run[n][0] = l_run[n][1] = 0.f;
                }
                whole_from = cur.tile == 0;
                fresh = false;
            }

            copy_wait<kStages - 2>();
            __syncwarp();
            issue(stage == 0 ? kStages - 1 : stage - 1);   // into the slot the tile before this one has left

            const uint32_t kt = ring_u + stage * (2 * S::kTileBytes), vt = kt + S::kTileBytes;
            const uint32_t rows = (uint32_t)seen & 0xffffu;
            seen >>= 16;
            --in_flight;

            // S^T = K q^T, in two chains of products
            float s[NT][2][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][0][e] = s[n][1][e] = 0.f;
            {
                const int row = (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
                for (int ks = 0; ks < kKs; ++ks) {
                    uint32_t a[4];
                    ldsm4(a, kt + row * S::kRow + (((2 * ks + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16x8x16<T>(s[n][ks & 1], a, qf[ks][n][0], qf[ks][n][1]);
                }
            }
            const bool in0 = (rows >> (lane >> 2)) & 1u, in1 = (rows >> ((lane >> 2) + 8)) & 1u;
            float alpha[NT][2], beta[NT][2];   // factors of what has been added up, and (fp16) of this tile
            uint32_t ph[NT][2], pl[NT][2];
            bool moved = false;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = (s[n][0][e] + s[n][1][e]) * s1;
                    if (p.cap > 0.f) x[e] = s2 * tanhf(x[e]);
                    if (!(e < 2 ? in0 : in1)) x[e] = -INFINITY;
                }
                float top[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])};
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    top[0] = fmaxf(top[0], __shfl_xor_sync(~0u, top[0], o));
                    top[1] = fmaxf(top[1], __shfl_xor_sync(~0u, top[1], o));
                }
                float w[4];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float m = fmaxf(m_run[n][c], top[c]);
                    const float base = m == -INFINITY ? 0.f : m;
                    moved |= m > m_run[n][c];
                    alpha[n][c] = exp2f(m_run[n][c] - base);
                    m_run[n][c] = m;
                    if constexpr (kOwnScale) {
                        const bool none = top[c] == -INFINITY;
                        const float one = none ? 0.f : top[c] - kLift;   // score of the weight 1
                        beta[n][c] = none ? 0.f : exp2f(one - base);
                        w[c] = exp2f(x[c] - one);
                        w[c + 2] = exp2f(x[c + 2] - one);
                        l_run[n][c] = l_run[n][c] * alpha[n][c] + (w[c] + w[c + 2]) * beta[n][c];
                    } else {
                        w[c] = exp2f(x[c] - base);
                        w[c + 2] = exp2f(x[c + 2] - base);
                        l_run[n][c] = l_run[n][c] * alpha[n][c] + w[c] + w[c + 2];
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t hi = pack2<T>(w[2 * r], w[2 * r + 1]);
                    float h0, h1;
                    unpack2<T>(hi, h0, h1);
                    ph[n][r] = transpose8x8(hi);
                    pl[n][r] = transpose8x8(pack2<T>(w[2 * r] - h0, w[2 * r + 1] - h1));
                }
            }
            if (__any_sync(~0u, moved)) {
#pragma unroll
                for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o_acc[ks][n][e] *= alpha[n][e & 1];
            }
            // O^T += V^T P^T
            {
                const int row = (lane & 7) + (lane >> 4) * 8;
#pragma unroll
                for (int ks = 0; ks < kKs; ++ks) {
                    uint32_t a[4];
                    ldsm4_trans(a, vt + row * S::kRow + (((2 * ks + ((lane >> 3) & 1)) ^ (row & 7)) << 4));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if constexpr (kOwnScale) {
                            float t[4] = {0.f, 0.f, 0.f, 0.f};
                            mma16x8x16<T>(t, a, ph[n][0], ph[n][1]);
                            mma16x8x16<T>(t, a, pl[n][0], pl[n][1]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o_acc[ks][n][e] = fmaf(t[e], beta[n][e & 1], o_acc[ks][n][e]);
                        } else {
                            mma16x8x16<T>(o_acc[ks][n], a, ph[n][0], ph[n][1]);
                            mma16x8x16<T>(o_acc[ks][n], a, pl[n][0], pl[n][1]);
                        }
                    }
                }
            }
            stage = stage + 1 == kStages ? 0 : stage + 1;
            --left;

            const bool last = cur.tile + 1 == cur.tiles;
            if (last || left == 0) {
                // the unit's end, or the stretch's
                int head0;
                const int nh = heads_of(p, cur.hu, kHeads, head0);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) l_run[n][c] += __shfl_xor_sync(~0u, l_run[n][c], o);
                if (last && whole_from) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int h = n * 8 + (lane & 3) * 2 + c;
                            if (h >= nh) continue;
                            T *o = reinterpret_cast<T *>(p.out) + cur.b * p.out_stride_seq +
                                   (head0 + h) * p.out_stride_head + (lane >> 2);
                            const float inv = l_run[n][c] > 0.f ? 1.f / l_run[n][c] : l_run[n][c] == 0.f ? 0.f : l_run[n][c];
#pragma unroll
                            for (int ks = 0; ks < kKs; ++ks) {
                                o[ks * 16] = from_float<T>(o_acc[ks][n][c] * inv);
                                o[ks * 16 + 8] = from_float<T>(o_acc[ks][n][c + 2] * inv);
                            }
                            if (p.lse && lane < 4)
                                p.lse[(int64_t)cur.b * (p.n_kv_heads * p.group) + head0 + h] =
                                    l_run[n][c] == 0.f ? -INFINITY : 0.6931471805599453f * m_run[n][c] + logf(l_run[n][c]);
                        }
                } else {
                    // a piece: a warp's first in its own place, its last (if it has two) in its ring, which no copy
                    // is on its way to any more
                    const int slot = 2 * warp + pieces;
                    float *dst = pieces ? reinterpret_cast<float *>(ring) : first_piece;
                    __syncwarp();
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int h = n * 8 + (lane & 3) * 2 + c;
#pragma unroll
                            for (int ks = 0; ks < kKs; ++ks) {
                                dst[h * D + ks * 16 + (lane >> 2)] = o_acc[ks][n][c];
                                dst[h * D + ks * 16 + 8 + (lane >> 2)] = o_acc[ks][n][c + 2];
                            }
                            if (lane < 4) piece_ml[slot * kHeads + h] = make_float2(m_run[n][c], l_run[n][c]);
                        }
                    if (lane == 0) {
                        piece_unit[slot] = cur.b * units + cur.hu;
                        piece_ends[slot] = (whole_from ? 1 : 0) | (last ? 2 : 0);
                    }
                    ++pieces;
                }
                fresh = true;
            }
            if (left > 0) advance(p, units, cur);
        }
        copy_wait<0>();
    }
    __syncthreads();

    // ---- join the block's pieces, unit by unit; they stand in the order of the line.  First a thread for each head of
    // each piece: what the piece counts for beside the unit's largest maximum.
    float *piece_top = reinterpret_cast<float *>(smem + S::kPiece);   // [2 kWarps][kHeads], in a ring that is no more used
    {
        const int j = threadIdx.x / kHeads, h = threadIdx.x % kHeads;
        float2 mine = make_float2(-INFINITY, 0.f);
        float top = -INFINITY;
        if (j < S::kPieces && piece_unit[j] >= 0) {
            const int u = piece_unit[j];
            mine = piece_ml[j * kHeads + h];
#pragma unroll 8
            for (int k = 0; k < S::kPieces; ++k)
                if (piece_unit[k] == u) top = fmaxf(top, piece_ml[k * kHeads + h].x);
        }
        __syncthreads();
        const float f = exp2f(mine.x - (top == -INFINITY ? 0.f : top));
        if (j < S::kPieces) piece_ml[j * kHeads + h] = make_float2(f, f * mine.y);
        if (j < S::kPieces) piece_top[j * kHeads + h] = top;
    }
    __syncthreads();
    // Then a thread has four channels of a head (or several times four) and walks the pieces; with more threads than that
    // takes, teams take units in turn.
    int open_unit = -1, goes_on = 0;
    constexpr int kThreads = kWarps * 32, kPer = kHeads * D / 4 <= kThreads ? 1 : kHeads * D / 4 <= 2 * kThreads ? 2 : 4;
    constexpr int kAcross = D / 4 / kPer, kCols = kHeads * kAcross, kTeams = kThreads / kCols;
    static_assert(kTeams >= 1, "a thread for each column");
    const int team = threadIdx.x / kCols, h = threadIdx.x % kCols / kAcross, c0 = threadIdx.x % kAcross * 4;
    if (team < kTeams) {
        int unit = -1, ends = 0, turn = -1;
        float m = -INFINITY, l = 0.f;
        float4 o[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        auto finish = [&]() {
            if (!(ends & 2)) {
                if (ends & 1) open_unit = unit;
                else goes_on = 1;
            }
            if (kTeams > 1 && turn % kTeams != team) return;
            const int b = (int)div_by(p.by_units, (uint32_t)unit), hu = unit - b * units;
            int head0;
            if (h >= heads_of(p, hu, kHeads, head0)) return;
            if (ends == 3) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                T *dst = reinterpret_cast<T *>(p.out) + b * p.out_stride_seq + (head0 + h) * p.out_stride_head + c0;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    *reinterpret_cast<uint2 *>(dst + i * kAcross * 4) =
                        make_uint2(pack2<T>(o[i].x * inv, o[i].y * inv), pack2<T>(o[i].z * inv, o[i].w * inv));
                if (p.lse && c0 == 0)
                    p.lse[(int64_t)b * (p.n_kv_heads * p.group) + head0 + h] =
                        l == 0.f ? -INFINITY : 0.6931471805599453f * m + logf(l);
            } else {
                // of the workspace: slot 1 for a unit that begins here, slot 0 for one that came in
                const int64_t w = ((int64_t)blockIdx.x * 2 + (ends & 1)) * kHeads + h;
#pragma unroll
                for (int i = 0; i < kPer; ++i) *reinterpret_cast<float4 *>(p.part_o + w * D + c0 + i * kAcross * 4) = o[i];
                if (c0 == 0) p.part_ml[w] = make_float2(m, l);
            }
        };
        constexpr int kBatch = kPer == 4 ? 2 : 4;
        static_assert(S::kPieces % kBatch == 0, "pieces");
        for (int j0 = 0; j0 < S::kPieces; j0 += kBatch) {
            int u[kBatch], e[kBatch];
            float2 f[kBatch];
            float4 v[kBatch][kPer];
            float t[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int j = j0 + k;
                u[k] = piece_unit[j];
                e[k] = piece_ends[j];
                f[k] = piece_ml[j * kHeads + h];
                t[k] = piece_top[j * kHeads + h];
                const uint8_t *src = j & 1 ? smem + (j >> 1) * S::kRing : smem + kWarps * S::kRing + (j >> 1) * S::kPiece;
#pragma unroll
                for (int i = 0; i < kPer; ++i) v[k][i] = *reinterpret_cast<const float4 *>(src + (h * D + c0 + i * kAcross * 4) * 4);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (u[k] < 0) continue;
                if (u[k] != unit) {
                    if (unit >= 0) finish();
                    unit = u[k];
                    ends = e[k] & 1;
                    ++turn;
                    m = t[k];
                    l = 0.f;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                ends = (ends & 1) | (e[k] & 2);
                l += f[k].y;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    o[i].x += v[k][i].x * f[k].x;
                    o[i].y += v[k][i].y * f[k].x;
                    o[i].z += v[k][i].z * f[k].x;
                    o[i].w += v[k][i].w * f[k].x;
                }
            }
        }
        if (unit >= 0) finish();
    }
    if (threadIdx.x == 0) {
        p.open_unit[blockIdx.x] = open_unit;
        p.goes_on[blockIdx.x] = goes_on;
    }

    // lengths beyond a row's pages are told; the empty sequences: zeros
    for (int b = blockIdx.x * kWarps + warp; b < p.n_seqs; b += gridDim.x * kWarps) {
        if (p.flags && lane == 0 && p.len[b] > p.max_tokens) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
        if (tiles_of(p, b)) continue;
        const int heads = p.n_kv_heads * p.group;
        for (int h = 0; h < heads; ++h) {
            T *o = reinterpret_cast<T *>(p.out) + b * p.out_stride_seq + h * p.out_stride_head;
            for (int c = lane; c < D / 2; c += 32) reinterpret_cast<uint32_t *>(o)[c] = 0u;
            if (p.lse && lane == 0) p.lse[(int64_t)b * heads + h] = -INFINITY;
        }
    }
}

// Joins the partial results of the units that cross a block's end: block (x, h) of this grid takes query head h of the
// unit that begins in block x of the kernel above and goes on behind it, if there is one.  Thread (g, c) adds up every
// kJoin-th partial result of four channels.
constexpr int kJoin = 8;
template <typename T, int D, int NT>
__global__ void __launch_bounds__(D / 4 * kJoin) kv_attend_join_kernel(const __grid_constant__ KvAttendParams p) {
    constexpr int kHeads = 8 * NT, kThreads = D / 4 * kJoin;
    __shared__ float weight[kMaxBlocks];
    __shared__ float warp_m[32], warp_l[32];
    __shared__ float4 sum[kJoin][D / 4];
    __shared__ int end_s;
    constexpr int kOwn = (kMaxBlocks + kThreads - 1) / kThreads;   // blocks a thread looks at
    if (threadIdx.x == 0) end_s = gridDim.x;
    grid_dependency_wait();
    const int first = blockIdx.x, h = blockIdx.y, blocks = gridDim.x;
    auto row_of = [&](int j) { return ((int64_t)(first + j) * 2 + (j == 0 ? 1 : 0)) * kHeads + h; };
    // all that may be needed is asked for at once: what turns out not to belong to the unit is not used
    const int unit = p.open_unit[first];
    int on[kOwn];
    float2 ml[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        const int j = threadIdx.x + k * kThreads;
        on[k] = first + j < blocks && j ? p.goes_on[first + j] : 1;
        ml[k] = first + j < blocks ? p.part_ml[row_of(j)] : make_float2(-INFINITY, 0.f);
    }
    if (unit < 0) return;
    const int units = p.n_kv_heads * p.blocks_per_head;
    const int b = (int)div_by(p.by_units, (uint32_t)unit), hu = unit - b * units;
    int head0;
    if (h >= heads_of(p, hu, kHeads, head0)) return;
    // the blocks it goes through: first, first + 1, ..., end - 1
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
        if (!on[k]) atomicMin(&end_s, first + (int)threadIdx.x + k * kThreads + 1);
    __syncthreads();
    const int n = end_s - first;
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        if ((int)threadIdx.x + k * kThreads >= n) ml[k] = make_float2(-INFINITY, 0.f);
        m = fmaxf(m, ml[k].x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    if ((threadIdx.x & 31) == 0) warp_m[threadIdx.x >> 5] = m;
    __syncthreads();
    m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kThreads / 32; ++j) m = fmaxf(m, warp_m[j]);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        const int j = threadIdx.x + k * kThreads;
        const float f = exp2f(ml[k].x - base);
        if (j < n) weight[j] = f;
        l += f * ml[k].y;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
    if ((threadIdx.x & 31) == 0) warp_l[threadIdx.x >> 5] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int j = 0; j < kThreads / 32; ++j) l += warp_l[j];
    const int c = threadIdx.x % (D / 4), g = threadIdx.x / (D / 4);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int j = g; j < n; j += kJoin) {
        const float4 v = *reinterpret_cast<const float4 *>(p.part_o + row_of(j) * D + c * 4);
        const float f = weight[j];
        o.x += f * v.x;
        o.y += f * v.y;
        o.z += f * v.z;
        o.w += f * v.w;
    }
    sum[g][c] = o;
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int k = 1; k < kJoin; ++k) {
        const float4 v = sum[k][c];
        o.x += v.x;
        o.y += v.y;
        o.z += v.z;
        o.w += v.w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *dst = reinterpret_cast<T *>(p.out) + b * p.out_stride_seq + (head0 + h) * p.out_stride_head + c * 4;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
    if (p.lse && c == 0)
        p.lse[(int64_t)b * (p.n_kv_heads * p.group) + head0 + h] =
            l == 0.f ? -INFINITY : 0.6931471805599453f * m + logf(l);
}

// Query heads per product: 8, or 16 where a kv head has more than 8 and the accumulators fit (head_dim <= 128); a
// larger group is cut into blocks of that many, which read the keys and values again (how much of it comes from L2 has not
// been measured).
int heads_per_unit(int group, int head_dim) { return group > 8 && head_dim <= 128 ? 16 : 8; }

int64_t round16(int64_t x) { return (x + 15) & ~(int64_t)15; }

template <typename T, int D, int NT>
int32_t launch(KvAttendParams &p, int sms, cudaStream_t stream) {
    using S = Shape<D, NT>;
    p.by_warps = fast_div((uint32_t)(sms * S::kWarps));
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(kv_attend_kernel<T, D, NT>), S::kSmem, allowed);
    if (e == cudaSuccess)
        e = launch_after_producer(kv_attend_kernel<T, D, NT>, dim3(sms), dim3(S::kWarps * 32), S::kSmem, stream, p);
    if (e == cudaSuccess)
        e = launch_after_producer(kv_attend_join_kernel<T, D, NT>, dim3(sms, min(p.group, 8 * NT)), dim3(D / 4 * kJoin), 0, stream,
                                  p);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}

template <typename T>
int32_t dispatch(KvAttendParams &p, int head_dim, int sms, cudaStream_t stream) {
    const bool two = heads_per_unit(p.group, head_dim) == 16;
    if (head_dim == 64) return two ? launch<T, 64, 2>(p, sms, stream) : launch<T, 64, 1>(p, sms, stream);
    if (head_dim == 128) return two ? launch<T, 128, 2>(p, sms, stream) : launch<T, 128, 1>(p, sms, stream);
    return launch<T, 256, 1>(p, sms, stream);
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int64_t stom_kv_attend_workspace_bytes(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t n_q_heads) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, false);
    if (rc) return rc;
    if (n_q_heads < 1 || n_q_heads % pool->n_kv_heads) return STOM_ERR_SHAPE;
    const int64_t rows = (int64_t)kMaxBlocks * 2 * heads_per_unit(n_q_heads / pool->n_kv_heads, pool->head_dim);
    return rows * pool->head_dim * 4 + rows * 8 + round16(kMaxBlocks * 8);
}

extern "C" int32_t stom_kv_attend(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t layer, int32_t n_q_heads,
                                  const void *q, int64_t q_stride_seq, int64_t q_stride_head, float softmax_scale,
                                  float softcap, int32_t window, void *out, int64_t out_stride_seq,
                                  int64_t out_stride_head, float *lse, void *workspace, int64_t workspace_bytes,
                                  uint32_t *dev_flags, void *stream) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, false);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->n_layers || n_q_heads < 1 || window < 0) return STOM_ERR_INVALID_ARG;
    // the factors that the kernel multiplies scores by have to be numbers, and one below binary32's normal ones lacks bits
    const float s1 = fabsf(softcap > 0.f ? softmax_scale / softcap : softmax_scale * 1.4426950408889634f);
    if (!(softcap >= 0.f) || !(softcap <= 2.0e38f) || !(s1 <= 3.0e38f) || (softcap > 0.f && s1 != 0.f && s1 < 1.2e-38f))
        return STOM_ERR_INVALID_ARG;
    if (n_q_heads % pool->n_kv_heads || n_q_heads / pool->n_kv_heads > 64) return STOM_ERR_SHAPE;
    if (seqs->n_seqs > STOM_KV_MAX_SEQS) return STOM_ERR_SHAPE;
    if (seqs->n_seqs == 0) return STOM_OK;
    if (!q || !out) return STOM_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !stride_ok(q_stride_seq, pool->dtype) || !stride_ok(q_stride_head, pool->dtype) ||
        !stride_ok(out_stride_seq, pool->dtype) || !stride_ok(out_stride_head, pool->dtype))
        return STOM_ERR_ALIGNMENT;
    const int32_t d = pool->head_dim, group = n_q_heads / pool->n_kv_heads;
    if (n_q_heads > 1 && (out_stride_head < d || q_stride_head < 0)) return STOM_ERR_INVALID_ARG;
    if (seqs->n_seqs > 1 && (out_stride_seq < d || q_stride_seq < 0)) return STOM_ERR_INVALID_ARG;
    const int64_t need = stom_kv_attend_workspace_bytes(pool, seqs, n_q_heads);
    if (!workspace || !aligned16(workspace) || workspace_bytes < need) return STOM_ERR_WORKSPACE;
    const int per = heads_per_unit(group, d);
    const int64_t units = (int64_t)pool->n_kv_heads * ((group + per - 1) / per);
    // the line of tiles is counted in 32 bits (with the grid's warps and a tile of each row to spare)
    const int64_t most = (int64_t)seqs->max_pages * pool->page_tokens;
    if (most > INT32_MAX - 32 || (most / kTile + 1) * seqs->n_seqs * units > INT32_MAX - 16 * kMaxBlocks) return STOM_ERR_SHAPE;
    int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    if (sms > kMaxBlocks) sms = kMaxBlocks;

    KvAttendParams p = {};
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
    p.group = group;
    p.blocks_per_head = (group + per - 1) / per;
    p.by_blocks = fast_div((uint32_t)p.blocks_per_head);
    p.by_units = fast_div((uint32_t)units);
    p.q = static_cast<const char *>(q);
    p.q_stride_seq = q_stride_seq;
    p.q_stride_head = q_stride_head;
    p.scale = softmax_scale;
    p.cap = softcap;
    p.window = window;
    p.out = static_cast<char *>(out);
    p.out_stride_seq = out_stride_seq;
    p.out_stride_head = out_stride_head;
    p.lse = lse;
    const int64_t rows = (int64_t)kMaxBlocks * 2 * per;
    p.part_o = static_cast<float *>(workspace);
    p.part_ml = reinterpret_cast<float2 *>(p.part_o + rows * d);
    p.open_unit = reinterpret_cast<int32_t *>(p.part_ml + rows);
    p.goes_on = p.open_unit + kMaxBlocks;
    p.flags = dev_flags;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return pool->dtype == STOM_BF16 ? dispatch<__nv_bfloat16>(p, d, sms, s) : dispatch<__half>(p, d, sms, s);
}
