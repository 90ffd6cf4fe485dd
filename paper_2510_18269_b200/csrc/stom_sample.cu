// The choice of the next token from a row of logits (stom_sample_tokens): temperature, top-k, top-p, min-p and a draw
// with a given random number, in the order "largest logit first, of equal ones the lowest index first".
//
// Nothing is sorted.  The tokens kept are a prefix of that order, and so is everything before the token drawn; each of
// the settings asks for ONE place in the order, given by a rank (top-k), by a mass (top-p, the draw) or by a logit
// (min-p).  A place is found through counts and masses of 4 096 or 2 048 ranges of KEYS (the logit's bits made to order as
// unsigned numbers), then among the keys of one range; within one key all weights are equal and the rest is a division.
//
// A row belongs to a cluster of up to 16 blocks, each with a slice of it.  Every block adds up its share of the ranges
// over the cluster (distributed shared memory), and the blocks agree on a place through one cluster barrier.
//   16-bit logits: one count per bit pattern (65 536 16-bit counters, hence slices below 65 536) in shared memory.  One
//     shared-memory atomic per logit is all the work that grows with the row; order, infinities and NaN are sorted out
//     when the counters are read, the exponential is taken per DISTINCT logit, and a mass is count times weight.
//   binary32 logits: ranges of equal width in (x_max - x) / T, so that the logits spread over them; counts, and masses as
//     sums of integers, three limbs of 16 bits or more (by the slice), so that the order of the atomics leaves no trace.
//     The keys of a range are gathered and ranked; a range with more than kGather of them is cut into 2 048
//     again.  With top-k everything else is decided among the keys ranked for it, if they are no more.
// With 100 000 tokens left to draw from, binary32 sums would move a border between two tokens by more than some tokens'
// whole weight.  The masses of ranges are whole numbers of UNITS in 64 bits, 2^-43 (the longest rows) to 2^-51 of the
// largest weight, the smallest that a row's sum has room for: their sums are
// exact and never fall, so that exactly one range holds a place and all blocks of a cluster see the same one.  A range is
// rounded to a unit once, after it has been added up (16 bits: in binary64; binary32: in units smaller by up to n / 512), so
// that the masses of a row are off by half a unit for each of 4 096 ranges (2 048, and 256 units) at most: 2^-34 of the
// largest weight up to 131 072 logits, 2^-32 for the longest rows.  Within the last few keys weights and sums are
// binary64.
//
// What bounds it: not memory (128 rows of 151 001 bf16 logits are 6 us at the copy rate) but the chain of steps a row has
// to go through, each a barrier, a look into another block's memory or a binary64 sum away from the next.  Measured: 128
// such rows with mixed settings 78 us, three rounds of 49 clusters of 3 blocks; a block's 24 us are 6 for its 50 000
// logits (4.3 cycles for a warp's shared-memory atomic, the rest the patterns' arithmetic), 5 for the ranges, 2 to 2.5 for
// every place asked for, 3 for the index.  One row of 128 000 logits on 16 blocks: bf16 21 us, binary32 20 us with top-k,
// 36 us with top-p alone (a ranking for each of two places).
#include "stom_kv.cuh"
#include "stom_sample.h"

#include <atomic>

namespace stom {

namespace {

constexpr int kMostRanges = 4096;
constexpr int kMaxCluster = 16;
constexpr uint32_t kGather = 1024;   // keys that are ranked at once (binary32)
constexpr int kSummers = 256;        // threads that add up a block's ranges

struct SampleParams {
    const char *logits;
    int64_t row_stride;
    int32_t n, slice;
    int32_t unit_bits, limb;     // a unit is 2^-unit_bits; bits of a limb (binary32)
    float per_nat;               // binary32: first ranges to a factor e of the weight
    uint32_t log2_per_range;     // and the powers of two from one to the next, in 2^-16
    int32_t most_lift;           // units that weights are rounded to are down to 2^-most_lift of those of the sums
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *logprob;
    uint32_t *flags;
};

// ---- keys: unsigned numbers in the order of the logits, the bits with the sign turned (positive) or all turned
// (negative).  -0 takes the key of +0; 0 stands for what is never drawn (NaN, -inf).
template <typename T>
struct Keys;
template <uint32_t INF>
struct Keys16 {
    static constexpr uint32_t kInf = INF, kZero = 0x8000u, kLowest = 0xffffu ^ (0x8000u | (INF - 1u));   // lowest: of a finite logit
    static __device__ __forceinline__ uint32_t bits(uint32_t key) { return key & 0x8000u ? key ^ 0x8000u : key ^ 0xffffu; }
    static __device__ __forceinline__ uint32_t of(uint32_t b, bool &nan) {
        const uint32_t mag = b & 0x7fffu, key = b & 0x8000u ? b ^ 0xffffu : b ^ 0x8000u;
        nan |= mag > INF;
        return mag > INF || b == (0x8000u | INF) ? 0u : mag ? key : kZero;
    }
};
template <>
struct Keys<__nv_bfloat16> : Keys16<0x7f80u> {
    static __device__ __forceinline__ double value(uint32_t k) { return (double)__uint_as_float(bits(k) << 16); }
};
template <>
struct Keys<__half> : Keys16<0x7c00u> {
    static __device__ __forceinline__ double value(uint32_t k) {
        return (double)__half2float(__ushort_as_half((unsigned short)bits(k)));
    }
};
template <>
struct Keys<float> {
    static constexpr uint32_t kLowest = 0xffffffffu ^ 0xff7fffffu;
    static __device__ __forceinline__ uint32_t of(uint32_t b, bool &nan) {
        const uint32_t mag = b & 0x7fffffffu, key = b & 0x80000000u ? b ^ 0xffffffffu : b ^ 0x80000000u;
        nan |= mag > 0x7f800000u;
        return mag > 0x7f800000u || b == 0xff800000u ? 0u : mag ? key : 0x80000000u;
    }
    static __device__ __forceinline__ float single(uint32_t k) {
        return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : k ^ 0xffffffffu);
    }
    static __device__ __forceinline__ double value(uint32_t k) { return (double)single(k); }
};

template <typename T>
struct Plan {
    static constexpr bool kHalf = sizeof(T) == 2;
    static constexpr int kRanges = kHalf ? kMostRanges : 2048;
    static constexpr int kThreads = kHalf ? 1024 : 512;
    static constexpr int kRaw = kHalf ? 65536 * 2 : kRanges * 16;     // counters
    // behind them: the list of ranges that are not empty (16 bits); the keys gathered, ranked, their sums (binary32)
    static constexpr int kList = kHalf ? kRanges * 2 : kGather * (4 + 4 + 4 + 4 + 8);
    static int share(int cluster) { return ((kRanges + cluster - 1) / cluster + 31) & ~31; }   // whole words of bits
    static int smem(int cluster) { return kRaw + kList + (kHalf ? 1 : 2) * share(cluster) * 12; }
};

// ---- distributed shared memory
__device__ __forceinline__ uint4 ld_cluster_u4(const void *mine, uint32_t rank) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(cluster_addr(mine, rank))
                 : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster_u(const uint32_t *mine, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr(mine, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_u(uint32_t *mine, uint32_t rank, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(mine, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_u64(uint64_t *mine, uint32_t rank, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(mine, rank)), "l"(v) : "memory");
}
// A block's memory may be written from another one only once it has begun: the two halves of a barrier for that
__device__ __forceinline__ void cluster_begun() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_all_begun() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// ---- what is asked for: a place in the order
enum Kind { BY_RANK, BY_MASS, PAST_MASS, BY_KEY };   // rank; first whose mass upto reaches / exceeds; up to a key
struct Query {
    Kind kind;
    uint32_t rank, key;
    double mass;
};
struct Place {           // the key of a place and what stands before that key
    uint32_t key, before, count;
    double mass_before, weight;
};
struct Cell {            // a range, and what stands before it
    uint32_t range, before, count;
    double mass_before;
};

struct Shared {
    uint32_t warp_count[32];
    uint64_t warp_mass[32];      // or the bits of binary64 sums
    uint32_t nan, lowest, listed;
    // what every block of the cluster tells all others: its ranges' counts, masses and last range that is not empty + 1
    // (per level), its largest and (binary32) least key, how many keys it has gathered, how many it has of the key drawn
    uint32_t all_count[2][kMaxCluster], all_lowest[2][kMaxCluster], all_max[kMaxCluster], all_min[kMaxCluster], all_listed[kMaxCluster], all_own[kMaxCluster];
    uint64_t all_mass[2][kMaxCluster];
    // 16 bits: ranges with logits of this block's slice; of this block's share, which of them every block has
    uint32_t occupied[kMostRanges / 32], held[kMostRanges / 32 + kMaxCluster];
    uint32_t ans_range[8], ans_before[8], ans_count[8];   // answers to queries, a slot each in turn
    double ans_mass[8];
    uint32_t first, last;
    double power[64];                              // 2^(j/64)
    Place place;
    // settled so far: tokens kept and their mass; the key drawn, how many equal ones come before it
    uint32_t count, nth;
    double mass;
};

// A row as one block of its cluster sees it
template <typename T>
struct Row {
    using K = Keys<T>;
    using P = Plan<T>;
    static constexpr int kThreads = P::kThreads;
    static constexpr bool kHalf = P::kHalf;
    static constexpr int kRanges = P::kRanges;
    Shared &sh;
    uint32_t *raw;               // counters
    uint8_t *list;
    uint32_t *cnt[2];            // of this block's share of the ranges, highest keys first: counts and masses, per level
    uint64_t *mass[2];
    const T *x;                  // this block's slice
    int n;
    uint32_t rank, blocks, share, mine;   // ranges of a block, and of this one
    double top, t, per_log2, unit;   // per_log2: log2(e) / t
    int unit_bits, limb;
    float half_top, per_range;   // binary32: half of top; ranges per two units of x
    uint32_t log2_per_range;     // powers of two from one range to the next, in 2^-16
    int most_lift;
    int tid;
    uint32_t slot = 0;
    // running sums of one level: before this thread's ranges, and with them
    struct Sums {
        uint32_t c0, c1, total;
        uint64_t m0, m1, all;
        uint32_t lowest;
    } sums[2];
    uint32_t low_key, high_key, shift;   // binary32: the keys that the second level covers, 2^shift to a range
    int inner;                           // and its units: 2^-inner of the first level's

    // Zero below e^-700: close to where binary64 ends, the last steps of an exponential would decide what is kept.
    __device__ __forceinline__ double weight(double v) const {
        const double y = v == top ? 0.0 : (v - top) / t;
        return y < -700.0 ? 0.0 : exp(y);
    }
    // The same in 2^-lift units (down to 2^-100), by 2^y = 2^(k/64) 2^r, |r| <= 1/128, the second factor by its Taylor polynomial
    // (the term left out is below 4e-17): without a branch, 11 binary64 operations in the place of a division and exp.
    __device__ __forceinline__ double units(double v, int lift = 0) const {
        const double y = v == top ? 0.0 : fmax((v - top) * per_log2, -100.0);
        const double shifted = fma(y, 64.0, 6755399441055744.0);          // 1.5 * 2^52: rounds to a whole number
        const int k = __double2loint(shifted);
        const double r = fma(shifted - 6755399441055744.0, -1.0 / 64.0, y);
        double e = 1.3333558146428443e-3;                                  // ln(2)^5 / 5!, and so on
        e = fma(e, r, 9.618129107628477e-3);
        e = fma(e, r, 5.5504108664821576e-2);
        e = fma(e, r, 2.402265069591007e-1);
        e = fma(e, r, 6.931471805599453e-1);
        e = fma(e, r, 1.0) * sh.power[k & 63];
        // times 2^(k >> 6) / unit, by the exponent
        return __hiloint2double(__double2hiint(e) + ((k >> 6) + unit_bits + lift) * (1 << 20), __double2loint(e));
    }

    // Block r of the cluster as the i-th to look at.  Every block begins with itself: if all began with block 0, they
    // would wait for that one's memory together, then for the next.
    __device__ __forceinline__ uint32_t turn(uint32_t i) const {
        const uint32_t r = rank + i;
        return r < blocks ? r : r - blocks;
    }
    // 16 bits: how many logits of the row have this key
    __device__ __forceinline__ uint32_t count16(uint32_t b, uint32_t r) const {
        return (ld_cluster_u(raw + (b >> 1), r) >> (16 * (b & 1))) & 0xffffu;
    }
    __device__ __forceinline__ uint32_t count_of(uint32_t key, bool &nan) const {
        const uint32_t b = K::bits(key), at = smem_u32(raw + (b >> 1)), half = 16 * (b & 1);
        uint32_t c = 0;
#pragma unroll 4
        for (uint32_t i = 0; i < blocks; ++i) {
            uint32_t a, w;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(turn(i)));
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(a) : "memory");
            c += (w >> half) & 0xffffu;
        }
        if (key == K::kZero)
            for (uint32_t i = 0; i < blocks; ++i) c += count16(0x8000u, turn(i));
        bool is_nan = false;
        if (K::of(b, is_nan) != key || key == 0) {   // NaN (all bits set is the one whose place is key 0), -inf, or -0
            nan |= is_nan && c;
            c = 0;
        }
        return c;
    }

    __device__ __forceinline__ uint32_t bits_at(int i) const {
        if constexpr (kHalf) return reinterpret_cast<const unsigned short *>(x)[i];
        else return reinterpret_cast<const uint32_t *>(x)[i];
    }
    // words(four words, index of the first logit) over the slice, 16 bytes at a time, one(bits, index) for its ends
    template <typename W, typename F>
    __device__ __forceinline__ void each(W words, F one) const {
        constexpr int kV = 16 / sizeof(T), kBatch = 4;
        const int off = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
        const int head = min(n, off ? kV - off : 0), vecs = (n - head) / kV;
        const uint4 *v = reinterpret_cast<const uint4 *>(x + head);
        for (int i = tid; i < vecs; i += kBatch * kThreads) {
            uint4 q[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (i + j * kThreads < vecs) q[j] = v[i + j * kThreads];
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (i + j * kThreads < vecs) words(q[j], head + (i + j * kThreads) * kV);
        }
        if (tid < head) one(bits_at(tid), tid);
        const int rest = head + vecs * kV + tid;
        if (rest < n) one(bits_at(rest), rest);
    }
    // f(bits, index) over the slice
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        each([&](const uint4 &q, int at) {
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (kHalf) {
                    f(w[e] & 0xffffu, at + 2 * e);
                    f(w[e] >> 16, at + 2 * e + 1);
                } else {
                    f(w[e], at + e);
                }
            }
        }, f);
    }
    // The index among the equal ones, in any order, of every logit with this key; how many there are
    __device__ __forceinline__ uint32_t collect(uint32_t key, uint32_t *found, uint32_t room) {
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        bool ignore = false;
        each([&](uint32_t b, int i) {
            if (K::of(b, ignore) == key) {
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                if (at < room) found[at] = i;
            }
        });
        __syncthreads();
        return sh.listed;
    }

    __device__ __forceinline__ void zero_raw() {
        for (int i = tid; i < P::kRaw / 16; i += kThreads) reinterpret_cast<uint4 *>(raw)[i] = make_uint4(0, 0, 0, 0);
    }

    // Sums of a level over the cluster, from cnt[level] and mass[level]
    __device__ __forceinline__ void sum_up(int level) {
        const int per = (share + kSummers - 1) / kSummers, first = tid * per, last = tid < kSummers ? min((int)mine, first + per) : 0;
        const int lane = tid & 31, warp = tid >> 5;
        Sums &s = sums[level];
        uint32_t c = 0, low = 0;
        uint64_t m = 0;
        for (int j = first; j < last; ++j) {
            c += cnt[level][j];
            m += mass[level][j];
            if (cnt[level][j]) low = j + 1;
        }
        s.c1 = c;
        s.m1 = m;
        if (tid == 0) sh.lowest = 0;
        __syncthreads();
        if (tid < kSummers) {
            low = __reduce_max_sync(~0u, low);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t vc = __shfl_up_sync(~0u, s.c1, o);
                const uint64_t vm = __shfl_up_sync(~0u, s.m1, o);
                if (lane >= o) {
                    s.c1 += vc;
                    s.m1 += vm;
                }
            }
            if (lane == 31) {
                sh.warp_count[warp] = s.c1;
                sh.warp_mass[warp] = s.m1;
                if (low) atomicMax(&sh.lowest, low);
            }
        }
        __syncthreads();
        uint32_t c_all = 0;
        uint64_t m_all = 0;
#pragma unroll
        for (int w = 0; w < kSummers / 32; ++w) {
            if (w == warp) {
                s.c1 += c_all;
                s.m1 += m_all;
            }
            c_all += sh.warp_count[w];
            m_all += sh.warp_mass[w];
        }
        s.c0 = s.c1 - c;
        s.m0 = s.m1 - m;
        if (tid < blocks) {
            st_cluster_u(&sh.all_count[level][rank], tid, c_all);
            st_cluster_u64(&sh.all_mass[level][rank], tid, m_all);
            st_cluster_u(&sh.all_lowest[level][rank], tid, sh.lowest);
        }
        cluster_sync();
        // a lane for each block
        const bool is = lane < (int)blocks;
        const uint32_t c_of = is ? sh.all_count[level][lane] : 0u, l_of = is ? sh.all_lowest[level][lane] : 0u;
        const uint64_t m_of = is ? sh.all_mass[level][lane] : 0ull;
        const uint32_t before = __reduce_add_sync(~0u, lane < (int)rank ? c_of : 0u);
        s.total = __reduce_add_sync(~0u, c_of);
        s.lowest = __reduce_max_sync(~0u, l_of ? lane * share + l_of : 0u);
        uint64_t mb = lane < (int)rank ? m_of : 0ull, all = m_of;
#pragma unroll
        for (int o = kMaxCluster / 2; o; o >>= 1) {
            mb += __shfl_xor_sync(~0u, mb, o);
            all += __shfl_xor_sync(~0u, all, o);
        }
        mb = __shfl_sync(~0u, mb, 0);
        s.all = __shfl_sync(~0u, all, 0);
        s.c0 += before;
        s.c1 += before;
        s.m0 += mb;
        s.m1 += mb;
    }

    // The range that holds the place asked for, with what stands before it; agreed on by all blocks
    __device__ __forceinline__ Cell find(int level, const Query &q, uint32_t base, double mass_base) {
        const Sums &s = sums[level];
        const double step = level ? __hiloint2double((1023 - unit_bits - inner) << 20, 0) : unit;
        const int per = (share + kSummers - 1) / kSummers, first = tid * per, last = tid < kSummers ? min((int)mine, first + per) : 0;
        const uint32_t at = slot++ & 7u;
        auto reached = [&](uint32_t c, uint64_t m) {   // never true and then false along the order
            if (c == 0) return false;
            if (c == s.total) return true;
            if (q.kind == BY_RANK) return base + c > q.rank;
            const double upto = mass_base + (double)m * step;
            return q.kind == BY_MASS ? upto >= q.mass : upto > q.mass;
        };
        bool holds = false;
        int wanted = -1;
        if (first < last) {
            if (q.kind == BY_KEY) {
                wanted = (int)range_of(level, q.key) - (int)(rank * share);
                holds = wanted >= first && wanted < last;
            } else {
                holds = s.c1 != s.c0 && reached(s.c1, s.m1) && !reached(s.c0, s.m0);
            }
        }
        if (holds) {
            uint32_t c = s.c0, hit_c = s.c0, hit = first;
            uint64_t m = s.m0, hit_m = s.m0;
            for (int j = first; j < last; ++j) {
                if (q.kind == BY_KEY ? j == wanted : cnt[level][j] != 0) {
                    hit = j, hit_c = c, hit_m = m;
                    if (q.kind == BY_KEY || reached(c + cnt[level][j], m + mass[level][j])) break;
                }
                c += cnt[level][j];
                m += mass[level][j];
            }
            for (uint32_t r = 0; r < blocks; ++r) {
                st_cluster_u(&sh.ans_range[at], r, rank * share + hit);
                st_cluster_u(&sh.ans_before[at], r, base + hit_c);
                st_cluster_u(&sh.ans_count[at], r, cnt[level][hit]);
                st_cluster_u64(reinterpret_cast<uint64_t *>(&sh.ans_mass[at]), r, (uint64_t)__double_as_longlong(mass_base + (double)hit_m * step));
            }
        }
        cluster_sync();
        return Cell{min(sh.ans_range[at], (uint32_t)kRanges - 1), sh.ans_before[at], sh.ans_count[at], sh.ans_mass[at]};
    }
    __device__ __forceinline__ uint32_t range_of(int level, uint32_t key) const {
        if constexpr (kHalf) return kRanges - 1 - (key >> 4);
        else return level ? (high_key - key) >> shift : range_at(K::single(key));
    }
    // binary32, first level: equal widths in x, about 64 of them to a factor e of the weight, down to half a unit.  Every
    // step of it is monotonous, so a range is a run of keys.  Halves, because the whole difference of two finite logits may
    // not be finite.
    __device__ __forceinline__ uint32_t range_at(float v) const {
        const float f = fmaf(v, -0.5f, half_top) * per_range;
        return 2.f * half_top == v ? 0u : (uint32_t)fminf(f, (float)(kRanges - 1));
    }

    // The weights of a range are at most 2^-(its place times log2_per_range), to 2^-15 by binary32's rounding of the place,
    // so that they can be added up in units that much smaller; as many as `most_lift` are enough for n of them.  (More
    // would cost: a weight is added limb by limb, those that are not zero.)
    __device__ __forceinline__ int lift_of(uint32_t range) const { return min((int)(range * log2_per_range >> 16), most_lift); }

    __device__ __forceinline__ Place ask(const Query &q) {
        if constexpr (!kHalf)
            if (all_ranked) {
                pick(q);
                return sh.place;
            }
        Cell cell = find(0, q, 0, 0.0);
        if constexpr (kHalf) {
            // 16 keys, a thread each; the first that reaches what is asked for, or (by key: always) the last
            if (tid < 32) {
                const uint32_t key = (kRanges - 1 - cell.range) * 16 + 15 - (tid & 15);
                bool nan = false;
                uint32_t c = tid < 16 ? count_of(key, nan) : 0u;
                const double w = c ? units(K::value(key)) * unit : 0.0;
                uint32_t c1 = c;
                double m1 = c * w;
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) {
                    const uint32_t vc = __shfl_up_sync(~0u, c1, o);
                    const double vm = __shfl_up_sync(~0u, m1, o);
                    if (tid >= o) {
                        c1 += vc;
                        m1 += vm;
                    }
                }
                const double mb = cell.mass_before, ahead = __shfl_up_sync(~0u, m1, 1);
                const bool in = c && (q.kind != BY_KEY || key >= q.key);
                const bool reached = in && (q.kind == BY_RANK ? cell.before + c1 > q.rank
                                            : q.kind == BY_MASS ? mb + m1 >= q.mass : q.kind == PAST_MASS && mb + m1 > q.mass);
                const uint32_t hits = __ballot_sync(~0u, reached), ins = __ballot_sync(~0u, in);
                const int pick = hits ? __ffs(hits) - 1 : ins ? 31 - __clz(ins) : -1;
                if (tid == max(pick, 0))
                    sh.place = pick < 0 ? Place{0, cell.before, 0, mb, 0.0}
                                        : Place{key, cell.before + c1 - c, c, mb + (tid ? ahead : 0.0), w};
            }
            __syncthreads();
        } else {
            // the keys of the range: from the lowest whose range is not beyond it to below the lowest of the one ahead
            low_key = lowest_within(cell.range);
            high_key = cell.range ? lowest_within(cell.range - 1) - 1 : best;
            inner = lift_of(cell.range);
            while (cell.count > kGather && low_key != high_key) {
                const uint32_t span = high_key - low_key;
                shift = max(0, 21 - __clz(span));                      // span >> shift < kRanges = 2^11
                tally<1, true>();
                cell = find(1, q, cell.before, cell.mass_before);
                high_key -= cell.range << shift;
                low_key = max(low_key, high_key - min(high_key, (1u << shift) - 1));
            }
            const double mb = cell.mass_before;
            if (low_key == high_key) {
                if (tid == 0) {
                    const bool in = cell.count && (q.kind != BY_KEY || high_key >= q.key);
                    sh.place = in ? Place{high_key, cell.before, cell.count, mb, units(K::value(high_key)) * unit}
                                  : Place{0, cell.before, 0, mb, 0.0};
                }
                __syncthreads();
            } else {
                rank_keys(cell.before, mb);
                pick(q);
            }
        }
        return sh.place;
    }

    // ---- binary32
    uint32_t best;               // the largest key
    __device__ __forceinline__ uint32_t lowest_within(uint32_t range) const {   // lowest key of a range up to this one
        uint32_t low = K::kLowest - 1, high = best;                             // low is beyond, high is within
        if (range >= kRanges - 1) return K::kLowest;
        while (high - low > 1) {
            const uint32_t step = (high - low + 31) / 32;
            const uint64_t k = (uint64_t)low + (uint64_t)step * ((tid & 31) + 1);
            const uint32_t yes = __ballot_sync(~0u, k >= high || range_at(K::single((uint32_t)k)) <= range);
            const int j = __ffs(yes) - 1;
            const uint64_t up = (uint64_t)low + (uint64_t)step * (j + 1);
            low = low + step * j;
            high = up < high ? (uint32_t)up : high;
        }
        return high;
    }

    // Counts and masses of a level (1: of the keys from low_key to high_key), summed over the cluster
    // MASSES false: counts alone, which is all that ranking the first top_k needs.
    template <int LEVEL, bool MASSES>
    __device__ __forceinline__ void tally() {
        zero_raw();
        __syncthreads();
        uint32_t beyond = 0;                                   // of the last range, where everything far down is
        uint64_t beyond_mass = 0;
        auto add = [&](uint32_t k, uint32_t range, uint64_t w) {
            if (!k || (LEVEL && (k < low_key || k > high_key))) return;
            if (LEVEL == 0 && range == kRanges - 1) {          // weights below half a unit of the sums
                ++beyond;
                beyond_mass += w;
                return;
            }
            uint32_t *r = raw + 4 * range;
            atomicAdd(r, 1u);
            if (!MASSES) return;
            const uint32_t mask = (1u << limb) - 1, w0 = (uint32_t)w & mask, w1 = (uint32_t)(w >> limb) & mask, w2 = (uint32_t)(w >> 2 * limb);
            if (w0) atomicAdd(r + 1, w0);
            if (w1) atomicAdd(r + 2, w1);
            if (w2) atomicAdd(r + 3, w2);
        };
        // to whole units of its range: 2^52 added leaves them in the low bits
        auto whole = [&](uint32_t k, uint32_t range) {
            const double w = units(K::value(k), LEVEL ? inner : lift_of(range));
            return (uint64_t)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffull;
        };
        each([&](const uint4 &q, int) {                        // four at a time: a weight is a chain of 12 operations
            const uint32_t b[4] = {q.x, q.y, q.z, q.w};
            uint32_t k[4], range[4];
            uint64_t w[4];
            bool nan = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                k[e] = K::of(b[e], nan);
                range[e] = range_of(LEVEL, k[e] ? k[e] : best);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = MASSES ? whole(k[e] ? k[e] : best, range[e]) : 0ull;
#pragma unroll
            for (int e = 0; e < 4; ++e) add(k[e], range[e], w[e]);
        }, [&](uint32_t b, int) {
            bool nan = false;
            const uint32_t k = K::of(b, nan), range = range_of(LEVEL, k ? k : best);
            add(k, range, MASSES ? whole(k ? k : best, range) : 0ull);
        });
        if (LEVEL == 0) {
            beyond = __reduce_add_sync(~0u, beyond);
            if (MASSES) {
#pragma unroll
                for (int o = 16; o; o >>= 1) beyond_mass += __shfl_xor_sync(~0u, beyond_mass, o);
            }
            if (beyond && (tid & 31) == 0) {
                uint32_t *r = raw + 4 * (kRanges - 1);
                const uint32_t mask = (1u << limb) - 1;
                atomicAdd(r, beyond);
                if (beyond_mass) {
                    atomicAdd(r + 1, (uint32_t)beyond_mass & mask);
                    atomicAdd(r + 2, (uint32_t)(beyond_mass >> limb) & mask);
                    atomicAdd(r + 3, (uint32_t)(beyond_mass >> 2 * limb));
                }
            }
        }
        cluster_sync();
        for (uint32_t j = tid; j < mine; j += kThreads) {
            const uint32_t *r = raw + 4 * (rank * share + j);
            uint32_t c = 0;
            uint64_t w = 0;
#pragma unroll
            for (uint32_t i = 0; i < kMaxCluster; ++i)
                if (i < blocks) {
                    const uint4 v = ld_cluster_u4(r, turn(i));
                    c += v.x;
                    w += (uint64_t)v.y + ((uint64_t)v.z << limb) + ((uint64_t)v.w << 2 * limb);
                }
            if (LEVEL == 0 && MASSES) {                        // to units of the sums, rounded
                const int lift = lift_of(rank * share + j);
                w = lift ? (w + (1ull << (lift - 1))) >> lift : w;
            }
            cnt[LEVEL][j] = c;
            mass[LEVEL][j] = w;
        }
        __syncthreads();
        sum_up(LEVEL);
    }

    // Every block gathers the at most kGather keys from low_key to high_key and ranks them, `base` and `mass_base` ahead of
    // them: afterwards order[i] is the i-th of them, upto[i] their mass up to it.  (`own` is read by the other blocks until
    // the next barrier of the cluster: a gathering always follows a find.)
    struct Ranked {
        uint32_t m, base;
        double mass_base;
    } ranked;
    __device__ __forceinline__ uint32_t *own() const { return reinterpret_cast<uint32_t *>(list); }
    __device__ __forceinline__ uint32_t *order() const { return own() + 2 * kGather; }
    __device__ __forceinline__ uint32_t *above() const { return own() + 3 * kGather; }   // keys above one; high half: equal ones
    __device__ __forceinline__ double *upto() const { return reinterpret_cast<double *>(own() + 4 * kGather); }
    __device__ __forceinline__ void rank_keys(uint32_t base, double mass_base) {
        uint32_t *keys = own() + kGather;                              // all blocks'
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        each([&](uint32_t b, int) {
            bool nan = false;
            const uint32_t k = K::of(b, nan);
            if (k && k >= low_key && k <= high_key) {
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                if (at < kGather) own()[at] = k;
            }
        });
        __syncthreads();
        if (tid < blocks) st_cluster_u(&sh.all_listed[rank], tid, min(sh.listed, kGather));
        cluster_sync();
        const int lane = tid & 31, warp = tid >> 5;
        const uint32_t of = lane < (int)blocks ? sh.all_listed[lane] : 0u;
        const uint32_t m = min(__reduce_add_sync(~0u, of), kGather);
        for (uint32_t r = warp; r < blocks; r += kThreads / 32) {      // a warp for each block
            const uint32_t first = __reduce_add_sync(~0u, lane < (int)r ? of : 0u), k = __shfl_sync(~0u, of, r);
            for (uint32_t i = lane; i < k; i += 32)
                if (first + i < kGather) keys[first + i] = ld_cluster_u(own() + i, r);
        }
        __syncthreads();
        for (uint32_t i = tid; i < m; i += kThreads) {
            const uint32_t k = keys[i];
            uint32_t more = 0, equal = 0, ahead = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < m; ++j) {
                const uint32_t o = keys[j];
                more += o > k;
                equal += o == k;
                ahead += o == k && j < i;
            }
            order()[more + ahead] = k;
            above()[more + ahead] = more | equal << 16;
        }
        __syncthreads();
        // masses up to each, in order: two neighbours a thread
        const uint32_t i0 = 2 * tid;
        const double w0 = i0 < m ? units(K::value(order()[i0])) * unit : 0.0;
        const double w1 = i0 + 1 < m ? units(K::value(order()[i0 + 1])) * unit : 0.0;
        double sum = w0 + w1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) sh.warp_mass[warp] = (uint64_t)__double_as_longlong(sum);
        __syncthreads();
        for (int w = 0; w < warp && 64 * warp < (int)m; ++w) sum += __longlong_as_double((long long)sh.warp_mass[w]);
        if (i0 < m) upto()[i0] = sum - w1;
        if (i0 + 1 < m) upto()[i0 + 1] = sum;
        ranked = Ranked{m, base, mass_base};
        __syncthreads();
    }
    // The place among them
    __device__ __forceinline__ void pick(const Query &q) {
        if (tid == 0) {
            sh.first = ~0u;
            sh.last = 0;
        }
        __syncthreads();
        for (uint32_t i = tid; i < ranked.m; i += kThreads) {
            const double mass_to = ranked.mass_base + upto()[i];
            const bool in = q.kind != BY_KEY || order()[i] >= q.key;
            const bool reached = q.kind == BY_RANK ? ranked.base + i + 1 > q.rank
                                 : q.kind == BY_MASS ? mass_to >= q.mass : q.kind == PAST_MASS && mass_to > q.mass;
            if (in && reached) atomicMin(&sh.first, i);
            if (in && (i + 1 == ranked.m || (q.kind == BY_KEY && order()[i + 1] < q.key))) sh.last = i + 1;
        }
        __syncthreads();
        if (tid == 0) {
            if (sh.first == ~0u && sh.last == 0) {
                sh.place = Place{0, ranked.base, 0, ranked.mass_base, 0.0};
            } else {
                const uint32_t i = sh.first != ~0u ? sh.first : sh.last - 1, more = above()[i] & 0xffffu;
                sh.place = Place{order()[i], ranked.base + more, above()[i] >> 16, ranked.mass_base + (more ? upto()[more - 1] : 0.0),
                                 units(K::value(order()[i])) * unit};
            }
        }
        __syncthreads();
    }
    // The keys of the first `rank` tokens and what shares their last range are ranked for good, if they are few enough
    bool all_ranked = false;
    __device__ __forceinline__ void rank_first(uint32_t rank_asked) {
        const Cell cell = find(0, Query{BY_RANK, rank_asked, 0, 0.0}, 0, 0.0);
        if (cell.before + cell.count > kGather) return;
        low_key = lowest_within(cell.range);
        high_key = best;
        rank_keys(0, 0.0);
        all_ranked = true;
    }

    // ---- 16 bits
    // One count per bit pattern.  The patterns that stand for a forbidden token, -inf and the type's lowest value, may be
    // most of a row, and atomics on one address wait for one another: the first is left out, the second counted aside.
    __device__ __forceinline__ void count_patterns() {
        const uint32_t base = smem_u32(raw);
        constexpr uint32_t kMinusInf = 0x8000u | K::kInf, kMin = kMinusInf - 1;
        uint32_t lowest = 0;
        auto add = [&](uint32_t b, uint32_t twice) {     // twice: the pattern times two, with anything above bit 16
            lowest += b == kMin;
            if (b < kMin || b > kMinusInf)
                asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(base + (twice & 0x1fffcu)), "r"(b & 1u ? 0x10000u : 1u) : "memory");
        };
        each([&](const uint4 &q, int) {
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                add(w[e] & 0xffffu, w[e] << 1);
                add(w[e] >> 16, w[e] >> 15);
            }
        }, [&](uint32_t b, int) { add(b, b << 1); });
        lowest = __reduce_add_sync(~0u, lowest);
        if (lowest && (tid & 31) == 0) atomicAdd(raw + (kMin >> 1), kMin & 1u ? lowest << 16 : lowest);
    }
    // Which ranges have logits of this block, and its largest key
    __device__ __forceinline__ uint32_t survey() {
        for (int i = tid; i < kRanges; i += kThreads) {
            const uint32_t block = K::bits((kRanges - 1 - i) * 16) >> 4;    // of 16 patterns, side by side
            const uint4 *c = reinterpret_cast<const uint4 *>(raw) + 2 * block;
            const uint4 a = c[0], b = c[1];
            bool some = a.x | a.y | a.z | a.w | b.x | b.y | b.z | b.w;
            if (i == kRanges - 1 - (int)(K::kZero >> 4)) some |= raw[0x8000u >> 1] & 0xffffu;   // -0 counts as +0
            const uint32_t bits = __ballot_sync(~0u, some);
            if ((tid & 31) == 0) sh.occupied[i >> 5] = bits;
        }
        __syncthreads();
        cluster_all_begun();
        if (tid < kRanges / 32) {
            const uint32_t words = share / 32, to = tid / words;
            st_cluster_u(&sh.held[rank * words + tid - to * words], to, sh.occupied[tid]);
        }
        uint32_t key = 0;
        if (tid < 32) {
            for (int w = 0; w < kRanges / 32 && !key; w += 32) {
                const uint32_t mine32 = sh.occupied[w + tid];
                uint32_t words = __ballot_sync(~0u, mine32 != 0);
                while (words && !key) {
                    const int j = __ffs(words) - 1;
                    words &= words - 1;
                    uint32_t bits = __shfl_sync(~0u, mine32, j);
                    while (bits && !key) {
                        const int i = (w + j) * 32 + __ffs(bits) - 1;
                        bits &= bits - 1;
                        const uint32_t k = (kRanges - 1 - i) * 16 + 15 - (tid & 15), b = K::bits(k);
                        uint32_t c = (raw[b >> 1] >> (16 * (b & 1))) & 0xffffu;
                        if (k == K::kZero) c += raw[0x8000u >> 1] & 0xffffu;
                        bool nan = false;
                        const uint32_t yes = __ballot_sync(~0u, c && K::of(b, nan) == k);
                        if (yes) key = (kRanges - 1 - i) * 16 + 15 - (__ffs(yes) - 1);
                    }
                }
            }
        }
        return key;
    }
    // Counts and masses of the ranges, summed over the cluster.  What is not empty in any block goes to a list, and 16
    // threads take one of its ranges, a key each.  True if there was a NaN.
    __device__ __forceinline__ bool tally16() {
        unsigned short *ranges = reinterpret_cast<unsigned short *>(list);
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        for (uint32_t j = tid; j < share; j += kThreads) {                  // share and mine: multiples of 32
            if (j >= mine) continue;
            cnt[0][j] = 0;
            mass[0][j] = 0;
            const uint32_t lane = tid & 31;
            uint32_t bits = lane < blocks ? sh.held[lane * (share / 32) + j / 32] : 0u;
            bits = __reduce_or_sync(~0u, bits);
            uint32_t at = 0;
            if (lane == 0 && bits) at = atomicAdd(&sh.listed, (uint32_t)__popc(bits));
            at = __shfl_sync(~0u, at, 0);
            if (bits >> lane & 1u) ranges[at + __popc(bits & ((1u << lane) - 1))] = (unsigned short)j;
        }
        __syncthreads();
        const uint32_t n_list = sh.listed;
        bool nan = false;
        constexpr int kAtOnce = 2;
        for (uint32_t base = 0; base < n_list; base += kAtOnce * (kThreads / 16)) {
            uint32_t c[kAtOnce];
            double m[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const uint32_t i = base + k * (kThreads / 16) + (tid >> 4);
                const uint32_t key = i < n_list ? (kRanges - 1 - (rank * share + ranges[i])) * 16 + (tid & 15) : 0u;
                c[k] = i < n_list ? count_of(key, nan) : 0u;
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const uint32_t i = base + k * (kThreads / 16) + (tid >> 4);
                const uint32_t key = c[k] ? (kRanges - 1 - (rank * share + ranges[i])) * 16 + (tid & 15) : K::kZero;
                m[k] = c[k] * units(K::value(key));
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const uint32_t i = base + k * (kThreads / 16) + (tid >> 4);
#pragma unroll
                for (int o = 8; o; o >>= 1) {
                    c[k] += __shfl_xor_sync(~0u, c[k], o);
                    m[k] += __shfl_xor_sync(~0u, m[k], o);
                }
                if ((tid & 15) == 0 && i < n_list) {
                    cnt[0][ranges[i]] = c[k];
                    mass[0][ranges[i]] = __double2ull_rn(m[k]);   // one rounding for the 16 keys
                }
            }
        }
        __syncthreads();
        sum_up(0);
        return nan;
    }
};

// RES: blocks that a multiprocessor is to hold (binary32: 2 where the rows take several rounds; 128 rows of 128 000:
// 136 us, with 1 it is 163; but one row on its own is a microsecond faster with 1, which spills no registers)
template <typename T, int RES>
__global__ void __launch_bounds__(Plan<T>::kThreads, RES) sample_kernel(const __grid_constant__ SampleParams p) {
    using K = Keys<T>;
    using P = Plan<T>;
    constexpr int kThreads = P::kThreads;
    constexpr bool kHalf = P::kHalf;
    constexpr int kRanges = P::kRanges;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t blocks = cluster_size(), rank = cluster_rank();
    const int64_t row = blockIdx.x / blocks;
    const int begin = min((int64_t)rank * p.slice, (int64_t)p.n);

    Row<T> r{sh};
    r.raw = reinterpret_cast<uint32_t *>(smem);
    r.list = smem + P::kRaw;
    r.share = ((kRanges + blocks - 1) / blocks + 31) & ~31;
    r.mine = min(r.share, kRanges - min((uint32_t)kRanges, rank * r.share));
    r.mass[0] = reinterpret_cast<uint64_t *>(smem + P::kRaw + P::kList);
    r.mass[1] = r.mass[0] + r.share;
    r.cnt[0] = reinterpret_cast<uint32_t *>(r.mass[0] + (kHalf ? 1 : 2) * r.share);
    r.cnt[1] = r.cnt[0] + r.share;
    r.tid = tid;
    r.rank = rank;
    r.blocks = blocks;
    r.n = min(p.slice, p.n - begin);
    r.x = reinterpret_cast<const T *>(p.logits) + row * p.row_stride + begin;

    cluster_begun();
    if (kHalf) r.zero_raw();
    if (tid == 0) sh.nan = 0;
    if (tid < 64) sh.power[tid] = exp2(tid * (1.0 / 64.0));
    __syncthreads();
    grid_dependency_wait();

    // ---- settings.  A NaN counts as not given.
    float temp = p.temperature ? p.temperature[row] : 1.f;
    float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f, u = p.u ? p.u[row] : 0.f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    bool bad = false;
    if (isnan(temp)) bad = true, temp = 1.f;
    if (isnan(top_p)) bad = true, top_p = 1.f;
    if (isnan(min_p)) bad = true, min_p = 0.f;
    if (isnan(u)) bad = true, u = 0.f;
    u = fminf(fmaxf(u, 0.f), 0x1.fffffep-1f);
    const bool cold = temp <= 0.f;

    // ---- the largest key, and for 16-bit logits the count of every pattern
    uint32_t best = 0, least_key = ~0u;
    if constexpr (kHalf) {
        r.count_patterns();
        __syncthreads();
        best = r.survey();
    } else {
        bool nan = false;
        r.each([&](uint32_t b, int) {
            const uint32_t k = K::of(b, nan);
            best = max(best, k);
            least_key = min(least_key, k - 1);                 // 0 is none: it becomes the largest
        });
        best = __reduce_max_sync(~0u, best);
        least_key = __reduce_min_sync(~0u, least_key);
        if (lane == 0) {
            sh.warp_count[warp] = best;
            sh.warp_mass[warp] = least_key;
        }
        if (nan) sh.nan = 1;
        __syncthreads();
        if (warp == 0) {
            best = __reduce_max_sync(~0u, lane < kThreads / 32 ? sh.warp_count[lane] : 0u);
            least_key = __reduce_min_sync(~0u, lane < kThreads / 32 ? (uint32_t)sh.warp_mass[lane] : ~0u);
        }
    }
    if constexpr (!kHalf) cluster_all_begun();
    if (tid < blocks) {
        st_cluster_u(&sh.all_max[rank], tid, best);
        if (!kHalf) st_cluster_u(&sh.all_min[rank], tid, least_key);
    }
    cluster_sync();
    best = __reduce_max_sync(~0u, lane < (int)blocks ? sh.all_max[lane] : 0u);
    if (tid == 0 && p.flags && (sh.nan || (bad && rank == 0))) atomicOr(p.flags, STOM_FLAG_BAD_VALUE);
    r.top = K::value(best ? best : K::kLowest);
    r.t = cold ? 1.0 : (double)temp;
    r.per_log2 = 1.4426950408889634 / r.t;
    r.unit_bits = p.unit_bits;
    r.unit = __hiloint2double((1023 - p.unit_bits) << 20, 0);
    r.limb = p.limb;
    if constexpr (!kHalf) {
        r.best = best;
        r.half_top = 0.5f * K::single(best ? best : K::kLowest);
        // not 0 at an infinite temperature, so that +inf stays ahead of all else
        r.per_range = fmaxf(fminf(2.f * p.per_nat / (cold ? 1.f : temp), 3.0e38f), 1e-38f);
        r.log2_per_range = p.log2_per_range;
        r.most_lift = p.most_lift;
    }

    // ---- the place drawn: key, and how many equal ones come before it
    uint32_t key = best, nth = 0, kept = 1;
    double weight = 1.0, total = 1.0;
    if (kHalf && (best == 0 || cold)) {                        // the masses are not needed, but a NaN has to be told
        bool nan = false;
        for (uint32_t b = tid; b < 65536 / 2; b += kThreads)
            if (r.raw[b]) {
                bool a = false, c = false;
                K::of(2 * b, a);
                K::of(2 * b + 1, c);
                nan |= (a && (r.raw[b] & 0xffffu)) || (c && (r.raw[b] >> 16));
            }
        if (nan && p.flags) atomicOr(p.flags, STOM_FLAG_BAD_VALUE);
    }
    if (best == 0) {
        if (rank == 0 && tid == 0) {
            p.token[row] = -1;
            if (p.kept) p.kept[row] = 0;
            if (p.logprob) p.logprob[row] = -INFINITY;
        }
        return;
    }
    if (!cold) {
        if constexpr (kHalf) {
            if (r.tally16() && p.flags) atomicOr(p.flags, STOM_FLAG_BAD_VALUE);
        } else {
            const bool few = top_k > 0 && top_k <= (int)kGather;
            if (few) {
                r.template tally<0, false>();
                if ((uint32_t)top_k < r.sums[0].total) r.rank_first((uint32_t)top_k - 1);
            }
            if (!r.all_ranked) r.template tally<0, true>();
        }
        // One warp decides after each answer; 32 would only wait for one another's binary64 operations.
        uint32_t count = r.sums[0].total;
        double mass = (double)r.sums[0].all * r.unit;
        auto settled = [&]() {
            __syncthreads();
            count = sh.count;
            mass = sh.mass;
        };
        if (top_k > 0 && (uint32_t)top_k < count) {
            const Place a = r.ask(Query{BY_RANK, (uint32_t)top_k - 1, 0, 0.0});
            count = top_k;
            mass = a.mass_before + (double)(top_k - a.before) * a.weight;
        }
        if (top_p < 1.f) {
            const double aim = (double)fmaxf(top_p, 0.f) * mass;
            const Place a = r.ask(Query{BY_MASS, 0, 0, aim});
            if (warp == 0) {
                // the fewest of the equal ones with which the mass is reached
                uint32_t c = 1;
                if (a.weight > 0.0) {
                    const double d = ceil((aim - a.mass_before) / a.weight);
                    c = d < 1.0 ? 1u : d > (double)a.count ? a.count : (uint32_t)d;
                    if (c > 1 && a.mass_before + (c - 1) * a.weight >= aim) --c;
                    else if (c < a.count && a.mass_before + c * a.weight < aim) ++c;
                }
                const bool less = a.before + c < count;
                if (lane == 0) {
                    sh.count = less ? a.before + c : count;
                    sh.mass = less ? a.mass_before + c * a.weight : mass;
                }
            }
            settled();
        }
        // min_p, and weights that vanish: the lowest key that is still kept, by a 33-way search
        uint32_t floor_key = K::kLowest;
        if constexpr (kHalf) floor_key = max(floor_key, (kRanges - r.sums[0].lowest) * 16);
        else floor_key = __reduce_min_sync(~0u, lane < (int)blocks ? sh.all_min[lane] : ~0u) + 1;
        const double least = fmin((double)min_p, 1.0);
        auto stays = [&](uint32_t k) {
            const double w = r.weight(K::value(k));
            return w > 0.0 && w >= least;
        };
        if (warp == 0) {
            uint32_t low = floor_key, high = best;             // low does not stay, high does
            if (stays(floor_key)) high = low;
            while (high - low > 1 && high != low) {
                const uint32_t step = (high - low + 31) / 32;
                const uint64_t k = (uint64_t)low + (uint64_t)step * (lane + 1);
                const uint32_t yes = __ballot_sync(~0u, k >= high || stays((uint32_t)k));
                const int j = __ffs(yes) - 1;                  // first probe that stays (the last one is at high or beyond)
                const uint64_t up = (uint64_t)low + (uint64_t)step * (j + 1);
                low = low + step * j;
                high = up < high ? (uint32_t)up : high;
            }
            if (lane == 0) sh.nth = high;
        }
        __syncthreads();
        const uint32_t last_key = sh.nth;
        if (last_key != floor_key) {
            const Place a = r.ask(Query{BY_KEY, 0, last_key, 0.0});
            if (a.before + a.count < count) {
                count = a.before + a.count;
                mass = a.mass_before + a.count * a.weight;
            }
        }
        if (count < 1) count = 1;
        const double aim = (double)u * mass;
        Place a = r.ask(Query{PAST_MASS, 0, 0, aim});
        if (warp == 0) {
            uint32_t q = 0;
            if (a.weight > 0.0) {
                const double d = floor((aim - a.mass_before) / a.weight);
                q = d < 0.0 ? 0u : d > (double)(a.count - 1) ? a.count - 1 : (uint32_t)d;
                if (q > 0 && a.mass_before + q * a.weight > aim) --q;
                else if (q + 1 < a.count && a.mass_before + (q + 1) * a.weight <= aim) ++q;
            }
            if (lane == 0) sh.nth = q;
        }
        __syncthreads();
        nth = sh.nth;
        if (a.before + nth >= count) {                         // rounding has led behind the last one kept
            a = r.ask(Query{BY_RANK, count - 1, 0, 0.0});
            nth = count - 1 - a.before;
        }
        key = a.key;
        kept = count;
        weight = a.weight;
        total = mass;
    }

    // ---- the index: the nth of the logits with this key, slice after slice
    constexpr uint32_t kRoom = 1024;
    uint32_t *found = reinterpret_cast<uint32_t *>(kHalf ? (uint8_t *)r.list : (uint8_t *)r.raw);
    uint32_t own;
    if constexpr (kHalf) {
        const uint32_t b = K::bits(key);
        own = (r.raw[b >> 1] >> (16 * (b & 1))) & 0xffffu;
        if (key == K::kZero) own += r.raw[0x8000u >> 1] & 0xffffu;
    } else {
        __syncthreads();
        own = r.collect(key, found, kRoom);
    }
    if (tid < blocks) st_cluster_u(&sh.all_own[rank], tid, own);
    cluster_sync();   // from here on nobody looks into another block's memory: the others may leave
    uint32_t ahead = 0;
    for (uint32_t k = 0; k < rank; ++k) ahead += sh.all_own[k];
    if (nth < ahead || nth >= ahead + own) return;
    const uint32_t want = nth - ahead;
    auto answer = [&](int index) {
        p.token[row] = begin + index;
        if (p.kept) p.kept[row] = (int32_t)kept;
        if (p.logprob) p.logprob[row] = (float)(log(weight) - log(total));
    };
    if (own <= kRoom) {
        if constexpr (kHalf) r.collect(key, found, kRoom);
        // the one that `want` others stand before
        for (uint32_t i = tid; i < own; i += kThreads) {
            uint32_t before = 0;
            for (uint32_t j = 0; j < own; ++j) before += found[j] < found[i];
            if (before == want) answer((int)found[i]);
        }
        return;
    }
    // many: every warp counts in a run of its own, then the run that holds it is walked again
    bool ignore = false;
    const int run = (r.n + kThreads / 32 - 1) / (kThreads / 32), i0 = warp * run, i1 = min(r.n, i0 + run);
    uint32_t c = 0;
    for (int i = i0 + lane; i < i1; i += 32) c += K::of(r.bits_at(i), ignore) == key;
    c = __reduce_add_sync(~0u, c);
    __syncthreads();
    if (lane == 0) sh.warp_count[warp] = c;
    __syncthreads();
    uint32_t before = 0;
    for (int k = 0; k < warp; ++k) before += sh.warp_count[k];
    if (want >= before && want < before + c) {
        uint32_t left = want - before;
        for (int i = i0; i < i1; i += 32) {
            const uint32_t hit = __ballot_sync(~0u, i + lane < i1 && K::of(r.bits_at(min(i + lane, i1 - 1)), ignore) == key);
            const uint32_t m = __popc(hit);
            if (left < m) {
                if (lane == 0) answer(i + (int)__fns(hit, 0, (int)left + 1));
                break;
            }
            left -= m;
        }
    }
}

template <typename T>
cudaLaunchConfig_t config(int rows, int cluster, cudaStream_t stream, cudaLaunchAttribute (&at)[2]) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(rows * cluster);
    lc.blockDim = dim3(Plan<T>::kThreads);
    lc.dynamicSmemBytes = Plan<T>::smem(cluster);
    lc.stream = stream;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 2;
    return lc;
}

// How many clusters of each size the current device runs at once (asked of the runtime once per device and type)
template <typename T>
cudaError_t resident(int (&most)[kMaxCluster + 1]) {
    static std::atomic<int> known[64][kMaxCluster + 1];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !known[dev][0].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(sample_kernel<T, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<T>::smem(1));
        if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<T, 1>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if constexpr (!Plan<T>::kHalf)
            if (e == cudaSuccess)
                e = cudaFuncSetAttribute(sample_kernel<T, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<T>::smem(1));
        for (int c = 1; c <= kMaxCluster && e == cudaSuccess; ++c) {
            cudaLaunchAttribute at[2];
            const cudaLaunchConfig_t lc = config<T>(1, c, nullptr, at);
            most[c] = 0;
            e = cudaOccupancyMaxActiveClusters(&most[c], sample_kernel<T, 1>, &lc);
            if (e != cudaSuccess && c > 8) {   // a device that runs none of this size
                cudaGetLastError();
                e = cudaSuccess;
                most[c] = 0;
            }
            if (dev < 64) known[dev][c].store(most[c], std::memory_order_relaxed);
        }
        if (e == cudaSuccess && dev < 64) known[dev][0].store(1, std::memory_order_release);
        return e;
    }
    for (int c = 1; c <= kMaxCluster; ++c) most[c] = known[dev][c].load(std::memory_order_relaxed);
    return cudaSuccess;
}

template <typename T>
int32_t launch(SampleParams &p, int rows, cudaStream_t stream) {
    int most[kMaxCluster + 1];
    cudaError_t e = resident<T>(most);
    // Blocks per row: as few as hold the row (a 16-bit counter counts to 65 535), but more as long as all rows run at
    // once and a slice stays long enough to be worth the blocks' exchange (128 000 logits in one row: 21 us with 16 blocks
    // of 8 000, 26 us with 8; 64 rows: 30 us with 2 blocks each, 37 with 3, which take two rounds).
    int cluster = (p.n + 65527) / 65528;
    if (e == cudaSuccess)
        for (int c = cluster + 1; c <= kMaxCluster && p.n / (c - 1) > 8192 && rows <= most[c]; ++c) cluster = c;
    if ((int64_t)rows * cluster > INT32_MAX) return STOM_ERR_SHAPE;
    p.slice = ((p.n + cluster - 1) / cluster + 7) & ~7;
    // a slice's sum of limbs takes 32 bits; three limbs hold a weight: 48 bits of 2^47 units at most (n > 2^14), 54 of 2^51
    p.limb = 32;
    while ((1ll << (32 - p.limb)) < p.slice) --p.limb;
    cudaLaunchAttribute at[2];
    const cudaLaunchConfig_t lc = config<T>(rows, cluster, stream, at);
    if (e == cudaSuccess) {
        if constexpr (Plan<T>::kHalf) {
            e = cudaLaunchKernelEx(&lc, sample_kernel<T, 1>, p);
        } else {
            e = rows <= most[cluster] ? cudaLaunchKernelEx(&lc, sample_kernel<T, 1>, p) : cudaLaunchKernelEx(&lc, sample_kernel<T, 2>, p);
        }
    }
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int32_t stom_sample_tokens(const void *logits, int32_t dtype, int32_t rows, int32_t n, int64_t row_stride,
                                      const float *temperature, const int32_t *top_k, const float *top_p,
                                      const float *min_p, const float *u, int32_t *token, int32_t *kept, float *logprob,
                                      uint32_t *dev_flags, void *stream) {
    if (rows < 0 || n < 1) return STOM_ERR_INVALID_ARG;
    if (dtype != STOM_BF16 && dtype != STOM_FP16 && dtype != STOM_FP32) return STOM_ERR_UNSUPPORTED;
    if (n > STOM_SAMPLE_MAX_N) return STOM_ERR_SHAPE;
    if (rows == 0) return STOM_OK;
    if (!logits || !token || (!u && !temperature) || row_stride < 0 || (rows > 1 && row_stride < n)) return STOM_ERR_INVALID_ARG;
    const uintptr_t all = reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) |
                          reinterpret_cast<uintptr_t>(top_p) | reinterpret_cast<uintptr_t>(min_p) |
                          reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(token) |
                          reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(logprob);
    if (all & 3u || reinterpret_cast<uintptr_t>(logits) % elem_bytes(dtype)) return STOM_ERR_ALIGNMENT;
    SampleParams p = {};
    int bits = 0;
    while ((1 << bits) < n) ++bits;
    p.unit_bits = 62 - bits < 51 ? 62 - bits : 51;    // 2^bits weights of 1 are 2^62 units; binary64 holds 2^52 of them
    p.most_lift = bits > 9 ? bits - 9 : 0;            // n halves of 2^-most_lift units are 2^8 units (ranges: 2^10 at most)
    p.per_nat = (Plan<float>::kRanges - 1) / ((p.unit_bits + 1) * 0.69314718f);
    p.log2_per_range = (uint32_t)(((p.unit_bits + 1) << 16) / (Plan<float>::kRanges - 1));
    p.logits = static_cast<const char *>(logits);
    p.row_stride = row_stride;
    p.n = n;
    p.temperature = temperature;
    p.top_k = top_k;
    p.top_p = top_p;
    p.min_p = min_p;
    p.u = u;
    p.token = token;
    p.kept = kept;
    p.logprob = logprob;
    p.flags = dev_flags;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == STOM_BF16) return launch<__nv_bfloat16>(p, rows, s);
    if (dtype == STOM_FP16) return launch<__half>(p, rows, s);
    return launch<float>(p, rows, s);
}
