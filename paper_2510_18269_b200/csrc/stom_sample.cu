// The choice of the next token from a row of logits (stom_sample_tokens): temperature, top-k, top-p, min-p and a draw
// with a given random number, in the order "largest logit first, of equal ones the lowest index first".
//
// Nothing is sorted.  The tokens kept are a prefix of that order, and so is everything before the token drawn; each of
// the settings asks for ONE place in the order, given by a rank (top-k), by a mass (top-p, the draw) or by a logit
// (min-p).  A place is found through counts and masses of ranges of KEYS (the logit's bits made to order as unsigned
// numbers), from 4 096 ranges down to a single key; within one key all weights are equal and the rest is a division.
//
// A row belongs to a cluster of up to 8 blocks, each with a slice of it; tables are added up over distributed shared
// memory, every block for its share of the ranges, and the blocks agree on a place through one cluster barrier.
//   16-bit logits: one count per possible key (65 536 16-bit counters, hence slices below 65 536) in shared memory.  One
//     shared-memory atomic per logit is all the work that grows with the row; the exponential is taken per DISTINCT
//     logit, and a mass is count times weight.
//   binary32 logits: the row is read again (from L2) for every level, 12 + 12 + 8 bits of the key: counts, and masses as
//     sums of integers, weight * 2^44 in three 16-bit limbs, so that the order of the atomics leaves no trace.
// With 100 000 tokens left to draw from, binary32 sums would move a border between two tokens by more than some tokens'
// whole weight.  The masses of ranges are whole multiples of 2^-44 (of the largest weight) in 64 bits: their sums are
// exact and never fall, so that exactly one range holds a place and all blocks of a cluster see the same one.  Within the
// last few keys weights and sums are binary64.
#include "stom_kv.cuh"
#include "stom_sample.h"

namespace stom {

namespace {

constexpr int kRanges = 4096;   // ranges of the first two levels
constexpr int kMaxCluster = 8;

struct SampleParams {
    const char *logits;
    int64_t row_stride;
    int32_t n, slice;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *logprob;
    uint32_t *flags;
};

// ---- keys: unsigned numbers in the order of the logits.  0 stands for what is never drawn (NaN, -inf); -0 is +0.
template <typename T>
struct Keys;
template <typename T>
__device__ __forceinline__ uint32_t key16(uint32_t b, uint32_t inf, bool &nan) {
    const uint32_t mag = b & 0x7fffu;
    nan |= mag > inf;
    const uint32_t k = b & 0x8000u ? 0x8000u - mag : 0x8000u + mag;   // -0 and +0: 0x8000
    return mag > inf || b == (0x8000u | inf) ? 0u : k;
}
__device__ __forceinline__ uint32_t bits16(uint32_t k) { return k >= 0x8000u ? k - 0x8000u : 0x8000u | (0x8000u - k); }
template <>
struct Keys<__nv_bfloat16> {
    static constexpr int kBits = 16;
    static constexpr uint32_t kLowest = 0x8000u - 0x7f7fu;   // of a finite logit
    static __device__ __forceinline__ uint32_t of(uint32_t b, bool &nan) { return key16<__nv_bfloat16>(b, 0x7f80u, nan); }
    static __device__ __forceinline__ double value(uint32_t k) { return (double)__uint_as_float(bits16(k) << 16); }
};
template <>
struct Keys<__half> {
    static constexpr int kBits = 16;
    static constexpr uint32_t kLowest = 0x8000u - 0x7bffu;
    static __device__ __forceinline__ uint32_t of(uint32_t b, bool &nan) { return key16<__half>(b, 0x7c00u, nan); }
    static __device__ __forceinline__ double value(uint32_t k) {
        return (double)__half2float(__ushort_as_half((unsigned short)bits16(k)));
    }
};
template <>
struct Keys<float> {
    static constexpr int kBits = 32;
    static constexpr uint32_t kLowest = 0x80000000u - 0x7f7fffffu;
    static __device__ __forceinline__ uint32_t of(uint32_t b, bool &nan) {
        const uint32_t mag = b & 0x7fffffffu;
        nan |= mag > 0x7f800000u;
        const uint32_t k = b & 0x80000000u ? 0x80000000u - mag : 0x80000000u + mag;
        return mag > 0x7f800000u || b == 0xff800000u ? 0u : k;
    }
    static __device__ __forceinline__ double value(uint32_t k) {
        return (double)__uint_as_float(k >= 0x80000000u ? k - 0x80000000u : 0x80000000u | (0x80000000u - k));
    }
};

template <typename T>
struct Plan {
    static constexpr int kThreads = sizeof(T) == 2 ? 1024 : 512;
    static constexpr int kRaw = sizeof(T) == 2 ? 65536 * 2 : kRanges * 16;   // counters in shared memory
    static int smem(int cluster) { return kRaw + (sizeof(T) == 2 ? 1 : 2) * (kRanges / cluster) * 12; }
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
__device__ __forceinline__ uint64_t ld_cluster_u64(const uint64_t *mine, uint32_t rank) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_addr(mine, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_u(uint32_t *mine, uint32_t rank, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(mine, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_u64(uint64_t *mine, uint32_t rank, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(mine, rank)), "l"(v) : "memory");
}
constexpr double kUnit = 0x1p-44, kUnits = 0x1p44;   // masses of ranges: whole multiples of kUnit

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

struct Shared {
    uint32_t max_key[32];
    uint32_t warp_count[32];
    uint64_t warp_mass[32];      // sums of units (ranges) or the bits of binary64 sums (keys)
    uint32_t nan;
    uint32_t count;              // of this block's ranges
    uint64_t mass;
    uint32_t lowest;             // last range of this block that is not empty, + 1
    uint32_t ans_range[8], ans_before[8];   // answers to queries, a slot each in turn
    uint64_t ans_mass[8];
    uint32_t first_hit, last_in; // thread of the key asked for
    uint32_t leaf[256];
    uint32_t row_max;
    Place place;
};

// A range of keys with all its tables, as one block of a cluster sees it
template <typename T>
struct Row {
    using K = Keys<T>;
    using P = Plan<T>;
    static constexpr int kThreads = P::kThreads;
    const SampleParams &p;
    Shared &sh;
    uint32_t *raw;               // counters
    uint32_t *cnt[2];            // of this block's share of the ranges, highest keys first: counts and masses, per level
    uint64_t *mass[2];
    const T *x;                  // this block's slice
    int n, begin;
    uint32_t rank, blocks, share;
    double top, t;
    int tid;
    uint32_t slot = 0;
    // running sums of one level: before this thread's ranges, and with them
    struct Sums {
        uint32_t c0, c1, total;
        uint64_t m0, m1, all;
        uint32_t lowest;
    } sums[2];
    int64_t have = -1;           // range whose second level is in cnt[1], mass[1] (binary32)

    // Zero below e^-700: close to where binary64 ends, the last steps of an exponential would decide what is kept.
    __device__ __forceinline__ double weight(double v) const {
        const double y = v == top ? 0.0 : (v - top) / t;
        return y < -700.0 ? 0.0 : exp(y);
    }

    // f(index in the slice, bits) over the slice, 16 bytes at a time
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        constexpr int kV = 16 / sizeof(T), kBatch = 4;
        const int off = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
        const int head = min(n, off ? kV - off : 0), vecs = (n - head) / kV;
        const uint4 *v = reinterpret_cast<const uint4 *>(x + head);
        auto part = [&](const uint4 &q, int at) {
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 2) {
                    f(at + 2 * e, w[e] & 0xffffu);
                    f(at + 2 * e + 1, w[e] >> 16);
                } else {
                    f(at + e, w[e]);
                }
            }
        };
        int i = tid;
        for (; i + (kBatch - 1) * kThreads < vecs; i += kBatch * kThreads) {
            uint4 q[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) q[j] = v[i + j * kThreads];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) part(q[j], head + (i + j * kThreads) * kV);
        }
        for (; i < vecs; i += kThreads) part(v[i], head + i * kV);
        for (int j = tid; j < head; j += kThreads) f(j, bits_at(j));
        for (int j = head + vecs * kV + tid; j < n; j += kThreads) f(j, bits_at(j));
    }
    __device__ __forceinline__ uint32_t bits_at(int i) const {
        if constexpr (sizeof(T) == 2) return reinterpret_cast<const unsigned short *>(x)[i];
        else return reinterpret_cast<const uint32_t *>(x)[i];
    }

    __device__ __forceinline__ void zero_raw() {
        for (int i = tid; i < P::kRaw / 16; i += kThreads) reinterpret_cast<uint4 *>(raw)[i] = make_uint4(0, 0, 0, 0);
    }

    __device__ static __forceinline__ uint64_t as_bits(uint64_t m) { return m; }
    __device__ static __forceinline__ uint64_t as_bits(double m) { return (uint64_t)__double_as_longlong(m); }
    __device__ static __forceinline__ void of_bits(uint64_t b, uint64_t &m) { m = b; }
    __device__ static __forceinline__ void of_bits(uint64_t b, double &m) { m = __longlong_as_double((long long)b); }

    // Sums over the block's threads: those of the threads ahead (c0, m0), and with the thread's own (c1, m1)
    template <typename M>
    __device__ __forceinline__ void block_sums(uint32_t c, M m, uint32_t &c0, uint32_t &c1, M &m0, M &m1) {
        const uint32_t c_own = c;
        const M m_own = m;
        const int lane = tid & 31, warp = tid >> 5;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t vc = __shfl_up_sync(~0u, c, o);
            const M vm = __shfl_up_sync(~0u, m, o);
            if (lane >= o) {
                c += vc;
                m += vm;
            }
        }
        __syncthreads();
        if (lane == 31) {
            sh.warp_count[warp] = c;
            sh.warp_mass[warp] = as_bits(m);
        }
        __syncthreads();
        uint32_t wc = lane < kThreads / 32 ? sh.warp_count[lane] : 0u;
        M wm = 0;
        if (lane < kThreads / 32) of_bits(sh.warp_mass[lane], wm);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t vc = __shfl_up_sync(~0u, wc, o);
            const M vm = __shfl_up_sync(~0u, wm, o);
            if (lane >= o) {
                wc += vc;
                wm += vm;
            }
        }
        const uint32_t bc = __shfl_sync(~0u, wc, (warp + 31) & 31);
        const M bm = __shfl_sync(~0u, wm, (warp + 31) & 31);
        c1 = c + (warp ? bc : 0u);
        m1 = m + (warp ? bm : M(0));
        c0 = c1 - c_own;
        m0 = m1 - m_own;
    }

    // Sums of a level over the cluster, from cnt[level] and mass[level]
    __device__ __forceinline__ void sum_up(int level) {
        const int per = max(1u, share / kThreads), first = tid * per;
        uint32_t c = 0, low = 0;
        uint64_t m = 0;
        if (first < (int)share)
            for (int j = 0; j < per; ++j) {
                c += cnt[level][first + j];
                m += mass[level][first + j];
                if (cnt[level][first + j]) low = first + j + 1;
            }
        Sums &s = sums[level];
        block_sums(c, m, s.c0, s.c1, s.m0, s.m1);
        if (tid == 0) sh.lowest = 0;
        __syncthreads();
        if (low) atomicMax(&sh.lowest, low);
        if (tid == kThreads - 1) {
            sh.count = s.c1;
            sh.mass = s.m1;
        }
        cluster_sync();
        uint32_t before = 0, total = 0, lowest = 0;
        uint64_t mb = 0, all = 0;
        for (uint32_t r = 0; r < blocks; ++r) {
            if (r == rank) {
                before = total;
                mb = all;
            }
            total += ld_cluster_u(&sh.count, r);
            all += ld_cluster_u64(&sh.mass, r);
            const uint32_t l = ld_cluster_u(&sh.lowest, r);
            if (l) lowest = r * share + l;
        }
        s.c0 += before;
        s.c1 += before;
        s.m0 += mb;
        s.m1 += mb;
        s.total = total;
        s.all = all;
        s.lowest = lowest;
    }

    // The range that holds the place asked for, with what stands before it; agreed on by all blocks
    __device__ __forceinline__ void find(int level, const Query &q, uint32_t &range, uint32_t &before, uint64_t &mass_before,
                                         uint32_t base, uint64_t mass_base) {
        const Sums &s = sums[level];
        const int per = max(1u, share / kThreads), first = tid * per;
        const uint32_t at = slot++ & 7u;
        auto reached = [&](uint32_t c, uint64_t m) {   // never true and then false along the order
            if (c == 0) return false;
            if (c == s.total) return true;
            if (q.kind == BY_RANK) return base + c > q.rank;
            const double upto = (double)(mass_base + m) * kUnit;
            return q.kind == BY_MASS ? upto >= q.mass : upto > q.mass;
        };
        bool mine = false;
        if (q.kind == BY_KEY) {
            const uint32_t r = range_of(level, q.key);
            mine = first < (int)share && r >= rank * share + first && r < rank * share + first + per;
        } else {
            mine = first < (int)share && s.c1 != s.c0 && reached(s.c1, s.m1) && !reached(s.c0, s.m0);
        }
        if (mine) {
            uint32_t c = s.c0, hit_c = s.c0, hit = first;
            uint64_t m = s.m0, hit_m = s.m0;
            for (int j = first; j < first + per; ++j) {
                if (q.kind == BY_KEY) {
                    if (rank * share + j == range_of(level, q.key)) {
                        hit = j, hit_c = c, hit_m = m;
                        break;
                    }
                } else if (cnt[level][j]) {
                    hit = j, hit_c = c, hit_m = m;
                    if (reached(c + cnt[level][j], m + mass[level][j])) break;
                }
                c += cnt[level][j];
                m += mass[level][j];
            }
            for (uint32_t r = 0; r < blocks; ++r) {
                st_cluster_u(&sh.ans_range[at], r, rank * share + hit);
                st_cluster_u(&sh.ans_before[at], r, base + hit_c);
                st_cluster_u64(&sh.ans_mass[at], r, mass_base + hit_m);
            }
        }
        cluster_sync();
        range = min(sh.ans_range[at], (uint32_t)kRanges - 1);
        before = sh.ans_before[at];
        mass_before = sh.ans_mass[at];
    }
    __device__ __forceinline__ uint32_t range_of(int level, uint32_t key) const {
        if constexpr (K::kBits == 16) return kRanges - 1 - (key >> 4);
        else return kRanges - 1 - (level == 0 ? key >> 20 : (key >> 8) & (kRanges - 1));
    }

    // Place among `keys` single keys, highest first: thread j has count c of key `key` (threads beyond: 0)
    __device__ __forceinline__ void settle(const Query &q, uint32_t key, uint32_t c, uint32_t base, double mass_base) {
        const double w = c ? weight(K::value(key)) : 0.0;
        if (tid == 0) {
            sh.place = Place{0, base, 0, mass_base, 0.0};
            sh.first_hit = ~0u;
            sh.last_in = 0;
        }
        uint32_t c0, c1;
        double m0, m1;
        block_sums(c, c * w, c0, c1, m0, m1);
        auto reached = [&](uint32_t cc, double mm) {
            if (q.kind == BY_RANK) return base + cc > q.rank;
            if (q.kind == BY_MASS) return mass_base + mm >= q.mass;
            if (q.kind == PAST_MASS) return mass_base + mm > q.mass;
            return false;   // BY_KEY: all that stands above
        };
        // by key: up to the last of the keys that are not below it; otherwise the first that reaches, or the last at all
        const bool in = c && (q.kind != BY_KEY || key >= q.key);
        if (in && q.kind != BY_KEY && reached(c1, m1)) atomicMin(&sh.first_hit, (uint32_t)tid);
        if (in) atomicMax(&sh.last_in, (uint32_t)tid);
        __syncthreads();
        const uint32_t pick = sh.first_hit != ~0u ? sh.first_hit : sh.last_in;
        if (in && (uint32_t)tid == pick) sh.place = Place{key, base + c0, c, mass_base + m0, w};
        __syncthreads();
    }

    __device__ __forceinline__ Place ask(const Query &q) {
        uint32_t range, before;
        uint64_t mb;
        find(0, q, range, before, mb, 0, 0);
        if constexpr (K::kBits == 16) {
            uint32_t key = 0, c = 0;
            if (tid < 16) {
                key = (kRanges - 1 - range) * 16 + 15 - tid;
                for (uint32_t r = 0; r < blocks; ++r)
                    c += (ld_cluster_u(raw + (key >> 1), r) >> (16 * (key & 1))) & 0xffffu;
            }
            settle(q, key, c, before, (double)mb * kUnit);
        } else {
            const uint32_t high = kRanges - 1 - range;
            if (have != (int64_t)high) {
                tally(1, high);
                have = high;
            }
            uint32_t range2;
            const uint32_t b0 = before;
            const uint64_t m0 = mb;
            find(1, q, range2, before, mb, b0, m0);
            const uint32_t mid = high << 12 | (kRanges - 1 - range2);
            __syncthreads();
            for (int i = tid; i < 256; i += kThreads) sh.leaf[i] = 0;
            __syncthreads();
            bool nan = false;
            each([&](int, uint32_t b) {
                const uint32_t k = K::of(b, nan);
                if (k && k >> 8 == mid) atomicAdd(&sh.leaf[k & 255u], 1u);
            });
            cluster_sync();
            uint32_t key = 0, c = 0;
            if (tid < 256) {
                key = mid << 8 | (255 - tid);
                for (uint32_t r = 0; r < blocks; ++r) c += ld_cluster_u(&sh.leaf[255 - tid], r);
            }
            settle(q, key, c, before, (double)mb * kUnit);
        }
        return sh.place;
    }

    // binary32: counts and masses of a level (of the keys that begin with `high`), summed over the cluster
    __device__ __forceinline__ void tally(int level, uint32_t high) {
        zero_raw();
        __syncthreads();
        bool nan = false;
        const double scale = 1.4426950408889634 / t;
        each([&](int, uint32_t b) {
            const uint32_t k = K::of(b, nan);
            if (!k || (level && k >> 20 != high)) return;
            uint32_t *r = raw + 4 * (level ? (k >> 8) & (kRanges - 1) : k >> 20);
            atomicAdd(r, 1u);
            const double v = K::value(k);
            const double y = v == top ? 0.0 : (v - top) * scale;
            if (y > -46.0) {
                const unsigned long long w = (unsigned long long)__double2ll_rn(exp2(y) * kUnits);
                atomicAdd(r + 1, (uint32_t)w & 0xffffu);
                atomicAdd(r + 2, (uint32_t)(w >> 16) & 0xffffu);
                atomicAdd(r + 3, (uint32_t)(w >> 32));
            }
        });
        cluster_sync();
        for (uint32_t j = tid; j < share; j += kThreads) {
            const uint32_t *r = raw + 4 * (kRanges - 1 - (rank * share + j));
            uint32_t c = 0;
            unsigned long long w = 0;
            for (uint32_t k = 0; k < blocks; ++k) {
                const uint4 v = ld_cluster_u4(r, k);
                c += v.x;
                w += (unsigned long long)v.y + ((unsigned long long)v.z << 16) + ((unsigned long long)v.w << 32);
            }
            cnt[level][j] = c;
            mass[level][j] = w;
        }
        __syncthreads();
        sum_up(level);
    }
    // 16 bits: the first level from the counts of single keys
    __device__ __forceinline__ void tally16() {
        for (uint32_t j = tid; j < share; j += kThreads) {
            const uint32_t first = (kRanges - 1 - (rank * share + j)) * 16;
            uint32_t c[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) c[e] = 0;
            for (uint32_t r = 0; r < blocks; ++r) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 v = ld_cluster_u4(raw + (first >> 1) + 4 * h, r);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        c[8 * h + 2 * e] += w[e] & 0xffffu;
                        c[8 * h + 2 * e + 1] += w[e] >> 16;
                    }
                }
            }
            uint32_t n_all = 0;
            uint64_t m = 0;
#pragma unroll 1
            for (int e = 15; e >= 0; --e) {
                uint32_t ce = 0;
#pragma unroll
                for (int f = 0; f < 16; ++f) ce = f == e ? c[f] : ce;
                if (ce) {
                    n_all += ce;
                    m += __double2ull_rn(ce * weight(K::value(first + e)) * kUnits);
                }
            }
            cnt[0][j] = n_all;
            mass[0][j] = m;
        }
        __syncthreads();
        sum_up(0);
    }
};

template <typename T>
__global__ void __launch_bounds__(Plan<T>::kThreads, 1) sample_kernel(const __grid_constant__ SampleParams p) {
    using K = Keys<T>;
    using P = Plan<T>;
    constexpr int kThreads = P::kThreads;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t blocks = cluster_size(), rank = cluster_rank();
    const int64_t row = blockIdx.x / blocks;

    Row<T> r{p, sh};
    r.raw = reinterpret_cast<uint32_t *>(smem);
    r.share = kRanges / blocks;
    r.mass[0] = reinterpret_cast<uint64_t *>(smem + P::kRaw);
    r.mass[1] = r.mass[0] + r.share;
    r.cnt[0] = reinterpret_cast<uint32_t *>(r.mass[0] + (sizeof(T) == 2 ? 1 : 2) * r.share);
    r.cnt[1] = r.cnt[0] + r.share;
    r.tid = tid;
    r.rank = rank;
    r.blocks = blocks;
    r.begin = min((int64_t)rank * p.slice, (int64_t)p.n);
    r.n = min(p.slice, p.n - r.begin);
    r.x = reinterpret_cast<const T *>(p.logits) + row * p.row_stride + r.begin;

    if (K::kBits == 16) r.zero_raw();
    if (tid == 0) sh.nan = 0;
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
    temp = fminf(temp, 3.0e38f);
    const bool cold = temp <= 0.f;

    // ---- the first pass: the largest key, and for 16-bit logits the count of every key
    uint32_t best = 0;
    bool nan = false;
    r.each([&](int, uint32_t b) {
        const uint32_t k = K::of(b, nan);
        best = max(best, k);
        if constexpr (K::kBits == 16)
            if (k) atomicAdd(r.raw + (k >> 1), k & 1u ? 0x10000u : 1u);
    });
    best = __reduce_max_sync(~0u, best);
    if (nan) sh.nan = 1;
    if (lane == 0) sh.max_key[warp] = best;
    __syncthreads();
    if (warp == 0) {
        uint32_t b = lane < kThreads / 32 ? sh.max_key[lane] : 0u;
        b = __reduce_max_sync(~0u, b);
        if (lane == 0) sh.row_max = b;
    }
    if (tid == 0 && p.flags && (sh.nan || (bad && rank == 0))) atomicOr(p.flags, STOM_FLAG_BAD_VALUE);
    cluster_sync();
    best = 0;
    for (uint32_t k = 0; k < blocks; ++k) best = max(best, ld_cluster_u(&sh.row_max, k));
    if (best == 0) {
        if (rank == 0 && tid == 0) {
            p.token[row] = -1;
            if (p.kept) p.kept[row] = 0;
            if (p.logprob) p.logprob[row] = -INFINITY;
        }
        cluster_sync();   // nobody leaves while its shared memory may still be read
        return;
    }
    r.top = K::value(best);
    r.t = temp;

    // ---- the place drawn: key, and how many equal ones come before it
    uint32_t key = best, nth = 0, kept = 1;
    double prob = 1.0;
    if (!cold) {
        if constexpr (K::kBits == 16) r.tally16();
        else r.tally(0, 0);
        uint32_t count = r.sums[0].total;
        double mass = (double)r.sums[0].all * kUnit;
        if (top_k > 0 && (uint32_t)top_k < count) {
            const Place a = r.ask(Query{BY_RANK, (uint32_t)top_k - 1, 0, 0.0});
            count = top_k;
            mass = a.mass_before + (double)(top_k - a.before) * a.weight;
        }
        if (top_p < 1.f) {
            const double aim = (double)fmaxf(top_p, 0.f) * mass;
            const Place a = r.ask(Query{BY_MASS, 0, 0, aim});
            // the fewest of the equal ones with which the mass is reached
            uint32_t c = 1;
            if (a.weight > 0.0) {
                const double d = ceil((aim - a.mass_before) / a.weight);
                c = d < 1.0 ? 1u : d > (double)a.count ? a.count : (uint32_t)d;
                if (c > 1 && a.mass_before + (c - 1) * a.weight >= aim) --c;
                else if (c < a.count && a.mass_before + c * a.weight < aim) ++c;
            }
            if (a.before + c < count) {
                count = a.before + c;
                mass = a.mass_before + c * a.weight;
            }
        }
        // min_p, and weights that vanish: the lowest key that is still kept, by a 33-way search
        const uint32_t floor_key = K::kBits == 16 ? (kRanges - r.sums[0].lowest) * 16 : (kRanges - r.sums[0].lowest) << 20;
        const double least = fmin((double)min_p, 1.0);
        auto stays = [&](uint32_t k) {
            if (k < K::kLowest) return false;
            const double w = r.weight(K::value(k));
            return w > 0.0 && w >= least;
        };
        if (!stays(max(floor_key, K::kLowest))) {
            uint32_t low = 0, high = best;                 // low does not stay, high does
            while (high - low > 1) {
                const uint32_t step = (high - low + 31) / 32;
                const uint64_t k = (uint64_t)low + (uint64_t)step * (lane + 1);
                const uint32_t yes = __ballot_sync(~0u, k >= high || stays((uint32_t)k));
                const int j = __ffs(yes) - 1;              // first probe that stays (the last one is at high or beyond)
                const uint64_t up = (uint64_t)low + (uint64_t)step * (j + 1);
                low = low + step * j;
                high = up < high ? (uint32_t)up : high;
            }
            const Place a = r.ask(Query{BY_KEY, 0, high, 0.0});
            if (a.before + a.count < count) {
                count = a.before + a.count;
                mass = a.mass_before + a.count * a.weight;
            }
        }
        if (count < 1) count = 1;
        const double aim = (double)u * mass;
        Place a = r.ask(Query{PAST_MASS, 0, 0, aim});
        uint32_t q = 0;
        if (a.weight > 0.0) {
            const double d = floor((aim - a.mass_before) / a.weight);
            q = d < 0.0 ? 0u : d > (double)(a.count - 1) ? a.count - 1 : (uint32_t)d;
            if (q > 0 && a.mass_before + q * a.weight > aim) --q;
            else if (q + 1 < a.count && a.mass_before + (q + 1) * a.weight <= aim) ++q;
        }
        if (a.before + q >= count) {                       // rounding has led behind the last one kept
            a = r.ask(Query{BY_RANK, count - 1, 0, 0.0});
            q = count - 1 - a.before;
        }
        key = a.key;
        nth = q;
        kept = count;
        prob = a.weight / mass;
    }

    // ---- the index: the nth of the logits with this key, slice after slice
    if constexpr (K::kBits == 32) {
        uint32_t c = 0;
        bool ignore = false;
        r.each([&](int, uint32_t b) { c += K::of(b, ignore) == key; });
        c = __reduce_add_sync(~0u, c);
        __syncthreads();
        if (lane == 0) sh.warp_count[warp] = c;
        __syncthreads();
        if (tid == 0) {
            uint32_t s = 0;
            for (int k = 0; k < kThreads / 32; ++k) s += sh.warp_count[k];
            sh.count = s;
        }
        cluster_sync();
    }
    uint32_t ahead = 0, own = 0;
    for (uint32_t k = 0; k <= rank; ++k) {
        const uint32_t c = K::kBits == 16 ? (ld_cluster_u(r.raw + ((key & 0xffffu) >> 1), k) >> (16 * (key & 1))) & 0xffffu
                                          : ld_cluster_u(&sh.count, k);
        if (k < rank) ahead += c;
        else own = c;
    }
    if (nth >= ahead && nth < ahead + own) {
        // every warp counts in a run of its own, then the run that holds it is walked again
        const uint32_t want = nth - ahead;
        const int run = (r.n + kThreads / 32 - 1) / (kThreads / 32), i0 = warp * run, i1 = min(r.n, i0 + run);
        uint32_t c = 0;
        bool ignore = false;
        for (int i = i0 + lane; i < i1; i += 32) c += K::of(r.bits_at(i), ignore) == key;
        c = __reduce_add_sync(~0u, c);
        __syncthreads();
        if (lane == 0) sh.max_key[warp] = c;
        __syncthreads();
        uint32_t before = 0;
        for (int k = 0; k < warp; ++k) before += sh.max_key[k];
        if (want >= before && want < before + c) {
            uint32_t left = want - before;
            for (int i = i0; i < i1; i += 32) {
                const uint32_t hit = __ballot_sync(~0u, i + lane < i1 && K::of(r.bits_at(min(i + lane, i1 - 1)), ignore) == key);
                const uint32_t m = __popc(hit);
                if (left < m) {
                    if (lane == 0) {
                        p.token[row] = r.begin + i + (int)__fns(hit, 0, (int)left + 1);
                        if (p.kept) p.kept[row] = (int32_t)kept;
                        if (p.logprob) p.logprob[row] = (float)log(prob);
                    }
                    break;
                }
                left -= m;
            }
        }
    }
    cluster_sync();
}

template <typename T>
int32_t launch(const SampleParams &p, int rows, int cluster, cudaStream_t stream) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(rows * cluster);
    lc.blockDim = dim3(Plan<T>::kThreads);
    lc.dynamicSmemBytes = Plan<T>::smem(cluster);
    lc.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 2;
    cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<T>::smem(1));
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&lc, sample_kernel<T>, p);
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
    const int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    // Blocks per row: as few as hold the row (a 16-bit counter counts to 65 535), but more where the rows alone would
    // leave multiprocessors idle and a slice stays long enough to be worth the blocks' exchange.
    int cluster = 1;
    while (cluster < kMaxCluster &&
           ((n + cluster - 1) / cluster > 65528 || (n / cluster > 8192 && (int64_t)rows * cluster * 2 <= sms)))
        cluster *= 2;
    if ((int64_t)rows * cluster > INT32_MAX) return STOM_ERR_SHAPE;
    SampleParams p = {};
    p.logits = static_cast<const char *>(logits);
    p.row_stride = row_stride;
    p.n = n;
    p.slice = ((n + cluster - 1) / cluster + 7) & ~7;
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
    if (dtype == STOM_BF16) return launch<__nv_bfloat16>(p, rows, cluster, s);
    if (dtype == STOM_FP16) return launch<__half>(p, rows, cluster, s);
    return launch<float>(p, rows, cluster, s);
}
