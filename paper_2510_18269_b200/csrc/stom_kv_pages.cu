// The pages of a cache: reserve (with copies of shared pages), fork, free, compact.
//
// Everything is decided on the device from refs, table and len, so that a decode step needs no host: one block plans
// (prefix sums over rows and pages), then a grid copies pages of all layers from the list the plan left in the
// workspace.  fork and free touch counts and tables only, one block per row.  What bounds them: the plans are chains of
// a few dependent memory round trips, the copies are memory (each byte read and written once, 16 bytes per access).
// Counts change by integer atomics, whose order leaves no trace; every page id is checked before it is used.
//
// Measured (B200, copy rate 6 458 GB/s), 28 layers, 4 heads of 128, pages of 50: eight sequences forked eight times, the
// 64 candidates given room for a token (free, fork, reserve): 30.9 us, 20 of them for the 164 MB of copies; 20 sequences'
// pages moved together: 69 to 74 us for 384 MB (5.2 to 5.6 TB/s).
#include "stom_kv.cuh"

namespace stom {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPerThread = 8;    // pages a thread of a plan looks at per round

struct Move {
    int32_t src, dst, tokens, pad;
};

// Workspace: head[0] the number of moves; ids [n_pages]: free pages, or (compaction) where a page goes, -1: it stays;
// then the moves.
struct PagesParams {
    char *k, *v;
    int64_t stride_layer, stride_page, stride_token, stride_head;
    int32_t n_layers, n_pages, page_tokens, n_kv_heads, chunk_bits;   // 2^chunk_bits 16-byte chunks make a row
    FastDiv by_page, by_head;
    int32_t *table, *len, *refs;
    int32_t n_seqs, max_pages;
    int64_t table_stride;
    const int32_t *wish;          // want, parent or drop
    int32_t *table_out, *refs_out, *n_live;
    int32_t *head, *ids;
    Move *moves;
    uint32_t *flags;
};

__device__ __forceinline__ void raise(const PagesParams &p, uint32_t bit) {
    if (p.flags) atomicOr(p.flags, bit);
}
// Pages of n tokens, never more than a row has
__device__ __forceinline__ int held_of(const PagesParams &p, int n) {
    if (n <= 0) return 0;
    return min((int)div_by(p.by_page, (uint32_t)n - 1) + 1, p.max_pages);
}
__device__ __forceinline__ bool is_page(const PagesParams &p, int id) { return (uint32_t)id < (uint32_t)p.n_pages; }

// Exclusive sum over the block's threads, and the total
template <typename N>
__device__ __forceinline__ N block_sum_before(N x, N &total) {
    __shared__ N warp_sum[kPlanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    N upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N v = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += v;
    }
    __syncthreads();   // the sums of the call before have been read
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    N mine = warp_sum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N v = __shfl_up_sync(~0u, mine, o);
        if (lane >= o) mine += v;
    }
    total = __shfl_sync(~0u, mine, 31);
    const N before = __shfl_sync(~0u, mine, (warp + 31) & 31);
    return upto - x + (warp ? before : 0);
}

__global__ void __launch_bounds__(128) kv_free_kernel(const __grid_constant__ PagesParams p) {
    grid_dependency_wait();
    const int i = blockIdx.x;
    if (!p.wish[i]) return;
    const int held = held_of(p, p.len[i]);
    int32_t *row = p.table + i * p.table_stride;
    for (int j = threadIdx.x; j < p.max_pages; j += blockDim.x) {
        if (j < held) {
            const int id = row[j];
            if (is_page(p, id)) {
                if (atomicSub(p.refs + id, 1) <= 0) {   // was free already: a table that does not fit its counts
                    atomicAdd(p.refs + id, 1);
                    raise(p, STOM_FLAG_BAD_INDEX);
                }
            } else {
                raise(p, STOM_FLAG_BAD_INDEX);
            }
        }
        row[j] = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0) p.len[i] = 0;
}

__global__ void __launch_bounds__(128) kv_fork_kernel(const __grid_constant__ PagesParams p) {
    grid_dependency_wait();
    const int i = blockIdx.x, from = p.wish[i];
    if (from == -1) return;
    // a row that is not forked is written by no block, so the parent's row stands still
    if ((uint32_t)from >= (uint32_t)p.n_seqs || p.wish[from] != -1 || p.len[i] > 0) {
        if (threadIdx.x == 0) raise(p, STOM_FLAG_BAD_INDEX);
        return;
    }
    const int n = p.len[from], held = held_of(p, n);
    const int32_t *src = p.table + from * p.table_stride;
    int32_t *row = p.table + i * p.table_stride;
    for (int j = threadIdx.x; j < p.max_pages; j += blockDim.x) {
        int id = -1;
        if (j < held) {
            id = src[j];
            if (is_page(p, id)) atomicAdd(p.refs + id, 1);
            else raise(p, STOM_FLAG_BAD_INDEX);
        }
        row[j] = id;
    }
    __syncthreads();
    if (threadIdx.x == 0) p.len[i] = max(n, 0);
}

// One block.  Shared memory, a word per row each: the partly filled page that a growing row holds together with others,
// or -1; how many hold it; and the row's first place in the list of free pages, with two bits on top.
constexpr uint32_t kStays = 0x80000000u, kCopies = 0x40000000u, kPlace = 0x3fffffffu;

__global__ void __launch_bounds__(kPlanThreads) kv_reserve_plan_kernel(const __grid_constant__ PagesParams p) {
    extern __shared__ int32_t plan_smem[];
    int32_t *share = plan_smem, *holders = share + p.n_seqs;
    uint32_t *need = reinterpret_cast<uint32_t *>(holders + p.n_seqs);   // first pages, then places
    __shared__ int n_moves;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t room = (int64_t)p.max_pages * p.page_tokens;
    if (tid == 0) n_moves = 0;
    grid_dependency_wait();

    for (int i = tid; i < p.n_seqs; i += kPlanThreads) {
        const int n = max(p.len[i], 0);
        int want = p.wish[i];
        if (want > room) {
            raise(p, STOM_FLAG_BAD_INDEX);
            want = 0;
        }
        int page = -1, with = 0;
        uint32_t pages = kStays;
        if (want > n) {
            const int held = held_of(p, n);
            pages = held_of(p, want) - held;
            if (n - (int)(div_by(p.by_page, (uint32_t)n) * p.by_page.d)) {
                page = p.table[i * p.table_stride + held - 1];
                if (is_page(p, page)) with = p.refs[page];
                else raise(p, STOM_FLAG_BAD_INDEX);
            }
        }
        share[i] = with > 1 ? page : -1;
        holders[i] = with;
        need[i] = pages;
    }
    __syncthreads();
    // who copies: all but the last of the growing rows that share a page, and that one too if a row stays behind
    for (int i = warp; i < p.n_seqs; i += kPlanThreads / 32) {
        const int page = share[i];
        if (page < 0) continue;
        int same = 0, later = 0;
        for (int j = lane; j < p.n_seqs; j += 32)
            if (share[j] == page) {
                ++same;
                later |= j > i;
            }
        same = __reduce_add_sync(~0u, same);
        later = __any_sync(~0u, later);
        if ((later || holders[i] > same) && lane == 0) need[i] |= kCopies;
    }
    __syncthreads();
    // places in the list of free pages, row after row
    long long wanted = 0;
    for (int base = 0; base < p.n_seqs; base += kPlanThreads) {
        const int i = base + tid;
        const uint32_t raw = i < p.n_seqs ? need[i] : kStays;
        const long long mine = raw & kStays ? 0 : (raw & kPlace) + (raw & kCopies ? 1 : 0);
        long long sum;
        const long long before = block_sum_before(mine, sum);
        if (i < p.n_seqs) need[i] = (uint32_t)((wanted + before) & kPlace) | (raw & (kStays | kCopies));
        wanted += sum;
    }
    const int total = (int)min(wanted, (long long)INT32_MAX);
    __syncthreads();
    if (wanted > p.n_pages) {   // more than there are at all
        if (tid == 0) {
            raise(p, STOM_FLAG_NO_PAGE);
            p.head[0] = 0;
        }
        return;
    }
    // the first `total` free pages in ascending order
    int found = 0;
    for (int base = 0; base < p.n_pages && found < total; base += kPlanThreads * kPerThread) {
        const int at = base + tid * kPerThread;
        int r[kPerThread], mine = 0;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            r[j] = at + j < p.n_pages ? p.refs[at + j] : 1;
            mine += r[j] == 0;
        }
        int sum;
        int rank = found + block_sum_before(mine, sum);
#pragma unroll
        for (int j = 0; j < kPerThread; ++j)
            if (r[j] == 0) {
                if (rank < total) p.ids[rank] = at + j;
                ++rank;
            }
        found += sum;
    }
    __syncthreads();
    if (found < total) {
        if (tid == 0) {
            raise(p, STOM_FLAG_NO_PAGE);
            p.head[0] = 0;
        }
        return;
    }
    // a thread for each page of the list: its row is the last whose first place is not behind it
    for (int at = tid; at < total; at += kPlanThreads) {
        int i = 0, high = p.n_seqs;
        while (high - i > 1) {
            const int mid = (i + high) >> 1;
            if ((need[mid] & kPlace) <= (uint32_t)at) i = mid;
            else high = mid;
        }
        const int copy = need[i] & kCopies ? 1 : 0, k = at - (int)(need[i] & kPlace), id = p.ids[at];
        const int n = max(p.len[i], 0);
        p.table[i * p.table_stride + held_of(p, n) - copy + k] = id;
        p.refs[id] = 1;
        if (copy && k == 0) {
            atomicSub(p.refs + share[i], 1);
            p.moves[atomicAdd(&n_moves, 1)] =
                Move{share[i], id, n - (int)(div_by(p.by_page, (uint32_t)n) * p.by_page.d), 0};
        }
    }
    __syncthreads();
    for (int i = tid; i < p.n_seqs; i += kPlanThreads)
        if (!(need[i] & kStays)) p.len[i] = p.wish[i];
    if (tid == 0) p.head[0] = n_moves;
}

__global__ void __launch_bounds__(kPlanThreads) kv_compact_plan_kernel(const __grid_constant__ PagesParams p) {
    const int tid = threadIdx.x;
    grid_dependency_wait();
    int mine = 0, live;
    for (int i = tid; i < p.n_pages; i += kPlanThreads) {
        const int r = p.refs[i];
        mine += r > 0;
        p.ids[i] = -1;
        if (p.refs_out != p.refs) p.refs_out[i] = r > 0 ? r : 0;
    }
    block_sum_before(mine, live);
    // the k-th live page behind the front, and the k-th free page of the front
    int from = 0, to = 0;
    for (int base = 0; base < p.n_pages; base += kPlanThreads * kPerThread) {
        const int at = base + tid * kPerThread;
        int r[kPerThread], hole = 0, behind = 0;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            r[j] = at + j < p.n_pages ? p.refs[at + j] : -1;
            if (at + j < live) hole += r[j] <= 0;
            else behind += r[j] > 0;
        }
        int holes, behinds;
        int h = to + block_sum_before(hole, holes);
        int b = from + block_sum_before(behind, behinds);
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            if (at + j < live) {
                if (r[j] <= 0) p.moves[h++].dst = at + j;
            } else if (r[j] > 0) {
                p.moves[b++].src = at + j;
            }
        }
        to += holes;
        from += behinds;
    }
    __syncthreads();
    for (int k = tid; k < from; k += kPlanThreads) {
        const Move m = p.moves[k];
        p.moves[k].tokens = p.page_tokens;
        p.ids[m.src] = m.dst;
        p.refs_out[m.dst] = p.refs[m.src];
        p.refs_out[m.src] = 0;
    }
    if (tid == 0) {
        p.head[0] = from;
        if (p.n_live) *p.n_live = live;
    }
}

// Copies what the plan listed: a block takes one (page, layer, keys or values) at a time.  RENAME: the tables too.
template <bool RENAME>
__global__ void __launch_bounds__(256) kv_move_kernel(const __grid_constant__ PagesParams p) {
    grid_dependency_wait();
    const int moves = p.head[0];
    const int64_t tasks = (int64_t)moves * p.n_layers * 2;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int m = (int)(task / (2 * p.n_layers)), rest = (int)(task - (int64_t)m * 2 * p.n_layers);
        const Move mv = p.moves[m];
        char *base = (rest & 1 ? p.v : p.k) + 2 * (rest >> 1) * p.stride_layer;
        const char *src = base + 2 * mv.src * p.stride_page;
        char *dst = base + 2 * mv.dst * p.stride_page;
        const int n = (mv.tokens * p.n_kv_heads) << p.chunk_bits;
        auto place = [&](int i) {
            const int row = i >> p.chunk_bits, c = i & ((1 << p.chunk_bits) - 1);
            const int t = (int)div_by(p.by_head, (uint32_t)row), h = row - t * p.n_kv_heads;
            return 2 * (t * p.stride_token + h * p.stride_head) + c * 16;
        };
        constexpr int kBatch = 4;
        for (int i = threadIdx.x; i < n; i += 256 * kBatch) {
            uint4 x[kBatch];
            int64_t at[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (i + j * 256 < n) {
                    at[j] = place(i + j * 256);
                    x[j] = *reinterpret_cast<const uint4 *>(src + at[j]);
                }
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (i + j * 256 < n) *reinterpret_cast<uint4 *>(dst + at[j]) = x[j];
        }
    }
    if (RENAME) {
        for (int i = blockIdx.x; i < p.n_seqs; i += gridDim.x) {
            const int held = held_of(p, p.len[i]);
            for (int j = threadIdx.x; j < p.max_pages; j += 256) {
                int id = -1;
                if (j < held) {
                    id = p.table[i * p.table_stride + j];
                    // a page id that is none stays what it is, and so does a page that has not moved
                    if (!is_page(p, id)) raise(p, STOM_FLAG_BAD_INDEX);
                    else if (p.ids[id] >= 0) id = p.ids[id];
                }
                p.table_out[i * p.table_stride + j] = id;
            }
        }
    }
}

int64_t round256(int64_t x) { return (x + 255) & ~(int64_t)255; }

int32_t prepare(PagesParams &p, const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *wish, uint32_t *flags) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, true);
    if (rc) return rc;
    if (reinterpret_cast<uintptr_t>(wish) & 3u) return STOM_ERR_ALIGNMENT;
    if ((int64_t)pool->page_tokens * pool->n_kv_heads * (pool->head_dim / 8) > (1 << 30)) return STOM_ERR_SHAPE;
    if (pool->n_pages >= (1 << 30) || seqs->max_pages >= (1 << 30)) return STOM_ERR_SHAPE;
    p = PagesParams{};
    p.k = static_cast<char *>(pool->k);
    p.v = static_cast<char *>(pool->v);
    p.stride_layer = pool->stride_layer;
    p.stride_page = pool->stride_page;
    p.stride_token = pool->stride_token;
    p.stride_head = pool->stride_head;
    p.n_layers = pool->n_layers;
    p.n_pages = pool->n_pages;
    p.page_tokens = pool->page_tokens;
    p.n_kv_heads = pool->n_kv_heads;
    p.chunk_bits = pool->head_dim == 64 ? 3 : pool->head_dim == 128 ? 4 : 5;
    p.by_page = fast_div((uint32_t)pool->page_tokens);
    p.by_head = fast_div((uint32_t)pool->n_kv_heads);
    p.table = seqs->table;
    p.len = seqs->len;
    p.refs = seqs->refs;
    p.n_seqs = seqs->n_seqs;
    p.max_pages = seqs->max_pages;
    p.table_stride = seqs->table_stride;
    p.wish = wish;
    p.flags = flags;
    return STOM_OK;
}

int32_t bind_workspace(PagesParams &p, const stom_kv_pool *pool, const stom_kv_seqs *seqs, void *ws, int64_t bytes) {
    if (!ws || !aligned16(ws) || bytes < stom_kv_pages_workspace_bytes(pool, seqs)) return STOM_ERR_WORKSPACE;
    p.head = static_cast<int32_t *>(ws);
    p.ids = p.head + 64;
    p.moves = reinterpret_cast<Move *>(static_cast<char *>(ws) + 256 + round256((int64_t)pool->n_pages * 4));
    return STOM_OK;
}

int32_t failed(cudaError_t e) {
    set_last_cuda_error(e);
    return STOM_ERR_CUDA;
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int64_t stom_kv_pages_workspace_bytes(const stom_kv_pool *pool, const stom_kv_seqs *seqs) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, false);
    if (rc) return rc;
    const int64_t moves = seqs->n_seqs > pool->n_pages ? seqs->n_seqs : pool->n_pages;
    return 256 + round256((int64_t)pool->n_pages * 4) + round256(moves * (int64_t)sizeof(Move));
}

extern "C" int32_t stom_kv_reserve(const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *want,
                                   void *workspace, int64_t workspace_bytes, uint32_t *dev_flags, void *stream) {
    PagesParams p;
    int32_t rc = prepare(p, pool, seqs, want, dev_flags);
    if (rc) return rc;
    if (seqs->n_seqs > STOM_KV_MAX_SEQS) return STOM_ERR_SHAPE;
    rc = bind_workspace(p, pool, seqs, workspace, workspace_bytes);
    if (rc) return rc;
    if (seqs->n_seqs == 0) return STOM_OK;
    if (!want) return STOM_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const size_t smem = (size_t)seqs->n_seqs * 12;
    cudaError_t e = cudaSuccess;
    static std::atomic<uint64_t> allowed{0};
    if (smem > 47 * 1024) e = allow_shared(reinterpret_cast<const void *>(kv_reserve_plan_kernel), STOM_KV_MAX_SEQS * 12, allowed);
    if (e == cudaSuccess) e = launch_after_producer(kv_reserve_plan_kernel, dim3(1), dim3(kPlanThreads), smem, s, p);
    if (e == cudaSuccess) e = launch_after_producer(kv_move_kernel<false>, dim3(sms * 8), dim3(256), 0, s, p);
    return e == cudaSuccess ? finish_launch() : failed(e);
}

extern "C" int32_t stom_kv_fork(const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *parent,
                                uint32_t *dev_flags, void *stream) {
    PagesParams p;
    int32_t rc = prepare(p, pool, seqs, parent, dev_flags);
    if (rc) return rc;
    if (seqs->n_seqs == 0) return STOM_OK;
    if (!parent) return STOM_ERR_INVALID_ARG;
    cudaError_t e = launch_after_producer(kv_fork_kernel, dim3(seqs->n_seqs), dim3(128), 0, static_cast<cudaStream_t>(stream), p);
    return e == cudaSuccess ? finish_launch() : failed(e);
}

extern "C" int32_t stom_kv_free(const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *drop,
                                uint32_t *dev_flags, void *stream) {
    PagesParams p;
    int32_t rc = prepare(p, pool, seqs, drop, dev_flags);
    if (rc) return rc;
    if (seqs->n_seqs == 0) return STOM_OK;
    if (!drop) return STOM_ERR_INVALID_ARG;
    cudaError_t e = launch_after_producer(kv_free_kernel, dim3(seqs->n_seqs), dim3(128), 0, static_cast<cudaStream_t>(stream), p);
    return e == cudaSuccess ? finish_launch() : failed(e);
}

extern "C" int32_t stom_kv_compact(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t *table_out,
                                   int32_t *refs_out, int32_t *n_live, void *workspace, int64_t workspace_bytes,
                                   uint32_t *dev_flags, void *stream) {
    PagesParams p;
    int32_t rc = prepare(p, pool, seqs, nullptr, dev_flags);
    if (rc) return rc;
    if ((!table_out && seqs->n_seqs > 0) || !refs_out) return STOM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(table_out) | reinterpret_cast<uintptr_t>(refs_out) | reinterpret_cast<uintptr_t>(n_live)) & 3u)
        return STOM_ERR_ALIGNMENT;
    rc = bind_workspace(p, pool, seqs, workspace, workspace_bytes);
    if (rc) return rc;
    p.table_out = table_out;
    p.refs_out = refs_out;
    p.n_live = n_live;
    const int sms = sm_count();
    if (!sms) return STOM_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_after_producer(kv_compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    if (e == cudaSuccess) e = launch_after_producer(kv_move_kernel<true>, dim3(sms * 8), dim3(256), 0, s, p);
    return e == cudaSuccess ? finish_launch() : failed(e);
}
