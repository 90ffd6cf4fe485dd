// The drafted path that is kept (stom_kv_accept): the walk through a sequence's tree, its keys and values moved together
// in all layers, lengths and page counts.
//
// One cluster of blocks per sequence, one launch: every block reads the tree and walks it (a warp looks at all nodes of a
// step at once; a handful of steps), the blocks share out the layers.  A thread has one 16-byte column of a layer's keys
// or values and moves it step by step: the k-th kept node goes from slot j_k to slot k <= j_k, and j_(k+1) > j_k >= k, so
// that no store touches a later step's source and all of a batch's loads may run ahead of its stores.  Page ids are read
// before a cluster barrier, behind which the first block writes length, table and counts.
//
// What bounds it: latency (length and range, then pages and tree, then rows).  Measured together with the stom_kv_reserve that
// makes room for the nodes, 28 layers, 4 heads of 128: one stream with a tree of 64 nodes 9 to 10 us, 40 streams of 33 nodes 12
// us (1 us of it the copies' bytes).
#include "stom_kv.cuh"

namespace stom {

namespace {

constexpr int kThreads = 256;
constexpr int kCluster = 8;

struct AcceptParams {
    char *k, *v;
    int64_t stride_layer, stride_page, stride_token, stride_head;
    int32_t n_layers, n_pages, n_kv_heads, chunk_bits;   // 2^chunk_bits 16-byte chunks make a row
    FastDiv by_page, by_head;
    int32_t *table, *len, *refs;
    int64_t table_stride, room;
    int32_t n_tokens;
    const int32_t *first, *parent, *draft, *chosen;
    int32_t *path, *n_accepted, *next;
    uint32_t *flags;
};

__global__ void __launch_bounds__(kThreads) kv_accept_kernel(const __grid_constant__ AcceptParams p) {
    __shared__ int parent[STOM_KV_MAX_TREE], draft[STOM_KV_MAX_TREE], chosen[STOM_KV_MAX_TREE], kept[STOM_KV_MAX_TREE];
    __shared__ int64_t row_of[STOM_KV_MAX_TREE];   // byte offset of each node's slot in a layer, -1: its page id is none
    __shared__ int n_kept;
    const int i = blockIdx.y, rank = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    grid_dependency_wait();
    const int a = p.first[i], b = p.first[i + 1], len = max(p.len[i], 0);
    const int n = b - a, base = len - n;
    const bool good = a >= 0 && a <= b && b <= p.n_tokens && n <= len && n <= STOM_KV_MAX_TREE && len <= p.room;
    const int nodes = good ? n : 0;
    int32_t *row = p.table + i * p.table_stride;
    if (tid < nodes) {
        parent[tid] = p.parent ? p.parent[a + tid] : tid - 1;
        draft[tid] = p.draft[a + tid];
        chosen[tid] = p.chosen[a + tid];
        const int t = base + tid, pg = (int)div_by(p.by_page, (uint32_t)t), id = row[pg];
        const bool is = (uint32_t)id < (uint32_t)p.n_pages;
        row_of[tid] = is ? 2 * (id * p.stride_page + (t - pg * (int64_t)p.by_page.d) * p.stride_token) : -1;
    }
    __syncthreads();
    if (tid < 32) {
        int at = 0, count = 0;
        while (at < nodes) {
            if (lane == 0) kept[count] = at;
            ++count;
            const int want = chosen[at];
            int child = nodes;
            for (int c0 = at + 1; c0 < nodes && child == nodes && want >= 0; c0 += 32) {
                const int c = c0 + lane;
                const uint32_t yes = __ballot_sync(~0u, c < nodes && parent[c] == at && draft[c] == want);
                if (yes) child = c0 + __ffs(yes) - 1;
            }
            at = child;
        }
        if (lane == 0) n_kept = count;
    }
    cluster_sync();   // every block has read the length and the pages; a block's own walk is done
    const int count = n_kept;

    if (rank == 0) {
        if (!good && p.flags && tid == 0) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
        if (tid < nodes) {
            if (p.path) p.path[a + tid] = tid < count ? kept[tid] : -1;
            // (a parent that is none counts as the context: the walk never finds it)
            if ((row_of[tid] < 0 || parent[tid] < -1 || parent[tid] >= tid) && p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
        }
        if (tid == 0) {
            if (p.n_accepted) p.n_accepted[i] = count;
            if (p.next) p.next[i] = count ? chosen[kept[count - 1]] : -1;
        }
        if (nodes) {
            if (tid == 0) p.len[i] = base + count;
            // pages of the old length that the new one does not reach (count >= 1: the new length is not 0)
            const int keep = (int)div_by(p.by_page, (uint32_t)(base + count - 1)) + 1;
            const int held = (int)div_by(p.by_page, (uint32_t)(len - 1)) + 1;
            for (int j = keep + tid; j < held; j += kThreads) {
                const int id = row[j];
                if ((uint32_t)id >= (uint32_t)p.n_pages) {
                    if (p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
                } else if (atomicSub(p.refs + id, 1) <= 0) {   // was free already: a table that does not fit its counts
                    atomicAdd(p.refs + id, 1);
                    if (p.flags) atomicOr(p.flags, STOM_FLAG_BAD_INDEX);
                }
                row[j] = -1;
            }
        }
    }
    if (count < 2) return;

    // columns: (layer, keys or values, head, chunk), chunks fastest
    const int64_t columns = ((int64_t)p.n_layers * 2 * p.n_kv_heads) << p.chunk_bits;
    for (int64_t col = rank * kThreads + tid; col < columns; col += kCluster * kThreads) {
        const int c = (int)(col & ((1 << p.chunk_bits) - 1));
        const uint32_t rest = (uint32_t)(col >> p.chunk_bits);
        const uint32_t lk = div_by(p.by_head, rest), h = rest - lk * (uint32_t)p.n_kv_heads;
        char *at = (lk & 1 ? p.v : p.k) + 2 * ((int64_t)(lk >> 1) * p.stride_layer + h * p.stride_head) + c * 16;
        constexpr int kBatch = 8;
        for (int s0 = 1; s0 < count; s0 += kBatch) {
            uint4 x[kBatch];
            int64_t to[kBatch];
#pragma unroll
            for (int s = 0; s < kBatch; ++s) {
                to[s] = -1;
                if (s0 + s < count) {
                    const int j = kept[s0 + s];
                    const int64_t from = row_of[j];
                    if (j != s0 + s && from >= 0 && row_of[s0 + s] >= 0) {
                        to[s] = row_of[s0 + s];
                        x[s] = *reinterpret_cast<const uint4 *>(at + from);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < kBatch; ++s)
                if (to[s] >= 0) *reinterpret_cast<uint4 *>(at + to[s]) = x[s];
        }
    }
}

}  // namespace

}  // namespace stom

using namespace stom;

extern "C" int32_t stom_kv_accept(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t n_tokens, const int32_t *first,
                                  const int32_t *parent, const int32_t *draft, const int32_t *chosen, int32_t *path,
                                  int32_t *n_accepted, int32_t *next, uint32_t *dev_flags, void *stream) {
    int32_t rc = check_pool(pool);
    if (!rc) rc = check_seqs(pool, seqs, true);
    if (rc) return rc;
    if (n_tokens < 0) return STOM_ERR_INVALID_ARG;
    const int64_t room = (int64_t)seqs->max_pages * pool->page_tokens;
    if (seqs->n_seqs > STOM_KV_MAX_SEQS || room > INT32_MAX - 32) return STOM_ERR_SHAPE;
    if ((int64_t)pool->n_layers * 2 * pool->n_kv_heads > INT32_MAX) return STOM_ERR_SHAPE;
    if (seqs->n_seqs == 0) return STOM_OK;
    if (!first || (n_tokens > 0 && (!draft || !chosen))) return STOM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(first) | reinterpret_cast<uintptr_t>(parent) | reinterpret_cast<uintptr_t>(draft) |
         reinterpret_cast<uintptr_t>(chosen) | reinterpret_cast<uintptr_t>(path) | reinterpret_cast<uintptr_t>(n_accepted) |
         reinterpret_cast<uintptr_t>(next)) & 3u)
        return STOM_ERR_ALIGNMENT;
    AcceptParams p = {};
    p.k = static_cast<char *>(pool->k);
    p.v = static_cast<char *>(pool->v);
    p.stride_layer = pool->stride_layer;
    p.stride_page = pool->stride_page;
    p.stride_token = pool->stride_token;
    p.stride_head = pool->stride_head;
    p.n_layers = pool->n_layers;
    p.n_pages = pool->n_pages;
    p.n_kv_heads = pool->n_kv_heads;
    p.chunk_bits = pool->head_dim == 64 ? 3 : pool->head_dim == 128 ? 4 : 5;
    p.by_page = fast_div((uint32_t)pool->page_tokens);
    p.by_head = fast_div((uint32_t)pool->n_kv_heads);
    p.table = seqs->table;
    p.len = seqs->len;
    p.refs = seqs->refs;
    p.table_stride = seqs->table_stride;
    p.room = room;
    p.n_tokens = n_tokens;
    p.first = first;
    p.parent = parent;
    p.draft = draft;
    p.chosen = chosen;
    p.path = path;
    p.n_accepted = n_accepted;
    p.next = next;
    p.flags = dev_flags;

    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(kCluster, seqs->n_seqs);
    lc.blockDim = dim3(kThreads);
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = kCluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&lc, kv_accept_kernel, p);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return STOM_ERR_CUDA;
    }
    return finish_launch();
}
