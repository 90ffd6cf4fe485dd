// Host-only part of the paged cache: checks of the descriptors and the rotation frequencies.
#include "stom_kv.cuh"

#include <math.h>

#include <atomic>

namespace stom {

int32_t check_pool(const stom_kv_pool *p) {
    if (!p || !p->k || !p->v) return STOM_ERR_INVALID_ARG;
    if (p->n_layers < 1 || p->n_pages < 1 || p->page_tokens < 1 || p->n_kv_heads < 1) return STOM_ERR_INVALID_ARG;
    if (p->dtype != STOM_BF16 && p->dtype != STOM_FP16) return STOM_ERR_UNSUPPORTED;
    if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return STOM_ERR_SHAPE;
    if (!aligned16(p->k) || !aligned16(p->v)) return STOM_ERR_ALIGNMENT;
    const int64_t stride[4] = {p->stride_layer, p->stride_page, p->stride_token, p->stride_head};
    const int32_t extent[4] = {p->n_layers, p->n_pages, p->page_tokens, p->n_kv_heads};
    for (int i = 0; i < 4; ++i) {
        if (!stride_ok(stride[i], p->dtype)) return STOM_ERR_ALIGNMENT;
        if (extent[i] > 1 && stride[i] < p->head_dim) return STOM_ERR_INVALID_ARG;  // rows would overlap
        if (stride[i] < 0) return STOM_ERR_INVALID_ARG;
    }
    return STOM_OK;
}

int32_t check_seqs(const stom_kv_pool *, const stom_kv_seqs *s, bool need_refs) {
    if (!s || s->n_seqs < 0 || s->max_pages < 1 || s->table_stride < s->max_pages) return STOM_ERR_INVALID_ARG;
    if ((s->n_seqs > 0 && (!s->table || !s->len)) || (need_refs && !s->refs)) return STOM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(s->table) | reinterpret_cast<uintptr_t>(s->len) | reinterpret_cast<uintptr_t>(s->refs)) & 3u)
        return STOM_ERR_ALIGNMENT;
    return STOM_OK;
}

int32_t sm_count() {
    static std::atomic<int32_t> known[64];   // a device's count does not change
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) {
        set_last_cuda_error(e);
        return 0;
    }
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

}  // namespace stom

using namespace stom;

extern "C" int32_t stom_kv_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double trained,
                                       double low, double high, double *freq) {
    if (rot_dim < 0 || !(theta > 0.0) || !isfinite(theta) || (rot_dim > 0 && !freq)) return STOM_ERR_INVALID_ARG;
    if (rot_dim % 16) return STOM_ERR_SHAPE;
    if (scaling < STOM_ROPE_PLAIN || scaling > STOM_ROPE_WAVES) return STOM_ERR_UNSUPPORTED;
    if (scaling != STOM_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return STOM_ERR_INVALID_ARG;
    if (scaling == STOM_ROPE_WAVES && (!(trained > 0.0) || !(low >= 0.0) || !(high > low) || !isfinite(trained * high)))
        return STOM_ERR_INVALID_ARG;
    const double r = rot_dim;
    const double base = scaling == STOM_ROPE_BASE ? theta * pow(factor, r / (r - 2.0)) : theta;
    for (int32_t i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / r);
        if (scaling == STOM_ROPE_LINEAR) f /= factor;
        if (scaling == STOM_ROPE_WAVES) {
            const double turns = trained * f / 6.283185307179586;
            const double keep = fmin(1.0, fmax(0.0, (turns - low) / (high - low)));
            f *= keep + (1.0 - keep) / factor;
        }
        freq[i] = f;
    }
    return STOM_OK;
}
