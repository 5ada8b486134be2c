// Paged cache, host side: validation, workspace size, table of the rotation.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {

seka_status validate_paged(const seka_paged_shape* s) {
    if (s == nullptr) return SEKA_ERR_INVALID_ARG;
    if (s->batch < 0 || s->total_new < 0 || s->max_new < 0 || s->n_pages < 0 || s->max_pages < 0) return SEKA_ERR_INVALID_ARG;
    if (s->batch > 0 && (s->n_pages < 1 || s->max_pages < 1)) return SEKA_ERR_INVALID_ARG;
    if (s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->n_q_heads % s->n_kv_heads != 0) return SEKA_ERR_INVALID_ARG;
    if (s->dtype != SEKA_F32 && s->dtype != SEKA_BF16) return SEKA_ERR_INVALID_ARG;
    if (!(s->softmax_scale >= 0.f) || isinf(s->softmax_scale)) return SEKA_ERR_INVALID_ARG;
    if (s->cu_new == nullptr && (long long)s->total_new != (long long)s->batch * s->max_new) return SEKA_ERR_INVALID_ARG;
    if (s->head_dim != 64 && s->head_dim != 128) return SEKA_ERR_UNSUPPORTED;
    if (s->page_size != 16 && s->page_size != 32 && s->page_size != 64 && s->page_size != 128 && s->page_size != 256)
        return SEKA_ERR_UNSUPPORTED;
    if (s->n_q_heads / s->n_kv_heads > 128 || s->n_q_heads > 32767 || s->batch > 65535) return SEKA_ERR_UNSUPPORTED;
    // rows of a sequence and of the pool, and tokens, are counted in 31 bits (bytes and elements in 64)
    if ((long long)s->max_pages * s->page_size > 0x7fff0000LL || (long long)s->n_pages * s->page_size > 0x7fff0000LL ||
        s->max_new > 0x7fff0000 || s->total_new > 0x7fff0000) return SEKA_ERR_UNSUPPORTED;
    // state rows, and with them the workspace, are counted in 64 bits
    const long long pairs = (long long)s->batch * s->n_kv_heads, cap = (long long)s->max_pages * s->page_size;
    if (pairs > 0x7fffffffLL || pairs * cap > 1LL << 40) return SEKA_ERR_UNSUPPORTED;
    return SEKA_OK;
}

PagedView paged_view(const seka_paged_shape* s, void* workspace) {
    PagedView v;
    v.table = s->block_table; v.lens = s->cache_lens; v.cu = s->cu_new;
    v.status = static_cast<int*>(workspace);
    v.B = s->batch; v.T = s->total_new; v.max_new = s->max_new;
    v.Hq = s->n_q_heads; v.Hkv = s->n_kv_heads; v.G = s->n_q_heads / s->n_kv_heads;
    v.max_pages = s->max_pages; v.n_pages = s->n_pages; v.cap = s->max_pages * s->page_size;
    v.page_shift = 0;
    while ((1 << v.page_shift) < s->page_size) ++v.page_shift;
    return v;
}

seka_status check_paged_call(const seka_paged_shape* s, const void* workspace, size_t workspace_bytes) {
    if (s->cache_lens == nullptr || (s->max_pages > 0 && s->block_table == nullptr)) return SEKA_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < paged_layout(s).total || ((uintptr_t)workspace & 255)) return SEKA_ERR_WORKSPACE;
    return SEKA_OK;
}

}  // namespace seka

extern "C" size_t seka_paged_workspace_bytes(const seka_paged_shape* shape) {
    if (seka::validate_paged(shape) != SEKA_OK) return 0;
    return seka::paged_layout(shape).total;
}

extern "C" seka_status seka_rope_turns(int32_t rot_dim, double base, int32_t scaling, double scale, double trained_len,
                                       double low_turns, double high_turns, double* h_turns) {
    if (h_turns == nullptr || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 128) return SEKA_ERR_INVALID_ARG;
    if (!(base > 1.0) || isinf(base) || scaling < SEKA_SCALE_PLAIN || scaling > SEKA_SCALE_WAVELENGTH) return SEKA_ERR_INVALID_ARG;
    if (scaling != SEKA_SCALE_PLAIN && (!(scale > 0.0) || isinf(scale))) return SEKA_ERR_INVALID_ARG;
    if (scaling == SEKA_SCALE_BASE && rot_dim == 2) return SEKA_ERR_INVALID_ARG;      // one pair: the exponent r / (r - 2) does not exist
    if (scaling == SEKA_SCALE_WAVELENGTH && (!(trained_len > 0.0) || !(high_turns > low_turns) || isinf(trained_len) || isinf(high_turns) || isinf(low_turns)))
        return SEKA_ERR_INVALID_ARG;
    const double r = rot_dim, two_pi = 6.283185307179586476925;
    if (scaling == SEKA_SCALE_BASE) base *= pow(scale, r / (r - 2.0));
    for (int i = 0; i < rot_dim / 2; ++i) {
        double t = pow(base, -2.0 * i / r) / two_pi;
        if (scaling == SEKA_SCALE_LINEAR) t /= scale;
        if (scaling == SEKA_SCALE_WAVELENGTH) {
            const double w = fmin(1.0, fmax(0.0, (trained_len * t - low_turns) / (high_turns - low_turns)));     // 1: left as it is
            t = t * w + t / scale * (1.0 - w);
        }
        h_turns[i] = t;
    }
    return SEKA_OK;
}
