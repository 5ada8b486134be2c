// Attention of new tokens over a paged cache.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {
namespace {

constexpr int PA_WARPS = 4;

struct PagedAttnParams {
    PagedView v;
    const __nv_bfloat16 *Q, *K, *V;
    __nv_bfloat16* O;
    float* lse;
    float scale_log2;
};

// A warp per (token, query head), a key at a time.
template <int D>
__global__ void __launch_bounds__(PA_WARPS * 32) paged_attn_kernel(const PagedAttnParams p) {
    constexpr int E = D / 32;
    pdl_wait();
    pdl_release();
    if (*p.v.status != 0) return;
    const long long w = (long long)blockIdx.x * PA_WARPS + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (w >= (long long)p.v.T * p.v.Hq) return;
    const int t = (int)(w / p.v.Hq), hq = (int)(w % p.v.Hq), h = hq / p.v.G;
    int b = -1, limit = -1;
    for (int i = 0; i < p.v.B; ++i) {
        const int q0 = p.v.cu ? p.v.cu[i] : i * p.v.max_new, q1 = p.v.cu ? p.v.cu[i + 1] : q0 + p.v.max_new;
        if (t >= q0 && t < q1) {
            const PagedSeq s = load_seq(p.v, i);
            if (s.valid) { b = i; limit = s.L - s.n + (t - q0); }
        }
    }
    float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) { q[e] = __bfloat162float(p.Q[(size_t)w * D + lane + 32 * e]); o[e] = 0.f; }
    for (int j = 0; j <= limit; ++j) {
        const long long row = load_pool_row(p.v, b, j);
        if (row < 0) break;
        const __nv_bfloat16 *k = p.K + ((size_t)row * p.v.Hkv + h) * D, *v = p.V + ((size_t)row * p.v.Hkv + h) * D;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(q[e], __bfloat162float(k[lane + 32 * e]), s);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= p.scale_log2;
        const float mn = fmaxf(m, s), f = mn == -INFINITY ? 1.f : exp2f(m - mn), pe = mn == -INFINITY ? 0.f : exp2f(s - mn);
        l = l * f + pe;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + pe * __bfloat162float(v[lane + 32 * e]);
        m = mn;
    }
    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
#pragma unroll
    for (int e = 0; e < E; ++e) p.O[(size_t)w * D + lane + 32 * e] = __float2bfloat16(o[e] * inv);
    if (p.lse != nullptr && lane == 0) p.lse[w] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
}

}  // namespace
}  // namespace seka

extern "C" seka_status seka_paged_attention(const seka_paged_shape* shape, const void* Q, const void* K_pages, const void* V_pages,
                                            void* O, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    using namespace seka;
    seka_status stc = validate_paged(shape);
    if (stc != SEKA_OK) return stc;
    if (shape->batch == 0 || shape->total_new == 0) return SEKA_OK;
    if (!Q || !O || ((!K_pages || !V_pages) && shape->n_pages > 0)) return SEKA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K_pages | (uintptr_t)V_pages | (uintptr_t)O) & 15) return SEKA_ERR_INVALID_ARG;
    stc = check_paged_call(shape, workspace, workspace_bytes);
    if (stc != SEKA_OK) return stc;
    PagedAttnParams p;
    p.v = paged_view(shape, workspace);
    p.Q = static_cast<const __nv_bfloat16*>(Q); p.K = static_cast<const __nv_bfloat16*>(K_pages); p.V = static_cast<const __nv_bfloat16*>(V_pages);
    p.O = static_cast<__nv_bfloat16*>(O); p.lse = lse;
    const float scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.f / sqrtf((float)shape->head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    const long long warps = (long long)shape->total_new * shape->n_q_heads;
    const unsigned grid = (unsigned)((warps + PA_WARPS - 1) / PA_WARPS);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return shape->head_dim == 128 ? launch_kernel(true, paged_attn_kernel<128>, grid, PA_WARPS * 32, 0, st, p)
                                  : launch_kernel(true, paged_attn_kernel<64>, grid, PA_WARPS * 32, 0, st, p);
}
