// Attention weight that the rows of a paged cache receive from new tokens, accumulated.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {
namespace {

constexpr int MS_WARPS = 4;

struct MassParams {
    PagedView v;
    const __nv_bfloat16 *Q, *K;
    const float *lse, *mass_in;
    float* mass_out;
    float scale_log2;
};

// A warp per (sequence, KV head, cached row), a query at a time.
template <int D>
__global__ void __launch_bounds__(MS_WARPS * 32) mass_kernel(const MassParams p) {
    constexpr int E = D / 32;
    pdl_wait();
    pdl_release();
    if (*p.v.status != 0) return;
    const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, G = p.v.G;
    const PagedSeq s = load_seq(p.v, b);
    for (int j = (int)blockIdx.x * MS_WARPS + (threadIdx.x >> 5); j < s.L; j += (int)gridDim.x * MS_WARPS) {
        const long long row = load_pool_row(p.v, b, j);
        if (row < 0) continue;
        float k[E], sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) k[e] = __bfloat162float(p.K[((size_t)row * p.v.Hkv + h) * D + lane + 32 * e]);
        const int old = s.L - s.n;
        for (int i = max(0, j - old); i < s.n; ++i)
            for (int g = 0; g < G; ++g) {
                const size_t q = (size_t)(s.q0 + i) * p.v.Hq + (size_t)h * G + g;
                float x = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) x = fmaf(k[e], __bfloat162float(p.Q[q * D + lane + 32 * e]), x);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
                sum += exp2f(x * p.scale_log2 - p.lse[q] * 1.4426950408889634f);
            }
        const size_t at = ((size_t)b * p.v.Hkv + h) * p.v.cap + j;
        if (lane == 0) p.mass_out[at] = (p.mass_in != nullptr && j < old ? p.mass_in[at] : 0.f) + sum;
    }
}

}  // namespace
}  // namespace seka

extern "C" seka_status seka_attention_mass(const seka_paged_shape* shape, const void* Q, const void* K_pages, const float* lse,
                                           const float* mass_in, float* mass_out, void* workspace, size_t workspace_bytes,
                                           void* cuda_stream) {
    using namespace seka;
    seka_status stc = validate_paged(shape);
    if (stc != SEKA_OK) return stc;
    if (shape->batch == 0 || shape->max_pages == 0) return SEKA_OK;
    if (!mass_out || (shape->total_new > 0 && (!Q || !lse)) || (!K_pages && shape->n_pages > 0)) return SEKA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K_pages) & 15) return SEKA_ERR_INVALID_ARG;
    stc = check_paged_call(shape, workspace, workspace_bytes);
    if (stc != SEKA_OK) return stc;
    MassParams p;
    p.v = paged_view(shape, workspace);
    p.Q = static_cast<const __nv_bfloat16*>(Q); p.K = static_cast<const __nv_bfloat16*>(K_pages);
    p.lse = lse; p.mass_in = mass_in; p.mass_out = mass_out;
    const float scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.f / sqrtf((float)shape->head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    const dim3 grid((unsigned)((p.v.cap + 127) / 128), (unsigned)p.v.Hkv, (unsigned)p.v.B);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return shape->head_dim == 128 ? launch_kernel(true, mass_kernel<128>, grid, MS_WARPS * 32, 0, st, p)
                                  : launch_kernel(true, mass_kernel<64>, grid, MS_WARPS * 32, 0, st, p);
}
