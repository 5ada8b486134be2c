// Rotary positions on new tokens' queries and keys, keys and values to their pages.
//
// Pair (x, x') of a head at position p turns by a = 2 pi p turns_i:  y = f (x cos a - x' sin a),  y' = f (x' cos a + x sin a).
// The angle in turns is reduced to [-1/2, 1/2] in fp64 (p turns_i is exact to 2^-53 of itself: 1e-9 of a turn at a position of
// 10^7) and only then becomes fp32; products are fp32, each output is rounded once.
//
// Bound by HBM: every element is read once and written once.  A block takes one token (for few tokens several blocks share it, a
// part of the heads each); its cosines and sines are computed once into shared memory.  A lane owns eight consecutive
// elements of a head; a rotation in halves finds the partners of its elements, which lie r/2 away at no alignment, through a
// copy of the row in shared memory that the lanes of one warp share.
#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {
namespace {

constexpr int ROPE_THREADS = 256;

struct RopeParams {
    PagedView v;
    const void *Q, *K, *V;
    long long q_stride, k_stride, v_stride;     // elements between tokens
    const int* positions;
    const double* turns;                        // null: nothing is rotated
    __nv_bfloat16 *Q_out, *K_pages, *V_pages;
    int* pos_cache;
    int r, layout;
    float magnitude;
};

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u[i]));
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    } else {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_kernel(const RopeParams p) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;          // lanes of a row, rows of a warp
    __shared__ float2 cs[D / 2];
    __shared__ float rows[ROPE_THREADS / 32][RPW][D];
    __shared__ int tok[4];                              // sequence, row in the cache (negative: padding), pool row
    const int t = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    pdl_release();
    const int status0 = *p.v.status;
    if (tid == 0) { tok[0] = -1; tok[1] = -1; tok[2] = -1; }
    __syncthreads();
    if (status0 != 0) return;
    // the sequence that owns the token
    for (int b = tid; b < p.v.B; b += ROPE_THREADS) {
        const int q0 = p.v.cu ? p.v.cu[b] : b * p.v.max_new, q1 = p.v.cu ? p.v.cu[b + 1] : q0 + p.v.max_new;
        if (t < q0 || t >= q1) continue;
        const PagedSeq s = check_seq(p.v, q0, q1, p.v.lens[b]);
        if (!s.valid) { report_invalid(p.v.status, kWhereSeq); continue; }
        const int j = s.L - s.n + (t - q0);
        tok[0] = b; tok[1] = j;
        if (j >= 0) tok[2] = (int)load_pool_row(p.v, b, j);
    }
    __syncthreads();
    const int b = tok[0], j = tok[1];
    const long long row = tok[2];
    if (p.turns != nullptr && tid < p.r / 2) {
        const int pos = p.positions ? p.positions[t] : j;
        double a = (double)pos * p.turns[tid];
        a -= rint(a);
        float s, c;
        sincospif(2.f * (float)a, &s, &c);
        cs[tid] = make_float2(c * p.magnitude, s * p.magnitude);
    }
    __syncthreads();
    const int Hq = p.v.Hq, Hkv = p.v.Hkv, n_rows = Hq + 2 * Hkv, r = p.turns ? p.r : 0, half = r / 2;
    const int sub = lane / LPR, e0 = (lane % LPR) * 8;
    const int first = ((int)blockIdx.y * (ROPE_THREADS / 32) + warp) * RPW;
    for (int h0 = first; h0 < n_rows; h0 += (int)gridDim.y * (ROPE_THREADS / 32) * RPW) {
        const int h = h0 + sub;
        const bool isq = h < Hq, isk = !isq && h < Hq + Hkv, have = h < n_rows && (isq || row >= 0);
        const bool turn = have && (isq || isk) && e0 < r;
        float x[8];
        if (have) {
            const T* src = isq ? static_cast<const T*>(p.Q) + t * p.q_stride + (size_t)h * D
                         : isk ? static_cast<const T*>(p.K) + t * p.k_stride + (size_t)(h - Hq) * D
                               : static_cast<const T*>(p.V) + t * p.v_stride + (size_t)(h - Hq - Hkv) * D;
            load8(src + e0, x);
        }
        if (p.layout == SEKA_ROPE_INTERLEAVED) {
            if (turn) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e0 + 2 * i < r) {
                        const float2 c = cs[e0 / 2 + i];
                        const float u = x[2 * i], w = x[2 * i + 1];
                        x[2 * i] = u * c.x - w * c.y; x[2 * i + 1] = w * c.x + u * c.y;
                    }
            }
        } else {
            float* mine = rows[warp][sub];
            __syncwarp();                               // the partners of the row before have been read
            if (turn) {
#pragma unroll
                for (int i = 0; i < 8; ++i) mine[e0 + i] = x[i];
            }
            __syncwarp();
            if (turn) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = e0 + i;
                    if (e < half) { const float2 c = cs[e]; x[i] = x[i] * c.x - mine[e + half] * c.y; }
                    else if (e < r) { const float2 c = cs[e - half]; x[i] = x[i] * c.x + mine[e - half] * c.y; }
                }
            }
        }
        if (have) {
            __nv_bfloat16* dst = isq ? p.Q_out + ((size_t)t * Hq + h) * D
                               : isk ? p.K_pages + ((size_t)row * Hkv + (h - Hq)) * D : p.V_pages + ((size_t)row * Hkv + (h - Hq - Hkv)) * D;
            *reinterpret_cast<uint4*>(dst + e0) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        }
    }
    if (p.pos_cache != nullptr && blockIdx.y == 0 && row >= 0)
        for (int h = tid; h < Hkv; h += ROPE_THREADS)
            p.pos_cache[((size_t)b * Hkv + h) * p.v.cap + j] = p.positions ? p.positions[t] : j;
}

template <typename T>
seka_status launch_rope(const RopeParams& p, int D, cudaStream_t st) {
    int n_sm = 0;
    if (!device_info(&n_sm)) return SEKA_ERR_CUDA;
    const int per = ROPE_THREADS / 32 * (32 * 8 / D), n_rows = p.v.Hq + 2 * p.v.Hkv;
    int split = 1;                  // blocks of a token: as many as fill the SMs, no more than it has rows for
    while (split * per < n_rows && (long long)p.v.T * split < 2LL * n_sm) ++split;
    const dim3 grid((unsigned)p.v.T, (unsigned)split);
    return D == 128 ? launch_kernel(true, rope_append_kernel<T, 128>, grid, ROPE_THREADS, 0, st, p)
                    : launch_kernel(true, rope_append_kernel<T, 64>, grid, ROPE_THREADS, 0, st, p);
}

}  // namespace
}  // namespace seka

extern "C" seka_status seka_rope_append(const seka_paged_shape* shape, const seka_rope* rope, const void* Q, int64_t q_stride,
                                        const void* K, int64_t k_stride, const void* V, int64_t v_stride, const int32_t* positions,
                                        void* Q_out, void* K_pages, void* V_pages, int32_t* pos_cache,
                                        void* workspace, size_t workspace_bytes, void* cuda_stream) {
    using namespace seka;
    seka_status stc = validate_paged(shape);
    if (stc != SEKA_OK) return stc;
    const int D = shape->head_dim, Hq = shape->n_q_heads, Hkv = shape->n_kv_heads;
    if (rope != nullptr) {
        if (rope->rot_dim < 2 || rope->rot_dim % 2 != 0 || rope->rot_dim > D || rope->turns == nullptr) return SEKA_ERR_INVALID_ARG;
        if (rope->layout != SEKA_ROPE_HALF && rope->layout != SEKA_ROPE_INTERLEAVED) return SEKA_ERR_INVALID_ARG;
        if (!(rope->magnitude >= 0.f) || isinf(rope->magnitude)) return SEKA_ERR_INVALID_ARG;
    }
    if (shape->batch == 0 || shape->total_new == 0) return SEKA_OK;
    const long long pq = (long long)Hq * D, pk = (long long)Hkv * D, unit = shape->dtype == SEKA_F32 ? 4 : 8;     // 16 bytes
    if (q_stride == 0) q_stride = pq;
    if (k_stride == 0) k_stride = pk;
    if (v_stride == 0) v_stride = pk;
    if (q_stride < pq || k_stride < pk || v_stride < pk || q_stride % unit || k_stride % unit || v_stride % unit) return SEKA_ERR_INVALID_ARG;
    if (!Q || !K || !V || !Q_out || ((!K_pages || !V_pages) && shape->n_pages > 0)) return SEKA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)Q_out | (uintptr_t)K_pages | (uintptr_t)V_pages) & 15) return SEKA_ERR_INVALID_ARG;
    if (Q == Q_out && (shape->dtype != SEKA_BF16 || q_stride != pq)) return SEKA_ERR_INVALID_ARG;
    stc = check_paged_call(shape, workspace, workspace_bytes);
    if (stc != SEKA_OK) return stc;

    RopeParams p;
    p.v = paged_view(shape, workspace);
    p.Q = Q; p.K = K; p.V = V; p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
    p.positions = positions; p.pos_cache = pos_cache;
    p.Q_out = static_cast<__nv_bfloat16*>(Q_out);
    p.K_pages = static_cast<__nv_bfloat16*>(K_pages); p.V_pages = static_cast<__nv_bfloat16*>(V_pages);
    p.turns = rope ? rope->turns : nullptr; p.r = rope ? rope->rot_dim : 0; p.layout = rope ? rope->layout : 0;
    p.magnitude = rope && rope->magnitude > 0.f ? rope->magnitude : 1.f;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return shape->dtype == SEKA_F32 ? launch_rope<float>(p, D, st) : launch_rope<__nv_bfloat16>(p, D, st);
}
