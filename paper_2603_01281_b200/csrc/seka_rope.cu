// Rotary positions on new tokens' queries and keys, keys and values to their pages.
//
// Pair (x, x') of a head at position p turns by a = 2 pi p turns_i:  y = f (x cos a - x' sin a),  y' = f (x' cos a + x sin a).
// The angle in turns is reduced to [-1/2, 1/2] in fp64 (p turns_i is exact to 2^-53 of itself: 1e-9 of a turn at a position of
// 10^7) and only then becomes fp32; products are fp32, each output is rounded once.
//
// Bound by HBM: every element is read once and written once.  A block takes a few tokens; their cosines and sines are computed once
// into shared memory.  A lane owns 16 elements of a head, as eight pairs where it can:
//   NEIGHBOURS  interleaved pairs: 16 consecutive elements, any r (also what is not rotated at all);
//   HALVES      pairs r/2 apart with r a multiple of 16: eight elements and their eight partners, both on 16-byte boundaries;
//   STAGED      pairs r/2 apart at no alignment: the warp's rows go through shared memory, a lane per pair there, three warp barriers a
//               row (16384 tokens of 32/8 heads of 128, r = 126 / 22 / 2: 101 / 89 / 90 us, HALVES at r = 128 81).
// The loads of the first rows are issued before the token's sequence, page and angles are known (100 -> 88 us); three groups of rows are in flight
// as bf16, two as fp32.  16384 tokens of 32/8 heads of 128 in bf16 (403 MB): 81 us, 5.0 TB/s; some 16000 tokens of 16/16 heads of 64 in fp32
// (313 MB): 56 us, 5.6 TB/s; 64 tokens: 6.3 us on the device, less than the call's work on the host.
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

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[16], int at) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u[i]));
            x[at + 2 * i] = f.x; x[at + 2 * i + 1] = f.y;
        }
    } else {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        x[at] = a.x; x[at + 1] = a.y; x[at + 2] = a.z; x[at + 3] = a.w;
        x[at + 4] = b.x; x[at + 5] = b.y; x[at + 6] = b.z; x[at + 7] = b.w;
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[16], int at) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[at], x[at + 1]), pack_bf16(x[at + 2], x[at + 3]), pack_bf16(x[at + 4], x[at + 5]), pack_bf16(x[at + 6], x[at + 7]));
}
// a lane's sixteen elements on their way: bf16 as it lies in memory, half the registers
template <typename T> struct Flying;
template <> struct Flying<float> {
    float v[16];
    __device__ __forceinline__ void fetch(const float* a, const float* b) { load8(a, v, 0); load8(b, v, 8); }
};
template <> struct Flying<__nv_bfloat16> {
    uint4 v[2];
    __device__ __forceinline__ void fetch(const __nv_bfloat16* a, const __nv_bfloat16* b) {
        v[0] = *reinterpret_cast<const uint4*>(a); v[1] = *reinterpret_cast<const uint4*>(b);
    }
    __device__ __forceinline__ void unpack(float (&x)[16]) const {
        load8(reinterpret_cast<const __nv_bfloat16*>(&v[0]), x, 0); load8(reinterpret_cast<const __nv_bfloat16*>(&v[1]), x, 8);
    }
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float& d, float x) { d = x; }
__device__ __forceinline__ void put(__nv_bfloat16& d, float x) { d = __float2bfloat16(x); }

enum RopeMode { NEIGHBOURS, HALVES, STAGED };
constexpr int ROPE_WARPS = ROPE_THREADS / 32, ROPE_TOKENS = 8;        // most tokens of a block

template <typename T, int D, RopeMode MODE>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_kernel(const RopeParams p, int tokens) {
    constexpr int LPR = D / 16, RPW = 32 / LPR;             // lanes of a row, rows of a warp
    __shared__ __align__(16) float2 cs[ROPE_TOKENS][D / 2];
    __shared__ int tok[ROPE_TOKENS][3];                     // sequence, row in the cache (negative: padding), pool row
    __shared__ __align__(16) T stage[MODE == STAGED ? ROPE_WARPS : 1][MODE == STAGED ? RPW : 1][D];
    const int t0 = (int)blockIdx.x * tokens, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nt = min(tokens, p.v.T - t0);
    pdl_wait();
    pdl_release();
    const int r = p.turns ? p.r : 0, half = r / 2;
    const int status0 = *p.v.status;
    if (tid < ROPE_TOKENS) { tok[tid][0] = -1; tok[tid][1] = -1; tok[tid][2] = -1; }
    __syncthreads();
    if (status0 != 0) return;
    const int Hq = p.v.Hq, Hkv = p.v.Hkv, n_rows = Hq + 2 * Hkv, groups = (n_rows + RPW - 1) / RPW;
    const int sub = lane / LPR, q = lane % LPR;
    // the lane's two runs of eight elements: pair i is (x[i], x[8 + i]) (HALVES) or (x[2 i], x[2 i + 1]) of them
    const bool apart = MODE == HALVES && 16 * q < r;
    const int e0 = apart ? 8 * q : 16 * q, e1 = apart ? half + 8 * q : 16 * q + 8;
    struct Row { int i, h; bool have; };                    // token, head (queries, keys, values one after another)
    auto row_of = [&](int k) -> Row {
        Row w;
        w.i = k / groups;
        w.h = (k - w.i * groups) * RPW + sub;
        w.have = w.i < nt && w.h < n_rows;
        return w;
    };
    auto load = [&](const Row& w, Flying<T>& x) {
        if (!w.have) return;
        const size_t t = (size_t)(t0 + w.i);
        const T* src = w.h < Hq ? static_cast<const T*>(p.Q) + t * p.q_stride + (size_t)w.h * D
                     : w.h < Hq + Hkv ? static_cast<const T*>(p.K) + t * p.k_stride + (size_t)(w.h - Hq) * D
                                      : static_cast<const T*>(p.V) + t * p.v_stride + (size_t)(w.h - Hq - Hkv) * D;
        x.fetch(src + e0, src + e1);
    };
    // the first rows are on their way while the tokens' sequences, pages and angles are found
    const int step = ROPE_WARPS * (int)gridDim.y;
    int k = (int)blockIdx.y * ROPE_WARPS + warp;
    constexpr int FLIGHT = sizeof(T) == 2 ? 3 : 2;          // groups of rows in flight
    Row w[FLIGHT];
    Flying<T> v[FLIGHT];
#pragma unroll
    for (int f = 0; f < FLIGHT; ++f) { w[f] = row_of(k + f * step); load(w[f], v[f]); }
    // the sequences that own the tokens
    for (int b = tid; b < p.v.B; b += ROPE_THREADS) {
        const int q0 = p.v.cu ? p.v.cu[b] : b * p.v.max_new, q1 = p.v.cu ? p.v.cu[b + 1] : q0 + p.v.max_new;
        const bool here = q0 < t0 + nt && q1 > t0;
        if (!here && (blockIdx.x != 0 || blockIdx.y != 0)) continue;                    // (the first block looks at every sequence)
        const PagedSeq s = check_seq(p.v, q0, q1, p.v.lens[b]);
        if (!s.valid) report_invalid(p.v.status, kWhereSeq);
        if (!s.valid || !here) continue;
        for (int i = max(0, q0 - t0); i < min(nt, q1 - t0); ++i) {
            const int j = s.L - s.n + (t0 + i - q0);
            tok[i][0] = b; tok[i][1] = j;
            if (j >= 0) tok[i][2] = (int)load_pool_row(p.v, b, j);
        }
    }
    if (p.positions == nullptr) __syncthreads();
    for (int x = tid; x < nt * half; x += ROPE_THREADS) {
        const int i = x / half, k = x - i * half;
        const int pos = p.positions ? p.positions[t0 + i] : tok[i][1];
        double a = (double)pos * p.turns[k];
        a -= rint(a);
        float sn, c;
        sincospif(2.f * (float)a, &sn, &c);
        cs[i][k] = make_float2(c * p.magnitude, sn * p.magnitude);
    }
    __syncthreads();
    auto finish = [&](const Row& w, float (&x)[16]) {
        const bool turn = w.have && w.h < Hq + Hkv;
        if (MODE == STAGED) {
            T* mine = stage[warp][sub];
            __syncwarp();                                   // the rows before have been read
            if (turn) {
#pragma unroll
                for (int i = 0; i < 16; i += 8) {
                    if constexpr (sizeof(T) == 2) store8(mine + e0 + i, x, i);
                    else {
                        *reinterpret_cast<float4*>(mine + e0 + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                        *reinterpret_cast<float4*>(mine + e0 + i + 4) = make_float4(x[i + 4], x[i + 5], x[i + 6], x[i + 7]);
                    }
                }
            }
            __syncwarp();
            const int i = min(w.i, nt - 1);                 // (the rows of a warp belong to one token)
            for (int k = lane; k < half; k += 32) {
                const float2 c = cs[i][k];
#pragma unroll
                for (int y = 0; y < RPW; ++y) {             // rows that are not turned hold what nobody reads
                    const float a = to_f32(stage[warp][y][k]), b = to_f32(stage[warp][y][k + half]);
                    put(stage[warp][y][k], a * c.x - b * c.y);
                    put(stage[warp][y][k + half], b * c.x + a * c.y);
                }
            }
            __syncwarp();
            if (turn) { load8(mine + e0, x, 0); load8(mine + e1, x, 8); }
        } else if (turn && 16 * q < r) {
            const float4* c4 = reinterpret_cast<const float4*>(&cs[w.i][8 * q]);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float4 c = c4[k / 2];                 // of pairs 8 q + k and the next; behind r/2: not used
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float cx = y ? c.z : c.x, sx = y ? c.w : c.y;
                    float& a = MODE == HALVES ? x[k + y] : x[2 * (k + y)];
                    float& b = MODE == HALVES ? x[8 + k + y] : x[2 * (k + y) + 1];
                    const float ya = a * cx - b * sx, yb = b * cx + a * sx;
                    if (MODE == HALVES || 8 * q + k + y < half) { a = ya; b = yb; }
                }
            }
        }
        if (!w.have) return;
        const long long row = tok[w.i][2];
        if (w.h >= Hq && row < 0) return;                   // padding, or no such page
        __nv_bfloat16* dst = w.h < Hq ? p.Q_out + ((size_t)(t0 + w.i) * Hq + w.h) * D
                           : w.h < Hq + Hkv ? p.K_pages + ((size_t)row * Hkv + (w.h - Hq)) * D
                                            : p.V_pages + ((size_t)row * Hkv + (w.h - Hq - Hkv)) * D;
        store8(dst + e0, x, 0);
        store8(dst + e1, x, 8);
    };
    while (true) {
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            if constexpr (sizeof(T) == 2) {
                float x[16];
                v[f].unpack(x);
                finish(w[f], x);
            } else {
                finish(w[f], v[f].v);
            }
        }
        k += FLIGHT * step;
        if (k >= nt * groups) break;
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) { w[f] = row_of(k + f * step); load(w[f], v[f]); }
    }
    if (p.pos_cache != nullptr && blockIdx.y == 0)
        for (int x = tid; x < nt * Hkv; x += ROPE_THREADS) {
            const int i = x % nt, h = x / nt;               // neighbouring tokens are neighbours in the cache
            if (tok[i][2] >= 0)
                p.pos_cache[((size_t)tok[i][0] * Hkv + h) * p.v.cap + tok[i][1]] = p.positions ? p.positions[t0 + i] : tok[i][1];
        }
}

template <typename T, int D>
seka_status launch_rope(const RopeParams& p, cudaStream_t st) {
    int n_sm = 0;
    if (!device_info(&n_sm)) return SEKA_ERR_CUDA;
    const int groups = (p.v.Hq + 2 * p.v.Hkv + 512 / D - 1) / (512 / D);        // of a token's rows: a warp's worth each
    // four tokens a block, in bf16 eight, where that still gives every SM four blocks (16384 tokens of 32/8 heads in bf16: 82 us, 83 with four,
    // 124 with one a block; 3000: 18 with four, 27 with one; some 16000 in fp32 56, 57 with eight); else one, and blocks share a token as far
    // as it has rows
    const long long each = 4LL * n_sm;
    const int tokens = sizeof(T) == 2 && p.v.T >= 8 * each ? 8 : p.v.T >= 4 * each ? 4 : 1;
    int split = 1;
    while (tokens == 1 && split * ROPE_WARPS < groups && (long long)p.v.T * split < 2LL * n_sm) ++split;
    const dim3 grid((unsigned)((p.v.T + tokens - 1) / tokens), (unsigned)split);
    const bool halves = p.turns != nullptr && p.layout == SEKA_ROPE_HALF;
    auto kern = !halves ? rope_append_kernel<T, D, NEIGHBOURS> : p.r % 16 == 0 ? rope_append_kernel<T, D, HALVES> : rope_append_kernel<T, D, STAGED>;
    return launch_kernel(true, kern, grid, ROPE_THREADS, 0, st, p, tokens);
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
    return shape->dtype == SEKA_F32 ? (D == 128 ? launch_rope<float, 128>(p, st) : launch_rope<float, 64>(p, st))
                                    : (D == 128 ? launch_rope<__nv_bfloat16, 128>(p, st) : launch_rope<__nv_bfloat16, 64>(p, st));
}
