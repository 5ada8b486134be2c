// Attention of new tokens over a paged cache: few rows (single tokens, a few tokens of a small group), and the merge of cut units.
//
//   paged_few_kernel      up to 16 rows (new tokens x query heads of a KV head) per unit: bound by HBM, every cached key and value is
//                         read once.  A producer warp streams 64-token stages of K and V through a ring in shared memory, a TMA box
//                         per page piece, its lanes issuing side by side; four consumer warps take 16 tokens of each stage, form
//                         the scores of all rows with mma.sync m16n8k16 (16 rows are too few for a tcgen05 tile), keep
//                         a private online softmax and P V in registers.  The CTA walks its equal share of all stages, unit after
//                         unit, without the ring running dry between them.
//                         64 contexts of 1024 to 4096 tokens, 32/8 heads of 128 (666 MB): 112 to 116 us from device to device, 5.7 to 5.9
//                         TB/s; the floor is 103.
//   paged_merge_kernel    merges the parts of a unit that a share boundary cut: some 3 us of a single sequence's 11, four trips to memory.
// Weights are rounded to bf16 for P V (half a step, 2^-8 of each); scores, sums and outputs stay in fp32 until the store.
#include <math.h>

#include "seka_paged_attn.cuh"

namespace seka {
namespace {

constexpr int FEW_KEYS = 64;                            // cached tokens of a stage
constexpr int FEW_CONSUMERS = 4, FEW_THREADS = (FEW_CONSUMERS + 1) * 32;

template <int D>
struct FewSmem {
    static constexpr int NSTAGE = D == 128 ? 3 : 4;
    static constexpr int CTAS_PER_SM = D == 128 ? 2 : 3;
    static constexpr int TILE_BYTES = FEW_KEYS * D * 2;
    static constexpr int BLOCK_BYTES = FEW_KEYS * 128;              // one [64 tokens x 64 elements] swizzled block
    static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
    static constexpr int MERGE_STRIDE = D + 2;                      // floats of a row: o[D], m, l
    static constexpr int MERGE_OFF = NSTAGE * STAGE_BYTES;          // [4 warps][8 rows]
    static constexpr int BAR_OFF = MERGE_OFF + FEW_CONSUMERS * 8 * MERGE_STRIDE * 4;
    static constexpr int WALK_OFF = BAR_OFF + 2 * NSTAGE * 8;
    static constexpr int BYTES = WALK_OFF + (FEW_CONSUMERS + 1) * 48 + 16;
    static_assert(BAR_OFF % 8 == 0 && WALK_OFF % 16 == 0 && sizeof(ShareScratch<FEW_THREADS>) <= BAR_OFF, "layout");
    static_assert(CTAS_PER_SM * (BYTES + 1024) <= 228 * 1024, "resident CTAs");
};

__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// ... and the same answer for all of them: has any given up?
__device__ __forceinline__ bool consumer_sync_or(bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(x ? 1u : 0u) : "memory");
    return r != 0;
}

// HALF: at most 8 rows, so rows 8..15 of every MMA are padding and their softmax is skipped (8 contexts of 1024 to 4096 tokens, a new token
// each: 23.1 us, 24.9 without; with 64 contexts HBM hides it, 115 and 116).
template <int D, bool HALF>
__global__ void __launch_bounds__(FEW_THREADS, FewSmem<D>::CTAS_PER_SM)
paged_few_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const __grid_constant__ PagedAttnParams p) {
    using SL = FewSmem<D>;
    constexpr int H = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + SL::BAR_OFF);
    uint64_t* empty = full + SL::NSTAGE;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SL::BYTES - 16);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < SL::NSTAGE; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], FEW_CONSUMERS); }
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
    }
    pdl_wait();
    pdl_release();
    const int status0 = *reinterpret_cast<volatile int*>(p.v.status);
    if (__syncthreads_or(status0 != 0)) return;             // an earlier launch gave up on this workspace
    const Share share = find_share<FEW_THREADS>(p.v, p.geo, p.n_shares, (int)blockIdx.x, *reinterpret_cast<ShareScratch<FEW_THREADS>*>(smem));
    if (tid == 0) write_cut(p.cuts, p.v, p.geo, share, (int)blockIdx.x);
    if (share.len == 0) return;
    Walk* walk = reinterpret_cast<Walk*>(smem + SL::WALK_OFF + warp * 48);
    if (lane == 0) walk_begin(p.v, share, *walk);
    __syncwarp();
    auto next = [&](Segment& s) -> bool {
        Walk w = *walk;
        __syncwarp();
        const bool ok = walk_next(p.v, p.geo, w, s);
        if (lane == 0) *walk = w;
        __syncwarp();
        return ok;
    };
    Segment sg = {};

    if (warp == FEW_CONSUMERS) {
        // ------------------------------------------------ producer: a lane per TMA box (K or V, 64 columns, a piece of a page)
        const int bx_shift = p.v.page_shift < 6 ? p.v.page_shift : 6, nb = FEW_KEYS >> bx_shift;
        const int box = lane % nb, blk = (lane / nb) % H, kv = lane / (nb * H);
        const uint32_t dst = (uint32_t)(kv * SL::TILE_BYTES + blk * SL::BLOCK_BYTES + (box << bx_shift) * 128);
        // first token of this lane's box of stage j; the entry of its page (not looked at where the box lies behind the cache)
        auto key_of = [&](int j) -> int { return j * FEW_KEYS + (box << bx_shift); };
        auto entry_of = [&](int j) -> int { return key_of(j) < sg.L ? table_entry(p.v, sg.b, key_of(j)) : 0; };
        int i = 0;
        bool ok = true;
        while (ok && next(sg)) {
            int entry = entry_of(sg.j);
#pragma unroll 1
            for (int t = 0; t < sg.n; ++t, ++i) {
                const int s = i % SL::NSTAGE, round = i / SL::NSTAGE;
                const int entry_next = t + 1 < sg.n ? entry_of(sg.j + t + 1) : 0, key = key_of(sg.j + t);
                if (round > 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], (uint32_t)(round - 1) & 1u, abort_flag, p.v.status, 60));
                    if (!ok) break;
                }
                if (lane == 0) {
                    const int keys = sg.L - (sg.j + t) * FEW_KEYS;
                    const int n_box = keys <= 0 ? 0 : min(nb, (keys + (1 << bx_shift) - 1) >> bx_shift);
                    mbar_expect_tx(&full[s], (uint32_t)(2 * H * n_box * 128) << bx_shift);
                }
                __syncwarp();
                if (key < sg.L && kv < 2) tma_load_3d(smem + s * SL::STAGE_BYTES + dst, kv ? &tv : &tk, &full[s], blk * 64, sg.h, box_row(p.v, entry, key));
                entry = entry_next;
            }
        }
        __syncwarp();
        if (lane == 0 && (!ok || *abort_flag)) {
            // a wait ran out somewhere: let the copies already issued land before the CTA's shared memory is released
            for (int k = i > SL::NSTAGE ? i - SL::NSTAGE : 0; k < i; ++k) {
                const uint64_t t0 = global_timer_ns();
                while (!mbar_try_wait(&full[k % SL::NSTAGE], (uint32_t)(k / SL::NSTAGE) & 1u) && global_timer_ns() - t0 < kWaitLimitNs) { }
            }
        }
        return;
    }

    // ---------------------------------------------------- consumers
    const int G = p.v.G, Hq = p.v.Hq;
    const int r0 = lane >> 2, cq = (lane & 3) * 2;          // accumulator rows r0 and r0 + 8, columns cq, cq + 1
    const int tok0 = r0 / G, tok1 = (r0 + 8) / G;           // new token of these rows
    // ldmatrix source rows of this lane inside the warp's 16 tokens of a stage
    const int key_k = 16 * warp + (lane & 7) + ((lane >> 4) << 3);         // K: matrices 2, 3 hold tokens 8..15
    const int key_v = 16 * warp + (lane & 7) + (((lane >> 3) & 1) << 3);   // V: matrices 1, 3 hold tokens 8..15
    const uint32_t k_row = (uint32_t)key_k * 128u, v_row = (uint32_t)key_v * 128u;
    const uint32_t k_sel = (uint32_t)((lane >> 3) & 1), v_sel = (uint32_t)(lane >> 4);
    const uint32_t smem_base = smem_u32(smem);
    float* mg = reinterpret_cast<float*>(smem + SL::MERGE_OFF);
    int i = 0;
    bool ok = true;
    while (ok && next(sg)) {
        const int rows = sg.n_new * G;
        uint32_t qa[D / 16][4];
        {
            const __nv_bfloat16* q0 = p.Q + ((size_t)(sg.q0 + tok0) * Hq + (size_t)sg.h * G + (r0 - tok0 * G)) * D;
            const __nv_bfloat16* q1 = p.Q + ((size_t)(sg.q0 + tok1) * Hq + (size_t)sg.h * G + (r0 + 8 - tok1 * G)) * D;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const int c = kk * 16 + cq;
                qa[kk][0] = r0 < rows ? *reinterpret_cast<const uint32_t*>(q0 + c) : 0u;
                qa[kk][2] = r0 < rows ? *reinterpret_cast<const uint32_t*>(q0 + c + 8) : 0u;
                qa[kk][1] = !HALF && r0 + 8 < rows ? *reinterpret_cast<const uint32_t*>(q1 + c) : 0u;
                qa[kk][3] = !HALF && r0 + 8 < rows ? *reinterpret_cast<const uint32_t*>(q1 + c + 8) : 0u;
            }
        }
        // last cached token that a row sees (padding rows: the last one)
        const int lim0 = r0 < rows ? sg.old + tok0 : sg.L - 1, lim1 = r0 + 8 < rows ? sg.old + tok1 : sg.L - 1;
        float o[D / 8][4];
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int j = 0; j < D / 8; ++j) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f; }
#pragma unroll 1
        for (int t = 0; t < sg.n; ++t, ++i) {
            const int s = i % SL::NSTAGE;
            ok = __all_sync(0xffffffffu, mbar_wait(&full[s], (uint32_t)(i / SL::NSTAGE) & 1u, abort_flag, p.v.status, 61));
            if (!ok) break;
            const uint32_t kt = smem_base + (uint32_t)(s * SL::STAGE_BYTES), vt = kt + SL::TILE_BYTES;
            // scores of the rows against the warp's 16 tokens: two 16 x 8 tiles
            float sc[2][4];
#pragma unroll
            for (int x = 0; x < 2; ++x) { sc[x][0] = sc[x][1] = sc[x][2] = sc[x][3] = 0.f; }
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t chunk = (uint32_t)((kk & 3) * 2) + k_sel;
                uint32_t b0, b1, b2, b3;
                ldsm_x4(kt + (uint32_t)((kk >> 2) * SL::BLOCK_BYTES) + k_row + (((chunk ^ (uint32_t)key_k) & 7u) << 4), b0, b1, b2, b3);
                mma_16816(sc[0], qa[kk], b0, b1);
                mma_16816(sc[1], qa[kk], b2, b3);
            }
            const int base = (sg.j + t) * FEW_KEYS + 16 * warp;
            if (base + 15 > sg.old) {                       // some row does not see all of the warp's tokens
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (base + 8 * x + cq + (e & 1) > (e < 2 ? lim0 : lim1)) sc[x][e] = -INFINITY;
                if (base + 16 > sg.L) {                     // values behind the cache may be anything, NaN too
                    for (int u = lane; u < 16 * H * 8; u += 32) {
                        const int row = u / (H * 8), c = u % (H * 8);
                        if (base + row >= sg.L)
                            *reinterpret_cast<uint4*>(smem + s * SL::STAGE_BYTES + SL::TILE_BYTES + (c >> 3) * SL::BLOCK_BYTES +
                                                      (16 * warp + row) * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    __syncwarp();
                }
            }
            // online softmax, private to the warp; the row sums stay per thread until the end
            float mx0 = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[1][0], sc[1][1]));
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
            const float mn0 = fmaxf(m0, mx0 * p.scale_log2);
            const float ms0 = mn0 == -INFINITY ? 0.f : mn0;
            const float f0 = fast_exp2(m0 - ms0);
            float mn1 = -INFINITY, ms1 = 0.f, f1 = 1.f;
            if (!HALF) {
                float mx1 = fmaxf(fmaxf(sc[0][2], sc[0][3]), fmaxf(sc[1][2], sc[1][3]));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
                mn1 = fmaxf(m1, mx1 * p.scale_log2);
                ms1 = mn1 == -INFINITY ? 0.f : mn1;
                f1 = fast_exp2(m1 - ms1);
            }
            const bool moved = (mn0 != m0) || (!HALF && mn1 != m1);
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int j = 0; j < D / 8; ++j) {
                    o[j][0] *= f0; o[j][1] *= f0;
                    if (!HALF) { o[j][2] *= f1; o[j][3] *= f1; }
                }
            }
            m0 = mn0; m1 = mn1;
            uint32_t pa[4];
            {
                const float p00 = fast_exp2(fmaf(sc[0][0], p.scale_log2, -ms0)), p01 = fast_exp2(fmaf(sc[0][1], p.scale_log2, -ms0));
                const float p10 = fast_exp2(fmaf(sc[1][0], p.scale_log2, -ms0)), p11 = fast_exp2(fmaf(sc[1][1], p.scale_log2, -ms0));
                l0 = fmaf(l0, f0, (p00 + p01) + (p10 + p11));
                pa[0] = pack_bf16(p00, p01); pa[2] = pack_bf16(p10, p11);
                if (!HALF) {
                    const float q00 = fast_exp2(fmaf(sc[0][2], p.scale_log2, -ms1)), q01 = fast_exp2(fmaf(sc[0][3], p.scale_log2, -ms1));
                    const float q10 = fast_exp2(fmaf(sc[1][2], p.scale_log2, -ms1)), q11 = fast_exp2(fmaf(sc[1][3], p.scale_log2, -ms1));
                    l1 = fmaf(l1, f1, (q00 + q01) + (q10 + q11));
                    pa[1] = pack_bf16(q00, q01); pa[3] = pack_bf16(q10, q11);
                } else {
                    pa[1] = 0u; pa[3] = 0u;
                }
            }
            // o[16 x D] += P[16 x 16 tokens] V[16 tokens x D]
#pragma unroll
            for (int jp = 0; jp < D / 16; ++jp) {
                const uint32_t chunk = (uint32_t)((jp & 3) * 2) + v_sel;
                uint32_t b0, b1, b2, b3;
                ldsm_x4_trans(vt + (uint32_t)((jp >> 2) * SL::BLOCK_BYTES) + v_row + (((chunk ^ (uint32_t)key_v) & 7u) << 4), b0, b1, b2, b3);
                mma_16816(o[2 * jp], pa, b0, b1);
                mma_16816(o[2 * jp + 1], pa, b2, b3);
            }
            fence_proxy_async();            // the reads (and zeros) of this stage come before the copies that refill it
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[s]);
        }
        // ------------------------------------------------ merge the four warps' states, eight rows at a time
        l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
        if (!HALF) {
            l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
        }
        const size_t slot = (size_t)blockIdx.x * 2 + (sg.first ? 0 : 1);
#pragma unroll
        for (int half = 0; half < (HALF ? 1 : 2); ++half) {
            if (half * 8 >= rows) break;
            ok = !consumer_sync_or(!ok || *abort_flag != 0);        // the area is free (its last readers are through)
            if (!ok) break;
            float* row = mg + ((size_t)warp * 8 + r0) * SL::MERGE_STRIDE;
#pragma unroll
            for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(row + 8 * j + cq) = half ? make_float2(o[j][2], o[j][3]) : make_float2(o[j][0], o[j][1]);
            if ((lane & 3) == 0) { row[D] = half ? m1 : m0; row[D + 1] = half ? l1 : l0; }
            consumer_sync();
            const int n = min(8, rows - half * 8);
            for (int idx = tid; idx < n * D; idx += FEW_CONSUMERS * 32) {
                const int r = idx / D, c = idx - r * D, ur = half * 8 + r;
                float mw[FEW_CONSUMERS], M = -INFINITY;
#pragma unroll
                for (int w = 0; w < FEW_CONSUMERS; ++w) { mw[w] = mg[((size_t)w * 8 + r) * SL::MERGE_STRIDE + D]; M = fmaxf(M, mw[w]); }
                float acc = 0.f, lsum = 0.f;
#pragma unroll
                for (int w = 0; w < FEW_CONSUMERS; ++w) {
                    const float f = mw[w] == -INFINITY ? 0.f : fast_exp2(mw[w] - M);
                    acc = fmaf(mg[((size_t)w * 8 + r) * SL::MERGE_STRIDE + c], f, acc);
                    lsum = fmaf(mg[((size_t)w * 8 + r) * SL::MERGE_STRIDE + D + 1], f, lsum);
                }
                if (sg.whole) {
                    const int tok = ur / G;
                    const size_t out = (size_t)(sg.q0 + tok) * Hq + (size_t)sg.h * G + (ur - tok * G);
                    p.O[out * D + c] = __float2bfloat16(lsum == 0.f ? 0.f : acc / lsum);
                    if (p.lse != nullptr && c == 0) p.lse[out] = lsum == 0.f ? -INFINITY : (M + log2f(lsum)) * 0.6931471805599453f;
                } else {
                    p.part_o[(slot * kFewRows + ur) * D + c] = acc;
                    if (c == 0) *reinterpret_cast<float2*>(p.part_ml + (slot * kFewRows + ur) * 2) = make_float2(M, lsum);
                }
            }
        }
    }
}

// Blocks of 8 warps for every cut: nothing to do where the share begins with a unit, or where an earlier cut of the same unit does it.
// The chain from the cut's record to the parts is four trips to memory long, so rows are merged a few at a time.
//   SPREAD false  units of a few parts: a block takes 32 rows, a warp four of them;
//   SPREAD true   units of many parts (a long context on few heads): a block takes two rows and each warp an eighth of the
//                 parts; the warps' sums are added in shared memory, in the order of the warps (four rows: 1 us more).
constexpr int MERGE_WARPS = 8;
constexpr int merge_rows(bool spread) { return spread ? 2 : 4; }                 // of a warp at a time
constexpr int merge_block_rows(bool spread) { return merge_rows(spread) * (spread ? 1 : MERGE_WARPS); }
template <int D, bool SPREAD>
__global__ void __launch_bounds__(MERGE_WARPS * 32) paged_merge_kernel(const __grid_constant__ PagedAttnParams p, int unit_rows, int live_rows) {
    constexpr int E = D / 32, ROWS = merge_rows(SPREAD);
    __shared__ __align__(16) float sums[SPREAD ? MERGE_WARPS : 1][ROWS][D];
    const int blocks = (live_rows + merge_block_rows(SPREAD) - 1) / merge_block_rows(SPREAD), cut = (int)blockIdx.x / blocks;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r0 = ((int)blockIdx.x - cut * blocks) * merge_block_rows(SPREAD) + (SPREAD ? 0 : warp * ROWS);
    pdl_wait();
    pdl_release();
    const int status0 = *p.v.status;
    const CutRecord c = p.cuts[cut];
    if (status0 != 0 || r0 >= live_rows || c.n == 0 || c.j == 0 || c.j > c.share) return;
    const PagedSeq s = paged_seq(p.v, c.b);
    // parts: the last segment of share cut - 1, then the first ones of the shares on
    const int parts = 1 + (c.n - c.j + c.share - 1) / c.share;
    auto slot = [&](int i) -> size_t { return i == 0 ? (size_t)(cut - 1) * 2 + (c.j < c.share ? 1 : 0) : (size_t)(cut - 1 + i) * 2; };
    size_t out[ROWS];
    bool real[ROWS];
    bool any = false;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {              // row -> new token and query head
        const int r = r0 + q, tile = r >> 7, rt = r & 127, t_tile = rt / p.v.G, tok = c.p * p.geo.tp + tile * p.tile_tokens + t_tile;
        real[q] = t_tile < p.tile_tokens && tok < s.n;
        out[q] = (size_t)(s.q0 + tok) * p.v.Hq + (size_t)c.h * p.v.G + (rt - t_tile * p.v.G);
        any |= real[q];
    }
    if (!any) return;                                       // (SPREAD: the same for the whole block)
    float M[ROWS], l[ROWS], acc[ROWS][E];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        M[q] = -INFINITY; l[q] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[q][e] = 0.f;
    }
    for (int i0 = 0; i0 < parts; i0 += 32) {
        const int n = min(32, parts - i0);
        float2 ml[ROWS];
        float f[ROWS];
#pragma unroll
        for (int q = 0; q < ROWS; ++q)
            ml[q] = lane < n ? *reinterpret_cast<const float2*>(p.part_ml + (slot(i0 + lane) * unit_rows + r0 + q) * 2) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            float mx = fmaxf(M[q], ml[q].x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float keep = M[q] == -INFINITY ? 0.f : fast_exp2(M[q] - mx);
            f[q] = ml[q].x == -INFINITY ? 0.f : fast_exp2(ml[q].x - mx);
            l[q] = fmaf(l[q], keep, ml[q].y * f[q]);    // per lane until the end
            M[q] = mx;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[q][e] *= keep;
        }
#pragma unroll 2
        for (int i = SPREAD ? warp : 0; i < n; i += SPREAD ? MERGE_WARPS : 1) {
            const float* src = p.part_o + (slot(i0 + i) * unit_rows + r0) * D + lane * E;
            float x[ROWS][E];
#pragma unroll
            for (int q = 0; q < ROWS; ++q) {
                if (E == 4) *reinterpret_cast<float4*>(x[q]) = *reinterpret_cast<const float4*>(src + q * D);
                else *reinterpret_cast<float2*>(x[q]) = *reinterpret_cast<const float2*>(src + q * D);
            }
#pragma unroll
            for (int q = 0; q < ROWS; ++q) {
                const float fi = __shfl_sync(0xffffffffu, f[q], i);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[q][e] = fmaf(x[q][e], fi, acc[q][e]);
            }
        }
    }
    if (SPREAD) {
#pragma unroll
        for (int q = 0; q < ROWS; ++q)
#pragma unroll
            for (int e = 0; e < E; ++e) sums[warp][q][lane * E + e] = acc[q][e];
        __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l[q] += __shfl_xor_sync(0xffffffffu, l[q], o);
        if (!real[q] || (SPREAD && warp != q)) continue;
        if (SPREAD) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                acc[q][e] = 0.f;
#pragma unroll
                for (int w = 0; w < MERGE_WARPS; ++w) acc[q][e] += sums[w][q][lane * E + e];
            }
        }
        const float inv = l[q] == 0.f ? 0.f : 1.f / l[q];
        uint32_t* dst = reinterpret_cast<uint32_t*>(p.O + out[q] * D + lane * E);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) dst[e] = pack_bf16(acc[q][2 * e] * inv, acc[q][2 * e + 1] * inv);
        if (p.lse != nullptr && lane == 0) p.lse[out[q]] = l[q] == 0.f ? -INFINITY : (M[q] + log2f(l[q])) * 0.6931471805599453f;
    }
}

template <int D, bool HALF>
seka_status launch_few(const CUtensorMap& tk, const CUtensorMap& tv, const PagedAttnParams& p, unsigned grid, cudaStream_t st) {
    using SL = FewSmem<D>;
    if (cudaFuncSetAttribute(paged_few_kernel<D, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, SL::BYTES) != cudaSuccess) return SEKA_ERR_CUDA;
    return launch_kernel(true, paged_few_kernel<D, HALF>, grid, FEW_THREADS, SL::BYTES, st, tk, tv, p);
}

}  // namespace
}  // namespace seka

extern "C" seka_status seka_paged_attention(const seka_paged_shape* shape, const void* Q, const void* K_pages, const void* V_pages,
                                            void* O, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    using namespace seka;
    seka_status stc = validate_paged(shape);
    if (stc != SEKA_OK) return stc;
    if (shape->batch == 0 || shape->total_new == 0 || shape->max_new == 0) return SEKA_OK;      // no sequence owns a token
    if (!Q || !O || !K_pages || !V_pages) return SEKA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K_pages | (uintptr_t)V_pages | (uintptr_t)O) & 15) return SEKA_ERR_INVALID_ARG;
    stc = check_paged_call(shape, workspace, workspace_bytes);
    if (stc != SEKA_OK) return stc;
    const PagedLayout w = paged_layout(shape);
    char* ws = static_cast<char*>(workspace);
    const int D = shape->head_dim, G = shape->n_q_heads / shape->n_kv_heads;
    const bool few = few_rows(shape);
    PagedAttnParams p;
    p.v = paged_view(shape, workspace);
    p.Q = static_cast<const __nv_bfloat16*>(Q); p.O = static_cast<__nv_bfloat16*>(O); p.lse = lse;
    const float scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.f / sqrtf((float)D);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.tile_tokens = few ? shape->max_new : 128 / G;
    // one tile of rows at most per sequence and KV head: units of one tile (SHARED tile kernel), else of two.  64 contexts of 2048 on 16 heads
    // of 64, 17 / 128 new tokens each: 178 / 184 us in units of two, 158 / 165 in units of one; 256 new tokens 253 / 297.  On 32/8 heads of
    // 128, 32 new tokens 134 / 123.
    p.geo.tp = few ? shape->max_new : shape->max_new <= p.tile_tokens ? p.tile_tokens : 2 * p.tile_tokens;
    p.geo.shift = few ? 6 : 7;
    // A share is worth a CTA of its own from two stages of 64 tokens on (one sequence of 128 / 777 / 2048 / 4096 tokens, 8 KV heads, in a graph: 7.8 /
    // 10.5 / 9.8 / 11.9 us; from four on 10.7 / 11.7 / 10.2 / 11.8), a share of tiles from four on (32 new tokens over 4096: 20.7 us, from two
    // on 22.5; over 1024 17.2 and 16.3).
    p.geo.min_share = few ? 2 : 4;
    p.geo.max_units = (shape->max_new + p.geo.tp - 1) / p.geo.tp;
    // shares that can have a step, from what the host knows
    const long long units = few ? shape->batch : (long long)shape->total_new / p.geo.tp + shape->batch;
    const long long steps = units * shape->n_kv_heads * ((p.v.cap + (1 << p.geo.shift) - 1) >> p.geo.shift);
    long long shares = (steps + p.geo.min_share - 1) / p.geo.min_share;
    if (shares > attention_shares(shape)) shares = attention_shares(shape);
    p.n_shares = (int)shares;
    p.cuts = reinterpret_cast<CutRecord*>(ws + w.cut_off);
    p.part_ml = reinterpret_cast<float*>(ws + w.part_ml_off);
    p.part_o = reinterpret_cast<float*>(ws + w.part_o_off);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (few) {
        const int box = shape->page_size < FEW_KEYS ? shape->page_size : FEW_KEYS;
        const long long rows = (long long)shape->n_pages * shape->page_size;
        CUtensorMap tk, tv;
        if (!make_tile_map(&tk, K_pages, D, shape->n_kv_heads, rows, box, 1, D == 64) ||
            !make_tile_map(&tv, V_pages, D, shape->n_kv_heads, rows, box, 1, D == 64)) return SEKA_ERR_CUDA;
        const bool half = shape->max_new * G <= 8;
        const unsigned grid = (unsigned)p.n_shares;
        stc = D == 128 ? (half ? launch_few<128, true>(tk, tv, p, grid, st) : launch_few<128, false>(tk, tv, p, grid, st))
                       : (half ? launch_few<64, true>(tk, tv, p, grid, st) : launch_few<64, false>(tk, tv, p, grid, st));
    } else {
        stc = D == 128 ? launch_paged_tiles<128>(p, Q, K_pages, V_pages, shape->page_size, st)
                       : launch_paged_tiles<64>(p, Q, K_pages, V_pages, shape->page_size, st);
    }
    if (stc != SEKA_OK || p.n_shares == 1) return stc;
    // Few rows and, from what the host knows, about two parts of a unit or more: spread over the warps.  One sequence of 777 / 4096 /
    // 65536 tokens on 8 KV heads, a new one: 12.9 / 20.2 / 62.1 us with a warp per four rows, 10.5 / 11.9 / 52.3 so; tiles
    // of rows have warps enough (128 rows over 8192 tokens, two sequences: 37.5 us, spread 51.7).
    const bool spread = few && p.n_shares >= 2 * units * shape->n_kv_heads;
    const int rows = unit_rows(shape), live = shape->max_new <= p.tile_tokens ? shape->max_new * G : rows;      // rows that can be real
    const unsigned grid = (unsigned)(p.n_shares * ((live + merge_block_rows(spread) - 1) / merge_block_rows(spread)));
    auto merge = D == 128 ? (spread ? paged_merge_kernel<128, true> : paged_merge_kernel<128, false>)
                          : (spread ? paged_merge_kernel<64, true> : paged_merge_kernel<64, false>);
    return launch_kernel(true, merge, grid, MERGE_WARPS * 32, 0, st, p, rows, live);
}
