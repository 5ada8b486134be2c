// Attention weight that the rows of a paged cache receive from new tokens, accumulated: for every cached token the sum over the queries
// that see it of exp(q.k scale - lse), queries of all heads of its group.
//
// The score tile is formed with the KEYS as its rows, so that the sum over queries runs along a thread's own row: no reduction
// between threads, no atomics, a fixed order.  K is read once, V not at all.
//   mass_few_kernel       up to 16 query rows: bound by HBM.  A producer warp streams 64-token stages of K (TMA, a box per piece of a
//                         page); four consumer warps take 16 tokens each, mma.sync m16n8k16 with K as A and the queries as B.  64 contexts of
//                         1024 to 4096 tokens, 32/8 heads of 128 (343 MB): 64 us, 5.3 TB/s; the floor is 53.
//   mass_tile_kernel      more rows, on tcgen05: 2 x 128 cached tokens stay in shared memory, tiles of 128 query rows (new token r / G,
//                         head r % G) pass by.  Bound by the exponentials (one per score, against 2 d flops).
//                         2 x 1024 tokens over 6000 to 8192, 32/8 heads of 128: 169 us; all exponentials at the rate of the special-function
//                         unit would take 105 (a quarter of them run on the multiply-add pipe instead; the unit is 59 % busy).  Two summing
//                         warps a scheduler, each a chain of multiply-add, exponential and sum, mostly wait for their own results.
//   mass_merge_kernel     adds the parts of a unit that a share boundary cut.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged_sched.cuh"

namespace seka {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct MassParams {
    PagedView v;
    const __nv_bfloat16* Q;
    const float *lse, *mass_in;
    float* mass_out;
    float scale_log2;
    int n_shares;
    KeyGeo key;
    RowGeo rowg;
    CutRecord* cuts;
    float* part;                // [n_shares, 2, 256]
};

__device__ __forceinline__ float mass_before(const MassParams& p, size_t at, int j, int old) { return p.mass_in != nullptr && j < old ? p.mass_in[at] : 0.f; }

// ---------------------------------------------------------------- few rows
constexpr int MF_KEYS = 64, MF_CONSUMERS = 4, MF_THREADS = (MF_CONSUMERS + 1) * 32;

template <int D>
struct MfSmem {
    static constexpr int NSTAGE = D == 128 ? 6 : 8, CTAS_PER_SM = D == 128 ? 2 : 3;
    static constexpr int STAGE_BYTES = MF_KEYS * D * 2, BLOCK_BYTES = MF_KEYS * 128;
    static constexpr int BAR_OFF = NSTAGE * STAGE_BYTES, WALK_OFF = BAR_OFF + 2 * NSTAGE * 8;
    static constexpr int BYTES = WALK_OFF + (MF_CONSUMERS + 1) * 48 + 16;
    static_assert(sizeof(ShareScratch<MF_THREADS>) <= BAR_OFF, "layout");
    static_assert(CTAS_PER_SM * (BYTES + 1024) <= 228 * 1024, "resident CTAs");
};

template <int D, bool HALF>
__global__ void __launch_bounds__(MF_THREADS, MfSmem<D>::CTAS_PER_SM)
mass_few_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ MassParams p) {
    using SL = MfSmem<D>;
    constexpr int H = D / 64, NB = HALF ? 1 : 2;            // query rows in groups of eight
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + SL::BAR_OFF);
    uint64_t* empty = full + SL::NSTAGE;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SL::BYTES - 16);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < SL::NSTAGE; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], MF_CONSUMERS); }
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tk);
    }
    pdl_wait();
    pdl_release();
    const int status0 = *reinterpret_cast<volatile int*>(p.v.status);
    if (__syncthreads_or(status0 != 0)) return;
    const Share share = find_share<MF_THREADS>(p.v, p.key, p.n_shares, (int)blockIdx.x, *reinterpret_cast<ShareScratch<MF_THREADS>*>(smem));
    if (share.len == 0) return;
    Walk* walk = reinterpret_cast<Walk*>(smem + SL::WALK_OFF + warp * 48);
    if (lane == 0) walk_begin(p.v, share, *walk);
    __syncwarp();
    auto next = [&](Segment& s) -> bool {
        Walk w = *walk;
        __syncwarp();
        const bool ok = walk_next(p.v, p.key, w, s);
        if (lane == 0) *walk = w;
        __syncwarp();
        return ok;
    };
    Segment sg = {};
    int i = 0;
    bool ok = true;

    if (warp == MF_CONSUMERS) {
        // ------------------------------------------------ producer: a lane per TMA box (64 columns, a piece of a page)
        const int bx_shift = p.v.page_shift < 6 ? p.v.page_shift : 6, nb = MF_KEYS >> bx_shift;
        const int box = lane % nb, blk = lane / nb;         // blk >= H: idle
        const uint32_t dst = (uint32_t)(blk * SL::BLOCK_BYTES + (box << bx_shift) * 128);
        // first token of this lane's box of stage j; the entry of its page (not looked at where the box lies behind the cache)
        auto key_of = [&](int j) -> int { return j * MF_KEYS + (box << bx_shift); };
        auto entry_of = [&](int j) -> int { return key_of(j) < sg.L ? table_entry(p.v, sg.b, key_of(j)) : 0; };
        while (ok && next(sg)) {
            int entry = entry_of(sg.j);
#pragma unroll 1
            for (int t = 0; t < sg.n; ++t, ++i) {
                const int s = i % SL::NSTAGE, round = i / SL::NSTAGE;
                const int entry_next = t + 1 < sg.n ? entry_of(sg.j + t + 1) : 0, key = key_of(sg.j + t);
                if (round > 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], (uint32_t)(round - 1) & 1u, abort_flag, p.v.status, 62));
                    if (!ok) break;
                }
                if (lane == 0) {
                    const int keys = sg.L - (sg.j + t) * MF_KEYS;          // at least one
                    mbar_expect_tx(&full[s], (uint32_t)(H * min(nb, (keys + (1 << bx_shift) - 1) >> bx_shift) * 128) << bx_shift);
                }
                __syncwarp();
                if (key < sg.L && blk < H) tma_load_3d(smem + s * SL::STAGE_BYTES + dst, &tk, &full[s], blk * 64, sg.h, box_row(p.v, entry, key));
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
    const int r0 = lane >> 2, cq = (lane & 3) * 2;          // accumulator rows (tokens) r0, r0 + 8; columns (query rows) cq, cq + 1
    const int key_k = 16 * warp + (lane & 7) + (((lane >> 3) & 1) << 3);   // ldmatrix row of this lane (matrices 1, 3: tokens 8..15)
    const uint32_t k_row = (uint32_t)key_k * 128u, k_sel = (uint32_t)(lane >> 4);
    const uint32_t smem_base = smem_u32(smem);
    while (ok && next(sg)) {
        const int rows = sg.n_new * G;
        uint32_t qb[NB][D / 16][2];
        float lse2[NB][2];
        int lim[NB][2];
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            const int r = r0 + 8 * x, tok = r / G;          // B fragment: this lane holds query row r
            const __nv_bfloat16* q = p.Q + ((size_t)(sg.q0 + tok) * Hq + (size_t)sg.h * G + (r - tok * G)) * D + cq;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                qb[x][kk][0] = r < rows ? *reinterpret_cast<const uint32_t*>(q + kk * 16) : 0u;
                qb[x][kk][1] = r < rows ? *reinterpret_cast<const uint32_t*>(q + kk * 16 + 8) : 0u;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = 8 * x + cq + e, tc = c / G;
                lse2[x][e] = c < rows ? p.lse[(size_t)(sg.q0 + tc) * Hq + (size_t)sg.h * G + (c - tc * G)] * kLog2e : 0.f;
                lim[x][e] = c < rows ? sg.old + tc : -1;    // last cached token that the row sees
            }
        }
        const size_t at0 = ((size_t)sg.b * p.v.Hkv + sg.h) * p.v.cap;
#pragma unroll 1
        for (int t = 0; t < sg.n; ++t, ++i) {
            const int s = i % SL::NSTAGE;
            // this lane stores token r0 (even lanes of its four) or r0 + 8
            const int j0 = (sg.j + t) * MF_KEYS + 16 * warp, mine = j0 + r0 + ((lane & 1) << 3);
            const bool store = (lane & 2) == 0 && mine < sg.L;
            const float before = store ? mass_before(p, at0 + mine, mine, sg.old) : 0.f;
            ok = __all_sync(0xffffffffu, mbar_wait(&full[s], (uint32_t)(i / SL::NSTAGE) & 1u, abort_flag, p.v.status, 63));
            if (!ok) break;
            const uint32_t kt = smem_base + (uint32_t)(s * SL::STAGE_BYTES);
            float sc[NB][4];
#pragma unroll
            for (int x = 0; x < NB; ++x) { sc[x][0] = sc[x][1] = sc[x][2] = sc[x][3] = 0.f; }
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t chunk = (uint32_t)((kk & 3) * 2) + k_sel;
                uint32_t a[4];
                ldsm_x4(kt + (uint32_t)((kk >> 2) * SL::BLOCK_BYTES) + k_row + (((chunk ^ (uint32_t)key_k) & 7u) << 4), a[0], a[1], a[2], a[3]);
#pragma unroll
                for (int x = 0; x < NB; ++x) mma_16816(sc[x], a, qb[x][kk][0], qb[x][kk][1]);
            }
            fence_proxy_async();            // the reads of this stage come before the copies that refill it
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[s]);
            float lo = 0.f, hi = 0.f;       // tokens r0 and r0 + 8
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    lo += j0 + r0 <= lim[x][e] ? fast_exp2(fmaf(sc[x][e], p.scale_log2, -lse2[x][e])) : 0.f;
                    hi += j0 + r0 + 8 <= lim[x][e] ? fast_exp2(fmaf(sc[x][2 + e], p.scale_log2, -lse2[x][e])) : 0.f;
                }
            lo += __shfl_xor_sync(0xffffffffu, lo, 1); hi += __shfl_xor_sync(0xffffffffu, hi, 1);
            lo += __shfl_xor_sync(0xffffffffu, lo, 2); hi += __shfl_xor_sync(0xffffffffu, hi, 2);
            if (store) p.mass_out[at0 + mine] = before + ((lane & 1) ? hi : lo);
        }
    }
}

// ---------------------------------------------------------------- many rows
constexpr int MT_THREADS = 384;
constexpr uint32_t BLK_BYTES = 128 * 128;
constexpr int MT_REGS_CTRL = 104, MT_REGS_SUM = 200;
constexpr int MT_POLY8 = 2;             // of eight pairs of exponentials, how many run on the multiply-add pipe

template <int D>
struct MtGeo {
    static constexpr int NQ = D == 128 ? 3 : 4;             // ring of query tiles
    static constexpr uint32_t TILE = (D / 64) * BLK_BYTES;
    static constexpr uint32_t Q_OFF = 4 * TILE;             // keys: two units of two tiles
    static constexpr uint32_t L_OFF = Q_OFF + NQ * TILE;    // lse (base 2) of the rows of each query tile
    static constexpr uint32_t BAR_OFF = L_OFF + NQ * 512;
    // mbarriers, by first index
    static constexpr uint32_t K_FULL = 0, K_FREE = K_FULL + 2, Q_FULL = K_FREE + 2, Q_FREE = Q_FULL + NQ, L_FREE = Q_FREE + NQ,
                              S_FULL = L_FREE + NQ, S_FREE = S_FULL + 4, DRAIN = S_FREE + 4, NBARS = DRAIN + 1;
    static constexpr uint32_t MISC_OFF = BAR_OFF + NBARS * 8, WALK_OFF = (MISC_OFF + 8 + 15) & ~15u;
    static constexpr uint32_t BYTES = WALK_OFF + 12 * 48;
    static_assert(sizeof(ShareScratch<MT_THREADS>) <= 4 * TILE, "layout");
    static_assert(BYTES <= 227 * 1024, "shared memory");
};

template <int D>
__global__ void __launch_bounds__(MT_THREADS, 1)
mass_tile_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ MassParams p) {
    using G = MtGeo<D>;
    constexpr int NQ = G::NQ, NBLK = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + G::BAR_OFF);
    uint64_t* k_full = bars + G::K_FULL;    // [2]      both key tiles of a unit landed
    uint64_t* k_free = bars + G::K_FREE;          // [2]      the tensor core is done with them
    uint64_t* q_full = bars + G::Q_FULL;          // [NQ]     query tile landed
    uint64_t* q_free = bars + G::Q_FREE;         // [NQ]
    uint64_t* l_free = bars + G::L_FREE;         // [NQ]     8 summing warps have read the lse of its rows
    uint64_t* s_full = bars + G::S_FULL;         // [2 x 2]  scores of key tile x, buffer s & 1 (the product and the lse of its rows: two arrivals)
    uint64_t* s_free = bars + G::S_FREE;          // [2 x 2]  4 summing warps have them in registers
    uint64_t* drain = bars + G::DRAIN;           // [1]      every product issued has finished
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + G::MISC_OFF);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + G::MISC_OFF + 4);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int Gq = p.v.G, TP = p.rowg.tp;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(k_full + i, 1); mbar_init(k_free + i, 1); }
        for (int i = 0; i < NQ; ++i) { mbar_init(q_full + i, 1); mbar_init(q_free + i, 1); mbar_init(l_free + i, 8); }
        for (int i = 0; i < 4; ++i) { mbar_init(s_full + i, 2); mbar_init(s_free + i, 4); }
        mbar_init(drain, 1);
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tmQ); tma_prefetch_desc(&tmK);
    }
    // rows of a query tile that no head fills (a group size that does not divide 128): zeros, so that their scores are finite
    for (int u = TP * Gq * 8 + tid; u < 128 * 8; u += MT_THREADS)
        for (int b = 0; b < NQ * NBLK; ++b) *reinterpret_cast<uint4*>(smem + G::Q_OFF + b * BLK_BYTES + u * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
    pdl_wait();
    const int status0 = *reinterpret_cast<volatile int*>(p.v.status);
    if (__syncthreads_or(status0 != 0)) return;
    const Share share = find_share<MT_THREADS>(p.v, p.rowg, p.n_shares, (int)blockIdx.x, *reinterpret_cast<ShareScratch<MT_THREADS>*>(smem));
    if (tid == 0) write_cut(p.cuts, p.v, p.rowg, share, (int)blockIdx.x);
    if (share.len == 0) return;
    if (warp == 0) { tmem_alloc(tmem_holder, 512); tmem_relinquish(); }
    Walk* walk = reinterpret_cast<Walk*>(smem + G::WALK_OFF + warp * 48);
    if (lane == 0) walk_begin(p.v, share, *walk);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, int where) -> bool {
        const bool ok = mbar_wait_limit(bar, parity, abort_flag, p.v.status, where, kWaitLimitNs, 1);
        return __all_sync(0xffffffffu, ok);
    };
    auto next = [&](Segment& s) -> bool {
        Walk w = *walk;
        __syncwarp();
        const bool ok = walk_next(p.v, p.rowg, w, s);
        if (lane == 0) *walk = w;
        __syncwarp();
        return ok;
    };
    Segment it;
    bool ok = true;
    uint32_t s = 0, u = 0;                  // steps and units so far, the same in every role

    if (warp < 4) {
        reg_dec<MT_REGS_CTRL>();
        const bool leader = elect_one();
        if (warp == 0) {
            // ------------------------------------------------------------ TMA producer
            const int bx_shift = p.v.page_shift < 7 ? p.v.page_shift : 7, nb = 256 >> bx_shift;     // boxes of a unit's 256 tokens
            const int box = lane % nb, blk = lane / nb;     // blk >= NBLK: idle
            const int key_in = box << bx_shift;
            const uint32_t dst = (uint32_t)(key_in >> 7) * G::TILE + (uint32_t)blk * BLK_BYTES + (uint32_t)((key_in & 127) * 128);
            const uint32_t q_bytes = (uint32_t)(TP * Gq) * 128u * NBLK;
            auto load_k = [&](const Segment& w, uint32_t n_u) {
                const int key = w.p * 256 + key_in, keys = w.L - w.p * 256;     // at least one
                const int entry = key < w.L ? table_entry(p.v, w.b, key) : 0;
                if (n_u >= 2) { ok = warp_wait(k_free + (n_u & 1), ((n_u >> 1) - 1) & 1, 70); if (!ok) return; }
                if (leader) mbar_expect_tx(k_full + (n_u & 1), (uint32_t)(min(nb, (keys + (1 << bx_shift) - 1) >> bx_shift) * 128 * NBLK) << bx_shift);
                __syncwarp();
                if (key < w.L && blk < NBLK) tma_load_3d(smem + (n_u & 1) * 2 * G::TILE + dst, &tmK, k_full + (n_u & 1), blk * 64, w.h, box_row(p.v, entry, key));
                __syncwarp();
            };
            uint32_t loaded_k = 0;          // units whose keys have been asked for
            bool have = next(it);
            load_k(it, 0); loaded_k = 1;
            while (ok && have) {
                Segment nx;
                const bool more = next(nx);
                const int t0 = p.rowg.first(it.L, it.n_new, it.p) + it.j;
#pragma unroll 1
                for (int j = 0; j < it.n; ++j, ++s) {
                    if (s >= NQ) { ok = warp_wait(q_free + s % NQ, (s / NQ - 1) & 1, 71); if (!ok) break; }
                    if (leader) {
                        uint64_t* bar = q_full + s % NQ;
                        mbar_expect_tx(bar, q_bytes);
#pragma unroll
                        for (int c = 0; c < NBLK; ++c)
                            tma_load_3d(smem + G::Q_OFF + (s % NQ) * G::TILE + c * BLK_BYTES, &tmQ, bar, c * 64, it.h * Gq, it.q0 + (t0 + j) * TP);
                    }
                    __syncwarp();
                    if (j == 0 && more) { load_k(nx, u + 1); if (!ok) break; loaded_k = u + 2; }
                }
                if (!ok) break;
                ++u;
                it = nx; have = more;
            }
            if (*abort_flag) {
                // loads that were armed may still be in flight: let them land before the shared memory is released
                auto settle = [&](uint64_t* bar, uint32_t n, uint32_t ring) {           // the last load of each stage
                    for (uint32_t k = n > ring ? n - ring : 0; k < n; ++k) mbar_wait_limit(bar + k % ring, (k / ring) & 1, nullptr, nullptr, 0, kWaitLimitNs);
                };
                settle(k_full, loaded_k, 2); settle(q_full, s, NQ);
            }
        } else if (warp == 1) {
            // ------------------------------------------------------------ MMA issuer
            constexpr uint32_t IDESC = umma_idesc_bf16(128, false), DESC_HI = umma_desc_hi_sw128(1024);
            const uint32_t dK = umma_desc_lo(smem_u32(smem), 16), dQ = umma_desc_lo(smem_u32(smem + G::Q_OFF), 16);
            while (ok && next(it)) {
                ok = warp_wait(k_full + (u & 1), (u >> 1) & 1, 72);
                if (!ok) break;
#pragma unroll 1
                for (int j = 0; j < it.n; ++j, ++s) {
                    ok = warp_wait(q_full + s % NQ, (s / NQ) & 1, 73);
                    if (!ok) break;
                    const uint32_t qd = dQ + (s % NQ) * (G::TILE >> 4);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t buf = 2 * x + (s & 1);
                        if (s >= 2) { ok = warp_wait(s_free + buf, ((s >> 1) - 1) & 1, 74); if (!ok) break; }
                        const uint32_t kd = dK + ((u & 1) * 2 + x) * (G::TILE >> 4);
                        tc_fence_after();
                        if (leader) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks) {
                                const uint32_t off = ((uint32_t)(ks >> 2) * BLK_BYTES + (uint32_t)(ks & 3) * 32) >> 4;
                                umma_ss(tmem_base + buf * 128, kd + off, DESC_HI, qd + off, DESC_HI, IDESC, ks > 0 ? 1u : 0u);
                            }
                            umma_commit(s_full + buf);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (leader) umma_commit(q_free + s % NQ);
                    __syncwarp();
                }
                if (!ok) break;
                if (leader) umma_commit(k_free + (u & 1));
                __syncwarp();
                ++u;
            }
        } else if (warp == 2) {
            // ------------------------------------------------------------ lse of the rows of each query tile, in base 2
            int tt[4], g[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { const int r = i * 32 + lane; tt[i] = r / Gq; g[i] = r - tt[i] * Gq; }
            while (ok && next(it)) {
                const int t0 = p.rowg.first(it.L, it.n_new, it.p) + it.j;
#pragma unroll 1
                for (int j = 0; j < it.n; ++j, ++s) {
                    const int tok0 = (t0 + j) * TP;
                    float l[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        l[i] = tt[i] < TP && tok0 + tt[i] < it.n_new ? p.lse[(size_t)(it.q0 + tok0 + tt[i]) * p.v.Hq + (size_t)it.h * Gq + g[i]] * kLog2e : INFINITY;
                    if (s >= NQ) { ok = warp_wait(l_free + s % NQ, (s / NQ - 1) & 1, 75); if (!ok) break; }
                    // one arrival per phase: the scores that used the buffers before are complete
                    for (int x = 0; x < 2 && ok && s >= 2; ++x) ok = warp_wait(s_full + 2 * x + (s & 1), ((s >> 1) - 1) & 1, 78);
                    if (!ok) break;
                    float* dst = reinterpret_cast<float*>(smem + G::L_OFF + (s % NQ) * 512);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dst[i * 32 + lane] = -l[i];
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(s_full + (s & 1)); mbar_arrive(s_full + 2 + (s & 1)); }
                }
            }
        }
    } else {
        // ------------------------------------------------------------ sums of key tile x, one cached token per thread
        reg_inc<MT_REGS_SUM>();
        const int x = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t tS = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + 256u * x;
        const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
        while (ok && next(it)) {
            const int key = it.p * 256 + x * 128 + row, t0 = p.rowg.first(it.L, it.n_new, it.p) + it.j;
            float2 sum[4] = {};
            // 32 columns at a time; the next 32 (at the end of a step the next step's first) are on their way from tensor memory meanwhile,
            // so that the special-function unit does not run dry
            uint32_t v[2][32];
            ok = warp_wait(s_full + 2 * x + (s & 1), (s >> 1) & 1, 76 + x);
            if (!ok) break;
            tc_fence_after();
            tmem_ld32(tS + (s & 1) * 128, v[0]);
            tmem_wait_ld_on(v[0]);
#pragma unroll 1
            for (int j = 0; j < it.n; ++j, ++s) {
                const int tok0 = (t0 + j) * TP;
                // columns [c_lo, c_hi) are rows of tokens that exist and see this thread's cached token
                const int d = key - it.old - tok0;
                const int c_lo = d <= 0 ? 0 : d >= TP ? 128 : d * Gq, c_hi = min(TP, it.n_new - tok0) * Gq;
                // of all columns of all rows of the warp: none masked, or none left
                const bool clean = !__any_sync(0xffffffffu, c_lo > 0 || c_hi < TP * Gq), none = !__any_sync(0xffffffffu, c_lo < c_hi);
                bool there = true;              // the next step's scores (asked for a while before they are needed)
                const float4* nl = reinterpret_cast<const float4*>(smem + G::L_OFF + (s % NQ) * 512);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t (&cur)[32] = v[c & 1];
                    if (c < 3) {
                        tmem_ld32(tS + (s & 1) * 128 + (c + 1) * 32, v[(c + 1) & 1]);
                        if (c == 2 && j + 1 < it.n) there = mbar_try_wait(s_full + 2 * x + ((s + 1) & 1), ((s + 1) >> 1) & 1);
                    } else if (j + 1 < it.n) {
                        if (!__all_sync(0xffffffffu, there)) ok = warp_wait(s_full + 2 * x + ((s + 1) & 1), ((s + 1) >> 1) & 1, 76 + x);
                        if (!ok) break;
                        tc_fence_after();
                        tmem_ld32(tS + ((s + 1) & 1) * 128, v[0]);
                    }
                    if (clean) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 n = nl[8 * c + e / 4];
                            const float2 a = __ffma2_rn(make_float2(__uint_as_float(cur[e]), __uint_as_float(cur[e + 1])), sc2, make_float2(n.x, n.y));
                            const float2 b = __ffma2_rn(make_float2(__uint_as_float(cur[e + 2]), __uint_as_float(cur[e + 3])), sc2, make_float2(n.z, n.w));
                            auto pw = [](float2 w, int pair) { return (pair & 7) < MT_POLY8 ? exp2_poly2(w) : make_float2(fast_exp2(w.x), fast_exp2(w.y)); };
                            sum[(e / 2) & 3] = __fadd2_rn(sum[(e / 2) & 3], pw(a, 3 * (e / 2)));
                            sum[(e / 2 + 1) & 3] = __fadd2_rn(sum[(e / 2 + 1) & 3], pw(b, 3 * (e / 2 + 1)));
                        }
                    } else if (!none) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 n = nl[8 * c + e / 4];
                            auto w = [&](int i, float m) -> float {
                                return 32 * c + e + i >= c_lo && 32 * c + e + i < c_hi ? fast_exp2(fmaf(__uint_as_float(cur[e + i]), p.scale_log2, m)) : 0.f;
                            };
                            sum[(e / 2) & 3] = __fadd2_rn(sum[(e / 2) & 3], make_float2(w(0, n.x), w(1, n.y)));
                            sum[(e / 2 + 1) & 3] = __fadd2_rn(sum[(e / 2 + 1) & 3], make_float2(w(2, n.z), w(3, n.w)));
                        }
                    }
                    tmem_wait_ld_on(v[(c + 1) & 1]);
                    if (c == 2) {                           // all scores of the step are in registers
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(s_free + 2 * x + (s & 1));
                    }
                }
                if (!ok) break;
                __syncwarp();
                if (lane == 0) mbar_arrive(l_free + s % NQ);
            }
            if (!ok) break;
            const float2 t = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
            if (it.whole) {
                const size_t at = ((size_t)it.b * p.v.Hkv + it.h) * p.v.cap + key;
                if (key < it.L) p.mass_out[at] = mass_before(p, at, key, it.old) + (t.x + t.y);
            } else {
                p.part[((size_t)blockIdx.x * 2 + (it.first ? 0 : 1)) * 256 + x * 128 + row] = t.x + t.y;
            }
        }
    }

    // ---------------------------------------------------------------- teardown (also after an abort)
    pdl_release();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        if (elect_one()) umma_commit(drain);
        __syncwarp();
        mbar_wait_limit(drain, 0, nullptr, p.v.status, 91, kWaitLimitNs);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

// A block per cut (see CutRecord): nothing to do where the share begins with a unit, or where an earlier cut of the same unit does it.
__global__ void __launch_bounds__(256) mass_merge_kernel(const __grid_constant__ MassParams p) {
    pdl_wait();
    pdl_release();
    if (*p.v.status != 0) return;
    const int cut = blockIdx.x, r = threadIdx.x;
    const CutRecord c = p.cuts[cut];
    if (c.n == 0 || c.j == 0 || c.j > c.share) return;
    const PagedSeq s = paged_seq(p.v, c.b);
    const int key = c.p * 256 + r;
    if (key >= s.L) return;
    const int parts = 1 + (c.n - c.j + c.share - 1) / c.share;
    const size_t at = ((size_t)c.b * p.v.Hkv + c.h) * p.v.cap + key;
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < parts; ++i)
        sum += p.part[(i == 0 ? (size_t)(cut - 1) * 2 + (c.j < c.share ? 1 : 0) : (size_t)(cut - 1 + i) * 2) * 256 + r];
    p.mass_out[at] = mass_before(p, at, key, s.L - s.n) + sum;
}

template <int D, bool HALF>
seka_status launch_mass_few(const CUtensorMap& tk, const MassParams& p, cudaStream_t st) {
    using SL = MfSmem<D>;
    if (cudaFuncSetAttribute(mass_few_kernel<D, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, SL::BYTES) != cudaSuccess) return SEKA_ERR_CUDA;
    return launch_kernel(true, mass_few_kernel<D, HALF>, (unsigned)p.n_shares, MF_THREADS, SL::BYTES, st, tk, p);
}
template <int D>
seka_status launch_mass_tiles(const CUtensorMap& tq, const CUtensorMap& tk, const MassParams& p, cudaStream_t st) {
    using G = MtGeo<D>;
    if (cudaFuncSetAttribute(mass_tile_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)G::BYTES) != cudaSuccess) return SEKA_ERR_CUDA;
    seka_status stc = launch_kernel(true, mass_tile_kernel<D>, (unsigned)p.n_shares, MT_THREADS, G::BYTES, st, tq, tk, p);
    if (stc != SEKA_OK || p.n_shares == 1) return stc;
    return launch_kernel(true, mass_merge_kernel, (unsigned)p.n_shares, 256, 0, st, p);
}

}  // namespace
}  // namespace seka

extern "C" seka_status seka_attention_mass(const seka_paged_shape* shape, const void* Q, const void* K_pages, const float* lse,
                                           const float* mass_in, float* mass_out, void* workspace, size_t workspace_bytes,
                                           void* cuda_stream) {
    using namespace seka;
    seka_status stc = validate_paged(shape);
    if (stc != SEKA_OK) return stc;
    if (shape->batch == 0) return SEKA_OK;
    if (!mass_out || (shape->total_new > 0 && (!Q || !lse)) || !K_pages) return SEKA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K_pages) & 15) return SEKA_ERR_INVALID_ARG;
    stc = check_paged_call(shape, workspace, workspace_bytes);
    if (stc != SEKA_OK) return stc;
    const PagedLayout w = paged_layout(shape);
    char* ws = static_cast<char*>(workspace);
    const int D = shape->head_dim, Hkv = shape->n_kv_heads, G = shape->n_q_heads / Hkv;
    MassParams p;
    p.v = paged_view(shape, workspace);
    p.Q = static_cast<const __nv_bfloat16*>(Q); p.lse = lse; p.mass_in = mass_in; p.mass_out = mass_out;
    const float scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.f / sqrtf((float)D);
    p.scale_log2 = scale * kLog2e;
    // Steps that a share has at least.  Few rows, one sequence of 128 / 777 / 2048 / 4096 tokens on 8 KV heads, launched and waited for: from one
    // on 19.0 / 19.0 / 19.6 / 20.2 us, from two 19.0 / 19.8 / 19.4 / 20.0, from four 19.8 / 20.6 / 20.3 / 20.6, from eight 23.0 / 22.2 / 21.6 /
    // 21.7; one behind the other all 8.0, the call's work on the host.  Tiles, 32 new tokens over 1024: from one on 11.7 us, from two 13.4,
    // from four 17.0; 128 over 4096 17.0 / 16.9 / 16.3; 512 over 2048 24.7 in each.
    p.key = KeyGeo{6, 4, 1};
    p.rowg = RowGeo{128 / G, 8, 2, (p.v.cap + 255) / 256};
    if (p.rowg.max_units <= 8 && p.rowg.tiles(shape->max_new) >= 1 << 28) p.rowg.max_units = 9;
    p.cuts = reinterpret_cast<CutRecord*>(ws + w.cut_off);
    p.part = reinterpret_cast<float*>(ws + w.mass_part_off);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const long long pool = (long long)shape->n_pages * shape->page_size, pairs = (long long)shape->batch * Hkv;
    CUtensorMap tq, tk;
    if (few_rows(shape) || shape->total_new == 0) {
        const int ctas = D == 128 ? MfSmem<128>::CTAS_PER_SM : MfSmem<64>::CTAS_PER_SM;
        const long long most = (pairs * ((p.v.cap + 63) / 64) + p.key.min_share - 1) / p.key.min_share;
        p.n_shares = (int)(most < kShareSms * ctas ? most : kShareSms * ctas);
        if (!make_tile_map(&tk, K_pages, D, Hkv, pool, shape->page_size < MF_KEYS ? shape->page_size : MF_KEYS, 1, D == 64)) return SEKA_ERR_CUDA;
        const bool half = shape->max_new * G <= 8;
        return D == 128 ? (half ? launch_mass_few<128, true>(tk, p, st) : launch_mass_few<128, false>(tk, p, st))
                        : (half ? launch_mass_few<64, true>(tk, p, st) : launch_mass_few<64, false>(tk, p, st));
    }
    const long long most = pairs * ((p.v.cap + 255) / 256) * p.rowg.tiles(shape->max_new);
    p.n_shares = (int)(most < kShareSms * p.rowg.min_share ? (most + p.rowg.min_share - 1) / p.rowg.min_share : kShareSms);
    if (!make_tile_map(&tk, K_pages, D, Hkv, pool, shape->page_size < 128 ? shape->page_size : 128, 1, D == 64) ||
        !make_tile_map(&tq, Q, D, shape->n_q_heads, shape->total_new, p.rowg.tp, G)) return SEKA_ERR_CUDA;
    return D == 128 ? launch_mass_tiles<128>(tq, tk, p, st) : launch_mass_tiles<64>(tq, tk, p, st);
}
