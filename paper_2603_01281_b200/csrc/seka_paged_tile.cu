// Attention of new tokens over a paged cache: many rows, on tcgen05.
//
// A tile of 128 rows packs the query heads of a KV head beside each other: row r is new token r / G, head r % G, so a chunk of any length
// fills its tiles and every key tile is read once for the whole group.  A unit is two such tiles ("A": the first 128 / G tokens, "B":
// the next) over the same keys; a step is one tile of 128 cached tokens.  One CTA (12 warps) per SM walks its equal share of all
// steps:
//   warp 0        TMA producer: Q (one box of G heads x 128 / G tokens per tile), K and V tiles through two rings, a box per piece
//                 of a page, the lanes issuing side by side; the page of the next tile is looked up a step ahead;
//   warp 1        MMA issuer: S_x = Q_x K^T, O_x += P_x V, all accumulators in tensor memory (S_A, S_B, O_A, O_B; P_x over S_x);
//   warp 2        operand relay: vouches for the operands of a step, so that the issuer waits on one barrier per hand-off; clears value
//                 rows behind the last cached token (pages may hold anything there, NaN included, and 0 times NaN is NaN);
//   warp 3        walks the share and publishes its segments in a small ring, ahead of everyone;
//   warps 4-7 / 8-11  softmax of tile A / B, one row per thread: mask by the row's own last visible token, online softmax in base 2
//                 with a lazily raised maximum, P back as bf16 over the consumed scores, O rescaled only when the maximum moved by
//                 more than 2^8.
// Both tiles take every step of their unit (the last may be masked for all of tile A): the roles then run in step.  Segments
// follow each other without a seam.
// SHARED: launches whose sequences have at most one tile of rows.  A CTA with a single tile would have half of its softmax warps idle
// and the others waiting for the tensor core and it for them: there "A" takes the first 64 keys of every step and "B" the others, for
// the same queries, each with its own maximum, sum and output; the scores of the next step are formed meanwhile, in the other tile's
// columns, and the softmax warps of A join the two states at the end.  A unit that lies in one share is normalised and stored, the parts of a cut one go to the workspace
// in fp32 for paged_merge_kernel.  Weights are rounded to bf16 (2^-8 of each), everything else is fp32.
// Bound by the special-function unit and the chain scores -> softmax -> P V: a step of two tiles is 2048 cycles of exponentials (16 a cycle and
// SM) beside 2048 of products at head_dim 128 (1024 at 64), and takes some 3000 to 3300, as every hand-over waits for the other side.
// 2048 new tokens over 32768, 28/4 heads of 128 (0.93 TFLOP): 725 us at 1.9 GHz, 1.28 PFLOP/s (tensor pipe 66 % busy, special-function
// unit 67 %); 840 us where the power limit holds the clock at 1.6 GHz.
// Every wait is bounded: a wait that runs out raises the CTA's abort flag, every role leaves its loop, the status word reports it.
#include <math.h>

#include "seka_paged_attn.cuh"

namespace seka {
namespace {

constexpr int NTHREADS = 384;
constexpr uint32_t BLK_BYTES = 128 * 128;               // one [128 x 64] bf16 block
constexpr float LAZY_RESCALE_LOG2 = 8.0f;
constexpr int REGS_CTRL = 104, REGS_SOFTMAX = 200;      // of 168 per thread at launch: 104 + 2 x 200 = 3 x 168
constexpr int PLAIN_POLLS = 1;

template <int D>
struct TGeo {
    static constexpr int KP1 = 6;                       // 16-key blocks of P handed over first, so that most of P V runs under the last exponentials
    static constexpr int NK = D == 128 ? 2 : 3;         // K and V ring depth
    static constexpr uint32_t TILE = (D / 64) * BLK_BYTES;
    static constexpr uint32_t K_OFF = 2 * TILE, V_OFF = K_OFF + NK * TILE, BAR_OFF = V_OFF + NK * TILE;
    static constexpr uint32_t NSEG = 8;                 // segments published ahead
    // mbarriers, by first index
    static constexpr uint32_t Q_FULL = 0, K0_FULL = Q_FULL + 2, KV_FULL = K0_FULL + 1, KV_FREE = KV_FULL + NK, S_FULL = KV_FREE + NK, P_FULL = S_FULL + 2,
                              P_LAST = P_FULL + 2, O_FULL = P_LAST + 2, O_DRAINED = O_FULL + 2, START_FULL = O_DRAINED + 2, DRAIN = START_FULL + 1,
                              HALF_READY = DRAIN + 1, O_STEP = HALF_READY + 1, SEG_FULL = O_STEP + 2, SEG_FREE = SEG_FULL + NSEG, NBARS = SEG_FREE + NSEG;
    static constexpr uint32_t MISC_OFF = BAR_OFF + NBARS * 8, SEG_OFF = (MISC_OFF + 16 + 15) & ~15u, STATE_OFF = SEG_OFF + NSEG * 48;       // (SHARED) maximum and sum of B's half, a row each
    static constexpr uint32_t BYTES = STATE_OFF + 128 * 8;
    static_assert(MISC_OFF % 8 == 0 && STATE_OFF % 8 == 0 && sizeof(ShareScratch<NTHREADS>) <= BAR_OFF, "layout");
    static_assert(BYTES <= 227 * 1024, "shared memory");
};

// 32 columns of the rows of a warp (lane = row), scaled, to global memory: four lanes write 64 contiguous bytes of a row.  `off`: the
// lane's row, in elements from `base` (negative: not stored).
template <typename OutT> __device__ __forceinline__ void store_rows32(OutT* base, int off, const uint32_t (&v)[32], float inv, int lane) {
    constexpr int EPU = 16 / (int)sizeof(OutT);
#pragma unroll
    for (int part = 0; part < 32 / (4 * EPU); ++part) {
        uint4 a[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t* w = &v[part * 4 * EPU + u * EPU];
            auto f = [&](int i) { return __uint_as_float(w[i]) * inv; };
            if constexpr (sizeof(OutT) == 2) a[u] = make_uint4(pack_bf16(f(0), f(1)), pack_bf16(f(2), f(3)), pack_bf16(f(4), f(5)), pack_bf16(f(6), f(7)));
            else a[u] = make_uint4(__float_as_uint(f(0)), __float_as_uint(f(1)), __float_as_uint(f(2)), __float_as_uint(f(3)));
        }
        transpose4(a, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int o = __shfl_sync(0xffffffffu, off, (lane & ~3) + k);
            if (o >= 0) *reinterpret_cast<uint4*>(base + o + part * 4 * EPU + (lane & 3) * EPU) = a[k];
        }
    }
}

template <int D, bool SHARED>
__global__ void __launch_bounds__(NTHREADS, 1)
paged_tile_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ PagedAttnParams p) {
    using G = TGeo<D>;
    constexpr int NK = G::NK, NBLK = D / 64;
    constexpr uint32_t TMEM_COLS = 512, COL_S = 0, COL_O = 256;        // S_x (and P_x) at COL_S + 128 x, O_x at COL_O + D x
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + G::BAR_OFF);
    uint64_t* q_full = bars + G::Q_FULL;                 // [2]   Q tile landed
    uint64_t* k0_full = bars + G::K0_FULL;          // [1]   first key tile of the share landed
    uint64_t* kv_full = bars + G::KV_FULL;         // [NK]  V(g) and K(g+1) landed
    uint64_t* kv_free = bars + G::KV_FREE;        // [NK]  one event per step: the tensor core is done with K(g+1) and V(g)
    uint64_t* s_full = bars + G::S_FULL;         // [2]   scores of tile x (SHARED: of the steps in turn) are in tensor memory
    uint64_t* p_full = bars + G::P_FULL;           // [2]   4 softmax warps (O_x rescaled, the first 16 KP1 keys of P_x written) + 1 relay
    uint64_t* p_last = bars + G::P_LAST;           // [2]   4 softmax warps: the other keys of P_x written
    uint64_t* o_full = bars + G::O_FULL;           // [2]   last P V of tile x finished
    uint64_t* o_drained = bars + G::O_DRAINED;        // [2]   4 softmax warps: O_x of the segment has been read
    uint64_t* start_full = bars + G::START_FULL;    // [1]   relay: Q tiles of the segment landed
    uint64_t* drain = bars + G::DRAIN;        // [1]   every product issued has finished
    uint64_t* half_ready = bars + G::HALF_READY;  // [1]  (SHARED) 4 softmax warps of B: the state of their half is complete
    uint64_t* o_step = bars + G::O_STEP;     // [2]   (SHARED) a P V of half x finished
    uint64_t* seg_full = bars + G::SEG_FULL; // [NSEG] segment published
    uint64_t* seg_free = bars + G::SEG_FREE; // [NSEG] 11 warps have read it
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + G::MISC_OFF);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + G::MISC_OFF + 4);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        mbar_init(q_full + 0, 1); mbar_init(q_full + 1, 1); mbar_init(k0_full, 1);
        for (int i = 0; i < NK; ++i) { mbar_init(kv_full + i, 1); mbar_init(kv_free + i, 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + i, 1); mbar_init(p_full + i, 5); mbar_init(p_last + i, 4); mbar_init(o_full + i, 1); mbar_init(o_drained + i, 4);
        }
        mbar_init(start_full, 1); mbar_init(drain, 1);
        mbar_init(half_ready, 4); mbar_init(o_step + 0, 1); mbar_init(o_step + 1, 1);
        for (int i = 0; i < (int)G::NSEG; ++i) { mbar_init(seg_full + i, 1); mbar_init(seg_free + i, 11); }
        *abort_flag = 0; *reinterpret_cast<volatile float*>(smem + G::MISC_OFF + 8) = p.scale_log2;
        mbar_fence_init();
        tma_prefetch_desc(&tmQ); tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV);
    }
    pdl_wait();
    const int status0 = *reinterpret_cast<volatile int*>(p.v.status), hook_skip = p.v.status[4], limit_us = p.v.status[5];
    if (__syncthreads_or(status0 != 0)) return;              // an earlier launch gave up on this workspace
    const Share share = find_share<NTHREADS>(p.v, p.geo, p.n_shares, (int)blockIdx.x, *reinterpret_cast<ShareScratch<NTHREADS>*>(smem));
    if (tid == 0) write_cut(p.cuts, p.v, p.geo, share, (int)blockIdx.x);
    if (share.len == 0) return;
    if (warp == 0) { tmem_alloc(tmem_holder, TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;

    auto limit_ns = [&]() -> uint64_t { return limit_us > 0 ? (uint64_t)limit_us * 1000ull : kWaitLimitNs; };
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, int where) -> bool {
        const bool ok = mbar_wait_within(bar, parity, abort_flag, p.v.status, where, limit_ns, PLAIN_POLLS);
        return __all_sync(0xffffffffu, ok);
    };
    const int TPT = p.tile_tokens;
    // the next segment, as published (n = 0: the share is through)
    struct Seg {
        int b, h, p, j, n, q0, L, old, n_new;      // as in Segment
        int flags;                                 // 1: whole, 2: first, 4: has a tile B
    };
    uint32_t n_seg = 0;
    auto published = [&]() -> bool { return warp_wait(seg_full + n_seg % G::NSEG, (n_seg / G::NSEG) & 1, 50); };
    auto look = [&](Seg& s) {
        const int4* r = reinterpret_cast<const int4*>(smem + G::SEG_OFF + (n_seg % G::NSEG) * 48);
        const int4 a = r[0], b = r[1], c = r[2];
        s.b = a.x; s.h = a.y; s.p = a.z; s.j = a.w; s.n = b.x; s.q0 = b.y; s.L = b.z; s.old = b.w; s.n_new = c.x; s.flags = c.y;
    };
    auto pass = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(seg_free + n_seg % G::NSEG);
        ++n_seg;
    };
    auto next = [&](Seg& s) -> bool {
        if (!published()) return false;
        look(s);
        pass();
        return s.n > 0;
    };
    auto has_b = [](const Seg& s) -> bool { return SHARED || (s.flags & 4) != 0; };       // (SHARED: B takes part in every segment)

    // Key tiles are numbered through, segment after segment: pair g is V(g) and K(g+1) (K(g+1) may be the next segment's first), in stage
    // g % NK of the V ring and (g + 1) % NK of the K ring; kv_free event g + 1 follows step g.
    Seg it;
    if (warp < 4) {
        reg_dec<REGS_CTRL>();
        const bool leader = elect_one();
        if (warp == 0) {
            // ------------------------------------------------------------ TMA producer
            const int bx_shift = p.v.page_shift < 7 ? p.v.page_shift : 7, nb = 128 >> bx_shift;
            const int box = lane % nb, blk = (lane / nb) % NBLK, kv = lane / (nb * NBLK);       // kv 0: K, 1: V, above: idle
            const uint32_t dst = (uint32_t)blk * BLK_BYTES + (uint32_t)((box << bx_shift) * 128);
            const int pool_rows = p.v.n_pages << p.v.page_shift;
            const uint32_t q_bytes = (uint32_t)(TPT * p.v.G) * 128u * NBLK;
            uint32_t pr = 0, n_it = 0, n_qb = 0, ev_seen = 0;
            uint32_t armed_q[2] = {0, 0}, armed_k0 = 0, armed_kv[NK];
#pragma unroll
            for (int i = 0; i < NK; ++i) armed_kv[i] = 0;
            bool ok = true;
            auto see_event = [&](uint32_t e, int where) {
                if (e < ev_seen) return;
                ok = warp_wait(kv_free + e % NK, (e / NK) & 1, where);
                ev_seen = e + 1;
            };
            // pool row of this lane's box of key tile j; -1: behind the cache.  A page that does not exist reads as zeros.
            auto row_of = [&](const Seg& s, int j) -> int {
                const int key = j * 128 + (box << bx_shift);
                if (key >= s.L) return -1;
                const long long r = load_pool_row(p.v, s.b, key);
                return r < 0 ? pool_rows : (int)r;
            };
            auto tile_bytes = [&](const Seg& s, int j) -> uint32_t {
                const int keys = s.L - j * 128;
                const int n_box = keys <= 0 ? 0 : min(nb, (keys + (1 << bx_shift) - 1) >> bx_shift);
                return (uint32_t)(n_box * 128 * NBLK) << bx_shift;
            };
            auto load_q = [&](const Seg& s) {
                const int t0 = s.q0 + s.p * p.geo.tp;
                const bool b2 = !SHARED && has_b(s);
                if (leader) {
                    mbar_expect_tx(q_full + 0, q_bytes);
#pragma unroll
                    for (int c = 0; c < NBLK; ++c) tma_load_3d(smem + c * BLK_BYTES, &tmQ, q_full + 0, c * 64, s.h * p.v.G, t0);
                    if (b2) {
                        mbar_expect_tx(q_full + 1, q_bytes);
#pragma unroll
                        for (int c = 0; c < NBLK; ++c) tma_load_3d(smem + G::TILE + c * BLK_BYTES, &tmQ, q_full + 1, c * 64, s.h * p.v.G, t0 + TPT);
                    }
                }
                __syncwarp();
                armed_q[0] = (n_it & 1) + 1; ++n_it;
                if (b2) { armed_q[1] = (n_qb & 1) + 1; ++n_qb; }
            };
            bool have = next(it), first = true;
            int row0 = -1, row1 = -1;                   // this step's tile; the next one (of this segment or the next)
            if (have) {
                load_q(it);
                row0 = row_of(it, it.j);
                if (it.n > 1) row1 = row_of(it, it.j + 1);
                if (leader) mbar_expect_tx(k0_full, tile_bytes(it, it.j));
                __syncwarp();
                if (kv == 0 && row0 >= 0) tma_load_3d(smem + G::K_OFF + dst, &tmK, k0_full, blk * 64, it.h, row0);
                armed_k0 = 1;
            }
            while (ok && have) {
                Seg nx;
                const bool more = next(nx);
                const int nx_row = more ? row_of(nx, nx.j) : -1;
#pragma unroll 1
                for (int t = 0; t < it.n; ++t) {
                    const uint32_t g = pr + (uint32_t)t;
                    const bool inside = t + 1 < it.n, any = inside || more;
                    if (!inside) row1 = nx_row;
                    const int row2 = t + 2 < it.n ? row_of(it, it.j + t + 2) : -1;
                    if (g >= NK - 1) {
                        see_event(g - (NK - 1), 10);
                        if (!ok) break;
                    }
                    uint64_t* bar = kv_full + g % NK;
                    // (test hook: one pair of the first segment of CTA 0 is left out altogether, so that its wait runs out)
                    const bool skip = hook_skip > 0 && first && blockIdx.x == 0 && t + 1 == hook_skip;
                    if (!skip) {
                        if (leader) mbar_expect_tx(bar, tile_bytes(it, it.j + t) + (inside ? tile_bytes(it, it.j + t + 1) : more ? tile_bytes(nx, nx.j) : 0u));
                        __syncwarp();
                        if (kv == 1 && row0 >= 0) tma_load_3d(smem + G::V_OFF + (g % NK) * G::TILE + dst, &tmV, bar, blk * 64, it.h, row0);
                        if (kv == 0 && any && row1 >= 0) tma_load_3d(smem + G::K_OFF + ((g + 1) % NK) * G::TILE + dst, &tmK, bar, blk * 64, inside ? it.h : nx.h, row1);
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < NK; ++i)
                            if ((int)(g % NK) == i) armed_kv[i] = ((g / NK) & 1) + 1;
                    }
                    row0 = row1; row1 = row2;
                }
                if (!ok) break;
                pr += it.n;
                if (more) {
                    row1 = nx.n > 1 ? row_of(nx, nx.j + 1) : -1;
                    see_event(pr - 1, 12);              // the last score products of the segment are through: its Q tiles may be replaced
                    if (!ok) break;
                    load_q(nx);
                }
                it = nx; have = more; first = false;
            }
            if (*abort_flag) {
                // loads that were armed may still be in flight: let them land before the shared memory is released
                auto settle = [&](uint64_t* bar, uint32_t armed) {
                    if (armed) mbar_wait_within(bar, armed - 1, nullptr, nullptr, 0, limit_ns);
                };
                settle(q_full + 0, armed_q[0]); settle(q_full + 1, armed_q[1]); settle(k0_full, armed_k0);
#pragma unroll
                for (int i = 0; i < NK; ++i) settle(kv_full + i, armed_kv[i]);
            }
        } else if (warp == 1) {
            // ------------------------------------------------------------ MMA issuer
            constexpr uint32_t IDESC_S = umma_idesc_bf16(128, false);
            constexpr uint32_t IDESC_PV = umma_idesc_bf16(D, true);
            constexpr uint32_t DESC_HI = umma_desc_hi_sw128(1024);
            const uint32_t dQ = umma_desc_lo(smem_u32(smem), 16), dK = umma_desc_lo(smem_u32(smem + G::K_OFF), 16);
            const uint32_t dV = umma_desc_lo(smem_u32(smem + G::V_OFF), BLK_BYTES);
            uint32_t n_it = 0, cx[2] = {0, 0}, n_o[2] = {0, 0};        // segments, steps of tile x, segments that had a tile x
            bool ok = true;
            // scores of the queries in tile q into columns x
            auto issue_S = [&](int x, int q, uint32_t st) {
                const uint32_t kd = dK + st * (G::TILE >> 4), qd = dQ + (uint32_t)q * (G::TILE >> 4), acc = tmem_base + COL_S + 128 * x;
                tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        const uint32_t off = ((uint32_t)(ks >> 2) * BLK_BYTES + (uint32_t)(ks & 3) * 32) >> 4;
                        umma_ss(acc, qd + off, DESC_HI, kd + off, DESC_HI, IDESC_S, ks > 0 ? 1u : 0u);
                    }
                    umma_commit(s_full + x);
                }
                __syncwarp();
            };
            // O_x (+)= P V over the blocks of 16 keys [ks0, ks1) of the value tile; their P starts in column `src`
            auto issue_PV = [&](int x, uint32_t src, uint32_t st, bool fresh, int ks0, int ks1, bool last) {
                const uint32_t vd = dV + st * (G::TILE >> 4) + (uint32_t)ks0 * (2048 >> 4), acc = tmem_base + COL_O + D * x;
                tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        if (ks < ks1 - ks0)
                            umma_ts(acc, tmem_base + src + (uint32_t)ks * 8, vd + (uint32_t)ks * (2048 >> 4), DESC_HI, IDESC_PV, (!fresh || ks > 0) ? 1u : 0u);
                    if (SHARED) umma_commit(o_step + x);
                    if (last) umma_commit(o_full + x);
                }
                __syncwarp();
            };
            // P of tile x and step j has been handed over.  Before a segment's first P V writes O_x, the O_x of the last segment
            // that had a tile x has been read (each phase is seen, in order).
            auto p_ready = [&](int x, int j) {
                ok = warp_wait(p_full + x, (cx[x] + j) & 1, 24 + 2 * x);
                if (ok && j == 0 && n_o[x] > 0) ok = warp_wait(o_drained + x, (n_o[x] - 1) & 1, 46 + x);
            };
            auto step_PV = [&](int x, uint32_t st, int j, int n) {
                p_ready(x, j);
                if (!ok) return;
                issue_PV(x, COL_S + 128 * x, st, j == 0, 0, G::KP1, false);
                ok = warp_wait(p_last + x, (cx[x] + j) & 1, 28 + x);
                if (!ok) return;
                issue_PV(x, COL_S + 128 * x + 8 * G::KP1, st, false, G::KP1, 8, j == n - 1);
            };
            // (SHARED) P of the 64 keys of half x lies over their scores, in buffer `buf`
            auto step_half = [&](int x, uint32_t buf, uint32_t st, int j, int n) {
                p_ready(x, j);
                if (ok) issue_PV(x, COL_S + 128 * buf + 64 * x, st, j == 0, 4 * x, 4 * x + 4, j == n - 1);
            };
            auto commit_event = [&](uint32_t st) {
                if (leader) umma_commit(kv_free + st);
                __syncwarp();
            };
            uint32_t st = 0, g = 0;       // stage of the present value tile, its number
            bool have = next(it);
            if (have) ok = warp_wait(start_full, 0, 20);
            if (ok && have) {
                issue_S(0, 0, 0);
                if (!SHARED && has_b(it)) issue_S(1, 1, 0);
                commit_event(0);
            }
            while (ok && have) {
                Seg nx;
                const bool more = next(nx), itB = has_b(it), nxB = more && has_b(nx);
                ++n_it;
#pragma unroll 1
                for (int j = 0; j < it.n; ++j, ++g) {
                    const uint32_t st1 = st + 1 == (uint32_t)NK ? 0u : st + 1;
                    const bool inside = j + 1 < it.n, turn = !inside && more;
                    if (SHARED) {
                        if (inside) {           // the next scores go first: they only need their keys
                            ok = warp_wait(kv_full + g % NK, (g / NK) & 1, 25);
                            if (!ok) break;
                            issue_S((j & 1) ^ 1, 0, st1);
                        }
                        step_half(0, j & 1, st, j, it.n);
                        if (ok) step_half(1, j & 1, st, j, it.n);
                        if (ok && turn) ok = warp_wait(start_full, n_it & 1, 21);
                        if (!ok) break;
                        if (turn) issue_S(0, 0, st1);
                    } else {
                        // V of this step and K of the next have landed once p_full completes: the relay vouches for them there
                        step_PV(0, st, j, it.n);
                        if (!ok) break;
                        if (turn) { ok = warp_wait(start_full, n_it & 1, 21); if (!ok) break; }
                        if (inside || turn) issue_S(0, 0, st1);
                        if (itB) { step_PV(1, st, j, it.n); if (!ok) break; }
                        if ((inside && itB) || (turn && nxB)) issue_S(1, 1, st1);
                    }
                    commit_event(st1);
                    st = st1;
                }
                if (!ok) break;
                cx[0] += it.n; ++n_o[0];
                if (itB) { cx[1] += it.n; ++n_o[1]; }
                it = nx; have = more;
            }
        } else if (warp == 2) {
            // ------------------------------------------------------------ operand relay
            uint32_t pr = 0, n_it = 0, n_qb = 0, cx[2] = {0, 0};
            bool ok = true;
            auto q_landed = [&](const Seg& s) {
                ok = warp_wait(q_full + 0, n_it & 1, 21);
                ++n_it;
                if (!SHARED && ok && has_b(s)) { ok = warp_wait(q_full + 1, n_qb & 1, 22); ++n_qb; }
                if (ok && n_it == 1) ok = warp_wait(k0_full, 0, 23);
                if (ok && lane == 0) mbar_arrive(start_full);
                __syncwarp();
            };
            bool have = next(it);
            if (have) q_landed(it);
            while (ok && have) {
                Seg nx;
                const bool more = next(nx), itB = has_b(it);
#pragma unroll 1
                for (int j = 0; j < it.n; ++j) {
                    const uint32_t g = pr + (uint32_t)j;
                    ok = warp_wait(kv_full + g % NK, (g / NK) & 1, 25);
                    if (!ok) break;
                    const int left = it.L - (it.j + j) * 128;              // value rows from here on lie behind the cache
                    if (left < 128) {
                        for (int u = max(left, 0) * 8 + lane; u < 128 * 8; u += 32) {
#pragma unroll
                            for (int c = 0; c < NBLK; ++c)
                                *reinterpret_cast<uint4*>(smem + G::V_OFF + (g % NK) * G::TILE + c * BLK_BYTES + u * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async();
                        __syncwarp();
                    }
                    if (lane == 0) {
                        mbar_arrive(p_full + 0);
                        if (itB) mbar_arrive(p_full + 1);
                    }
                    __syncwarp();
                    // the next segment's Q tiles land while the last softmax of this one runs
                    if (j + 1 == it.n && more) { q_landed(nx); if (!ok) break; }
                    // stay within the phase: the next arrival may only come after this phase has completed and the issuer has seen it
                    // (SHARED, where the next weights do not wait for the issuer: after the event of the step)
                    if (SHARED) ok = warp_wait(kv_free + (g + 1) % NK, ((g + 1) / NK) & 1, 35);
                    else ok = warp_wait(p_full + 0, (cx[0] + j) & 1, 33);
                    if (!SHARED && ok && itB) ok = warp_wait(p_full + 1, (cx[1] + j) & 1, 34);
                    if (!ok) break;
                }
                pr += it.n; cx[0] += it.n;
                if (itB) cx[1] += it.n;
                it = nx; have = more;
            }
        } else {
            // ------------------------------------------------------------ walk
            Walk w;
            walk_begin(p.v, share, w);
            bool more = true;
            for (uint32_t k = 0; more; ++k) {
                Segment s;
                s.n = 0;
                more = walk_next(p.v, p.geo, w, s);
                const uint32_t i = k % G::NSEG;
                if (k >= G::NSEG && !warp_wait(seg_free + i, (k / G::NSEG - 1) & 1, 51)) break;
                if (lane == 0) {
                    const int flags = more ? (s.whole ? 1 : 0) | (s.first ? 2 : 0) | (s.p * p.geo.tp + TPT < s.n_new ? 4 : 0) : 0;
                    int4* r = reinterpret_cast<int4*>(smem + G::SEG_OFF + i * 48);
                    r[0] = make_int4(s.b, s.h, s.p, s.j); r[1] = make_int4(s.n, s.q0, s.L, s.old); r[2] = make_int4(s.n_new, flags, 0, 0);
                    mbar_arrive(seg_full + i);
                }
                __syncwarp();
            }
        }
    } else {
        // ------------------------------------------------------------ softmax of tile x, one row per thread
        reg_inc<REGS_SOFTMAX>();
        const int x = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t t_lane = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t tS = t_lane + COL_S + 128 * x, tO = t_lane + COL_O + D * x;
        const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
        constexpr int NC = SHARED ? 64 : 128;        // scores of a row that one thread takes
        uint32_t cX = 0, n_o = 0, n_s[2] = {0, 0};    // steps; phases of o_full; (SHARED) phases of the two score buffers
        float2* half_state = reinterpret_cast<float2*>(smem + G::STATE_OFF);
        bool ok = true;
        // (the segment is read from the ring twice, for its steps and for its end: its ten words would not fit beside the scores)
        while (ok && published()) {
            look(it);
            const int n = it.n;
            if (n == 0 || (x == 1 && !has_b(it))) {
                pass();
                if (n == 0) break;
                continue;
            }
            const int tok = it.p * p.geo.tp + (SHARED ? 0 : x * TPT) + row / p.v.G;
            // last cached token that the row sees, counted from its first key of the step (rows without a token: as the last one)
            int lim = it.old + min(tok, it.n_new - 1) - it.j * 128 - (SHARED ? 64 * x : 0);
            float m_run = -INFINITY, l_run = 0.f;
#pragma unroll 1
            for (int j = 0; j < n; ++j, lim -= 128) {
                // (SHARED) the steps of a segment use the two buffers in turn
                const uint32_t tc = SHARED ? t_lane + COL_S + 128 * (j & 1) + 64 * x : tS;
                ok = SHARED ? warp_wait(s_full + (j & 1), (((j & 1) ? n_s[1] : n_s[0]) + (j >> 1)) & 1, 40 + x) : warp_wait(s_full + x, (cX + j) & 1, 40 + x);
                if (!ok) break;
                tc_fence_after();
                uint32_t v[NC];
#pragma unroll
                for (int c = 0; c < NC / 32; ++c) tmem_ld32(tc + c * 32, reinterpret_cast<uint32_t(&)[32]>(v[32 * c]));
                tmem_wait_ld();
                if (__any_sync(0xffffffffu, lim < NC - 1)) {
#pragma unroll
                    for (int e = 0; e < NC; ++e)
                        if (e > lim) v[e] = 0xff800000u;
                }
                float mx[NC / 16];
#pragma unroll
                for (int q = 0; q < NC / 16; ++q) {
                    mx[q] = fmaxf(__uint_as_float(v[16 * q]), __uint_as_float(v[16 * q + 1]));
#pragma unroll
                    for (int e = 2; e < 16; e += 2) mx[q] = max3(mx[q], __uint_as_float(v[16 * q + e]), __uint_as_float(v[16 * q + e + 1]));
                }
                float mx_all;
                if constexpr (SHARED) mx_all = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                else mx_all = fmaxf(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], max3(mx[5], mx[6], mx[7])));
                const float m_new = fmaxf(m_run, mx_all * p.scale_log2);
                // raise the running maximum only when it moved a lot; p may then exceed 1 (up to 2^8), which is harmless
                const bool raise = (m_new - m_run) > LAZY_RESCALE_LOG2;      // (both -inf: false)
                const float factor = raise ? fast_exp2(m_run - m_new) : 1.f;
                if (raise) m_run = m_new;
                if (j > 0 && __any_sync(0xffffffffu, raise)) {
                    // O_x is rescaled behind the P V before.  (SHARED) These scores did not wait for that one, but for the one before it
                    // (so the barrier is in this phase or just through it: its parity tells)
                    if (SHARED) {
                        ok = warp_wait(o_step + x, (cX + j - 1) & 1, 48 + x);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    uint32_t o[32];
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        tmem_ld32(tO + c * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                        tmem_st32(tO + c * 32, o);
                    }
                }
                float2 sc_piece = sc2;
                const float nm = m_run == -INFINITY ? 0.f : -m_run;          // nothing visible so far: all weights are exp2(-inf)
                const float2 nm2 = make_float2(nm, nm);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < NC / 32; ++c) {
                    uint32_t pk16[16];
#pragma unroll
                    for (int e2 = 0; e2 < 16; ++e2) {
                        const int e = 32 * c + 2 * e2;
                        const float2 arg = __ffma2_rn(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), sc_piece, nm2);
                        const float2 pe = make_float2(fast_exp2(arg.x), fast_exp2(arg.y));
                        sum[e2 & 1] = __fadd2_rn(sum[e2 & 1], pe);
                        pk16[e2] = pack_bf16(pe.x, pe.y);
                    }
                    tmem_st16(tc + c * 16, pk16);          // P (bf16 pairs) over score columns that are already in registers
                    if (!SHARED && 2 * c + 2 == G::KP1) {             // the first piece is in place: the tensor core may start on it
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(p_full + x);
                        // the scale of the other keys is read again here, so that their exponentials are not moved ahead of the hand-over
                        float again;
                        asm volatile("ld.volatile.shared.f32 %0, [%1];" : "=f"(again) : "r"(smem_u32(smem + G::MISC_OFF + 8)) : "memory");
                        sc_piece = make_float2(again, again);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                if (SHARED && j > 0) {
                    // these weights may be there before the step before has been handed over (its values are still on the way): their
                    // arrival must not count for that one
                    ok = warp_wait(p_full + x, (cX + j - 1) & 1, 43);
                    if (!ok) break;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive((SHARED ? p_full : p_last) + x);
                const float2 s2 = __fadd2_rn(sum[0], sum[1]);
                l_run = l_run * factor + (s2.x + s2.y);
            }
            if (!ok) break;
            cX += n; n_s[0] += (n + 1) / 2; n_s[1] += n / 2;
            look(it);
            pass();
            ok = warp_wait(o_full + x, n_o & 1, 44 + x);
            if (!ok) break;
            ++n_o;
            tc_fence_after();
            if (SHARED) {
                if (x == 1) {               // hand the state of B's half to A's warps
                    half_state[row] = make_float2(m_run, l_run);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(half_ready);
                    continue;
                }
                ok = warp_wait(half_ready, (n_o - 1) & 1, 49);
                if (!ok) break;
                tc_fence_after();
                const float2 st = half_state[row];
                const float m = fmaxf(m_run, st.x), f_a = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m);
                const float f_b = st.x == -INFINITY ? 0.f : fast_exp2(st.x - m);
                l_run = l_run * f_a + st.y * f_b;
                m_run = m;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {          // O_A = f_a O_A + f_b O_B
                    uint32_t a[32], b[32];
                    tmem_ld32(tO + c * 32, a);
                    tmem_ld32(tO + D + c * 32, b);
                    tmem_wait_ld_on(a);
                    tmem_wait_ld_on(b);
#pragma unroll
                    for (int e = 0; e < 32; ++e) a[e] = __float_as_uint(fmaf(__uint_as_float(b[e]), f_b, __uint_as_float(a[e]) * f_a));
                    tmem_st32(tO + c * 32, a);
                }
                tmem_wait_st();
            }
            const int xt = SHARED ? 0 : x;
            if (it.flags & 1) {
                const int tt = row / p.v.G, g = row - tt * p.v.G, tk = it.p * p.geo.tp + xt * TPT + tt;
                const bool real = tt < TPT && tk < it.n_new;
                const size_t row_at = (size_t)(it.q0 + it.p * p.geo.tp + xt * TPT) * p.v.Hq + (size_t)it.h * p.v.G;       // row 0 of the tile
                const int off = real ? (tt * p.v.Hq + g) * D : -1;
                const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
                if (real && p.lse != nullptr)
                    p.lse[row_at + (size_t)(tt * p.v.Hq + g)] = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * 0.6931471805599453f;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tO + c * 32, o);
                    tmem_wait_ld_on(o);
                    store_rows32<__nv_bfloat16>(p.O + row_at * D + c * 32, off, o, inv, lane);
                }
            } else {
                const size_t part = (((size_t)blockIdx.x * 2 + ((it.flags & 2) ? 0 : 1)) * 2 + x) * 128;
                *reinterpret_cast<float2*>(p.part_ml + (part + row) * 2) = make_float2(m_run, l_run);
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tO + c * 32, o);
                    tmem_wait_ld_on(o);
                    store_rows32<float>(p.part_o + part * D + c * 32, row * D, o, 1.f, lane);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) { mbar_arrive(o_drained + x); if (SHARED) mbar_arrive(o_drained + 1); }
        }
    }

    // ---------------------------------------------------------------- teardown (also after an abort)
    pdl_release();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        // every product issued has finished before tensor and shared memory are released
        if (elect_one()) umma_commit(drain);
        __syncwarp();
        mbar_wait_within(drain, 0, nullptr, p.v.status, 90, limit_ns);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem_base, TMEM_COLS);
}

}  // namespace

template <int D>
seka_status launch_paged_tiles(const PagedAttnParams& p, const void* Q, const void* K, const void* V, int page_size, cudaStream_t st) {
    using G = TGeo<D>;
    const int box = page_size < 128 ? page_size : 128;
    const long long rows = (long long)p.v.n_pages * page_size;
    CUtensorMap tq, tk, tv;
    if (!make_tile_map(&tq, Q, D, p.v.Hq, p.v.T, p.tile_tokens, p.v.G) || !make_tile_map(&tk, K, D, p.v.Hkv, rows, box, 1, D == 64) ||
        !make_tile_map(&tv, V, D, p.v.Hkv, rows, box, 1, D == 64)) return SEKA_ERR_CUDA;
    auto kern = p.geo.tp == p.tile_tokens ? paged_tile_kernel<D, true> : paged_tile_kernel<D, false>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)G::BYTES) != cudaSuccess) return SEKA_ERR_CUDA;
    return launch_kernel(true, kern, (unsigned)p.n_shares, NTHREADS, G::BYTES, st, tq, tk, tv, p);
}

template seka_status launch_paged_tiles<64>(const PagedAttnParams&, const void*, const void*, const void*, int, cudaStream_t);
template seka_status launch_paged_tiles<128>(const PagedAttnParams&, const void*, const void*, const void*, int, cudaStream_t);

}  // namespace seka
