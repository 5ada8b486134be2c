// Eviction: every (sequence, KV head) of more than `keep` cached rows is cut to the `keep` that come first by (class, weight, row).
//
//   evict_select_kernel   a cluster of 1 to 8 CTAs per (sequence, KV head), a run of consecutive rows each.  A row's rank is its class (2:
//                         recent, 1: highlighted, 0) above its weight mapped to 32 bits whose unsigned order is the order of the
//                         weights; both are formed once and kept in shared memory (where they fit).  The class that the keep-th row
//                         belongs to follows from the counts, and makes one 32-bit key of both.  The key is narrowed down in digits of
//                         eight bits, from the first bit that differs between the smallest and the largest weight on (a CTA's
//                         histogram has 16 columns, so that a warp's updates meet in pairs at most; the CTAs add their totals through
//                         distributed shared memory) until at most 256 rows are left, which are then
//                         compared with one another, row numbers included.  Only more than 256 equal weights go through all four
//                         digits and a count of ties in row order.  Last the lists of the freed rows below `keep` and of the
//                         kept ones behind, every warp on consecutive rows so that ranks come from ballots.  Four rows a lane
//                         at a time: with many pairs the passes are bound by instructions, not by memory.
//   evict_move_kernel     copies K, V, weight and position of the kept rows behind into the freed rows.
// 64 contexts of 1024 to 4096 rows, 8 KV heads of 128, cut to 2048: 80 us = 30 (selection) + 50 (233 MB, 4.1 TB/s: a chain of list, table and
// row, four rows of a warp in flight); one of 65536 cut to 16384: 60 us, of which 27 are the selection (a chain of passes and cluster
// barriers on 64 SMs) and 24 the moves.
// What is kept below `keep` does not move: a cache that is cut often, by a little each time, moves only that little.  Sources lie at or
// behind `keep`, destinations below it, so the copies need no order.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {
namespace {

constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_MAX_CLUSTER = 8;
constexpr int EV_COLS = 16;                             // columns of the histogram (lanes l and l + 16 share one)
constexpr int EV_CAND = 256;                            // rows that are compared with one another, at most one per thread
constexpr int EV_MAX_CACHED = 40 * 1024;                // rows of a CTA whose ranks fit in shared memory beside the histogram
constexpr uint32_t EV_IN = 0xffffffffu, EV_OUT = 0u;    // keys of rows of a higher / lower class than the cut's (no weight has them)

struct EvictParams {
    PagedView v;
    __nv_bfloat16 *K, *V;
    const float* mass_in;
    float* mass_out;
    const int* pos_in;
    int* pos_out;
    const uint8_t* protect;
    int protect_len;
    const int* next_pos;
    int keep, recent;
    int cluster, cached;        // CTAs of a (sequence, KV head) in the first launch; rows whose ranks are kept in shared memory
    int move_blocks, move_rows; // blocks of a (sequence, KV head) in the second launch; rows of a warp at a time
    int* lens_out;
    int* count;                 // [B, Hkv] rows that move
    int* list;                  // [B, Hkv, cap]
};

// weight -> 32 bits in the same order (NaN first, then -inf; the two zeros equal), between EV_OUT and EV_IN
SEKA_HD uint32_t mass_order(float x, uint32_t bits) {
    if (x != x) return 1u;
    if (x == 0.f) return 0x80000000u;
    return (bits & 0x80000000u) ? ~bits : bits | 0x80000000u;
}

struct EvSmem {
    int hist[256][EV_COLS];
    int tot[2][256];            // this CTA's totals of a digit (read by the cluster; two, so that one barrier per digit is enough)
    int sum[256];               // ... added up over the cluster
    int xch[4][4];              // what the CTAs tell each other: class counts and status; ties; freed and late rows; candidates and extreme weights
    uint2 cand[EV_CAND];        // rows that are left in this CTA: number, negated (the lowest first among equals), and key
    unsigned long long all[EV_CAND];    // ... of the cluster, as one number that grows with the rank
    int warp_a[EV_WARPS], warp_b[EV_WARPS];
    uint32_t warp_min[EV_WARPS], warp_max[EV_WARPS];
    int found[4];
};
constexpr size_t EV_MAX_BYTES = sizeof(EvSmem) + (size_t)EV_MAX_CACHED * 5;
static_assert(EV_MAX_BYTES <= 227 * 1024, "shared memory");

__device__ __forceinline__ int ld_cluster(const int* local, int rank) {
    uint32_t a;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier(int C) {
    if (C == 1) { __syncthreads(); return; }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const EvictParams p) {
    extern __shared__ __align__(16) uint8_t smem[];
    EvSmem& sm = *reinterpret_cast<EvSmem*>(smem);
    uint32_t* ord_s = reinterpret_cast<uint32_t*>(smem + sizeof(EvSmem));
    uint8_t* cls_s = reinterpret_cast<uint8_t*>(ord_s + p.cached);
    const int C = p.cluster, pair = (int)blockIdx.x / C, rank = (int)blockIdx.x - pair * C, b = pair / p.v.Hkv;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned all = 0xffffffffu, below = (1u << lane) - 1;
    pdl_wait();
    pdl_release();
    const int status0 = *reinterpret_cast<volatile int*>(p.v.status);
    const int L = p.v.lens[b], keep = p.keep;
    if (L < 0 || L > p.v.cap) {                         // (the same for the whole cluster)
        if (tid == 0 && rank == 0) { report_invalid(p.v.status, kWhereSeq); p.count[pair] = 0; }
        return;
    }
    const size_t base = (size_t)pair * p.v.cap;
    const float* mass = p.mass_in + base;
    const int* pos = p.pos_in + base;
    if (L <= keep) {
        if (status0 == 0)
            for (int j = rank * EV_THREADS + tid; j < L; j += C * EV_THREADS) {
                if (p.mass_out != p.mass_in) p.mass_out[base + j] = mass[j];
                if (p.pos_out != p.pos_in) p.pos_out[base + j] = pos[j];
            }
        if (tid == 0 && rank == 0) p.count[pair] = 0;
        return;
    }
    // rows of this CTA [lo, hi), of this warp [wlo, whi): consecutive, multiples of 128
    const int wrows = ((L + C * EV_WARPS - 1) / (C * EV_WARPS) + 127) & ~127, chunk = wrows * EV_WARPS;
    const long long lo_l = (long long)rank * chunk;
    const int lo = (int)(lo_l < L ? lo_l : L), hi = L - lo < chunk ? L : lo + chunk;
    const int wlo = hi - lo < warp * wrows ? hi : lo + warp * wrows, whi = hi - wlo < wrows ? hi : wlo + wrows;
    const bool cached = chunk <= p.cached;
    const long long recent_from = (long long)p.next_pos[b] - p.recent;
    const uint8_t* prot = p.protect != nullptr ? p.protect + (size_t)b * p.protect_len : nullptr;
    auto flag_of = [&](int x) -> int {                  // (any valid address where the position has no flag)
        const bool inside = x >= 0 && x < p.protect_len;
        const int f = prot != nullptr ? (int)prot[inside ? x : 0] : 0;
        return inside && f != 0 ? 1 : 0;
    };
    auto class_of = [&](int x, int flag) -> uint32_t { return (long long)x >= recent_from ? 2u : (uint32_t)flag; };
    // of a value per warp: the sum, and the sum over the warps before this one
    auto over_warps = [&](const int* w, int& total) -> int {
        const int x = lane < EV_WARPS ? w[lane] : 0;
        total = __reduce_add_sync(all, x);
        return __reduce_add_sync(all, lane < warp ? x : 0);
    };

    // weights and positions once from memory, eight rows of a lane in flight; rows below `keep` are passed on as they are (what is freed
    // is written over by the second launch).  (Rows up to the next multiple of four behind the last one are read and not used: a state
    // row has 16-byte units.)
    int n2 = 0, n1 = 0;
    uint32_t o_min = 0xffffffffu, o_max = 0u;
    const bool copy_m = p.mass_out != p.mass_in, copy_p = p.pos_out != p.pos_in;
    for (int j0 = wlo + 4 * lane; j0 - 4 * lane < whi; j0 += 256) {
        float4 m[2];
        int4 x[2];
        int f[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = j0 + 128 * h < whi ? j0 + 128 * h : wlo;
            m[h] = *reinterpret_cast<const float4*>(mass + j); x[h] = *reinterpret_cast<const int4*>(pos + j);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) { f[h][0] = flag_of(x[h].x); f[h][1] = flag_of(x[h].y); f[h][2] = flag_of(x[h].z); f[h][3] = flag_of(x[h].w); }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = j0 + 128 * h, n = min(4, whi - j);
            if (n <= 0) continue;
            const float mv[4] = {m[h].x, m[h].y, m[h].z, m[h].w};
            const int xv[4] = {x[h].x, x[h].y, x[h].z, x[h].w};
            uint32_t o[4], c4 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = class_of(xv[i], f[h][i]);
                o[i] = mass_order(mv[i], __float_as_uint(mv[i]));
                c4 |= c << (8 * i);
                n2 += i < n && c == 2; n1 += i < n && c == 1;
                if (i < n) { o_min = min(o_min, o[i]); o_max = max(o_max, o[i]); }
            }
            if (cached) {
                *reinterpret_cast<uint4*>(ord_s + (j - lo)) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint32_t*>(cls_s + (j - lo)) = c4;
            }
            if (j + 4 <= keep && n == 4) {
                if (copy_m) *reinterpret_cast<float4*>(p.mass_out + base + j) = m[h];
                if (copy_p) *reinterpret_cast<int4*>(p.pos_out + base + j) = x[h];
            } else {
                for (int i = 0; i < n && j + i < keep; ++i) {
                    if (copy_m) p.mass_out[base + j + i] = mv[i];
                    if (copy_p) p.pos_out[base + j + i] = xv[i];
                }
            }
        }
    }
    n2 = __reduce_add_sync(all, n2); n1 = __reduce_add_sync(all, n1);
    o_min = __reduce_min_sync(all, o_min); o_max = __reduce_max_sync(all, o_max);
    if (lane == 0) { sm.warp_a[warp] = n2; sm.warp_b[warp] = n1; sm.warp_min[warp] = o_min; sm.warp_max[warp] = o_max; }
    __syncthreads();
    over_warps(sm.warp_a, n2); over_warps(sm.warp_b, n1);
    o_min = __reduce_min_sync(all, lane < EV_WARPS ? sm.warp_min[lane] : 0xffffffffu);
    o_max = __reduce_max_sync(all, lane < EV_WARPS ? sm.warp_max[lane] : 0u);
    int bad = status0;
    if (C > 1) {
        if (tid == 0) { sm.xch[0][0] = n2; sm.xch[0][1] = n1; sm.xch[0][2] = status0; sm.xch[3][1] = (int)o_min; sm.xch[3][2] = (int)o_max; }
        cluster_barrier(C);
        n2 = 0; n1 = 0; bad = 0;
        for (int r = 0; r < C; ++r) { n2 += ld_cluster(&sm.xch[0][0], r); n1 += ld_cluster(&sm.xch[0][1], r); bad |= ld_cluster(&sm.xch[0][2], r); }
        for (int r = 0; r < C; ++r) { o_min = min(o_min, (uint32_t)ld_cluster(&sm.xch[3][1], r)); o_max = max(o_max, (uint32_t)ld_cluster(&sm.xch[3][2], r)); }
    }
    bad = __syncthreads_or(bad);                        // (one CTA's threads may have read the status at different times)
    if (bad) { cluster_barrier(C); return; }            // an earlier launch gave up (decided together: nobody leaves while others read)
    const uint32_t cut_class = n2 >= keep ? 2u : n2 + n1 >= keep ? 1u : 0u;
    auto merge = [&](uint32_t c, uint32_t o) -> uint32_t { return c == cut_class ? o : c > cut_class ? EV_IN : EV_OUT; };
    // keys of the rows j .. j + 3 of this lane (behind the last row: EV_OUT)
    auto keys = [&](int j, uint32_t (&k)[4]) {
        if (cached) {
            const uint4 o = *reinterpret_cast<const uint4*>(ord_s + (j - lo));
            k[0] = o.x; k[1] = o.y; k[2] = o.z; k[3] = o.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                k[i] = EV_OUT;
                if (j + i < whi) { const float w = mass[j + i]; const int x = pos[j + i]; k[i] = merge(class_of(x, flag_of(x)), mass_order(w, __float_as_uint(w))); }
            }
        }
    };
    if (cached)
        for (int j = wlo + 4 * lane; j < whi; j += 128) {
            const uint4 o = *reinterpret_cast<const uint4*>(ord_s + (j - lo));
            const uint32_t c = *reinterpret_cast<const uint32_t*>(cls_s + (j - lo));
            uint32_t k[4] = {merge(c & 255, o.x), merge((c >> 8) & 255, o.y), merge((c >> 16) & 255, o.z), merge(c >> 24, o.w)};
#pragma unroll
            for (int i = 1; i < 4; ++i)
                if (j + i >= whi) k[i] = EV_OUT;
            *reinterpret_cast<uint4*>(ord_s + (j - lo)) = make_uint4(k[0], k[1], k[2], k[3]);
        }

    // `need` rows are still to be taken among the `left` ones that agree with the digits so far (bits `above` of `cut`)
    int need = keep - (cut_class < 2 ? n2 : 0) - (cut_class < 1 ? n1 : 0), left = cut_class == 2 ? n2 : cut_class == 1 ? n1 : L - n2 - n1;
    int bits = 32 - __clz((int)(o_min ^ o_max));        // that may differ
    uint32_t above = bits == 32 ? 0u : ~0u << bits, cut = o_min & above;
    for (int digit = 0; bits > 0 && left > EV_CAND; ++digit) {
        const int shift = bits > 8 ? bits - 8 : 0;
        const uint32_t mask = bits > 8 ? 255u : (1u << bits) - 1;
        for (int i = tid; i < 256 * EV_COLS / 4; i += EV_THREADS) reinterpret_cast<int4*>(&sm.hist[0][0])[i] = make_int4(0, 0, 0, 0);
        __syncthreads();
        for (int j = wlo + 4 * lane; j < whi; j += 128) {
            uint32_t k[4];
            keys(j, k);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((k[i] & above) == cut && k[i] != EV_OUT && k[i] != EV_IN) atomicAdd(&sm.hist[(k[i] >> shift) & mask][lane % EV_COLS], 1);
        }
        __syncthreads();
        if (tid < 256) {                                // (rotated: neighbouring bins start in other banks)
            int x = 0;
#pragma unroll
            for (int i = 0; i < EV_COLS; ++i) x += sm.hist[tid][(i + (tid >> 1)) % EV_COLS];
            sm.tot[digit & 1][tid] = x;
        }
        cluster_barrier(C);
        const int* totals = sm.tot[digit & 1];
        if (C > 1) {
            if (tid < 256) {
                int x = 0;
                for (int r = 0; r < C; ++r) x += ld_cluster(&sm.tot[digit & 1][tid], r);
                sm.sum[tid] = x;
            }
            __syncthreads();
            totals = sm.sum;                            // (written again behind the next digit's barriers)
        }
        // the bin, counted from the top, in which the need-th row lies: eight bins a lane, every warp for itself
        int x[8], t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i] = totals[255 - 8 * lane - i]; t += x[i]; }
        int inc = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(all, inc, o);
            if (lane >= o) inc += y;
        }
        int before = inc - t, bin = -1, n_need = 0, n_left = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (before < need && before + x[i] >= need) { bin = 255 - 8 * lane - i; n_need = need - before; n_left = x[i]; }
            before += x[i];
        }
        const int src = __ffs(__ballot_sync(all, bin >= 0)) - 1;
        cut |= (uint32_t)__shfl_sync(all, bin, src) << shift;
        need = __shfl_sync(all, n_need, src);
        left = __shfl_sync(all, n_left, src);
        above |= mask << shift;
        bits = shift;
    }
    // the last row that stays: key `cut`, row `cut_row`.  Few rows left: each is compared with all the others.
    const bool ranked = left <= EV_CAND;
    int cut_row = -1;
    if (ranked) {
        if (tid == 0) sm.found[2] = 0;
        __syncthreads();
        for (int j = wlo + 4 * lane; j < whi; j += 128) {
            uint32_t k[4];
            keys(j, k);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((k[i] & above) == cut && k[i] != EV_OUT && k[i] != EV_IN) sm.cand[atomicAdd(&sm.found[2], 1)] = make_uint2(~(uint32_t)(j + i), k[i]);
        }
        __syncthreads();
        if (C > 1) {
            if (tid == 0) sm.xch[3][0] = sm.found[2];
            cluster_barrier(C);
        }
        unsigned long long me = 0;
        if (tid < left) {
            uint2 c;
            if (C == 1) c = sm.cand[tid];
            else {
                int r = 0, at = tid;
                for (int n = ld_cluster(&sm.xch[3][0], 0); r + 1 < C && at >= n; n = ld_cluster(&sm.xch[3][0], r)) { at -= n; ++r; }
                c.x = (uint32_t)ld_cluster(reinterpret_cast<const int*>(&sm.cand[at].x), r); c.y = (uint32_t)ld_cluster(reinterpret_cast<const int*>(&sm.cand[at].y), r);
            }
            me = ((unsigned long long)c.y << 32) | c.x;
            sm.all[tid] = me;
        }
        __syncthreads();
        if (tid < left) {
            int before = 0;
#pragma unroll 8
            for (int i = 0; i < left; ++i) before += sm.all[i] > me;
            if (before == need - 1) { sm.found[0] = (int)(me >> 32); sm.found[1] = (int)~(uint32_t)me; }
        }
        __syncthreads();
        cut = (uint32_t)sm.found[0]; cut_row = sm.found[1];
    }
    // more equal weights than that: the first `need` of them, in row order
    int ties = 0;
    if (!ranked) {
        int mine = 0;
        for (int j = wlo + 4 * lane; j < whi; j += 128) {
            uint32_t k[4];
            keys(j, k);
#pragma unroll
            for (int i = 0; i < 4; ++i) mine += k[i] == cut;
        }
        mine = __reduce_add_sync(all, mine);
        if (lane == 0) sm.warp_a[warp] = mine;
        __syncthreads();
        int total;
        ties = over_warps(sm.warp_a, total);
        if (C > 1) {
            if (tid == 0) sm.xch[1][0] = total;
            cluster_barrier(C);
            for (int r = 0; r < rank; ++r) ties += ld_cluster(&sm.xch[1][0], r);
        }
        __syncthreads();                                // warp_a has been read
    }
    // of a bit per row (four a lane): the rows before this lane's, and all of the warp's
    auto before_lane = [&](uint32_t bits, int& total) -> int {
        int n = 0;
        total = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned bal = __ballot_sync(all, (bits >> i) & 1);
            n += __popc(bal & below); total += __popc(bal);
        }
        return n;
    };
    // who stays, a bit per row of this lane (whole warp: j of lanes behind the last row too); `t` counts the ties before
    auto decide = [&](int j, int& t) -> uint32_t {
        uint32_t k[4] = {EV_OUT, EV_OUT, EV_OUT, EV_OUT}, in = 0, tie = 0;
        if (j < whi) keys(j, k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            in |= (uint32_t)(k[i] > cut) << i;
            tie |= (uint32_t)(k[i] == cut && j + i < whi) << i;
        }
        if (ranked) {
#pragma unroll
            for (int i = 0; i < 4; ++i) in |= (uint32_t)(((tie >> i) & 1) && j + i <= cut_row) << i;
        } else {
            int total, r = before_lane(tie, total) + t;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((tie >> i) & 1) { in |= (uint32_t)(r < need) << i; ++r; }
            t += total;
        }
        return in;
    };
    // of its rows: those below `keep`, and those that exist
    auto low = [&](int j) -> uint32_t { const int n = keep - j; return n <= 0 ? 0u : n >= 4 ? 15u : (1u << n) - 1; };
    auto real = [&](int j) -> uint32_t { const int n = whi - j; return n <= 0 ? 0u : n >= 4 ? 15u : (1u << n) - 1; };
    int freed = 0, late = 0;
    {
        int t = ties;
        for (int j = wlo + 4 * lane; j - 4 * lane < whi; j += 128) {
            const uint32_t in = decide(j, t), ok = real(j), lw = low(j);
            freed += __popc(ok & lw & ~in); late += __popc(ok & ~lw & in);
        }
    }
    freed = __reduce_add_sync(all, freed); late = __reduce_add_sync(all, late);
    if (lane == 0) { sm.warp_a[warp] = freed; sm.warp_b[warp] = late; }
    __syncthreads();
    int moved, all_late;
    int at_f = over_warps(sm.warp_a, moved), at_l = over_warps(sm.warp_b, all_late);
    if (C > 1) {
        if (tid == 0) { sm.xch[2][0] = moved; sm.xch[2][1] = all_late; }
        cluster_barrier(C);
        moved = 0;
        for (int r = 0; r < C; ++r) {
            const int a = ld_cluster(&sm.xch[2][0], r), c = ld_cluster(&sm.xch[2][1], r);
            if (r < rank) { at_f += a; at_l += c; }
            moved += a;
        }
    }
    int* list = p.list + base;
    for (int j = wlo + 4 * lane; j - 4 * lane < whi; j += 128) {
        const uint32_t in = decide(j, ties), ok = real(j), lw = low(j);
        uint32_t gone = ok & lw & ~in, back = ok & ~lw & in;
        int total, at = at_f + before_lane(gone, total);
        at_f += total;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((gone >> i) & 1) list[at++] = j + i;
        at = at_l + before_lane(back, total);
        at_l += total;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((back >> i) & 1) list[p.v.cap - 1 - at++] = j + i;
    }
    if (tid == 0 && rank == 0) p.count[pair] = moved;
    if (C > 1) cluster_barrier(C);                      // nobody leaves while its shared memory is read
}

// A warp takes up to 32 rows of the list (eight where there are few rows for many warps): its lanes look up places and pages of a row
// each, then the rows are copied four at a time (eight: more registers, a batch of 64 sequences 94 -> 101 us).
constexpr int MV_WARPS = 8;

template <int D>
__global__ void __launch_bounds__(MV_WARPS * 32) evict_move_kernel(const EvictParams p) {
    constexpr int LPR = D / 8, LANES = 2 * LPR, TOGETHER = 32 / LANES, FLIGHT = 4;      // 16-byte units of a row; lanes of a row of K and one of V
    pdl_wait();
    pdl_release();
    const int status0 = *p.v.status;
    const int pair = blockIdx.x / p.move_blocks, block = blockIdx.x % p.move_blocks, b = pair / p.v.Hkv, h = pair % p.v.Hkv;
    const int n = p.count[pair], lane = threadIdx.x & 31;
    if (status0 != 0) return;
    if (block == 0 && h == 0 && threadIdx.x == 0) p.lens_out[b] = min(p.v.lens[b], p.keep);
    const size_t base = (size_t)pair * p.v.cap;
    const int unit = lane % LANES, which = lane / LANES;
    __nv_bfloat16* T = (unit < LPR ? p.K : p.V) + (size_t)h * D + (unit % LPR) * 8;
    const size_t pitch = (size_t)p.v.Hkv * D;
    for (int i0 = (block * MV_WARPS + (threadIdx.x >> 5)) * p.move_rows; i0 < n; i0 += p.move_blocks * MV_WARPS * p.move_rows) {
        const int i = i0 + lane, rows = min(p.move_rows, n - i0);
        int to = -1, from = -1;
        if (lane < rows) {
            const int dst = p.list[base + i], src = p.list[base + p.v.cap - 1 - i];
            const float m = p.mass_in[base + src];
            const int x = p.pos_in[base + src];
            to = (int)load_pool_row(p.v, b, dst); from = (int)load_pool_row(p.v, b, src);
            if (from < 0) to = -1;
            p.mass_out[base + dst] = m;
            p.pos_out[base + dst] = x;
        }
        for (int k0 = 0; k0 < rows; k0 += FLIGHT * TOGETHER) {
            uint4 x[FLIGHT];
            int t[FLIGHT];
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) {
                const int k = k0 + f * TOGETHER + which;                    // (below 32; rows that do not exist have no place)
                t[f] = __shfl_sync(0xffffffffu, to, k & 31);
                const int s = __shfl_sync(0xffffffffu, from, k & 31);
                if (t[f] >= 0) x[f] = *reinterpret_cast<const uint4*>(T + (size_t)s * pitch);
            }
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f)
                if (t[f] >= 0) *reinterpret_cast<uint4*>(T + (size_t)t[f] * pitch) = x[f];
        }
    }
}

}  // namespace
}  // namespace seka

extern "C" seka_status seka_evict_cache(const seka_paged_shape* shape, void* K_pages, void* V_pages, const float* mass_in, float* mass_out,
                                        const int32_t* pos_in, int32_t* pos_out, const uint8_t* protect, int32_t protect_len,
                                        const int32_t* next_pos, int32_t keep, int32_t recent, int32_t* lens_out,
                                        void* workspace, size_t workspace_bytes, void* cuda_stream) {
    using namespace seka;
    seka_status stc = validate_paged(shape);
    if (stc != SEKA_OK) return stc;
    if (keep < 1 || recent < 0 || protect_len < 0) return SEKA_ERR_INVALID_ARG;
    if (shape->batch == 0) return SEKA_OK;
    if (!mass_in || !mass_out || !pos_in || !pos_out || !next_pos || !lens_out || ((!K_pages || !V_pages) && shape->n_pages > 0))
        return SEKA_ERR_INVALID_ARG;
    if (((uintptr_t)K_pages | (uintptr_t)V_pages | (uintptr_t)mass_in | (uintptr_t)mass_out | (uintptr_t)pos_in | (uintptr_t)pos_out) & 15)
        return SEKA_ERR_INVALID_ARG;
    stc = check_paged_call(shape, workspace, workspace_bytes);
    if (stc != SEKA_OK) return stc;
    const PagedLayout w = paged_layout(shape);
    char* ws = static_cast<char*>(workspace);
    EvictParams p;
    p.v = paged_view(shape, workspace);
    p.K = static_cast<__nv_bfloat16*>(K_pages); p.V = static_cast<__nv_bfloat16*>(V_pages);
    p.mass_in = mass_in; p.mass_out = mass_out; p.pos_in = pos_in; p.pos_out = pos_out;
    p.protect = protect_len > 0 ? protect : nullptr; p.protect_len = protect_len;
    p.next_pos = next_pos; p.keep = keep; p.recent = recent; p.lens_out = lens_out;
    p.count = reinterpret_cast<int*>(ws + w.evict_count_off);
    p.list = reinterpret_cast<int*>(ws + w.evict_list_off);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const unsigned pairs = (unsigned)shape->batch * (unsigned)shape->n_kv_heads;
    int n_sm = 0;
    if (!device_info(&n_sm)) return SEKA_ERR_CUDA;
    // CTAs of a pair: more while they still find SMs and have 2048 rows each (a cache may be filled to its last page).  One context of 65536
    // rows: 60 us, 239 with one CTA a pair; 8 of 8192: 51 and 55.
    p.cluster = 1;
    while (p.cluster < EV_MAX_CLUSTER && 2LL * p.cluster * pairs <= 2LL * n_sm && p.v.cap > 4 * 1024 * p.cluster) p.cluster *= 2;
    const int lanes = p.cluster * EV_WARPS * 128;
    const long long rows = ((long long)p.v.cap + lanes - 1) / lanes * (EV_WARPS * 128);     // most rows of a CTA
    // longer: ranks are formed again in every pass (one context of 65536 that way: 82 us, 60 cached; 64 of 1024 to 4096: 92 and 80)
    p.cached = rows <= EV_MAX_CACHED ? (int)rows : 0;
    const size_t bytes = sizeof(EvSmem) + (size_t)p.cached * 5;
    // the limit belongs to the function, not to the launch: always the most that any call asks for, so that a call of another host thread
    // between this line and the launch does not lower it
    if (cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)EV_MAX_BYTES) != cudaSuccess) return SEKA_ERR_CUDA;
    stc = launch_cluster(true, (unsigned)p.cluster, evict_select_kernel, dim3(pairs * (unsigned)p.cluster), EV_THREADS, bytes, st, p);
    if (stc != SEKA_OK) return stc;
    const int D = shape->head_dim;
    const long long most = p.v.cap - keep < keep ? p.v.cap - keep : keep;          // rows of a pair that can move
    const long long fill = (16LL * n_sm + pairs - 1) / pairs;
    // rows of a warp: eight while that leaves fewer than eight warps per SM, up to 32 (64 contexts 80 us, 86 with eight always; one of
    // 1500 14.2, 16.4 with 32 always; one of 65536 60, 58 with eight)
    p.move_rows = 32;
    while (p.move_rows > 8 && (long long)pairs * most < 8LL * n_sm * p.move_rows) p.move_rows /= 2;
    long long blocks = most > 0 ? (most + MV_WARPS * p.move_rows - 1) / (MV_WARPS * p.move_rows) : 1;
    if (blocks > fill) blocks = fill;
    p.move_blocks = (int)blocks;
    const dim3 grid(pairs * (unsigned)blocks);
    return D == 128 ? launch_kernel(true, evict_move_kernel<128>, grid, MV_WARPS * 32, 0, st, p)
                    : launch_kernel(true, evict_move_kernel<64>, grid, MV_WARPS * 32, 0, st, p);
}
