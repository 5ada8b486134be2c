// Eviction: every (sequence, KV head) of more than `keep` cached rows is cut to the `keep` that come first by (class, weight, row).
//
//   evict_select_kernel   a cluster of 1 to 8 CTAs per (sequence, KV head), a run of consecutive rows each.  A row's rank is its class (2:
//                         recent, 1: highlighted, 0) above its weight mapped to 32 bits whose unsigned order is the order of the
//                         weights; both are formed once and kept in shared memory (where they fit).  The class that the keep-th row
//                         belongs to follows from the counts, its weight is found in four digits of eight bits: a CTA's
//                         histogram has 16 columns (a warp's updates meet in pairs at most), the CTAs add their totals through
//                         distributed shared memory.  Then ties by row, and the lists of the freed rows below `keep` and the
//                         kept ones behind, every warp on consecutive rows so that ranks come from ballots.
//   evict_move_kernel     copies K, V, weight and position of the kept rows behind into the freed rows.
// What is kept below `keep` does not move: a cache that is cut often, by a little each time, moves only that little.  Sources lie at or
// behind `keep`, destinations below it, so the copies need no order.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {
namespace {

constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_MAX_CLUSTER = 8;
constexpr int EV_COLS = 16;                             // columns of the histogram (lanes l and l + 16 share one); 32 leave too little room for four CTAs per SM
constexpr int EV_FLIGHT = 8;                            // rows of a lane whose loads are in flight together
constexpr int EV_MAX_CACHED = 40 * 1024;                // rows of a CTA whose ranks fit in shared memory beside the histogram

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
    int move_blocks;            // blocks of a (sequence, KV head) in the second launch
    int* lens_out;
    int* count;                 // [B, Hkv] rows that move
    int* list;                  // [B, Hkv, cap]
};

// weight -> 32 bits in the same order (NaN first, then -inf; the two zeros equal)
SEKA_HD uint32_t mass_order(float x, uint32_t bits) {
    if (x != x) return 0u;
    if (x == 0.f) return 0x80000000u;
    return (bits & 0x80000000u) ? ~bits : bits | 0x80000000u;
}

struct EvSmem {
    int hist[256][EV_COLS];
    int tot[2][256];            // this CTA's totals of a digit (read by the cluster; two, so that one barrier per digit is enough)
    int sum[256];
    int xch[3][4];              // what the CTAs tell each other: class counts and status; ties; freed and late rows
    int warp_a[EV_WARPS], warp_b[EV_WARPS];
    int found[2];
};

__device__ __forceinline__ int ld_cluster(const int* local, int rank) {
    uint32_t a;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
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
    // rows of this CTA [lo, hi), of this warp [wlo, whi): consecutive, multiples of 32
    const int wrows = ((L + C * EV_WARPS - 1) / (C * EV_WARPS) + 31) & ~31, chunk = wrows * EV_WARPS;
    const long long lo_l = (long long)rank * chunk;
    const int lo = (int)(lo_l < L ? lo_l : L), hi = L - lo < chunk ? L : lo + chunk;
    const int wlo = hi - lo < warp * wrows ? hi : lo + warp * wrows, whi = hi - wlo < wrows ? hi : wlo + wrows;
    const bool cached = chunk <= p.cached;
    const long long recent_from = (long long)p.next_pos[b] - p.recent;
    auto class_of = [&](int x, int flag) -> int { return (long long)x >= recent_from ? 2 : flag; };
    // where the flag of a position lies (any valid address where it has none), and whether it has one
    const uint8_t* prot = p.protect != nullptr ? p.protect + (size_t)b * p.protect_len : nullptr;
    auto flag_of = [&](int x) -> int {
        const bool inside = x >= 0 && x < p.protect_len;
        const int f = prot != nullptr ? (int)prot[inside ? x : 0] : 0;
        return inside && f != 0 ? 1 : 0;
    };
    auto get = [&](int j, uint32_t& o) -> int {         // class, and the weight's order
        if (cached) { o = ord_s[j - lo]; return cls_s[j - lo]; }
        const float m = mass[j];
        const int x = pos[j];
        o = mass_order(m, __float_as_uint(m));
        return class_of(x, flag_of(x));
    };
    // weights and positions once from memory, several rows' loads in flight; rows below `keep` are passed on as they are (what is freed
    // is written over by the second launch)
    int n2 = 0, n1 = 0;
    const bool copy_m = p.mass_out != p.mass_in, copy_p = p.pos_out != p.pos_in;
    for (int j0 = wlo + lane; j0 - lane < whi; j0 += 32 * EV_FLIGHT) {
        float m[EV_FLIGHT];
        int x[EV_FLIGHT], f[EV_FLIGHT];
#pragma unroll
        for (int i = 0; i < EV_FLIGHT; ++i) {
            const int j = min(j0 + 32 * i, whi - 1);    // (the last row again where there is none)
            m[i] = mass[j]; x[i] = pos[j];
        }
#pragma unroll
        for (int i = 0; i < EV_FLIGHT; ++i) f[i] = flag_of(x[i]);
#pragma unroll
        for (int i = 0; i < EV_FLIGHT; ++i) {
            const int j = j0 + 32 * i;
            if (j >= whi) continue;
            const int c = class_of(x[i], f[i]);
            if (cached) { ord_s[j - lo] = mass_order(m[i], __float_as_uint(m[i])); cls_s[j - lo] = (uint8_t)c; }
            n2 += c == 2; n1 += c == 1;
            if (j < keep) {
                if (copy_m) p.mass_out[base + j] = m[i];
                if (copy_p) p.pos_out[base + j] = x[i];
            }
        }
    }
    n2 = __reduce_add_sync(all, n2); n1 = __reduce_add_sync(all, n1);
    if (lane == 0) { sm.warp_a[warp] = n2; sm.warp_b[warp] = n1; }
    __syncthreads();
    if (tid == 0) {
        int a = 0, c = 0;
        for (int w = 0; w < EV_WARPS; ++w) { a += sm.warp_a[w]; c += sm.warp_b[w]; }
        sm.xch[0][0] = a; sm.xch[0][1] = c; sm.xch[0][2] = status0;
    }
    cluster_barrier();
    n2 = 0; n1 = 0;
    int bad = 0;
    for (int r = 0; r < C; ++r) { n2 += ld_cluster(&sm.xch[0][0], r); n1 += ld_cluster(&sm.xch[0][1], r); bad |= ld_cluster(&sm.xch[0][2], r); }
    if (bad) { cluster_barrier(); return; }             // an earlier launch gave up (decided together: nobody leaves while others read)
    const int cut_class = n2 >= keep ? 2 : n2 + n1 >= keep ? 1 : 0;
    // `need` rows are still to be taken among those of the class that agree with the digits so far
    int need = keep - (cut_class < 2 ? n2 : 0) - (cut_class < 1 ? n1 : 0);
    uint32_t cut = 0;
    for (int digit = 0; digit < 4; ++digit) {
        const int shift = 24 - 8 * digit;
        const uint32_t above = digit == 0 ? 0u : 0xffffffffu << (shift + 8);
        for (int i = tid; i < 256 * EV_COLS / 4; i += EV_THREADS) reinterpret_cast<int4*>(&sm.hist[0][0])[i] = make_int4(0, 0, 0, 0);
        __syncthreads();
#pragma unroll 4
        for (int j = wlo + lane; j < whi; j += 32) {
            uint32_t o;
            const int c = get(j, o);
            if (c == cut_class && (o & above) == cut) atomicAdd(&sm.hist[(o >> shift) & 255][lane % EV_COLS], 1);
        }
        __syncthreads();
        if (tid < 256) {                                // (rotated: neighbouring bins start in other banks)
            int x = 0;
#pragma unroll
            for (int i = 0; i < EV_COLS; ++i) x += sm.hist[tid][(i + (tid >> 1)) % EV_COLS];
            sm.tot[digit & 1][tid] = x;
        }
        cluster_barrier();
        if (tid < 256) {
            int x = 0;
            for (int r = 0; r < C; ++r) x += ld_cluster(&sm.tot[digit & 1][tid], r);
            sm.sum[tid] = x;
        }
        __syncthreads();
        // the bin, counted from the top, in which the need-th row lies: eight bins a lane
        if (warp == 0) {
            int x[8], t = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) { x[i] = sm.sum[255 - 8 * lane - i]; t += x[i]; }
            int inc = t;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(all, inc, o);
                if (lane >= o) inc += y;
            }
            int before = inc - t;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < need && before + x[i] >= need) { sm.found[0] = 255 - 8 * lane - i; sm.found[1] = need - before; }
                before += x[i];
            }
        }
        __syncthreads();
        cut |= (uint32_t)sm.found[0] << shift;
        need = sm.found[1];
        // (found and sum are written again behind the next digit's barriers)
    }
    // ties: the first `need` rows, in row order, of those whose rank is the cut's
    int mine = 0;
    for (int j = wlo + lane; j - lane < whi; j += 32) {
        uint32_t o = 0;
        const bool tie = j < whi && get(j, o) == cut_class && o == cut;
        mine += __popc(__ballot_sync(all, tie));
    }
    if (lane == 0) sm.warp_a[warp] = mine;
    __syncthreads();
    if (tid == 0) {
        int a = 0;
        for (int w = 0; w < EV_WARPS; ++w) a += sm.warp_a[w];
        sm.xch[1][0] = a;
    }
    cluster_barrier();
    int ties = 0;
    for (int r = 0; r < rank; ++r) ties += ld_cluster(&sm.xch[1][0], r);
    for (int w = 0; w < warp; ++w) ties += sm.warp_a[w];
    // who is in; `t` counts the ties before the rows of this step
    auto decide = [&](int j, int& t) -> bool {
        uint32_t o = 0;
        int c = -1;
        if (j < whi) c = get(j, o);
        const bool tie = c == cut_class && o == cut;
        const unsigned bal = __ballot_sync(all, tie);
        const bool in = c > cut_class || (c == cut_class && o > cut) || (tie && t + __popc(bal & below) < need);
        t += __popc(bal);
        return in;
    };
    int freed = 0, late = 0;
    {
        int t = ties;
        for (int j = wlo + lane; j - lane < whi; j += 32) {
            const bool in = decide(j, t);
            freed += __popc(__ballot_sync(all, j < whi && j < keep && !in));
            late += __popc(__ballot_sync(all, j < whi && j >= keep && in));
        }
    }
    __syncthreads();                                    // warp_a has been read
    if (lane == 0) { sm.warp_a[warp] = freed; sm.warp_b[warp] = late; }
    __syncthreads();
    if (tid == 0) {
        int a = 0, c = 0;
        for (int w = 0; w < EV_WARPS; ++w) { a += sm.warp_a[w]; c += sm.warp_b[w]; }
        sm.xch[2][0] = a; sm.xch[2][1] = c;
    }
    cluster_barrier();
    int at_f = 0, at_l = 0, moved = 0;
    for (int r = 0; r < C; ++r) {
        const int a = ld_cluster(&sm.xch[2][0], r), c = ld_cluster(&sm.xch[2][1], r);
        if (r < rank) { at_f += a; at_l += c; }
        moved += a;
    }
    for (int w = 0; w < warp; ++w) { at_f += sm.warp_a[w]; at_l += sm.warp_b[w]; }
    int* list = p.list + base;
    for (int j = wlo + lane; j - lane < whi; j += 32) {
        const bool in = decide(j, ties), gone = j < whi && j < keep && !in, back = j < whi && j >= keep && in;
        const unsigned bf = __ballot_sync(all, gone), bl = __ballot_sync(all, back);
        if (gone) list[at_f + __popc(bf & below)] = j;
        if (back) list[p.v.cap - 1 - (at_l + __popc(bl & below))] = j;
        at_f += __popc(bf); at_l += __popc(bl);
    }
    if (tid == 0 && rank == 0) p.count[pair] = moved;
    cluster_barrier();                                  // nobody leaves while its shared memory is read
}

// A warp takes 32 rows of the list: its lanes look up places and pages of a row each, then the rows are copied eight at a time.
constexpr int MV_WARPS = 8;

template <int D>
__global__ void __launch_bounds__(MV_WARPS * 32) evict_move_kernel(const EvictParams p) {
    constexpr int LPR = D / 8, LANES = 2 * LPR, TOGETHER = 32 / LANES, FLIGHT = 8;      // 16-byte units of a row; lanes of a row of K and one of V
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
    for (int i0 = (block * MV_WARPS + (threadIdx.x >> 5)) * 32; i0 < n; i0 += p.move_blocks * MV_WARPS * 32) {
        const int i = i0 + lane, rows = min(32, n - i0);
        int to = -1, from = -1;
        if (i < n) {
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
    if (((uintptr_t)K_pages | (uintptr_t)V_pages) & 15) return SEKA_ERR_INVALID_ARG;
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
    // CTAs of a pair: more while they still find SMs and have 1024 rows each (a cache may be filled to its last page)
    p.cluster = 1;
    while (p.cluster < EV_MAX_CLUSTER && 2LL * p.cluster * pairs <= 2LL * n_sm && p.v.cap > 2 * 1024 * p.cluster) p.cluster *= 2;
    const int lanes = p.cluster * EV_WARPS * 32;
    const long long rows = ((long long)p.v.cap + lanes - 1) / lanes * (EV_WARPS * 32);      // most rows of a CTA
    p.cached = rows <= EV_MAX_CACHED ? (int)rows : 0;                                       // longer: ranks are formed again in every pass
    const size_t bytes = sizeof(EvSmem) + (size_t)p.cached * 5;
    if (cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return SEKA_ERR_CUDA;
    stc = launch_cluster(true, (unsigned)p.cluster, evict_select_kernel, dim3(pairs * (unsigned)p.cluster), EV_THREADS, bytes, st, p);
    if (stc != SEKA_OK) return stc;
    const int D = shape->head_dim;
    const long long most = p.v.cap - keep < keep ? p.v.cap - keep : keep;          // rows of a pair that can move
    long long blocks = most > 0 ? (most + MV_WARPS * 32 - 1) / (MV_WARPS * 32) : 1;
    const long long fill = (16LL * n_sm + pairs - 1) / pairs;
    if (blocks > fill) blocks = fill;
    p.move_blocks = (int)blocks;
    const dim3 grid(pairs * (unsigned)blocks);
    return D == 128 ? launch_kernel(true, evict_move_kernel<128>, grid, MV_WARPS * 32, 0, st, p)
                    : launch_kernel(true, evict_move_kernel<64>, grid, MV_WARPS * 32, 0, st, p);
}
