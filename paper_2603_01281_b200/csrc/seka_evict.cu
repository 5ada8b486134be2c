// Eviction: every (sequence, KV head) of more than `keep` cached rows is cut to the `keep` that come first by (class, weight, row).
//
//   evict_select_kernel   one CTA per (sequence, KV head).  A row's rank is a number of 34 bits: its class (2: recent, 1: highlighted,
//                         0) above its weight mapped so that unsigned order is the order of the weights.  The number of the
//                         keep-th row is found digit by digit (the class, then 11, 11 and 10 bits) from histograms in shared memory;
//                         a last pass in row order lists the freed rows below `keep` and the kept ones behind, ties by
//                         row, and writes weights and positions.
//   evict_move_kernel     copies K and V of the kept rows behind into the freed rows, a warp per row.
// What is kept below `keep` does not move: a cache that is cut often, by a little each time, moves only that little.  Sources lie at or
// behind `keep`, destinations below it, so the copies need no order.
#include <math.h>

#include "seka_kernels.h"
#include "seka_paged.cuh"

namespace seka {
namespace {

constexpr int EV_THREADS = 1024, EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;

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

__device__ __forceinline__ int block_sum_scan(int x, int* warp_tot, int& total) {      // exclusive scan over the block
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();                        // warp_tot of the scan before has been read
    if (lane == 31) warp_tot[warp] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < EV_WARPS; ++w) {
        if (w < warp) before += warp_tot[w];
        total += warp_tot[w];
    }
    return before + inc - x;
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const EvictParams p) {
    __shared__ int hist[EV_BINS];
    __shared__ int warp_tot[EV_WARPS];
    __shared__ int found[2];
    const int b = blockIdx.x / p.v.Hkv, tid = threadIdx.x;
    pdl_wait();
    pdl_release();
    if (*p.v.status != 0) return;
    int L = p.v.lens[b];
    if (L < 0 || L > p.v.cap) {
        if (tid == 0) { report_invalid(p.v.status, kWhereSeq); p.count[blockIdx.x] = 0; }
        return;
    }
    const size_t base = (size_t)blockIdx.x * p.v.cap;
    const float* mass = p.mass_in + base;
    const int* pos = p.pos_in + base;
    const int keep = p.keep;
    if (L <= keep) {
        for (int j = tid; j < L; j += EV_THREADS) {
            if (p.mass_out != p.mass_in) p.mass_out[base + j] = mass[j];
            if (p.pos_out != p.pos_in) p.pos_out[base + j] = pos[j];
        }
        if (tid == 0) p.count[blockIdx.x] = 0;
        return;
    }
    const long long recent_from = (long long)p.next_pos[b] - p.recent;
    auto klass = [&](int j) -> int {
        const int x = pos[j];
        if ((long long)x >= recent_from) return 2;
        return (p.protect != nullptr && x >= 0 && x < p.protect_len && p.protect[(size_t)b * p.protect_len + x] != 0) ? 1 : 0;
    };
    auto order = [&](int j) -> uint32_t { const float x = mass[j]; return mass_order(x, __float_as_uint(x)); };

    // digit 0: the class; digits 1 to 3: the weight.  `need` rows are still to be taken among those that agree with the digits so far.
    int need = keep, cut_class = 0;
    uint32_t cut = 0;
    for (int digit = 0; digit < 4; ++digit) {
        const int shift = digit == 1 ? 21 : digit == 2 ? 10 : 0, bins = digit == 0 ? 3 : digit == 3 ? 1024 : 2048;
        const uint32_t above = digit <= 1 ? 0u : digit == 2 ? 0xffe00000u : 0xfffffc00u;
        for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < L; j += EV_THREADS) {
            const int c = klass(j);
            if (digit == 0) { atomicAdd(&hist[c], 1); continue; }
            if (c != cut_class) continue;
            const uint32_t o = order(j);
            if ((o & above) == (cut & above)) atomicAdd(&hist[(o >> shift) & (uint32_t)(bins - 1)], 1);
        }
        __syncthreads();
        // the bin, counted from the top, in which the need-th row lies: two bins a thread, highest first
        int x0 = 0, x1 = 0;
        const int i0 = EV_BINS - 1 - 2 * tid, i1 = i0 - 1;
        x0 = hist[i0]; x1 = hist[i1];
        int total;
        const int before = block_sum_scan(x0 + x1, warp_tot, total);
        if (before < need && before + x0 >= need) { found[0] = i0; found[1] = need - before; }
        else if (before + x0 < need && before + x0 + x1 >= need) { found[0] = i1; found[1] = need - before - x0; }
        __syncthreads();
        need = found[1];
        if (digit == 0) cut_class = found[0];
        else cut |= (uint32_t)found[0] << shift;
        __syncthreads();
    }
    // in row order: ties by row, freed rows below `keep` to the front of the list, kept rows behind to its back
    int* list = p.list + base;
    int ties = 0, freed = 0, late = 0;
    for (int j0 = 0; j0 < L; j0 += EV_THREADS) {
        const int j = j0 + tid;
        bool in = false, tie = false;
        if (j < L) {
            const int c = klass(j);
            if (c == cut_class) { const uint32_t o = order(j); in = o > cut; tie = o == cut; }
            else in = c > cut_class;
        }
        int total;
        const int rank = ties + block_sum_scan(tie ? 1 : 0, warp_tot, total);
        ties += total;
        if (tie && rank < need) in = true;
        const bool gone = j < keep && !in, back = j >= keep && j < L && in;
        const int at_f = freed + block_sum_scan(gone ? 1 : 0, warp_tot, total);
        freed += total;
        const int at_b = late + block_sum_scan(back ? 1 : 0, warp_tot, total);
        late += total;
        if (gone) list[at_f] = j;
        if (back) list[p.v.cap - 1 - at_b] = j;
        if (j < keep && in) {
            if (p.mass_out != p.mass_in) p.mass_out[base + j] = mass[j];
            if (p.pos_out != p.pos_in) p.pos_out[base + j] = pos[j];
        }
    }
    __syncthreads();
    for (int i = tid; i < freed; i += EV_THREADS) {
        const int dst = list[i], src = list[p.v.cap - 1 - i];
        p.mass_out[base + dst] = mass[src];
        p.pos_out[base + dst] = pos[src];
    }
    if (tid == 0) p.count[blockIdx.x] = freed;
}

constexpr int MV_WARPS = 8;

template <int D>
__global__ void __launch_bounds__(MV_WARPS * 32) evict_move_kernel(const EvictParams p) {
    constexpr int LPR = D / 8;                          // lanes of a row of 16-byte units; K and V side by side fill a warp (d = 128)
    pdl_wait();
    pdl_release();
    if (*p.v.status != 0) return;
    const int pair = blockIdx.x / p.move_blocks, block = blockIdx.x % p.move_blocks, b = pair / p.v.Hkv, h = pair % p.v.Hkv;
    if (block == 0 && h == 0 && threadIdx.x == 0) p.lens_out[b] = min(p.v.lens[b], p.keep);
    const int n = p.count[pair];
    const int* list = p.list + (size_t)pair * p.v.cap;
    const int unit = threadIdx.x % (2 * LPR), per = MV_WARPS * 32 / (2 * LPR);
    __nv_bfloat16* T = unit < LPR ? p.K : p.V;
    const int e0 = (unit % LPR) * 8;
    for (int i = block * per + threadIdx.x / (2 * LPR); i < n; i += p.move_blocks * per) {
        const long long to = load_pool_row(p.v, b, list[i]), from = load_pool_row(p.v, b, list[p.v.cap - 1 - i]);
        if (to < 0 || from < 0) continue;
        *reinterpret_cast<uint4*>(T + ((size_t)to * p.v.Hkv + h) * D + e0) = *reinterpret_cast<const uint4*>(T + ((size_t)from * p.v.Hkv + h) * D + e0);
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
    stc = launch_kernel(true, evict_select_kernel, dim3(pairs), EV_THREADS, 0, st, p);
    if (stc != SEKA_OK) return stc;
    int n_sm = 0;
    if (!device_info(&n_sm)) return SEKA_ERR_CUDA;
    const int D = shape->head_dim, per = MV_WARPS * 32 / (D / 4);
    const long long most = p.v.cap - keep < keep ? p.v.cap - keep : keep;          // rows of a pair that can move
    long long blocks = most > 0 ? (most + per - 1) / per : 1;
    const long long fill = (8LL * n_sm + pairs - 1) / pairs;
    if (blocks > fill) blocks = fill;
    p.move_blocks = (int)blocks;
    const dim3 grid(pairs * (unsigned)blocks);
    return D == 128 ? launch_kernel(true, evict_move_kernel<128>, grid, MV_WARPS * 32, 0, st, p)
                    : launch_kernel(true, evict_move_kernel<64>, grid, MV_WARPS * 32, 0, st, p);
}
