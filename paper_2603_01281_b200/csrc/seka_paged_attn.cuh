// Attention of new tokens over a paged cache: what its two kernels and the merge of cut units share.
#pragma once

#include "seka_kernels.h"
#include "seka_paged_sched.cuh"

namespace seka {

struct PagedAttnParams {
    PagedView v;
    StepGeo geo;
    const __nv_bfloat16* Q;
    __nv_bfloat16* O;
    float* lse;                 // [T, Hq] or null
    float scale_log2;
    int tile_tokens;            // new tokens of a tile of rows (geo.tp: of a unit)
    int n_shares;
    CutRecord* cuts;            // [n_shares]
    float* part_ml;             // [n_shares, 2, rows of a unit, 2]
    float* part_o;              // [n_shares, 2, rows of a unit, D]
};

// many rows: tcgen05 tiles
template <int D> seka_status launch_paged_tiles(const PagedAttnParams& p, const void* Q, const void* K, const void* V, int page_size, cudaStream_t st);

}  // namespace seka
