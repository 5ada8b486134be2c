// Paged cache: what the kernels of the paged calls share (view of the cache, checks of what only the device knows, workspace).
#pragma once

#include "seka_common.cuh"

namespace seka {

struct PagedView {
    const int* table;           // [B, max_pages]
    const int* lens;            // [B] cached tokens, the new ones included
    const int* cu;              // [B + 1] or null
    int* status;
    int B, T, max_new, Hq, Hkv, G;
    int max_pages, n_pages, page_shift, cap;
};

// One sequence of a call: its new tokens are q0 .. q0 + n - 1 and the last n of its L cached ones.
struct PagedSeq {
    int q0, n, L;
    bool valid;                 // false: a length or an offset lies outside its range; the sequence is empty then
};

SEKA_HD PagedSeq check_seq(const PagedView& v, int q0, int q1, int L) {
    PagedSeq s;
    s.valid = q0 >= 0 && q1 >= q0 && q1 <= v.T && q1 - q0 <= v.max_new && L >= 0 && L <= v.cap;
    s.q0 = s.valid ? q0 : 0; s.n = s.valid ? q1 - q0 : 0; s.L = s.valid ? L : 0;
    return s;
}
SEKA_HD PagedSeq paged_seq(const PagedView& v, int b) {
    return check_seq(v, v.cu ? v.cu[b] : b * v.max_new, v.cu ? v.cu[b + 1] : (b + 1) * v.max_new, v.lens[b]);
}

// Pool row (page * page_size + offset) of cached token j (0 <= j < cap) of a sequence given the entry of its page; -1: no such page.
SEKA_HD long long pool_row(const PagedView& v, int page, int j) {
    if (page < 0 || page >= v.n_pages) return -1;
    return ((long long)page << v.page_shift) + (j & ((1 << v.page_shift) - 1));
}
SEKA_HD int table_entry(const PagedView& v, int b, int j) { return v.table[(long long)b * v.max_pages + (j >> v.page_shift)]; }

// Attention and accumulated weights: up to this many rows (new tokens x query heads of a KV head) of a sequence the few-row kernel runs, else
// the tile kernel.  It takes all that the few-row kernels hold: with 16 rows and 64 contexts of 1024 to 4096 tokens, 32/8 heads of 128,
// attention takes 127 us (tiles 150), weights 66 (163); one context of 4096 16.7 (19.9) and 7.8 (14.9).
constexpr int kFewRows = 16;
static inline bool few_rows(const seka_paged_shape* s) {
    return (long long)s->max_new * (s->n_q_heads / s->n_kv_heads) <= kFewRows;
}
// Shares of a launch (one per CTA: one CTA per SM in the tile kernel, two or three in the few-row kernel) and rows of a unit.  148 SMs;
// a device with fewer runs the same shares in more than one wave.
constexpr int kShareSms = 148;
static inline int attention_shares(const seka_paged_shape* s) { return few_rows(s) ? kShareSms * (s->head_dim == 128 ? 2 : 3) : kShareSms; }
static inline int unit_rows(const seka_paged_shape* s) { return few_rows(s) ? kFewRows : 256; }

// Workspace of the paged calls (one at a time): status block, then the lists of the eviction or the partial results of
// the attention or of the accumulated weights.
struct PagedLayout {
    size_t evict_count_off;     // int32 [B, Hkv]: rows that move
    size_t evict_list_off;      // int32 [B, Hkv, cap]: freed rows from the front, rows that take their place from the back
    size_t cut_off;             // CutRecord [shares]
    size_t part_ml_off;         // fp32 [shares, 2, rows, 2]: running maximum (log2 domain) and sum of the cut units of each share
    size_t part_o_off;          // fp32 [shares, 2, rows, d]: their outputs, not normalised
    size_t mass_part_off;       // fp32 [148, 2, 256]: weights of the cut units of each share
    size_t total;
};
static inline PagedLayout paged_layout(const seka_paged_shape* s) {
    PagedLayout w;
    const size_t pairs = (size_t)s->batch * s->n_kv_heads, cap = (size_t)s->max_pages * s->page_size;
    w.evict_count_off = 1024;
    w.evict_list_off = w.evict_count_off + align_up(pairs * 4 + 4, 256);
    const size_t evict = w.evict_list_off + align_up(pairs * cap * 4 + 4, 256);
    const size_t shares = (size_t)attention_shares(s), rows = (size_t)unit_rows(s);
    w.cut_off = 1024;
    w.part_ml_off = w.cut_off + align_up(shares * 32, 256);
    w.part_o_off = w.part_ml_off + shares * 2 * rows * 2 * 4;
    const size_t attend = w.part_o_off + shares * 2 * rows * s->head_dim * 4;
    w.mass_part_off = w.cut_off + align_up((size_t)kShareSms * 32, 256);
    const size_t mass = w.mass_part_off + (size_t)kShareSms * 2 * 256 * 4;
    w.total = evict > attend ? evict : attend;
    if (mass > w.total) w.total = mass;
    return w;
}

#ifdef __CUDACC__

// Records an argument that only the device could see to be wrong.
__device__ __forceinline__ void report(int* status, seka_status what, int where) {
    if (atomicCAS(status, (int)SEKA_OK, (int)what) == (int)SEKA_OK) status[1] = where;
}
__device__ __forceinline__ void report_invalid(int* status, int where) { report(status, SEKA_ERR_INVALID_ARG, where); }
// codes of status[1]
constexpr int kWhereSeq = 200, kWherePage = 201, kWhereSteps = 202;

__device__ __forceinline__ PagedSeq load_seq(const PagedView& v, int b) {
    const PagedSeq s = paged_seq(v, b);
    if (!s.valid) report_invalid(v.status, kWhereSeq);
    return s;
}
// Row for a TMA box at cached token j, given the entry of its page: a page that does not exist is reported and reads as zeros (the row
// behind the pool).  Apart from the load of the entry, so that it can be under way while the box before is waited for.
__device__ __forceinline__ int box_row(const PagedView& v, int entry, int j) {
    const long long r = pool_row(v, entry, j);
    if (r >= 0) return (int)r;
    report_invalid(v.status, kWherePage);
    return v.n_pages << v.page_shift;
}
__device__ __forceinline__ long long load_pool_row(const PagedView& v, int b, int j) {
    const long long r = pool_row(v, table_entry(v, b, j), j);
    if (r < 0) report_invalid(v.status, kWherePage);
    return r;
}

#endif  // __CUDACC__

seka_status validate_paged(const seka_paged_shape* s);
// the view of a validated shape; the status block is the workspace's first
PagedView paged_view(const seka_paged_shape* s, void* workspace);
// workspace and device arrays that every call needs
seka_status check_paged_call(const seka_paged_shape* s, const void* workspace, size_t workspace_bytes);

}  // namespace seka
