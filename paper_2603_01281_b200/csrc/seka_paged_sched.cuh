// Division of a paged call's work among CTAs.
//
// A unit is a piece of a sequence and one KV head that one CTA can finish by itself; it takes a number of steps.  Units are numbered
// sequence by sequence, KV head by KV head; their steps, laid end to end, are one line that is cut into equal shares, one per CTA,
// wherever the cuts fall: every CTA has the same number of steps whatever the lengths are.  A unit that lies in one share is
// finished there; the parts of one that was cut are merged behind.  Only the device knows the lengths: every CTA adds up the steps
// itself and finds where its share begins.  What a unit and a step are is the geometry's to say:
//   units(L, n)      units of a sequence with L cached tokens, the last n of them new, per KV head
//   steps(L, n, u)   steps of its unit u (at least 1)
//   max_units        no sequence has more units (from what the host knows); more than 8 where the steps of so many could pass 31 bits
#pragma once

#include "seka_paged.cuh"

namespace seka {

// Attention: the queries of `tp` consecutive new tokens (with their whole query group); a step is a tile of 2^shift cached tokens, up
// to the last one that the unit's last token sees (a unit that sees none has one step, all masked).
struct StepGeo {
    int tp, shift;
    int min_share;      // steps that a share has at least
    int max_units;      // (2^24 steps of 128 tokens each at most: eight fit 31 bits)
    SEKA_HD int steps_to(int L, int n, int last) const {
        const int x = L - n + last;
        return x <= (1 << shift) ? 1 : (int)(((long long)x + (1 << shift) - 1) >> shift);
    }
    SEKA_HD int units(int, int n) const { return (n + tp - 1) / tp; }
    SEKA_HD int steps(int L, int n, int p) const {
        const int last = (p + 1) * tp;
        return steps_to(L, n, last < n ? last : n);
    }
};

// Accumulated weights, few rows: all cached tokens of a sequence; a step is 2^shift of them.
struct KeyGeo {
    int shift, min_share, max_units;
    SEKA_HD int units(int L, int) const { return L > 0 ? 1 : 0; }
    SEKA_HD int steps(int L, int, int) const { return (int)(((long long)L + (1 << shift) - 1) >> shift); }
};

// Accumulated weights, many rows: 2^shift cached tokens; a step is the queries of `tp` new tokens, from the first that sees any of
// them (a sequence without new tokens has one empty step).
struct RowGeo {
    int tp, shift, min_share, max_units;
    SEKA_HD int tiles(int n) const { return n > 0 ? (n + tp - 1) / tp : 1; }
    SEKA_HD int first(int L, int n, int u) const {
        const long long x = ((long long)u << shift) - (L - n);
        return x > 0 ? (int)((uint32_t)x / (uint32_t)tp) : 0;       // (keys and tokens are counted in 31 bits)
    }
    SEKA_HD int units(int L, int) const { return (int)(((long long)L + (1 << shift) - 1) >> shift); }
    SEKA_HD int steps(int L, int n, int u) const { return tiles(n) - first(L, n, u); }
};

// Steps of the units first, first + stride, .. of a sequence, per KV head.  A unit's steps fit 31 bits, their sum need not: a prompt of a million
// tokens with 128 query heads on a KV head has more than 2^31.
template <typename Sum = long long, typename Geo> SEKA_HD Sum steps_of_units(const Geo& g, int L, int n, int first, int stride) {
    Sum t = 0;
    for (int u = first, U = g.units(L, n); u < U; u += stride) t += g.steps(L, n, u);
    return t;
}
// Steps of a full share of a line of `all` among n_cta.
SEKA_HD long long share_of(long long all, int n_cta, int min_share) {
    const long long share = (all + n_cta - 1) / n_cta;
    return share < min_share ? min_share : share;
}
// Steps of a CTA, its segments' and the merge's sums are counted in 31 bits.  2^30 steps would take more than twenty minutes.
constexpr long long kMaxShare = 1LL << 30;

// A place on the line: step `j` of unit p of KV head h of sequence b.
struct LinePos { int b, h, p, j; };

// What the merge needs of the cut where a share begins: the unit it falls into (n: its steps; 0: the share is empty).
struct CutRecord { int b, h, p, j, n, share; };

#ifdef __CUDACC__

struct Share {
    long long len;          // steps of this CTA
    LinePos at;
    int share;              // steps of a full share
};

// What find_share needs of shared memory, before anything else is in it.
template <int NT> struct ShareScratch {
    long long warp_sum[NT / 32];
    long long rest;                     // steps into the KV head that the share begins in
    int b, L, n, h, p, j;
    int len[NT], new_tokens[NT];
    long long steps[NT];
};

// exclusive scan over the block; `all` receives the sum
template <int NT> __device__ __forceinline__ long long block_scan(long long x, long long* warp_sum, long long& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();                    // the sums of the scan before have been read
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) before += warp_sum[w];
        all += warp_sum[w];
    }
    return before + inc - x;
}

// Every thread of a block of NT calls: the block's share of the line among `n_cta`.  Sequences by thread, NT at a time, then the units of
// the one that the share begins in; the steps of a sequence of many units are added up by a warp.  (In closed form, sums of floors by
// Euclid's algorithm, the 64-bit divisions and a binary search over them took 10 us.)
template <int NT, typename Geo>
__device__ inline Share find_share(const PagedView& v, const Geo& g, int n_cta, int cta, ShareScratch<NT>& sc) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long mine = 0;                 // steps of this thread's sequence; with up to NT sequences it stays in a register
    int L = 0, n = 0;
    auto count = [&](int b0) {
        const int b = b0 + tid;
        L = 0; n = 0;
        if (b < v.B) { const PagedSeq s = load_seq(v, b); L = s.L; n = s.n; }
        long long per = 0;
        if (g.max_units <= 8) {
            if (b < v.B) per = steps_of_units<int>(g, L, n, 0, 1);
        } else {
            sc.len[tid] = L; sc.new_tokens[tid] = n;
            __syncthreads();
            for (int k = warp; k < NT && b0 + k < v.B; k += NT / 32) {
                long long t = steps_of_units(g, sc.len[k], sc.new_tokens[k], lane, 32);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
                if (lane == 0) sc.steps[k] = t;
            }
            __syncthreads();
            if (b < v.B) per = sc.steps[tid];
        }
        mine = per * v.Hkv;
    };
    long long total = 0, all;
    for (int b0 = 0; b0 < v.B; b0 += NT) { count(b0); total += mine; }
    block_scan<NT>(total, sc.warp_sum, all);
    const long long share = share_of(all, n_cta, g.min_share);
    Share r;
    r.share = (int)share;
    const long long x = share * cta;
    r.len = all - x < share ? all - x : share;
    r.at = LinePos{0, 0, 0, 0};
    if (r.len <= 0 || share > kMaxShare) {              // (the same for the whole block; too long: for all blocks)
        if (share > kMaxShare) report(v.status, SEKA_ERR_UNSUPPORTED, kWhereSteps);
        r.len = 0;
        return r;
    }
    long long before = 0;
    for (int b0 = 0; b0 < v.B; b0 += NT) {
        if (v.B > NT) count(b0);
        const long long at = before + block_scan<NT>(mine, sc.warp_sum, all);
        if (mine > 0 && x >= at && x < at + mine) {
            sc.b = b0 + tid; sc.L = L; sc.n = n;
            const long long per = mine / v.Hkv;
            sc.h = (int)((x - at) / per);
            sc.rest = x - at - sc.h * per;
        }
        before += all;
        if (before > x) break;                          // (the same for the whole block)
    }
    __syncthreads();
    const int U = g.units(sc.L, sc.n);
    before = 0;
    for (int u0 = 0; u0 < U; u0 += NT) {
        const int st = u0 + tid < U ? g.steps(sc.L, sc.n, u0 + tid) : 0;
        const long long at = before + block_scan<NT>(st, sc.warp_sum, all);
        if (sc.rest >= at && sc.rest < at + st) { sc.p = u0 + tid; sc.j = (int)(sc.rest - at); }
        before += all;
        if (before > sc.rest) break;
    }
    __syncthreads();
    r.at = LinePos{sc.b, sc.h, sc.p, sc.j};
    fence_proxy_async();                // the scratch lies where copies will land
    __syncthreads();
    return r;
}

template <typename Geo> __device__ __forceinline__ void write_cut(CutRecord* cuts, const PagedView& v, const Geo& g, const Share& s, int cta) {
    CutRecord c = {s.at.b, s.at.h, s.at.p, s.at.j, 0, s.share};
    if (s.len > 0) {
        const PagedSeq q = paged_seq(v, s.at.b);
        c.n = g.steps(q.L, q.n, s.at.p);
    }
    cuts[cta] = c;
}

// Walks the segments of a share: per unit, the steps [j, j + n) of it.
struct Segment {
    int b, h, p;            // unit
    int j, n;               // first step, steps
    int q0, L, old;         // first new token and cached tokens of the sequence, cached tokens before the new ones (may be negative)
    int n_new;
    bool whole;             // all of the unit
    bool first;             // first segment of the share
};
struct Walk {
    LinePos at;
    int left, first;        // (a share is at most kMaxShare)
    int q0, L, n;
};
__device__ __forceinline__ void walk_load(const PagedView& v, Walk& w) {
    const PagedSeq s = paged_seq(v, w.at.b);
    w.q0 = s.q0; w.L = s.L; w.n = s.n;
}
__device__ __forceinline__ void walk_begin(const PagedView& v, const Share& s, Walk& w) {
    w.at = s.at; w.left = (int)s.len; w.first = 1; w.q0 = 0; w.L = 0; w.n = 0;
    if (w.left > 0) walk_load(v, w);
}
template <typename Geo> __device__ __forceinline__ bool walk_next(const PagedView& v, const Geo& g, Walk& w, Segment& s) {
    if (w.left <= 0) return false;
    const int steps = g.steps(w.L, w.n, w.at.p), rest = steps - w.at.j;
    s.b = w.at.b; s.h = w.at.h; s.p = w.at.p; s.j = w.at.j;
    s.n = rest < w.left ? rest : w.left;
    s.q0 = w.q0; s.L = w.L; s.n_new = w.n; s.old = w.L - w.n;
    s.whole = s.j == 0 && s.n == steps;
    s.first = w.first != 0;
    w.first = 0; w.left -= s.n; w.at.j = 0;
    if (w.left > 0) {                       // the unit is through
        ++w.at.p;
        if (w.at.p >= g.units(w.L, w.n)) {
            w.at.p = 0;
            if (++w.at.h == v.Hkv) {
                w.at.h = 0;
                do { ++w.at.b; if (w.at.b >= v.B) { w.left = 0; break; } walk_load(v, w); } while (g.units(w.L, w.n) == 0);
            }
        }
    }
    return true;
}

#endif  // __CUDACC__

}  // namespace seka
