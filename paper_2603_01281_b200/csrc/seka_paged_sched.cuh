// Division of the paged attention among CTAs.
//
// A unit is the queries of `tp` consecutive new tokens of a sequence and one KV head (with their whole query group); it walks
// the key tiles of the cached tokens that its last token sees, one tile a step.  Units are numbered sequence by
// sequence, KV head by KV head, tokens ascending; their steps, laid end to end, are one line that is cut into equal shares, one per CTA,
// wherever the cuts fall: every CTA has the same number of steps whatever the lengths are.  A unit that lies in one share is
// finished there; the parts of one that was cut are merged behind (combine).  Only the device knows the lengths: every CTA adds
// up the steps itself and finds where its share begins.
#pragma once

#include "seka_paged.cuh"

namespace seka {

struct StepGeo {
    int tp;             // new tokens of a unit
    int shift;          // log2 of the keys of a step
    int min_share;      // steps that a share has at least
};

// steps of the unit that ends before new token `last` (a unit that sees no key has one step, all masked)
SEKA_HD int steps_to(const StepGeo& g, int L, int n, int last) {
    const int x = L - n + last;
    return x <= (1 << g.shift) ? 1 : (int)(((long long)x + (1 << g.shift) - 1) >> g.shift);
}
SEKA_HD int seq_units(const StepGeo& g, int n) { return (n + g.tp - 1) / g.tp; }
SEKA_HD int unit_steps(const StepGeo& g, int L, int n, int p) {
    const int last = (p + 1) * g.tp;
    return steps_to(g, L, n, last < n ? last : n);
}

// sum of floor((a i + b) / m) over 0 <= i < n, all non-negative, m > 0 (Euclid's algorithm on the lattice points below the line)
SEKA_HD unsigned long long floor_sum(unsigned long long n, unsigned long long m, unsigned long long a, unsigned long long b) {
    unsigned long long ans = 0;
    while (n > 0) {
        if (a >= m) { ans += n * (n - 1) / 2 * (a / m); a %= m; }
        if (b >= m) { ans += n * (b / m); b %= m; }
        const unsigned long long y = a * n + b;
        if (y < m) break;
        n = y / m; b = y % m;
        const unsigned long long t = m; m = a; a = t;
    }
    return ans;
}

// steps of the first `u` units of a sequence with n new tokens and L cached ones (one KV head)
SEKA_HD long long head_steps(const StepGeo& g, int L, int n, int u) {
    if (u <= 0) return 0;
    const int U = seq_units(g, n), old = L - n;
    long long s = 0;
    int full = u < U ? u : U - 1;           // units of exactly tp tokens
    int p = 0;
    while (p < full && (long long)old + (long long)(p + 1) * g.tp < 1) { ++s; ++p; }      // padding: units without a key
    if (p < full)
        s += (long long)floor_sum((unsigned long long)(full - p), 1ull << g.shift, (unsigned long long)g.tp,
                                  (unsigned long long)((long long)old + (long long)(p + 1) * g.tp + (1 << g.shift) - 1));
    if (u >= U) s += unit_steps(g, L, n, U - 1);
    return s;
}

// A place on the line: step `j` of unit p of KV head h of sequence b.
struct LinePos { int b, h, p, j; };

// `r` steps into the sequence b (0 <= r < Hkv * steps of a head)
SEKA_HD LinePos place_in_seq(const StepGeo& g, int b, int L, int n, long long per_head, long long r) {
    LinePos c;
    c.b = b; c.h = (int)(r / per_head);
    r -= c.h * per_head;
    int lo = 0, hi = seq_units(g, n) - 1;               // largest p with head_steps(p) <= r
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (head_steps(g, L, n, mid) <= r) lo = mid; else hi = mid - 1;
    }
    c.p = lo; c.j = (int)(r - head_steps(g, L, n, lo));
    return c;
}

// What the merge needs of the cut where a share begins: the unit it falls into (n: its steps; 0: the share is empty).
struct CutRecord { int b, h, p, j, n, share; };

#ifdef __CUDACC__

constexpr long long kNoPlace = -1;

struct Share {
    long long len;          // steps of this CTA
    LinePos at;
    int share;              // steps of a full share
};

// Every thread of a block of NT calls; the block's share of the line among `n_cta`.  `scratch`: NT / 32 + 4 words of 8 bytes.
template <int NT>
__device__ inline Share find_share(const PagedView& v, const StepGeo& g, int n_cta, int cta, long long* scratch) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int NW = NT / 32;
    // steps of the sequences, a block's worth at a time; with up to NT sequences they stay in a register
    long long mine = 0;
    int L = 0, n = 0;
    auto steps_of = [&](int b) -> long long {
        if (b >= v.B) { n = 0; L = 0; return 0; }
        const PagedSeq s = load_seq(v, b);
        n = s.n; L = s.L;
        return n > 0 ? head_steps(g, L, n, seq_units(g, n)) * v.Hkv : 0;
    };
    long long total = 0;
    for (int b0 = 0; b0 < v.B; b0 += NT) { mine = steps_of(b0 + tid); total += mine; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (lane == 0) scratch[warp] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += scratch[w];
    long long share = (total + n_cta - 1) / n_cta;
    if (share < g.min_share) share = g.min_share;
    Share r;
    r.share = (int)share;
    const long long x = share * cta;
    r.len = total - x < share ? total - x : share;
    r.at = LinePos{0, 0, 0, 0};
    if (r.len <= 0) { r.len = 0; return r; }            // (uniform)
    int* place = reinterpret_cast<int*>(scratch + NW);
    long long before = 0;
    for (int b0 = 0; b0 < v.B; b0 += NT) {
        if (v.B > NT) mine = steps_of(b0 + tid);
        long long inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += y;
        }
        __syncthreads();
        if (lane == 31) scratch[warp] = inc;
        __syncthreads();
        long long mybase = before, all = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < warp) mybase += scratch[w];
            all += scratch[w];
        }
        mybase += inc - mine;
        if (mine > 0 && x >= mybase && x < mybase + mine) {
            const LinePos c = place_in_seq(g, b0 + tid, L, n, mine / v.Hkv, x - mybase);
            place[0] = c.b; place[1] = c.h; place[2] = c.p; place[3] = c.j;
        }
        before += all;
        if (before > x) break;                          // (uniform)
    }
    __syncthreads();
    r.at = LinePos{place[0], place[1], place[2], place[3]};
    return r;
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
    int left, first;        // (a share is below 2^31 steps: a line of 2^31 steps of 128 keys would take hours)
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
__device__ __forceinline__ bool walk_next(const PagedView& v, const StepGeo& g, Walk& w, Segment& s) {
    if (w.left <= 0) return false;
    const int steps = unit_steps(g, w.L, w.n, w.at.p), rest = steps - w.at.j;
    s.b = w.at.b; s.h = w.at.h; s.p = w.at.p; s.j = w.at.j;
    s.n = rest < w.left ? rest : w.left;
    s.q0 = w.q0; s.L = w.L; s.n_new = w.n; s.old = w.L - w.n;
    s.whole = s.j == 0 && s.n == steps;
    s.first = w.first != 0;
    w.first = 0; w.left -= s.n; w.at.j = 0;
    if (w.left > 0) {                       // the unit is through
        ++w.at.p;
        if (w.at.p * g.tp >= w.n) {
            w.at.p = 0;
            if (++w.at.h == v.Hkv) {
                w.at.h = 0;
                do { ++w.at.b; if (w.at.b >= v.B) { w.left = 0; break; } walk_load(v, w); } while (w.n == 0);
            }
        }
    }
    return true;
}

#endif  // __CUDACC__

}  // namespace seka
