// Division of a paged call's work among CTAs.
//
// A unit is a piece of a sequence and one KV head that one CTA can finish by itself; it takes a number of steps.  Units are numbered
// sequence by sequence, KV head by KV head; their steps, laid end to end, are one line that is cut into equal shares, one per CTA,
// wherever the cuts fall: every CTA has the same number of steps whatever the lengths are.  A unit that lies in one share is
// finished there; the parts of one that was cut are merged behind.  Only the device knows the lengths: every CTA adds up the steps
// itself and finds where its share begins.  What a unit and a step are is the geometry's to say:
//   units(L, n)      units of a sequence with L cached tokens, the last n of them new, per KV head
//   steps(L, n, u)   steps of its unit u (at least 1)
//   prefix(L, n, u)  steps of its first u units
#pragma once

#include "seka_paged.cuh"

namespace seka {

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

// Attention: the queries of `tp` consecutive new tokens (with their whole query group); a step is a tile of 2^shift cached tokens, up
// to the last one that the unit's last token sees (a unit that sees none has one step, all masked).
struct StepGeo {
    int tp, shift;
    int min_share;      // steps that a share has at least
    SEKA_HD int steps_to(int L, int n, int last) const {
        const int x = L - n + last;
        return x <= (1 << shift) ? 1 : (int)(((long long)x + (1 << shift) - 1) >> shift);
    }
    SEKA_HD int units(int, int n) const { return (n + tp - 1) / tp; }
    SEKA_HD int steps(int L, int n, int p) const {
        const int last = (p + 1) * tp;
        return steps_to(L, n, last < n ? last : n);
    }
    SEKA_HD long long prefix(int L, int n, int u) const {
        if (u <= 0) return 0;
        const int U = units(L, n), old = L - n;
        long long s = 0;
        const int full = u < U ? u : U - 1;     // units of exactly tp tokens
        int p = 0;
        while (p < full && (long long)old + (long long)(p + 1) * tp < 1) { ++s; ++p; }      // padding: units without a key
        if (p < full)
            s += (long long)floor_sum((unsigned long long)(full - p), 1ull << shift, (unsigned long long)tp,
                                      (unsigned long long)((long long)old + (long long)(p + 1) * tp + (1 << shift) - 1));
        if (u >= U) s += steps(L, n, U - 1);
        return s;
    }
};

// Accumulated weights, few rows: all cached tokens of a sequence; a step is 2^shift of them.
struct KeyGeo {
    int shift, min_share;
    SEKA_HD int units(int L, int) const { return L > 0 ? 1 : 0; }
    SEKA_HD int steps(int L, int, int) const { return (int)(((long long)L + (1 << shift) - 1) >> shift); }
    SEKA_HD long long prefix(int L, int n, int u) const { return u > 0 ? steps(L, n, 0) : 0; }
};

// Accumulated weights, many rows: 2^shift cached tokens; a step is the queries of `tp` new tokens, from the first that sees any of
// them (a sequence without new tokens has one empty step).
struct RowGeo {
    int tp, shift, min_share;
    SEKA_HD int tiles(int n) const { return n > 0 ? (n + tp - 1) / tp : 1; }
    SEKA_HD int first(int L, int n, int u) const {
        const long long x = ((long long)u << shift) - (L - n);
        return x > 0 ? (int)(x / tp) : 0;
    }
    SEKA_HD int units(int L, int) const { return (int)(((long long)L + (1 << shift) - 1) >> shift); }
    SEKA_HD int steps(int L, int n, int u) const { return tiles(n) - first(L, n, u); }
    SEKA_HD long long prefix(int L, int n, int u) const {
        const long long old = L - n, k0 = old <= 0 ? 0 : (old + (1 << shift) - 1) >> shift;
        long long s = (long long)tiles(n) * u;
        if (u > k0) s -= (long long)floor_sum((unsigned long long)(u - k0), (unsigned long long)tp, 1ull << shift, (unsigned long long)((k0 << shift) - old));
        return s;
    }
};

// A place on the line: step `j` of unit p of KV head h of sequence b.
struct LinePos { int b, h, p, j; };

// `r` steps into the sequence b (0 <= r < Hkv * steps of a head)
template <typename Geo> SEKA_HD LinePos place_in_seq(const Geo& g, int b, int L, int n, long long per_head, long long r) {
    LinePos c;
    c.b = b; c.h = (int)(r / per_head);
    r -= c.h * per_head;
    int lo = 0, hi = g.units(L, n) - 1;                 // largest p with prefix(p) <= r
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (g.prefix(L, n, mid) <= r) lo = mid; else hi = mid - 1;
    }
    c.p = lo; c.j = (int)(r - g.prefix(L, n, lo));
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
template <int NT, typename Geo>
__device__ inline Share find_share(const PagedView& v, const Geo& g, int n_cta, int cta, long long* scratch) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int NW = NT / 32;
    // steps of the sequences, a block's worth at a time; with up to NT sequences they stay in a register
    long long mine = 0;
    int L = 0, n = 0;
    auto steps_of = [&](int b) -> long long {
        if (b >= v.B) { n = 0; L = 0; return 0; }
        const PagedSeq s = load_seq(v, b);
        n = s.n; L = s.L;
        return g.prefix(L, n, g.units(L, n)) * v.Hkv;
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
