"""Paged calls without a GPU: refusals before anything is launched, the table of the rotation, and the checks of what only the device
knows (sequence bounds, pages), compiled for the host from the header that the kernels include."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2603_01281_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)        # never dereferenced: the checks come first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def shape(**kw):
    base = dict(batch=2, total_new=6, max_new=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=40, max_pages=8,
                dtype=binding.SEKA_BF16, softmax_scale=0.0, block_table=256, cache_lens=256, cu_new=256)
    base.update(kw)
    return binding.SekaPagedShape(*[base[f[0]] for f in binding.SekaPagedShape._fields_])


def rope(**kw):
    base = dict(rot_dim=64, layout=0, magnitude=1.0, turns=256)
    base.update(kw)
    return binding.SekaRope(*[base[f[0]] for f in binding.SekaRope._fields_])


def append(lib, s, r=None, Q=ONE, qs=0, K=ONE, ks=0, V=ONE, vs=0, Qo=ctypes.c_void_p(512), Kp=ONE, Vp=ONE, ws=ONE, n=BIG):
    return lib.seka_rope_append(ctypes.byref(s), ctypes.byref(r) if r is not None else None, Q, qs, K, ks, V, vs, None, Qo, Kp, Vp, None, ws, n, None)


def attend(lib, s, Q=ONE, K=ONE, V=ONE, O=ONE, ws=ONE, n=BIG):
    return lib.seka_paged_attention(ctypes.byref(s), Q, K, V, O, None, ws, n, None)


def mass(lib, s, Q=ONE, K=ONE, lse=ONE, out=ONE, ws=ONE, n=BIG):
    return lib.seka_attention_mass(ctypes.byref(s), Q, K, lse, None, out, ws, n, None)


def evict(lib, s, K=ONE, V=ONE, m=ONE, p=ONE, nxt=ONE, keep=10, recent=2, plen=0, lens=ONE, ws=ONE, n=BIG):
    return lib.seka_evict_cache(ctypes.byref(s), K, V, m, m, p, p, None, plen, nxt, keep, recent, lens, ws, n, None)


BAD_SHAPES = [dict(batch=-1), dict(total_new=-1), dict(max_new=-1), dict(n_q_heads=7), dict(n_kv_heads=0), dict(head_dim=96), dict(page_size=24),
              dict(page_size=8), dict(page_size=512), dict(n_pages=-1), dict(max_pages=-2), dict(dtype=5), dict(softmax_scale=-1.0),
              dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(n_q_heads=258), dict(cu_new=None, total_new=7),
              dict(max_pages=1 << 28), dict(n_pages=1 << 28), dict(batch=70000)]


@pytest.mark.parametrize("bad", BAD_SHAPES)
def test_bad_shapes(lib, bad):
    s = shape(**bad)
    assert binding.seka_paged_workspace_bytes(s) == 0
    for call in (append, attend, mass, evict):
        assert call(lib, s) in (binding.SEKA_ERR_INVALID_ARG, binding.SEKA_ERR_UNSUPPORTED)
    assert binding.seka_launch_count() == 0


def test_bad_arguments(lib):
    s, bad, ws = shape(), binding.SEKA_ERR_INVALID_ARG, binding.SEKA_ERR_WORKSPACE
    for call in (append, attend, mass, evict):
        assert call(lib, s, ws=None) == ws and call(lib, s, n=300) == ws and call(lib, s, ws=ODD) == ws
        assert call(lib, shape(block_table=None)) == bad and call(lib, shape(cache_lens=None)) == bad
        assert call(lib, shape(batch=0, total_new=0, cu_new=None, cache_lens=None), ws=None) == binding.SEKA_OK
    for k in ("Q", "K", "V", "Qo", "Kp", "Vp"):
        assert append(lib, s, **{k: None}) == bad and append(lib, s, **{k: ODD}) == bad
    for k in ("qs", "ks", "vs"):
        assert append(lib, s, **{k: 8}) == bad and append(lib, s, **{k: 8 * 128 + 4}) == bad and append(lib, s, **{k: -2048}) == bad
    for r in (rope(rot_dim=0), rope(rot_dim=63), rope(rot_dim=130), rope(layout=2), rope(magnitude=-1.0), rope(magnitude=math.nan), rope(turns=None)):
        assert append(lib, s, r) == bad
    assert append(lib, s, Qo=ONE, qs=12 * 128) == bad                               # in place needs packed queries
    assert append(lib, shape(dtype=binding.SEKA_F32), Qo=ONE) == bad                # ... of the output's type
    for k in ("Q", "K", "V", "O"):
        assert attend(lib, s, **{k: None}) == bad and attend(lib, s, **{k: ODD}) == bad
    for k in ("Q", "K", "lse", "out"):
        assert mass(lib, s, **{k: None}) == bad
    for k in ("K", "V", "m", "p", "nxt", "lens"):
        assert evict(lib, s, **{k: None}) == bad
    assert evict(lib, s, keep=0) == bad and evict(lib, s, recent=-1) == bad and evict(lib, s, plen=-1) == bad
    assert attend(lib, shape(total_new=0, max_new=0), Q=None, O=None, ws=None) == binding.SEKA_OK
    assert binding.seka_launch_count() == 0


def test_misaligned_state_is_refused(lib):
    off = ctypes.c_void_p(ONE.value + 4)
    assert evict(lib, shape(), m=off) == binding.SEKA_ERR_INVALID_ARG
    assert evict(lib, shape(), p=off) == binding.SEKA_ERR_INVALID_ARG


def test_binding_refuses_wrong_tensors():
    with pytest.raises(ValueError):
        binding.make_paged_shape(batch=1, max_new=1, total_new=1, n_q_heads=2, n_kv_heads=1, head_dim=64, page_size=16, n_pages=4,
                                 block_table=torch.zeros((1, 2), dtype=torch.int32), cache_lens=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.make_rope(torch.zeros(32))
    x = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    binding._fits("x", x, torch.bfloat16, (3, 4, 64), x.device)
    binding._fits("x", x[:, :2], torch.bfloat16, (3, 2, 64), x.device, packed=False)
    for t, shp in ((x.float(), (3, 4, 64)), (x, (3, 4, 128)), (x, (3, 4)), (x[:, :2], (3, 2, 64)), (x.to("meta"), (3, 4, 64))):
        with pytest.raises(ValueError):
            binding._fits("x", t, torch.bfloat16, shp, torch.device("cpu"))


def test_rope_turns(lib):
    for r in (2, 32, 126, 128):
        i = torch.arange(r // 2, dtype=torch.float64)
        plain = 10000.0 ** (-2 * i / r) / (2 * math.pi)
        torch.testing.assert_close(binding.seka_rope_turns(r), plain, rtol=1e-14, atol=0)
        torch.testing.assert_close(binding.seka_rope_turns(r, scaling="linear", scale=4.0), plain / 4, rtol=1e-14, atol=0)
        w = ((4096 * plain - 1) / 3).clamp(0, 1)
        torch.testing.assert_close(binding.seka_rope_turns(r, scaling="wavelength", scale=8.0, trained_len=4096), plain * w + plain / 8 * (1 - w),
                                   rtol=1e-13, atol=0)
        if r > 2:
            t = binding.seka_rope_turns(r, scaling="base", scale=4.0)
            assert t[0] == binding.seka_rope_turns(r)[0] and abs(float(t[-1] / plain[-1]) - 0.25) < 1e-12
    bad = [dict(rot_dim=0), dict(rot_dim=5), dict(rot_dim=130), dict(rot_dim=32, base=1.0), dict(rot_dim=32, base=math.nan),
           dict(rot_dim=32, scaling="linear", scale=0.0), dict(rot_dim=2, scaling="base", scale=2.0),
           dict(rot_dim=32, scaling="wavelength", scale=2.0, trained_len=0.0),
           dict(rot_dim=32, scaling="wavelength", scale=2.0, low_turns=4.0, high_turns=4.0)]
    for kw in bad:
        with pytest.raises(binding.SekaError):
            binding.seka_rope_turns(**kw)


PROBE = r'''
#include <stdio.h>
#include "seka_paged.cuh"
using namespace seka;
int main() {
    int table[2 * 4] = {3, 0, 9, 10, -1, 7, 2147483647, 5}, lens[2], cu[3];
    PagedView v = {};
    v.table = table; v.lens = lens; v.cu = cu;
    v.B = 2; v.T = 10; v.max_new = 6; v.max_pages = 4; v.n_pages = 10; v.page_shift = 4; v.cap = 64;
    int bad = 0;
    auto expect = [&](bool ok, int line) { if (!ok) { printf("line %d\n", line); ++bad; } };
    // every combination of offsets and lengths around the bounds: valid exactly where nothing can leave the buffers
    const int offs[] = {-2147483647, -1, 0, 1, 4, 6, 7, 9, 10, 11, 2147483647}, ls[] = {-2147483647, -1, 0, 1, 5, 63, 64, 65, 2147483647};
    for (int a : offs) for (int b : offs) for (int l : ls) {
        cu[0] = a; cu[1] = b; cu[2] = 10; lens[0] = l; lens[1] = 0;
        const PagedSeq s = paged_seq(v, 0);
        const bool ok = a >= 0 && b >= a && b <= 10 && (long long)b - a <= 6 && l >= 0 && l <= 64;
        expect(s.valid == ok, __LINE__);
        expect(s.q0 >= 0 && s.n >= 0 && s.q0 + s.n <= v.T && s.n <= v.max_new && s.L >= 0 && s.L <= v.cap, __LINE__);
        if (!ok) expect(s.n == 0 && s.L == 0, __LINE__);
    }
    v.cu = nullptr; lens[0] = 5; lens[1] = 64; v.T = 12;
    expect(paged_seq(v, 1).valid && paged_seq(v, 1).q0 == 6 && paged_seq(v, 1).n == 6, __LINE__);
    // pages: a row of the pool or -1
    const long long want[2][4] = {{48, 0, 144, -1}, {-1, 112, -1, 80}};
    for (int b = 0; b < 2; ++b) for (int j = 0; j < 64; ++j) {
        const long long r = pool_row(v, table_entry(v, b, j), j), w = want[b][j / 16];
        expect(r == (w < 0 ? -1 : w + j % 16), __LINE__);
        expect(r < 160, __LINE__);
    }
    v.n_pages = 0x7fff0000 / 256; v.page_shift = 8;
    expect(pool_row(v, v.n_pages - 1, 511) == (long long)v.n_pages * 256 - 1, __LINE__);
    return bad ? 1 : 0;
}
'''


def test_device_checks_on_the_host(tmp_path):
    src, exe = tmp_path / "probe.cpp", tmp_path / "probe"
    src.write_text(PROBE)
    cuda = os.path.join(os.path.dirname(os.path.dirname(build.NVCC)), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, "-I", cuda, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


SCHED = r'''
#include <stdio.h>
#include <stdlib.h>
#include "seka_paged_sched.cuh"
using namespace seka;
int main() {
    unsigned seed = 12345;
    auto rnd = [&](int lo, int hi) { seed = seed * 1664525u + 1013904223u; return lo + (int)((seed >> 8) % (unsigned)(hi - lo + 1)); };
    int bad = 0;
    auto expect = [&](bool ok, int line) { if (!ok && bad++ < 5) printf("line %d\n", line); };
    for (int rep = 0; rep < 3000; ++rep) {
        StepGeo g;
        g.shift = rnd(6, 7); g.tp = rep % 3 == 0 ? rnd(1, 9) : rep % 3 == 1 ? 256 / rnd(1, 128) : rnd(1, 4096); g.min_share = 1;
        if (g.tp < 1) g.tp = 1;
        const int n = rnd(1, rep % 2 ? 40 : 3000), L = rep % 5 == 0 ? rnd(0, n + 100) : n + rnd(0, 9000), U = g.units(L, n);
        for (int u = 0; u < U; ++u) {
            const int last = (u + 1) * g.tp < n ? (u + 1) * g.tp : n, keys = L - n + last, K = 1 << g.shift;
            const int want = keys <= 0 ? 1 : (keys + K - 1) / K;
            expect(g.steps(L, n, u) == want, __LINE__);
        }
    }
    for (int rep = 0; rep < 3000; ++rep) {
        RowGeo g;
        g.shift = 8; g.tp = rep % 2 ? 128 / rnd(1, 128) : rnd(1, 128); g.min_share = 1;
        const int n = rep % 7 == 0 ? 0 : rnd(1, rep % 2 ? 40 : 3000), L = rep % 5 == 0 ? rnd(0, n + 100) : n + rnd(0, 9000), U = g.units(L, n);
        expect(U == (L + 255) / 256, __LINE__);
        for (int u = 0; u < U; ++u) {
            // row tiles that hold a token which sees the unit's first key (token i sees key j: j <= L - n + i)
            int want = 0;
            for (int t = 0; t * g.tp < (n > 0 ? n : 1); ++t) {
                const int last = (t + 1) * g.tp < n ? (t + 1) * g.tp - 1 : n - 1;
                want += n == 0 || u * 256 <= L - n + last;
            }
            expect(want >= 1 && g.steps(L, n, u) == want, __LINE__);
        }
        const KeyGeo k = {6, 1, 1};
        expect(k.units(L, n) * k.steps(L, n, 0) == (L + 63) / 64, __LINE__);
    }
    StepGeo g = {1, 7, 1, 1};          // the longest cache
    expect(g.steps(0x7fff0000, 1, 0) == 0x7fff0000 / 128, __LINE__);
    return bad ? 1 : 0;
}
'''


def test_division_among_ctas_on_the_host(tmp_path):
    src, exe = tmp_path / "sched.cpp", tmp_path / "sched"
    src.write_text(SCHED)
    cuda = os.path.join(os.path.dirname(os.path.dirname(build.NVCC)), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, "-I", cuda, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_no_sequence_has_new_tokens(lib):
    # a padded packed step in which every sequence is idle: tokens that nobody owns, nothing to attend to
    assert attend(lib, shape(max_new=0)) == binding.SEKA_OK


def test_counts_beyond_their_bits_are_refused(lib):
    for bad in (dict(max_new=(1 << 31) - 1), dict(total_new=(1 << 31) - 1), dict(batch=60000, n_kv_heads=30000, n_q_heads=30000, max_pages=1 << 24, n_pages=1 << 20)):
        s = shape(**bad)
        assert lib.seka_paged_workspace_bytes(ctypes.byref(s)) == 0
        for call in (append, attend, mass, evict):
            assert call(lib, s) == binding.SEKA_ERR_UNSUPPORTED, (bad, call)


SUMS = r'''
#include <stdio.h>
#include "seka_paged_sched.cuh"
using namespace seka;
int main() {
    int bad = 0;
    auto expect = [&](bool ok, int line) { if (!ok && bad++ < 5) printf("line %d\n", line); };
    // the steps of a sequence against sums in 128 bits in closed form: a unit's last token sees L - n + last keys, every 2^shift are a step
    auto floors = [](__int128 count, __int128 a, __int128 b, __int128 m) {          // sum of (a i + b) / m over i < count
        __int128 t = 0;
        while (true) {
            t += (a / m) * count * (count - 1) / 2 + (b / m) * count;
            a %= m; b %= m;
            const __int128 top = a * count + b;
            if (top < m) return t;
            count = top / m; b = top % m;
            const __int128 x = m; m = a; a = x;
        }
    };
    const int cases[][3] = {{1100000, 1100000, 2}, {2304000, 270336, 2}, {4300000, 4300000, 32}, {6000000, 6000000, 64}, {2000000, 1900001, 4}, {300000, 299999, 2},
                            {40000000, 3000000, 2}, {1000, 1000, 16}};
    for (const auto& c : cases) {
        const int L = c[0], n = c[1], tp = c[2];
        const StepGeo g = {tp, 7, 4, 0};
        const int U = g.units(L, n);
        expect(U == (n + tp - 1) / tp, __LINE__);
        __int128 want = floors(U - 1, tp, (__int128)L - n + tp + 127, 128) + (L + 127) / 128;
        long long got = 0;
        for (int lane = 0; lane < 32; ++lane) got += steps_of_units(g, L, n, lane, 32);
        expect((__int128)got == want && got == steps_of_units(g, L, n, 0, 1), __LINE__);
        const RowGeo r = {tp / 2, 8, 2, 0};
        const int V = r.units(L, n), T = r.tiles(n);
        __int128 rows = 0;
        for (int u = 0; u < V; ++u) { const long long x = 256LL * u - (L - n); rows += T - (x > 0 ? x / r.tp : 0); }
        got = 0;
        for (int lane = 0; lane < 32; ++lane) got += steps_of_units(r, L, n, lane, 32);
        expect((__int128)got == rows, __LINE__);
    }
    expect(steps_of_units(StepGeo{2, 7, 4, 0}, 1100000, 1100000, 0, 1) > 0x7fffffffLL, __LINE__);
    // shares cover the line, and what a CTA cannot count is above the limit
    for (long long all : {1LL, 3LL, 4LL, 147LL * 4, 1LL << 31, (1LL << 32) + 5, 148LL << 30, (148LL << 30) + 1, 1LL << 44})
        for (int ctas : {1, 7, 148, 444}) {
            const long long s = share_of(all, ctas, 4);
            expect(s >= 4 && s * ctas >= all && (s == 4 || (s - 1) * ctas < all), __LINE__);
        }
    expect(share_of(148LL << 30, 148, 4) == kMaxShare && share_of((148LL << 30) + 1, 148, 4) > kMaxShare, __LINE__);
    // the merge: parts of the longest unit in shares at the limit
    const int n = 0x7fff0000 / 64, j = 1;
    expect((long long)n - j + kMaxShare - 1 <= 0x7fffffffLL, __LINE__);
    return bad ? 1 : 0;
}
'''


def test_sums_of_steps_on_the_host(tmp_path):
    src, exe = tmp_path / "sums.cpp", tmp_path / "sums"
    src.write_text(SUMS)
    cuda = os.path.join(os.path.dirname(os.path.dirname(build.NVCC)), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, "-I", cuda, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
