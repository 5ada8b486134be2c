"""Paged cache on the GPU against plain implementations in 64 bits (tests/paged_ref.py), through the binding.

Tolerances.  Half a step of bf16 is 2^-8 of the value.  A score is a sum of d products accumulated in fp32, off by at most d 2^-23 of
the sum of their magnitudes (`dq` below, scaled): delta = d 2^-23 dq.  Attention rounds its weights to bf16, so an output is
off by at most 2^-8 |o| + (2^-8 + 2 delta + 2^-16) sum_j p_j |v_j|, the 2^-16 for the fp32 sums and the approximate exponential."""
import math

import pytest
import torch

from paper_2603_01281_b200 import binding

import paged_ref as R

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    binding.load()


# lens, new tokens, query heads, KV heads, head_dim, page
SINGLE = [
    ([1, 16, 17, 777], [1, 1, 1, 1], 8, 2, 128, 16),
    ([5, 0, 300, 64, 65, 1024, 63], [1] * 7, 4, 4, 64, 32),
    ([2000, 1], [1, 1], 7, 1, 128, 128),
    ([900, 130], [1, 1], 16, 1, 64, 64),
    ([333, 40, 129], [1, 1, 1], 17, 1, 128, 16),
    ([700], [1], 128, 1, 64, 256),
    ([50, 3], [1, 1], 3, 3, 128, 16),
    ([40] * 70, [1] * 70, 4, 2, 64, 16),
    ([6001, 12, 4096], [1, 1, 1], 32, 8, 128, 64),
]
CHUNK = [
    ([300, 5, 129, 40], [3, 5, 2, 1], 8, 2, 128, 16),             # few rows; a whole sequence that is new
    ([1000], [300], 4, 2, 128, 64),
    ([257, 64, 0, 500, 31], [257, 10, 0, 1, 31], 8, 8, 64, 32),     # ragged: whole prompts, an empty sequence, a single token
    ([700, 650], [129, 128], 7, 1, 128, 128),
    ([3, 200], [6, 4], 4, 1, 64, 16),                              # more new tokens than rows: the first three are padding
    ([900, 901], [65, 63], 9, 3, 64, 16),
    ([520], [20], 128, 1, 128, 16),
    ([260, 30], [33, 1], 40, 2, 64, 256),                          # twenty heads per KV head
    ([2500, 1300, 100], [700, 1, 100], 28, 4, 128, 128),
    ([1500] * 6, [17] * 6, 6, 2, 64, 32),
    ([4000, 130], [4, 4], 16, 4, 128, 64),
    ([385, 384, 383], [384, 384, 383], 5, 1, 64, 64),
]


def check_attention(c, O, lse):
    ref, L, A, dq = R.attention(c)
    delta = c.d * 2.0 ** -23 * dq
    tol = HALF * ref.abs() + (HALF + 2 * delta[..., None] + 2.0 ** -16) * A
    err = (O.double() - ref).abs()
    assert torch.isfinite(O).all()
    assert (err <= tol).all(), "worst ratio %.3f" % float((err / tol.clamp_min(1e-30)).max())
    if lse is not None:
        seen = torch.isfinite(L)
        assert torch.equal(torch.isneginf(lse), ~seen)
        assert ((lse.double() - L)[seen].abs() <= (delta + 2.0 ** -17 + 2.0 ** -21 * L.abs())[seen]).all()


def attend(c, with_lse=True):
    O = torch.full_like(c.Q, float("nan"))
    lse = torch.full((c.T, c.Hq), float("nan"), device="cuda") if with_lse else None
    binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, O, lse, c.ws)
    assert c.status() == binding.SEKA_OK
    return O, lse


@pytest.mark.parametrize("case", SINGLE + CHUNK)
def test_attention(case):
    c = R.Cache(*case, seed=1)
    O, lse = attend(c)
    check_attention(c, O, lse)
    again, _ = attend(c, with_lse=False)
    assert torch.equal(O, again)


def test_attention_fixed_count_wide_table_scale_and_in_place():
    # four new tokens each without offsets, a table with room for more pages, a scale of its own, the output over the queries
    c = R.Cache([200, 64, 4, 333], [4] * 4, 8, 4, 64, 32, seed=2, packed=False, max_pages=40, scale=0.31)
    O, lse = attend(c)
    check_attention(c, O, lse)
    Q = c.Q.clone()
    binding.seka_paged_attention(c.shape, Q, c.K, c.V, Q, None, c.ws)
    assert torch.equal(Q, O)


def test_attention_shared_pages():
    # two sequences that share the pages of a common prefix
    c = R.Cache([200, 210], [1, 12], 8, 2, 128, 64, seed=3)
    c.table[1, :3] = c.table[0, :3]
    c.table_d.copy_(c.table)
    c.V.view(-1, c.Hkv, c.d)[c.rows(1)] = c.V.view(-1, c.Hkv, c.d)[c.rows(1)].nan_to_num()
    O, lse = attend(c)
    check_attention(c, O, lse)


def test_attention_rising_and_extreme_scores():
    # keys that grow along the cache (the running maximum moves at every step) and scores far beyond the range of exp
    for d, n in ((128, 1), (64, 90), (128, 90)):
        c = R.Cache([1500], [n], 4, 2, d, 64, seed=4)
        K = c.K.view(-1, c.Hkv, d)
        r = c.rows(0).cuda()
        K[r] = (K[r].float() * torch.linspace(0.1, 30.0, 1500, device="cuda")[:, None, None]).bfloat16()
        O, lse = attend(c)
        check_attention(c, O, lse)


@pytest.mark.parametrize("case", SINGLE + CHUNK)
def test_mass(case):
    c = R.Cache(*case, seed=5)
    _, L, _, _ = R.attention(c)
    lse = L.float()
    m0 = torch.rand((c.B, c.Hkv, c.cap), generator=c.g).cuda()
    out = torch.full_like(m0, -7.0)
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, m0, out, c.ws)
    assert c.status() == binding.SEKA_OK
    ref, err = R.mass(c, lse, m0)
    inside = (torch.arange(c.cap, device="cuda")[None] < c.lens_d[:, None])[:, None].expand_as(out)
    # per weight: delta (through err), 2^-16 of the argument's fp32 arithmetic and the exponential; the sum: 2^-24 of itself per term
    terms = c.G * max(c.new + [1])
    tol = c.d * 2.0 ** -23 * err + (2.0 ** -16 + (terms + 2) * 2.0 ** -24) * ref.abs() + 1e-30
    assert (((out.double() - ref).abs() <= tol) | ~inside).all(), "worst ratio %.3f" % float(((out.double() - ref).abs() / tol)[inside].max())
    assert (out[~inside] == -7.0).all()                       # rows behind the sequences are left
    same = m0.clone()
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, same, same, c.ws)
    assert torch.equal(same[inside], out[inside]) and torch.equal(same[~inside], m0[~inside])
    zero = torch.full_like(m0, float("nan"))
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, zero, c.ws)
    ref0, _ = R.mass(c, lse, None)
    assert (((zero.double() - ref0).abs() <= tol) | ~inside).all()


ROPE = [
    # rot_dim, layout, scaling, dtype, head_dim, query heads, KV heads
    (128, "half", "plain", "bf16", 128, 8, 2), (128, "interleaved", "wavelength", "bf16", 128, 8, 2), (32, "interleaved", "linear", "f32", 64, 4, 4),
    (64, "half", "base", "f32", 64, 7, 1), (2, "half", "plain", "bf16", 64, 4, 2), (2, "interleaved", "linear", "f32", 128, 3, 3),
    (22, "half", "base", "bf16", 128, 5, 1), (22, "interleaved", "base", "bf16", 64, 4, 1), (126, "half", "wavelength", "f32", 128, 4, 2),
    (48, "half", "linear", "bf16", 64, 16, 16), (96, "half", "plain", "f32", 128, 32, 8), (0, "half", "plain", "bf16", 128, 4, 2), (0, "half", "plain", "f32", 64, 4, 4),
]


@pytest.mark.parametrize("r,layout,scaling,dtype,d,Hq,Hkv", ROPE)
@pytest.mark.parametrize("lens,new,page", [([40, 300, 16, 0, 5], [1, 37, 16, 0, 9], 16), ([900], [200], 256), ([7, 9], [1, 1], 32)])
def test_rope_append(r, layout, scaling, dtype, d, Hq, Hkv, lens, new, page):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    c = R.Cache(lens, new, Hq, Hkv, d, page, seed=6, dtype=dt)
    turns = binding.seka_rope_turns(r, 500000.0, scaling, 8.0).cuda() if r else None
    rope = binding.make_rope(turns, layout, 1.25) if r else None
    qkv = torch.randn((c.T, (Hq + 2 * Hkv) * d), generator=c.g).to(dt).cuda()
    q, k, v = qkv[:, :Hq * d].view(c.T, Hq, d), qkv[:, Hq * d:(Hq + Hkv) * d].view(c.T, Hkv, d), qkv[:, (Hq + Hkv) * d:].view(c.T, Hkv, d)
    pos = torch.randint(-5, 1000000, (c.T,), generator=c.g, dtype=torch.int32).cuda()
    Q_out = torch.full((c.T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    K0, V0 = c.K.clone(), c.V.clone()
    pc = torch.full((c.B, Hkv, c.cap), -9, dtype=torch.int32, device="cuda")
    binding.seka_rope_append(c.shape, rope, q, k, v, pos, Q_out, c.K, c.V, pc, c.ws)
    assert c.status() == binding.SEKA_OK

    def check(got, x):
        if rope is None:
            assert torch.equal(got, x.to(torch.bfloat16))
            return
        ref, size = R.rotate(x, pos, turns, layout, 1.25)
        # the reduced angle as fp32, its sine and cosine (2 ulp), two products and a sum: below 2^-20 of the magnitudes
        assert ((got.double() - ref).abs() <= HALF * ref.abs() + 2.0 ** -20 * size).all()
        assert torch.equal(got[..., r:], x[..., r:].to(torch.bfloat16))

    check(Q_out, q)
    K1, V1, p1 = K0.clone().view(-1, Hkv, d), V0.clone().view(-1, Hkv, d), torch.full_like(pc, -9)
    for b in range(c.B):
        l, n = lens[b], min(new[b], lens[b])            # tokens without a row are padding
        rows = c.rows(b)[l - n:].cuda()
        t = slice(c.cu[b + 1] - n, c.cu[b + 1])
        if n:
            x = c.K.view(-1, Hkv, d)[rows]
            if rope is None:
                assert torch.equal(x, k[t].to(torch.bfloat16))
            else:
                ref, size = R.rotate(k[t], pos[t], turns, layout, 1.25)
                assert ((x.double() - ref).abs() <= HALF * ref.abs() + 2.0 ** -20 * size).all()
        K1[rows], V1[rows] = c.K.view(-1, Hkv, d)[rows], v[t].to(torch.bfloat16)
        p1[b, :, l - n:l] = pos[t]
    same = lambda a, b: torch.equal(a.view(torch.int16), b.reshape(a.shape).view(torch.int16))
    assert same(c.K, K1) and same(c.V, V1) and torch.equal(pc, p1)       # other rows are left, bit for bit
    # without positions: the row in the cache; and in place over packed bf16 queries
    if dt == torch.bfloat16 and rope is not None:
        Q = q.contiguous()
        binding.seka_rope_append(c.shape, rope, Q, k, v, pos, Q, c.K, c.V, None, c.ws)
        assert torch.equal(Q, Q_out)
        own = torch.cat([torch.arange(lens[b] - new[b], lens[b]) for b in range(c.B)]).to(torch.int32).cuda()
        a, b2 = torch.empty_like(Q_out), torch.empty_like(Q_out)
        binding.seka_rope_append(c.shape, rope, q, k, v, None, a, c.K, c.V, pc, c.ws)
        binding.seka_rope_append(c.shape, rope, q, k, v, own, b2, c.K, c.V, None, c.ws)
        assert torch.equal(a, b2)
        for b in range(c.B):
            n = min(new[b], lens[b])
            assert torch.equal(pc[b, 0, lens[b] - n:lens[b]].cpu(), own[c.cu[b + 1] - n:c.cu[b + 1]].cpu())


def test_rope_padding_tokens():
    # idle sequences of a padded decode batch: nothing is stored for them
    c = R.Cache([0, 5, 0], [1, 1, 1], 4, 2, 64, 16, seed=7, packed=False)
    K0 = c.K.clone()
    turns = binding.seka_rope_turns(64).cuda()
    x = torch.randn((3, 8, 64), generator=c.g).bfloat16().cuda()
    Q_out = torch.full((3, 4, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([0, 4, 0], dtype=torch.int32, device="cuda")
    binding.seka_rope_append(c.shape, binding.make_rope(turns), x[:, :4], x[:, 4:6], x[:, 6:], pos, Q_out, c.K, c.V, None, c.ws)
    assert c.status() == binding.SEKA_OK and torch.isfinite(Q_out).all()
    row = int(c.rows(1)[4])
    changed = (c.K.view(torch.int16) != K0.view(torch.int16)).view(-1, 2 * 64).any(1).nonzero().flatten().tolist()
    assert changed == [row]


EVICT = [
    # lens, KV heads, head_dim, page, keep, recent, highlighted share
    ([1500], 8, 128, 16, 1024, 64, 0.1), ([100, 1000, 37, 0, 513], 2, 64, 32, 100, 10, 0.3), ([40, 41], 3, 64, 16, 40, 40, 0.0),
    ([5000, 4999], 1, 128, 128, 1, 0, 0.0), ([3000], 4, 64, 256, 2999, 5, 0.9), ([700, 300], 2, 128, 64, 256, 1000, 0.2), ([9000], 2, 64, 64, 3000 + 7, 100, 0.6),
]


def run_evict(c, mass_in, pos_in, protect, next_pos, keep, recent, inplace=False):
    K0, V0 = c.K.clone(), c.V.clone()
    mo = mass_in if inplace else torch.full_like(mass_in, -7.0)
    po = pos_in if inplace else torch.full_like(pos_in, -7)
    m0, p0 = mass_in.clone(), pos_in.clone()
    lens = c.lens_d if inplace else torch.full_like(c.lens_d, -1)
    want = R.evict(c, m0, p0, protect, next_pos, keep, recent)
    binding.seka_evict_cache(c.shape, c.K, c.V, mass_in, mo, pos_in, po, protect, next_pos, keep, recent, lens, c.ws)
    assert c.status() == binding.SEKA_OK
    assert lens.tolist() == [min(l, keep) for l in c.lens]
    K1, V1 = K0.clone().view(-1, c.Hkv, c.d), V0.clone().view(-1, c.Hkv, c.d)
    for b in range(c.B):
        rows = c.rows(b).cuda()
        for h in range(c.Hkv):
            src = torch.tensor(want[b][h], dtype=torch.long, device="cuda")
            n = len(src)
            assert torch.equal(mo[b, h, :n].view(torch.int32), m0[b, h, src].view(torch.int32))
            assert torch.equal(po[b, h, :n], p0[b, h, src])
            if inplace:
                assert torch.equal(mo[b, h, n:].view(torch.int32), m0[b, h, n:].view(torch.int32)) and torch.equal(po[b, h, n:], p0[b, h, n:])
            else:
                assert (mo[b, h, n:] == -7.0).all() and (po[b, h, n:] == -7).all()
            K1[rows[:n], h] = K0.view(-1, c.Hkv, c.d)[rows[src], h]
            V1[rows[:n], h] = V0.view(-1, c.Hkv, c.d)[rows[src], h]
    assert torch.equal(c.K.view(torch.int16), K1.view_as(c.K).view(torch.int16)) and torch.equal(c.V.view(torch.int16), V1.view_as(c.V).view(torch.int16))


@pytest.mark.parametrize("lens,Hkv,d,page,keep,recent,share", EVICT)
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(lens, Hkv, d, page, keep, recent, share, kind):
    c = R.Cache(lens, [0] * len(lens), Hkv, Hkv, d, page, seed=8)
    size = (c.B, Hkv, c.cap)
    if kind == "spread":
        m = torch.randn(size, generator=c.g).mul(2.0).exp()
    elif kind == "ties":
        m = torch.randint(0, 3, size, generator=c.g).float()
    else:                       # zeros of both signs, negative numbers, infinities, NaN, subnormal numbers
        vals = torch.tensor([0.0, -0.0, -1.5, float("inf"), float("-inf"), float("nan"), 1e-42, -1e-42, 2.0, 2.0000002])
        m = vals[torch.randint(0, len(vals), size, generator=c.g)]
    pos = torch.stack([torch.stack([torch.randperm(2 * c.cap, generator=c.g)[:c.cap] for _ in range(Hkv)]) for _ in range(c.B)]).to(torch.int32)
    next_pos = torch.full((c.B,), 2 * c.cap, dtype=torch.int32)
    protect = (torch.rand((c.B, c.cap), generator=c.g) < share).to(torch.uint8) if share else None      # positions behind it: not protected
    run_evict(c, m.cuda(), pos.cuda(), None if protect is None else protect.cuda(), next_pos.cuda(), keep, recent)


def test_evict_long_rows_and_many_pairs():
    # one sequence whose ranks do not fit in a CTA's shared memory, in a batch that leaves each pair one CTA
    c = R.Cache([44000] + [20] * 37, [0] * 38, 4, 4, 64, 256, seed=12)
    m = torch.randn((c.B, 4, c.cap), generator=c.g).mul(1.5).exp().cuda()
    pos = torch.arange(c.cap, dtype=torch.int32).expand(c.B, 4, -1).contiguous().cuda()
    protect = (torch.rand((c.B, 30000), generator=c.g) < 0.2).to(torch.uint8).cuda()
    run_evict(c, m, pos, protect, c.lens_d.clone(), 15000, 100)


def test_evict_in_place_and_again():
    c = R.Cache([900, 64], [0, 0], 2, 2, 64, 16, seed=9)
    m = torch.rand((2, 2, c.cap), generator=c.g).cuda()
    pos = torch.arange(c.cap, dtype=torch.int32).expand(2, 2, -1).contiguous().cuda()
    nxt = torch.tensor([900, 64], dtype=torch.int32, device="cuda")
    for keep in (500, 499, 30):
        run_evict(c, m, pos, None, nxt, keep, 8, inplace=True)
        c.lens = [min(l, keep) for l in c.lens]


def test_refusals_on_the_device():
    # lengths, offsets and pages that only the device sees; every one is reported and nothing outside the buffers is touched
    def fresh():
        c = R.Cache([100, 90], [3, 2], 4, 2, 64, 16, seed=10)
        c.m = torch.arange(c.cap, dtype=torch.float32, device="cuda").expand(2, 2, -1).contiguous()
        c.p = torch.zeros((2, 2, c.cap), dtype=torch.int32, device="cuda")
        c.x = torch.zeros((5, 4, 64), dtype=torch.bfloat16, device="cuda")
        return c

    calls = {
        "append": lambda c: binding.seka_rope_append(c.shape, None, c.x, c.x[:, :2], c.x[:, 2:], None, c.x.clone(), c.K, c.V, None, c.ws),
        "attend": lambda c: binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, torch.empty_like(c.Q), None, c.ws),
        "mass": lambda c: binding.seka_attention_mass(c.shape, c.Q, c.K, torch.zeros((5, 4), device="cuda"), None, c.m, c.ws),
        "evict": lambda c: binding.seka_evict_cache(c.shape, c.K, c.V, c.m, c.m, c.p, c.p, None, c.lens_d, 50, 4, c.lens_d.clone(), c.ws),
    }
    bad = {
        "too long": lambda c: c.lens_d.copy_(torch.tensor([c.cap + 1, 90])),
        "negative": lambda c: c.lens_d.copy_(torch.tensor([-1, 90])),
        "page": lambda c: c.table_d[0].fill_(c.n_pages),
        "no page": lambda c: c.table_d[1].fill_(-1),
        "offsets": lambda c: c.cu_d.copy_(torch.tensor([0, 4, 5])),          # four new tokens where three is the most
        "behind": lambda c: c.cu_d.copy_(torch.tensor([0, 3, 6])),
    }
    for what, spoil in bad.items():
        for name, call in calls.items():
            if name == "evict" and what in ("offsets", "behind"):
                continue                        # it has no new tokens
            c = fresh()
            spoil(c)
            call(c)
            assert c.status() == binding.SEKA_ERR_INVALID_ARG, (what, name)
            # the next launch on this workspace does nothing until the status is cleared
            O = torch.full_like(c.Q, 3.0)
            binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, O, None, c.ws)
            assert (O == 3.0).all()
            binding.seka_reset_status(c.ws)
            assert c.status() == binding.SEKA_OK


def test_far_pages():
    # pages whose elements lie beyond 2^31 of the pool's first
    page, Hkv, d = 256, 8, 128
    n_pages = (1 << 31) // (page * Hkv * d) + 40
    c = R.Cache([600, 50], [20, 1], 16, Hkv, d, page, seed=11, n_pages=n_pages)
    assert int(c.table.max()) * page * Hkv * d > 1 << 31
    turns = binding.seka_rope_turns(d).cuda()
    pos = torch.arange(c.T, dtype=torch.int32, device="cuda")
    x = torch.randn((c.T, 16 + 2 * Hkv, d), generator=c.g).bfloat16().cuda()
    binding.seka_rope_append(c.shape, binding.make_rope(turns), x[:, :16], x[:, 16:24], x[:, 24:], pos, c.Q, c.K, c.V, None, c.ws)
    ref, size = R.rotate(x[:20, 16:24], pos[:20], turns, "half")
    got = c.K.view(-1, Hkv, d)[c.rows(0)[580:].cuda()].double()
    assert ((got - ref).abs() <= HALF * ref.abs() + 2.0 ** -20 * size).all()
    O, lse = attend(c)
    check_attention(c, O, lse)
    m = torch.zeros((c.B, Hkv, c.cap), device="cuda")
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, m, c.ws)
    ref, err = R.mass(c, lse)
    assert ((m.double() - ref).abs() <= d * 2.0 ** -23 * err + (2.0 ** -16 + 2 * 20 * 2.0 ** -24) * ref + 1e-30).all()
    r = c.rows(0).cuda()
    before = c.K.view(-1, Hkv, d)[r]
    p = torch.arange(c.cap, dtype=torch.int32).expand(2, Hkv, -1).contiguous().cuda()
    lens = c.lens_d.clone()
    want = R.evict(c, m, p, None, lens, 300, 10)
    binding.seka_evict_cache(c.shape, c.K, c.V, m, m, p, p, None, lens, 300, 10, lens, c.ws)
    assert c.status() == binding.SEKA_OK and lens.tolist() == [300, 50]
    for h in range(Hkv):
        assert torch.equal(c.K.view(-1, Hkv, d)[r[:300], h], before[torch.tensor(want[0][h], device="cuda"), h])
