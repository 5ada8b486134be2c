"""Rotation and append in launches whose blocks take several tokens (four, in bf16 eight, where that still gives every SM four blocks):
sequences that share a block, a short last block, padding and tokens that nobody owns inside a block, all forms of the rotation."""
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


FORMS = [
    # rot_dim, layout, head_dim, query heads, KV heads
    (128, "half", 128, 8, 2), (64, "half", 64, 7, 1), (48, "half", 64, 4, 4), (96, "half", 128, 3, 1), (128, "interleaved", 128, 28, 4), (20, "interleaved", 64, 5, 1),
    (22, "half", 128, 6, 2), (2, "half", 64, 4, 2), (126, "half", 128, 5, 1), (50, "half", 64, 17, 1), (0, "half", 128, 4, 2),
]


def ragged(T, kind, g):
    """New tokens of sequences that add up to T."""
    new, left = [], T
    while left > 0:
        n = int(torch.randint(*{"short": (0, 10), "mixed": (1, 700)}[kind], (1,), generator=g))
        new.append(min(n, left))
        left -= new[-1]
    return new


@pytest.mark.parametrize("r,layout,d,Hq,Hkv", FORMS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["short", "mixed", "one"])
@pytest.mark.parametrize("per_block", [4, 8])
def test_several_tokens_a_block(r, layout, d, Hq, Hkv, dtype, kind, per_block):
    sm = torch.cuda.get_device_properties(0).multi_processor_count
    g = torch.Generator().manual_seed(50 + per_block)
    own = per_block * 4 * sm + 3                                 # just above the threshold of four, or of eight, and no multiple
    tail = 6                                                     # tokens behind the last sequence
    new = [own] if kind == "one" else ragged(own, kind, g)
    # a part of the sequences has fewer rows than new tokens (the first ones are padding), a few are idle
    lens = [0 if i % 11 == 5 else n // 2 if i % 7 == 3 else n + (i * 13) % 40 for i, n in enumerate(new)]
    c = R.Cache(lens, new, Hq, Hkv, d, 16, seed=51)
    T = own + tail
    shape = binding.make_paged_shape(batch=c.B, max_new=max(new), total_new=T, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_size=16,
                                     n_pages=c.n_pages, block_table=c.table_d, cache_lens=c.lens_d, cu_new=c.cu_d, dtype=dtype)
    ws = binding.new_paged_workspace(shape)
    turns = binding.seka_rope_turns(r, 500000.0).cuda() if r else None
    rope = binding.make_rope(turns, layout, 0.75) if r else None
    qkv = torch.randn((T, Hq + 2 * Hkv, d), generator=g).to(dtype).cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    own_rows = torch.cat([torch.arange(l - n, l) for l, n in zip(lens, new)] + [torch.full((tail,), -1)]).to(torch.int32).cuda()
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(new)]).cuda()
    real = own_rows[:own] >= 0
    pool = c.table_d.long()[seq, (own_rows[:own].long().clamp_min(0)) // 16] * 16 + own_rows[:own].long() % 16
    rows = pool[real]
    far = torch.randint(-5, 1000000, (T,), generator=g, dtype=torch.int32).cuda()
    K0, V0 = c.K.clone(), c.V.clone()
    for pos in (far, None):
        at = far if pos is not None else own_rows
        c.K.copy_(K0); c.V.copy_(V0)
        Q_out = torch.full((T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        pc = torch.full((c.B, Hkv, c.cap), -9, dtype=torch.int32, device="cuda")
        binding.seka_rope_append(shape, rope, q, k, v, pos, Q_out, c.K, c.V, pc, ws)
        assert binding.seka_poll_status(ws) == binding.SEKA_OK

        def check(got, x, p):
            if rope is None:
                assert torch.equal(got, x.to(torch.bfloat16))
                return
            ref, size = R.rotate(x, p, turns, layout, 0.75)
            assert ((got.double() - ref).abs() <= HALF * ref.abs() + 2.0 ** -20 * size).all()          # as in test_gpu_paged.py
            assert torch.equal(got[..., r:], x[..., r:].to(torch.bfloat16))

        check(Q_out[:own], q[:own], at[:own])
        assert torch.isfinite(Q_out).all()                                   # tokens that nobody owns are written too
        check(c.K.view(-1, Hkv, d)[rows], k[:own][real], at[:own][real])
        K1, V1, p1 = K0.clone().view(-1, Hkv, d), V0.clone().view(-1, Hkv, d), torch.full_like(pc, -9)
        K1[rows], V1[rows] = c.K.view(-1, Hkv, d)[rows], v[:own][real].to(torch.bfloat16)
        p1[seq[real], :, own_rows[:own][real].long()] = at[:own][real][:, None].expand(-1, Hkv)
        same = lambda a, b: torch.equal(a.view(torch.int16), b.view_as(a).view(torch.int16))
        assert same(c.K, K1) and same(c.V, V1) and torch.equal(pc, p1)       # other rows are left, bit for bit
        if dtype == torch.bfloat16:                                          # in place over packed queries
            Q = q.contiguous()
            binding.seka_rope_append(shape, rope, Q, k, v, pos, Q, c.K, c.V, pc, ws)
            assert torch.equal(Q, Q_out) and same(c.K, K1) and same(c.V, V1) and torch.equal(pc, p1)


@pytest.mark.parametrize("r,layout", [(128, "half"), (128, "interleaved"), (22, "half")])
def test_more_groups_than_are_in_flight(r, layout):
    # many heads: a warp of a block comes back for further groups of rows, with several tokens a block and with several blocks a token
    sm = torch.cuda.get_device_properties(0).multi_processor_count
    for T in (16 * sm + 1, 3):
        c = R.Cache([T + 5], [T], 64, 32, 128, 64, seed=52)
        turns = binding.seka_rope_turns(r).cuda()
        x = torch.randn((T, 128, 128), generator=c.g).bfloat16().cuda()
        pos = torch.randint(0, 100000, (T,), generator=c.g, dtype=torch.int32).cuda()
        Q = torch.full((T, 64, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        binding.seka_rope_append(c.shape, binding.make_rope(turns, layout), x[:, :64], x[:, 64:96], x[:, 96:], pos, Q, c.K, c.V, None, c.ws)
        assert c.status() == binding.SEKA_OK
        rows = c.rows(0)[5:].cuda()
        for got, want in ((Q, x[:, :64]), (c.K.view(-1, 32, 128)[rows], x[:, 64:96])):
            ref, size = R.rotate(want, pos, turns, layout)
            assert ((got.double() - ref).abs() <= HALF * ref.abs() + 2.0 ** -20 * size).all()
        assert torch.equal(c.V.view(-1, 32, 128)[rows], x[:, 96:])


def test_a_bad_sequence_inside_a_block():
    # offsets out of range in the middle of a long launch are reported whichever block holds them
    sm = torch.cuda.get_device_properties(0).multi_processor_count
    n = (16 * sm + 100) // 5
    c = R.Cache([n] * 5, [n] * 5, 4, 2, 64, 64, seed=53)
    x = torch.zeros((c.T, 8, 64), dtype=torch.bfloat16, device="cuda")
    for spoil in (lambda: c.lens_d[3:4].fill_(c.cap + 1), lambda: c.table_d[3].fill_(c.n_pages), lambda: c.cu_d[3:4].fill_(c.T + 1)):
        keep = [t.clone() for t in (c.lens_d, c.table_d, c.cu_d)]
        spoil()
        binding.seka_rope_append(c.shape, None, x[:, :4], x[:, 4:6], x[:, 6:], None, torch.empty_like(c.Q), c.K, c.V, None, c.ws)
        assert c.status() == binding.SEKA_ERR_INVALID_ARG
        binding.seka_reset_status(c.ws)
        for t, k in zip((c.lens_d, c.table_d, c.cu_d), keep):
            t.copy_(k)
    binding.seka_rope_append(c.shape, None, x[:, :4], x[:, 4:6], x[:, 6:], None, torch.empty_like(c.Q), c.K, c.V, None, c.ws)
    assert c.status() == binding.SEKA_OK
