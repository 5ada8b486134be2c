"""The paged calls as they are used: one after another on one cache behind the key edit, on other streams, side by side, in captured
graphs, in padded batches, with cold caches, and with a wait that runs out.  Tolerances are those of test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from oracle import edit_keys
from paper_2603_01281_b200 import binding

import paged_ref as R
from test_gpu_paged import CHUNK, HALF, SINGLE, attend, check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    binding.load()


class Server:
    """One layer of a server: its cache, the state per cached row, the calls of a step in their order."""

    def __init__(self, lens, new, Hq, Hkv, d, page, seed, max_pages=None, n_pages=None):
        self.c = c = R.Cache(lens, new, Hq, Hkv, d, page, seed=seed, max_pages=max_pages, n_pages=n_pages)
        self.qkv = torch.randn((c.T, Hq + 2 * Hkv, d), generator=c.g).bfloat16().cuda()
        self.turns = binding.seka_rope_turns(d, scaling="linear", scale=2.0).cuda()
        self.rope = binding.make_rope(self.turns)
        self.O, self.lse = torch.full_like(c.Q, float("nan")), torch.full((c.T, Hq), float("nan"), device="cuda")
        self.mass = torch.rand((c.B, Hkv, c.cap), generator=c.g).cuda()
        self.pos = torch.arange(c.cap, dtype=torch.int32, device="cuda").expand(c.B, Hkv, -1).contiguous()
        self.protect = (torch.rand((c.B, c.cap), generator=c.g) < 0.1).to(torch.uint8).cuda()
        self.next = c.lens_d.clone()
        self.positions = torch.cat([torch.arange(l - n, l) for l, n in zip(lens, new)]).to(torch.int32).cuda()

    def slices(self):
        Hq, Hkv = self.c.Hq, self.c.Hkv
        return self.qkv[:, :Hq], self.qkv[:, Hq:Hq + Hkv], self.qkv[:, Hq + Hkv:]

    def append(self):
        c = self.c
        binding.seka_rope_append(c.shape, self.rope, *self.slices(), self.positions, c.Q, c.K, c.V, self.pos, c.ws)

    def attend(self):
        c = self.c
        binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, self.O, self.lse, c.ws)

    def weigh(self):
        c = self.c
        binding.seka_attention_mass(c.shape, c.Q, c.K, self.lse, self.mass, self.mass, c.ws)

    def cut(self, keep):
        c = self.c
        binding.seka_evict_cache(c.shape, c.K, c.V, self.mass, self.mass, self.pos, self.pos, self.protect, self.next, keep, 16, c.lens_d, c.ws)

    def step(self, keep):
        self.append()
        self.attend()
        self.weigh()
        self.cut(keep)

    def everything(self):
        c = self.c
        return [x.clone() for x in (c.K, c.V, c.Q, self.O, self.lse, self.mass, self.pos, c.lens_d)]


def same(a, b):
    ints = {torch.bfloat16: torch.int16, torch.float32: torch.int32, torch.int32: torch.int32}
    return all(torch.equal(x.view(ints[x.dtype]), y.view(ints[y.dtype])) for x, y in zip(a, b))


# few rows, and many
STEPS = [([300, 41, 130], [1, 1, 1], 8, 2, 128, 16, 100), ([700, 90, 40, 513], [257, 90, 1, 13], 14, 2, 64, 32, 64)]


@pytest.mark.parametrize("lens,new,Hq,Hkv,d,page,keep", STEPS)
def test_a_step_after_another(lens, new, Hq, Hkv, d, page, keep):
    s = Server(lens, new, Hq, Hkv, d, page, seed=20)
    c = s.c
    # the highlighted new keys are edited where the projection left them (a copy of the slice: the edit takes packed keys)
    rng = np.random.default_rng(1)
    U = np.linalg.qr(rng.standard_normal((1, Hkv, d, 8)))[0].astype(np.float32)
    mask, gain = (rng.random(c.T) < 0.5).astype(np.uint8), np.linspace(0.5, 1.5, c.B).astype(np.float32)
    es = binding.make_shape(batch=c.B, max_seqlen=max(new), n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=d, rank=8, total_tokens=c.T, cu_seqlens=c.cu_d)
    K = s.slices()[1].contiguous()
    K0 = K.float().cpu().numpy()
    ews = binding.new_workspace(es)
    binding.seka_edit_keys(es, K, K, torch.from_numpy(mask).cuda(), torch.from_numpy(U).cuda(), None, torch.from_numpy(gain).cuda(), None, ews)
    assert binding.seka_poll_status(ews) == binding.SEKA_OK
    ref = edit_keys(K0, mask, np.asarray(c.cu, dtype=np.int32), U, gain=gain)
    assert (np.abs(K.double().cpu().numpy() - ref) / np.abs(ref).max(axis=-1, keepdims=True)).max() <= 2.0 ** -8
    s.qkv[:, Hq:Hq + Hkv] = K
    # rotation and append: the pages hold the rotated edited keys, the positions of the new rows are noted
    s.append()
    assert c.status() == binding.SEKA_OK
    want, size = R.rotate(K, s.positions, s.turns, "half")
    for b in range(c.B):
        rows, t = c.rows(b)[lens[b] - new[b]:].cuda(), slice(c.cu[b], c.cu[b + 1])
        got = c.K.view(-1, Hkv, d)[rows].double()
        assert ((got - want[t]).abs() <= HALF * want[t].abs() + 2.0 ** -20 * size[t]).all()
        assert torch.equal(c.V.view(-1, Hkv, d)[rows], s.slices()[2][t])
        assert torch.equal(s.pos[b, 0, lens[b] - new[b]:lens[b]], s.positions[t])
    s.attend()
    assert c.status() == binding.SEKA_OK
    check_attention(c, s.O, s.lse)
    before = s.mass.clone()
    s.weigh()
    assert c.status() == binding.SEKA_OK
    inside = (torch.arange(c.cap, device="cuda")[None] < c.lens_d[:, None])[:, None].expand_as(s.mass)
    ref, err = R.mass(c, s.lse, before)
    tol = d * 2.0 ** -23 * err + (2.0 ** -16 + (c.G * max(new) + 2) * 2.0 ** -24) * ref.abs() + 1e-30
    assert (((s.mass.double() - ref).abs() <= tol) | ~inside).all() and torch.equal(s.mass[~inside], before[~inside])
    want = R.evict(c, s.mass, s.pos, s.protect, s.next, keep, 16)
    K1, m1, p1 = c.K.clone().view(-1, Hkv, d), s.mass.clone(), s.pos.clone()
    s.cut(keep)
    assert c.status() == binding.SEKA_OK and c.lens_d.tolist() == [min(l, keep) for l in lens]
    for b in range(c.B):
        for h in range(Hkv):
            src = torch.tensor(want[b][h], device="cuda")
            rows = c.rows(b).cuda()
            assert torch.equal(c.K.view(-1, Hkv, d)[rows[:len(src)], h], K1[rows[src], h])
            assert torch.equal(s.mass[b, h, :len(src)], m1[b, h, src]) and torch.equal(s.pos[b, h, :len(src)], p1[b, h, src])
    # the next token of every sequence: one more row behind what was kept, at the position that follows the text
    c.lens, c.new, c.T, c.cu = [min(l, keep) + 1 for l in lens], [1] * c.B, c.B, list(range(c.B + 1))
    c.lens_d += 1
    c.shape = binding.make_paged_shape(batch=c.B, max_new=1, total_new=c.B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_size=page,
                                       n_pages=c.n_pages, block_table=c.table_d, cache_lens=c.lens_d)
    c.ws, c.Q = binding.new_paged_workspace(c.shape), c.Q[:c.B].clone()
    s.qkv, s.positions = s.qkv[:c.B], s.next.clone()
    s.O, s.lse = torch.full_like(c.Q, float("nan")), torch.full((c.T, Hq), float("nan"), device="cuda")
    s.append()
    s.attend()
    assert c.status() == binding.SEKA_OK
    check_attention(c, s.O, s.lse)
    want, size = R.rotate(s.slices()[1], s.positions, s.turns, "half")
    for b in range(c.B):
        row = int(c.rows(b)[-1])
        assert ((c.K.view(-1, Hkv, d)[row].double() - want[b]).abs() <= HALF * want[b].abs() + 2.0 ** -20 * size[b]).all()


@pytest.mark.parametrize("lens,new,Hq,Hkv,d,page,keep", STEPS)
def test_captured_step(lens, new, Hq, Hkv, d, page, keep):
    # the graph is captured once; lengths, pages, offsets and data then change under it
    s = Server(lens, new, Hq, Hkv, d, page, seed=21, max_pages=60, n_pages=200)
    c = s.c
    Server(lens, new, Hq, Hkv, d, page, seed=21).step(keep)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        s.step(keep)
    for seed, other, fresh in ((22, lens, new), (23, [l + 150 for l in lens[::-1]], new[::-1]), (24, [max(n, 1) for n in new], new)):
        e = Server(other, fresh, Hq, Hkv, d, page, seed=seed, max_pages=60, n_pages=200)
        for dst, src in ((c.K, e.c.K), (c.V, e.c.V), (c.table_d, e.c.table_d), (c.lens_d, e.c.lens_d), (c.cu_d, e.c.cu_d),
                         (s.qkv, e.qkv), (s.mass, e.mass), (s.pos, e.pos), (s.protect, e.protect), (s.next, e.next), (s.positions, e.positions)):
            dst.copy_(src)
        s.O.fill_(float("nan")); s.lse.fill_(float("nan"))
        e.step(keep)
        torch.cuda.synchronize()
        assert e.c.status() == binding.SEKA_OK
        graph.replay()
        torch.cuda.synchronize()
        assert c.status() == binding.SEKA_OK
        assert same(s.everything(), e.everything()) and torch.isfinite(s.O).all()


def test_other_streams_and_side_by_side():
    # the calls run on the current stream, behind what that stream has still to do; two servers at a time, a workspace each
    args = [([900, 130, 1100], [1, 1, 1], 16, 4, 128, 64, 256), ([700, 650, 90], [129, 128, 60], 7, 1, 64, 16, 200)]
    want = []
    for i, a in enumerate(args):
        s = Server(*a[:6], seed=25 + i)
        s.step(a[6])
        torch.cuda.synchronize()
        want.append(s.everything())
    for _ in range(5):
        servers = [Server(*a[:6], seed=25 + i) for i, a in enumerate(args)]
        late = [s.qkv.clone() for s in servers]
        for s in servers:
            s.qkv.fill_(float("nan"))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in servers]
        for s, st, x in zip(servers, streams, late):
            with torch.cuda.stream(st):
                torch.cuda._sleep(2_000_000)                # about a millisecond, then the data the calls need
                s.qkv.copy_(x)
        for part in ("append", "attend", "weigh"):
            for s, st in zip(servers, streams):
                with torch.cuda.stream(st):
                    getattr(s, part)()
        for s, st, a in zip(servers, streams, args):
            with torch.cuda.stream(st):
                s.cut(a[6])
        torch.cuda.synchronize()
        for s, w in zip(servers, want):
            assert s.c.status() == binding.SEKA_OK and same(s.everything(), w)


def test_padded_batches():
    # tokens behind the last sequence, idle sequences, tables wider than needed: rows that nobody owns are left as they were
    for new, T in (([1, 0, 1, 0], 4), ([40, 0, 65, 0], 160)):
        lens = [100, 0, 300, 0]
        c = R.Cache(lens, new, 8, 2, 128, 16, seed=30, max_pages=64)
        own = sum(new)
        shape = binding.make_paged_shape(batch=4, max_new=max(new), total_new=T, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16,
                                         n_pages=c.n_pages, block_table=c.table_d, cache_lens=c.lens_d, cu_new=c.cu_d)
        ws = binding.new_paged_workspace(shape)
        qkv = torch.full((T, 12, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        qkv[:own] = torch.randn((own, 12, 128), generator=c.g).bfloat16().cuda()
        Q, O, lse = torch.zeros((T, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.full((T, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, 8), 3.0, device="cuda")
        rope = binding.make_rope(binding.seka_rope_turns(128).cuda())
        K0 = c.K.clone()
        binding.seka_rope_append(shape, rope, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], None, Q, c.K, c.V, None, ws)
        written = torch.cat([c.rows(b)[lens[b] - new[b]:] for b in range(4)]).sort().values.tolist()
        assert (c.K.view(torch.int16) != K0.view(torch.int16)).view(-1, 256).any(1).nonzero().flatten().tolist() == written
        binding.seka_paged_attention(shape, Q, c.K, c.V, O, lse, ws)
        assert binding.seka_poll_status(ws) == binding.SEKA_OK
        assert (O[own:] == 3.0).all() and (lse[own:] == 3.0).all()
        c.Q = Q[:own].contiguous()
        check_attention(c, O[:own], lse[:own])
        m = torch.full((4, 2, c.cap), -7.0, device="cuda")
        binding.seka_attention_mass(shape, Q, c.K, lse, None, m, ws)
        assert binding.seka_poll_status(ws) == binding.SEKA_OK
        ref, err = R.mass(c, lse[:own])
        inside = (torch.arange(c.cap, device="cuda")[None] < c.lens_d[:, None])[:, None].expand_as(m)
        tol = 128 * 2.0 ** -23 * err + (2.0 ** -16 + (4 * max(new) + 2) * 2.0 ** -24) * ref + 1e-30
        assert (((m.double() - ref).abs() <= tol) | ~inside).all() and (m[~inside] == -7.0).all()


def test_a_page_twice():
    # a sequence whose table names a page twice (a repeated passage): attention and weights read it at both places
    for n in (1, 70):
        c = R.Cache([200], [n], 4, 2, 64, 32, seed=31)
        c.table[0, 1] = c.table[0, 0]
        c.table_d.copy_(c.table)
        O, lse = attend(c)
        check_attention(c, O, lse)
        m = torch.zeros((1, 2, c.cap), device="cuda")
        binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, m, c.ws)
        assert c.status() == binding.SEKA_OK
        ref, err = R.mass(c, lse)
        assert ((m.double() - ref).abs() <= 64 * 2.0 ** -23 * err + (2.0 ** -16 + (2 * n + 2) * 2.0 ** -24) * ref + 1e-30).all()


def test_cold_caches_give_the_same():
    # data that comes late from memory, behind a buffer larger than the L2 cache full of NaN: every result as it was
    cs = [R.Cache(*case, seed=32) for case in SINGLE + CHUNK]
    first = [attend(c) for c in cs]
    masses = []
    for c, (_, lse) in zip(cs, first):
        m = torch.zeros((c.B, c.Hkv, c.cap), device="cuda")
        binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, m, c.ws)
        masses.append(m)
    flush = torch.empty(200 << 20, dtype=torch.uint8, device="cuda")
    for turn in range(6):
        for c, (O0, lse0), m0 in zip(cs, first, masses):
            O, lse, m = torch.full_like(O0, 7.0), torch.full_like(lse0, 7.0), torch.zeros_like(m0)
            flush.fill_(0xff if turn % 2 else 0x7f)
            torch.cuda.synchronize()
            binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, O, lse, c.ws)
            torch.cuda.synchronize()
            flush.fill_(0x7f)
            torch.cuda.synchronize()
            binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, m, c.ws)
            assert c.status() == binding.SEKA_OK
            assert same([O, lse, m], [O0, lse0, m0]), c.lens


@pytest.mark.parametrize("lens,new,d", [([600, 400], [200, 300], 128), ([600, 400], [200, 300], 64), ([700], [100], 128), ([700], [100], 64)])
def test_a_wait_that_runs_out(lens, new, d):
    c = R.Cache(lens, new, 4, 4, d, 64, seed=33)
    good, _ = attend(c)
    words = c.ws[:256].view(torch.int32)
    words[4] = 1                        # the first pair of key and value tiles of CTA 0 never comes
    words[5] = 5000                     # every wait gives up after 5 ms
    O = torch.full_like(c.Q, float("nan"))
    torch.cuda.synchronize()
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, O, None, c.ws)
    t1.record()
    assert c.status() == binding.SEKA_ERR_TIMEOUT
    assert t0.elapsed_time(t1) < 2000.0
    O.fill_(float("nan"))
    binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, O, None, c.ws)             # does nothing
    assert c.status() == binding.SEKA_ERR_TIMEOUT and torch.isnan(O).all()
    binding.seka_reset_status(c.ws)
    again, _ = attend(c)
    assert torch.equal(again, good)


def test_refused_tensors():
    s = Server([100, 40], [30, 40], 4, 2, 64, 16, seed=34)
    c = s.c
    q, k, v = s.slices()
    before = s.everything()

    def append(q=q, k=k, v=v, ws=c.ws, out=c.Q, pos=s.positions):
        binding.seka_rope_append(c.shape, s.rope, q, k, v, pos, out, c.K, c.V, s.pos, ws)

    wide = torch.zeros((c.T, 4, 128), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q[:1].expand(c.T, -1, -1)), dict(k=k.transpose(1, 2)), dict(v=v.float()), dict(q=wide[..., ::2]), dict(ws=c.ws.cpu()), dict(ws=None),
                dict(ws=c.ws.view(torch.int32)), dict(out=torch.empty_like(q.float())), dict(pos=s.positions.long())):
        with pytest.raises(ValueError):
            append(**bad)
    odd = torch.zeros(c.T * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(c.T, 4, 64)
    with pytest.raises(binding.SekaError):
        append(q=odd)                                       # not on a 16-byte boundary
    with pytest.raises(binding.SekaError):
        append(ws=c.ws[:1024])
    m = torch.zeros(s.mass.numel() + 1, device="cuda")[1:].view_as(s.mass)
    with pytest.raises(binding.SekaError):
        binding.seka_evict_cache(c.shape, c.K, c.V, m, s.mass, s.pos, s.pos, None, s.next, 20, 4, c.lens_d, c.ws)
    with pytest.raises(ValueError):
        binding.seka_paged_attention(c.shape, c.Q, c.K[1:], c.V, s.O, s.lse, c.ws)
    with pytest.raises(ValueError):
        binding.seka_attention_mass(c.shape, c.Q, c.K, s.lse, s.mass[:, :, :-1], s.mass, c.ws)
    assert c.status() == binding.SEKA_OK and same(s.everything(), before)


def test_a_step_without_new_tokens():
    # a padded packed step in which every sequence is idle: tokens are rotated, nothing is stored, attended to or weighed
    c = R.Cache([100, 40], [0, 0], 4, 2, 64, 16, seed=35)
    shape = binding.make_paged_shape(batch=2, max_new=0, total_new=3, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, n_pages=c.n_pages,
                                     block_table=c.table_d, cache_lens=c.lens_d, cu_new=c.cu_d)
    ws = binding.new_paged_workspace(shape)
    qkv = torch.randn((3, 8, 64), generator=c.g).bfloat16().cuda()
    Q, O, lse = torch.zeros_like(qkv[:, :4]), torch.full((3, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((3, 4), 3.0, device="cuda")
    Q, K0, V0 = Q.contiguous(), c.K.clone(), c.V.clone()
    pos = torch.tensor([7, 8, 9], dtype=torch.int32, device="cuda")
    turns = binding.seka_rope_turns(64).cuda()
    binding.seka_rope_append(shape, binding.make_rope(turns), qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], pos, Q, c.K, c.V, None, ws)
    binding.seka_paged_attention(shape, Q, c.K, c.V, O, lse, ws)
    m0 = torch.rand((2, 2, c.cap), generator=c.g).cuda()
    m = torch.full_like(m0, -7.0)
    binding.seka_attention_mass(shape, Q, c.K, lse, m0, m, ws)
    assert binding.seka_poll_status(ws) == binding.SEKA_OK
    want, size = R.rotate(qkv[:, :4], pos, turns, "half")
    assert ((Q.double() - want).abs() <= HALF * want.abs() + 2.0 ** -20 * size).all()
    assert same([c.K, c.V], [K0, V0]) and (O == 3.0).all() and (lse == 3.0).all()
    inside = (torch.arange(c.cap, device="cuda")[None] < c.lens_d[:, None])[:, None].expand_as(m)
    assert torch.equal(m[inside], m0[inside]) and (m[~inside] == -7.0).all()


def test_every_sequence_is_looked_at():
    # offsets and lengths out of range that own none of the call's tokens are reported too
    for spoil in (lambda c: c.lens_d[2:].fill_(c.cap + 1), lambda c: c.lens_d[2:].fill_(-5), lambda c: c.cu_d[2:].copy_(torch.tensor([33, 1000]))):
        c = R.Cache([100, 40, 30], [30, 3, 0], 4, 2, 64, 16, seed=36)
        spoil(c)
        x = torch.zeros((c.T, 8, 64), dtype=torch.bfloat16, device="cuda")
        calls = [lambda: binding.seka_rope_append(c.shape, None, x[:, :4], x[:, 4:6], x[:, 6:], None, torch.empty_like(c.Q), c.K, c.V, None, c.ws),
                 lambda: binding.seka_paged_attention(c.shape, c.Q, c.K, c.V, torch.empty_like(c.Q), None, c.ws),
                 lambda: binding.seka_attention_mass(c.shape, c.Q, c.K, torch.zeros((c.T, 4), device="cuda"), None, torch.zeros((3, 2, c.cap), device="cuda"), c.ws)]
        for call in calls:
            call()
            assert c.status() == binding.SEKA_ERR_INVALID_ARG
            binding.seka_reset_status(c.ws)
