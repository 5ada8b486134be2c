"""Edges of the paged calls: NaN among the queries of the accumulated weights and the exponential of every column, more than 2^31 steps, host
threads side by side, more sequences than threads.  Tolerances are those of test_gpu_paged.py where nothing else is said."""
import ctypes
import math
import sys
import threading

import pytest
import torch

from paper_2603_01281_b200 import binding

import paged_ref as R
from test_gpu_paged import attend, check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    binding.load()


@pytest.mark.parametrize("where", ["query", "lse"])
@pytest.mark.parametrize("n,G", [(64, 4), (8, 4), (36, 7), (4, 4), (2, 4)])
def test_a_nan_query_reaches_the_weights_of_the_keys_it_sees(n, G, where):
    # sequence i has one bad row, in another column of its tile of rows each: the keys that its token sees get NaN, all others
    # what they would have had (64, 36 and 8 new tokens: tiles; 4 and 2: few rows)
    B, L, Hkv, d = 32, 520, 2, 64
    c = R.Cache([L] * B, [n] * B, G * Hkv, Hkv, d, 64, seed=40)
    _, lse, _, _ = R.attention(c)
    lse = lse.float()
    ref, err = R.mass(c, lse)
    want = torch.zeros((B, Hkv, c.cap), dtype=torch.bool, device="cuda")
    for b in range(B):
        row = (b * 5 + (b // 8) * 32) % (n * G)
        t, h = row // G, b % Hkv
        at = (c.cu[b] + t, h * G + row % G)
        if where == "query":
            c.Q[at[0], at[1], b % d] = float("nan")
        lse[at] = float("nan")
        want[b, h, :L - n + t + 1] = True
    out = torch.zeros((B, Hkv, c.cap), device="cuda")
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, out, c.ws)
    assert c.status() == binding.SEKA_OK
    assert torch.equal(torch.isnan(out), want)
    inside = (torch.arange(c.cap, device="cuda") < L).expand_as(out) & ~want
    tol = d * 2.0 ** -23 * err + (2.0 ** -16 + (G * n + 2) * 2.0 ** -24) * ref + 1e-30
    # (a column's sum without its bad row's part: only other heads and unseen keys are compared, where the bad row adds nothing)
    assert ((out.double() - ref).abs() <= tol)[inside].all()


def test_the_exponential_of_every_column():
    # One query row of a tile counts (the others have an lse of +infinity: weight 0), another column in every sequence, and the scores
    # are known exactly: the weight of a key is 2^x of x in [-140, 60].  Special-function unit: 2^-22 of the value;
    # polynomial: 2.1e-7, below that.  Below 2^-126 both may be off by as much as 2^-126, and nothing is added for -infinity.
    B, old, d = 64, 2048, 64
    n = 128                                                      # one query head: a tile of 128 new tokens
    c = R.Cache([old + n] * B, [n] * B, 1, 1, d, 64, seed=41, scale=math.log(2.0))
    whole = torch.randint(-140, 61, (B, old), generator=c.g).float()
    part = torch.randint(0, 256, (B, old), generator=c.g).float() / 256
    c.Q.zero_(); c.Q[:, 0, 0] = 1.0; c.Q[:, 0, 1] = 1.0
    K = c.K.view(-1, d)
    for b in range(B):
        k = torch.zeros((old + n, d))
        k[:old, 0], k[:old, 1] = whole[b], part[b]
        K[c.rows(b).cuda()] = k.bfloat16().cuda()
    lse = torch.full((c.T, 1), float("inf"), device="cuda")
    for b in range(B):
        lse[c.cu[b] + (b if b < 32 else (7 * b) % 128), 0] = 0.0
    out = torch.full((B, 1, c.cap), float("nan"), device="cuda")
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, out, c.ws)
    assert c.status() == binding.SEKA_OK
    log2e, scale = torch.tensor(1.4426950408889634), torch.tensor(math.log(2.0), dtype=torch.float32)
    x = ((whole + part).double() * (scale * log2e).double()).float().double()          # one rounding, as in the multiply-add
    ref = torch.exp2(x)
    err = (out[:, 0, :old].cpu().double() - ref).abs()
    assert (err <= 2.0 ** -22 * ref + 2.0 ** -126).all(), float((err / ref)[ref > 2.0 ** -120].max())
    # no row that counts sees the chunk's last keys in sequences whose row is not the last one: their weights are exactly zero
    for b in range(B):
        t = b if b < 32 else (7 * b) % 128
        assert (out[b, 0, old + t + 1:old + n] == 0).all()
    # no row at all that counts
    lse.fill_(float("inf"))
    out.fill_(float("nan"))
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, out, c.ws)
    assert c.status() == binding.SEKA_OK and (out[:, 0, :old + n] == 0).all()


def test_more_than_2_31_steps_of_a_sequence():
    # 128 query heads on one KV head: 270336 new tokens over a cache of 2.3 million rows are 2.4e9 steps of attention (units of two tokens) and as
    # many of the weights.  The cache repeats eight pages, so that the sums over a token's keys are sums over 2048 rows and how often
    # it sees each.
    G, d, page, period = 128, 64, 256, 2048
    L, n = 9000 * page - 3, 270336
    cap, old = 9000 * page, L - n
    attn_steps = sum((old + 2 * u + 2 + 127) // 128 for u in range(n // 2))
    mass_steps = sum(n - max(0, 256 * u - old) for u in range(cap // 256))
    assert attn_steps > 1 << 31 and mass_steps > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(42)
    K, V = (torch.randn((8, page, 1, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    V += 1
    Q = torch.randn((n, G, d), generator=g, device="cuda", dtype=torch.bfloat16)
    table = (torch.arange(9000, dtype=torch.int32, device="cuda") % 8).view(1, -1).contiguous()
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    shape = binding.make_paged_shape(batch=1, max_new=n, total_new=n, n_q_heads=G, n_kv_heads=1, head_dim=d, page_size=page, n_pages=8,
                                     block_table=table, cache_lens=lens)
    ws = binding.new_paged_workspace(shape)
    O, lse = torch.full_like(Q, float("nan")), torch.full((n, G), float("nan"), device="cuda")
    binding.seka_paged_attention(shape, Q, K, V, O, lse, ws)
    assert binding.seka_poll_status(ws) == binding.SEKA_OK
    assert bool(torch.isfinite(lse).all()) and bool(torch.isfinite(O).all())
    k, v, at = K.view(period, d).double(), V.view(period, d).double(), torch.arange(period, device="cuda")
    t = torch.cat([torch.tensor([0, 1, 2, n - 2, n - 1]), torch.randint(0, n, (60,), generator=torch.Generator().manual_seed(1))]).cuda()
    often = ((old + t)[:, None] - at[None, :]).div(period, rounding_mode="floor").double() + 1            # rows j = at (mod 2048) up to old + t
    s = Q[t].double() @ k.T / math.sqrt(d)                                                               # [tokens, heads, 2048]
    ref_lse = torch.logsumexp(s + often.log()[:, None], 2)
    p = torch.exp(s - ref_lse[..., None]) * often[:, None]
    ref, A = p @ v, p @ v.abs()
    dq = (Q[t].double().abs() @ k.abs().T / math.sqrt(d)).amax(2)
    delta = d * 2.0 ** -23 * dq
    # Beside the bounds of the other sizes: a row's sum takes 18000 steps, off by at most 2^-24 of it each; its output 16 keys
    # at a time, 144000 additions inside the tensor core of at most 2^-23 of the sum of magnitudes each.
    steps = cap // 128
    assert ((lse[t].double() - ref_lse).abs() <= delta + 2.0 ** -17 + 2.0 ** -21 * ref_lse.abs() + steps * 2.0 ** -24).all()
    err = (O[t].double() - ref).abs()
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * delta[..., None] + 2.0 ** -16 + steps * 2.0 ** -24 + 8 * steps * 2.0 ** -23) * A
    assert (err <= tol).all(), float((err / tol).max())
    del O
    out = torch.full((1, 1, cap), float("nan"), device="cuda")
    binding.seka_attention_mass(shape, Q, K, lse, None, out, ws)
    assert binding.seka_poll_status(ws) == binding.SEKA_OK
    assert bool(torch.isfinite(out[0, 0, :L]).all())
    keys = torch.tensor([0, 1, 255, 256, 70000, old - 1, old, old + 1, old + 1000, old + n // 2, L - 5000, L - 2], device="cuda")
    ref = torch.zeros(len(keys), dtype=torch.float64, device="cuda")
    for t0 in range(0, n, 8192):
        w = torch.exp(Q[t0:t0 + 8192].double() @ k[keys % period].T / math.sqrt(d) - lse[t0:t0 + 8192].double()[..., None]).sum(1)
        ref += w.masked_fill(keys[None, :] > (old + torch.arange(t0, min(t0 + 8192, n), device="cuda"))[:, None], 0.0).sum(0)
    # eight sums side by side of up to 270336 x 128 / 8 terms of about the same size: off by 2^-24 of the sum each at the very most, which
    # would be a quarter; roundings of both signs leave the square root of that many, 2^-24 sqrt(4.3e6) = 1.2e-4, here with a factor of 32
    err = (out[0, 0, keys].double() - ref).abs()
    assert (err <= (delta.max() * 2 + 2.0 ** -16 + 32 * 1.3e-4) * ref).all(), float((err / ref).max())


def test_work_beyond_what_a_cta_counts_is_refused():
    # 20000 new tokens with 128 query heads over the longest cache: more than 2^30 steps a CTA; nothing is computed
    G, d, page, n = 128, 64, 256, 20000
    pages = 0x7fff0000 // page
    assert sum((0x7fff0000 - n + 2 * u + 2 + 127) // 128 for u in range(n // 2)) > 148 << 30
    K = torch.zeros((1, page, 1, d), dtype=torch.bfloat16, device="cuda")
    Q = torch.zeros((n, G, d), dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros((1, pages), dtype=torch.int32, device="cuda"), torch.tensor([0x7fff0000], dtype=torch.int32, device="cuda")
    shape = binding.make_paged_shape(batch=1, max_new=n, total_new=n, n_q_heads=G, n_kv_heads=1, head_dim=d, page_size=page, n_pages=1,
                                     block_table=table, cache_lens=lens)
    ws = binding.new_paged_workspace(shape)
    O, lse = torch.full_like(Q, 3.0), torch.full((n, G), 3.0, device="cuda")
    binding.seka_paged_attention(shape, Q, K, K, O, lse, ws)
    assert binding.seka_poll_status(ws) == binding.SEKA_ERR_UNSUPPORTED
    assert bool((O == 3.0).all()) and bool((lse == 3.0).all())
    # the same launch on a shorter cache
    binding.seka_reset_status(ws)
    lens.fill_(n)
    binding.seka_paged_attention(shape, Q, K, K, O, lse, ws)
    assert binding.seka_poll_status(ws) == binding.SEKA_OK
    want = torch.arange(1, n + 1, device="cuda").double().log()[:, None]
    assert bool((O == 0).all()) and bool(((lse.double() - want).abs() <= 2.0 ** -17 + 2.0 ** -21 * want).all())


def test_evictions_of_several_host_threads():
    # caches of very different lengths side by side: the selections ask for 200 KB of shared memory and for 34 KB
    def cache(lens, seed):
        c = R.Cache(lens, [0] * len(lens), 1, 1, 64, 256, seed=seed)
        c.m = torch.rand((c.B, 1, c.cap), generator=c.g).cuda()
        c.p = torch.arange(c.cap, dtype=torch.int32).expand(c.B, 1, -1).contiguous().cuda()
        c.mo, c.po, c.lo = torch.empty_like(c.m), torch.empty_like(c.p), torch.empty_like(c.lens_d)
        return c

    caches = [cache([290000], 43), cache([300, 20], 44), cache([280000], 45), cache([400], 46)]
    streams = [torch.cuda.Stream() for _ in caches]
    call, begin, seen = binding.load().seka_evict_cache, threading.Barrier(len(caches)), [set() for _ in caches]

    def cut(c, stream, statuses):
        torch.cuda.set_device(0)
        args = (ctypes.byref(c.shape), *(x.data_ptr() for x in (c.K, c.V, c.m, c.mo, c.p, c.po)), None, 0, c.lens_d.data_ptr(), 200, 10,
                c.lo.data_ptr(), c.ws.data_ptr(), c.ws.numel(), stream.cuda_stream)
        begin.wait(timeout=60)
        for _ in range(4000):
            statuses.add(call(*args))

    torch.cuda.synchronize()
    every = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=cut, args=a) for a in zip(caches, streams, seen)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(every)
    torch.cuda.synchronize()
    assert seen == [{binding.SEKA_OK}] * len(caches), seen
    for c in caches:
        assert c.status() == binding.SEKA_OK and c.lo.tolist() == [min(l, 200) for l in c.lens]
    for c in caches[1::2]:                      # (the long ones are compared elsewhere)
        kept = R.evict(c, c.m, c.p, None, c.lens_d, 200, 10)
        for b in range(c.B):
            assert c.po[b, 0, :min(c.lens[b], 200)].tolist() == kept[b][0]


@pytest.mark.parametrize("B,new,Hq,Hkv,d,page", [(330, (1, 1), 8, 2, 64, 16), (400, (1, 30), 8, 2, 64, 16), (790, (0, 150), 16, 1, 128, 32), (1200, (0, 3), 4, 1, 64, 16)])
def test_more_sequences_than_threads(B, new, Hq, Hkv, d, page):
    # the shares are found sequences by thread, a block's worth at a time: some batches that take several turns, up to eight units a sequence and
    # more, sequences without new tokens and without any token among them
    g = torch.Generator().manual_seed(47)
    n = torch.randint(new[0], new[1] + 1, (B,), generator=g).tolist()
    n[B // 2] = new[1]
    old = torch.randint(0, 90, (B,), generator=g).tolist()
    lens = [0 if i % 37 == 5 else a + b for i, (a, b) in enumerate(zip(n, old))]
    c = R.Cache(lens, n, Hq, Hkv, d, page, seed=48)
    O, lse = attend(c)
    check_attention(c, O, lse)
    ref, err = R.mass(c, lse)
    out = torch.full((B, Hkv, c.cap), -7.0, device="cuda")
    binding.seka_attention_mass(c.shape, c.Q, c.K, lse, None, out, c.ws)
    assert c.status() == binding.SEKA_OK
    inside = (torch.arange(c.cap, device="cuda")[None] < c.lens_d[:, None])[:, None].expand_as(out)
    tol = d * 2.0 ** -23 * err + (2.0 ** -16 + (c.G * max(n) + 2) * 2.0 ** -24) * ref + 1e-30
    assert (((out.double() - ref).abs() <= tol) | ~inside).all() and (out[~inside] == -7.0).all()
