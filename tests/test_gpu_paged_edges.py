"""Edges of the paged calls: NaN among the queries of the accumulated weights and the exponential of every column."""
import math

import pytest
import torch

from paper_2603_01281_b200 import binding

import paged_ref as R

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
