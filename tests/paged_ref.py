"""Paged caches for the tests and plain implementations of the paged calls in 64 bits."""
import math

import torch

from paper_2603_01281_b200 import binding


class Cache:
    """A pool of pages with the sequences of a test in scattered pages; unused pages and rows behind a sequence hold NaN."""

    def __init__(self, lens, new, n_q_heads, n_kv_heads, head_dim, page, seed=0, dtype=torch.bfloat16, max_pages=None, packed=True,
                 device="cuda", n_pages=None, scale=0.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.Hq, self.Hkv, self.d, self.page = list(lens), list(new), n_q_heads, n_kv_heads, head_dim, page
        self.B, self.T, self.G = len(lens), sum(new), n_q_heads // n_kv_heads
        self.cu = [0]
        for n in new:
            self.cu.append(self.cu[-1] + n)
        pages = [(l + page - 1) // page for l in lens]
        self.max_pages = max_pages or max(pages + [1])
        self.cap = self.max_pages * page
        self.n_pages = n_pages or sum(pages) + 3
        lo = max(0, self.n_pages - sum(pages) - 3)               # a larger pool: its last pages
        order = torch.randperm(self.n_pages - lo, generator=g) + lo
        self.table = torch.full((self.B, self.max_pages), -1, dtype=torch.int32)
        at = 0
        for b in range(self.B):
            self.table[b, :pages[b]] = order[at:at + pages[b]].to(torch.int32)
            at += pages[b]
        shape = (self.n_pages, page, n_kv_heads, head_dim)
        self.K, self.V = torch.empty(shape, dtype=torch.bfloat16, device=device), torch.empty(shape, dtype=torch.bfloat16, device=device)
        self.K[lo:].fill_(float("nan")); self.V[lo:].fill_(float("nan"))
        for b in range(self.B):
            r = self.rows(b).to(device)
            for x in (self.K, self.V):
                x.view(-1, n_kv_heads, head_dim)[r] = torch.randn((len(r), n_kv_heads, head_dim), generator=g).to(torch.bfloat16).to(device)
        self.Q = torch.randn((self.T, n_q_heads, head_dim), generator=g).to(torch.bfloat16).to(device)
        self.g = g
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
        self.table_d, self.lens_d, self.cu_d = self.table.to(device), dev(self.lens), dev(self.cu)
        fixed = not packed
        assert not fixed or len(set(new)) <= 1
        self.shape = binding.make_paged_shape(batch=self.B, max_new=max(new + [0]), total_new=self.T, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads,
                                              head_dim=head_dim, page_size=page, n_pages=self.n_pages, block_table=self.table_d,
                                              cache_lens=self.lens_d, cu_new=None if fixed else self.cu_d, dtype=dtype, softmax_scale=scale)
        self.scale = scale or 1.0 / math.sqrt(head_dim)
        self.ws = binding.new_paged_workspace(self.shape)

    def rows(self, b, n=None):
        j = torch.arange(self.lens[b] if n is None else n)
        return self.table[b, j // self.page].long() * self.page + j % self.page

    def cached(self, x, b):
        return x.view(-1, self.Hkv, self.d)[self.rows(b).to(x.device)].double()

    def status(self):
        return binding.seka_poll_status(self.ws)


def attention(c):
    """O [T, Hq, d], lse [T, Hq], and two sums that the tolerances need: sum_j p |v| [T, Hq, d] and the largest sum |q_i k_i| scale of a
    row over the keys that it sees [T, Hq]."""
    dev = c.Q.device
    O = torch.zeros((c.T, c.Hq, c.d), dtype=torch.float64, device=dev)
    A, lse, dq = torch.zeros_like(O), torch.full((c.T, c.Hq), -math.inf, dtype=torch.float64, device=dev), torch.zeros((c.T, c.Hq), dtype=torch.float64, device=dev)
    for b in range(c.B):
        k, v, old = c.cached(c.K, b), c.cached(c.V, b), c.lens[b] - c.new[b]
        for i0 in range(0, c.new[b], 256):
            i = torch.arange(i0, min(i0 + 256, c.new[b]), device=dev)
            seen = torch.arange(c.lens[b], device=dev)[None, :] <= (old + i)[:, None]
            some = seen.any(1)
            t = c.cu[b] + i[some]
            if len(t) == 0:
                continue
            for hq in range(c.Hq):
                q, h = c.Q[t, hq].double(), hq // c.G
                s = (q @ k[:, h].T * c.scale).masked_fill(~seen[some], -math.inf)
                lse[t, hq] = torch.logsumexp(s, 1)
                p = torch.softmax(s, 1)
                O[t, hq], A[t, hq] = p @ v[:, h], p @ v[:, h].abs()
                dq[t, hq] = (q.abs() @ k[:, h].abs().T * c.scale).masked_fill(~seen[some], 0.0).amax(1)
    return O, lse, A, dq


def mass(c, lse, mass_in=None):
    """[B, Hkv, cap] (rows behind a sequence: 0), and the same sums weighted by sum |q_i k_i| scale (for the tolerance)."""
    dev = c.Q.device
    out, err = (torch.zeros((c.B, c.Hkv, c.cap), dtype=torch.float64, device=dev) for _ in range(2))
    for b in range(c.B):
        k, n, l = c.cached(c.K, b), c.new[b], c.lens[b]
        seen = torch.arange(l, device=dev)[None, :] <= (l - n + torch.arange(n, device=dev))[:, None]
        for hq in range(c.Hq):
            q, h = c.Q[c.cu[b]:c.cu[b + 1], hq].double(), hq // c.G
            w = torch.exp(q @ k[:, h].T * c.scale - lse[c.cu[b]:c.cu[b + 1], hq].double()[:, None]).masked_fill(~seen, 0.0)
            out[b, h, :l] += w.sum(0)
            err[b, h, :l] += (w * (q.abs() @ k[:, h].abs().T * c.scale)).sum(0)
        if mass_in is not None and l > n:
            out[b, :, :l - n] += mass_in[b, :, :l - n].double()
    return out, err


def rotate(x, pos, turns, layout, f=1.0):
    """The rotated heads in 64 bits and |x| + |partner| of every element (0 where it is not rotated)."""
    x = x.double().clone()
    r = 2 * len(turns)
    a = 2 * math.pi * torch.remainder(pos.double()[:, None] * turns.double(), 1.0)
    cos, sin = a.cos()[:, None] * f, a.sin()[:, None] * f
    i = torch.arange(r // 2, device=x.device)
    i0, i1 = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    size = torch.zeros_like(x)
    u, w = x[..., i0].clone(), x[..., i1].clone()
    size[..., i0] = size[..., i1] = (u.abs() + w.abs()) * f
    x[..., i0], x[..., i1] = u * cos - w * sin, w * cos + u * sin
    return x, size


def evict(c, mass_in, pos_in, protect, next_pos, keep, recent):
    """Source row of every row below min(L, keep), [B][Hkv], by sorting plain Python tuples."""
    out = []
    for b in range(c.B):
        l, per = c.lens[b], []
        for h in range(c.Hkv):
            if l <= keep:
                per.append(list(range(l)))
                continue
            m, x = mass_in[b, h, :l].tolist(), pos_in[b, h, :l].tolist()

            def rank(j):
                inside = protect is not None and 0 <= x[j] < protect.shape[1]
                k = 2 if x[j] >= int(next_pos[b]) - recent else 1 if inside and int(protect[b, x[j]]) else 0
                return (-k, 1 if m[j] != m[j] else 0, 0.0 if m[j] != m[j] else -m[j], j)

            kept = set(sorted(range(l), key=rank)[:keep])
            late = iter(j for j in range(keep, l) if j in kept)
            per.append([j if j in kept else next(late) for j in range(keep)])
        out.append(per)
    return out
