"""Measured cases of the paged cache: what a server does that keeps the steered prompts' keys and values in pages.

Four kinds of pass, each one call of the library:

  append   rotary positions on the queries and keys of new tokens; keys and values go to their pages (`seka_rope_append`)
  attend   attention of the new tokens over the paged cache, a single token or a chunk per sequence (`seka_paged_attention`)
  mass     the attention weight that the cached tokens receive from the new ones, accumulated (`seka_attention_mass`)
  evict    the cache cut to its heaviest, recent and highlighted tokens (`seka_evict_cache`)

Sizes are those of this repository's configurations and decode benchmark (32 query heads on 8 of 128, 28 on 4 of 128, 16 on 16 of
64), with page sizes from 16 to 128.  With `own` false every pass is computed by elementary torch operations.
"""
import math

import torch

own = False

PAD = 2                 # pages of the pool that no sequence owns


# ------------------------------------------------------------------------------------------------ cases
def _case(kind, **kw):
    c = dict(kind=kind, batch=1, new_min=1, new_max=1, len_min=4096, len_max=4096, q_heads=32, kv_heads=8, head_dim=128, page=64)
    c.update(kw)
    return c


def _append(**kw):
    return _case("append", **{**dict(dtype="bf16", rot_dim=128, layout="half", base=500000.0, scaling="plain", scale=1.0, far=0), **kw})


def _attend(**kw):
    return _case("attend", **kw)


def _mass(**kw):
    return _case("mass", **kw)


def _evict(**kw):
    return _case("evict", **{**dict(keep=1024, recent=64, highlight=0.1), **kw})


def listed():
    return [
        # one generation step of a full batch: a token per sequence is rotated and cached; launch latency counts
        _append(name="append_decode_batch", batch=64, len_min=1024, len_max=4096),
        # a batch of long-context prompts: rotation scaled by wavelength, positions far beyond the trained range
        _append(name="append_prompts_scaled", batch=4, new_min=4096, new_max=4096, scaling="wavelength", scale=8.0, far=120000),
        # a small model in single precision: ragged chunks, half of each head rotated, neighbours paired, small pages
        _append(name="append_ragged_fp32", batch=64, new_min=1, new_max=512, len_min=512, len_max=2048, q_heads=16, kv_heads=16, head_dim=64,
                page=16, dtype="f32", rot_dim=32, layout="interleaved", base=10000.0, scaling="linear", scale=4.0),
        # one user, one generated token, a short conversation: the smallest call
        _attend(name="attend_one_user", len_min=777, len_max=777, page=16),
        # a generation step of a full batch of ragged contexts: the cache is read once
        _attend(name="attend_decode_batch", batch=64, len_min=1024, len_max=4096),
        # a chunk of a long document: the last 2048 of 32768 tokens are new, odd group of query heads
        _attend(name="attend_chunk_long", new_min=2048, new_max=2048, len_min=32768, len_max=32768, q_heads=28, kv_heads=4, page=128),
        # a mixed batch of a small model: some sequences decode, others bring a chunk
        _attend(name="attend_mixed_batch", batch=64, new_min=1, new_max=512, len_min=512, len_max=2048, q_heads=16, kv_heads=16, head_dim=64,
                page=32),
        # weights of a generation step over ragged contexts
        _mass(name="mass_decode_batch", batch=64, len_min=1024, len_max=4096),
        # weights of a prompt chunk over its context, pages smaller than a tile
        _mass(name="mass_chunk", batch=2, new_min=1024, new_max=1024, len_min=6000, len_max=8192, page=16),
        # one user's cache cut back after a prompt
        _evict(name="evict_one_user", len_min=1500, len_max=1500, keep=1024, page=16),
        # a full batch cut to half of its longest context
        _evict(name="evict_batch", batch=64, len_min=1024, len_max=4096, keep=2048, recent=256),
        # one long context cut to a quarter, most of its rows move
        _evict(name="evict_long", len_min=65536, len_max=65536, keep=16384, recent=1024, page=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads = rng.choice([(32, 8, 128), (28, 4, 128), (16, 16, 64), (8, 2, 128), (24, 8, 64), (9, 3, 64), (16, 1, 128)])
    c = dict(q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], page=rng.choice([16, 32, 64, 128, 256]))
    kind = rng.choice(["append", "attend", "attend", "mass", "evict"])
    if kind == "append":
        c["batch"] = _log_int(rng, 1, 64)
        c["new_max"] = _log_int(rng, 1, max(1, 16384 // c["batch"]))
        c["new_min"] = rng.randint(1, c["new_max"])
        c["len_min"] = c["new_max"]
        c["len_max"] = c["new_max"] + rng.randint(0, 1000)
        c["rot_dim"] = 2 * rng.randint(1, c["head_dim"] // 2)
        c["layout"] = rng.choice(["half", "interleaved"])
        c["base"] = rng.choice([10000.0, 500000.0])
        c["scaling"] = rng.choice(["plain", "linear", "base", "wavelength"]) if c["rot_dim"] > 2 else "plain"
        c["scale"] = rng.choice([2.0, 4.0, 8.0])
        c["far"] = _log_int(rng, 1, 1000000)
        c["dtype"] = rng.choice(["bf16", "f32"])
        return _append(**c)
    if kind == "evict":
        c["len_max"] = _log_int(rng, 16, 65536)
        c["batch"] = _log_int(rng, 1, max(1, min(64, 262144 // c["len_max"])))
        c["len_min"] = rng.randint(1, c["len_max"])
        c["keep"] = rng.randint(1, c["len_max"])
        c["recent"] = _log_int(rng, 1, c["keep"])
        c["highlight"] = rng.choice([0.0, 0.05, 0.15, 0.7])
        return _evict(**c)
    c["batch"] = _log_int(rng, 1, 64)
    c["new_max"] = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 2048)])
    c["new_min"] = rng.randint(1, c["new_max"])
    # query-key pairs and cached tokens stay below those of the largest listed cases
    most = min(32768, 262144 // c["batch"], (2048 * 32768 * 28 // 4) // (c["batch"] * c["new_max"] * c["q_heads"]) + c["new_max"])
    c["len_max"] = _log_int(rng, c["new_max"], max(c["new_max"], most))
    c["len_min"] = rng.randint(c["new_max"], c["len_max"])
    return _attend(**c) if kind == "attend" else _mass(**c)


def _lengths(case):
    """New and cached tokens of each sequence (plain numbers that follow from the case alone)."""
    B = case["batch"]
    def spread(lo, hi, step):
        return [hi if b == 0 else lo + (b * step) % (hi - lo + 1) for b in range(B)]
    new = spread(case["new_min"], case["new_max"], 97)
    lens = spread(case["len_min"], case["len_max"], 1237)
    return new, [max(n, l) for n, l in zip(new, lens)]


# ------------------------------------------------------------------------------------------------ inputs
def _turns(case):
    """Turns per position of each rotated pair, in 64 bits: base^(-2i/r) / 2 pi, scaled for long contexts."""
    r, base, s = case["rot_dim"], case["base"], case["scale"]
    i = torch.arange(r // 2, dtype=torch.float64)
    if case["scaling"] == "base":
        base = base * s ** (r / (r - 2))
    t = base ** (-2.0 * i / r) / (2.0 * math.pi)
    if case["scaling"] == "linear":
        t = t / s
    elif case["scaling"] == "wavelength":        # between 1 and 4 turns over 8192 positions: from fully scaled to not at all
        keep = ((8192.0 * t - 1.0) / 3.0).clamp(0.0, 1.0)
        t = t * keep + t / s * (1.0 - keep)
    return t


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, lens = _lengths(case)
    B, Hq, Hkv, d, ps = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    T = sum(new)
    pages = [(l + ps - 1) // ps for l in lens]
    max_pages, n_pages = max(pages), sum(pages) + PAD
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]

    def normal(*shape, dtype=torch.bfloat16):
        out = torch.empty(shape, dtype=dtype, device="cuda")
        for part in out.flatten().split(1 << 28):
            part.normal_(generator=g)
        return out

    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    st = dict(case=case, new=new, lens=lens, cu=cu, T=T, cap=max_pages * ps, n_pages=n_pages, table=table, lens_dev=i32(lens), cu_dev=i32(cu),
              K=normal(n_pages, ps, Hkv, d), V=normal(n_pages, ps, Hkv, d))
    if case["kind"] == "append":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        qkv = normal(T, (Hq + 2 * Hkv) * d, dtype=dt)            # the projection's output: queries, keys, values of a token side by side
        st.update(q=qkv[:, :Hq * d].view(T, Hq, d), k=qkv[:, Hq * d:(Hq + Hkv) * d].view(T, Hkv, d), v=qkv[:, (Hq + Hkv) * d:].view(T, Hkv, d),
                  turns=_turns(case).cuda(), Q=torch.empty((T, Hq, d), dtype=torch.bfloat16, device="cuda"),
                  pos_cache=torch.zeros((B, Hkv, st["cap"]), dtype=torch.int32, device="cuda"))
        far = torch.randint(0, case["far"] + 1, (B,), generator=g, device="cuda").tolist()
        st["pos"] = torch.cat([torch.arange(far[b] + lens[b] - new[b], far[b] + lens[b], device="cuda") for b in range(B)]).to(torch.int32)
    elif case["kind"] == "evict":
        mass = torch.empty((B, Hkv, st["cap"]), device="cuda").normal_(generator=g).mul_(1.5).exp_()
        mass[torch.rand(mass.shape, generator=g, device="cuda") < 0.05] = 0.0       # never attended: equal weights
        P = max(lens)
        st.update(mass=mass, mass_out=torch.zeros_like(mass), lens_out=torch.zeros_like(st["lens_dev"]), next_pos=st["lens_dev"].clone(),
                  pos=torch.arange(st["cap"], dtype=torch.int32, device="cuda").expand(B, Hkv, -1).contiguous(),
                  protect=(torch.rand((B, P), generator=g, device="cuda") < case["highlight"]).to(torch.uint8))
        st["pos_out"] = torch.zeros_like(st["pos"])
    else:
        st["Q"] = normal(T, Hq, d)
        if case["kind"] == "attend":
            st.update(O=torch.empty_like(st["Q"]), lse=torch.empty((T, Hq), device="cuda"))
        else:
            st["lse"] = _attention(st, torch.float32, with_output=False)[1]
            st["mass"] = torch.rand((B, Hkv, st["cap"]), generator=g, device="cuda")
            st["mass_out"] = torch.zeros_like(st["mass"])
    if own:
        _handle(st)
    return st


def _handle(st):
    """What a program of the framework keeps: the shape, the workspace and the table of the rotation."""
    if "shape" not in st:
        from paper_2603_01281_b200 import binding
        c = st["case"]
        st["binding"] = binding
        dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
        st["shape"] = binding.make_paged_shape(batch=c["batch"], max_new=max(st["new"]), total_new=st["T"], n_q_heads=c["q_heads"],
                                               n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], page_size=c["page"], n_pages=st["n_pages"],
                                               block_table=st["table"], cache_lens=st["lens_dev"], cu_new=st["cu_dev"], dtype=dt)
        st["ws"] = binding.new_paged_workspace(st["shape"])
        if c["kind"] == "append":
            turns = binding.seka_rope_turns(c["rot_dim"], base=c["base"], scaling=c["scaling"], scale=c["scale"], trained_len=8192,
                                            low_turns=1.0, high_turns=4.0).cuda()
            st["rope"] = binding.make_rope(turns, layout=c["layout"])
    return st["binding"]


# ------------------------------------------------------------------------------------------------ plain forms
def _rows(st, b, n):
    """Pool rows (page * page_size + offset) of the first n cached tokens of sequence b."""
    ps = st["case"]["page"]
    j = torch.arange(n, device="cuda")
    return st["table"][b, j // ps].long() * ps + j % ps


def _pool(st, name):
    t = st[name]
    return t.view(-1, *t.shape[2:])


def _visible(n, l):
    """[n, l]: cached token j is visible to new token i."""
    return torch.arange(l, device="cuda") <= (l - n + torch.arange(n, device="cuda"))[:, None]


def _attention(st, dt, with_output=True):
    c = st["case"]
    Hq, Hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    G = Hq // Hkv
    O = torch.zeros((st["T"], Hq, d), dtype=dt, device="cuda") if with_output else None
    lse = torch.empty((st["T"], Hq), dtype=dt, device="cuda")
    for b in range(c["batch"]):
        n, l, t0 = st["new"][b], st["lens"][b], st["cu"][b]
        rows = _rows(st, b, l)
        k, v = _pool(st, "K")[rows].to(dt), _pool(st, "V")[rows].to(dt)
        q = st["Q"][t0:t0 + n].to(dt)
        seen = _visible(n, l)
        for h in range(Hkv):
            s = torch.einsum("igd,jd->gij", q[:, h * G:(h + 1) * G], k[:, h]) / math.sqrt(d)
            s.masked_fill_(~seen, float("-inf"))
            top = s.amax(-1, keepdim=True)
            s.sub_(top).exp_()
            total = s.sum(-1, keepdim=True)
            lse[t0:t0 + n, h * G:(h + 1) * G] = (top + total.log())[..., 0].T
            if with_output:
                O[t0:t0 + n, h * G:(h + 1) * G] = (torch.matmul(s, v[:, h]) / total).permute(1, 0, 2)
    return O, lse


def _mass_sums(st, dt):
    """The weights that the cached tokens of each sequence receive: a list of [Hkv, l]."""
    c = st["case"]
    Hkv, d, G = c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"]
    out = []
    for b in range(c["batch"]):
        n, l, t0 = st["new"][b], st["lens"][b], st["cu"][b]
        k, q = _pool(st, "K")[_rows(st, b, l)].to(dt), st["Q"][t0:t0 + n].to(dt)
        seen = _visible(n, l)
        w = torch.empty((Hkv, l), dtype=dt, device="cuda")
        for h in range(Hkv):
            s = torch.einsum("igd,jd->gij", q[:, h * G:(h + 1) * G], k[:, h]) / math.sqrt(d)
            s.sub_(st["lse"][t0:t0 + n, h * G:(h + 1) * G].to(dt).T[..., None]).exp_()
            w[h] = s.masked_fill_(~seen, 0.0).sum((0, 1))
        out.append(w)
    return out


def _mass_plain(st):
    out = st["mass_out"]
    for b, w in enumerate(_mass_sums(st, torch.float32)):
        n, l = st["new"][b], st["lens"][b]
        w[:, :l - n] += st["mass"][b, :, :l - n]
        out[b, :, :l] = w
    return out


def _rotate(x, cos, sin, layout):
    """The first 2 * cos.shape[-1] elements of the heads of x [T, H, d], rotated; the others as they are."""
    r = 2 * cos.shape[-1]
    y, c, s = x.clone(), cos[:, None], sin[:, None]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    ya, yb = a * c - b * s, b * c + a * s
    if layout == "half":
        y[..., :r // 2], y[..., r // 2:r] = ya, yb
    else:
        y[..., 0:r:2], y[..., 1:r:2] = ya, yb
    return y


def _append_plain(st):
    c = st["case"]
    angle = st["pos"].double()[:, None] * st["turns"]
    angle = (angle - angle.round()) * (2.0 * math.pi)
    cos, sin = angle.cos().float(), angle.sin().float()
    st["Q"].copy_(_rotate(st["q"].float(), cos, sin, c["layout"]))
    k = _rotate(st["k"].float(), cos, sin, c["layout"]).bfloat16()
    v = st["v"].bfloat16()
    for b in range(c["batch"]):
        n, l, t0 = st["new"][b], st["lens"][b], st["cu"][b]
        rows = _rows(st, b, l)[l - n:]
        _pool(st, "K")[rows] = k[t0:t0 + n]
        _pool(st, "V")[rows] = v[t0:t0 + n]
        st["pos_cache"][b, :, l - n:l] = st["pos"][t0:t0 + n]
    return st["Q"], st["K"], st["V"], st["pos_cache"]


def _evict_plain(st):
    c = st["case"]
    keep = c["keep"]
    for b in range(c["batch"]):
        l = st["lens"][b]
        m = min(l, keep)
        mass, pos = st["mass"][b, :, :l], st["pos"][b, :, :l]
        if l > keep:
            klass = torch.where(pos >= st["next_pos"][b] - c["recent"], 2, (st["protect"][b][pos.long()] != 0).to(torch.int64))
            by_mass = mass.sort(dim=1, descending=True, stable=True).indices
            order = by_mass.gather(1, klass.gather(1, by_mass).sort(dim=1, descending=True, stable=True).indices)
            kept = torch.zeros_like(mass, dtype=torch.bool).scatter_(1, order[:, :keep], True)
            # the i-th freed row takes the i-th kept row from behind the cut
            back = (~kept[:, keep:]).to(torch.int8).sort(dim=1, stable=True).indices + keep
            turn = ((~kept[:, :keep]).cumsum(1) - 1).clamp(0, l - keep - 1)
            here = torch.arange(keep, device="cuda")
            src = torch.where(kept[:, :keep], here, back.gather(1, turn))
            rows = _rows(st, b, l)
            for name in ("K", "V"):
                pool = _pool(st, name)
                moved = pool[rows].gather(0, src.T[..., None].expand(-1, -1, c["head_dim"]))
                pool[rows[:keep]] = moved
            mass, pos = mass.gather(1, src), pos.gather(1, src)
        st["mass_out"][b, :, :m] = mass
        st["pos_out"][b, :, :m] = pos
    torch.clamp(st["lens_dev"], max=keep, out=st["lens_out"])
    return st["K"], st["V"], st["mass_out"], st["pos_out"], st["lens_out"]


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    c = st["case"]
    kind = c["kind"]
    if not own:
        if kind == "append":
            return _append_plain(st)
        if kind == "attend":
            O, lse = _attention(st, torch.float32)
            return O.bfloat16(), lse
        return _mass_plain(st) if kind == "mass" else _evict_plain(st)
    lib = _handle(st)
    if kind == "append":
        lib.seka_rope_append(st["shape"], st["rope"], st["q"], st["k"], st["v"], st["pos"], st["Q"], st["K"], st["V"], st["pos_cache"], st["ws"])
        return st["Q"], st["K"], st["V"], st["pos_cache"]
    if kind == "attend":
        lib.seka_paged_attention(st["shape"], st["Q"], st["K"], st["V"], st["O"], st["lse"], st["ws"])
        return st["O"], st["lse"]
    if kind == "mass":
        lib.seka_attention_mass(st["shape"], st["Q"], st["K"], st["lse"], st["mass"], st["mass_out"], st["ws"])
        return st["mass_out"]
    lib.seka_evict_cache(st["shape"], st["K"], st["V"], st["mass"], st["mass_out"], st["pos"], st["pos_out"], st["protect"], st["next_pos"],
                         c["keep"], c["recent"], st["lens_out"], st["ws"])
    return st["K"], st["V"], st["mass_out"], st["pos_out"], st["lens_out"]


def work(case):
    new, lens = _lengths(case)
    Hq, Hkv, d, T = case["q_heads"], case["kv_heads"], case["head_dim"], sum(new)
    pairs = sum(n * l - n * (n - 1) // 2 for n, l in zip(new, lens))
    if case["kind"] == "append":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": T * (Hq + 2 * Hkv) * d * (size + 2) + 4 * T * (1 + Hkv), "flops": 3 * T * (Hq + Hkv) * case["rot_dim"]}
    if case["kind"] == "attend":
        return {"bytes": 4 * sum(lens) * Hkv * d + T * Hq * (4 * d + 4), "flops": 4 * pairs * Hq * d}
    if case["kind"] == "mass":
        return {"bytes": sum(lens) * Hkv * (2 * d + 8) + T * Hq * (2 * d + 4), "flops": 2 * pairs * Hq * d}
    # weights and positions read once and written once; rows that move are read and written (as many as a random choice moves)
    keep = case["keep"]
    moved = sum(min(keep, l) * max(0, l - keep) // l for l in lens)
    return {"bytes": Hkv * (8 * sum(lens) + 8 * sum(min(l, keep) for l in lens) + 8 * d * moved), "flops": Hkv * sum(lens)}


# ------------------------------------------------------------------------------------------------ definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    ps, new, lens, cu = case["page"], st["new"], st["lens"], st["cu"]
    Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    G = Hq // Hkv
    table = st["table"].cpu()

    def cached(name, b, first=0):
        """Rows [first, l) of sequence b, page by page."""
        parts = [st[name][int(table[b, p])] for p in range((lens[b] + ps - 1) // ps)]
        return torch.cat(parts)[first:lens[b]]

    if kind in ("attend", "mass"):
        O = torch.zeros((st["T"], Hq, d), dtype=torch.float64, device="cuda")
        lse = torch.zeros((st["T"], Hq), dtype=torch.float64, device="cuda")
        out = torch.zeros((case["batch"], Hkv, st["cap"]), dtype=torch.float64, device="cuda")
        for b in range(case["batch"]):
            n, l = new[b], lens[b]
            k, v = cached("K", b).double(), cached("V", b).double()
            old = l - n
            future = torch.ones((n, l), dtype=torch.bool, device="cuda").triu(old + 1)
            for hq in range(Hq):
                z = st["Q"][cu[b]:cu[b + 1], hq].double() @ k[:, hq // G].T * d ** -0.5
                z[future] = -math.inf
                if kind == "attend":
                    lse[cu[b]:cu[b + 1], hq] = torch.logsumexp(z, 1)
                    O[cu[b]:cu[b + 1], hq] = torch.softmax(z, 1) @ v[:, hq // G]
                else:
                    out[b, hq // G, :l] += torch.exp(z - st["lse"][cu[b]:cu[b + 1], hq].double()[:, None]).sum(0)
            if kind == "mass":
                out[b, :, :old] += st["mass"][b, :, :old].double()
        return (O, lse) if kind == "attend" else out
    if kind == "append":
        phase = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                            2.0 * math.pi * torch.remainder(st["pos"].double()[:, None] * st["turns"], 1.0))

        def turned(x):
            x, r = x.double().clone(), case["rot_dim"]
            part = x[..., :r]
            pairs = part.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else part.unflatten(-1, (r // 2, 2))
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * phase[:, None])
            x[..., :r] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
            return x

        K, V, pos = st["K"].double(), st["V"].double(), st["pos_cache"].clone()
        k, v = turned(st["k"]), st["v"].double()
        for b in range(case["batch"]):
            at = [divmod(j, ps) for j in range(lens[b] - new[b], lens[b])]
            page, off = torch.tensor([int(table[b, p]) for p, _ in at]).cuda(), torch.tensor([o for _, o in at]).cuda()
            K[page, off], V[page, off] = k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]]
            pos[b, :, lens[b] - new[b]:lens[b]] = st["pos"][cu[b]:cu[b + 1]]
        return turned(st["q"]), K, V, pos
    return None             # whole numbers and rows that are moved as they are
