"""Calls of several host threads side by side whose launches ask for different amounts of shared memory of the same kernel: every call
succeeds and gives the bits that it gives alone."""
import ctypes
import sys
import threading

import pytest
import torch

from paper_2603_01281_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    binding.load()


class Prompt:
    """A small prompt and raw arguments of the calls on it (ranks and experts decide the shared memory)."""

    def __init__(self, seed, d, rank, experts, tokens, kv=2, steered=True, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")        # noqa: E731
        self.shp = binding.make_shape(batch=1, max_seqlen=tokens, n_q_heads=2 * kv, n_kv_heads=kv, head_dim=d, rank=rank, n_experts=experts, dtype=dtype)
        self.Q, self.K, self.V = rnd(tokens, 2 * kv, d).to(dtype), rnd(tokens, kv, d).to(dtype), rnd(tokens, kv, d).to(dtype)
        self.U = torch.linalg.qr(rnd(experts, kv, d, d))[0][..., :rank].contiguous() if experts <= 8 else rnd(experts, kv, d, rank) / 32
        self.sigma = rnd(experts, kv, rank).abs() + 0.5
        self.mask = (torch.rand(tokens, generator=g, device="cuda") < 0.3).to(torch.uint8) if steered else torch.zeros(tokens, dtype=torch.uint8, device="cuda")
        self.gain, self.steered = torch.full((1,), 0.5, device="cuda"), steered
        self.alpha = torch.zeros((1, kv, experts), device="cuda")
        self.given = torch.full((1, kv, experts), 0.25, device="cuda")
        self.O, self.K2 = torch.zeros_like(self.Q), torch.zeros_like(self.K)
        self.ws = binding.new_workspace(self.shp)
        self.stream = torch.cuda.Stream()
        torch.cuda.synchronize()

    def call(self, what):
        lib, st, p = binding.load(), self.stream.cuda_stream, lambda t: t.data_ptr()            # noqa: E731
        shp, ws = ctypes.byref(self.shp), (self.ws.data_ptr(), self.ws.numel())
        if what == "forward":
            steer = (p(self.mask), p(self.U), p(self.given), p(self.gain), None) if self.steered else (None,) * 5
            return lib.seka_attention_fwd, (shp, p(self.Q), p(self.K), p(self.V), p(self.O), None, *steer, *ws, st)
        if what == "routed":
            return lib.seka_attention_fwd_routed, (shp, p(self.Q), p(self.K), p(self.V), p(self.O), None, p(self.mask), p(self.U), p(self.sigma), 0,
                                                   p(self.alpha), p(self.gain), None, *ws, st)
        if what == "edit":
            return lib.seka_edit_keys, (shp, p(self.K), p(self.K2), p(self.mask), p(self.U), p(self.given), p(self.gain), None, *ws, st)
        return lib.adaseka_route, (shp, p(self.Q), p(self.U), p(self.sigma), 0, p(self.alpha), st)

    def results(self):
        return [x.clone() for x in (self.O, self.K2, self.alpha)]


# what is called; head_dim, rank, experts, tokens, steered of each thread
CASES = [
    ("forward", [(128, 16, 1, 300, True), (128, 16, 1, 300, False), (128, 64, 2, 300, True), (128, 8, 1, 200, False)]),
    ("forward", [(64, 16, 1, 300, True), (64, 16, 1, 300, False), (64, 64, 2, 300, True), (64, 8, 1, 200, False)]),
    ("routed", [(64, 64, 2, 300, True), (64, 8, 2, 300, True), (64, 32, 4, 300, True), (64, 16, 1, 200, True)]),
    ("routed", [(128, 128, 8, 300, True), (128, 8, 2, 300, True), (128, 16, 200, 300, True), (128, 16, 1, 200, True)]),
    ("edit", [(64, 64, 2, 700, True), (64, 16, 1, 700, True), (64, 64, 2, 300, True), (64, 8, 1, 300, True)]),
    ("route", [(128, 1, 4096, 64, True), (128, 1, 3500, 64, True), (128, 1, 4000, 64, True), (128, 1, 3700, 64, True)]),
]


@pytest.mark.parametrize("what,prompts", CASES)
def test_calls_of_several_host_threads(what, prompts):
    ps = [Prompt(60 + i, *a[:4], steered=a[4]) for i, a in enumerate(prompts)]
    alone = []
    for p in ps:
        f, args = p.call(what)
        assert f(*args) == binding.SEKA_OK
        torch.cuda.synchronize()
        alone.append(p.results())
    begin, seen = threading.Barrier(len(ps)), [set() for _ in ps]

    def work(p, statuses):
        torch.cuda.set_device(0)
        f, args = p.call(what)
        begin.wait(timeout=60)
        for _ in range(3000):
            statuses.add(f(*args))

    every = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=work, args=a) for a in zip(ps, seen)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(every)
    torch.cuda.synchronize()
    assert seen == [{binding.SEKA_OK}] * len(ps), seen
    for p, want in zip(ps, alone):
        assert binding.seka_poll_status(p.ws) == binding.SEKA_OK
        assert all(torch.equal(a, b) for a, b in zip(p.results(), want))
