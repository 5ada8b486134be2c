"""Thin ctypes binding over ``libseka_b200.so`` (the C ABI declared in ``include/seka.h``).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
PyTorch supplies device memory and the current stream.  There is no fallback: if the
compiled library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libseka_b200.so")

SEKA_OK, SEKA_ERR_INVALID_ARG, SEKA_ERR_UNSUPPORTED, SEKA_ERR_WORKSPACE, SEKA_ERR_CUDA, SEKA_ERR_TIMEOUT = range(6)
SEKA_F32, SEKA_BF16 = 0, 1

EXPORTS = ["seka_workspace_bytes", "seka_edit_keys", "adaseka_route", "seka_attention_fwd",
           "seka_host_staging_bytes", "seka_attention_fwd_host", "seka_reset_status", "seka_poll_status",
           "seka_status_string", "seka_launch_count", "seka_edit_keys_static", "seka_decode_workspace_bytes",
           "seka_decode_attention", "seka_attention_fwd_routed", "seka_learn_workspace_bytes", "seka_learn_projections",
           "seka_paged_workspace_bytes", "seka_rope_turns", "seka_rope_append", "seka_paged_attention", "seka_attention_mass",
           "seka_evict_cache"]
SEKA_STATIC_MAX_TOKENS = 262144


class SekaShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_seqlen", ctypes.c_int32), ("total_tokens", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rank", ctypes.c_int32), ("n_experts", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("cu_seqlens", ctypes.c_void_p)]


class SekaLearnShape(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("n_slots", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("gamma", ctypes.c_float)]


class SekaPagedShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("total_new", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float), ("block_table", ctypes.c_void_p),
                ("cache_lens", ctypes.c_void_p), ("cu_new", ctypes.c_void_p)]


class SekaRope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("turns", ctypes.c_void_p)]


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "wavelength": 3}


class SekaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


_lib = None


def load() -> ctypes.CDLL:
    """Load the compiled CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("CUDA library %s is missing: run __graft_entry__.build() "
                               "(python -m paper_2603_01281_b200.build); there is no CPU fallback" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        vp, sp = ctypes.c_void_p, ctypes.POINTER(SekaShape)
        lib.seka_workspace_bytes.argtypes = [sp]; lib.seka_workspace_bytes.restype = ctypes.c_size_t
        lib.seka_host_staging_bytes.argtypes = [sp]; lib.seka_host_staging_bytes.restype = ctypes.c_size_t
        lib.seka_edit_keys.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lib.seka_edit_keys.restype = ctypes.c_int
        lib.seka_edit_keys_static.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.seka_edit_keys_static.restype = ctypes.c_int
        lib.adaseka_route.argtypes = [sp, vp, vp, vp, ctypes.c_int32, vp, vp]
        lib.adaseka_route.restype = ctypes.c_int
        lib.seka_attention_fwd.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lib.seka_attention_fwd.restype = ctypes.c_int
        lib.seka_attention_fwd_routed.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp, vp,
                                                  ctypes.c_size_t, vp]
        lib.seka_attention_fwd_routed.restype = ctypes.c_int
        lib.seka_attention_fwd_host.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t,
                                                vp, ctypes.c_size_t, vp]
        lib.seka_attention_fwd_host.restype = ctypes.c_int
        lib.seka_decode_workspace_bytes.argtypes = [sp]; lib.seka_decode_workspace_bytes.restype = ctypes.c_size_t
        lib.seka_decode_attention.argtypes = [sp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lib.seka_decode_attention.restype = ctypes.c_int
        lp = ctypes.POINTER(SekaLearnShape)
        lib.seka_learn_workspace_bytes.argtypes = [lp]; lib.seka_learn_workspace_bytes.restype = ctypes.c_size_t
        lib.seka_learn_projections.argtypes = [lp] + [vp] * 14 + [ctypes.c_size_t, vp]
        lib.seka_learn_projections.restype = ctypes.c_int
        pp, i32, i64, f64, sz = ctypes.POINTER(SekaPagedShape), ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
        lib.seka_paged_workspace_bytes.argtypes = [pp]; lib.seka_paged_workspace_bytes.restype = sz
        lib.seka_rope_turns.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp]; lib.seka_rope_turns.restype = ctypes.c_int
        lib.seka_rope_append.argtypes = [pp, ctypes.POINTER(SekaRope), vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.seka_rope_append.restype = ctypes.c_int
        lib.seka_paged_attention.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, vp]; lib.seka_paged_attention.restype = ctypes.c_int
        lib.seka_attention_mass.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, vp]; lib.seka_attention_mass.restype = ctypes.c_int
        lib.seka_evict_cache.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, sz, vp]
        lib.seka_evict_cache.restype = ctypes.c_int
        lib.seka_reset_status.argtypes = [vp, vp]; lib.seka_reset_status.restype = ctypes.c_int
        lib.seka_poll_status.argtypes = [vp, vp]; lib.seka_poll_status.restype = ctypes.c_int
        lib.seka_status_string.argtypes = [ctypes.c_int]; lib.seka_status_string.restype = ctypes.c_char_p
        lib.seka_launch_count.argtypes = []; lib.seka_launch_count.restype = ctypes.c_uint64
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().seka_status_string(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the library must be contiguous"
    return t.data_ptr()


def _stream() -> int:
    """The current stream of the current device, as torch.cuda.current_stream().cuda_stream gives it, without building the
    stream object (3.2 us of a call; the raw lookup takes 0.1)."""
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(status: int, where: str) -> None:
    if status != SEKA_OK:
        raise SekaError(status, where)


def make_shape(*, batch: int, max_seqlen: int, n_q_heads: int, n_kv_heads: int, head_dim: int, rank: int,
               n_experts: int = 1, dtype: torch.dtype = torch.bfloat16, total_tokens: int = 0,
               cu_seqlens: Optional[torch.Tensor] = None, softmax_scale: float = 0.0) -> SekaShape:
    """Fill the POD shape struct; ``cu_seqlens`` is a device int32 tensor [B+1] or None."""
    if cu_seqlens is not None:
        assert cu_seqlens.dtype == torch.int32 and cu_seqlens.is_cuda and cu_seqlens.is_contiguous()
    code = {torch.float32: SEKA_F32, torch.bfloat16: SEKA_BF16}[dtype]
    s = SekaShape(batch, max_seqlen, total_tokens, n_q_heads, n_kv_heads, head_dim, rank, n_experts, code,
                  softmax_scale, cu_seqlens.data_ptr() if cu_seqlens is not None else None)
    s._keepalive = cu_seqlens
    return s


def seka_workspace_bytes(shape: SekaShape) -> int:
    return int(load().seka_workspace_bytes(ctypes.byref(shape)))


def seka_host_staging_bytes(shape: SekaShape) -> int:
    return int(load().seka_host_staging_bytes(ctypes.byref(shape)))


def new_workspace(shape: SekaShape, device="cuda") -> torch.Tensor:
    """Allocate (with torch) and clear a workspace of the size the library asks for."""
    n = seka_workspace_bytes(shape)
    if n == 0:
        raise SekaError(SEKA_ERR_INVALID_ARG, "seka_workspace_bytes")
    ws = torch.zeros(n, dtype=torch.uint8, device=device)
    return ws


def seka_edit_keys(shape: SekaShape, K_in, K_out, mask, U, alpha, gain, head_enable, workspace) -> None:
    _check(load().seka_edit_keys(ctypes.byref(shape), _ptr(K_in), _ptr(K_out), _ptr(mask), _ptr(U), _ptr(alpha),
                                 _ptr(gain), _ptr(head_enable), _ptr(workspace),
                                 workspace.numel() if workspace is not None else 0, _stream()), "seka_edit_keys")


def seka_edit_keys_static(shape: SekaShape, K_in, K_out, mask, U, alpha, gain, head_enable) -> None:
    """seka_edit_keys for callers that cannot allocate: one launch without scratch (at most SEKA_STATIC_MAX_TOKENS tokens)."""
    _check(load().seka_edit_keys_static(ctypes.byref(shape), _ptr(K_in), _ptr(K_out), _ptr(mask), _ptr(U),
                                        _ptr(alpha), _ptr(gain), _ptr(head_enable), _stream()),
           "seka_edit_keys_static")


def adaseka_route(shape: SekaShape, Q, U, sigma, k_route: int, alpha_out) -> None:
    _check(load().adaseka_route(ctypes.byref(shape), _ptr(Q), _ptr(U), _ptr(sigma), int(k_route), _ptr(alpha_out),
                                _stream()), "adaseka_route")


def seka_attention_fwd(shape: SekaShape, Q, K, V, O, lse, mask, U, alpha, gain, head_enable, workspace) -> None:
    _check(load().seka_attention_fwd(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(lse), _ptr(mask),
                                     _ptr(U), _ptr(alpha), _ptr(gain), _ptr(head_enable), _ptr(workspace),
                                     workspace.numel() if workspace is not None else 0, _stream()),
           "seka_attention_fwd")


def seka_attention_fwd_routed(shape: SekaShape, Q, K, V, O, lse, mask, U, sigma, k_route: int, alpha_out, gain,
                              head_enable, workspace) -> None:
    """AdaSEKA in one call: the routing of Eq. 6 runs inside the operand-preparation launch."""
    _check(load().seka_attention_fwd_routed(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(lse),
                                            _ptr(mask), _ptr(U), _ptr(sigma), int(k_route), _ptr(alpha_out), _ptr(gain),
                                            _ptr(head_enable), _ptr(workspace),
                                            workspace.numel() if workspace is not None else 0, _stream()),
           "seka_attention_fwd_routed")


def seka_attention_fwd_host(shape: SekaShape, h_Q, h_K, h_V, h_O, h_lse, h_mask, U, alpha, gain, head_enable,
                            staging, workspace) -> None:
    """Host-buffer variant: h_* are CPU tensors (pinned for asynchronous copies)."""
    for t in (h_Q, h_K, h_V, h_O, h_lse, h_mask):
        assert t is None or not t.is_cuda
    _check(load().seka_attention_fwd_host(ctypes.byref(shape), _ptr(h_Q), _ptr(h_K), _ptr(h_V), _ptr(h_O),
                                          _ptr(h_lse), _ptr(h_mask), _ptr(U), _ptr(alpha), _ptr(gain),
                                          _ptr(head_enable), _ptr(staging), staging.numel(), _ptr(workspace),
                                          workspace.numel(), _stream()), "seka_attention_fwd_host")


def seka_decode_workspace_bytes(shape: SekaShape) -> int:
    return int(load().seka_decode_workspace_bytes(ctypes.byref(shape)))


def seka_decode_attention(shape: SekaShape, Q, K, V, O, lse, workspace) -> None:
    """One decode step over the (already edited) cache: Q and O are [B, Hq, d], K and V the packed caches."""
    _check(load().seka_decode_attention(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(lse),
                                        _ptr(workspace), workspace.numel() if workspace is not None else 0,
                                        _stream()), "seka_decode_attention")


def seka_learn_projections(h, h_pos, h_neg, answer_tokens, gamma: float) -> dict:
    """Offline spectral learning for every slot of bf16 embeddings [n, slots, d]; allocates the outputs with torch
    and returns them in a dict (omega_pos, omega_neg, U_pos, U_neg, S_pos, S_neg, k_pos, k_neg, D)."""
    n, slots, d = h.shape
    assert h.dtype == torch.bfloat16 and h_pos.shape == h.shape and h_neg.shape == h.shape
    shp = SekaLearnShape(n, slots, d, gamma)
    nbytes = int(load().seka_learn_workspace_bytes(ctypes.byref(shp)))
    if nbytes == 0:
        raise SekaError(SEKA_ERR_UNSUPPORTED, "seka_learn_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=h.device)
    ws[:256].zero_()                        # the status block; the launches write the rest before they read it
    f32 = dict(dtype=torch.float32, device=h.device)
    out = {"omega_pos": torch.empty((slots, d, d), **f32), "omega_neg": torch.empty((slots, d, d), **f32),
           "U_pos": torch.empty((slots, d, d), **f32), "U_neg": torch.empty((slots, d, d), **f32),
           "S_pos": torch.empty((slots, d), **f32), "S_neg": torch.empty((slots, d), **f32),
           "k_pos": torch.empty(slots, dtype=torch.int32, device=h.device),
           "k_neg": torch.empty(slots, dtype=torch.int32, device=h.device), "D": torch.empty(slots, **f32)}
    _check(load().seka_learn_projections(ctypes.byref(shp), _ptr(h), _ptr(h_pos), _ptr(h_neg), _ptr(answer_tokens),
                                         _ptr(out["omega_pos"]), _ptr(out["omega_neg"]), _ptr(out["U_pos"]),
                                         _ptr(out["U_neg"]), _ptr(out["S_pos"]), _ptr(out["S_neg"]), _ptr(out["k_pos"]),
                                         _ptr(out["k_neg"]), _ptr(out["D"]), _ptr(ws), ws.numel(), _stream()),
           "seka_learn_projections")
    st = seka_poll_status(ws)
    if st != SEKA_OK:
        raise SekaError(st, "seka_learn_projections (device status)")
    out["workspace"] = ws
    return out


def seka_reset_status(workspace) -> None:
    _check(load().seka_reset_status(_ptr(workspace), _stream()), "seka_reset_status")


def seka_poll_status(workspace) -> int:
    return int(load().seka_poll_status(_ptr(workspace), _stream()))


def seka_launch_count() -> int:
    return int(load().seka_launch_count())


# ---------------------------------------------------------------- paged cache
def _fits(name: str, t: Optional[torch.Tensor], dtype, shape, device, packed: bool = True) -> None:
    """A tensor of a paged call: type, device, sizes (None: any) and, unless ``packed`` is false, contiguous."""
    if t is None or (t.dtype is dtype and t.shape == shape and t.device == device and (not packed or t.is_contiguous())):
        return
    if t.dtype != dtype or t.device != device or t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError("%s must be %s %s on %s, not %s %s on %s" % (name, dtype, list(shape), device, t.dtype, list(t.shape), t.device))
    if packed and not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _scratch(t: torch.Tensor, device):
    """The workspace of a paged call and its bytes."""
    if t is None or t.dtype is not torch.uint8 or t.device != device or not t.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on %s (new_paged_workspace)" % device)
    return t.data_ptr(), t.numel()


def make_paged_shape(*, batch: int, max_new: int, total_new: int, n_q_heads: int, n_kv_heads: int, head_dim: int, page_size: int,
                     n_pages: int, block_table: torch.Tensor, cache_lens: torch.Tensor, cu_new: Optional[torch.Tensor] = None,
                     dtype: torch.dtype = torch.bfloat16, softmax_scale: float = 0.0) -> SekaPagedShape:
    """Fill the struct of the paged calls.  The tables are device int32 tensors: ``block_table`` [B, max_pages], ``cache_lens`` [B]
    (new tokens included), ``cu_new`` [B+1] or None (every sequence has ``max_new`` new tokens).  They may change between calls;
    the shape keeps them alive."""
    dev = cache_lens.device
    if dev.type != "cuda":
        raise ValueError("cache_lens must be a device tensor")
    _fits("cache_lens", cache_lens, torch.int32, (batch,), dev)
    _fits("block_table", block_table, torch.int32, (batch, None), dev)
    _fits("cu_new", cu_new, torch.int32, (batch + 1,), dev)
    code = {torch.float32: SEKA_F32, torch.bfloat16: SEKA_BF16}[dtype]
    s = SekaPagedShape(batch, total_new, max_new, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, block_table.shape[1], code,
                       softmax_scale, block_table.data_ptr(), cache_lens.data_ptr(), cu_new.data_ptr() if cu_new is not None else None)
    s._keepalive = (block_table, cache_lens, cu_new)
    s._dtype, s._device = dtype, dev
    s._pages = (n_pages, page_size, n_kv_heads, head_dim)
    s._state = (batch, n_kv_heads, block_table.shape[1] * page_size)
    s._q = (total_new, n_q_heads, head_dim)
    return s


def seka_paged_workspace_bytes(shape: SekaPagedShape) -> int:
    return int(load().seka_paged_workspace_bytes(ctypes.byref(shape)))


def new_paged_workspace(shape: SekaPagedShape) -> torch.Tensor:
    """A workspace of the paged calls on the shape's device, its status block cleared."""
    n = seka_paged_workspace_bytes(shape)
    if n == 0:
        raise SekaError(SEKA_ERR_UNSUPPORTED, "seka_paged_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=shape._device)
    ws[:256].zero_()
    return ws


def _on_device(shape: SekaPagedShape) -> int:
    """The current stream; the shape's device must be the current one (the launches go to it)."""
    st = _stream()
    if shape._device.index is not None and shape._device.index != torch._C._cuda_getDevice():
        raise ValueError("the tensors are on %s, which is not the current device" % shape._device)
    return st


def seka_rope_turns(rot_dim: int, base: float = 10000.0, scaling: str = "plain", scale: float = 1.0, trained_len: float = 8192.0,
                    low_turns: float = 1.0, high_turns: float = 4.0) -> torch.Tensor:
    """Turns per position of the rotated pairs, a CPU fp64 tensor [rot_dim / 2]; move it to the device once."""
    out = torch.empty(max(rot_dim // 2, 0), dtype=torch.float64)
    _check(load().seka_rope_turns(rot_dim, base, ROPE_SCALINGS[scaling], scale, trained_len, low_turns, high_turns, out.data_ptr()),
           "seka_rope_turns")
    return out


def make_rope(turns: torch.Tensor, layout: str = "half", magnitude: float = 1.0) -> SekaRope:
    """Rotation of the first ``2 * len(turns)`` elements of each head; ``turns`` is a device fp64 tensor."""
    if turns.dtype != torch.float64 or turns.dim() != 1 or not turns.is_cuda or not turns.is_contiguous():
        raise ValueError("turns must be a contiguous 1-D device fp64 tensor")
    r = SekaRope(2 * turns.numel(), ROPE_LAYOUTS[layout], magnitude, turns.data_ptr())
    r._keepalive = turns
    return r


def seka_rope_append(shape: SekaPagedShape, rope: Optional[SekaRope], Q, K, V, positions, Q_out, K_pages, V_pages, pos_cache,
                     workspace) -> None:
    """Rotate the new queries and keys, cache keys and values.  Q, K, V may be slices of one projection (heads contiguous)."""
    st, dev, (T, Hq, d), Hkv = _on_device(shape), shape._device, shape._q, shape.n_kv_heads
    strides = []
    for name, x, H in (("Q", Q, Hq), ("K", K, Hkv), ("V", V, Hkv)):
        _fits(name, x, shape._dtype, (T, H, d), dev, packed=False)
        token, head, one = x.stride()
        if T > 0 and (one != 1 or (H > 1 and head != d) or (T > 1 and token < H * d)):
            raise ValueError("%s: the heads of a token must be contiguous, its tokens apart" % name)
        strides.append(token if T > 1 else 0)
    if rope is not None and rope._keepalive.device != dev:
        raise ValueError("the turns are on %s, not on %s" % (rope._keepalive.device, dev))
    _fits("positions", positions, torch.int32, (T,), dev)
    _fits("Q_out", Q_out, torch.bfloat16, (T, Hq, d), dev)
    _fits("K_pages", K_pages, torch.bfloat16, shape._pages, dev)
    _fits("V_pages", V_pages, torch.bfloat16, shape._pages, dev)
    _fits("pos_cache", pos_cache, torch.int32, shape._state, dev)
    _check(load().seka_rope_append(ctypes.byref(shape), ctypes.byref(rope) if rope is not None else None, Q.data_ptr(), strides[0],
                                   K.data_ptr(), strides[1], V.data_ptr(), strides[2], _ptr(positions), _ptr(Q_out), _ptr(K_pages),
                                   _ptr(V_pages), _ptr(pos_cache), *_scratch(workspace, dev), st), "seka_rope_append")


def seka_paged_attention(shape: SekaPagedShape, Q, K_pages, V_pages, O, lse, workspace) -> None:
    """Attention of the new tokens over the paged cache; Q and O are bf16 [T, Hq, d], lse fp32 [T, Hq] or None."""
    st, dev = _on_device(shape), shape._device
    _fits("Q", Q, torch.bfloat16, shape._q, dev)
    _fits("K_pages", K_pages, torch.bfloat16, shape._pages, dev)
    _fits("V_pages", V_pages, torch.bfloat16, shape._pages, dev)
    _fits("O", O, torch.bfloat16, shape._q, dev)
    _fits("lse", lse, torch.float32, shape._q[:2], dev)
    _check(load().seka_paged_attention(ctypes.byref(shape), _ptr(Q), _ptr(K_pages), _ptr(V_pages), _ptr(O), _ptr(lse),
                                       *_scratch(workspace, dev), st), "seka_paged_attention")


def seka_attention_mass(shape: SekaPagedShape, Q, K_pages, lse, mass_in, mass_out, workspace) -> None:
    """Add the attention weight that the cached rows receive from the new tokens; mass is fp32 [B, Hkv, cap]."""
    st, dev = _on_device(shape), shape._device
    _fits("Q", Q, torch.bfloat16, shape._q, dev)
    _fits("K_pages", K_pages, torch.bfloat16, shape._pages, dev)
    _fits("lse", lse, torch.float32, shape._q[:2], dev)
    _fits("mass_in", mass_in, torch.float32, shape._state, dev)
    _fits("mass_out", mass_out, torch.float32, shape._state, dev)
    _check(load().seka_attention_mass(ctypes.byref(shape), _ptr(Q), _ptr(K_pages), _ptr(lse), _ptr(mass_in), _ptr(mass_out),
                                      *_scratch(workspace, dev), st), "seka_attention_mass")


def seka_evict_cache(shape: SekaPagedShape, K_pages, V_pages, mass_in, mass_out, pos_in, pos_out, protect, next_pos, keep: int,
                     recent: int, lens_out, workspace) -> None:
    """Cut every sequence to ``keep`` cached rows per KV head; ``protect`` is uint8 [B, P] over positions (or None)."""
    st, dev, B = _on_device(shape), shape._device, shape.batch
    _fits("K_pages", K_pages, torch.bfloat16, shape._pages, dev)
    _fits("V_pages", V_pages, torch.bfloat16, shape._pages, dev)
    for name, x, dt in (("mass_in", mass_in, torch.float32), ("mass_out", mass_out, torch.float32), ("pos_in", pos_in, torch.int32),
                        ("pos_out", pos_out, torch.int32)):
        _fits(name, x, dt, shape._state, dev)
    _fits("protect", protect, torch.uint8, (B, None), dev)
    _fits("next_pos", next_pos, torch.int32, (B,), dev)
    _fits("lens_out", lens_out, torch.int32, (B,), dev)
    _check(load().seka_evict_cache(ctypes.byref(shape), _ptr(K_pages), _ptr(V_pages), _ptr(mass_in), _ptr(mass_out), _ptr(pos_in),
                                   _ptr(pos_out), _ptr(protect), protect.shape[1] if protect is not None else 0, _ptr(next_pos),
                                   int(keep), int(recent), _ptr(lens_out), *_scratch(workspace, dev), st),
           "seka_evict_cache")
