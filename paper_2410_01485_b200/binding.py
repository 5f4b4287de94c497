"""Thin ctypes binding of the C-ABI library (argument marshalling only).

PyTorch supplies device memory and streams; every step of the attention path runs in
the library's CUDA kernels.  There is no CPU fallback: if the shared library is missing
or the device is not sm_100, calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblg_sparse_attn.so")

LG_OK = 0
MODE_FULL_CAUSAL, MODE_SINK_WINDOW, MODE_STRIDED_LOCAL = 0, 1, 2


class LgError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__("%s failed: %s (%d)" % (what, status_string(code), code))
        self.code = code


class AttnParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("L", C.c_int32), ("D", C.c_int32),
                ("block", C.c_int32), ("mode", C.c_int32), ("sink_tokens", C.c_int32),
                ("window_tokens", C.c_int32), ("stride_blocks", C.c_int32), ("local_blocks", C.c_int32),
                ("window_exact", C.c_int32), ("lists_prepared", C.c_int32), ("scale", C.c_float),
                ("q_strides", C.c_int64 * 3), ("k_strides", C.c_int64 * 3), ("v_strides", C.c_int64 * 3),
                ("o_strides", C.c_int64 * 3), ("doc_start", C.c_void_p)]


class DeviceStepBuffers(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("d_o", C.c_void_p),
                ("o", C.c_void_p), ("lse", C.c_void_p), ("dq", C.c_void_p), ("dk", C.c_void_p), ("dv", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class DecodeParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("sink_tokens", C.c_int32), ("window_tokens", C.c_int32), ("block_tokens", C.c_int32),
                ("scale", C.c_float)]


class PagedParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("sink_tokens", C.c_int32), ("window_tokens", C.c_int32), ("block_tokens", C.c_int32),
                ("scale", C.c_float), ("page_tokens", C.c_int32), ("num_pages", C.c_int32),
                ("table_stride", C.c_int32)]


_lib = None

# every symbol include/lg.h declares: (restype, argtypes)
_vp, _sz = C.c_void_p, C.c_size_t
SYMBOLS = {
    "lg_block_index_nnz": (C.c_int64, [C.POINTER(AttnParams)]),
    "lg_block_index_bytes": (_sz, [C.POINTER(AttnParams)]),
    "lg_build_block_index": (C.c_int, [C.POINTER(AttnParams), _vp, _vp, _vp, _vp, C.POINTER(C.c_int64), _vp]),
    "lg_sparse_attn_workspace_bytes": (_sz, [C.POINTER(AttnParams), C.c_int]),
    "lg_sparse_attn_prepare": (C.c_int, [C.POINTER(AttnParams), _vp, _sz, C.c_int, _vp]),
    "lg_sparse_attn_bwd_variant": (C.c_int32, [C.POINTER(AttnParams)]),
    "lg_sparse_attn_fwd": (C.c_int, [C.POINTER(AttnParams), _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "lg_sparse_attn_bwd": (C.c_int, [C.POINTER(AttnParams)] + [_vp] * 9 + [_vp, _sz, _vp]),
    "lg_sparse_attn_bwd_marked": (C.c_int, [C.POINTER(AttnParams)] + [_vp] * 9 + [_vp, _sz, _vp, C.POINTER(_vp)]),
    "lg_sparse_attn_fwd_bwd_host_workspace_bytes": (_sz, [C.POINTER(AttnParams), C.c_int]),
    "lg_sparse_attn_fwd_bwd_host": (C.c_int, [C.POINTER(AttnParams)] + [_vp] * 9 + [_vp, C.c_int, _vp, _vp, _vp]),
    "lg_kv_ring_append": (C.c_int, [C.POINTER(DecodeParams), _vp, _vp, _vp, _vp, C.c_int32, _vp, _vp]),
    "lg_sparse_decode_workspace_bytes": (_sz, [C.POINTER(DecodeParams)]),
    "lg_sparse_decode_workspace_init": (C.c_int, [_vp, _sz, _vp]),
    "lg_sparse_decode": (C.c_int, [C.POINTER(DecodeParams), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "lg_chunk_prefill_workspace_bytes": (_sz, [C.POINTER(DecodeParams), C.c_int32, C.c_int64]),
    "lg_chunk_prefill": (C.c_int, [C.POINTER(DecodeParams), _vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int64, _vp, _vp,
                                   _vp, _sz, _vp]),
    "lg_sparse_decode_static": (C.c_int, [C.POINTER(DecodeParams), _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "lg_sparse_decode_static_reset": (C.c_int, [_vp]),
    "lg_paged_table_extend": (C.c_int, [C.POINTER(PagedParams), _vp, _vp, C.c_int32, _vp, C.c_int32, _vp, _vp, _vp, _vp]),
    "lg_paged_slot_map": (C.c_int, [C.POINTER(PagedParams), _vp, _vp, _vp, C.c_int32, _vp, _vp, _vp]),
    "lg_paged_append": (C.c_int, [C.POINTER(PagedParams)] + [_vp] * 8 + [C.c_int32, _vp, _vp, _vp]),
    "lg_paged_gather": (C.c_int, [C.POINTER(PagedParams)] + [_vp] * 5 + [C.c_int32, _vp, _vp, _vp]),
    "lg_paged_decode_workspace_bytes": (_sz, [C.POINTER(PagedParams)]),
    "lg_paged_decode": (C.c_int, [C.POINTER(PagedParams)] + [_vp] * 10 + [_sz, _vp]),
    "lg_paged_chunk_prefill_workspace_bytes": (_sz, [C.POINTER(PagedParams), C.c_int32, _vp]),
    "lg_paged_chunk_prefill": (C.c_int, [C.POINTER(PagedParams)] + [_vp] * 8 + [C.c_int32] + [_vp] * 4 + [_sz, _vp]),
    "lg_selftest_wait_timeout": (C.c_int, [_vp, _vp]),
    "lg_last_status": (C.c_int, [_vp, _vp]),
    "lg_status_string": (C.c_char_p, [C.c_int]),
    "lg_debug_kernel_launches": (C.c_int64, []),
}


def load_library() -> C.CDLL:
    """Load the in-tree shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("CUDA library %s is missing: run `python -m paper_2410_01485_b200.build` "
                               "(there is no CPU fallback)" % LIB_PATH)
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def status_string(code: int) -> str:
    return load_library().lg_status_string(code).decode()


def _check(code: int, what: str):
    if code != LG_OK:
        raise LgError(code, what)


try:   # the handle alone: building a torch.cuda.Stream object for it costs three microseconds of a call
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _device
except ImportError:
    _raw_stream = None


def _stream() -> int:
    if _raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


_pack_strides = struct.Struct("=12q").pack_into      # q_strides .. o_strides, which lie side by side
_STRIDES_AT = AttnParams.q_strides.offset
assert AttnParams.o_strides.offset == _STRIDES_AT + 72


def _set_strides(p: AttnParams, q, k, v, o):
    """Strides of the four tensors [B, H, L, D] into p (one packed write: field by field it took 8 us); returns them."""
    qs, ks, vs, os_ = q.stride(), k.stride(), v.stride(), o.stride()
    assert len(qs) == len(ks) == len(vs) == len(os_) == 4 and qs[3] == ks[3] == vs[3] == os_[3] == 1, \
        "expect [B, H, L, D] with contiguous D"
    for t, s in ((q, qs), (k, ks), (v, vs), (o, os_)):     # (the library takes three zeros for a contiguous tensor)
        assert s[0] or s[1] or s[2] or t.is_contiguous(), "expect q, k, v, o not broadcast over B, H and L at once"
    _pack_strides(p, _STRIDES_AT, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], os_[0], os_[1], os_[2])
    return qs, ks, vs, os_


def attn_params(B, Hq, Hkv, L, D, block, mode, sink_tokens=0, window_tokens=0, stride_blocks=0, local_blocks=0,
                scale=0.0, window_exact=False, doc_start=None) -> AttnParams:
    """doc_start: optional CUDA int32 tensor [B, L] (first position of each token's document); the params
    object keeps a reference to it."""
    p = AttnParams()
    if doc_start is not None:
        assert doc_start.dtype == torch.int32 and doc_start.is_contiguous() and tuple(doc_start.shape) == (B, L)
        p.doc_start = doc_start.data_ptr()
        p._doc_start_ref = doc_start
    p.B, p.Hq, p.Hkv, p.L, p.D, p.block, p.mode = B, Hq, Hkv, L, D, block, mode
    p.sink_tokens, p.window_tokens, p.stride_blocks, p.local_blocks = sink_tokens, window_tokens, stride_blocks, local_blocks
    p.scale = scale
    p.window_exact = int(bool(window_exact))
    return p


def params_of(cfg, scale: float = 0.0, doc_start=None) -> AttnParams:
    """AttnParams from a synth.AttnConfig-like object."""
    return attn_params(cfg.B, cfg.Hq, cfg.Hkv, cfg.L, cfg.D, cfg.block, cfg.mode, cfg.sink_tokens,
                       cfg.window_tokens, cfg.stride_blocks, cfg.local_blocks, scale,
                       getattr(cfg, "window_exact", False), doc_start)


# ------------------------------------------------------------------------------ index

def lg_block_index_nnz(p: AttnParams) -> int:
    n = load_library().lg_block_index_nnz(C.byref(p))
    if n < 0:
        raise LgError(int(n), "lg_block_index_nnz")
    return int(n)


def lg_build_block_index(p: AttnParams, device="cuda") -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Returns device int32 tensors (row_ptr, col_idx, col_ptr, row_idx)."""
    lib = load_library()
    nnz = lg_block_index_nnz(p)
    nB = -(-p.L // p.block)
    assert lib.lg_block_index_bytes(C.byref(p)) == 4 * (2 * (nB + 1) + 2 * nnz)
    row_ptr = torch.empty(nB + 1, dtype=torch.int32, device=device)
    col_ptr = torch.empty(nB + 1, dtype=torch.int32, device=device)
    col_idx = torch.empty(max(nnz, 1), dtype=torch.int32, device=device)
    row_idx = torch.empty(max(nnz, 1), dtype=torch.int32, device=device)
    out = C.c_int64(-1)
    _check(lib.lg_build_block_index(C.byref(p), row_ptr.data_ptr(), col_idx.data_ptr(), col_ptr.data_ptr(),
                                    row_idx.data_ptr(), C.byref(out), _stream()), "lg_build_block_index")
    assert out.value == nnz
    return row_ptr, col_idx[:nnz], col_ptr, row_idx[:nnz]


# ------------------------------------------------------------------------- fwd / bwd

def attn_workspace(p: AttnParams, want_bwd: bool, device="cuda") -> torch.Tensor:
    n = load_library().lg_sparse_attn_workspace_bytes(C.byref(p), int(want_bwd))
    if n == 0:
        raise LgError(-1, "lg_sparse_attn_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def lg_sparse_attn_prepare(p: AttnParams, workspace: torch.Tensor, want_bwd: bool) -> AttnParams:
    """Build lists and schedules once into `workspace`; sets p.lists_prepared so that later forward /
    backward calls with this params object and workspace launch their attention kernels only."""
    p.lists_prepared = 0
    _check(load_library().lg_sparse_attn_prepare(C.byref(p), workspace.data_ptr(), workspace.numel(), int(want_bwd),
                                                 _stream()), "lg_sparse_attn_prepare")
    p.lists_prepared = 1
    return p


def bwd_variant_name(p: AttnParams) -> str:
    """Which backward variant lg_sparse_attn_bwd runs for these parameters."""
    v = load_library().lg_sparse_attn_bwd_variant(C.byref(p))
    if v < 0:
        raise LgError(int(v), "lg_sparse_attn_bwd_variant")
    return {0: "two_pass", 2: "keep_ds"}[int(v)]


def lg_sparse_attn_fwd(p: AttnParams, q, k, v, o=None, lse=None, workspace=None):
    """q [B,Hq,L,D], k, v [B,Hkv,L,D] bf16 CUDA tensors -> (o bf16, lse fp32 [B,Hq,L])."""
    lib = load_library()
    o = torch.empty_like(q) if o is None else o
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if lse is None else lse
    ws = attn_workspace(p, False, q.device) if workspace is None else workspace
    _set_strides(p, q, k, v, o)
    _check(lib.lg_sparse_attn_fwd(C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                  lse.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "lg_sparse_attn_fwd")
    return o, lse


def lg_sparse_attn_bwd(p: AttnParams, q, k, v, o, lse, d_o, dq=None, dk=None, dv=None, workspace=None):
    """Gradients (dq, dk, dv) bf16 of sum(O * dO)."""
    lib = load_library()
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    ws = attn_workspace(p, True, q.device) if workspace is None else workspace
    qs, ks, vs, os_ = _set_strides(p, q, k, v, o)
    assert d_o.stride() == os_ and dq.stride() == qs
    assert dk.stride() == ks and dv.stride() == vs
    _check(lib.lg_sparse_attn_bwd(C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                  lse.data_ptr(), d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                  ws.data_ptr(), ws.numel(), _stream()), "lg_sparse_attn_bwd")
    return dq, dk, dv


def lg_sparse_attn_bwd_marked(p: AttnParams, q, k, v, o, lse, d_o, dq, dk, dv, workspace, events):
    """As lg_sparse_attn_bwd; records the caller's four torch.cuda.Event objects (timing enabled, each
    recorded once before so that its handle exists) around the delta, dK/dV and dQ kernels.  Does not
    synchronise: read event durations after the stream has passed them."""
    _set_strides(p, q, k, v, o)
    assert len(events) == 4
    ev = (C.c_void_p * 4)(*[e.cuda_event for e in events])
    _check(load_library().lg_sparse_attn_bwd_marked(
        C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(),
        dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream(), ev),
        "lg_sparse_attn_bwd_marked")


def timing_events(n: int = 4):
    """n CUDA events with timing, each recorded once so that the driver object behind it exists."""
    evs = [torch.cuda.Event(enable_timing=True) for _ in range(n)]
    for e in evs:
        e.record()
    return evs


def host_step_workspace(p: AttnParams, head_groups: int, device="cuda") -> torch.Tensor:
    n = load_library().lg_sparse_attn_fwd_bwd_host_workspace_bytes(C.byref(p), head_groups)
    if n == 0:
        raise LgError(-1, "lg_sparse_attn_fwd_bwd_host_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def host_step_groups(p: AttnParams, head_groups: int) -> int:
    """The number of head groups a step can be cut into: `head_groups` if it divides Hkv, else 1."""
    return head_groups if (head_groups > 1 and p.Hkv % head_groups == 0) else 1


def sparse_attn_fwd_bwd_host(p: AttnParams, host_in, host_out, dev=None, head_groups: int = 4):
    """End-to-end training step with HOST buffers through lg_sparse_attn_fwd_bwd_host: pinned q, k, v, do
    go to the device, forward and backward run there, and o, lse, dq, dk, dv come back into the pinned
    tensors of `host_out`; head groups are pipelined over three streams inside the library call.
    `dev` optionally supplies preallocated device buffers (inputs dict, o, lse, dq, dk, dv, workspace of
    host_step_workspace(p, groups) bytes).  This wrapper only marshals pointers and streams."""
    n_groups = host_step_groups(p, head_groups)
    if dev is None:
        d_in = {k: torch.empty(v.shape, dtype=v.dtype, device="cuda") for k, v in host_in.items()}
        o = torch.empty_like(d_in["q"])
        lse = torch.empty(d_in["q"].shape[:3], dtype=torch.float32, device="cuda")
        dq, dk, dv = torch.empty_like(d_in["q"]), torch.empty_like(d_in["k"]), torch.empty_like(d_in["v"])
        ws = host_step_workspace(p, n_groups)
    else:
        d_in, o, lse, dq, dk, dv, ws = dev
    for t in list(host_in.values()) + list(host_out.values()) + list(d_in.values()) + [o, lse, dq, dk, dv]:
        assert t.is_contiguous()
    bufs = DeviceStepBuffers(d_in["q"].data_ptr(), d_in["k"].data_ptr(), d_in["v"].data_ptr(), d_in["do"].data_ptr(),
                             o.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                             ws.data_ptr(), ws.numel())
    cur = torch.cuda.current_stream()
    s_in, s_cmp, s_out = (_side_stream(i) for i in range(3))
    for st in (s_in, s_cmp, s_out):
        st.wait_stream(cur)
    _check(load_library().lg_sparse_attn_fwd_bwd_host(
        C.byref(p), host_in["q"].data_ptr(), host_in["k"].data_ptr(), host_in["v"].data_ptr(), host_in["do"].data_ptr(),
        host_out["o"].data_ptr(), host_out["lse"].data_ptr(), host_out["dq"].data_ptr(), host_out["dk"].data_ptr(),
        host_out["dv"].data_ptr(), C.byref(bufs), n_groups, s_in.cuda_stream, s_cmp.cuda_stream, s_out.cuda_stream),
        "lg_sparse_attn_fwd_bwd_host")
    for st in (s_in, s_cmp, s_out):
        cur.wait_stream(st)
    return host_out


_side_streams = {}


def _side_stream(i: int) -> "torch.cuda.Stream":
    key = (torch.cuda.current_device(), i)
    if key not in _side_streams:
        _side_streams[key] = torch.cuda.Stream()
    return _side_streams[key]


# ---------------------------------------------------------------------- decode / ring

def decode_params(B, Hq, Hkv, D, sink_tokens, window_tokens, scale=0.0, block_tokens=0) -> DecodeParams:
    """block_tokens: 0 = attend every token the cache holds; Bs = the block-granular window of training."""
    p = DecodeParams()
    p.B, p.Hq, p.Hkv, p.D, p.sink_tokens, p.window_tokens, p.scale = B, Hq, Hkv, D, sink_tokens, window_tokens, scale
    p.block_tokens = block_tokens
    return p


def lg_kv_ring_append(p: DecodeParams, k_cache, v_cache, k_new, v_new, n_tokens_before):
    """Append k_new, v_new [B,Hkv,T,D] in place; n_tokens_before int64 device [B]."""
    assert k_cache.is_contiguous() and v_cache.is_contiguous() and k_new.is_contiguous() and v_new.is_contiguous()
    _check(load_library().lg_kv_ring_append(C.byref(p), k_cache.data_ptr(), v_cache.data_ptr(), k_new.data_ptr(),
                                            v_new.data_ptr(), k_new.shape[2], n_tokens_before.data_ptr(),
                                            _stream()), "lg_kv_ring_append")


def decode_workspace(p: DecodeParams, device="cuda") -> torch.Tensor:
    """A workspace ready for lg_sparse_decode (allocated and zero-filled through the library's own call)."""
    n = load_library().lg_sparse_decode_workspace_bytes(C.byref(p))
    if n == 0:
        raise LgError(-1, "lg_sparse_decode_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _check(load_library().lg_sparse_decode_workspace_init(ws.data_ptr(), ws.numel(), _stream()),
           "lg_sparse_decode_workspace_init")
    return ws


def lg_sparse_decode(p: DecodeParams, q, k_cache, v_cache, n_tokens, o=None, lse=None, workspace=None,
                     want_lse: bool = True):
    """q [B,Hq,D] bf16 -> (o [B,Hq,D] bf16, lse [B,Hq] fp32 or None)."""
    assert q.is_contiguous() and k_cache.is_contiguous() and v_cache.is_contiguous()
    o = torch.empty_like(q) if o is None else o
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    ws = decode_workspace(p, q.device) if workspace is None else workspace
    _check(load_library().lg_sparse_decode(C.byref(p), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                           n_tokens.data_ptr(), o.data_ptr(), lse.data_ptr() if lse is not None else None,
                                           ws.data_ptr(), ws.numel(), _stream()), "lg_sparse_decode")
    return o, lse


def decode_call(p: DecodeParams, q, k_cache, v_cache, n_tokens, o, lse, workspace, stream=None):
    """lg_sparse_decode on fixed buffers (a serving loop's): every argument is marshalled once, the stream
    included (`stream`, default: the stream that is current now).  The returned function takes no arguments,
    launches on that stream and returns nothing (the results are in o, lse).  The tensors must stay alive
    and in place."""
    assert q.is_contiguous() and k_cache.is_contiguous() and v_cache.is_contiguous()
    fn = load_library().lg_sparse_decode
    handle = (torch.cuda.current_stream() if stream is None else stream).cuda_stream
    args = (C.byref(p), C.c_void_p(q.data_ptr()), C.c_void_p(k_cache.data_ptr()), C.c_void_p(v_cache.data_ptr()),
            C.c_void_p(n_tokens.data_ptr()), C.c_void_p(o.data_ptr()),
            C.c_void_p(lse.data_ptr() if lse is not None else None), C.c_void_p(workspace.data_ptr()),
            C.c_size_t(workspace.numel()), C.c_void_p(handle))
    keep = (p, q, k_cache, v_cache, n_tokens, o, lse, workspace)

    def call(_keep=keep):
        code = fn(*args)
        if code != LG_OK:
            raise LgError(code, "lg_sparse_decode")

    return call


def chunk_prefill_workspace(p: DecodeParams, T: int, n_tokens_before: int, device="cuda") -> torch.Tensor:
    n = load_library().lg_chunk_prefill_workspace_bytes(C.byref(p), T, n_tokens_before)
    if n == 0:
        raise LgError(-1, "lg_chunk_prefill_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def lg_chunk_prefill(p: DecodeParams, q_chunk, k_chunk, v_chunk, k_cache, v_cache, n_tokens_before: int,
                     o=None, lse=None, workspace=None):
    """q_chunk [B,Hq,T,D], k_chunk, v_chunk [B,Hkv,T,D] bf16 against the ring caches (None while empty);
    n_tokens_before is a host integer.  Returns (o [B,Hq,T,D] bf16, lse [B,Hq,T] fp32)."""
    assert q_chunk.is_contiguous() and k_chunk.is_contiguous() and v_chunk.is_contiguous()
    assert k_cache is None or (k_cache.is_contiguous() and v_cache.is_contiguous())
    T = q_chunk.shape[2]
    o = torch.empty_like(q_chunk) if o is None else o
    lse = torch.empty(q_chunk.shape[:3], dtype=torch.float32, device=q_chunk.device) if lse is None else lse
    ws = chunk_prefill_workspace(p, T, n_tokens_before, q_chunk.device) if workspace is None else workspace
    _check(load_library().lg_chunk_prefill(
        C.byref(p), q_chunk.data_ptr(), k_chunk.data_ptr(), v_chunk.data_ptr(),
        k_cache.data_ptr() if k_cache is not None else None, v_cache.data_ptr() if v_cache is not None else None,
        T, n_tokens_before, o.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "lg_chunk_prefill")
    return o, lse


DECODE_STATIC_SCRATCH_BYTES = 4 << 20   # LG_DECODE_STATIC_SCRATCH_BYTES of include/lg.h


def lg_sparse_decode_static(p: DecodeParams, q, k_cache, v_cache, n_tokens, o, lse=None):
    """lg_sparse_decode for callers that cannot allocate: no workspace argument, the split
    partials live in a fixed array inside the library (see include/lg.h).  `o` (and `lse`, if
    wanted) must be supplied by the caller, so this wrapper allocates nothing either."""
    assert q.is_contiguous() and k_cache.is_contiguous() and v_cache.is_contiguous() and o.is_contiguous()
    _check(load_library().lg_sparse_decode_static(C.byref(p), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                                  n_tokens.data_ptr(), o.data_ptr(),
                                                  lse.data_ptr() if lse is not None else None, _stream()),
           "lg_sparse_decode_static")
    return o, lse


# ------------------------------------------------------------------------- paged 8-bit cache

def paged_params(B, Hq, Hkv, D, sink_tokens, window_tokens, page_tokens, num_pages, scale=0.0, block_tokens=0,
                 table_stride=0) -> PagedParams:
    """Pools are float8_e4m3fn (or uint8) tensors [num_pages, Hkv, page_tokens, D], scales fp32 [num_pages, Hkv], the
    block table int32 [B, table_stride] (table_stride 0: ceil((sink_tokens + window_tokens) / page_tokens))."""
    return PagedParams(B, Hq, Hkv, D, sink_tokens, window_tokens, block_tokens, scale, page_tokens, num_pages, table_stride)


_I32, _I64, _F32, _BF16, _F8, _U8 = torch.int32, torch.int64, torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.uint8


# (The checks of a call are a microsecond or two of the host's time: every attribute of a tensor is asked for once.)
def _check_cache(p: PagedParams, k_pool, v_pool, k_scale, v_scale):
    pages, heads = p.num_pages, p.Hkv
    pool, scale, code = (pages, heads, p.page_tokens, p.D), (pages, heads), k_pool.dtype
    assert k_pool.shape == pool and v_pool.shape == pool and k_scale.shape == scale and v_scale.shape == scale, \
        "expect pools [num_pages, Hkv, page_tokens, D] and scales [num_pages, Hkv]"
    assert k_pool.is_contiguous() and v_pool.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()
    assert (code is _F8 or code is _U8) and v_pool.dtype is code and k_scale.dtype is _F32 and v_scale.dtype is _F32
    _check_device(k_pool, v_pool, k_scale, v_scale)


def _check_device(*tensors):
    """All of a call's tensors lie on the device whose stream it goes to (a host tensor's address would fault the GPU)."""
    dev = _device() if _raw_stream is not None else torch.cuda.current_device()
    for t in tensors:
        assert t.get_device() == dev, "expect tensors on the current CUDA device"


def _check_table(p: PagedParams, block_table):
    columns = p.table_stride or -(-(p.sink_tokens + p.window_tokens) // max(1, p.page_tokens))
    assert block_table.shape == (p.B, columns) and block_table.dtype is _I32 and block_table.is_contiguous(), \
        "expect an int32 block table [B, table_stride]"


def _check_counts(B, dtype, n):
    assert n.dtype is dtype and n.numel() == B and n.is_contiguous()


_Strides = C.c_int64 * 3


def _ptr(t):
    return None if t is None else t.data_ptr()


def lg_paged_table_extend(p: PagedParams, n_tokens_before, n_new, free_pages, free_start, block_table, free_next,
                          T_new: Optional[int] = None):
    """New pages from free_pages (int32) into block_table for sequences that grow from n_tokens_before (int64 [B]) by n_new
    (int32 [B]; None: T_new each) tokens; free_start, free_next: int32 tensors of one element each."""
    _check_counts(p.B, _I64, n_tokens_before)
    if n_new is not None:
        _check_counts(p.B, _I32, n_new)
    else:
        assert T_new is not None
    _check_table(p, block_table)
    assert free_pages.dtype is _I32 and free_start.dtype is _I32 and free_next.dtype is _I32 and free_pages.is_contiguous()
    _check_device(n_tokens_before, block_table, free_pages, free_start, free_next, n_new if n_new is not None else free_next)
    code = load_library().lg_paged_table_extend(
        C.byref(p), n_tokens_before.data_ptr(), _ptr(n_new), 0x7fffffff if T_new is None else T_new, free_pages.data_ptr(),
        free_pages.numel(), free_start.data_ptr(), block_table.data_ptr(), free_next.data_ptr(), _stream())
    if code != LG_OK:
        raise LgError(code, "lg_paged_table_extend")


def lg_paged_slot_map(p: PagedParams, n_tokens, first, count, block_table, slot_map):
    """slot_map (int64 [B, T]): where the cache holds positions first .. first + count - 1 (count int32 [B]; None: T)."""
    B, T = slot_map.shape
    _check_counts(B, _I64, n_tokens)
    _check_counts(B, _I64, first)
    if count is not None:
        _check_counts(B, _I32, count)
    _check_table(p, block_table)
    assert B == p.B and slot_map.dtype is _I64 and slot_map.is_contiguous()
    _check_device(n_tokens, first, block_table, slot_map, count if count is not None else first)
    code = load_library().lg_paged_slot_map(C.byref(p), n_tokens.data_ptr(), first.data_ptr(), _ptr(count), T, block_table.data_ptr(),
                                            slot_map.data_ptr(), _stream())
    if code != LG_OK:
        raise LgError(code, "lg_paged_slot_map")
    return slot_map


def _append_args(p: PagedParams, k_pool, v_pool, k_scale, v_scale, block_table, k_new, v_new, n_tokens_before, n_new):
    _check_cache(p, k_pool, v_pool, k_scale, v_scale)
    _check_table(p, block_table)
    B, H, T, D = shape = k_new.shape
    _check_counts(B, _I64, n_tokens_before)
    if n_new is not None:
        _check_counts(B, _I32, n_new)
    assert B == p.B and H == p.Hkv and D == p.D and v_new.shape == shape and k_new.dtype is _BF16 and v_new.dtype is _BF16
    _check_device(block_table, k_new, v_new, n_tokens_before, n_new if n_new is not None else n_tokens_before)
    if k_new.is_contiguous() and v_new.is_contiguous():
        st = None
    else:
        strides, other = k_new.stride(), v_new.stride()
        if 1 in shape:         # (the stride of a dimension of one element says nothing)
            whole = (H * T * D, T * D, D, 1)
            strides, other = (tuple(w if n == 1 else s for s, n, w in zip(x, shape, whole)) for x in (strides, other))
        assert strides == other, "k_new and v_new must have the same strides"
        assert strides[3] == 1, "expect contiguous D"
        st = _Strides(strides[0], strides[1], strides[2])
    return (C.byref(p), k_pool.data_ptr(), v_pool.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), block_table.data_ptr(),
            k_new.data_ptr(), v_new.data_ptr(), st, T, n_tokens_before.data_ptr(), _ptr(n_new))


def lg_paged_append(p: PagedParams, k_pool, v_pool, k_scale, v_scale, block_table, k_new, v_new, n_tokens_before, n_new=None):
    """Append k_new, v_new [B,Hkv,T,D] (any strides of 8 elements with contiguous D) in place; n_tokens_before int64 [B], n_new
    int32 [B] or None for T tokens each."""
    _check(load_library().lg_paged_append(*_append_args(p, k_pool, v_pool, k_scale, v_scale, block_table, k_new, v_new,
                                                        n_tokens_before, n_new), _stream()), "lg_paged_append")


def paged_append_call(p: PagedParams, k_pool, v_pool, k_scale, v_scale, block_table, k_new, v_new, n_tokens_before, n_new=None,
                      stream=None):
    """lg_paged_append on fixed buffers, every argument marshalled once (as decode_call)."""
    args = _append_args(p, k_pool, v_pool, k_scale, v_scale, block_table, k_new, v_new, n_tokens_before, n_new)
    return _fixed_call("lg_paged_append", args, stream,
                       (p, k_pool, v_pool, k_scale, v_scale, block_table, k_new, v_new, n_tokens_before, n_new))


def lg_paged_gather(p: PagedParams, k_pool, v_pool, k_scale, v_scale, slot_map, k_out=None, v_out=None):
    """Rows of the cache at slot_map (int64 [B, T]) as bf16 [B, Hkv, T, D]; zeros where it is negative."""
    _check_cache(p, k_pool, v_pool, k_scale, v_scale)
    B, T = slot_map.shape
    assert B == p.B and slot_map.dtype is _I64 and slot_map.is_contiguous()
    shape = (B, p.Hkv, T, p.D)
    if k_out is None:
        k_out = torch.empty(shape, dtype=torch.bfloat16, device=k_pool.device)
    if v_out is None:
        v_out = torch.empty_like(k_out)
    for t in (k_out, v_out):
        assert t.shape == shape and t.dtype is _BF16 and t.is_contiguous()
    _check_device(slot_map, k_out, v_out)
    _check(load_library().lg_paged_gather(C.byref(p), k_pool.data_ptr(), v_pool.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                          slot_map.data_ptr(), T, k_out.data_ptr(), v_out.data_ptr(), _stream()), "lg_paged_gather")
    return k_out, v_out


def paged_decode_workspace(p: PagedParams, device="cuda") -> torch.Tensor:
    """A workspace ready for lg_paged_decode (allocated and zero-filled)."""
    n = load_library().lg_paged_decode_workspace_bytes(C.byref(p))
    if n == 0:
        raise LgError(-1, "lg_paged_decode_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _check(load_library().lg_sparse_decode_workspace_init(ws.data_ptr(), ws.numel(), _stream()),
           "lg_sparse_decode_workspace_init")
    return ws


def _decode_args(p: PagedParams, q, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens, o, lse, workspace):
    _check_cache(p, k_pool, v_pool, k_scale, v_scale)
    _check_table(p, block_table)
    _check_counts(p.B, _I64, n_tokens)
    shape = (p.B, p.Hq, p.D)
    for t in (q, o):
        assert t.shape == shape and t.dtype is _BF16 and t.is_contiguous()
    assert lse is None or (lse.shape == shape[:2] and lse.dtype is _F32 and lse.is_contiguous())
    _check_device(q, block_table, n_tokens, o, workspace, lse if lse is not None else o)
    return (C.byref(p), q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
            block_table.data_ptr(), n_tokens.data_ptr(), o.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel())


def lg_paged_decode(p: PagedParams, q, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens, o=None, lse=None, workspace=None,
                    want_lse: bool = True):
    """q [B,Hq,D] bf16 over the paged cache -> (o [B,Hq,D] bf16, lse [B,Hq] fp32 or None)."""
    o = torch.empty_like(q) if o is None else o
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    ws = paged_decode_workspace(p) if workspace is None else workspace
    _check(load_library().lg_paged_decode(*_decode_args(p, q, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens, o, lse, ws),
                                          _stream()), "lg_paged_decode")
    return o, lse


def paged_decode_call(p: PagedParams, q, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens, o, lse, workspace, stream=None):
    """lg_paged_decode on fixed buffers, every argument marshalled once (as decode_call)."""
    args = _decode_args(p, q, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens, o, lse, workspace)
    return _fixed_call("lg_paged_decode", args, stream,
                       (p, q, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens, o, lse, workspace))


def _fixed_call(name, args, stream, keep):
    """A function without arguments that makes the call on `stream` (default: the one current now); `keep` stays alive."""
    fn = getattr(load_library(), name)
    handle = (torch.cuda.current_stream() if stream is None else stream).cuda_stream
    args = tuple(t(a) if isinstance(a, int) else a for t, a in zip(fn.argtypes, args)) + (C.c_void_p(handle),)

    def call(_keep=keep):
        code = fn(*args)
        if code != LG_OK:
            raise LgError(code, name)

    return call


def _host_counts(p: PagedParams, n_tokens_before):
    n = [int(x) for x in n_tokens_before]
    assert len(n) == p.B
    return (C.c_int64 * p.B)(*n)


def paged_chunk_prefill_workspace(p: PagedParams, T: int, n_tokens_before, device="cuda") -> torch.Tensor:
    n = load_library().lg_paged_chunk_prefill_workspace_bytes(C.byref(p), T, _host_counts(p, n_tokens_before))
    if n == 0:
        raise LgError(-1, "lg_paged_chunk_prefill_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def lg_paged_chunk_prefill(p: PagedParams, q_chunk, k_chunk, v_chunk, k_pool, v_pool, k_scale, v_scale, block_table, n_tokens_before,
                           o=None, lse=None, workspace=None):
    """q_chunk [B,Hq,T,D], k_chunk, v_chunk [B,Hkv,T,D] bf16 against the paged cache; n_tokens_before: B host integers.
    Returns (o [B,Hq,T,D] bf16, lse [B,Hq,T] fp32)."""
    _check_cache(p, k_pool, v_pool, k_scale, v_scale)
    _check_table(p, block_table)
    B, T, D = p.B, q_chunk.shape[2], p.D
    for t, H in ((q_chunk, p.Hq), (k_chunk, p.Hkv), (v_chunk, p.Hkv)):
        assert t.shape == (B, H, T, D) and t.dtype is _BF16 and t.is_contiguous()
    _check_device(q_chunk, k_chunk, v_chunk, block_table)
    o = torch.empty_like(q_chunk) if o is None else o
    lse = torch.empty(q_chunk.shape[:3], dtype=torch.float32, device=q_chunk.device) if lse is None else lse
    ws = paged_chunk_prefill_workspace(p, T, n_tokens_before) if workspace is None else workspace
    assert o.shape == q_chunk.shape and o.dtype is _BF16 and o.is_contiguous()
    assert lse.shape == q_chunk.shape[:3] and lse.dtype is _F32 and lse.is_contiguous()
    _check_device(o, lse, ws)
    _check(load_library().lg_paged_chunk_prefill(
        C.byref(p), q_chunk.data_ptr(), k_chunk.data_ptr(), v_chunk.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
        k_scale.data_ptr(), v_scale.data_ptr(), block_table.data_ptr(), T, _host_counts(p, n_tokens_before), o.data_ptr(),
        lse.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "lg_paged_chunk_prefill")
    return o, lse


def lg_selftest_wait_timeout(workspace: torch.Tensor) -> None:
    """Launch the one-warp kernel whose bounded wait must expire (see include/lg.h)."""
    _check(load_library().lg_selftest_wait_timeout(workspace.data_ptr(), _stream()), "lg_selftest_wait_timeout")


def kernel_launches() -> int:
    """Kernels launched by the library in this process so far (diagnostic counter)."""
    return int(load_library().lg_debug_kernel_launches())


def lg_last_status(workspace: torch.Tensor) -> int:
    return int(load_library().lg_last_status(workspace.data_ptr(), _stream()))
