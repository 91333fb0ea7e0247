"""Thin Python binding of the C ABI (include/provip.h), same names.

Argument marshalling only: torch tensors give device pointers, the current
torch stream gives the cudaStream_t, and torch allocates the workspace and the
outputs. Every step of the pruning path runs in the CUDA library; there is no
CPU or PyTorch fallback - if ``libprovip.so`` is missing or a call fails, a
``ProvipError`` is raised.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libprovip.so")

OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED = -2
ERR_WORKSPACE = -3
ERR_CUDA = -4
ERR_TIMEOUT = -5
DEVSTAT_TIMEOUT, DEVSTAT_BAD_ARG = 1, 2  # bits of the device status word
F32, BF16 = 0, 1
ALGO_AUTO, ALGO_SIMT, ALGO_TCGEN05, ALGO_TCGEN05_TWOPASS = 0, 1, 2, 3
ALGO_TCGEN05_STREAM, ALGO_TCGEN05_CLUSTER = 4, 5
PRUNE_OVERLAP_PREVIOUS = 1
PRUNE_CONCURRENT = 2
PRUNE_HOST_ROWS = 4

_P = ctypes.c_void_p
_I = ctypes.c_int
_L = ctypes.c_longlong
_F = ctypes.c_float
_Z = ctypes.c_size_t

# name -> (restype, argtypes); mirrors include/provip.h
_SIGS = {
    "provip_status_string": (ctypes.c_char_p, [_I]),
    "provip_last_error": (ctypes.c_char_p, []),
    "provip_version": (_I, []),
    "provip_set_option": (_I, [_I, _I]),
    "provip_device_status": (_I, [_P, _I]),
    "provip_selftest_wait_timeout": (_I, [_P]),
    "provip_crit_text_workspace_size": (_Z, [_I, _I, _I]),
    "provip_crit_text": (_I, [_P, _I, _I, _I, _P, _I, _P, _P, _P, _Z, _P]),
    "provip_relevance_workspace_size": (_Z, [_I, _I, _I, _I]),
    "provip_relevance": (_I, [_P, _I, _I, _I, _P, _P, _I, _P, _I, _P, _P, _Z, _P]),
    "provip_topk": (_I, [_P, _I, _I, _I, _P, _P]),
    "provip_merge_workspace_size": (_Z, [_I, _I, _I, _I]),
    "provip_merge": (_I, [_P, _I, _I, _I, _P, _I, _I, _P, _P, _P, _Z, _P]),
    "provip_similarity_reduce_workspace_size": (_Z, [_I, _I, _I, _I, _I]),
    "provip_similarity_reduce": (_I, [_P, _I, _I, _I, _P, _P, _I, _P, _I, _I, _P, _P, _P, _P, _P, _P, _Z,
                                      _P]),
    "provip_head_scores_workspace_size": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "provip_head_scores": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _I, _P, _P, _P, _I, _I, _I, _P, _I, _I,
                                _P, _P, _Z, _P]),
    "provip_head_scores_noalloc": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _I, _P, _P, _P, _I, _I, _I, _P, _I,
                                        _I, _P, _P]),
    "provip_compact": (_I, [_P, _I, _I, _I, _P, _I, _P, _P, _I, _I, _P, _I, _P, _I, _I, _I, _P, _P, _P,
                            _P, _P, _P]),
    "provip_topk_compact": (_I, [_P, _I, _I, _I, _P, _I, _P, _P, _I, _I, _P, _I, _P, _I, _I, _I, _P, _P,
                                 _P, _P, _P, _P, _P]),
    "provip_head_topk": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _I, _P, _P, _P, _I, _I, _I, _P, _I, _I, _I,
                              _P, _P, _P, _Z, _P]),
    "provip_prune_workspace_size": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "provip_prune": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P, _I, _P, _P, _P, _I, _I, _I, _P, _P,
                          _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _Z, ctypes.c_uint, _P]),
    "provip_visual_heads_workspace_size": (_Z, [_I, _I, _I, _I, _I, _I, _I, _I]),
    "provip_head_confidence": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _I, _I, _P, _I, _I, _I,
                                    _P, _P, _P, _Z, _P]),
    "provip_prune_visual_heads": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P, _P, _P, _I, _I, _I, _P,
                                       _P, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _Z,
                                       ctypes.c_uint, _P]),
    "provip_prompt_attention_workspace_size": (_Z, [_I] * 9),
    "provip_prompt_attention": (_I, [_P, _L, _P, _L, _P, _L, _I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _I, _I, _P, _L, _P,
                                     _L, _I, _I, _F, _I, _I, _P, _L, _P, _P, _Z, _P]),
    "provip_page_tables": (_I, [_P, _P, _I, _I, _P, _I, _P, _P, _I, _I, _P, _P, _P, _P, _P]),
    "provip_kv_append": (_I, [_P, _L, _P, _L, _I, _I, _I, _P, _I, _I, _I, _P, _P, _P]),
    "provip_decode_attention_workspace_size": (_Z, [_I] * 7),
    "provip_decode_attention": (_I, [_P, _L, _I, _I, _I, _I, _P, _P, _I, _I, _P, _I, _P, _I, _P, _I, _F, _I, _I, _P, _L,
                                     _P, _P, _Z, _P]),
    "provip_rotate": (_I, [_P, _L, _P, _L, _I, _P, _I, _I, _I, _P, _L, _I, _P, _P, _F, _P, _P, _F, _I, _P, _L, _P, _L, _P]),
    "provip_rotate_append": (_I, [_P, _L, _P, _L, _P, _L, _I, _P, _I, _I, _I, _P, _L, _I, _P, _P, _F, _P, _P, _F, _I, _P, _L,
                                  _P, _L, _P, _I, _I, _I, _P, _P, _P]),
    "provip_kv_append4": (_I, [_P, _L, _P, _L, _I, _I, _I, _P, _I, _I, _I, _P, _P, _P]),
    "provip_kv_read4": (_I, [_P, _I, _I, _I, _P, _P, _I, _I, _I, _P, _L, _P, _L, _P]),
    "provip_decode_attention4_workspace_size": (_Z, [_I] * 6),
    "provip_decode_attention4": (_I, [_P, _L, _I, _I, _I, _I, _P, _P, _I, _I, _P, _I, _P, _I, _P, _I, _F, _I, _P, _L, _P, _P,
                                      _Z, _P]),
}


class ProvipError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{msg} (status {code})")
        self.code = code


_lib = None
_lock = threading.Lock()


def lib():
    """Loads libprovip.so (raises if it has not been built: there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise ProvipError(ERR_UNSUPPORTED, f"CUDA library not built: {LIB_PATH} is missing "
                                  "(run __graft_entry__.build())")
            L = ctypes.CDLL(LIB_PATH)
            for name, (res, args) in _SIGS.items():
                f = getattr(L, name)
                f.restype = res
                f.argtypes = args
            _lib = L
    return _lib


def _check(rc, what):
    if rc != OK:
        L = lib()
        msg = L.provip_last_error().decode() or L.provip_status_string(rc).decode()
        raise ProvipError(rc, f"{what}: {msg}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise ProvipError(ERR_UNSUPPORTED, f"unsupported dtype {t.dtype}")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ProvipError(ERR_INVALID_ARG, "tensor must live on the GPU")
    if not t.is_contiguous():
        raise ProvipError(ERR_INVALID_ARG, "tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _ptr_host_ok(t):
    """a device tensor, or a pinned host tensor (mapped into the device's
    address space) for the arguments PROVIP_PRUNE_HOST_ROWS allows there"""
    if t is not None and not t.is_cuda:
        if not t.is_pinned():
            raise ProvipError(ERR_INVALID_ARG, "a host tensor must be pinned (pin_memory())")
        if not t.is_contiguous():
            raise ProvipError(ERR_INVALID_ARG, "tensor must be contiguous")
        return ctypes.c_void_p(t.data_ptr())
    return _ptr(t)


def _stream(device):
    """The device's current stream as torch has it. (torch.cuda.current_stream builds an object
    around the same handle, 2 us of a 10 us call; it is the way where the handle has no
    accessor, and for a device given by its name or number.)"""
    if _raw_stream is None or not isinstance(device, torch.device):
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index if device.index is not None else torch.cuda.current_device())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _i32(t):
    if t is None:
        return None
    if t.dtype != torch.int32:
        raise ProvipError(ERR_INVALID_ARG, "index/length tensors must be int32")
    return _ptr(t)


def _i32_host_ok(t):
    if t is None:
        return None
    if t.dtype != torch.int32:
        raise ProvipError(ERR_INVALID_ARG, "index/length tensors must be int32")
    return _ptr_host_ok(t)


def _u8(t):
    if t is None:
        return None
    if t.dtype != torch.uint8:
        raise ProvipError(ERR_INVALID_ARG, "masks must be uint8")
    return _ptr(t)


def workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------
# status
# ---------------------------------------------------------------------------
def provip_device_status(clear: bool = True):
    """Synchronises and returns (status code, device status bits)."""
    bits = ctypes.c_uint(0)
    rc = lib().provip_device_status(ctypes.byref(bits), 1 if clear else 0)
    return rc, bits.value


def provip_selftest_wait_timeout(device="cuda:0"):
    """Enqueues the failure-detection self test: a bounded wait that nothing
    completes gives up after 2 s and sets the TIMEOUT bit of the device status
    word (read it with provip_device_status)."""
    _check(lib().provip_selftest_wait_timeout(_stream(torch.device(device))), "provip_selftest_wait_timeout")


def provip_version() -> int:
    return lib().provip_version()


OPT_MERGE_PAIRS = 1


def provip_set_option(option: int, value: int) -> None:
    """Process-wide kernel-choice switch (PROVIP_OPT_*), for calls enqueued after it."""
    _check(lib().provip_set_option(int(option), int(value)), "provip_set_option")


# ---------------------------------------------------------------------------
# pre-LLM pass
# ---------------------------------------------------------------------------
def provip_crit_text(emb_t, text_len, want_r=False, out=None, ws=None):
    """Sec. 4.2: the critical-row mask T [B, N_t_max] (and r when want_r); out: a
    pre-allocated mask to write, ws: a pre-allocated workspace."""
    B, Ntm, D = emb_t.shape
    dev = emb_t.device
    mask = out if out is not None else torch.empty((B, Ntm), dtype=torch.uint8, device=dev)
    r = torch.empty((B, Ntm), dtype=torch.float32, device=dev) if want_r else None
    L = lib()
    need = L.provip_crit_text_workspace_size(B, Ntm, D)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    rc = L.provip_crit_text(_ptr(emb_t), B, Ntm, D, _i32(text_len), _dtype_code(emb_t), _u8(mask),
                            _ptr(r), _ptr(ws), ws.numel(), _stream(dev))
    _check(rc, "provip_crit_text")
    return (mask, r) if want_r else mask


def provip_relevance(emb_v, emb_t, text_len, crit_mask):
    B, Nv, D = emb_v.shape
    Ntm = emb_t.shape[1]
    dev = emb_v.device
    p = torch.empty((B, Nv), dtype=torch.float32, device=dev)
    L = lib()
    ws = workspace(L.provip_relevance_workspace_size(B, Nv, D, Ntm), dev)
    rc = L.provip_relevance(_ptr(emb_v), B, Nv, D, _ptr(emb_t), _i32(text_len), Ntm, _u8(crit_mask),
                            _dtype_code(emb_v), _ptr(p), _ptr(ws), ws.numel(), _stream(dev))
    _check(rc, "provip_relevance")
    return p


def provip_topk(scores, k):
    B, N = scores.shape
    idx = torch.empty((B, k), dtype=torch.int32, device=scores.device)
    rc = lib().provip_topk(_ptr(scores), B, N, k, _ptr(idx), _stream(scores.device))
    _check(rc, "provip_topk")
    return idx


def provip_merge(emb_v, keep_idx, want_merged=True):
    B, Nv, D = emb_v.shape
    keep = keep_idx.shape[1]
    dev = emb_v.device
    assign = torch.empty((B, Nv), dtype=torch.int32, device=dev)
    merged = torch.empty((B, keep, D), dtype=emb_v.dtype, device=dev) if want_merged else None
    L = lib()
    ws = workspace(L.provip_merge_workspace_size(B, Nv, D, keep), dev)
    rc = L.provip_merge(_ptr(emb_v), B, Nv, D, _i32(keep_idx), keep, _dtype_code(emb_v), _ptr(assign),
                        _ptr(merged), _ptr(ws), ws.numel(), _stream(dev))
    _check(rc, "provip_merge")
    return assign, merged


def provip_similarity_reduce(emb_v, emb_t, text_len, keep_pre, crit_mask=None, want_merged=True,
                             ws=None, out=None, want_assign=False):
    """Sec. 4.2-4.3 end to end. Returns dict(idx, merged, p, mask, assign); out:
    the same dict of pre-allocated outputs to write instead (assign optional:
    the merge's nearest-centroid positions [B, N_v], with want_assign or given
    in out)."""
    B, Nv, D = emb_v.shape
    Ntm = emb_t.shape[1]
    dev = emb_v.device
    if out is not None:
        idx, merged, p, mask = out["idx"], out.get("merged"), out["p"], out["mask"]
        assign = out.get("assign")
    else:
        idx = torch.empty((B, keep_pre), dtype=torch.int32, device=dev)
        merged = torch.empty((B, keep_pre, D), dtype=emb_v.dtype, device=dev) if want_merged else None
        p = torch.empty((B, Nv), dtype=torch.float32, device=dev)
        mask = torch.empty((B, Ntm), dtype=torch.uint8, device=dev)
        assign = torch.empty((B, Nv), dtype=torch.int32, device=dev) if (want_assign and want_merged) else None
    L = lib()
    need = L.provip_similarity_reduce_workspace_size(B, Nv, D, Ntm, keep_pre)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    rc = L.provip_similarity_reduce(_ptr(emb_v), B, Nv, D, _ptr(emb_t), _i32(text_len), Ntm,
                                    _u8(crit_mask), keep_pre, _dtype_code(emb_v), _ptr(idx),
                                    _ptr(merged), _i32(assign), _ptr(p), _ptr(mask), _ptr(ws),
                                    ws.numel(), _stream(dev))
    _check(rc, "provip_similarity_reduce")
    return dict(idx=idx, merged=merged, p=p, mask=mask, assign=assign)


# ---------------------------------------------------------------------------
# in-LLM pass
# ---------------------------------------------------------------------------
def _heads_arg(head_list, H_q):
    """head_list is read on the host (a list, a CPU tensor, or a device tensor copied once);
    None means every head (a NULL list with H_sel = H_q)."""
    if head_list is None:
        return None, int(H_q)
    hl = [int(h) for h in (head_list.tolist() if hasattr(head_list, "tolist") else head_list)]
    arr = (ctypes.c_int * len(hl))(*hl)
    return arr, len(hl)


def provip_head_scores(Q, K, head_list, text_start, text_len, seq_len, vis_start, N_v,
                       row_mask=None, algo=ALGO_AUTO, N_t_max=None, ws=None):
    B, Lm, Hq, dh = Q.shape
    Hkv = K.shape[2]
    dev = Q.device
    heads, hs = _heads_arg(head_list, Hq)
    Ntm = int(N_t_max if N_t_max is not None else (row_mask.shape[1] if row_mask is not None
                                                   else int(text_len.max().item())))
    scores = torch.empty((B, N_v), dtype=torch.float32, device=dev)
    L = lib()
    dt = _dtype_code(Q)
    need = L.provip_head_scores_workspace_size(B, Lm, hs, Ntm, N_v, algo, dt)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    rc = L.provip_head_scores(_ptr(Q), _ptr(K), B, Lm, Hq, Hkv, dh, heads, hs, _i32(text_start),
                              _i32(text_len), _u8(row_mask), Ntm, vis_start, N_v, _i32(seq_len), dt,
                              algo, _ptr(scores), _ptr(ws), ws.numel(), _stream(dev))
    _check(rc, "provip_head_scores")
    return scores


def _outs(hidden, K, V, pos, B, L_out, device=None):
    dev = hidden.device if device is None else device
    ho = torch.empty((B, L_out) + tuple(hidden.shape[2:]), dtype=hidden.dtype, device=dev)
    ko = torch.empty((B, L_out) + tuple(K.shape[2:]), dtype=K.dtype, device=dev) if K is not None else None
    vo = torch.empty((B, L_out) + tuple(V.shape[2:]), dtype=V.dtype, device=dev) if V is not None else None
    po = torch.full((pos.shape[0], B, L_out), -1, dtype=torch.int32, device=dev) if pos is not None else None
    return ho, ko, vo, po


def provip_compact(idx, hidden, K, V, pos, seq_len, vis_start, N_v, out=None):
    """hidden, K, V, pos and the outputs may be device tensors or pinned host
    tensors (the library detects host memory); idx and seq_len live on the
    device, and the outputs default to device tensors."""
    B, Lm, D = hidden.shape
    keep = idx.shape[1]
    Hkv, dh = (K.shape[2], K.shape[3]) if K is not None else (0, 0)
    P = pos.shape[0] if pos is not None else 0
    ho, ko, vo, po = out if out is not None else _outs(hidden, K, V, pos, B, Lm - N_v + keep, idx.device)
    slo = torch.empty(B, dtype=torch.int32, device=idx.device)
    rc = lib().provip_compact(_i32(idx), B, N_v, keep, _ptr_host_ok(hidden), D, _ptr_host_ok(K), _ptr_host_ok(V),
                              Hkv, dh, _i32_host_ok(pos), P, _i32(seq_len), Lm, vis_start, _dtype_code(hidden),
                              _ptr_host_ok(ho), _ptr_host_ok(ko), _ptr_host_ok(vo), _i32_host_ok(po), _i32(slo),
                              _stream(idx.device))
    _check(rc, "provip_compact")
    return dict(hidden=ho, K=ko, V=vo, pos=po, seq_len=slo)


def provip_topk_compact(scores, keep, hidden, K, V, pos, seq_len, vis_start):
    B, Lm, D = hidden.shape
    N_v = scores.shape[1]
    Hkv, dh = (K.shape[2], K.shape[3]) if K is not None else (0, 0)
    P = pos.shape[0] if pos is not None else 0
    ho, ko, vo, po = _outs(hidden, K, V, pos, B, Lm - N_v + keep)
    idx = torch.empty((B, keep), dtype=torch.int32, device=hidden.device)
    slo = torch.empty(B, dtype=torch.int32, device=hidden.device)
    rc = lib().provip_topk_compact(_ptr(scores), B, N_v, keep, _ptr(hidden), D, _ptr(K), _ptr(V), Hkv,
                                   dh, _i32(pos), P, _i32(seq_len), Lm, vis_start,
                                   _dtype_code(hidden), _ptr(ho), _ptr(ko), _ptr(vo), _i32(po),
                                   _ptr(idx), _i32(slo), _stream(hidden.device))
    _check(rc, "provip_topk_compact")
    return dict(hidden=ho, K=ko, V=vo, pos=po, idx=idx, seq_len=slo)


class PruneStep:
    """Pre-allocated outputs + workspace for repeated provip_prune calls (one shape)."""

    def __init__(self, Q, K, V, hidden, pos, head_list, N_t_max, N_v, keep, algo=ALGO_AUTO,
                 want_scores=True, flags=0, ws=None, device=None, host_rows=False):
        """Q, K, V, hidden, pos give the shapes and dtypes (meta tensors are fine
        with device=...). host_rows: the compacted outputs are pinned host
        tensors, and hidden, V and pos may be pinned host tensors too
        (PROVIP_PRUNE_HOST_ROWS)."""
        B, Lm, Hq, dh = Q.shape
        self.shape = (B, Lm, Hq, K.shape[2], dh, hidden.shape[2])
        self.heads, self.H_sel = _heads_arg(head_list, Q.shape[2])
        self.N_t_max, self.N_v, self.keep, self.algo = int(N_t_max), int(N_v), int(keep), algo
        self.flags = int(flags) | (PRUNE_HOST_ROWS if host_rows else 0)
        dev = Q.device if device is None else torch.device(device)
        self.dtype = _dtype_code(Q)
        L_out = Lm - N_v + keep
        self.hidden_out, self.K_out, self.V_out, self.pos_out = _outs(hidden, K, V, pos, B, L_out, dev)
        if host_rows:
            self.hidden_out, self.K_out, self.V_out, self.pos_out = (
                None if t is None else torch.empty(t.shape, dtype=t.dtype, pin_memory=True)
                for t in (self.hidden_out, self.K_out, self.V_out, self.pos_out))
        self.idx = torch.empty((B, keep), dtype=torch.int32, device=dev)
        self.seq_len_out = torch.empty(B, dtype=torch.int32, device=dev)
        self.scores = torch.empty((B, N_v), dtype=torch.float32, device=dev) if want_scores else None
        need = lib().provip_prune_workspace_size(B, Lm, self.H_sel, self.N_t_max, N_v, algo, self.dtype)
        self.ws = ws if ws is not None and ws.numel() >= need else workspace(need, dev)

    def __call__(self, Q, K, V, hidden, pos, text_start, text_len, seq_len, vis_start,
                 row_mask=None, stream=None):
        B, Lm, Hq, Hkv, dh, D = self.shape
        P = pos.shape[0] if pos is not None else 0
        st = ctypes.c_void_p(stream.cuda_stream) if stream is not None else _stream(Q.device)
        hp = _ptr_host_ok if self.flags & PRUNE_HOST_ROWS else _ptr
        rc = lib().provip_prune(_ptr(Q), _ptr(K), hp(V), hp(hidden), B, Lm, Hq, Hkv, dh, D,
                                self.heads, self.H_sel, _i32(text_start), _i32(text_len),
                                _u8(row_mask), self.N_t_max, vis_start, self.N_v, _i32(seq_len),
                                _i32_host_ok(pos) if hp is _ptr_host_ok else _i32(pos), P, self.keep,
                                self.dtype, self.algo, hp(self.hidden_out), hp(self.K_out),
                                hp(self.V_out),
                                _i32_host_ok(self.pos_out) if hp is _ptr_host_ok else _i32(self.pos_out),
                                _ptr(self.idx), _i32(self.seq_len_out), _ptr(self.scores),
                                _ptr(self.ws), self.ws.numel(), self.flags, st)
        _check(rc, "provip_prune")
        return dict(hidden=self.hidden_out, K=self.K_out, V=self.V_out, pos=self.pos_out,
                    idx=self.idx, seq_len=self.seq_len_out, scores=self.scores)


def provip_prune(Q, K, V, hidden, pos, head_list, text_start, text_len, seq_len, vis_start, N_v,
                 keep, row_mask=None, algo=ALGO_AUTO, N_t_max=None):
    Ntm = int(N_t_max if N_t_max is not None else int(text_len.max().item()))
    step = PruneStep(Q, K, V, hidden, pos, head_list, Ntm, N_v, keep, algo)
    return step(Q, K, V, hidden, pos, text_start, text_len, seq_len, vis_start, row_mask)


def provip_head_topk(Q, K, head_list, text_start, text_len, seq_len, vis_start, N_v, keep,
                     row_mask=None, algo=ALGO_AUTO, N_t_max=None, ws=None, want_scores=True):
    B, Lm, Hq, dh = Q.shape
    Hkv = K.shape[2]
    dev = Q.device
    heads, hs = _heads_arg(head_list, Hq)
    Ntm = int(N_t_max if N_t_max is not None else int(text_len.max().item()))
    idx = torch.empty((B, keep), dtype=torch.int32, device=dev)
    scores = torch.empty((B, N_v), dtype=torch.float32, device=dev) if want_scores else None
    L = lib()
    dt = _dtype_code(Q)
    need = L.provip_head_scores_workspace_size(B, Lm, hs, Ntm, N_v, algo, dt)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    rc = L.provip_head_topk(_ptr(Q), _ptr(K), B, Lm, Hq, Hkv, dh, heads, hs, _i32(text_start),
                            _i32(text_len), _u8(row_mask), Ntm, vis_start, N_v, _i32(seq_len), keep, dt,
                            algo, _ptr(idx), _ptr(scores), _ptr(ws), ws.numel(), _stream(dev))
    _check(rc, "provip_head_topk")
    return idx, scores


def provip_head_scores_noalloc(Q, K, head_list, text_start, text_len, seq_len, vis_start, N_v,
                               row_mask=None, algo=ALGO_AUTO, N_t_max=None):
    """provip_head_scores without a workspace: the scratch is the library's own
    static device array (for hosts that cannot allocate device memory; shapes
    needing more than PROVIP_NOALLOC_SCRATCH_BYTES are rejected)."""
    B, Lm, Hq, dh = Q.shape
    Hkv = K.shape[2]
    dev = Q.device
    heads, hs = _heads_arg(head_list, Hq)
    Ntm = int(N_t_max if N_t_max is not None else int(text_len.max().item()))
    scores = torch.empty((B, N_v), dtype=torch.float32, device=dev)
    rc = lib().provip_head_scores_noalloc(_ptr(Q), _ptr(K), B, Lm, Hq, Hkv, dh, heads, hs, _i32(text_start),
                                          _i32(text_len), _u8(row_mask), Ntm, vis_start, N_v, _i32(seq_len),
                                          _dtype_code(Q), algo, _ptr(scores), _stream(dev))
    _check(rc, "provip_head_scores_noalloc")
    return scores


# ---------------------------------------------------------------------------
# visual-head identification (Sec. 4.4)
# ---------------------------------------------------------------------------
def provip_head_confidence(Q, K, text_start, text_len, seq_len, vis_start, N_v, N_vis,
                           crit_mask=None, algo=ALGO_AUTO, N_t_max=None, ws=None, want_conf=True):
    """Head confidence C [B, H_q] over the critical rows and the N_vis visual heads
    [B, N_vis] (ascending) of every sample. Returns (vis_heads, conf or None)."""
    B, Lm, Hq, dh = Q.shape
    Hkv = K.shape[2]
    dev = Q.device
    Ntm = int(N_t_max if N_t_max is not None else (crit_mask.shape[1] if crit_mask is not None
                                                   else int(text_len.max().item())))
    vis = torch.empty((B, N_vis), dtype=torch.int32, device=dev)
    conf = torch.empty((B, Hq), dtype=torch.float32, device=dev) if want_conf else None
    L = lib()
    dt = _dtype_code(Q)
    need = L.provip_visual_heads_workspace_size(B, Lm, Hq, Ntm, N_v, N_vis, algo, dt)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    rc = L.provip_head_confidence(_ptr(Q), _ptr(K), B, Lm, Hq, Hkv, dh, _i32(text_start),
                                  _i32(text_len), _u8(crit_mask), Ntm, vis_start, N_v, _i32(seq_len),
                                  N_vis, dt, algo, _ptr(conf), _ptr(vis), _ptr(ws), ws.numel(),
                                  _stream(dev))
    _check(rc, "provip_head_confidence")
    return vis, conf


class VisualHeadsPruneStep:
    """Pre-allocated outputs + workspace for repeated provip_prune_visual_heads calls."""

    def __init__(self, Q, K, V, hidden, pos, N_t_max, N_v, keep, N_vis, algo=ALGO_AUTO,
                 want_scores=True, want_conf=True, flags=0, ws=None, device=None):
        """Q, K, V, hidden, pos give the shapes and dtypes (meta tensors are fine
        with device=...)."""
        B, Lm, Hq, dh = Q.shape
        self.shape = (B, Lm, Hq, K.shape[2], dh, hidden.shape[2])
        self.N_t_max, self.N_v, self.keep, self.N_vis, self.algo = int(N_t_max), int(N_v), int(keep), int(N_vis), algo
        self.flags = int(flags)
        dev = Q.device if device is None else torch.device(device)
        self.dtype = _dtype_code(Q)
        L_out = Lm - N_v + keep
        self.hidden_out, self.K_out, self.V_out, self.pos_out = _outs(hidden, K, V, pos, B, L_out, dev)
        self.idx = torch.empty((B, keep), dtype=torch.int32, device=dev)
        self.seq_len_out = torch.empty(B, dtype=torch.int32, device=dev)
        self.scores = torch.empty((B, N_v), dtype=torch.float32, device=dev) if want_scores else None
        self.vis_heads = torch.empty((B, self.N_vis), dtype=torch.int32, device=dev)
        self.conf = torch.empty((B, Hq), dtype=torch.float32, device=dev) if want_conf else None
        need = lib().provip_visual_heads_workspace_size(B, Lm, Hq, self.N_t_max, N_v, self.N_vis, algo,
                                                        self.dtype)
        self.ws = ws if ws is not None and ws.numel() >= need else workspace(need, dev)

    def __call__(self, Q, K, V, hidden, pos, text_start, text_len, seq_len, vis_start,
                 crit_mask=None, stream=None):
        B, Lm, Hq, Hkv, dh, D = self.shape
        P = pos.shape[0] if pos is not None else 0
        st = ctypes.c_void_p(stream.cuda_stream) if stream is not None else _stream(Q.device)
        rc = lib().provip_prune_visual_heads(
            _ptr(Q), _ptr(K), _ptr(V), _ptr(hidden), B, Lm, Hq, Hkv, dh, D, _i32(text_start),
            _i32(text_len), _u8(crit_mask), self.N_t_max, vis_start, self.N_v, _i32(seq_len),
            _i32(pos), P, self.N_vis, self.keep, self.dtype, self.algo, _ptr(self.hidden_out),
            _ptr(self.K_out), _ptr(self.V_out), _i32(self.pos_out), _ptr(self.idx),
            _i32(self.seq_len_out), _ptr(self.scores), _ptr(self.vis_heads), _ptr(self.conf),
            _ptr(self.ws), self.ws.numel(), self.flags, st)
        _check(rc, "provip_prune_visual_heads")
        return dict(hidden=self.hidden_out, K=self.K_out, V=self.V_out, pos=self.pos_out,
                    idx=self.idx, seq_len=self.seq_len_out, scores=self.scores,
                    vis_heads=self.vis_heads, conf=self.conf)


def provip_prune_visual_heads(Q, K, V, hidden, pos, text_start, text_len, seq_len, vis_start, N_v,
                              keep, N_vis, crit_mask=None, algo=ALGO_AUTO, N_t_max=None):
    Ntm = int(N_t_max if N_t_max is not None else (crit_mask.shape[1] if crit_mask is not None
                                                   else int(text_len.max().item())))
    step = VisualHeadsPruneStep(Q, K, V, hidden, pos, Ntm, N_v, keep, N_vis, algo)
    return step(Q, K, V, hidden, pos, text_start, text_len, seq_len, vis_start, crit_mask)


# ---------------------------------------------------------------------------
# behind the pruning: attention over prompts, paged cache, decoding
# ---------------------------------------------------------------------------
def _rows(t, H, dtype, what):
    """pointer and row stride (elements) of a [T, H, 128] tensor whose heads lie next to each
    other; a slice of a fused query/key/value buffer is fine"""
    if not t.is_cuda:
        raise ProvipError(ERR_INVALID_ARG, "tensor must live on the GPU")
    if t.dtype is not dtype:
        raise ProvipError(ERR_INVALID_ARG, f"{what}: dtype {t.dtype}, not {dtype}")
    n, h, d = t.shape
    s0, s1, s2 = t.stride()
    if h != H or d != 128:
        raise ProvipError(ERR_INVALID_ARG, f"{what}: shape {tuple(t.shape)}, not [rows, {H}, 128]")
    if n and (s2 != 1 or (s1 != 128 and h > 1)):
        raise ProvipError(ERR_INVALID_ARG, f"{what}: the heads of a row must lie next to each other")
    return t.data_ptr(), (s0 if n > 1 else h * 128)


def _ints(t, n, what):
    if t.dtype is not torch.int32 or not t.is_cuda or not t.is_contiguous() or t.numel() < n:
        raise ProvipError(ERR_INVALID_ARG, f"{what} must be a contiguous int32 GPU tensor of {n} entries")
    return t.data_ptr()


def _dtype_of(dtype):
    if dtype is torch.bfloat16:
        return BF16
    if dtype is torch.float32:
        return F32
    raise ProvipError(ERR_UNSUPPORTED, f"unsupported dtype {dtype}")


class PromptAttention:
    """Pre-allocated outputs + workspace for repeated provip_prompt_attention calls (one shape):
    T_q query rows of B sequences, at most q_len_max rows and k_len_max own keys each, behind
    prefix_len shared keys. With T_q = B * L_max, q_start = b * L_max and the lengths of a
    pruning step it takes that step's padded layout."""

    def __init__(self, T_q, B, H_q, H_kv, q_len_max, k_len_max, prefix_len=0, causal=True, scale=None,
                 dtype=torch.bfloat16, device="cuda", algo=ALGO_AUTO, want_lse=True):
        self.shape = (int(T_q), int(B), int(H_q), int(H_kv), int(q_len_max), int(k_len_max), int(prefix_len))
        self.causal, self.algo, self.dtype, self._dt = int(bool(causal)), int(algo), dtype, _dtype_of(dtype)
        self.scale = 128 ** -0.5 if scale is None else float(scale)
        dev = torch.device(device)
        self.out = torch.empty((T_q, H_q, 128), dtype=dtype, device=dev)
        self.lse = torch.empty((T_q, H_q), dtype=torch.float32, device=dev) if want_lse else None
        self.ws = workspace(lib().provip_prompt_attention_workspace_size(*self.shape, self._dt, self.algo), dev)

    def __call__(self, Q, K, V, q_start, q_len, k_start, k_len, K_prefix=None, V_prefix=None):
        """Q [T_q, H_q, 128], K and V [T_k, H_kv, 128], the prefix's [prefix_len, H_kv, 128];
        starts and lengths int32 [B] on the device. Returns dict(out, lse)."""
        T_q, B, H_q, H_kv, qm, km, P = self.shape
        if Q.shape[0] != T_q or K.shape[0] != V.shape[0]:
            raise ProvipError(ERR_INVALID_ARG, "prompt_attention: Q, K or V has another number of rows")
        q, qs = _rows(Q, H_q, self.dtype, "Q")
        k, ks = _rows(K, H_kv, self.dtype, "K")
        v, vs = _rows(V, H_kv, self.dtype, "V")
        kp = vp = None
        kps = vps = 0
        if P:
            if K_prefix is None or V_prefix is None or K_prefix.shape[0] < P or V_prefix.shape[0] < P:
                raise ProvipError(ERR_INVALID_ARG, f"prompt_attention: the prefix needs {P} rows")
            kp, kps = _rows(K_prefix, H_kv, self.dtype, "K_prefix")
            vp, vps = _rows(V_prefix, H_kv, self.dtype, "V_prefix")
        rc = lib().provip_prompt_attention(
            q, qs, k, ks, v, vs, T_q, K.shape[0], B, H_q, H_kv, 128, _ints(q_start, B, "q_start"),
            _ints(q_len, B, "q_len"), _ints(k_start, B, "k_start"), _ints(k_len, B, "k_len"), qm, km, kp, kps, vp, vps, P,
            self.causal, self.scale, self._dt, self.algo, self.out.data_ptr(), H_q * 128,
            None if self.lse is None else self.lse.data_ptr(), self.ws.data_ptr(), self.ws.numel(), _stream(Q.device))
        _check(rc, "provip_prompt_attention")
        return dict(out=self.out, lse=self.lse)


def provip_prompt_attention(Q, K, V, q_start, q_len, k_start, k_len, q_len_max, k_len_max, K_prefix=None,
                            V_prefix=None, causal=True, scale=None, algo=ALGO_AUTO, want_lse=True):
    """One call of PromptAttention, its outputs and workspace allocated here."""
    step = PromptAttention(Q.shape[0], q_len.numel(), Q.shape[1], K.shape[1], q_len_max, k_len_max,
                           0 if K_prefix is None else K_prefix.shape[0], causal, scale, Q.dtype, Q.device, algo, want_lse)
    return step(Q, K, V, q_start, q_len, k_start, k_len, K_prefix, V_prefix)


class PageTables:
    """Pre-allocated outputs for repeated provip_page_tables calls: B requests, pages of
    page_size rows, at most T_max new tokens a step."""

    def __init__(self, B, page_size, T_max, device="cuda"):
        dev = torch.device(device)
        self.B, self.page_size, self.T_max = int(B), int(page_size), int(T_max)
        self.kv_len = torch.empty(B, dtype=torch.int32, device=dev)
        self.row_start = torch.empty(B + 1, dtype=torch.int32, device=dev)
        self.slot_map = torch.empty(T_max, dtype=torch.int32, device=dev)
        self.free_count = torch.empty(1, dtype=torch.int32, device=dev)

    def __call__(self, kv_len, new_len, free_pages, free_count, block_table, inplace=False):
        """kv_len, new_len [B], free_pages (the stack) and block_table [B, max_pages] (both updated),
        free_count [1]: int32 on the device. inplace: kv_len and free_count are updated too instead
        of leaving the new ones in self. Returns dict(kv_len, row_start, slot_map, free_count)."""
        B = self.B
        kv_out, fc_out = (kv_len, free_count) if inplace else (self.kv_len, self.free_count)
        if block_table.dim() != 2 or block_table.shape[0] != B:
            raise ProvipError(ERR_INVALID_ARG, f"block_table must be [{B}, max_pages]")
        rc = lib().provip_page_tables(
            _ints(kv_len, B, "kv_len"), _ints(new_len, B, "new_len"), B, self.page_size,
            _ints(free_pages, 0, "free_pages"), free_pages.numel(), _ints(free_count, 1, "free_count"),
            _ints(block_table, 0, "block_table"), block_table.shape[1], self.T_max, kv_out.data_ptr(),
            self.row_start.data_ptr(), self.slot_map.data_ptr(), fc_out.data_ptr(), _stream(kv_len.device))
        _check(rc, "provip_page_tables")
        return dict(kv_len=kv_out, row_start=self.row_start, slot_map=self.slot_map, free_count=fc_out)


def _pages(t, dtype, what):
    if not t.is_cuda or not t.is_contiguous() or t.dim() != 4 or t.dtype is not dtype:
        raise ProvipError(ERR_INVALID_ARG, f"{what} must be a contiguous {dtype} GPU tensor [n_pages, page_size, H_kv, d_h]")
    return t.data_ptr()


def provip_kv_append(K, V, slot_map, k_pages, v_pages):
    """Rows of K and V [T, H_kv, d_h] into the slots slot_map [T] of k_pages and v_pages
    [n_pages, page_size, H_kv, d_h]; negative slots are skipped."""
    dtype = K.dtype
    kp, vp = _pages(k_pages, dtype, "k_pages"), _pages(v_pages, dtype, "v_pages")
    T, H, d = K.shape
    pages = k_pages.shape
    if V.shape != K.shape or V.dtype is not dtype or pages[2] != H or pages[3] != d or v_pages.shape != pages:
        raise ProvipError(ERR_INVALID_ARG, "kv_append: K, V and the pages must agree in shape and dtype")
    if not (K.is_cuda and V.is_cuda):
        raise ProvipError(ERR_INVALID_ARG, "tensor must live on the GPU")
    k0, k1, k2 = K.stride()
    v0, v1, v2 = V.stride()
    if T and (k2 != 1 or v2 != 1 or (H > 1 and (k1 != d or v1 != d))):
        raise ProvipError(ERR_INVALID_ARG, "kv_append: the heads of a row must lie next to each other")
    if T <= 1:
        k0 = v0 = H * d
    rc = lib().provip_kv_append(K.data_ptr(), k0, V.data_ptr(), v0, T, H, d, _ints(slot_map, T, "slot_map"), pages[0],
                                pages[1], _dtype_of(dtype), kp, vp, _stream(K.device))
    _check(rc, "provip_kv_append")


class DecodeAttention:
    """Pre-allocated outputs + workspace for repeated provip_decode_attention calls: one token of
    B requests, each behind prefix_len shared tokens and at most kv_len_max of its own."""

    def __init__(self, B, H_q, H_kv, kv_len_max, prefix_len=0, scale=None, dtype=torch.bfloat16, device="cuda",
                 algo=ALGO_AUTO, want_lse=True):
        self.shape = (int(B), int(H_q), int(H_kv), int(kv_len_max), int(prefix_len))
        self.algo, self.dtype, self._dt = int(algo), dtype, _dtype_of(dtype)
        self.scale = 128 ** -0.5 if scale is None else float(scale)
        dev = torch.device(device)
        self.out = torch.empty((B, H_q, 128), dtype=dtype, device=dev)
        self.lse = torch.empty((B, H_q), dtype=torch.float32, device=dev) if want_lse else None
        self.ws = workspace(lib().provip_decode_attention_workspace_size(*self.shape, self._dt, self.algo), dev)

    def __call__(self, Q, k_pages, v_pages, block_table, kv_len, prefix_table=None):
        """Q [B, H_q, 128]; k_pages, v_pages [n_pages, page_size, H_kv, 128]; block_table
        [B, max_pages], kv_len [B] and the prefix's pages int32 on the device. Returns dict(out, lse)."""
        B, H_q, H_kv, km, P = self.shape
        if Q.shape[0] != B or block_table.dim() != 2 or block_table.shape[0] != B:
            raise ProvipError(ERR_INVALID_ARG, f"decode_attention: Q and block_table must have {B} rows")
        if k_pages.shape[2:] != (H_kv, 128) or v_pages.shape != k_pages.shape:
            raise ProvipError(ERR_INVALID_ARG, f"decode_attention: pages must be [n_pages, page_size, {H_kv}, 128]")
        q, qs = _rows(Q, H_q, self.dtype, "Q")
        if P and prefix_table is None:
            raise ProvipError(ERR_INVALID_ARG, "decode_attention: the prefix needs its pages' table")
        ps = k_pages.shape[1]
        rc = lib().provip_decode_attention(
            q, qs, B, H_q, H_kv, 128, _pages(k_pages, self.dtype, "k_pages"), _pages(v_pages, self.dtype, "v_pages"),
            k_pages.shape[0], ps, _ints(block_table, 0, "block_table"), block_table.shape[1], _ints(kv_len, B, "kv_len"),
            km, _ints(prefix_table, -(-P // ps), "prefix_table") if P else None, P, self.scale, self._dt, self.algo,
            self.out.data_ptr(), H_q * 128, None if self.lse is None else self.lse.data_ptr(), self.ws.data_ptr(),
            self.ws.numel(), _stream(Q.device))
        _check(rc, "provip_decode_attention")
        return dict(out=self.out, lse=self.lse)


def provip_decode_attention(Q, k_pages, v_pages, block_table, kv_len, kv_len_max, prefix_table=None, prefix_len=0,
                            scale=None, algo=ALGO_AUTO, want_lse=True):
    """One call of DecodeAttention, its outputs and workspace allocated here."""
    step = DecodeAttention(Q.shape[0], Q.shape[1], k_pages.shape[2], kv_len_max, prefix_len, scale, Q.dtype, Q.device,
                           algo, want_lse)
    return step(Q, k_pages, v_pages, block_table, kv_len, prefix_table)


# ---------------------------------------------------------------------------
# position rotation, and a cache held in 4 bits
# ---------------------------------------------------------------------------
ROW4 = 72  # bytes of a head's row of 128 values in 4 bits: 64 of codes, 8 of scales


class Rotary:
    """What a model's position rotation goes by: inv_freq, the 64 pairs' frequencies in radians a
    position (default base^(-i/64)), axis, the axis of position ids that each pair turns with
    (default: the first), or sections, the numbers of pairs that turn with each axis in order
    (such as (16, 24, 24) for time, height and width), and factor, by which rotated queries and
    keys are multiplied. Held on the host: one object serves every device and stream. Its values stay as
    they are made (calls, and graphs of them, hold what they were given): another plan is another object."""

    def __init__(self, inv_freq=None, axis=None, sections=None, base=10000.0, factor=1.0):
        freq = [float(base) ** (-i / 64) for i in range(64)] if inv_freq is None else \
            [float(f) for f in (inv_freq.tolist() if hasattr(inv_freq, "tolist") else inv_freq)]
        if axis is not None and sections is not None:
            raise ProvipError(ERR_INVALID_ARG, "Rotary: axis or sections, not both")
        if sections is not None:
            axis = [a for a, n in enumerate(sections) for _ in range(n)]
        axis = [0] * 64 if axis is None else [int(a) for a in (axis.tolist() if hasattr(axis, "tolist") else axis)]
        if len(freq) != 64 or len(axis) != 64 or min(axis) < 0:
            raise ProvipError(ERR_INVALID_ARG, "Rotary: 64 frequencies and 64 axes from 0 on, one a pair")
        n_axes, factor, inv_freq, axis = max(axis) + 1, float(factor), (ctypes.c_double * 64)(*freq), (ctypes.c_int * 64)(*axis)
        self.__dict__.update(n_axes=n_axes, factor=factor, inv_freq=inv_freq, axis=axis, args=(n_axes, inv_freq, axis, factor))

    def __setattr__(self, name, value):
        raise ProvipError(ERR_INVALID_ARG, f"Rotary: {name} is set when it is made")

    def __reduce__(self):  # (copies and pickles: with arrays of their own)
        return Rotary, (list(self.inv_freq), list(self.axis), None, 1.0, self.factor)


# (The checks below look at each property of a tensor once, and at its device by number: a property takes
# 0.1 to 0.2 us, and a call has up to nine tensors and 8 us on the GPU's side.)
_raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _dims(what, *tensors):
    """the refusal of tensors whose sizes could not even be taken apart (the others are refused one by one)"""
    return ProvipError(ERR_INVALID_ARG, f"{what}: rows must be [T, H, 128], pages three- or four-dimensional: got " +
                       " and ".join(str(list(t.shape)) for t in tensors))


def _heads(t, T, H, dtype, dev, what):
    """pointer and row stride (elements) of rows [T, H, 128] as _rows takes them, on device number dev"""
    if t.dtype is not dtype or t.get_device() != dev or dev < 0 or t.shape != (T, H, 128):
        raise ProvipError(ERR_INVALID_ARG, f"{what} must be {dtype} [{T}, {H}, 128] on GPU {dev}: got {t.dtype} {list(t.shape)} on {t.device}")
    s0, s1, s2 = t.stride()
    if (s2 != 1 or (s1 != 128 and H > 1)) and T:
        raise ProvipError(ERR_INVALID_ARG, f"{what}: the heads of a row must lie next to each other")
    return t.data_ptr(), (s0 if T > 1 else H * 128)


def _norm(w, dtype, dev, what):
    if w is None:
        return None
    if w.dtype is not dtype or w.get_device() != dev or w.numel() != 128 or not w.is_contiguous():
        raise ProvipError(ERR_INVALID_ARG, f"{what} must be a contiguous {dtype} tensor of 128 entries on GPU {dev}")
    return w.data_ptr()


def _positions(pos, T, n_axes, dev):
    """pointer and axis stride of position ids [axes, T] (or [axes, B, L] with T = B L)"""
    if pos.dim() == 3 and pos.is_contiguous():
        pos = pos.view(pos.shape[0], -1)
    shape, stride = pos.shape, pos.stride()
    if pos.dtype is not torch.int32 or pos.get_device() != dev or len(shape) != 2 or shape[0] < n_axes or shape[1] != T or \
            (T > 1 and stride[1] != 1):
        raise ProvipError(ERR_INVALID_ARG, f"pos must be an int32 tensor of at least {n_axes} axes by {T} rows on GPU {dev}")
    # (one axis alone may have any stride)
    return pos.data_ptr(), stride[0] if n_axes > 1 and T > 0 else T


def _index(t, n, dev, what):
    if t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous() or t.numel() < n:
        raise ProvipError(ERR_INVALID_ARG, f"{what} must be a contiguous int32 tensor of {n} entries on GPU {dev}")
    return t.data_ptr()


def _call(dev, what, call, *args):
    """a library call with its tensors' device current, whichever the caller's is, on that device's stream"""
    if dev == _raw_device():
        rc = call(*args, _raw_stream(dev) if _raw_stream is not None else _stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = call(*args, _stream(dev))
    if rc != OK:
        _check(rc, what)


def _rotate_args(Q, K, pos, rotary, q_norm, k_norm, eps, n_rows, q_out, k_out):
    """the arguments that the rotating calls share: inputs, what goes by positions, outputs, their device"""
    try:
        dtype, dev, (T, H_q, _), H = Q.dtype, Q.get_device(), Q.shape, K.shape[1]
    except (ValueError, IndexError):
        raise _dims("rotate", Q, K) from None
    q, qs = _heads(Q, T, H_q, dtype, dev, "Q")
    k, ks = _heads(K, T, H, dtype, dev, "K")
    qo, qos = _heads(q_out, T, H_q, dtype, dev, "q_out")
    ko, kos = (None, 0) if k_out is None else _heads(k_out, T, H, dtype, dev, "k_out")
    p, ps = _positions(pos, T, rotary.n_axes, dev)
    by = (None if n_rows is None else _index(n_rows, 1, dev, "n_rows"), H_q, H, 128, p, ps, *rotary.args,
          _norm(q_norm, dtype, dev, "q_norm"), _norm(k_norm, dtype, dev, "k_norm"), eps, _dtype_of(dtype))
    return (q, qs, k, ks), by, (qo, qos, ko, kos), dev


def provip_rotate(Q, K, pos, rotary, q_norm=None, k_norm=None, eps=1e-6, out=None, n_rows=None):
    """Norms (where given, [128]) and rotation of Q [T, H_q, 128] and K [T, H_kv, 128] by the position
    ids pos [axes, T] (or a compaction's [axes, B, L]). out: (q_out, k_out) to write, which may be (Q, K)
    themselves; n_rows: device count of rows (such as row_start[B:]), past which rows are left untouched.
    Returns (q_out, k_out)."""
    q_out, k_out = out if out is not None else (Q.new_empty(Q.shape), K.new_empty(K.shape))
    ins, by, outs, dev = _rotate_args(Q, K, pos, rotary, q_norm, k_norm, eps, n_rows, q_out, k_out)
    _call(dev, "provip_rotate", lib().provip_rotate, *ins, Q.shape[0], *by, *outs)
    return q_out, k_out


def pages4(n_pages, page_size, H_kv, device="cuda"):
    """A pool of 4-bit pages [n_pages, H_kv, page_size * 72] bytes, whose rows stand for zeros."""
    return torch.zeros(n_pages, H_kv, page_size * ROW4, dtype=torch.uint8, device=device)


def _pages4(k_pages, v_pages, H, dev):
    """pointers of two 4-bit pools, their pages and rows a page"""
    shape = k_pages.shape
    for t in (k_pages, v_pages):
        if t.dtype is not torch.uint8 or t.get_device() != dev or dev < 0 or t.shape != shape or len(shape) != 3 or shape[1] != H or \
                shape[2] % ROW4 or not t.is_contiguous():
            raise ProvipError(ERR_INVALID_ARG, f"4-bit pages must be contiguous uint8 tensors [n_pages, {H}, page_size * {ROW4}] on GPU {dev}")
    return k_pages.data_ptr(), v_pages.data_ptr(), shape[0], shape[2] // ROW4


def provip_rotate_append(Q, K, V, pos, rotary, slot_map, k_pages, v_pages, q_norm=None, k_norm=None, eps=1e-6, out=None,
                         want_k=False, n_rows=None):
    """provip_rotate, with the rotated keys and the values V [T, H_kv, 128] into the slots slot_map [T] of
    pages on the way: [n_pages, page_size, H_kv, 128] of the rows' type, or 4-bit ones (uint8, see pages4).
    out: (q_out, k_out or None) to write. Returns (q_out, k_out), the latter None unless given or want_k."""
    q_out, k_out = out if out is not None else (Q.new_empty(Q.shape), K.new_empty(K.shape) if want_k else None)
    ins, by, outs, dev = _rotate_args(Q, K, pos, rotary, q_norm, k_norm, eps, n_rows, q_out, k_out)
    T, H, dtype = Q.shape[0], K.shape[1], Q.dtype
    v, vs = _heads(V, T, H, dtype, dev, "V")
    four = k_pages.dtype is torch.uint8
    if four:
        kp, vp, n, ps = _pages4(k_pages, v_pages, H, dev)
    else:
        kp, vp = _pages(k_pages, dtype, "k_pages"), _pages(v_pages, dtype, "v_pages")
        n, ps = k_pages.shape[:2]  # (four dimensions: checked there)
        if k_pages.shape[2:] != (H, 128) or v_pages.shape != k_pages.shape or k_pages.get_device() != dev or v_pages.get_device() != dev:
            raise ProvipError(ERR_INVALID_ARG, f"rotate_append: pages must be [n_pages, page_size, {H}, 128] on GPU {dev}")
    _call(dev, "provip_rotate_append", lib().provip_rotate_append, *ins, v, vs, T, *by, *outs, _index(slot_map, T, dev, "slot_map"), n,
          ps, int(four), kp, vp)
    return q_out, k_out


def provip_kv_append4(K, V, slot_map, k_pages, v_pages):
    """Rows of K and V [T, H_kv, 128] into the slots slot_map [T] of 4-bit pages (uint8, see pages4);
    negative slots are skipped."""
    try:
        (T, H, _), dtype, dev = K.shape, K.dtype, K.get_device()
    except ValueError:
        raise _dims("kv_append4", K) from None
    k, ks = _heads(K, T, H, dtype, dev, "K")
    v, vs = _heads(V, T, H, dtype, dev, "V")
    kp, vp, n, ps = _pages4(k_pages, v_pages, H, dev)
    _call(dev, "provip_kv_append4", lib().provip_kv_append4, k, ks, v, vs, T, H, 128, _index(slot_map, T, dev, "slot_map"), n, ps,
          _dtype_of(dtype), kp, vp)


def provip_kv_read4(slot_map, k_pages, v_pages, dtype=torch.bfloat16, out=None):
    """What the rows at the slots slot_map [T] of 4-bit pages stand for: K and V [T, H_kv, 128]. out: (K, V)
    to write, whose type counts then; rows of a negative slot are left untouched (zeros, unless out is given)."""
    if k_pages.dim() != 3:
        raise _dims("kv_read4", k_pages)
    T, H, dev = slot_map.numel(), k_pages.shape[1], k_pages.get_device()
    if out is None:
        out = tuple(torch.zeros(T, H, 128, dtype=dtype, device=k_pages.device) for _ in range(2))
    k_out, v_out = out
    dtype = k_out.dtype
    k, ks = _heads(k_out, T, H, dtype, dev, "K")
    v, vs = _heads(v_out, T, H, dtype, dev, "V")
    kp, vp, n, ps = _pages4(k_pages, v_pages, H, dev)
    _call(dev, "provip_kv_read4", lib().provip_kv_read4, _index(slot_map, T, dev, "slot_map"), T, H, 128, kp, vp, n, ps,
          _dtype_of(dtype), k, ks, v, vs)
    return k_out, v_out


class DecodeAttention4:
    """Pre-allocated outputs + workspace for repeated provip_decode_attention4 calls: DecodeAttention
    over 4-bit pages (uint8, see pages4). dtype: of the queries and the output."""

    def __init__(self, B, H_q, H_kv, kv_len_max, prefix_len=0, scale=None, dtype=torch.bfloat16, device="cuda", want_lse=True):
        self.shape = (int(B), int(H_q), int(H_kv), int(kv_len_max), int(prefix_len))
        self.dtype, self._dt = dtype, _dtype_of(dtype)
        self.scale = 128 ** -0.5 if scale is None else float(scale)
        dev = torch.device(device)
        self.out = torch.empty((B, H_q, 128), dtype=dtype, device=dev)
        self.lse = torch.empty((B, H_q), dtype=torch.float32, device=dev) if want_lse else None
        self.ws = workspace(lib().provip_decode_attention4_workspace_size(*self.shape, self._dt), dev)

    def __call__(self, Q, k_pages, v_pages, block_table, kv_len, prefix_table=None):
        """Q [B, H_q, 128]; k_pages, v_pages [n_pages, H_kv, page_size * 72] bytes; block_table
        [B, max_pages], kv_len [B] and the prefix's pages int32 on the device. Returns dict(out, lse)."""
        B, H_q, H_kv, km, P = self.shape
        dev = self.out.get_device()
        q, qs = _heads(Q, B, H_q, self.dtype, dev, "Q")
        kp, vp, n, ps = _pages4(k_pages, v_pages, H_kv, dev)
        table = block_table.shape
        if len(table) != 2 or table[0] != B:
            raise ProvipError(ERR_INVALID_ARG, f"decode_attention4: block_table must have {B} rows")
        if P and prefix_table is None:
            raise ProvipError(ERR_INVALID_ARG, "decode_attention4: the prefix needs its pages' table")
        _call(dev, "provip_decode_attention4", lib().provip_decode_attention4, q, qs, B, H_q, H_kv, 128, kp, vp, n, ps,
              _index(block_table, 0, dev, "block_table"), table[1], _index(kv_len, B, dev, "kv_len"), km,
              _index(prefix_table, -(-P // ps), dev, "prefix_table") if P else None, P, self.scale, self._dt,
              self.out.data_ptr(), H_q * 128, None if self.lse is None else self.lse.data_ptr(), self.ws.data_ptr(), self.ws.numel())
        return dict(out=self.out, lse=self.lse)


def provip_decode_attention4(Q, k_pages, v_pages, block_table, kv_len, kv_len_max, prefix_table=None, prefix_len=0,
                             scale=None, want_lse=True):
    """One call of DecodeAttention4, its outputs and workspace allocated here."""
    if Q.dim() != 3 or k_pages.dim() != 3:
        raise _dims("decode_attention4", Q, k_pages)
    step = DecodeAttention4(Q.shape[0], Q.shape[1], k_pages.shape[1], kv_len_max, prefix_len, scale, Q.dtype, Q.device, want_lse)
    return step(Q, k_pages, v_pages, block_table, kv_len, prefix_table)
