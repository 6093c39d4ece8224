"""Thin Python binding of libssd's C ABI (argument marshalling only).

Every function here takes torch tensors that already live on the CUDA device, passes their
addresses to the C entry point of the same name and returns the output tensors; all
computation happens in the library's CUDA kernels.  There is no CPU fallback: importing this
module without a built libssd.so, or calling it with host tensors, raises.

The calls of a decoding step, with result buffers given and no launch options, are marshalled by
_ssd_call (csrc/ssd_call.cpp); whatever it does not take -- it answers None -- goes the general way
through ctypes, which is also where wrong arguments are named.  Without _ssd_call.so, or with one
built for another torch, every call goes that way.
"""
import ctypes as C
import os
import warnings
from typing import Callable, Dict, List, Optional

import torch

from . import build as _build

F32, BF16, F16 = 0, 1, 2
UTT_NONFINITE, UTT_BAD_DRAFT_ID, UTT_BAD_OFFSETS, UTT_INTERNAL = 1, 2, 4, 0x80000000
UTT_BAD_PARENT, UTT_BAD_CACHE, UTT_CACHE_FULL = 8, 16, 32
OK, ERR_NULL, ERR_ARG, ERR_DTYPE, ERR_WORKSPACE, ERR_CUDA, ERR_ALIGN, ERR_TOO_LARGE = range(8)
VERIFY_STATIC_SCRATCH_BYTES = 8 << 20

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libssd.so")


class SsdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().ssd_status_string(code).decode()
        if code == ERR_CUDA:
            msg += " (cudaError %d)" % lib().ssd_last_cuda_error()
        super().__init__("%s: %s" % (where, msg))


class LaunchOpts(C.Structure):
    """Mirror of ssd_launch_opts (include/ssd.h)."""
    _fields_ = [("kernel", C.c_int32), ("ctas", C.c_int32), ("warps", C.c_int32),
                ("stages", C.c_int32), ("stage_bytes", C.c_int32), ("split", C.c_int32),
                ("ev_begin", C.c_void_p), ("ev_end", C.c_void_p), ("fma_exp", C.c_int32),
                ("finish", C.c_int32)]


class Heads(C.Structure):
    """Mirror of ssd_heads (include/ssd.h)."""
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("heads", C.c_int32)]


class KvCache(C.Structure):
    """Mirror of ssd_kv_cache (include/ssd.h)."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("head_stride", C.c_int64), ("pages", C.c_int32), ("page_size", C.c_int32), ("heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int), ("max_pages", C.c_int32), ("page_table", C.c_void_p),
                ("table_stride", C.c_int64), ("len", C.c_void_p)]


_lib = None
_call = None


class _Declines:
    """In the place of a _ssd_call that cannot be used: every call goes the general way."""
    def __getattr__(self, name):
        return lambda *args: None


def _native():
    global _call
    if _call is None:
        lib()
        try:
            from . import _ssd_call as call
            want = "_ssd_call for " + _build.built_for()
            if call.built_for != want:
                raise ImportError("it is %r, not %r" % (call.built_for, want))
        except ImportError as e:
            warnings.warn("_ssd_call.so cannot be used (%s): calls are marshalled through ctypes, which takes "
                          "several times longer; run `python -m paper_2603_11243_b200.build`" % e, RuntimeWarning)
            call = _Declines()
        _call = call
    return _call


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                "libssd.so is not built: run `python -m paper_2603_11243_b200.build` "
                "(needs nvcc); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        L.ssd_status_string.restype = C.c_char_p
        L.ssd_status_string.argtypes = [C.c_int32]
        L.ssd_last_cuda_error.restype = C.c_int32
        L.ssd_version.restype = C.c_int32
        L.ssd_launch_count.restype = C.c_uint64
        for f in (L.ssd_ctc_draft_workspace_bytes, L.ssd_verify_workspace_bytes):
            f.restype = C.c_size_t
            f.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int, C.c_void_p]
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.ssd_ctc_draft.restype = i32
        L.ssd_ctc_draft.argtypes = [vp, C.c_int, i32, i64, vp, i32, i64, i32, i32,
                                    vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                    vp, C.c_size_t, vp, vp]
        L.ssd_entropy_gate.restype = i32
        L.ssd_entropy_gate.argtypes = [vp, vp, i32, i64, C.c_float, vp, vp, vp, vp, vp, vp]
        L.ssd_verify.restype = i32
        L.ssd_verify.argtypes = [vp, C.c_int, i32, i64, vp, vp, i32, i64, C.c_float, vp,
                                 vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        L.ssd_verify_static.restype = i32
        L.ssd_verify_static.argtypes = [vp, C.c_int, i32, i64, vp, vp, i32, i64, C.c_float, vp,
                                        vp, vp, vp, vp, vp, vp, vp]
        L.ssd_verify_early_exit_workspace_bytes.restype = C.c_size_t
        L.ssd_verify_early_exit_workspace_bytes.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int, C.c_void_p]
        L.ssd_verify_early_exit.restype = i32
        L.ssd_verify_early_exit.argtypes = [vp, C.c_int, i32, i64, vp, vp, i32, i64, C.c_float, vp,
                                            vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        for f in (L.ssd_ctc_draft_read_span, L.ssd_verify_read_span):
            f.restype = i32
        L.ssd_ctc_draft_read_span.argtypes = [C.c_uint64, C.c_int, i32, i64, i64, vp, vp]
        L.ssd_verify_read_span.argtypes = [C.c_uint64, C.c_int, i32, i64, i64, i32, vp, vp]
        L.ssd_verify_shard.restype = i32
        L.ssd_verify_shard.argtypes = [vp, C.c_int, i32, i64, i64, vp, vp, i32, i64, vp, vp, vp,
                                       C.c_size_t, vp, vp]
        L.ssd_verify_combine.restype = i32
        L.ssd_verify_combine.argtypes = [vp, i32, i64, vp, vp, i32, i64, C.c_float, vp, vp, vp, vp,
                                         vp, vp, vp]
        L.ssd_threshold_sweep.restype = i32
        L.ssd_threshold_sweep.argtypes = [vp, vp, vp, i32, i64, vp, vp, i32, vp, vp, vp, vp, vp]
        L.ssd_assemble.restype = i32
        L.ssd_assemble.argtypes = [vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ssd_greedy_step_workspace_bytes.restype = C.c_size_t
        L.ssd_greedy_step_workspace_bytes.argtypes = [i64, i32, C.c_int, vp]
        L.ssd_greedy_step.restype = i32
        L.ssd_greedy_step.argtypes = [vp, C.c_int, i32, i64, i64, vp, vp, vp, vp, vp, C.c_size_t,
                                      vp, vp]
        L.ssd_tree_attention.restype = i32
        L.ssd_tree_attention.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, i32, C.c_float, C.c_float, vp, vp, vp,
                                         vp, C.c_size_t, vp]
        L.ssd_tree_attention_workspace_bytes.restype = C.c_size_t
        L.ssd_tree_attention_workspace_bytes.argtypes = [i32, i32, i32, i64, i32]
        L.ssd_verify_tree.restype = i32
        L.ssd_verify_tree.argtypes = [vp, C.c_int, i32, i64, vp, vp, vp, i32, i64, C.c_float, vp,
                                      vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        L.ssd_cache_append.restype = i32
        L.ssd_cache_append.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, vp, i64, i32, vp, vp, vp]
        L.ssd_cache_weights.restype = i32
        L.ssd_cache_weights.argtypes = [vp, vp, vp, vp, i32, i64, i32, C.c_float, C.c_float, vp, vp, i64, i32, vp, vp]
        L.ssd_cache_evict.restype = i32
        L.ssd_cache_evict.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, i64, vp, vp, vp]
        _lib = L
    return _lib


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("logits must be float32 or bfloat16, got %s" % t.dtype)


def _dev(t: Optional[torch.Tensor], name: str):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor: libssd has no host path" % name)
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _opts(o: Optional[LaunchOpts]):
    return None if o is None else C.cast(C.pointer(o), C.c_void_p)


def _rows_ld(logits: torch.Tensor):
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be a 2-D row-major matrix (unit stride along the vocabulary)")
    return logits.shape[0], (logits.stride(0) if logits.shape[0] > 1 else max(logits.stride(0), logits.shape[1]))


def ssd_ctc_draft_workspace_bytes(B, N, V, dtype_code, opts=None) -> int:
    return int(lib().ssd_ctc_draft_workspace_bytes(B, N, V, dtype_code, _opts(opts)))


def ssd_verify_workspace_bytes(B, M, V, dtype_code, opts=None) -> int:
    return int(lib().ssd_verify_workspace_bytes(B, M, V, dtype_code, _opts(opts)))


class ReadSpan(C.Structure):
    """Mirror of ssd_read_span (include/ssd.h)."""
    _fields_ = [("lo", C.c_uint64), ("hi", C.c_uint64), ("faults", C.c_int64),
                ("kernel", C.c_int32), ("direct", C.c_int32)]


def ssd_ctc_draft_read_span(base_addr: int, dtype_code: int, V: int, ld: int, N: int,
                            opts: Optional[LaunchOpts] = None) -> ReadSpan:
    """Host-only: the addresses ssd_ctc_draft's streaming kernel would read (see ssd.h)."""
    out = ReadSpan()
    rc = lib().ssd_ctc_draft_read_span(base_addr, dtype_code, V, ld, N, _opts(opts),
                                       C.cast(C.pointer(out), C.c_void_p))
    if rc != OK:
        raise SsdError(rc, "ssd_ctc_draft_read_span")
    return out


def ssd_verify_read_span(base_addr: int, dtype_code: int, V: int, ld: int, M: int, B: int = 1,
                         opts: Optional[LaunchOpts] = None) -> ReadSpan:
    """Host-only: the addresses ssd_verify's streaming kernel would read (see ssd.h)."""
    out = ReadSpan()
    rc = lib().ssd_verify_read_span(base_addr, dtype_code, V, ld, M, B, _opts(opts),
                                    C.cast(C.pointer(out), C.c_void_p))
    if rc != OK:
        raise SsdError(rc, "ssd_verify_read_span")
    return out


def alloc_ctc_outputs(N: int, B: int, device, logprob_ld: int = 0) -> Dict[str, torch.Tensor]:
    e = lambda n, dt: torch.empty((n,), dtype=dt, device=device)
    # ssd_ctc_draft_workspace_bytes is 2048 whatever the sizes are (the tile counters)
    out = dict(workspace=torch.empty((2048,), dtype=torch.uint8, device=device),
               frame_entropy=e(N, torch.float32), frame_argmax=e(N, torch.int32),
               frame_lse=e(N, torch.float32), draft_tokens=e(N, torch.int32),
               draft_frames=e(N, torch.int32), draft_len=e(B, torch.int32),
               draft_full_len=e(B, torch.int32), utt_max_entropy=e(B, torch.float32),
               utt_status=e(B, torch.int32))
    if logprob_ld:
        out["frame_logprob"] = torch.empty((N, logprob_ld), dtype=torch.float32, device=device)
    return out


def ssd_ctc_draft(logits: torch.Tensor, frame_off: torch.Tensor, blank_id: int,
                  max_draft_len: int, V: Optional[int] = None, out=None, want_logprob=False,
                  opts: Optional[LaunchOpts] = None) -> Dict[str, torch.Tensor]:
    """Stage 1 (Section 2.1, Eq. 2, Eq. 3): frame statistics and the collapsed draft."""
    if out is not None and opts is None:
        rc = (_call or _native()).ctc_draft(logits, frame_off, blank_id, max_draft_len, V, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_ctc_draft")
    N, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = frame_off.shape[0] - 1
    if frame_off.dtype != torch.int64:
        raise TypeError("frame_off must be int64")
    if out is None:
        out = alloc_ctc_outputs(N, B, logits.device, ld if want_logprob else 0)
    ws = out.get("workspace")
    rc = lib().ssd_ctc_draft(
        _dev(logits, "logits"), _dtype_code(logits), V, ld, _dev(frame_off, "frame_off"), B, N,
        blank_id, max_draft_len, _dev(out["frame_entropy"], "frame_entropy"),
        _dev(out["frame_argmax"], "frame_argmax"), _dev(out.get("frame_lse"), "frame_lse"),
        _dev(out.get("frame_logprob"), "frame_logprob"),
        _dev(out["draft_tokens"], "draft_tokens"), _dev(out.get("draft_frames"), "draft_frames"),
        _dev(out["draft_len"], "draft_len"), _dev(out["draft_full_len"], "draft_full_len"),
        _dev(out["utt_max_entropy"], "utt_max_entropy"), _dev(out["utt_status"], "utt_status"),
        _dev(ws, "workspace"), 0 if ws is None else ws.numel(), _stream(), _opts(opts))
    if rc != OK:
        raise SsdError(rc, "ssd_ctc_draft")
    return out


def alloc_gate_outputs(B: int, device) -> Dict[str, torch.Tensor]:
    return dict(gate_accept=torch.empty((B,), dtype=torch.uint8, device=device),
                max_entropy=torch.empty((B,), dtype=torch.float32, device=device),
                argmax_frame=torch.empty((B,), dtype=torch.int32, device=device))


def ssd_entropy_gate(frame_entropy: torch.Tensor, frame_off: torch.Tensor, tau_ctc: float,
                     out=None) -> Dict[str, torch.Tensor]:
    """The entropy gate (Eq. 3): accept iff every frame entropy is below tau_ctc."""
    B, N = frame_off.shape[0] - 1, frame_entropy.shape[0]
    if frame_entropy.dtype != torch.float32 or frame_off.dtype != torch.int64:
        raise TypeError("frame_entropy must be float32 and frame_off int64")
    if out is None:
        out = alloc_gate_outputs(B, frame_entropy.device)
    rc = lib().ssd_entropy_gate(
        _dev(frame_entropy, "frame_entropy"), _dev(frame_off, "frame_off"), B, N,
        C.c_float(tau_ctc), _dev(out["gate_accept"], "gate_accept"),
        _dev(out["max_entropy"], "max_entropy"), _dev(out.get("argmax_frame"), "argmax_frame"),
        None, None, _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_entropy_gate")
    return out


def _gate_from_maxima_args(utt_max_entropy, utt_status, tau_ctc, out):
    B = utt_max_entropy.shape[0]
    if utt_max_entropy.dtype != torch.float32 or utt_status.dtype != torch.int32:
        raise TypeError("utt_max_entropy must be float32 and utt_status int32 (the bits of a uint32)")
    return [None, None, B, 0, C.c_float(tau_ctc), _dev(out["gate_accept"], "gate_accept"),
            _dev(out["max_entropy"], "max_entropy"), None,
            _dev(utt_max_entropy, "utt_max_entropy"), _dev(utt_status, "utt_status"), _stream()]


def ssd_entropy_gate_from_maxima(utt_max_entropy: torch.Tensor, utt_status: torch.Tensor,
                                 tau_ctc: float, out=None) -> Dict[str, torch.Tensor]:
    """The entropy gate (Eq. 3) through ssd_entropy_gate's second form: from the utterance
    maxima and status words ssd_ctc_draft left behind (B values instead of N frame entropies).
    `out` needs gate_accept and max_entropy only."""
    if out is not None:
        rc = (_call or _native()).gate_from_maxima(utt_max_entropy, utt_status, tau_ctc, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_entropy_gate")
    if out is None:
        B, dev = utt_max_entropy.shape[0], utt_max_entropy.device
        out = dict(gate_accept=torch.empty((B,), dtype=torch.uint8, device=dev),
                   max_entropy=torch.empty((B,), dtype=torch.float32, device=dev))
    rc = lib().ssd_entropy_gate(*_gate_from_maxima_args(utt_max_entropy, utt_status, tau_ctc, out))
    if rc != OK:
        raise SsdError(rc, "ssd_entropy_gate")
    return out


def alloc_verify_outputs(M: int, B: int, device, workspace_bytes: int) -> Dict[str, torch.Tensor]:
    e = lambda n, dt: torch.empty((n,), dtype=dt, device=device)
    return dict(token_logp=e(M, torch.float32), row_lse=e(M, torch.float32),
                accepted_len=e(B, torch.int32), all_accepted=e(B, torch.uint8),
                utt_status=e(B, torch.int32),
                workspace=torch.empty((max(workspace_bytes, 256),), dtype=torch.uint8,
                                      device=device))


def ssd_verify(logits: torch.Tensor, tok_off: torch.Tensor, draft_ids: torch.Tensor,
               tau_slm: float, skip: Optional[torch.Tensor] = None, V: Optional[int] = None,
               out=None, opts: Optional[LaunchOpts] = None) -> Dict[str, torch.Tensor]:
    """Stage 2 (Eq. 5, Section 2.3): draft-token log-likelihoods and the accepted prefix."""
    if out is not None and opts is None:
        rc = (_call or _native()).verify(logits, tok_off, draft_ids, tau_slm, skip, V, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_verify")
    M, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = tok_off.shape[0] - 1
    if tok_off.dtype != torch.int64 or draft_ids.dtype != torch.int32:
        raise TypeError("tok_off must be int64 and draft_ids int32")
    if skip is not None and skip.dtype != torch.uint8:
        raise TypeError("skip must be uint8")
    code = _dtype_code(logits)
    if out is None:
        out = alloc_verify_outputs(M, B, logits.device,
                                   ssd_verify_workspace_bytes(B, M, V, code, opts))
    ws = out["workspace"]
    rc = lib().ssd_verify(
        _dev(logits, "logits"), code, V, ld, _dev(tok_off, "tok_off"),
        _dev(draft_ids, "draft_ids"), B, M, C.c_float(tau_slm), _dev(skip, "skip"),
        _dev(out["token_logp"], "token_logp"), _dev(out.get("row_lse"), "row_lse"),
        _dev(out["accepted_len"], "accepted_len"), _dev(out["all_accepted"], "all_accepted"),
        _dev(out["utt_status"], "utt_status"), _dev(ws, "workspace"), ws.numel(), _stream(),
        _opts(opts))
    if rc != OK:
        raise SsdError(rc, "ssd_verify")
    return out


def ssd_verify_static(logits: torch.Tensor, tok_off: torch.Tensor, draft_ids: torch.Tensor,
                      tau_slm: float, out: Dict[str, torch.Tensor],
                      skip: Optional[torch.Tensor] = None, V: Optional[int] = None,
                      opts: Optional[LaunchOpts] = None) -> Dict[str, torch.Tensor]:
    """ssd_verify for callers that cannot allocate: the scratch is the library's own fixed
    device array, so `out` holds only the result tensors (token_logp, row_lse, accepted_len,
    all_accepted, utt_status), which the caller owns and must pass in.  This wrapper allocates
    nothing either.  Sizes beyond the fixed array raise SsdError with code ERR_TOO_LARGE."""
    M, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = tok_off.shape[0] - 1
    if tok_off.dtype != torch.int64 or draft_ids.dtype != torch.int32:
        raise TypeError("tok_off must be int64 and draft_ids int32")
    if skip is not None and skip.dtype != torch.uint8:
        raise TypeError("skip must be uint8")
    rc = lib().ssd_verify_static(
        _dev(logits, "logits"), _dtype_code(logits), V, ld, _dev(tok_off, "tok_off"),
        _dev(draft_ids, "draft_ids"), B, M, C.c_float(tau_slm), _dev(skip, "skip"),
        _dev(out["token_logp"], "token_logp"), _dev(out.get("row_lse"), "row_lse"),
        _dev(out["accepted_len"], "accepted_len"), _dev(out["all_accepted"], "all_accepted"),
        _dev(out["utt_status"], "utt_status"), _stream(), _opts(opts))
    if rc != OK:
        raise SsdError(rc, "ssd_verify_static")
    return out


def ssd_verify_shard(logits: torch.Tensor, col0: int, tok_off: torch.Tensor,
                     draft_ids: torch.Tensor, skip: Optional[torch.Tensor] = None,
                     V_local: Optional[int] = None, stats: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None,
                     opts: Optional[LaunchOpts] = None) -> torch.Tensor:
    """Stage 2 over a vocabulary-parallel LLM head, this rank's part: `logits` holds columns
    [col0, col0 + V_local) of the whole vocabulary; returns [M, 3] (max, sum, draft logit)."""
    if stats is not None and workspace is not None and opts is None:
        rc = (_call or _native()).verify_shard(logits, col0, tok_off, draft_ids, skip, V_local, stats,
                                               workspace)
        if rc == OK:
            return stats
        if rc is not None:
            raise SsdError(rc, "ssd_verify_shard")
    M, ld = _rows_ld(logits)
    V_local = logits.shape[1] if V_local is None else V_local
    B = tok_off.shape[0] - 1
    if tok_off.dtype != torch.int64 or draft_ids.dtype != torch.int32:
        raise TypeError("tok_off must be int64 and draft_ids int32")
    if skip is not None and skip.dtype != torch.uint8:
        raise TypeError("skip must be uint8")
    if stats is None:
        stats = torch.zeros((M, 3), dtype=torch.float32, device=logits.device)
    if workspace is None:
        need = ssd_verify_workspace_bytes(B, M, V_local, _dtype_code(logits), opts)
        workspace = torch.empty((max(need, 256),), dtype=torch.uint8, device=logits.device)
    rc = lib().ssd_verify_shard(
        _dev(logits, "logits"), _dtype_code(logits), V_local, ld, col0, _dev(tok_off, "tok_off"),
        _dev(draft_ids, "draft_ids"), B, M, _dev(skip, "skip"), _dev(stats, "shard_stats"),
        _dev(workspace, "workspace"), workspace.numel(), _stream(), _opts(opts))
    if rc != OK:
        raise SsdError(rc, "ssd_verify_shard")
    return stats


def ssd_verify_combine(stats_all: torch.Tensor, V_total: int, tok_off: torch.Tensor,
                       draft_ids: torch.Tensor, tau_slm: float,
                       skip: Optional[torch.Tensor] = None, out=None) -> Dict[str, torch.Tensor]:
    """After the all-gather of every rank's ssd_verify_shard result into stats_all [R, M, 3]:
    log-likelihoods (Eq. 5) and the accepted prefix, as ssd_verify returns them."""
    if out is not None:
        rc = (_call or _native()).verify_combine(stats_all, V_total, tok_off, draft_ids, tau_slm, skip,
                                                 out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_verify_combine")
    if stats_all.dim() != 3 or stats_all.shape[2] != 3 or not stats_all.is_contiguous() \
            or stats_all.dtype != torch.float32:
        raise ValueError("stats_all must be a contiguous float32 tensor [R, M, 3]")
    R, M = stats_all.shape[0], stats_all.shape[1]
    B = tok_off.shape[0] - 1
    if tok_off.dtype != torch.int64 or draft_ids.dtype != torch.int32:
        raise TypeError("tok_off must be int64 and draft_ids int32")
    if out is None:
        out = alloc_verify_outputs(M, B, stats_all.device, 0)
    rc = lib().ssd_verify_combine(
        _dev(stats_all, "stats_all"), R, V_total, _dev(tok_off, "tok_off"),
        _dev(draft_ids, "draft_ids"), B, M, C.c_float(tau_slm), _dev(skip, "skip"),
        _dev(out["token_logp"], "token_logp"), _dev(out.get("row_lse"), "row_lse"),
        _dev(out["accepted_len"], "accepted_len"), _dev(out["all_accepted"], "all_accepted"),
        _dev(out["utt_status"], "utt_status"), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_verify_combine")
    return out


def ssd_verify_early_exit_workspace_bytes(B, M, V, dtype_code, opts=None) -> int:
    return int(lib().ssd_verify_early_exit_workspace_bytes(B, M, V, dtype_code, _opts(opts)))


def _early_exit_args(logits, tok_off, draft_ids, tau_slm, out, skip, V, opts):
    M, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = tok_off.shape[0] - 1
    if tok_off.dtype != torch.int64 or draft_ids.dtype != torch.int32:
        raise TypeError("tok_off must be int64 and draft_ids int32")
    if skip is not None and skip.dtype != torch.uint8:
        raise TypeError("skip must be uint8")
    ws = out["workspace"]
    return [_dev(logits, "logits"), _dtype_code(logits), V, ld, _dev(tok_off, "tok_off"),
            _dev(draft_ids, "draft_ids"), B, M, C.c_float(tau_slm), _dev(skip, "skip"),
            _dev(out["token_logp"], "token_logp"), _dev(out.get("row_lse"), "row_lse"),
            _dev(out["accepted_len"], "accepted_len"), _dev(out["all_accepted"], "all_accepted"),
            _dev(out["utt_status"], "utt_status"), _dev(out.get("rows_read"), "rows_read"),
            _dev(ws, "workspace"), ws.numel(), _stream(), _opts(opts)]


def alloc_early_exit_outputs(M, B, V, dtype_code, device, opts=None) -> Dict[str, torch.Tensor]:
    out = alloc_verify_outputs(M, B, device,
                               ssd_verify_early_exit_workspace_bytes(B, M, V, dtype_code, opts))
    out["rows_read"] = torch.empty((B,), dtype=torch.int32, device=device)
    return out


def ssd_verify_early_exit(logits: torch.Tensor, tok_off: torch.Tensor, draft_ids: torch.Tensor,
                          tau_slm: float, skip: Optional[torch.Tensor] = None,
                          V: Optional[int] = None, out=None,
                          opts: Optional[LaunchOpts] = None) -> Dict[str, torch.Tensor]:
    """Stage 2 with early exit (Section 2.3 needs only the first reject): same decisions as
    ssd_verify; token_logp only for the rows that were read."""
    if out is not None and opts is None:
        rc = (_call or _native()).verify_early_exit(logits, tok_off, draft_ids, tau_slm, skip, V, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_verify_early_exit")
    if out is None:
        M = logits.shape[0]
        out = alloc_early_exit_outputs(M, tok_off.shape[0] - 1,
                                       logits.shape[1] if V is None else V, _dtype_code(logits),
                                       logits.device, opts)
    rc = lib().ssd_verify_early_exit(*_early_exit_args(logits, tok_off, draft_ids, tau_slm, out,
                                                       skip, V, opts))
    if rc != OK:
        raise SsdError(rc, "ssd_verify_early_exit")
    return out


def bind_verify_early_exit(logits, tok_off, draft_ids, tau_slm, out, skip=None, V=None,
                           opts: Optional[LaunchOpts] = None):
    args = _early_exit_args(logits, tok_off, draft_ids, tau_slm, out, skip, V, opts)
    return BoundCall(lib().ssd_verify_early_exit, "ssd_verify_early_exit", args,
                     (logits, tok_off, draft_ids, out, skip, opts), True)


def ssd_threshold_sweep(utt_max_entropy: torch.Tensor, token_logp: torch.Tensor,
                        tok_off: torch.Tensor, tau_ctc, tau_slm, out=None,
                        want_counts: bool = True) -> Dict[str, torch.Tensor]:
    """Gate and first reject for every (tau_ctc[p], tau_slm[p]) pair from stored maxima and
    log-likelihoods (Section 3.2's operating-point sweep).  tau_ctc / tau_slm: host sequences."""
    B, M = tok_off.shape[0] - 1, token_logp.shape[0]
    P = len(tau_ctc)
    if len(tau_slm) != P:
        raise ValueError("tau_ctc and tau_slm must have the same length")
    if utt_max_entropy.dtype != torch.float32 or token_logp.dtype != torch.float32:
        raise TypeError("utt_max_entropy and token_logp must be float32")
    if tok_off.dtype != torch.int64:
        raise TypeError("tok_off must be int64")
    dev = token_logp.device if M else utt_max_entropy.device
    if out is None:
        out = dict(gate_accept=torch.empty((P, B), dtype=torch.uint8, device=dev),
                   accepted_len=torch.empty((P, B), dtype=torch.int32, device=dev),
                   all_accepted=torch.empty((P, B), dtype=torch.uint8, device=dev))
        if want_counts:
            out["counts"] = torch.empty((P, 3), dtype=torch.int32, device=dev)
    tc = (C.c_float * max(P, 1))(*[float(v) for v in tau_ctc])
    ts = (C.c_float * max(P, 1))(*[float(v) for v in tau_slm])
    rc = lib().ssd_threshold_sweep(
        _dev(utt_max_entropy, "utt_max_entropy"), _dev(token_logp, "token_logp"),
        _dev(tok_off, "tok_off"), B, M, C.cast(tc, C.c_void_p), C.cast(ts, C.c_void_p), P,
        _dev(out["gate_accept"], "gate_accept"), _dev(out["accepted_len"], "accepted_len"),
        _dev(out["all_accepted"], "all_accepted"), _dev(out.get("counts"), "counts"), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_threshold_sweep")
    return out


def ssd_assemble(tokens: torch.Tensor, tok_off: torch.Tensor, gate_accept: torch.Tensor,
                 accepted_len: torch.Tensor, all_accepted: torch.Tensor,
                 out=None) -> Dict[str, torch.Tensor]:
    """Eq. 7: final hypotheses and the ordered list of utterances left to the AR pass."""
    if out is not None:
        rc = (_call or _native()).assemble(tokens, tok_off, gate_accept, accepted_len, all_accepted, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_assemble")
    B, M = tok_off.shape[0] - 1, tokens.shape[0]
    if tokens.dtype != torch.int32 or accepted_len.dtype != torch.int32:
        raise TypeError("tokens and accepted_len must be int32")
    if gate_accept.dtype != torch.uint8 or all_accepted.dtype != torch.uint8:
        raise TypeError("gate_accept and all_accepted must be uint8")
    if tok_off.dtype != torch.int64:
        raise TypeError("tok_off must be int64")
    dev = tok_off.device
    if out is None:
        e = lambda n, dt: torch.empty((n,), dtype=dt, device=dev)
        out = dict(final_tokens=e(M, torch.int32), final_len=e(B, torch.int32),
                   is_final=e(B, torch.uint8), ar_count=e(1, torch.int32),
                   ar_utt=e(B, torch.int32), ar_resume=e(B, torch.int32))
    rc = lib().ssd_assemble(
        _dev(tokens, "tokens"), _dev(tok_off, "tok_off"), B, M, _dev(gate_accept, "gate_accept"),
        _dev(accepted_len, "accepted_len"), _dev(all_accepted, "all_accepted"),
        _dev(out["final_tokens"], "final_tokens"), _dev(out["final_len"], "final_len"),
        _dev(out["is_final"], "is_final"), _dev(out["ar_count"], "ar_count"),
        _dev(out["ar_utt"], "ar_utt"), _dev(out["ar_resume"], "ar_resume"), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_assemble")
    return out


def ssd_greedy_step_workspace_bytes(R, V, dtype_code, opts=None) -> int:
    return int(lib().ssd_greedy_step_workspace_bytes(R, V, dtype_code, _opts(opts)))


def ssd_greedy_step(logits: torch.Tensor, V: Optional[int] = None, out=None,
                    opts: Optional[LaunchOpts] = None) -> Dict[str, torch.Tensor]:
    """One greedy decoding step (Eq. 6) per row: most likely token and its log-likelihood."""
    if out is not None and opts is None:
        rc = (_call or _native()).greedy_step(logits, V, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_greedy_step")
    R, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    code = _dtype_code(logits)
    if out is None:
        dev = logits.device
        e = lambda n, dt: torch.empty((n,), dtype=dt, device=dev)
        out = dict(next_token=e(R, torch.int32), next_logp=e(R, torch.float32),
                   row_lse=e(R, torch.float32), row_status=e(R, torch.int32),
                   workspace=torch.empty((max(ssd_greedy_step_workspace_bytes(R, V, code, opts), 256),),
                                         dtype=torch.uint8, device=dev))
    ws = out["workspace"]
    rc = lib().ssd_greedy_step(
        _dev(logits, "logits"), code, V, ld, R, _dev(out["next_token"], "next_token"),
        _dev(out.get("next_logp"), "next_logp"), _dev(out.get("row_lse"), "row_lse"),
        _dev(out.get("row_status"), "row_status"), _dev(ws, "workspace"), ws.numel(), _stream(),
        _opts(opts))
    if rc != OK:
        raise SsdError(rc, "ssd_greedy_step")
    return out


# ---- draft trees and their cache ---------------------------------------------------------------

def _here(t: Optional[torch.Tensor], name: str):
    """Address of a tensor on the current device, which is the one that the library launches on."""
    p = _dev(t, name)
    if t is not None and t.device.index != torch.cuda.current_device():
        raise ValueError("%s is on %s, which is not the current device" % (name, t.device))
    return p


def _flat(t: Optional[torch.Tensor], name: str, dtype, n: int):
    """Address of a contiguous [n] of a type, or None for None."""
    if t is not None and (t.dtype != dtype or t.shape != (n,) or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s [%d]" % (name, dtype, n))
    return _here(t, name)


def _heads(x: torch.Tensor, name: str) -> Heads:
    if x.dim() != 3 or (x.shape[2] > 1 and x.stride(2) != 1):
        raise ValueError("%s must be [rows, heads, head_dim] with contiguous heads" % name)
    return Heads(_here(x, name), x.stride(0), x.stride(1), x.shape[1])


def _kv_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float16:
        return F16
    raise TypeError("keys and values must be bfloat16 or float16, got %s" % t.dtype)


def _kv_cache(k_cache: torch.Tensor, v_cache: Optional[torch.Tensor], page_table: torch.Tensor,
              cache_len: torch.Tensor, B: int) -> KvCache:
    if k_cache.dim() != 4 or (k_cache.shape[3] > 1 and k_cache.stride(3) != 1):
        raise ValueError("k_cache must be [pages, page_size, heads, head_dim] with contiguous heads")
    if v_cache is not None and (v_cache.dtype != k_cache.dtype or v_cache.shape != k_cache.shape or
                                any(n > 1 and a != b for n, a, b in zip(k_cache.shape, v_cache.stride(), k_cache.stride()))):
        raise ValueError("v_cache must have k_cache's type, shape and strides")
    if page_table.dtype != torch.int32 or cache_len.dtype != torch.int32:
        raise TypeError("page_table and cache_len must be int32")
    if page_table.dim() != 2 or page_table.shape[0] != B or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table must be [B, max_pages] with contiguous rows")
    if cache_len.dim() != 1 or cache_len.shape[0] != B or (B > 1 and cache_len.stride(0) != 1):
        raise ValueError("cache_len must be a contiguous [B]")
    pages, page, heads, D = k_cache.shape
    return KvCache(_here(k_cache, "k_cache"), _here(v_cache, "v_cache"), k_cache.stride(0), k_cache.stride(1),
                   k_cache.stride(2), pages, page, heads, D, _kv_code(k_cache), page_table.shape[1],
                   _here(page_table, "page_table"), max(page_table.stride(0), page_table.shape[1]) if B <= 1 else page_table.stride(0),
                   _here(cache_len, "cache_len"))


def _ref(x):
    return C.cast(C.pointer(x), C.c_void_p)


def _nodes(tok_off: torch.Tensor, parent: Optional[torch.Tensor], M: int) -> int:
    if tok_off.dtype != torch.int64 or tok_off.dim() != 1 or not tok_off.is_contiguous():
        raise TypeError("tok_off must be a contiguous int64 [B + 1]")
    if parent is not None and (parent.dtype != torch.int32 or parent.shape != (M,) or not parent.is_contiguous()):
        raise TypeError("parent must be a contiguous int32 [M]")
    return tok_off.shape[0] - 1


def ssd_tree_attention_workspace_bytes(heads: int, kv_heads: int, head_dim: int, M: int, max_nodes: int) -> int:
    return int(lib().ssd_tree_attention_workspace_bytes(heads, kv_heads, head_dim, M, max_nodes))


def alloc_tree_attention_outputs(M: int, B: int, heads: int, head_dim: int, dtype, device, kv_heads: int = 1,
                                 max_nodes: Optional[int] = None) -> Dict[str, torch.Tensor]:
    """kv_heads and max_nodes size the workspace: without them it is enough for any."""
    ws = max([256] + [ssd_tree_attention_workspace_bytes(heads, kv, head_dim, M, M if max_nodes is None else max_nodes)
                      for kv in range(kv_heads, heads + 1) if heads % kv == 0 and heads // kv <= 128])
    return dict(out=torch.empty((M, heads, head_dim), dtype=dtype, device=device),
                lse=torch.empty((M, heads), dtype=torch.float32, device=device),
                utt_status=torch.empty((B,), dtype=torch.int32, device=device),
                workspace=torch.empty((ws,), dtype=torch.uint8, device=device))


def ssd_tree_attention(q: torch.Tensor, tree_k: torch.Tensor, tree_v: torch.Tensor, k_cache: torch.Tensor,
                       v_cache: torch.Tensor, page_table: torch.Tensor, cache_len: torch.Tensor,
                       tok_off: torch.Tensor, max_nodes: int, parent: Optional[torch.Tensor] = None,
                       scale: Optional[float] = None, cap: float = 0.0, out=None) -> Dict[str, torch.Tensor]:
    """Attention of every draft node to its utterance's paged cache and to its own line of descent
    (one layer of the pass that Section 2.2 verifies with).  q [M, Hq, D]; tree_k, tree_v [M, Hkv, D];
    k_cache, v_cache [pages, page_size, Hkv, D]; parent None: chains; scale None: D ** -0.5; scores capped
    at cap by a tanh where cap > 0.  Returns out [M, Hq, D], lse [M, Hq] and utt_status [B]."""
    if out is not None:
        rc = (_call or _native()).tree_attention(
            q, tree_k, tree_v, k_cache, v_cache, page_table, cache_len, tok_off, max_nodes, parent,
            q.shape[-1] ** -0.5 if scale is None else scale, cap, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_tree_attention")
    M, B = q.shape[0], _nodes(tok_off, parent, q.shape[0])
    if tree_k.dtype != q.dtype or tree_v.dtype != q.dtype or k_cache.dtype != q.dtype:
        raise TypeError("q, tree_k, tree_v and the cache must have one type")
    for name, x in (("tree_k", tree_k), ("tree_v", tree_v)):
        if x.dim() != 3 or x.shape[0] != M or x.shape[2] != q.shape[2]:
            raise ValueError("%s must be [M, heads, head_dim] like q" % name)
    if k_cache.dim() != 4 or k_cache.shape[3] != q.shape[2]:
        raise ValueError("the cache's heads are not as long as q's")
    if out is None:
        out = alloc_tree_attention_outputs(M, B, q.shape[1], q.shape[2], q.dtype, q.device, tree_k.shape[1], max_nodes)
    o, lse, ws = out["out"], out.get("lse"), out["workspace"]
    if o.dtype != q.dtype or o.shape != q.shape:
        raise ValueError("out must have q's type and shape")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [M, heads]")
    cache = _kv_cache(k_cache, v_cache, page_table, cache_len, B)
    rc = lib().ssd_tree_attention(
        _ref(_heads(q, "q")), _ref(_heads(tree_k, "tree_k")), _ref(_heads(tree_v, "tree_v")), _ref(cache),
        _here(tok_off, "tok_off"), _here(parent, "parent"), B, M, max_nodes,
        q.shape[2] ** -0.5 if scale is None else scale, cap, _ref(_heads(o, "out")), _here(lse, "lse"),
        _flat(out["utt_status"], "utt_status", torch.int32, B), _here(ws, "workspace"), ws.numel(), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_tree_attention")
    return out


def alloc_verify_tree_outputs(M: int, B: int, device, workspace_bytes: int) -> Dict[str, torch.Tensor]:
    e = lambda n, dt: torch.empty((n,), dtype=dt, device=device)
    return dict(token_logp=e(M, torch.float32), row_lse=e(M, torch.float32), path=e(M, torch.int32),
                path_len=e(B, torch.int32), on_path=e(M, torch.uint8), utt_status=e(B, torch.int32),
                workspace=e(max(workspace_bytes, 256), torch.uint8))


def ssd_verify_tree(logits: torch.Tensor, tok_off: torch.Tensor, draft_ids: torch.Tensor,
                    parent: Optional[torch.Tensor], tau_slm: float, skip: Optional[torch.Tensor] = None,
                    V: Optional[int] = None, out=None, opts: Optional[LaunchOpts] = None) -> Dict[str, torch.Tensor]:
    """Stage 2 along a draft tree (Eq. 5 on every path): logits row i is the LLM's output after node i;
    returns the nodes' log-likelihoods and the longest accepted path.  parent None: chains."""
    if out is not None and opts is None:
        rc = (_call or _native()).verify_tree(logits, tok_off, draft_ids, parent, tau_slm, skip, V, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_verify_tree")
    M, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = _nodes(tok_off, parent, M)
    code = _dtype_code(logits)
    if out is None:
        out = alloc_verify_tree_outputs(M, B, logits.device, ssd_verify_workspace_bytes(B, M, V, code, opts))
    ws = out["workspace"]
    rc = lib().ssd_verify_tree(
        _here(logits, "logits"), code, V, ld, _here(tok_off, "tok_off"), _flat(draft_ids, "draft_ids", torch.int32, M),
        _here(parent, "parent"), B, M, C.c_float(tau_slm), _flat(skip, "skip", torch.uint8, B), _flat(out["token_logp"], "token_logp", torch.float32, M),
        _flat(out.get("row_lse"), "row_lse", torch.float32, M), _flat(out["path"], "path", torch.int32, M), _flat(out["path_len"], "path_len", torch.int32, B),
        _flat(out["on_path"], "on_path", torch.uint8, M), _flat(out["utt_status"], "utt_status", torch.int32, B), _here(ws, "workspace"), ws.numel(),
        _stream(), _opts(opts))
    if rc != OK:
        raise SsdError(rc, "ssd_verify_tree")
    return out


def _weights(weight: Optional[torch.Tensor], name: str, B: int, device):
    """Address, stride and columns of [B, slots] weights."""
    if weight is None:
        return None, 0, 0
    if weight.dtype != torch.float32 or weight.dim() != 2 or weight.shape[0] != B or \
            (weight.shape[1] > 1 and weight.stride(1) != 1):
        raise ValueError("%s must be float32 [B, slots] with contiguous rows" % name)
    return _here(weight, name), (weight.stride(0) if B > 1 else max(weight.stride(0), weight.shape[1])), weight.shape[1]


def alloc_cache_append_outputs(B: int, device) -> Dict[str, torch.Tensor]:
    return dict(new_len=torch.empty((B,), dtype=torch.int32, device=device),
                utt_status=torch.empty((B,), dtype=torch.int32, device=device))


def ssd_cache_append(tree_k: torch.Tensor, tree_v: torch.Tensor, tok_off: torch.Tensor, path: Optional[torch.Tensor],
                     path_len: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor,
                     cache_len: torch.Tensor, weight: Optional[torch.Tensor] = None, out=None) -> Dict[str, torch.Tensor]:
    """The accepted path's keys and values enter the cache, in place (the K/V of Eq. 7's verified prefix); path and
    path_len as ssd_verify_tree leaves them, path None: an utterance's first path_len nodes.  weight [B, slots]
    is set to 0 for the new slots.  Returns new_len, which is not cache_len, and utt_status."""
    if out is not None:
        rc = (_call or _native()).cache_append(tree_k, tree_v, tok_off, path, path_len, k_cache, v_cache,
                                                page_table, cache_len, weight, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_cache_append")
    M, B = tree_k.shape[0], _nodes(tok_off, path, tree_k.shape[0])
    if tree_k.dtype != k_cache.dtype or tree_v.dtype != k_cache.dtype:
        raise TypeError("tree_k, tree_v and the cache must have one type")
    for name, x in (("tree_k", tree_k), ("tree_v", tree_v)):
        if x.dim() != 3 or x.shape[0] != M or x.shape[2] != k_cache.shape[3]:
            raise ValueError("%s must be [M, heads, head_dim] like the cache" % name)
    if path_len.dtype != torch.int32 or path_len.shape != (B,) or not path_len.is_contiguous():
        raise TypeError("path_len must be a contiguous int32 [B]")
    if out is None:
        out = alloc_cache_append_outputs(B, k_cache.device)
    rc = lib().ssd_cache_append(
        _ref(_heads(tree_k, "tree_k")), _ref(_heads(tree_v, "tree_v")),
        _ref(_kv_cache(k_cache, v_cache, page_table, cache_len, B)), _here(tok_off, "tok_off"), _here(path, "path"),
        _here(path_len, "path_len"), B, M, *_weights(weight, "weight", B, k_cache.device),
        _flat(out["new_len"], "new_len", torch.int32, B), _flat(out["utt_status"], "utt_status", torch.int32, B), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_cache_append")
    return out


def alloc_cache_weights_outputs(B: int, device) -> Dict[str, torch.Tensor]:
    return dict(utt_status=torch.empty((B,), dtype=torch.int32, device=device))


def ssd_cache_weights(q: torch.Tensor, lse: torch.Tensor, k_cache: torch.Tensor, page_table: torch.Tensor,
                      cache_len: torch.Tensor, tok_off: torch.Tensor, max_nodes: int, weight: torch.Tensor,
                      use: Optional[torch.Tensor] = None, scale: Optional[float] = None, cap: float = 0.0,
                      out=None) -> Dict[str, torch.Tensor]:
    """Adds to weight [B, slots], in place, the attention weight that every cached slot receives from the
    nodes with use != 0 (None: all), summed over their heads; lse as ssd_tree_attention returns it."""
    if out is not None:
        rc = (_call or _native()).cache_weights(
            q, lse, k_cache, page_table, cache_len, tok_off, max_nodes, weight, use,
            q.shape[-1] ** -0.5 if scale is None else scale, cap, out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_cache_weights")
    M, B = q.shape[0], _nodes(tok_off, None, q.shape[0])
    if q.dim() != 3 or q.dtype != k_cache.dtype or k_cache.dim() != 4 or k_cache.shape[3] != q.shape[2]:
        raise ValueError("q must be [M, heads, head_dim] of the cache's type")
    if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [M, heads]")
    if use is not None and (use.dtype != torch.uint8 or use.shape != (M,) or not use.is_contiguous()):
        raise TypeError("use must be a contiguous uint8 [M]")
    if out is None:
        out = alloc_cache_weights_outputs(B, q.device)
    rc = lib().ssd_cache_weights(
        _ref(_heads(q, "q")), _here(lse, "lse"), _ref(_kv_cache(k_cache, None, page_table, cache_len, B)),
        _here(tok_off, "tok_off"), B, M, max_nodes, q.shape[2] ** -0.5 if scale is None else scale, cap,
        _here(use, "use"), *_weights(weight, "weight", B, q.device), _flat(out["utt_status"], "utt_status", torch.int32, B), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_cache_weights")
    return out


def alloc_cache_evict_outputs(B: int, budget: int, device) -> Dict[str, torch.Tensor]:
    e = lambda shape, dt: torch.empty(shape, dtype=dt, device=device)
    return dict(kept=e((B, budget), torch.int32), weight=e((B, budget), torch.float32),
                new_len=e((B,), torch.int32), utt_status=e((B,), torch.int32))


def ssd_cache_evict(k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, cache_len: torch.Tensor,
                    weight: torch.Tensor, budget: int, sink: int = 0, recent: int = 0, out=None) -> Dict[str, torch.Tensor]:
    """Caches of more than `budget` slots keep the first `sink`, the last `recent` and the heaviest between, moved
    down in place and in order.  Returns kept [B, budget], the kept slots' weight [B, budget], new_len and
    utt_status."""
    if out is not None:
        rc = (_call or _native()).cache_evict(k_cache, v_cache, page_table, cache_len, weight, budget, sink, recent,
                                               out)
        if rc == OK:
            return out
        if rc is not None:
            raise SsdError(rc, "ssd_cache_evict")
    B = cache_len.shape[0]
    if out is None:
        out = alloc_cache_evict_outputs(B, budget, k_cache.device)
    kept = out["kept"]
    if kept.dtype != torch.int32 or kept.shape != (B, budget) or not kept.is_contiguous():
        raise ValueError("kept must be a contiguous int32 [B, budget]")
    w_out, out_stride, out_cols = _weights(out.get("weight"), "out['weight']", B, k_cache.device)
    if w_out is not None and out_cols < budget:
        raise ValueError("out['weight'] must have a column for every kept slot")
    rc = lib().ssd_cache_evict(
        _ref(_kv_cache(k_cache, v_cache, page_table, cache_len, B)), *_weights(weight, "weight", B, k_cache.device),
        B, budget, sink, recent, _here(kept, "kept"), w_out, out_stride, _flat(out["new_len"], "new_len", torch.int32, B),
        _flat(out["utt_status"], "utt_status", torch.int32, B), _stream())
    if rc != OK:
        raise SsdError(rc, "ssd_cache_evict")
    return out


class BoundCall:
    """One C-ABI call with its arguments already marshalled, for loops that issue the same call
    many times (benchmarks, serving loops): calling it enqueues the work again on the stream
    that was current when it was bound.  `opts` replaces the launch options for one call."""

    def __init__(self, fn, name: str, args: List, keep: tuple, has_opts: bool):
        self._fn, self._name, self._args, self._keep, self._has_opts = fn, name, args, keep, has_opts

    def __call__(self, opts: Optional[LaunchOpts] = None) -> None:
        a = self._args
        if opts is not None:
            if not self._has_opts:
                raise TypeError(self._name + " takes no launch options")
            a = a[:-1] + [C.cast(C.pointer(opts), C.c_void_p)]
        rc = self._fn(*a)
        if rc != OK:
            raise SsdError(rc, self._name)


def bind_ctc_draft(logits, frame_off, blank_id, max_draft_len, out, V=None,
                   opts: Optional[LaunchOpts] = None) -> BoundCall:
    N, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = frame_off.shape[0] - 1
    args = [_dev(logits, "logits"), _dtype_code(logits), V, ld, _dev(frame_off, "frame_off"), B, N,
            blank_id, max_draft_len, _dev(out["frame_entropy"], "frame_entropy"),
            _dev(out["frame_argmax"], "frame_argmax"), _dev(out.get("frame_lse"), "frame_lse"),
            None, _dev(out["draft_tokens"], "draft_tokens"),
            _dev(out.get("draft_frames"), "draft_frames"), _dev(out["draft_len"], "draft_len"),
            _dev(out["draft_full_len"], "draft_full_len"),
            _dev(out["utt_max_entropy"], "utt_max_entropy"), _dev(out["utt_status"], "utt_status"),
            _dev(out.get("workspace"), "workspace"),
            0 if out.get("workspace") is None else out["workspace"].numel(), _stream(), _opts(opts)]
    return BoundCall(lib().ssd_ctc_draft, "ssd_ctc_draft", args, (logits, frame_off, out, opts), True)


def bind_entropy_gate(frame_entropy, frame_off, tau_ctc, out) -> BoundCall:
    B, N = frame_off.shape[0] - 1, frame_entropy.shape[0]
    args = [_dev(frame_entropy, "frame_entropy"), _dev(frame_off, "frame_off"), B, N,
            C.c_float(tau_ctc), _dev(out["gate_accept"], "gate_accept"),
            _dev(out["max_entropy"], "max_entropy"), _dev(out.get("argmax_frame"), "argmax_frame"),
            None, None, _stream()]
    return BoundCall(lib().ssd_entropy_gate, "ssd_entropy_gate", args,
                     (frame_entropy, frame_off, out), False)


def bind_entropy_gate_from_maxima(utt_max_entropy, utt_status, tau_ctc, out) -> BoundCall:
    return BoundCall(lib().ssd_entropy_gate, "ssd_entropy_gate",
                     _gate_from_maxima_args(utt_max_entropy, utt_status, tau_ctc, out),
                     (utt_max_entropy, utt_status, out), False)


def bind_verify(logits, tok_off, draft_ids, tau_slm, out, skip=None, V=None,
                opts: Optional[LaunchOpts] = None) -> BoundCall:
    M, ld = _rows_ld(logits)
    V = logits.shape[1] if V is None else V
    B = tok_off.shape[0] - 1
    ws = out["workspace"]
    args = [_dev(logits, "logits"), _dtype_code(logits), V, ld, _dev(tok_off, "tok_off"),
            _dev(draft_ids, "draft_ids"), B, M, C.c_float(tau_slm), _dev(skip, "skip"),
            _dev(out["token_logp"], "token_logp"), _dev(out.get("row_lse"), "row_lse"),
            _dev(out["accepted_len"], "accepted_len"), _dev(out["all_accepted"], "all_accepted"),
            _dev(out["utt_status"], "utt_status"), _dev(ws, "workspace"), ws.numel(), _stream(),
            _opts(opts)]
    return BoundCall(lib().ssd_verify, "ssd_verify", args,
                     (logits, tok_off, draft_ids, out, skip, opts), True)
