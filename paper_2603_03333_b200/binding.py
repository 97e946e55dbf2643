"""Thin ctypes binding of libdropmatch's C ABI (include/dropmatch.h).

Argument marshalling only: torch tensors give device pointers and the current stream; every
step of the verification path runs inside the library's CUDA kernels.  There is no CPU
fallback: if the shared library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

OK, EINVAL, EUNSUPPORTED, ECUDA, EWORKSPACE, EDEVICE, ENOHEAD, ESTATICLIMIT = 0, -1, -2, -3, -4, -5, -6, -7
STATIC_MAX_ROWS = 256
F32, BF16 = 0, 1
RULE_NAIVE, RULE_MAJORITY = 0, 1
IMPL_AUTO, IMPL_SIMT, IMPL_TCGEN05 = 0, 1, 2
MASK_PER_POSITION, MASK_PER_PATH = 0, 1
TAIL_RENORM, TAIL_BUCKET = 0, 1
MAX_TOP = 128

_LIB_PATH = Path(__file__).resolve().parent / "libdropmatch.so"
_lib = None

_vp, _ci, _cf, _u64, _i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_uint64, ctypes.c_int64

# name -> (restype, argtypes); mirrors include/dropmatch.h declaration by declaration
SIGNATURES = {
    "dm_create": (_ci, [ctypes.POINTER(_vp), _ci]),
    "dm_destroy": (_ci, [_vp]),
    "dm_set_head": (_ci, [_vp, _vp, _ci, _ci, _ci, _ci, _ci]),
    "dm_set_impl": (_ci, [_vp, _ci]),
    "dm_set_pdl": (_ci, [_vp, _ci]),
    "dm_set_mask_mode": (_ci, [_vp, _ci]),
    "dm_set_vocab_offset": (_ci, [_vp, _ci]),
    "dropmatch_partial_best": (_ci, [_vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _vp, _vp]),
    "dropmatch_finalize_packed": (_ci, [_vp, _vp, _ci, _vp, _ci, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_verify": (_ci, [_vp, _vp, _vp, _ci, _ci, _cf, _u64, _ci, _vp, _vp, _vp, _vp]),
    "dropmatch_verify_batched": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _ci, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_verify_batched_sampled": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _ci, _cf, _cf,
                                               _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_verify_batched_next": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _u64, _u64, _ci,
                                            _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_verify_batched_host": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _ci, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_verify_batched_static": (_ci, [_ci, _vp, _ci, _ci, _ci, _vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _ci,
                                              _vp, _vp, _vp, _vp, _vp]),
    "dm_enable_js": (_ci, [_vp, _ci, _ci]),
    "dropmatch_verify_js": (_ci, [_vp, _vp, _vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dm_enable_score": (_ci, [_vp, _ci, _ci]),
    "dropmatch_score": (_ci, [_vp, _vp, _vp, _ci, _ci, _cf, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_logprobs": (_ci, [_vp, _vp, _ci, _i64, _ci, _ci, _vp, _ci, _cf, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_logprobs_grad": (_ci, [_vp, _vp, _ci, _i64, _ci, _ci, _vp, _cf, _vp, _vp, _vp, _i64, _vp]),
    "dropmatch_distill": (_ci, [_vp, _vp, _ci, _i64, _ci, _ci, _vp, _vp, _ci, _ci, _cf, _vp, _vp, _vp, _i64, _vp]),
    "dropmatch_verify_lossless": (_ci, [_vp, _vp, _ci, _i64, _vp, _ci, _i64, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _cf, _vp, _vp,
                                        _vp, _vp, _vp, _vp]),
    "dropmatch_dropout": (_ci, [_vp, _vp, _ci, _i64, _ci, _ci, _ci, _ci, _cf, _u64, _u64, _vp, _i64, _vp]),
    "dropmatch_dropout_grad": (_ci, [_vp, _vp, _ci, _i64, _ci, _ci, _ci, _ci, _cf, _u64, _u64, _vp, _i64, _vp]),
    "dropmatch_quantize_i8": (_ci, [_vp, _vp, _ci, _i64, _ci, _ci, _vp, _i64, _vp, _vp]),
    "dropmatch_matmul_i8": (_ci, [_vp, _vp, _i64, _vp, _ci, _vp, _i64, _vp, _ci, _ci, _vp, _ci, _i64, _vp]),
    "dropmatch_linear_i8": (_ci, [_vp, _vp, _ci, _i64, _ci, _vp, _i64, _vp, _ci, _ci, _vp, _i64, _vp, _vp, _ci, _i64, _vp]),
    "dropmatch_verify_tree": (_ci, [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _u64, _u64, _ci,
                                    _vp, _vp, _vp, _vp, _vp, _vp]),
    "dropmatch_verify_tree_next": (_ci, [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _u64, _u64, _ci,
                                         _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dm_debug_logits": (_ci, [_vp, _vp, _ci, _ci, _vp, _ci, _cf, _u64, _u64, _vp, _vp]),
    "dm_debug_masks": (_ci, [_vp, _ci, _ci, _ci, _ci, _cf, _u64, _u64, _vp, _vp]),
    "dm_debug_masked_operand": (_ci, [_vp, _vp, _ci, _ci, _ci, _cf, _u64, _u64, _vp, _vp]),
    "dm_debug_read_stream": (_ci, [_vp, _vp, ctypes.c_size_t, _vp]),
    "dm_device_error": (_ci, [_vp, _vp, ctypes.POINTER(ctypes.c_uint32)]),
    "dm_debug_set_wait_limit": (_ci, [_vp, _u64]),
    "dm_profile_head": (_ci, [_vp, _ci]),
    "dm_profile_read": (_ci, [_vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_ci)]),
    "dm_workspace_bytes": (ctypes.c_size_t, [_vp]),
    "dm_last_impl": (_ci, [_vp]),
    "dm_last_launches": (_ci, [_vp]),
    "dm_strerror": (ctypes.c_char_p, [_ci]),
}


class DropMatchError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


def lib() -> ctypes.CDLL:
    """Load libdropmatch.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise ImportError(f"{_LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(str(_LIB_PATH))
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().dm_strerror(status).decode()


def _check(status: int, where: str):
    if status != OK:
        raise DropMatchError(status, where)


def _ptr(t):
    # the address as a plain int: ctypes converts it for pointer parameters, and building a
    # c_void_p object per argument would cost more than the rest of the marshalling together
    return None if t is None else t.data_ptr()


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}   # of tensors of logits

_empty = torch.empty    # called with sizes, not a tuple of them: half the time

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device) -> int:
    # the handle of torch's current stream on `device` (the short way where this torch has it)
    if _raw_stream is not None:
        index = device if isinstance(device, int) else torch.device(device).index
        if index is not None:
            return _raw_stream(index)
    return torch.cuda.current_stream(device).cuda_stream


def _dev(t: torch.Tensor, dtype, what: str) -> torch.Tensor:
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise TypeError(f"{what} must be a contiguous CUDA tensor of {dtype}")
    return t


def verify_batched_static(W, H, draft, K, p, seed, seq_base=0, rule=RULE_NAIVE, out=None):
    """dropmatch_verify_batched_static: chain verification without a context and without any
    device allocation inside the library (the output tensors are the caller's; pass `out` to
    reuse them).  B*T*K may not exceed STATIC_MAX_ROWS."""
    if W.dtype not in (torch.float32, torch.bfloat16) or not W.is_cuda or not W.is_contiguous() or W.dim() != 2:
        raise TypeError("W must be a contiguous 2-D CUDA tensor of float32 or bfloat16")
    dtype = F32 if W.dtype == torch.float32 else BF16
    _dev(H, W.dtype, "H"); _dev(draft, torch.int32, "draft")
    B, T, _ = H.shape
    V, d = W.shape
    if out is None:
        i32 = dict(dtype=torch.int32, device=W.device)
        out = dict(tokens=torch.empty((B, T, K), **i32), counts=torch.empty((B, T, K), **i32),
                   hits=torch.empty((B, T), **i32), accept_len=torch.empty((B,), **i32))
    _check(lib().dropmatch_verify_batched_static(W.device.index, _ptr(W), V, d, dtype, _ptr(H), _ptr(draft), B, T, K,
                                                 p, seed, seq_base, rule, _ptr(out["tokens"]), _ptr(out["counts"]),
                                                 _ptr(out["hits"]), _ptr(out["accept_len"]), _stream(W.device)),
           "dropmatch_verify_batched_static")
    return out


class Context:
    """One dm_ctx: a device, an LM head, and the library-owned workspace."""

    def __init__(self, device: int = 0):
        self._h = ctypes.c_void_p()
        self.device = torch.device("cuda", device)
        _check(lib().dm_create(ctypes.byref(self._h), device), "dm_create")
        self._W = None
        self.dtype = None

    def close(self):
        if self._h:
            lib().dm_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _tdtype(self):
        return torch.float32 if self.dtype == F32 else torch.bfloat16

    # -- dm_set_head / dm_set_impl
    def set_head(self, W: torch.Tensor, max_rows: int, max_hidden_rows: int | None = None):
        """W must be complete before a verify call is enqueued and must not be written by work that
        is still in flight on the stream (see set_pdl)."""
        if W.dtype not in (torch.float32, torch.bfloat16) or not W.is_cuda or not W.is_contiguous() or W.dim() != 2:
            raise TypeError("W must be a contiguous 2-D CUDA tensor of float32 or bfloat16")
        dtype = F32 if W.dtype == torch.float32 else BF16
        V, d = W.shape
        _check(lib().dm_set_head(self._h, _ptr(W), V, d, dtype, max_rows, max_hidden_rows or max_rows), "dm_set_head")
        self._W, self.dtype, self.V, self.d = W, dtype, V, d   # keep W alive

    def set_impl(self, impl: int):
        _check(lib().dm_set_impl(self._h, impl), "dm_set_impl")

    def set_pdl(self, enable: bool):
        """Off: verify kernels never start before earlier work of the stream has completed (needed when
        that work writes W; by default the kernel streams W while the kernel ahead is still finishing)."""
        _check(lib().dm_set_pdl(self._h, int(enable)), "dm_set_pdl")

    def set_mask_mode(self, mode: int):
        _check(lib().dm_set_mask_mode(self._h, mode), "dm_set_mask_mode")

    # -- vocabulary-sharded heads
    def set_vocab_offset(self, offset: int):
        _check(lib().dm_set_vocab_offset(self._h, offset), "dm_set_vocab_offset")

    def partial_best(self, H, K, p, seed, seq_base=0):
        """-> int64 tensor [B*T*K] holding the packed (key, inverted token id) words bit for bit."""
        B, T, _ = H.shape
        _dev(H, self._tdtype(), "H")
        out = torch.empty((B * T * K,), dtype=torch.int64, device=self.device)
        _check(lib().dropmatch_partial_best(self._h, _ptr(H), B, T, K, p, seed, seq_base, _ptr(out),
                                            _stream(self.device)), "dropmatch_partial_best")
        return out

    def finalize_packed(self, packed, draft, K, rule=RULE_NAIVE):
        """packed: int64 [n_parts, B*T*K] (or [B*T*K]); draft[B,T] -> the outputs of verify_batched."""
        _dev(draft, torch.int32, "draft")
        B, T = draft.shape
        if packed.dim() == 1:
            packed = packed.unsqueeze(0)
        _dev(packed, torch.int64, "packed")
        if packed.shape[1] != B * T * K:
            raise TypeError("packed must have B*T*K words per part")
        out = self.alloc_outputs(B, T, K)
        _check(lib().dropmatch_finalize_packed(self._h, _ptr(packed), packed.shape[0], _ptr(draft), B, T, K, rule,
                                               _ptr(out["tokens"]), _ptr(out["counts"]), _ptr(out["hits"]),
                                               _ptr(out["accept_len"]), _stream(self.device)),
               "dropmatch_finalize_packed")
        return out

    # -- dropmatch_verify
    def verify(self, H, draft, K, p, seed, rule=RULE_NAIVE):
        T = H.shape[0]
        _dev(H, self._tdtype(), "H"); _dev(draft, torch.int32, "draft")
        tokens = torch.empty((T, K), dtype=torch.int32, device=self.device)
        counts = torch.empty_like(tokens)
        alen = torch.empty((1,), dtype=torch.int32, device=self.device)
        _check(lib().dropmatch_verify(self._h, _ptr(H), _ptr(draft), T, K, p, seed, rule, _ptr(tokens),
                                      _ptr(counts), _ptr(alen), _stream(self.device)), "dropmatch_verify")
        return dict(tokens=tokens, counts=counts, accept_len=alen)

    # -- dropmatch_verify_batched
    def verify_batched(self, H, draft, K, p, seed, seq_base=0, rule=RULE_NAIVE, out=None):
        B, T, _ = H.shape
        _dev(H, self._tdtype(), "H"); _dev(draft, torch.int32, "draft")
        if out is None:
            out = self.alloc_outputs(B, T, K)
        _check(lib().dropmatch_verify_batched(self._h, _ptr(H), _ptr(draft), B, T, K, p, seed, seq_base, rule,
                                              _ptr(out["tokens"]), _ptr(out["counts"]), _ptr(out["hits"]),
                                              _ptr(out["accept_len"]), _stream(self.device)),
               "dropmatch_verify_batched")
        return out

    # -- dropmatch_verify_batched_sampled
    def verify_batched_sampled(self, H, draft, K, p, seed, temperature=1.0, top_p=1.0, seq_base=0, rule=RULE_NAIVE,
                               out=None):
        B, T, _ = H.shape
        _dev(H, self._tdtype(), "H"); _dev(draft, torch.int32, "draft")
        if out is None:
            out = self.alloc_outputs(B, T, K)
        _check(lib().dropmatch_verify_batched_sampled(self._h, _ptr(H), _ptr(draft), B, T, K, p, seed, seq_base, rule,
                                                      temperature, top_p, _ptr(out["tokens"]), _ptr(out["counts"]),
                                                      _ptr(out["hits"]), _ptr(out["accept_len"]),
                                                      _stream(self.device)), "dropmatch_verify_batched_sampled")
        return out

    # -- dropmatch_verify_batched_next
    def verify_batched_next(self, H, draft, K, p, seed, seq_base=0, rule=RULE_NAIVE):
        """H[B,T_h,d] with T_h = T or T+1 (bonus row), draft[B,T].  Adds plain[B,T_h], next[B]."""
        B, T_h, _ = H.shape
        T = draft.shape[1]
        if T_h - T not in (0, 1):
            raise TypeError("H must have T or T+1 hidden rows per sequence")
        _dev(H, self._tdtype(), "H"); _dev(draft, torch.int32, "draft")
        i32 = dict(dtype=torch.int32, device=self.device)
        out = dict(tokens=torch.empty((B, T_h, K), **i32), counts=torch.empty((B, T_h, K), **i32),
                   hits=torch.empty((B, T), **i32), accept_len=torch.empty((B,), **i32),
                   plain=torch.empty((B, T_h), **i32), next=torch.empty((B,), **i32))
        _check(lib().dropmatch_verify_batched_next(self._h, _ptr(H), _ptr(draft), B, T, T_h - T, K, p, seed, seq_base,
                                                   rule, _ptr(out["tokens"]), _ptr(out["counts"]), _ptr(out["hits"]),
                                                   _ptr(out["accept_len"]), _ptr(out["plain"]), _ptr(out["next"]),
                                                   _stream(self.device)), "dropmatch_verify_batched_next")
        return out

    def alloc_outputs(self, B, T, K):
        i32 = dict(dtype=torch.int32, device=self.device)
        return dict(tokens=torch.empty((B, T, K), **i32), counts=torch.empty((B, T, K), **i32),
                    hits=torch.empty((B, T), **i32), accept_len=torch.empty((B,), **i32))

    # -- dropmatch_verify_batched_host
    def verify_batched_host(self, H, draft, K, p, seed, seq_base=0, rule=RULE_NAIVE, out=None):
        """H, draft and outputs are CPU tensors (pinned for speed); returns after the results are on the host."""
        B, T, _ = H.shape
        if H.is_cuda or draft.is_cuda or not H.is_contiguous() or not draft.is_contiguous():
            raise TypeError("host entry point takes contiguous CPU tensors")
        if H.dtype != self._tdtype() or draft.dtype != torch.int32:
            raise TypeError("H must have the head's dtype and draft must be int32")
        if out is None:
            out = self.alloc_host_outputs(B, T, K)
        _check(lib().dropmatch_verify_batched_host(self._h, _ptr(H), _ptr(draft), B, T, K, p, seed, seq_base, rule,
                                                   _ptr(out["tokens"]), _ptr(out["counts"]), _ptr(out["hits"]),
                                                   _ptr(out["accept_len"]), _stream(self.device)),
               "dropmatch_verify_batched_host")
        return out

    @staticmethod
    def alloc_host_outputs(B, T, K, pin=True):
        mk = lambda *s: torch.empty(s, dtype=torch.int32, pin_memory=pin)
        return dict(tokens=mk(B, T, K), counts=mk(B, T, K), hits=mk(B, T), accept_len=mk(B))

    # -- dm_enable_js / dropmatch_verify_js
    def enable_js(self, max_rows: int, max_hidden_rows: int):
        _check(lib().dm_enable_js(self._h, max_rows, max_hidden_rows), "dm_enable_js")

    def verify_js(self, H, draft, draft_prob, K, p, seed, seq_base=0):
        """Algorithm 1 (JS test, else majority).  draft_prob[B,T,V] float32 on the device."""
        B, T, _ = H.shape
        _dev(H, self._tdtype(), "H"); _dev(draft, torch.int32, "draft"); _dev(draft_prob, torch.float32, "draft_prob")
        if tuple(draft_prob.shape) != (B, T, self.V):
            raise TypeError("draft_prob must have shape [B, T, V]")
        i32 = dict(dtype=torch.int32, device=self.device)
        out = dict(tokens=torch.empty((B, T, K), **i32), counts=torch.empty((B, T, K), **i32),
                   js=torch.empty((B, T, K + 1), dtype=torch.float32, device=self.device),
                   js_ok=torch.empty((B, T), **i32), accept_len=torch.empty((B,), **i32))
        _check(lib().dropmatch_verify_js(self._h, _ptr(H), _ptr(draft), _ptr(draft_prob), B, T, K, p, seed, seq_base,
                                         _ptr(out["tokens"]), _ptr(out["counts"]), _ptr(out["js"]), _ptr(out["js_ok"]),
                                         _ptr(out["accept_len"]), _stream(self.device)), "dropmatch_verify_js")
        return out

    # -- dm_enable_score / dropmatch_score
    def enable_score(self, max_rows: int, max_top: int = 0):
        _check(lib().dm_enable_score(self._h, max_rows, max_top), "dm_enable_score")

    def score(self, H, tokens=None, n_top=0, temperature=1.0):
        """H[...,d] through the head, without dropout; tokens[...] int32 or None.  -> dict of float32
        tensors of the leading shape: lse, entropy, logprob (with tokens), and for n_top > 0
        top_ids[...,n_top] (int32) and top_logprob[...,n_top]."""
        self._on_device(_dev(H, self._tdtype(), "H"), "H")
        if H.dim() < 2 or H.shape[-1] != self.d:
            raise TypeError("H must have shape [..., d]")
        out = self._row_outputs(H.shape[:-1], tokens, n_top)
        _check(lib().dropmatch_score(self._h, _ptr(H), _ptr(tokens), H.numel() // self.d, n_top, temperature,
                                     *self._row_pointers(out), _stream(self.device)), "dropmatch_score")
        return out

    # -- dropmatch_logprobs / dropmatch_logprobs_grad / dropmatch_distill
    def logprobs(self, logits, tokens=None, n_top=0, temperature=1.0):
        """The outputs of `score` for logits[...,V] in memory (float32 or bfloat16; the last dimension
        dense, one stride between rows).  Autograd does not see this call, nor the two below: what they
        return carries no graph, and a gradient written into `out` does not count as a change of it."""
        rows, ld = self._rows(logits, "logits")
        out = self._row_outputs(logits.shape[:-1], tokens, n_top)
        _check(lib().dropmatch_logprobs(self._h, _ptr(logits), _DTYPES[logits.dtype], ld, rows, logits.shape[-1],
                                        _ptr(tokens), n_top, temperature, *self._row_pointers(out),
                                        _stream(self.device)), "dropmatch_logprobs")
        return out

    def logprobs_grad(self, logits, tokens, grad_logprob, grad_entropy=None, temperature=1.0, out=None):
        """-> gradient of sum(grad_logprob * logprob + grad_entropy * entropy) for the logits, in their
        dtype.  Either factor may be None; `out` may be the logits themselves."""
        rows, ld = self._rows(logits, "logits")
        lead = logits.shape[:-1]
        self._per_row(tokens, torch.int32, lead, "tokens")
        self._per_row(grad_logprob, torch.float32, lead, "grad_logprob")
        self._per_row(grad_entropy, torch.float32, lead, "grad_entropy")
        out, ld_out = self._grad_target(logits, out)
        _check(lib().dropmatch_logprobs_grad(self._h, _ptr(logits), _DTYPES[logits.dtype], ld, rows, logits.shape[-1],
                                             _ptr(tokens), temperature, _ptr(grad_logprob), _ptr(grad_entropy),
                                             _ptr(out), ld_out, _stream(self.device)), "dropmatch_logprobs_grad")
        return out

    def distill(self, logits, teacher_ids, teacher_logprob, tail=TAIL_RENORM, temperature=1.0, weight=None, loss=True,
                grad=False, out=None):
        """KL(teacher || student) per row of logits[...,V] for teacher_ids[...,k] (int32, outside [0,V):
        absent) and teacher_logprob[...,k] (float32).  -> dict: loss[...] (unless loss=False) and, with
        `grad`, the gradient of sum(weight * loss) for the logits, in their dtype, into `out` if given
        (which may be the logits themselves)."""
        rows, ld = self._rows(logits, "logits")
        lead = logits.shape[:-1]
        k = teacher_ids.shape[-1]
        self._per_row(teacher_ids, torch.int32, (*lead, k), "teacher_ids")
        self._per_row(teacher_logprob, torch.float32, (*lead, k), "teacher_logprob")
        self._per_row(weight, torch.float32, lead, "weight")
        if not grad and out is not None:
            raise TypeError("out is the gradient's: it needs grad=True")
        res = {}
        if loss:
            res["loss"] = _empty(*lead, dtype=torch.float32, device=self.device)
        ld_out = 0
        if grad:
            res["grad"], ld_out = self._grad_target(logits, out)
        _check(lib().dropmatch_distill(self._h, _ptr(logits), _DTYPES[logits.dtype], ld, rows, logits.shape[-1],
                                       _ptr(teacher_ids), _ptr(teacher_logprob), k, tail, temperature, _ptr(weight),
                                       _ptr(res.get("loss")), _ptr(res.get("grad")), ld_out, _stream(self.device)),
               "dropmatch_distill")
        return res

    # -- dropmatch_verify_lossless
    def verify_lossless(self, target, draft, u_accept, u_next, draft_logits=None, draft_len=None, temperature=1.0,
                        draft_temperature=1.0):
        """Drafted tokens against the target's distribution.  target[B,T,V] or, with a row behind the last drafted
        token, [B,T+1,V] and draft_logits[B,T,V] (float32 or bfloat16, as in `logprobs`; None: a drafter without a
        distribution), draft[B,T] int32, draft_len[B] int32 or None, u_accept[B,T] and u_next[B] float32 in [0,1).
        -> dict: accept_len[B], next[B] (int32), accept_prob[B,T]."""
        if target.dim() != 3 or draft.dim() != 2:
            raise TypeError("target must have shape [B, T or T+1, V] and draft [B, T]")
        B, rows, V = target.shape
        T = draft.shape[1]
        if draft.shape[0] != B or rows - T not in (0, 1):
            raise TypeError("target must have T or T+1 rows for each of draft's sequences")
        _, ld = self._rows(target, "target")
        self._per_row(draft, torch.int32, (B, T), "draft")
        self._per_row(u_accept, torch.float32, (B, T), "u_accept")
        self._per_row(u_next, torch.float32, (B,), "u_next")
        self._per_row(draft_len, torch.int32, (B,), "draft_len")
        draft_dtype, ld_draft = F32, V
        if draft_logits is not None:
            if draft_logits.shape != (B, T, V):
                raise TypeError("draft_logits must have shape [B, T, V]")
            _, ld_draft = self._rows(draft_logits, "draft_logits")
            draft_dtype = _DTYPES[draft_logits.dtype]
        dev = self.device
        out = dict(accept_len=_empty(B, dtype=torch.int32, device=dev), next=_empty(B, dtype=torch.int32, device=dev),
                   accept_prob=_empty(B, T, dtype=torch.float32, device=dev))
        _check(lib().dropmatch_verify_lossless(self._h, _ptr(target), _DTYPES[target.dtype], ld, _ptr(draft_logits),
                                               draft_dtype, ld_draft, _ptr(draft), _ptr(draft_len), B, T, rows - T, V,
                                               temperature, draft_temperature, _ptr(u_accept), _ptr(u_next),
                                               _ptr(out["accept_len"]), _ptr(out["next"]), _ptr(out["accept_prob"]),
                                               _stream(dev)), "dropmatch_verify_lossless")
        return out

    # -- dropmatch_dropout / dropmatch_dropout_grad
    def dropout(self, x, K, p, seed, seq_base=0, out=None):
        """x[B,T,d] (float32 or bfloat16) -> out[B,T,K,d]: K masked copies of every row, scaled by 1/(1-p), with the
        masks of the verify calls.  Autograd does not see this call; `dropout_grad` is its gradient."""
        if x.dim() != 3:
            raise TypeError("x must have shape [B, T, d]")
        B, T, d = x.shape
        _, ld = self._rows(x, "x")
        if out is None:
            out, ld_out = _empty(B, T, K, d, dtype=x.dtype, device=self.device), d
        else:
            if out.shape != (B, T, K, d) or out.dtype != x.dtype:
                raise TypeError("out must have shape [B, T, K, d] and x's dtype")
            ld_out = self._rows(out, "out")[1]
        _check(lib().dropmatch_dropout(self._h, _ptr(x), _DTYPES[x.dtype], ld, B, T, K, d, p, seed, seq_base, _ptr(out),
                                       ld_out, _stream(self.device)), "dropmatch_dropout")
        return out

    def dropout_grad(self, grad, p, seed, seq_base=0, out=None):
        """grad[B,T,K,d] of `dropout`'s copies -> [B,T,d]: the gradient of x, summed over the copies."""
        if grad.dim() != 4:
            raise TypeError("grad must have shape [B, T, K, d]")
        B, T, K, d = grad.shape
        _, ld = self._rows(grad, "grad")
        if out is None:
            out, ld_out = _empty(B, T, d, dtype=grad.dtype, device=self.device), d
        else:
            if out.shape != (B, T, d) or out.dtype != grad.dtype:
                raise TypeError("out must have shape [B, T, d] and grad's dtype")
            ld_out = self._rows(out, "out")[1]
        _check(lib().dropmatch_dropout_grad(self._h, _ptr(grad), _DTYPES[grad.dtype], ld, B, T, K, d, p, seed, seq_base,
                                            _ptr(out), ld_out, _stream(self.device)), "dropmatch_dropout_grad")
        return out

    # -- dropmatch_quantize_i8 / dropmatch_matmul_i8 / dropmatch_linear_i8
    def quantize_i8(self, x):
        """x[..., n] (float32 or bfloat16, as in `logprobs`) -> (q[..., n] int8, scale[...] float32): a scale for each row.
        q's rows start 16 bytes apart at least, as the products want them (q is a view of whole 16-byte rows)."""
        rows, ld = self._rows(x, "x")
        n = x.shape[-1]
        ld_q = -(-n // 16) * 16
        q = _empty(*x.shape[:-1], ld_q, dtype=torch.int8, device=self.device)
        scale = _empty(*x.shape[:-1], dtype=torch.float32, device=self.device)
        _check(lib().dropmatch_quantize_i8(self._h, _ptr(x), _DTYPES[x.dtype], ld, rows, n, _ptr(q), ld_q, _ptr(scale),
                                           _stream(self.device)), "dropmatch_quantize_i8")
        return q[..., :n], scale

    def matmul_i8(self, q, q_scale, W, w_scale, dtype=torch.float32):
        """q[..., d] and q_scale[...], W[V, d] and w_scale[V], as quantize_i8 gives them -> q W^T with the scales applied,
        [..., V] in `dtype` (float32 or bfloat16)."""
        rows, ld = self._rows_i8(q, "q")
        V, ld_w = self._weights_i8(W, w_scale, q.shape[-1])
        self._per_row(q_scale, torch.float32, q.shape[:-1], "q_scale")
        out = self._product(q.shape[:-1], V, dtype)
        _check(lib().dropmatch_matmul_i8(self._h, _ptr(q), ld, _ptr(q_scale), rows, _ptr(W), ld_w, _ptr(w_scale), V, q.shape[-1],
                                         _ptr(out), _DTYPES[dtype], V, _stream(self.device)), "dropmatch_matmul_i8")
        return out

    def linear_i8(self, x, W, w_scale, dtype=None):
        """x[..., d] (float32 or bfloat16) through W[V, d], w_scale[V] as quantize_i8 gives them: x is quantised row by row,
        then multiplied.  -> [..., V] in `dtype` (x's by default)."""
        rows, ld = self._rows(x, "x")
        d = x.shape[-1]
        V, ld_w = self._weights_i8(W, w_scale, d)
        ld_q = -(-d // 16) * 16
        scratch = _empty(rows * (ld_q + 4), dtype=torch.int8, device=self.device)      # the rows, then their scales
        out = self._product(x.shape[:-1], V, x.dtype if dtype is None else dtype)
        _check(lib().dropmatch_linear_i8(self._h, _ptr(x), _DTYPES[x.dtype], ld, rows, _ptr(W), ld_w, _ptr(w_scale), V, d,
                                         _ptr(scratch), ld_q, scratch.data_ptr() + rows * ld_q, _ptr(out), _DTYPES[out.dtype], V,
                                         _stream(self.device)), "dropmatch_linear_i8")
        return out

    def _rows_i8(self, t, what):
        """(rows, row stride) of int8 rows one stride apart."""
        if not t.is_cuda or t.dtype != torch.int8 or t.dim() < 2:
            raise TypeError(f"{what} must be a CUDA tensor [..., d] of int8")
        rows, ld = self._strided_rows(self._on_device(t, what), what)
        if rows == 1:
            ld = -(-ld // 16) * 16
        if ld % 16 or t.data_ptr() % 16:
            raise TypeError(f"{what} must have rows that start on 16-byte boundaries (see quantize_i8)")
        return rows, ld

    def _weights_i8(self, W, w_scale, d):
        if W.dim() != 2 or W.shape[1] != d:
            raise TypeError(f"W must have shape [V, {d}]")
        V, ld_w = self._rows_i8(W, "W")
        self._per_row(w_scale, torch.float32, (V,), "w_scale")
        return V, ld_w

    def _product(self, lead, V, dtype):
        if dtype not in _DTYPES:
            raise TypeError("the product's dtype must be float32 or bfloat16")
        return _empty(*lead, V, dtype=dtype, device=self.device)

    # the calls on rows are short: these checks are written for few Python-level operations
    def _on_device(self, t, what):
        if t.get_device() != self.device.index:
            raise TypeError(f"{what} must be on the context's device {self.device}")
        return t

    def _rows(self, t, what):
        """(rows, row stride) of a tensor [..., V] whose rows lie one stride apart."""
        if not t.is_cuda or t.dtype not in _DTYPES or t.dim() < 2:
            raise TypeError(f"{what} must be a CUDA tensor [..., V] of float32 or bfloat16")
        return self._strided_rows(self._on_device(t, what), what)

    @staticmethod
    def _strided_rows(t, what):
        V = t.shape[-1]
        if t.is_contiguous():
            return (t.numel() // V if V else 0), V
        if V > 1 and t.stride(-1) != 1:
            raise TypeError(f"{what} must be dense along the last dimension")
        rows, ld = 1, None
        for n, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
            if n != 1:
                if ld is None:
                    ld = stride
                elif stride != ld * rows:
                    raise TypeError(f"{what} must have one stride between rows")
            rows *= n
        ld = V if ld is None else ld
        if rows > 1 and ld < V:
            raise TypeError(f"{what} must not have overlapping rows")
        return rows, max(ld, V)

    def _per_row(self, t, dtype, shape, what):
        if t is None:
            return
        if not (t.dtype is dtype and t.get_device() == self.device.index and t.is_contiguous()):
            self._on_device(_dev(t, dtype, what), what)
        if t.shape != shape:
            raise TypeError(f"{what} must have shape {tuple(shape)}")

    def _grad_target(self, logits, out):
        if out is None:
            return _empty(*logits.shape, dtype=logits.dtype, device=self.device), logits.shape[-1]
        if out.shape != logits.shape or out.dtype != logits.dtype:
            raise TypeError("out must have the logits' shape and dtype")
        return out, self._rows(out, "out")[1]

    def _row_outputs(self, lead, tokens, n_top):
        dev, f32 = self.device, torch.float32
        out = dict(lse=_empty(*lead, dtype=f32, device=dev), entropy=_empty(*lead, dtype=f32, device=dev))
        if tokens is not None:
            self._per_row(tokens, torch.int32, lead, "tokens")
            out["logprob"] = _empty(*lead, dtype=f32, device=dev)
        if n_top > 0:
            out["top_ids"] = _empty(*lead, n_top, dtype=torch.int32, device=dev)
            out["top_logprob"] = _empty(*lead, n_top, dtype=f32, device=dev)
        return out

    @staticmethod
    def _row_pointers(out):
        get = out.get
        return (_ptr(get("logprob")), out["lse"].data_ptr(), out["entropy"].data_ptr(), _ptr(get("top_ids")),
                _ptr(get("top_logprob")))

    # -- dropmatch_verify_tree
    def verify_tree(self, H, node_token, node_parent, node_hrow, K, p, seed, seq_base=0, rule=RULE_NAIVE):
        B, N_h, _ = H.shape
        N = node_token.shape[1]
        _dev(H, self._tdtype(), "H")
        for name, t in (("node_token", node_token), ("node_parent", node_parent), ("node_hrow", node_hrow)):
            _dev(t, torch.int32, name)
        i32 = dict(dtype=torch.int32, device=self.device)
        out = dict(tokens=torch.empty((B, N_h, K), **i32), counts=torch.empty((B, N_h, K), **i32),
                   node_ok=torch.empty((B, N), **i32), best_node=torch.empty((B,), **i32),
                   accept_len=torch.empty((B,), **i32))
        _check(lib().dropmatch_verify_tree(self._h, _ptr(H), _ptr(node_token), _ptr(node_parent), _ptr(node_hrow),
                                           B, N_h, N, K, p, seed, seq_base, rule, _ptr(out["tokens"]),
                                           _ptr(out["counts"]), _ptr(out["node_ok"]), _ptr(out["best_node"]),
                                           _ptr(out["accept_len"]), _stream(self.device)), "dropmatch_verify_tree")
        return out

    def verify_tree_next(self, H, node_token, node_parent, node_hrow, K, p, seed, seq_base=0, rule=RULE_NAIVE):
        """verify_tree plus plain[B,N_h]: the undropped greedy token of every hidden row."""
        B, N_h, _ = H.shape
        N = node_token.shape[1]
        _dev(H, self._tdtype(), "H")
        for name, t in (("node_token", node_token), ("node_parent", node_parent), ("node_hrow", node_hrow)):
            _dev(t, torch.int32, name)
        i32 = dict(dtype=torch.int32, device=self.device)
        out = dict(tokens=torch.empty((B, N_h, K), **i32), counts=torch.empty((B, N_h, K), **i32),
                   node_ok=torch.empty((B, N), **i32), best_node=torch.empty((B,), **i32),
                   accept_len=torch.empty((B,), **i32), plain=torch.empty((B, N_h), **i32))
        _check(lib().dropmatch_verify_tree_next(self._h, _ptr(H), _ptr(node_token), _ptr(node_parent),
                                                _ptr(node_hrow), B, N_h, N, K, p, seed, seq_base, rule,
                                                _ptr(out["tokens"]), _ptr(out["counts"]), _ptr(out["node_ok"]),
                                                _ptr(out["best_node"]), _ptr(out["accept_len"]), _ptr(out["plain"]),
                                                _stream(self.device)), "dropmatch_verify_tree_next")
        return out

    # -- debug
    def debug_logits(self, H, row_sel, p, seed, seq_base=0):
        B, T, _ = H.shape
        _dev(H, self._tdtype(), "H"); _dev(row_sel, torch.int32, "row_sel")
        n = row_sel.shape[0]
        out = torch.empty((n, self.V), dtype=torch.float32, device=self.device)
        _check(lib().dm_debug_logits(self._h, _ptr(H), B, T, _ptr(row_sel), n, p, seed, seq_base, _ptr(out),
                                     _stream(self.device)), "dm_debug_logits")
        return out

    def debug_masks(self, B, T, K, d, p, seed, seq_base=0):
        out = torch.empty((B, T, K, (d + 31) // 32), dtype=torch.int32, device=self.device)
        _check(lib().dm_debug_masks(self._h, B, T, K, d, p, seed, seq_base, _ptr(out), _stream(self.device)),
               "dm_debug_masks")
        return out

    def debug_masked_operand(self, H, K, p, seed, seq_base=0):
        """-> [B*T*K, d] tensor of the head's dtype: every path's hidden row with its dropped elements zeroed."""
        B, T, d = H.shape
        _dev(H, self._tdtype(), "H")
        out = torch.empty((B * T * K, d), dtype=H.dtype, device=self.device)
        _check(lib().dm_debug_masked_operand(self._h, _ptr(H), B, T, K, p, seed, seq_base, _ptr(out),
                                             _stream(self.device)), "dm_debug_masked_operand")
        return out

    def debug_read_stream(self, t: torch.Tensor):
        """One read-only pass over a CUDA tensor's bytes (for measuring the read-only HBM rate)."""
        _check(lib().dm_debug_read_stream(self._h, _ptr(t), t.numel() * t.element_size(), _stream(self.device)),
               "dm_debug_read_stream")

    def device_error(self) -> int:
        code = ctypes.c_uint32()
        _check(lib().dm_device_error(self._h, _stream(self.device), ctypes.byref(code)), "dm_device_error")
        return code.value

    def debug_set_wait_limit(self, cycles: int):
        _check(lib().dm_debug_set_wait_limit(self._h, cycles), "dm_debug_set_wait_limit")

    def profile_head(self, enable: bool):
        _check(lib().dm_profile_head(self._h, int(enable)), "dm_profile_head")

    def profile_read(self):
        """-> (summed head-kernel milliseconds, number of calls) since the last read."""
        ms, n = ctypes.c_double(), ctypes.c_int()
        _check(lib().dm_profile_read(self._h, ctypes.byref(ms), ctypes.byref(n)), "dm_profile_read")
        return ms.value, n.value

    def workspace_bytes(self) -> int:
        return lib().dm_workspace_bytes(self._h)

    def last_impl(self) -> int:
        return lib().dm_last_impl(self._h)

    def last_launches(self) -> int:
        return lib().dm_last_launches(self._h)
