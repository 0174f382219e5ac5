"""Thin ctypes binding of libcospec.so (include/cospec.h).

Marshalling only: torch tensors supply device memory and the current stream,
this module turns them into pointers and sizes and calls the C ABI.  Every step
of the computation runs in the library's HIP kernels.  There is no fallback: if
the library cannot be loaded or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from . import _build

__all__ = ["lib", "verify_block", "verify_block_static", "verify_tree", "arbitrate", "CospecError", "Prepared",
           "prepare_block", "prepare_tree", "prepare_sps", "SplitBlock", "sps_block", "hybrid_mask",
           "hybrid_attention", "PagedCache", "CacheCall", "prepare_cache_append", "cache_append",
           "prepare_cache_keep", "cache_keep", "prepare_hybrid_attention_paged", "hybrid_attention_paged",
           "prepare_tree_attention", "tree_attention", "LatentCache", "prepare_latent_append", "latent_append",
           "prepare_latent_keep", "latent_keep", "prepare_latent_attention", "latent_attention",
           "prepare_latent_tree_attention", "latent_tree_attention", "prepare_expanded_attention",
           "expanded_attention", "PagePool", "PoolCall", "prepare_pages_fork", "pages_fork", "prepare_pages_reserve",
           "pages_reserve", "prepare_pages_release", "pages_release", "prepare_pages_compact", "pages_compact",
           "prepare_pages_copy", "pages_copy", "status_string", "MAX_K",
           "MAX_N", "MAX_SPLITS"]

MAX_K, MAX_N, MAX_SPLITS = 64, 256, 64
_F32, _BF16, _F8E4M3 = 0, 1, 2
_lib = None


class CospecError(RuntimeError):
    pass


class _Head(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("h", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("w1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("w2", ctypes.c_void_p),
                ("b2", ctypes.c_float)]


_FEATURE_FIELDS = ["tgt_argmax", "tgt_max", "tgt_lse", "tgt_entropy", "drf_argmax", "drf_max",
                   "drf_lse", "drf_entropy", "logp_tgt", "logp_drf", "delta", "z_tilde", "policy",
                   "accept", "tgt_candidate", "logp_action"]


class _Features(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in _FEATURE_FIELDS]


class _RL(ctypes.Structure):
    _fields_ = [("correct", ctypes.c_void_p), ("alpha", ctypes.c_float), ("beta", ctypes.c_float),
                ("effective", ctypes.c_void_p), ("in_s_acc", ctypes.c_void_p),
                ("first_mismatch", ctypes.c_void_p), ("first_reject", ctypes.c_void_p),
                ("rho", ctypes.c_void_p), ("reward", ctypes.c_void_p),
                ("round_return", ctypes.c_void_p)]


class _Options(ctypes.Structure):
    _fields_ = [("reduce_begin", ctypes.c_void_p), ("reduce_end", ctypes.c_void_p),
                ("reduce2_begin", ctypes.c_void_p), ("reduce2_end", ctypes.c_void_p),
                ("splits", ctypes.c_int32),
                ("sample_uniform", ctypes.c_void_p), ("policy_uniform", ctypes.c_void_p),
                ("rl", ctypes.POINTER(_RL)), ("hidden_row0", ctypes.c_void_p),
                ("hidden_rows", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("page", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("d", ctypes.c_int32), ("n_pages", ctypes.c_int64), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("max_pages", ctypes.c_int32)]


class _LatentCache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("page", ctypes.c_int32), ("d_c", ctypes.c_int32),
                ("n_pages", ctypes.c_int64), ("c", ctypes.c_void_p), ("r", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("table", ctypes.c_void_p), ("max_pages", ctypes.c_int32)]


class _Pool(ctypes.Structure):
    _fields_ = [("refs", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("page", ctypes.c_int32)]


class _Plane(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_bytes", ctypes.c_int64)]


class _Rope(ctypes.Structure):
    _fields_ = [("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("inv_freq", ctypes.c_void_p)]


def _event_handle(ev) -> int:
    """Raw hipEvent_t of a torch event (torch creates it at its first record)."""
    if ev.cuda_event == 0:
        ev.record()
    return ev.cuda_event


def lib():
    """The loaded library, built first if no build exists.  A build whose id (the hash
    of the sources it was compiled from) differs from the sources on disk is refused:
    the kernels it holds are not the ones in csrc/."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            _build.build()
        L = ctypes.CDLL(_build.LIB)
        P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        HP = ctypes.POINTER(_Head)
        L.cospec_build_id.restype = ctypes.c_char_p
        L.cospec_build_id.argtypes = []
        built, want = L.cospec_build_id().decode(), _build.source_hash()
        if built != want:
            raise CospecError(f"{_build.LIB} is stale: built from sources {built}, the sources on disk are "
                              f"{want}; rebuild it (python -m paper_2605_24793_amd._build)")
        L.cospec_abi_version.restype = I32
        L.cospec_abi_version.argtypes = []
        L.cospec_workspace_bytes.restype = SZ
        L.cospec_workspace_bytes.argtypes = [I32, I32, I32, I32, HP]
        L.cospec_status_string.restype = ctypes.c_char_p
        L.cospec_status_string.argtypes = [I32]
        L.cospec_verify_block_workspace_size.restype = SZ
        L.cospec_verify_block_workspace_size.argtypes = [I32, I32, I32, HP]
        L.cospec_verify_tree_workspace_size.restype = SZ
        L.cospec_verify_tree_workspace_size.argtypes = [I32, I32, I32, HP]
        L.cospec_arbitrate_workspace_size.restype = SZ
        L.cospec_arbitrate_workspace_size.argtypes = [I64, HP]
        L.cospec_verify_block.restype = I32
        L.cospec_verify_block.argtypes = [P, P, I32, I64, P, P, HP, ctypes.c_float, I32, I32, I32,
                                          P, P, ctypes.POINTER(_Features),
                                          ctypes.POINTER(_Options), P, SZ, P]
        L.cospec_verify_tree.restype = I32
        L.cospec_verify_tree.argtypes = [P, P, I32, I64, P, P, P, HP, ctypes.c_float, I32, I32,
                                         I32, P, P, P, ctypes.POINTER(_Features),
                                         ctypes.POINTER(_Options), P, SZ, P]
        L.cospec_verify_block_static.restype = I32
        L.cospec_verify_block_static.argtypes = [P, P, I32, I64, P, P, HP, ctypes.c_float, I32, I32, I32,
                                                 P, P, ctypes.POINTER(_Features), ctypes.POINTER(_Options), P]
        L.cospec_verify_block_reduce.restype = I32
        L.cospec_verify_block_reduce.argtypes = [P, P, I32, I64, P, HP, I32, I32, I32, P,
                                                 ctypes.POINTER(_Features), ctypes.POINTER(_Options),
                                                 P, SZ, P]
        L.cospec_verify_block_arbitrate.restype = I32
        L.cospec_verify_block_arbitrate.argtypes = L.cospec_verify_block.argtypes
        L.cospec_verify_block_sps_workspace_size.restype = SZ
        L.cospec_verify_block_sps_workspace_size.argtypes = [I32, I32, I32]
        L.cospec_verify_block_sps.restype = I32
        L.cospec_verify_block_sps.argtypes = [P, P, I32, I64, P, P, I32, I32, I32, P, P,
                                              ctypes.POINTER(_Features), ctypes.POINTER(_Options), P,
                                              SZ, P]
        L.cospec_hybrid_mask.restype = I32
        L.cospec_hybrid_mask.argtypes = [P, I32, I32, I32, P, P]
        L.cospec_hybrid_attention.restype = I32
        L.cospec_hybrid_attention.argtypes = [P, P, P, P, P, I32, I32, I32, I32, I32, I32, I32,
                                              ctypes.c_float, P, P]
        L.cospec_hybrid_attention_workspace_size.restype = SZ
        L.cospec_hybrid_attention_workspace_size.argtypes = [I32] * 6
        L.cospec_hybrid_attention_ws.restype = I32
        L.cospec_hybrid_attention_ws.argtypes = [P, P, P, P, P, I32, I32, I32, I32, I32, I32, I32,
                                                 ctypes.c_float, P, P, SZ, P]
        L.cospec_head_tile_groups.restype = I32
        L.cospec_head_tile_groups.argtypes = [I32, I32, I32, I32, I32, HP]
        L.cospec_arbitrate.restype = I32
        L.cospec_arbitrate.argtypes = [P, I64, P, I64, HP, ctypes.c_float, P, P, P, SZ, P]
        CP = ctypes.POINTER(_Cache)
        L.cospec_cache_append.restype = I32
        L.cospec_cache_append.argtypes = [CP, P, P, P, I64, P, I64, ctypes.POINTER(_Rope), P, I32, I32, P, I64, I32,
                                          P, P]
        L.cospec_cache_keep.restype = I32
        L.cospec_cache_keep.argtypes = [CP, P, P, I32, I32, P]
        L.cospec_paged_attention_workspace_size.restype = SZ
        L.cospec_paged_attention_workspace_size.argtypes = [CP, I32, I32, I32]
        L.cospec_hybrid_attention_paged.restype = I32
        L.cospec_hybrid_attention_paged.argtypes = [P, CP, P, P, I32, I32, I32, I32, ctypes.c_float, P, P, SZ, P]
        L.cospec_tree_attention.restype = I32
        L.cospec_tree_attention.argtypes = [P, CP, P, P, I32, I32, I32, ctypes.c_float, P, P, SZ, P]
        LP, F32 = ctypes.POINTER(_LatentCache), ctypes.c_float
        L.cospec_latent_append.restype = I32
        L.cospec_latent_append.argtypes = [LP, P, P, P, I64, P, I64, P, F32, ctypes.POINTER(_Rope), P, I32, I32, P, I64,
                                           I64, I32, P, I64, P, P, P]
        L.cospec_latent_keep.restype = I32
        L.cospec_latent_keep.argtypes = [LP, P, P, I32, I32, P]
        L.cospec_latent_attention_workspace_size.restype = SZ
        L.cospec_latent_attention_workspace_size.argtypes = [LP, I32, I32, I32]
        L.cospec_latent_attention.restype = I32
        L.cospec_latent_attention.argtypes = [P, LP, P, P, I32, I32, I32, I32, F32, P, P, SZ, P]
        L.cospec_latent_tree_attention.restype = I32
        L.cospec_latent_tree_attention.argtypes = [P, LP, P, P, I32, I32, I32, F32, P, P, SZ, P]
        L.cospec_expanded_attention.restype = I32
        L.cospec_expanded_attention.argtypes = [P, P, I64, I64, P, I64, I64, P, I64, P, P, I32, I32, I32, I32, I32, I32,
                                                F32, P, P]
        OP = ctypes.POINTER(_Pool)
        L.cospec_pages_fork.restype = I32
        L.cospec_pages_fork.argtypes = [OP, P, I32, P, P, I32, I32, P, P]
        L.cospec_pages_reserve_workspace_size.restype = SZ
        L.cospec_pages_reserve_workspace_size.argtypes = [OP, I32, I32]
        L.cospec_pages_reserve.restype = I32
        L.cospec_pages_reserve.argtypes = [OP, P, I32, P, P, I32, I32, P, P, P, SZ, P]
        L.cospec_pages_release.restype = I32
        L.cospec_pages_release.argtypes = [OP, P, I32, P, I32, P]
        L.cospec_pages_compact_workspace_size.restype = SZ
        L.cospec_pages_compact_workspace_size.argtypes = [OP]
        L.cospec_pages_compact.restype = I32
        L.cospec_pages_compact.argtypes = [OP, P, I32, I32, P, P, P, SZ, P]
        L.cospec_pages_copy.restype = I32
        L.cospec_pages_copy.argtypes = [ctypes.POINTER(_Plane), I32, I64, P, I32, P, P]
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().cospec_status_string(code).decode()


def _check(code: int, what: str):
    if code != 0:
        raise CospecError(f"{what}: {status_string(code)} ({code})")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return _BF16
    if t.dtype == torch.float32:
        return _F32
    raise TypeError(f"logits, hidden states and head weights are bf16 or f32, got {t.dtype}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _head_struct(head) -> _Head:
    w1, b1, w2, b2 = head.w1, head.b1, head.w2, head.b2
    for t in (w1, w2) + ((b1,) if b1 is not None else ()):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("head weights must be contiguous device tensors")
    return _Head(int(w1.shape[1]), int(w1.shape[0]), _dtype_code(w1), _ptr(w1), _ptr(b1),
                 _ptr(w2), float(b2))


def head_tile_groups(is_tree: bool, B: int, n: int, V: int, logit_dtype: torch.dtype, head) -> int:
    """How many workgroups share a tile of the head's first layer beside the reduction of a
    whole step (n: draft tokens of a chain, nodes of a tree); 0: not in tiles."""
    return lib().cospec_head_tile_groups(int(is_tree), int(B), int(n), int(V),
                                         _BF16 if logit_dtype == torch.bfloat16 else _F32,
                                         ctypes.byref(_head_struct(head)))


def _row_stride(t: torch.Tensor) -> int:
    """Row stride in elements of a [B, R, V] logit tensor whose rows may be padded."""
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError("logits must be [B, R, V] with unit element stride")
    if t.shape[0] > 1 and t.shape[1] > 0 and t.stride(0) != t.shape[1] * t.stride(1):
        raise ValueError("logit rows must be uniformly spaced: stride(0) == R * stride(1)")
    return int(t.stride(1))


# torch's current stream as a raw hipStream_t, without the Stream object that
# torch.cuda.current_stream() builds on every call (measured: 0.3 against 2.75 us of the 11 us
# a small call takes).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


class Prepared:
    """Pre-marshalled arguments of one verify call: outputs, features, workspace and
    are allocated once, so
    `launch()` enqueues the step with no allocation."""

    def __init__(self, fn, args_before_feats, outputs, feats, feats_struct, workspace, splits,
                 uniform=None, policy_u=None, rl=None):
        self._fn = fn
        self._args = args_before_feats
        self.outputs = outputs
        self.features = feats
        self._feats = feats_struct
        self.workspace = workspace
        self.splits = int(splits)
        self.uniform = uniform
        self.policy_u = policy_u
        self.rl = rl                    # (struct, output tensors, correct tensor) or None
        self.hidden_row0 = None         # packed hidden rows: int64 [B] device tensor, and
        self.hidden_rows = 0            # the rows of the packed array
        self._keep = []

    def _options(self, timing):
        if (timing is None and not self.splits and self.uniform is None
                and self.policy_u is None and self.rl is None and self.hidden_row0 is None):
            return None
        ev = [None] * 4 if timing is None else [None if e is None else _event_handle(e) for e in timing]
        rl = None if self.rl is None else ctypes.pointer(self.rl[0])
        return _Options(ev[0], ev[1], ev[2], ev[3], self.splits, _ptr(self.uniform),
                        _ptr(self.policy_u), rl, _ptr(self.hidden_row0), int(self.hidden_rows))

    def launch(self, timing=None):
        """Enqueue the step on torch's current stream.  `timing` = four torch events
        recorded around the target-row and the draft-row reduction launches."""
        opts = self._options(timing)
        code = self._fn(*self._args, ctypes.byref(self._feats) if self._feats is not None else None,
                        ctypes.byref(opts) if opts is not None else None,
                        _ptr(self.workspace), self.workspace.numel(), _stream())
        _check(code, self._fn.__name__)

    def result(self) -> dict:
        out = dict(self.outputs)
        out.update(self.features or {})
        if self.rl is not None:
            out.update({"rl_" + k: v for k, v in self.rl[1].items()})
        return out


def _features(alloc: bool, dev, B, RT, RD, D):
    if not alloc:
        return None, None
    i32, f32, u8 = torch.int32, torch.float32, torch.uint8
    shapes = dict(tgt_argmax=((B, RT), i32), tgt_max=((B, RT), f32), tgt_lse=((B, RT), f32),
                  tgt_entropy=((B, RT), f32), drf_argmax=((B, RD), i32), drf_max=((B, RD), f32),
                  drf_lse=((B, RD), f32), drf_entropy=((B, RD), f32), logp_tgt=((B, D), f32),
                  logp_drf=((B, D), f32), delta=((B, D), u8), z_tilde=((B, D), f32),
                  policy=((B, D), f32), accept=((B, D), u8), tgt_candidate=((B, RT), i32),
                  logp_action=((B, D), f32))
    feats = {k: torch.empty(s, dtype=t, device=dev) for k, (s, t) in shapes.items()}
    st = _Features(*[_ptr(feats[f]) for f in _FEATURE_FIELDS])
    return feats, st


def _uniforms(u: Optional[torch.Tensor], B: int, RT: int):
    if u is None:
        return None
    if tuple(u.shape) != (B, RT) or u.dtype != torch.float32 or not u.is_contiguous() or not u.is_cuda:
        raise ValueError("sample_u must be a contiguous float32 device tensor [B, target rows]")
    return u


def _policy_uniforms(u: Optional[torch.Tensor], B: int, D: int):
    if u is None:
        return None
    if tuple(u.shape) != (B, D) or u.dtype != torch.float32 or not u.is_contiguous() or not u.is_cuda:
        raise ValueError("policy_u must be a contiguous float32 device tensor [B, decisions]")
    return u


def _rl(correct: Optional[torch.Tensor], alpha: float, beta: float, B: int, K: int, dev):
    if correct is None:
        return None
    if tuple(correct.shape) != (B,) or correct.dtype != torch.uint8 or not correct.is_cuda:
        raise ValueError("correct must be a uint8 device tensor [B]")
    correct = correct.contiguous()
    outs = dict(effective=torch.empty((B, K), dtype=torch.uint8, device=dev),
                in_s_acc=torch.empty((B, K), dtype=torch.uint8, device=dev),
                first_mismatch=torch.empty(B, dtype=torch.int32, device=dev),
                first_reject=torch.empty(B, dtype=torch.int32, device=dev),
                rho=torch.empty(B, dtype=torch.float32, device=dev),
                reward=torch.empty((B, K), dtype=torch.float32, device=dev),
                round_return=torch.empty(B, dtype=torch.float32, device=dev))
    st = _RL(_ptr(correct), float(alpha), float(beta), *[_ptr(outs[k]) for k in (
        "effective", "in_s_acc", "first_mismatch", "first_reject", "rho", "reward", "round_return")])
    return st, outs, correct


def prepare_block(target, draft, draft_tokens, hidden, head, lam: float, features: bool = True,
                  splits: int = 0,
                  sample_u: Optional[torch.Tensor] = None,
                  policy_u: Optional[torch.Tensor] = None,
                  correct: Optional[torch.Tensor] = None, alpha: float = 1.0,
                  beta: float = 0.25, hidden_row0: Optional[torch.Tensor] = None) -> Prepared:
    """sample_u: one uniform per target row [B, K+1] for temperature-1 candidates
    (cospec_options.sample_uniform); None for the greedy argmax.  policy_u: one
    uniform per decision [B, K] for sampled arbitration.  correct: uint8 [B]
    rollout correctness; turns on the per-round RL statistics (returned with an
    "rl_" prefix) with failure-reward weights alpha and beta.  hidden_row0: int64 [B]
    device tensor; hidden is then a packed [rows, d] array and decision i of sequence
    b reads row hidden_row0[b] + i - 1 (cospec_options.hidden_row0)."""
    B, R, V = target.shape
    K = R - 1
    ld = _row_stride(target)
    if K > 0 and _row_stride(draft) != ld:
        raise ValueError("target and draft rows must share one stride")
    if hidden_row0 is not None:
        if tuple(hidden_row0.shape) != (B,) or hidden_row0.dtype != torch.int64 or not hidden_row0.is_cuda:
            raise ValueError("hidden_row0 must be an int64 device tensor [B]")
        if hidden.dim() != 2 or not hidden.is_contiguous():
            raise ValueError("with hidden_row0, hidden must be a contiguous [rows, d] array")
        hidden_row0 = hidden_row0.contiguous()
    packed_ok = hidden_row0 is not None or (hidden.shape[:2] == (B, K) and hidden.is_contiguous())
    if K > 0 and (tuple(draft.shape) != (B, K, V) or tuple(draft_tokens.shape) != (B, K)
                  or draft_tokens.dtype != torch.int32 or not draft_tokens.is_contiguous()
                  or not packed_ok):
        raise ValueError("shape/dtype mismatch between target, draft, draft_tokens and hidden")
    dev = target.device
    hs = _head_struct(head)
    L = lib()
    ws_bytes = L.cospec_verify_block_workspace_size(B, K, V, ctypes.byref(hs))
    if ws_bytes == 0 and B > 0:
        raise CospecError("invalid sizes for cospec_verify_block")
    workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
    outputs = dict(accept_len=torch.empty(B, dtype=torch.int32, device=dev),
                   tokens=torch.empty((B, K + 1), dtype=torch.int32, device=dev))
    feats, fst = _features(features, dev, B, K + 1, K, K)
    args = (_ptr(target), _ptr(draft) if K > 0 else None, _dtype_code(target), ld,
            _ptr(draft_tokens) if K > 0 else None, _ptr(hidden) if K > 0 else None,
            ctypes.byref(hs), float(lam), B, K, V, _ptr(outputs["accept_len"]),
            _ptr(outputs["tokens"]))
    p = Prepared(L.cospec_verify_block, args, outputs, feats, fst, workspace, splits,
                 _uniforms(sample_u, B, K + 1), _policy_uniforms(policy_u, B, K),
                 _rl(correct, alpha, beta, B, K, dev))
    if hidden_row0 is not None:
        p.hidden_row0, p.hidden_rows = hidden_row0, hidden.shape[0]
    p._keep = [hs, target, draft, draft_tokens, hidden, head]
    return p


def prepare_tree(target, draft, parent, node_tokens, hidden, head, lam: float,
                 features: bool = True, splits: int = 0,
                 sample_u: Optional[torch.Tensor] = None,
                 policy_u: Optional[torch.Tensor] = None) -> Prepared:
    """sample_u: one uniform per target row [B, N] for temperature-1 candidates;
    policy_u: one uniform per node [B, N] for sampled arbitration."""
    B, N, V = target.shape
    ld = _row_stride(target)
    if _row_stride(draft) != ld or tuple(draft.shape) != (B, N, V):
        raise ValueError("target and draft must both be [B, N, V] with one row stride")
    for t in (parent, node_tokens):
        if tuple(t.shape) != (B, N) or t.dtype != torch.int32 or not t.is_contiguous():
            raise ValueError("parent and node_tokens must be contiguous int32 [B, N]")
    if hidden.shape[:2] != (B, N) or not hidden.is_contiguous():
        raise ValueError("hidden must be contiguous [B, N, d]")
    dev = target.device
    hs = _head_struct(head)
    L = lib()
    ws_bytes = L.cospec_verify_tree_workspace_size(B, N, V, ctypes.byref(hs))
    if ws_bytes == 0 and B > 0:
        raise CospecError("invalid sizes for cospec_verify_tree")
    workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
    outputs = dict(accept_len=torch.empty(B, dtype=torch.int32, device=dev),
                   tokens=torch.empty((B, N), dtype=torch.int32, device=dev),
                   path=torch.empty((B, N), dtype=torch.int32, device=dev))
    feats, fst = _features(features, dev, B, N, N, N)
    args = (_ptr(target), _ptr(draft), _dtype_code(target), ld, _ptr(parent), _ptr(node_tokens),
            _ptr(hidden), ctypes.byref(hs), float(lam), B, N, V, _ptr(outputs["accept_len"]),
            _ptr(outputs["tokens"]), _ptr(outputs["path"]))
    p = Prepared(L.cospec_verify_tree, args, outputs, feats, fst, workspace, splits,
                 _uniforms(sample_u, B, N), _policy_uniforms(policy_u, B, N))
    p._keep = [hs, target, draft, parent, node_tokens, hidden, head]
    return p


def verify_block(target, draft, draft_tokens, hidden, head, lam: float, features: bool = True,
                 splits: int = 0,
                 sample_u: Optional[torch.Tensor] = None,
                 policy_u: Optional[torch.Tensor] = None,
                 correct: Optional[torch.Tensor] = None, alpha: float = 1.0,
                 beta: float = 0.25, hidden_row0: Optional[torch.Tensor] = None) -> dict:
    """cospec_verify_block on device tensors; returns accept_len, tokens (+ features,
    + rl_* statistics when `correct` is given)."""
    p = prepare_block(target, draft, draft_tokens, hidden, head, lam, features, splits,
                      sample_u, policy_u, correct, alpha, beta, hidden_row0)
    p.launch()
    return p.result()


def verify_block_static(target, draft, draft_tokens, hidden, head, lam: float, features: bool = True,
                        splits: int = 0, sample_u: Optional[torch.Tensor] = None) -> dict:
    """cospec_verify_block_static: the chain step on the library's static scratch buffer
    (no workspace is allocated here or in the library).  Same results as verify_block."""
    B, R, V = target.shape
    K = R - 1
    ld = _row_stride(target)
    if K > 0 and (_row_stride(draft) != ld or tuple(draft.shape) != (B, K, V)
                  or tuple(draft_tokens.shape) != (B, K) or draft_tokens.dtype != torch.int32
                  or not draft_tokens.is_contiguous() or hidden.shape[:2] != (B, K)
                  or not hidden.is_contiguous()):
        raise ValueError("shape/dtype mismatch between target, draft, draft_tokens and hidden")
    dev = target.device
    hs = _head_struct(head)
    outputs = dict(accept_len=torch.empty(B, dtype=torch.int32, device=dev),
                   tokens=torch.empty((B, K + 1), dtype=torch.int32, device=dev))
    feats, fst = _features(features, dev, B, K + 1, K, K)
    u = _uniforms(sample_u, B, K + 1)
    opts = _Options(splits=int(splits), sample_uniform=_ptr(u)) if (splits or u is not None) else None
    code = lib().cospec_verify_block_static(
        _ptr(target), _ptr(draft) if K > 0 else None, _dtype_code(target), ld,
        _ptr(draft_tokens) if K > 0 else None, _ptr(hidden) if K > 0 else None, ctypes.byref(hs), float(lam),
        B, K, V, _ptr(outputs["accept_len"]), _ptr(outputs["tokens"]),
        ctypes.byref(fst) if fst is not None else None, ctypes.byref(opts) if opts is not None else None,
        _stream())
    _check(code, "cospec_verify_block_static")
    out = dict(outputs)
    out.update(feats or {})
    return out


def verify_tree(target, draft, parent, node_tokens, hidden, head, lam: float,
                features: bool = True, splits: int = 0,
                sample_u: Optional[torch.Tensor] = None,
                policy_u: Optional[torch.Tensor] = None) -> dict:
    """cospec_verify_tree on device tensors; returns accept_len, tokens, path (+ features)."""
    p = prepare_tree(target, draft, parent, node_tokens, hidden, head, lam, features, splits,
                     sample_u, policy_u)
    p.launch()
    return p.result()


def arbitrate(hidden, head, lam: float, row_index: Optional[torch.Tensor] = None) -> dict:
    """cospec_arbitrate: head logits and threshold decisions for selected hidden rows."""
    h2 = hidden.reshape(-1, hidden.shape[-1])
    if not h2.is_contiguous():
        raise ValueError("hidden must be contiguous")
    n_rows = h2.shape[0]
    if row_index is not None and (row_index.dtype != torch.int32 or not row_index.is_contiguous()):
        raise ValueError("row_index must be contiguous int32")
    n_sel = n_rows if row_index is None else row_index.numel()
    hs = _head_struct(head)
    L = lib()
    ws = torch.empty(max(L.cospec_arbitrate_workspace_size(n_sel, ctypes.byref(hs)), 256),
                     dtype=torch.uint8, device=hidden.device)
    z = torch.empty(n_sel, dtype=torch.float32, device=hidden.device)
    acc = torch.empty(n_sel, dtype=torch.uint8, device=hidden.device)
    code = L.cospec_arbitrate(_ptr(h2), n_rows, _ptr(row_index), n_sel, ctypes.byref(hs),
                              float(lam), _ptr(z), _ptr(acc), _ptr(ws), ws.numel(), _stream())
    _check(code, "cospec_arbitrate")
    return dict(z=z, accept=acc)


class SplitBlock:
    """The chain step in two phases around the caller's arbitrator
    (cospec_verify_block_reduce, then cospec_verify_block_arbitrate).  Creating it
    enqueues phase 1; `candidates` ([B, K+1] int32) then holds the target's
    candidates the arbitrator's input needs; `arbitrate()` enqueues phase 2 on the
    hidden states and returns the results of the whole step."""

    def __init__(self, target, draft, draft_tokens, head, features: bool = True, splits: int = 0,
                 sample_u: Optional[torch.Tensor] = None):
        B, R, V = target.shape
        K = R - 1
        ld = _row_stride(target)
        if K > 0 and (_row_stride(draft) != ld or tuple(draft.shape) != (B, K, V)
                      or tuple(draft_tokens.shape) != (B, K) or draft_tokens.dtype != torch.int32
                      or not draft_tokens.is_contiguous()):
            raise ValueError("shape/dtype mismatch between target, draft and draft_tokens")
        dev = target.device
        self._hs = _head_struct(head)
        L = lib()
        ws_bytes = L.cospec_verify_block_workspace_size(B, K, V, ctypes.byref(self._hs))
        if ws_bytes == 0 and B > 0:
            raise CospecError("invalid sizes for cospec_verify_block_reduce")
        self.workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
        self.candidates = torch.empty((B, K + 1), dtype=torch.int32, device=dev)
        self.features, self._fst = _features(features, dev, B, K + 1, K, K)
        self.splits = int(splits)
        self._u = _uniforms(sample_u, B, K + 1)
        self._common = (_ptr(target), _ptr(draft) if K > 0 else None, _dtype_code(target), ld,
                        _ptr(draft_tokens) if K > 0 else None)
        self._sizes = (B, K, V)
        self._keep = [target, draft, draft_tokens, head]
        opts = _Options(splits=self.splits, sample_uniform=_ptr(self._u))
        code = L.cospec_verify_block_reduce(*self._common, ctypes.byref(self._hs), B, K, V,
                                            _ptr(self.candidates),
                                            ctypes.byref(self._fst) if self._fst is not None else None,
                                            ctypes.byref(opts), _ptr(self.workspace),
                                            self.workspace.numel(), _stream())
        _check(code, "cospec_verify_block_reduce")

    def arbitrate(self, hidden, lam: float, policy_u: Optional[torch.Tensor] = None,
                  correct: Optional[torch.Tensor] = None, alpha: float = 1.0, beta: float = 0.25,
                  hidden_row0: Optional[torch.Tensor] = None) -> dict:
        """Phase 2.  hidden: [B, K, d], or with hidden_row0 (int64 [B]) a packed
        [rows, d] array where decision i of sequence b reads row hidden_row0[b] + i - 1."""
        B, K, V = self._sizes
        dev = self.workspace.device
        if not hidden.is_contiguous():
            raise ValueError("hidden must be contiguous")
        if hidden_row0 is not None:
            if tuple(hidden_row0.shape) != (B,) or hidden_row0.dtype != torch.int64 or not hidden_row0.is_cuda:
                raise ValueError("hidden_row0 must be an int64 device tensor [B]")
            hidden_row0 = hidden_row0.contiguous()
            n_hidden = hidden.reshape(-1, hidden.shape[-1]).shape[0]
        elif K > 0 and tuple(hidden.shape[:2]) != (B, K):
            raise ValueError("hidden must be [B, K, d] without hidden_row0")
        outputs = dict(accept_len=torch.empty(B, dtype=torch.int32, device=dev),
                       tokens=torch.empty((B, K + 1), dtype=torch.int32, device=dev))
        pu = _policy_uniforms(policy_u, B, K)
        rl = _rl(correct, alpha, beta, B, K, dev)
        opts = _Options(splits=self.splits, policy_uniform=_ptr(pu),
                        rl=None if rl is None else ctypes.pointer(rl[0]),
                        hidden_row0=_ptr(hidden_row0),
                        hidden_rows=n_hidden if hidden_row0 is not None else 0)
        code = lib().cospec_verify_block_arbitrate(
            *self._common, _ptr(hidden) if K > 0 else None, ctypes.byref(self._hs), float(lam), B, K, V,
            _ptr(outputs["accept_len"]), _ptr(outputs["tokens"]),
            ctypes.byref(self._fst) if self._fst is not None else None, ctypes.byref(opts),
            _ptr(self.workspace), self.workspace.numel(), _stream())
        _check(code, "cospec_verify_block_arbitrate")
        out = dict(outputs)
        out.update(self.features or {})
        out["tgt_candidate"] = self.candidates
        if rl is not None:
            out.update({"rl_" + k: v for k, v in rl[1].items()})
        self._keep += [hidden, pu, rl, hidden_row0]
        return out


def prepare_sps(target, draft, draft_tokens, uniforms, features: bool = True,
                splits: int = 0) -> Prepared:
    """Pre-marshalled cospec_verify_block_sps (standard speculative sampling over
    chain blocks).  uniforms: float32 [B, K+1] on the device (K acceptance tests,
    then the draw of the last token).  The result holds accept_len, tokens and the
    features; `policy` holds the acceptance probabilities min(1, p_T / p_D)."""
    B, R, V = target.shape
    K = R - 1
    ld = _row_stride(target)
    if K > 0 and (_row_stride(draft) != ld or tuple(draft.shape) != (B, K, V)
                  or tuple(draft_tokens.shape) != (B, K) or draft_tokens.dtype != torch.int32
                  or not draft_tokens.is_contiguous()):
        raise ValueError("shape/dtype mismatch between target, draft and draft_tokens")
    u = _uniforms(uniforms, B, K + 1)
    if u is None:
        raise ValueError("speculative sampling needs uniforms [B, K+1]")
    dev = target.device
    L = lib()
    ws = torch.empty(max(L.cospec_verify_block_sps_workspace_size(B, K, V), 256), dtype=torch.uint8,
                     device=dev)
    outputs = dict(accept_len=torch.empty(B, dtype=torch.int32, device=dev),
                   tokens=torch.empty((B, K + 1), dtype=torch.int32, device=dev))
    feats, fst = _features(features, dev, B, K + 1, K, K)
    unwritten = {}
    if feats is not None:        # members the baseline leaves untouched (kept alive: fst points at them)
        unwritten = {k: feats.pop(k) for k in ("z_tilde", "logp_action")}
    args = (_ptr(target), _ptr(draft) if K > 0 else None, _dtype_code(target), ld,
            _ptr(draft_tokens) if K > 0 else None, _ptr(u), B, K, V, _ptr(outputs["accept_len"]),
            _ptr(outputs["tokens"]))
    p = Prepared(L.cospec_verify_block_sps, args, outputs, feats, fst, ws, splits)
    p._keep = [target, draft, draft_tokens, u, unwritten]
    return p


def sps_block(target, draft, draft_tokens, uniforms, features: bool = True, splits: int = 0) -> dict:
    """cospec_verify_block_sps on device tensors (see prepare_sps)."""
    p = prepare_sps(target, draft, draft_tokens, uniforms, features, splits)
    p.launch()
    return p.result()


def _i32(t: torch.Tensor, n: int, what: str) -> torch.Tensor:
    if tuple(t.shape) != (n,) or t.dtype != torch.int32 or not t.is_cuda:
        raise ValueError(f"{what} must be an int32 device tensor [{n}]")
    return t.contiguous()


def hybrid_mask(ctx_len: torch.Tensor, K: int, L: int) -> torch.Tensor:
    """cospec_hybrid_mask: the arbitrator's attention mask [B, L, L] (uint8, 1 = attend)."""
    B = ctx_len.shape[0]
    ctx = _i32(ctx_len, B, "ctx_len")
    out = torch.empty((B, L, L), dtype=torch.uint8, device=ctx.device)
    _check(lib().cospec_hybrid_mask(_ptr(ctx), B, int(K), int(L), _ptr(out), _stream()), "cospec_hybrid_mask")
    return out


def hybrid_attention(q, k, v, ctx_len, q_start, K: int, scale: float) -> torch.Tensor:
    """cospec_hybrid_attention: q [B, n_q, Hq, D], k and v [B, L, Hkv, D] (bf16, contiguous)
    -> [B, n_q, Hq, D] bf16, under the arbitrator's hybrid mask."""
    B, nq, Hq, D = q.shape
    L, Hkv = k.shape[1], k.shape[2]
    for t in (q, k, v):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("q, k and v must be contiguous bf16 device tensors")
    if tuple(k.shape) != (B, L, Hkv, D) or tuple(v.shape) != (B, L, Hkv, D):
        raise ValueError("k and v must be [B, L, Hkv, D]")
    ctx = _i32(ctx_len, B, "ctx_len")
    qs = _i32(q_start, B, "q_start")
    out = torch.empty_like(q)
    lb = lib()
    ws_bytes = lb.cospec_hybrid_attention_workspace_size(B, nq, L, Hq, Hkv, D)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device) if ws_bytes else None
    code = lb.cospec_hybrid_attention_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(ctx), _ptr(qs), B, nq, L, Hq, Hkv,
                                         D, int(K), float(scale), _ptr(out), _ptr(ws), ws_bytes, _stream())
    _check(code, "cospec_hybrid_attention")
    return out


class PagedCache:
    """Pages of keys and values of one attention layer (cospec_cache): k [n_pages, heads, page, d]
    and v [n_pages, heads, d, page], both bf16, or both float8_e4m3fn with f32 scales
    [n_pages, heads] (powers of two).  page is 16, 32, 64 or 128, d 64 or 128."""

    def __init__(self, k, v, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        if k.dim() != 4 or v.dim() != 4:
            raise ValueError("k must be [n_pages, heads, page, d] and v [n_pages, heads, d, page]")
        n, heads, page, d = k.shape
        if tuple(v.shape) != (n, heads, d, page) or v.dtype != k.dtype:
            raise ValueError("v must be [n_pages, heads, d, page], of k's type")
        if k.dtype == torch.float8_e4m3fn:
            self.dtype = _F8E4M3
            for t in (k_scale, v_scale):
                if t is None or tuple(t.shape) != (n, heads) or t.dtype != torch.float32:
                    raise ValueError("float8_e4m3fn pages need float32 scales [n_pages, heads]")
        elif k.dtype == torch.bfloat16:
            self.dtype = _BF16
            if k_scale is not None or v_scale is not None:
                raise ValueError("bf16 pages have no scales")
        else:
            raise TypeError(f"pages are bf16 or float8_e4m3fn, got {k.dtype}")
        for t in (k, v, k_scale, v_scale):
            if t is not None and (not t.is_cuda or not t.is_contiguous() or t.device != k.device):
                raise ValueError("pages and scales must be contiguous tensors of one device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads, self.page, self.d = int(n), int(heads), int(page), int(d)

    @classmethod
    def empty(cls, n_pages: int, heads: int, d: int, page: int = 64, dtype: torch.dtype = torch.bfloat16,
              device="cuda") -> "PagedCache":
        """A cache with nothing in it (its memory is not cleared: every place is written before
        it is read)."""
        k = torch.empty((n_pages, heads, page, d), dtype=dtype, device=device)
        v = torch.empty((n_pages, heads, d, page), dtype=dtype, device=device)
        scales = [None, None]
        if dtype == torch.float8_e4m3fn:
            scales = [torch.empty((n_pages, heads), dtype=torch.float32, device=device) for _ in range(2)]
        return cls(k, v, *scales)

    def _planes(self):
        return [self.k, self.v] + ([] if self.k_scale is None else [self.k_scale, self.v_scale])

    def _struct(self, table: torch.Tensor, B: int) -> _Cache:
        if table.dim() != 2 or table.shape[0] != B or table.dtype != torch.int32 or not table.is_contiguous():
            raise ValueError("table must be contiguous int32 [B, pages of a sequence]")
        _same_device(self.k, table)
        return _Cache(self.dtype, self.page, self.heads, self.d, self.n_pages, _ptr(self.k), _ptr(self.v),
                      _ptr(self.k_scale), _ptr(self.v_scale), _ptr(table), int(table.shape[1]))


def _same_device(first: torch.Tensor, *others: Optional[torch.Tensor]):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("every tensor of a call must be on one device")


def _on_current(dev: torch.device):
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {dev}, the current device is cuda:{torch.cuda.current_device()}")


class CacheCall:
    """Pre-marshalled arguments of one call on a paged cache: `outputs` and the workspace are
    allocated once, so `launch()` enqueues it, on torch's current stream, with no allocation.  The
    tensors it was prepared with are kept, and read anew by every launch.  Launches that may overlap in
    time (two streams, two captured graphs) need calls of their own: they would share these."""

    def __init__(self, fn, args, outputs, device, keep, workspace=None, ws_bytes=None):
        self._fn, self._device, self._keep = fn, device, keep
        self.outputs = outputs
        self.workspace = workspace
        self._args = args if ws_bytes is None else args + (_ptr(workspace), ws_bytes)
        self._index = device.index
        _on_current(device)
        self._stream = _stream()                           # where the tensors allocated here are at home

    def launch(self):
        if torch.cuda.current_device() != self._index:
            _on_current(self._device)
        stream = _stream()
        if stream != self._stream:
            # used on another stream than their own: the allocator must not hand the memory out early
            for t in (self.workspace, *self.outputs.values()):
                if t is not None:
                    t.record_stream(torch.cuda.current_stream())
        code = self._fn(*self._args, stream)
        if code:
            _check(code, self._fn.__name__)

    def result(self):
        return self.outputs


def _tokens(t: torch.Tensor, B: int, n: int, d: int, what: str) -> int:
    """Distance in elements between tokens of a [B, n, heads, d] bf16 tensor whose heads lie side
    by side (a slice of a projection's output will do)."""
    if t.dim() != 4 or tuple(t.shape[:2]) != (B, n) or t.shape[3] != d or t.dtype != torch.bfloat16 or not t.is_cuda:
        raise ValueError(f"{what} must be a bf16 device tensor [B, n, heads, {d}]")
    heads = t.shape[2]
    if t.stride(3) != 1 or (heads > 1 and t.stride(2) != d):
        raise ValueError(f"the heads of a token of {what} must lie side by side")
    if B * n <= 1:
        return max(heads * d, 8)
    ld = t.stride(1) if n > 1 else t.stride(0)
    if B > 1 and n > 1 and t.stride(0) != n * ld:
        raise ValueError(f"the tokens of {what} must be evenly spaced: stride(0) == n * stride(1)")
    return int(ld)


def _i32_kept(t: torch.Tensor, n: int, what: str) -> torch.Tensor:
    """_i32, for a call that reads the tensor anew at every launch: no copy of it will do."""
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return _i32(t, n, what)


def prepare_cache_append(cache: PagedCache, table, start, k, v, count: Optional[torch.Tensor] = None,
                         inv_freq: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                         interleaved: bool = False, q: Optional[torch.Tensor] = None) -> CacheCall:
    """Pre-marshalled cospec_cache_append: tokens k, v [B, n, heads, d] go to positions start[b] ..
    start[b] + count[b] - 1 (int32 [B]; count None: n), keys rotated with inv_freq (f32
    [rot / 2]; None: not rotated) to positions (int32 [B, n]; None: where they go).  q
    [B, n, Hq, d]: queries to rotate as well, into outputs["q"].  In float8_e4m3fn pages, positions
    behind the new ones are no longer the sequence's (their page's scale may change)."""
    if k.dim() != 4:
        raise ValueError("k must be [B, n, heads, d]")
    B, n = int(k.shape[0]), int(k.shape[1])
    ld_k, ld_v = _tokens(k, B, n, cache.d, "k"), _tokens(v, B, n, cache.d, "v")
    if k.shape[2] != cache.heads or v.shape[2] != cache.heads:
        raise ValueError(f"k and v must have the cache's {cache.heads} heads")
    cs = cache._struct(table, B)
    start = _i32_kept(start, B, "start")
    if count is not None:
        count = _i32_kept(count, B, "count")
    if positions is not None and (tuple(positions.shape) != (B, n) or positions.dtype != torch.int32
                                  or not positions.is_contiguous()):
        raise ValueError("positions must be contiguous int32 [B, n]")
    rope = None
    if inv_freq is not None:
        if inv_freq.dim() != 1 or inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be contiguous float32 [rot / 2]")
        rope = _Rope(2 * int(inv_freq.shape[0]), int(bool(interleaved)), _ptr(inv_freq))
    ld_q, Hq, out = 0, 0, None
    if q is not None:
        ld_q, Hq = _tokens(q, B, n, cache.d, "q"), int(q.shape[2])
        out = torch.empty((B, n, Hq, cache.d), dtype=torch.bfloat16, device=k.device)
    _same_device(cache.k, k, v, start, count, positions, inv_freq, q)
    args = (ctypes.byref(cs), _ptr(start), _ptr(count), _ptr(k), ld_k, _ptr(v), ld_v,
            None if rope is None else ctypes.byref(rope), _ptr(positions), B, n, _ptr(q), ld_q, Hq, _ptr(out))
    return CacheCall(lib().cospec_cache_append, args, {} if out is None else dict(q=out), cache.k.device,
                     [cache, table, start, count, k, v, inv_freq, positions, q, cs, rope])


def cache_append(cache: PagedCache, table, start, k, v, count: Optional[torch.Tensor] = None,
                 inv_freq: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                 interleaved: bool = False, q: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """cospec_cache_append (see prepare_cache_append); returns the rotated queries, if any."""
    p = prepare_cache_append(cache, table, start, k, v, count, inv_freq, positions, interleaved, q)
    p.launch()
    return p.outputs.get("q")


def prepare_cache_keep(cache: PagedCache, table, ctx_len, path) -> CacheCall:
    """Pre-marshalled cospec_cache_keep: the nodes path [B, N] (int32, as verify_tree returns
    it) of each tree at positions ctx_len[b] .. move to its front."""
    if path.dim() != 2 or path.dtype != torch.int32 or not path.is_contiguous():
        raise ValueError("path must be contiguous int32 [B, N]")
    B, N = int(path.shape[0]), int(path.shape[1])
    cs = cache._struct(table, B)
    ctx = _i32_kept(ctx_len, B, "ctx_len")
    _same_device(cache.k, ctx, path)
    return CacheCall(lib().cospec_cache_keep, (ctypes.byref(cs), _ptr(ctx), _ptr(path), B, N), {}, cache.k.device,
                     [cache, table, ctx, path, cs])


def cache_keep(cache: PagedCache, table, ctx_len, path) -> None:
    """cospec_cache_keep (see prepare_cache_keep)."""
    prepare_cache_keep(cache, table, ctx_len, path).launch()


def _attention_call(fn, q, cache, table, ctx_len, more, K, scale) -> CacheCall:
    if q.dim() != 4 or q.shape[3] != cache.d or q.dtype != torch.bfloat16 or not q.is_contiguous():
        raise ValueError(f"q must be contiguous bf16 [B, n, Hq, {cache.d}]")
    B, n, Hq = int(q.shape[0]), int(q.shape[1]), int(q.shape[2])
    cs = cache._struct(table, B)
    ctx = _i32_kept(ctx_len, B, "ctx_len")
    _same_device(cache.k, q, ctx, more)
    out = torch.empty_like(q)
    ws_bytes = lib().cospec_paged_attention_workspace_size(ctypes.byref(cs), B, n, Hq)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device) if ws_bytes else None
    args = (_ptr(q), ctypes.byref(cs), _ptr(ctx), _ptr(more), B, n, Hq) + K + (float(scale), _ptr(out))
    return CacheCall(fn, args, dict(out=out), q.device, [q, cache, table, ctx, more, cs], ws, ws_bytes)


def prepare_hybrid_attention_paged(q, cache: PagedCache, table, ctx_len, q_start, K: int, scale: float) -> CacheCall:
    """Pre-marshalled cospec_hybrid_attention_paged: q [B, n_q, Hq, d] (bf16, contiguous) at positions
    q_start[b] .. q_start[b] + n_q - 1 against the cache, under the arbitrator's hybrid mask;
    outputs["out"] has q's shape."""
    return _attention_call(lib().cospec_hybrid_attention_paged, q, cache, table, ctx_len,
                           _i32_kept(q_start, int(q.shape[0]), "q_start"), (int(K),), scale)


def hybrid_attention_paged(q, cache: PagedCache, table, ctx_len, q_start, K: int, scale: float) -> torch.Tensor:
    """cospec_hybrid_attention_paged (see prepare_hybrid_attention_paged) -> [B, n_q, Hq, d] bf16."""
    p = prepare_hybrid_attention_paged(q, cache, table, ctx_len, q_start, K, scale)
    p.launch()
    return p.outputs["out"]


def prepare_tree_attention(q, cache: PagedCache, table, ctx_len, parent, scale: float) -> CacheCall:
    """Pre-marshalled cospec_tree_attention: q [B, N, Hq, d] (bf16, contiguous) of the nodes kept at
    positions ctx_len[b] .. ctx_len[b] + N - 1, parent [B, N] as verify_tree takes it;
    outputs["out"] has q's shape."""
    if tuple(parent.shape) != tuple(q.shape[:2]) or parent.dtype != torch.int32 or not parent.is_contiguous():
        raise ValueError("parent must be contiguous int32 [B, N]")
    return _attention_call(lib().cospec_tree_attention, q, cache, table, ctx_len, parent, (), scale)


def tree_attention(q, cache: PagedCache, table, ctx_len, parent, scale: float) -> torch.Tensor:
    """cospec_tree_attention (see prepare_tree_attention) -> [B, N, Hq, d] bf16."""
    p = prepare_tree_attention(q, cache, table, ctx_len, parent, scale)
    p.launch()
    return p.outputs["out"]


# ------------------------------------------------------------------ latent vectors

_ROT = 64       # components of a latent cache's rotated keys


class LatentCache:
    """Pages of latent vectors of one attention layer (cospec_latent_cache): c [n_pages, page, d_c], bf16 or
    float8_e4m3fn with f32 scales [n_pages, page] (one a position), and r [n_pages, page, 64] bf16, the rotated
    keys.  page is 16, 32, 64 or 128, d_c 256 or 512."""

    def __init__(self, c, r, scale: Optional[torch.Tensor] = None):
        if c.dim() != 3:
            raise ValueError("c must be [n_pages, page, d_c]")
        n, page, d_c = c.shape
        if tuple(r.shape) != (n, page, _ROT) or r.dtype != torch.bfloat16:
            raise ValueError(f"r must be bf16 [n_pages, page, {_ROT}]")
        if c.dtype == torch.float8_e4m3fn:
            self.dtype = _F8E4M3
            if scale is None or tuple(scale.shape) != (n, page) or scale.dtype != torch.float32:
                raise ValueError("float8_e4m3fn latents need float32 scales [n_pages, page]")
        elif c.dtype == torch.bfloat16:
            self.dtype = _BF16
            if scale is not None:
                raise ValueError("bf16 latents have no scales")
        else:
            raise TypeError(f"latents are bf16 or float8_e4m3fn, got {c.dtype}")
        for t in (c, r, scale):
            if t is not None and (not t.is_cuda or not t.is_contiguous() or t.device != c.device):
                raise ValueError("latents, rotated keys and scales must be contiguous tensors of one device")
        self.c, self.r, self.scale = c, r, scale
        self.n_pages, self.page, self.d_c = int(n), int(page), int(d_c)

    @classmethod
    def empty(cls, n_pages: int, d_c: int, page: int = 64, dtype: torch.dtype = torch.bfloat16,
              device="cuda") -> "LatentCache":
        """A cache with nothing in it (its memory is not cleared: every place is written before
        it is read)."""
        c = torch.empty((n_pages, page, d_c), dtype=dtype, device=device)
        r = torch.empty((n_pages, page, _ROT), dtype=torch.bfloat16, device=device)
        scale = torch.empty((n_pages, page), dtype=torch.float32, device=device) if dtype == torch.float8_e4m3fn else None
        return cls(c, r, scale)

    def _struct(self, table: torch.Tensor, B: int) -> _LatentCache:
        if table.dim() != 2 or table.shape[0] != B or table.dtype != torch.int32 or not table.is_contiguous():
            raise ValueError("table must be contiguous int32 [B, pages of a sequence]")
        _same_device(self.c, table)
        return _LatentCache(self.dtype, self.page, self.d_c, self.n_pages, _ptr(self.c), _ptr(self.r),
                            _ptr(self.scale), _ptr(table), int(table.shape[1]))

    def _planes(self):
        return [self.c, self.r] + ([] if self.scale is None else [self.scale])


def _token_stride(t: torch.Tensor, what: str) -> int:
    """Distance in elements between the tokens of t [B, n, ...], evenly spaced."""
    B, n = t.shape[0], t.shape[1]
    if B * n <= 1:
        return -1                                           # one token, or none: no distance
    ld = t.stride(1) if n > 1 else t.stride(0)
    if B > 1 and n > 1 and t.stride(0) != n * ld:
        raise ValueError(f"the tokens of {what} must be evenly spaced: stride(0) == n * stride(1)")
    return int(ld)


def _token_rows(t: torch.Tensor, B: int, n: int, d: int, what: str) -> int:
    """Distance in elements between tokens of a [B, n, d] bf16 tensor."""
    if tuple(t.shape) != (B, n, d) or t.dtype != torch.bfloat16 or not t.is_cuda or t.stride(2) != 1:
        raise ValueError(f"{what} must be a bf16 device tensor [B, n, {d}] with unit element stride")
    ld = _token_stride(t, what)
    return d if ld < 0 else ld


def _head_rows(t: torch.Tensor, B: int, n: int, d: int, what: str):
    """Distances in elements between tokens, and between heads, of a [B, n, heads, d] bf16 tensor."""
    if t.dim() != 4 or tuple(t.shape[:2]) != (B, n) or t.shape[3] != d or t.dtype != torch.bfloat16 or not t.is_cuda \
            or t.stride(3) != 1:
        raise ValueError(f"{what} must be a bf16 device tensor [B, n, heads, {d}] with unit element stride")
    head = int(t.stride(2)) if t.shape[2] > 1 else d
    ld = _token_stride(t, what)
    return (head * int(t.shape[2]) if ld < 0 else ld), head


def prepare_latent_append(cache: LatentCache, table, start, c, k_r, weight: Optional[torch.Tensor] = None,
                          eps: float = 1e-6, count: Optional[torch.Tensor] = None,
                          inv_freq: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                          interleaved: bool = False, q: Optional[torch.Tensor] = None,
                          q_out: Optional[torch.Tensor] = None, dense: bool = False) -> CacheCall:
    """Pre-marshalled cospec_latent_append: tokens c [B, n, d_c] (bf16; normalised and taken times weight
    [d_c] unless that is None) and k_r [B, n, 64] go to positions start[b] .. start[b] + count[b] - 1 (int32
    [B]; count None: n), k_r rotated with inv_freq (f32 [rot / 2]; None: not rotated) to positions (int32
    [B, n]; None: where they go).  q [B, n, Hq, 64]: queries' rotated part, into outputs["q"]: q_out
    [B, n, Hq, 64] (such as the last components of the attention's queries), or a new tensor.  dense: outputs["c"]
    [B, n, d_c] and outputs["k_r"] [B, n, 64] hold the same latents and keys side by side, bf16."""
    if c.dim() != 3:
        raise ValueError("c must be [B, n, d_c]")
    B, n = int(c.shape[0]), int(c.shape[1])
    ld_c, ld_r = _token_rows(c, B, n, cache.d_c, "c"), _token_rows(k_r, B, n, _ROT, "k_r")
    cs = cache._struct(table, B)
    start = _i32_kept(start, B, "start")
    if count is not None:
        count = _i32_kept(count, B, "count")
    if positions is not None and (tuple(positions.shape) != (B, n) or positions.dtype != torch.int32
                                  or not positions.is_contiguous()):
        raise ValueError("positions must be contiguous int32 [B, n]")
    if weight is not None and (tuple(weight.shape) != (cache.d_c,) or weight.dtype != torch.bfloat16
                               or not weight.is_contiguous()):
        raise ValueError("weight must be contiguous bf16 [d_c]")
    rope = None
    if inv_freq is not None:
        if inv_freq.dim() != 1 or inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be contiguous float32 [rot / 2]")
        rope = _Rope(2 * int(inv_freq.shape[0]), int(bool(interleaved)), _ptr(inv_freq))
    ld_q = head_q = Hq = head_out = 0
    outputs = {}
    if q is not None:
        Hq = int(q.shape[2]) if q.dim() == 4 else 0
        ld_q, head_q = _head_rows(q, B, n, _ROT, "q")
        if q_out is None:
            q_out = torch.empty((B, n, Hq, _ROT), dtype=torch.bfloat16, device=c.device)
        if tuple(q_out.shape) != (B, n, Hq, _ROT):
            raise ValueError("q_out must have q's shape")
        ld_out, head_out = _head_rows(q_out, B, n, _ROT, "q_out")
        if Hq == 1:
            head_out = ld_out                               # one head: the distance of its tokens
        if B * n > 1 and ld_out != Hq * head_out:
            raise ValueError("q_out's tokens must lie one after the other")
        outputs["q"] = q_out
    elif q_out is not None:
        raise ValueError("q_out without q")
    if dense:
        outputs["c"] = torch.empty((B, n, cache.d_c), dtype=torch.bfloat16, device=c.device)
        outputs["k_r"] = torch.empty((B, n, _ROT), dtype=torch.bfloat16, device=c.device)
    _same_device(cache.c, c, k_r, weight, start, count, positions, inv_freq, q, q_out)
    args = (ctypes.byref(cs), _ptr(start), _ptr(count), _ptr(c), ld_c, _ptr(k_r), ld_r, _ptr(weight), float(eps),
            None if rope is None else ctypes.byref(rope), _ptr(positions), B, n, _ptr(q), ld_q, head_q, Hq, _ptr(q_out),
            head_out, _ptr(outputs.get("c")), _ptr(outputs.get("k_r")))
    return CacheCall(lib().cospec_latent_append, args, outputs, cache.c.device,
                     [cache, table, start, count, c, k_r, weight, inv_freq, positions, q, q_out, cs, rope])


def latent_append(cache: LatentCache, table, start, c, k_r, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  count: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
                  positions: Optional[torch.Tensor] = None, interleaved: bool = False,
                  q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, dense: bool = False) -> dict:
    """cospec_latent_append (see prepare_latent_append); returns its outputs: "q", "c" and "k_r", as far as they
    were asked for."""
    p = prepare_latent_append(cache, table, start, c, k_r, weight, eps, count, inv_freq, positions, interleaved, q, q_out,
                              dense)
    p.launch()
    return p.outputs


def prepare_latent_keep(cache: LatentCache, table, ctx_len, path) -> CacheCall:
    """Pre-marshalled cospec_latent_keep: the nodes path [B, N] (int32, as verify_tree returns
    it) of each tree at positions ctx_len[b] .. move to its front."""
    if path.dim() != 2 or path.dtype != torch.int32 or not path.is_contiguous():
        raise ValueError("path must be contiguous int32 [B, N]")
    B, N = int(path.shape[0]), int(path.shape[1])
    cs = cache._struct(table, B)
    ctx = _i32_kept(ctx_len, B, "ctx_len")
    _same_device(cache.c, ctx, path)
    return CacheCall(lib().cospec_latent_keep, (ctypes.byref(cs), _ptr(ctx), _ptr(path), B, N), {}, cache.c.device,
                     [cache, table, ctx, path, cs])


def latent_keep(cache: LatentCache, table, ctx_len, path) -> None:
    """cospec_latent_keep (see prepare_latent_keep)."""
    prepare_latent_keep(cache, table, ctx_len, path).launch()


def _latent_call(fn, q, cache, table, ctx_len, more, K, scale) -> CacheCall:
    if q.dim() != 4 or q.shape[3] != cache.d_c + _ROT or q.dtype != torch.bfloat16 or not q.is_contiguous():
        raise ValueError(f"q must be contiguous bf16 [B, n, Hq, {cache.d_c + _ROT}]")
    B, n, Hq = int(q.shape[0]), int(q.shape[1]), int(q.shape[2])
    cs = cache._struct(table, B)
    ctx = _i32_kept(ctx_len, B, "ctx_len")
    _same_device(cache.c, q, ctx, more)
    out = torch.empty((B, n, Hq, cache.d_c), dtype=torch.bfloat16, device=q.device)
    ws_bytes = lib().cospec_latent_attention_workspace_size(ctypes.byref(cs), B, n, Hq)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device) if ws_bytes else None
    args = (_ptr(q), ctypes.byref(cs), _ptr(ctx), _ptr(more), B, n, Hq) + K + (float(scale), _ptr(out))
    return CacheCall(fn, args, dict(out=out), q.device, [q, cache, table, ctx, more, cs], ws, ws_bytes)


def prepare_latent_attention(q, cache: LatentCache, table, ctx_len, q_start, K: int, scale: float) -> CacheCall:
    """Pre-marshalled cospec_latent_attention: q [B, n_q, Hq, d_c + 64] (bf16, contiguous) at positions
    q_start[b] .. q_start[b] + n_q - 1 against the latents, under the arbitrator's hybrid mask;
    outputs["out"] is [B, n_q, Hq, d_c] bf16."""
    return _latent_call(lib().cospec_latent_attention, q, cache, table, ctx_len,
                        _i32_kept(q_start, int(q.shape[0]), "q_start"), (int(K),), scale)


def latent_attention(q, cache: LatentCache, table, ctx_len, q_start, K: int, scale: float) -> torch.Tensor:
    """cospec_latent_attention (see prepare_latent_attention) -> [B, n_q, Hq, d_c] bf16."""
    p = prepare_latent_attention(q, cache, table, ctx_len, q_start, K, scale)
    p.launch()
    return p.outputs["out"]


def prepare_latent_tree_attention(q, cache: LatentCache, table, ctx_len, parent, scale: float) -> CacheCall:
    """Pre-marshalled cospec_latent_tree_attention: q [B, N, Hq, d_c + 64] (bf16, contiguous) of the nodes kept
    at positions ctx_len[b] .. ctx_len[b] + N - 1, parent [B, N] as verify_tree takes it;
    outputs["out"] is [B, N, Hq, d_c] bf16."""
    if tuple(parent.shape) != tuple(q.shape[:2]) or parent.dtype != torch.int32 or not parent.is_contiguous():
        raise ValueError("parent must be contiguous int32 [B, N]")
    return _latent_call(lib().cospec_latent_tree_attention, q, cache, table, ctx_len, parent, (), scale)


def latent_tree_attention(q, cache: LatentCache, table, ctx_len, parent, scale: float) -> torch.Tensor:
    """cospec_latent_tree_attention (see prepare_latent_tree_attention) -> [B, N, Hq, d_c] bf16."""
    p = prepare_latent_tree_attention(q, cache, table, ctx_len, parent, scale)
    p.launch()
    return p.outputs["out"]


def prepare_expanded_attention(q, k, v, k_r, ctx_len, q_start, K: int, scale: float) -> CacheCall:
    """Pre-marshalled cospec_expanded_attention: q [B, n_q, H, d + 64] (bf16, contiguous), k and v [B, L, H, d]
    (bf16; halves of one projection's heads will do) and the heads' shared rotated key k_r [B, L, 64], under the
    arbitrator's hybrid mask; outputs["out"] is [B, n_q, H, d] bf16."""
    if k.dim() != 4 or q.dim() != 4 or q.dtype != torch.bfloat16 or not q.is_contiguous() or not q.is_cuda:
        raise ValueError("q must be contiguous bf16 [B, n_q, H, d + 64] on the device, k [B, L, H, d]")
    B, n, H, L, d = int(q.shape[0]), int(q.shape[1]), int(q.shape[2]), int(k.shape[1]), int(k.shape[3])
    if q.shape[3] != d + _ROT or k.shape[2] != H or tuple(v.shape) != tuple(k.shape):
        raise ValueError("q must be [B, n_q, H, d + 64], k and v [B, L, H, d]")
    ld_k, head_k = _head_rows(k, B, L, d, "k")
    ld_v, head_v = _head_rows(v, B, L, d, "v")
    ld_r = _token_rows(k_r, B, L, _ROT, "k_r")
    ctx, qs = _i32_kept(ctx_len, B, "ctx_len"), _i32_kept(q_start, B, "q_start")
    _same_device(q, k, v, k_r, ctx, qs)
    out = torch.empty((B, n, H, d), dtype=torch.bfloat16, device=q.device)
    args = (_ptr(q), _ptr(k), ld_k, head_k, _ptr(v), ld_v, head_v, _ptr(k_r), ld_r, _ptr(ctx), _ptr(qs), B, n, L, H, d,
            int(K), float(scale), _ptr(out))
    return CacheCall(lib().cospec_expanded_attention, args, dict(out=out), q.device, [q, k, v, k_r, ctx, qs])


def expanded_attention(q, k, v, k_r, ctx_len, q_start, K: int, scale: float) -> torch.Tensor:
    """cospec_expanded_attention (see prepare_expanded_attention) -> [B, n_q, H, d] bf16."""
    p = prepare_expanded_attention(q, k, v, k_r, ctx_len, q_start, K, scale)
    p.launch()
    return p.outputs["out"]


# ------------------------------------------------------------------ the pages under the caches

class PagePool:
    """Which pages of the caches of a model's layers are in use (cospec_page_pool): refs [n_pages] int32 counts for
    each page the table entries that name it, 0: free.  One table serves all layers."""

    def __init__(self, refs: torch.Tensor, page: int):
        if refs.dim() != 1 or refs.dtype != torch.int32 or not refs.is_cuda or not refs.is_contiguous():
            raise ValueError("refs must be a contiguous int32 device tensor [n_pages]")
        self.refs, self.n_pages, self.page = refs, int(refs.shape[0]), int(page)
        self._struct = _Pool(_ptr(refs), self.n_pages, self.page)

    @classmethod
    def empty(cls, n_pages: int, page: int = 64, device="cuda") -> "PagePool":
        """A pool of free pages."""
        return cls(torch.zeros(n_pages, dtype=torch.int32, device=device), page)

    def _table(self, table: torch.Tensor, rows: Optional[int] = None):
        if table.dim() != 2 or table.dtype != torch.int32 or not table.is_contiguous() \
                or (rows is not None and table.shape[0] != rows):
            raise ValueError("table must be contiguous int32 [rows, pages of a sequence]")
        _same_device(self.refs, table)
        return int(table.shape[0]), int(table.shape[1])


class PoolCall(CacheCall):
    """Calls on a pool's pages, launched one after the other as one CacheCall."""

    def __init__(self, fn, args, outputs, device, keep, workspace=None, ws_bytes=None, then=None):
        super().__init__(fn, args, outputs, device, keep, workspace, ws_bytes)
        self._then = then

    def launch(self):
        super().launch()
        if self._then is not None:
            fn, args = self._then
            code = fn(*args, _stream())
            if code:
                _check(code, fn.__name__)


def _planes_of(pool_pages: int, page: int, caches, device):
    """The planes of the caches' pages, as the library takes them, and how many."""
    tensors = []
    for cache in caches:
        if cache.n_pages != pool_pages or cache.page != page:
            raise ValueError("every cache must have the pool's pages")
        tensors += cache._planes()
    for t in tensors:
        if t.device != device:
            raise ValueError("every tensor of a call must be on one device")
    planes = (_Plane * max(len(tensors), 1))()
    for p, t in zip(planes, tensors):
        p.data, p.page_bytes = t.data_ptr(), t[0].numel() * t.element_size()
    return planes, len(tensors)


def _copy_args(pool: PagePool, caches, pairs, count):
    planes, n = _planes_of(pool.n_pages, pool.page, caches, pool.refs.device)
    return (planes, n, pool.n_pages, _ptr(pairs), int(pairs.shape[0]), _ptr(count))


def prepare_pages_copy(pool: PagePool, caches, pairs, count: Optional[torch.Tensor] = None) -> CacheCall:
    """Pre-marshalled cospec_pages_copy: pages pairs[i, 0] -> pairs[i, 1] (int32 [n, 2]; the first count[0] of
    them if count, int32 [1], is given) in all of the caches."""
    if pairs.dim() != 2 or pairs.shape[1] != 2 or pairs.dtype != torch.int32 or not pairs.is_contiguous():
        raise ValueError("pairs must be contiguous int32 [n, 2]")
    if count is not None:
        count = _i32_kept(count, 1, "count")
    caches = list(caches)
    _same_device(pool.refs, pairs, count)
    args = _copy_args(pool, caches, pairs, count)
    return CacheCall(lib().cospec_pages_copy, args, {}, pool.refs.device, [pool, caches, pairs, count])


def pages_copy(pool: PagePool, caches, pairs, count: Optional[torch.Tensor] = None) -> None:
    """cospec_pages_copy (see prepare_pages_copy)."""
    prepare_pages_copy(pool, caches, pairs, count).launch()


def prepare_pages_fork(pool: PagePool, table, row, length) -> CacheCall:
    """Pre-marshalled cospec_pages_fork: outputs["table"] [B, pages] shares the pages of the first length[b]
    positions of row row[b] of table (int32 [B] both)."""
    rows, T = pool._table(table)
    B = int(row.shape[0])
    row, length = _i32_kept(row, B, "row"), _i32_kept(length, B, "length")
    _same_device(pool.refs, row, length)
    out = torch.empty((B, T), dtype=torch.int32, device=table.device)
    args = (ctypes.byref(pool._struct), _ptr(table), rows, _ptr(row), _ptr(length), B, T, _ptr(out))
    return CacheCall(lib().cospec_pages_fork, args, dict(table=out), pool.refs.device, [pool, table, row, length])


def pages_fork(pool: PagePool, table, row, length) -> torch.Tensor:
    """cospec_pages_fork (see prepare_pages_fork); returns the new table."""
    p = prepare_pages_fork(pool, table, row, length)
    p.launch()
    return p.outputs["table"]


def prepare_pages_reserve(pool: PagePool, table, start, n: int, count: Optional[torch.Tensor] = None,
                          caches=()) -> PoolCall:
    """Pre-marshalled cospec_pages_reserve: positions start[b] .. start[b] + count[b] - 1 (int32 [B]; count
    None: n) get pages of their sequence's own in table, and the caches' pages are copied where a sequence leaves a
    page that others share inside it.  outputs: copies [B, 2], lacking [1] (0: done; else nothing was).
    Caches that are left out have to take the copies by pages_copy before the pool's next reserve or compact and before
    new positions are written: a page that all its holders left is free."""
    B, T = pool._table(table)
    start = _i32_kept(start, B, "start")
    if count is not None:
        count = _i32_kept(count, B, "count")
    _same_device(pool.refs, start, count)
    caches = list(caches)
    dev = pool.refs.device
    copies = torch.empty((B, 2), dtype=torch.int32, device=dev)
    lacking = torch.empty(1, dtype=torch.int32, device=dev)
    L = lib()
    ws_bytes = L.cospec_pages_reserve_workspace_size(ctypes.byref(pool._struct), B, int(n))
    ws = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
    args = (ctypes.byref(pool._struct), _ptr(table), T, _ptr(start), _ptr(count), B, int(n), _ptr(copies), _ptr(lacking))
    then = (L.cospec_pages_copy, _copy_args(pool, caches, copies, None)) if caches else None
    return PoolCall(L.cospec_pages_reserve, args, dict(copies=copies, lacking=lacking), dev,
                    [pool, table, start, count, caches], ws, ws.numel(), then)


def pages_reserve(pool: PagePool, table, start, n: int, count: Optional[torch.Tensor] = None, caches=()) -> dict:
    """cospec_pages_reserve and, for the caches, cospec_pages_copy (see prepare_pages_reserve)."""
    p = prepare_pages_reserve(pool, table, start, n, count, caches)
    p.launch()
    return p.outputs


def prepare_pages_release(pool: PagePool, table, keep) -> CacheCall:
    """Pre-marshalled cospec_pages_release: gives back the pages behind each row's first keep[b] positions."""
    B, T = pool._table(table)
    keep = _i32_kept(keep, B, "keep")
    _same_device(pool.refs, keep)
    args = (ctypes.byref(pool._struct), _ptr(table), T, _ptr(keep), B)
    return CacheCall(lib().cospec_pages_release, args, {}, pool.refs.device, [pool, table, keep])


def pages_release(pool: PagePool, table, keep) -> None:
    """cospec_pages_release (see prepare_pages_release)."""
    prepare_pages_release(pool, table, keep).launch()


def prepare_pages_compact(pool: PagePool, table, caches=()) -> PoolCall:
    """Pre-marshalled cospec_pages_compact: the pages in use move to the pool's front, in table (which must hold
    every entry that names one) and in the caches.  outputs: moves [n_pages // 2, 2] and n_moves [1].  Caches that are
    left out have to take the moves by pages_copy (with n_moves) before they are used again."""
    B, T = pool._table(table)
    caches = list(caches)
    dev = pool.refs.device
    moves = torch.empty((max(pool.n_pages // 2, 1), 2), dtype=torch.int32, device=dev)
    n_moves = torch.empty(1, dtype=torch.int32, device=dev)
    L = lib()
    ws_bytes = L.cospec_pages_compact_workspace_size(ctypes.byref(pool._struct))
    ws = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
    args = (ctypes.byref(pool._struct), _ptr(table), T, B, _ptr(moves), _ptr(n_moves))
    then = (L.cospec_pages_copy, _copy_args(pool, caches, moves, n_moves)) if caches else None
    return PoolCall(L.cospec_pages_compact, args, dict(moves=moves, n_moves=n_moves), dev, [pool, table, caches], ws,
                    ws.numel(), then)


def pages_compact(pool: PagePool, table, caches=()) -> dict:
    """cospec_pages_compact and, for the caches, cospec_pages_copy (see prepare_pages_compact)."""
    p = prepare_pages_compact(pool, table, caches)
    p.launch()
    return p.outputs
