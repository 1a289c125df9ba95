"""Thin ctypes binding of libsprinter: argument marshalling only.

Every function takes CUDA ``torch`` tensors (used here purely as device buffers), passes
their pointers to the C ABI declared in ``include/sprinter.h`` and returns the output
tensors.  All arithmetic happens in the CUDA kernels of the library; there is no fallback:
if the library is missing or the device is not a compute-capability-10 GPU the call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

from . import build as _build

F32, BF16 = 0, 1
OP_SPRINTER_VERIFY, OP_REPLACE_SAMPLE, OP_SD_VERIFY, OP_SPRINTER_STEP, OP_SD_SHARD = 0, 1, 2, 3, 4
OP_VERIFIER_LABELS, OP_VERIFIER_TRAIN = 5, 6
OP_HEAD_LOSS, OP_HEAD_LOSS_GRAD, OP_VERIFIER_LABELS_HEAD, OP_VERIFIER_TRAIN8 = 7, 8, 10, 11
OP_CACHE_APPEND, OP_TREE_ATTENTION, OP_LOGITS_RULES = 12, 13, 14
PATH_AUTO, PATH_SIMT, PATH_TENSOR = 0, 1, 2

EXPORTS = [
    "spr_workspace_bytes", "spr_workspace_init", "sprinter_verify", "replace_sample", "sd_verify",
    "spr_device_status", "spr_status_string", "spr_last_cuda_error", "spr_version", "spr_sd_verify_launches",
    "spr_host_arena_bytes", "sprinter_verify_host", "replace_sample_host", "sd_verify_host",
    "spr_set_stage_events", "replace_sample_static", "sprinter_step", "sprinter_simulate",
    "sd_shard_stats", "sd_shard_decide", "sd_shard_weights", "sd_shard_draw", "sd_shard_decide_weights",
    "verifier_labels", "verifier_train_step", "spr_test_sprinter_verify", "spr_test_verifier_train_step",
    "head_loss", "head_loss_grad", "verifier_labels_head", "spr_pack8_pitch", "hidden_pack8", "hidden_unpack8",
    "verifier_train_step8", "spr_test_verifier_train_step8", "spr_test_pair_kernels",
    "cache_append", "tree_attention", "logits_rules", "spr_draft_pass_call", "spr_test_tree_attention",
]


class SprinterError(RuntimeError):
    def __init__(self, fn: str, status: int):
        L = lib()
        msg = L.spr_status_string(status).decode()
        if status == 4:
            msg += " (" + L.spr_last_cuda_error().decode() + ")"
        super().__init__(f"{fn}: status {status}: {msg}")
        self.status = status


_lib = None


def lib_path() -> str:
    return _build.LIB


def lib():
    """Loads libsprinter.so (never builds it implicitly on a machine without nvcc)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(
                f"{path} is missing: build it with `python -m paper_2502_04557_b200.build`")
        L = C.CDLL(path)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_size_t
        L.spr_workspace_bytes.restype = sz
        L.spr_workspace_bytes.argtypes = [i32] * 7
        L.spr_workspace_init.restype = i32
        L.spr_workspace_init.argtypes = [vp, sz, vp]
        L.sprinter_verify.restype = i32
        L.sprinter_verify.argtypes = [vp, vp, vp, vp, vp, f32, i32, i32, i32, i32, i32, i32,
                                      vp, vp, vp, vp, sz, vp]
        L.spr_test_sprinter_verify.restype = i32
        L.spr_test_sprinter_verify.argtypes = [vp, vp, vp, vp, vp, f32, i32, i32, i32, i32, i32,
                                               vp, vp, vp, vp, sz, vp, i32, i32, i32, i32, i32, C.c_uint]
        L.sprinter_step.restype = i32
        L.sprinter_step.argtypes = [vp, vp, vp, vp, vp, f32, i32, i32, i32, i32, vp, i64, i32, i32, vp,
                                    i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.sprinter_simulate.restype = i32
        L.sprinter_simulate.argtypes = [C.c_uint64, i64, i64, i32, f32, f32, i32, vp, vp, vp]
        L.replace_sample.restype = i32
        L.replace_sample.argtypes = [vp, i64, i32, i64, vp, vp, i32, i32, i32, vp, i32, vp, vp, sz, vp]
        L.sd_verify.restype = i32
        L.sd_verify.argtypes = [vp, vp, i64, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                vp, sz, vp]
        L.sd_shard_stats.restype = i32
        L.sd_shard_stats.argtypes = [vp, vp, i64, i32, i32, vp, i32, i32, i32, i32, vp, vp, sz, vp]
        L.sd_shard_decide.restype = i32
        L.sd_shard_decide.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.sd_shard_weights.restype = i32
        L.sd_shard_weights.argtypes = [vp, vp, i64, i32, vp, vp, i32, i32, i32, i32, vp, vp, sz, vp]
        L.sd_shard_decide_weights.restype = i32
        L.sd_shard_decide_weights.argtypes = [vp, vp, i64, i32, vp, i32, vp, vp, i32, i32, i32, i32, i32,
                                              vp, vp, vp, vp, vp, vp, sz, vp]
        L.sd_shard_draw.restype = i32
        L.sd_shard_draw.argtypes = [vp, vp, i64, i32, i32, vp, vp, i32, i32, vp, vp, i32, i32, i32, i32,
                                    vp, vp, vp, sz, vp]
        L.verifier_labels.restype = i32
        L.verifier_labels.argtypes = [vp, vp, i64, vp, i32, i32, i32, i32, i32, vp, i32, vp, vp, vp, sz, vp]
        L.verifier_train_step.restype = i32
        L.verifier_train_step.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, i32, f32, f32, f32, f32, vp, vp, sz, vp]
        L.spr_test_verifier_train_step.restype = i32
        L.spr_test_verifier_train_step.argtypes = L.verifier_train_step.argtypes + [i32, C.c_uint]
        L.head_loss.restype = i32
        L.head_loss.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, sz, vp]
        L.head_loss_grad.restype = i32
        L.head_loss_grad.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, sz, vp]
        L.verifier_labels_head.restype = i32
        L.verifier_labels_head.argtypes = [vp, vp, i32, vp, vp, i32, vp, i32, i32, i32, vp, i32, vp, vp, vp, sz, vp]
        L.spr_pack8_pitch.restype = sz
        L.spr_pack8_pitch.argtypes = [i32]
        for fn in (L.hidden_pack8, L.hidden_unpack8):
            fn.restype = i32
            fn.argtypes = [vp, i64, i32, i32, vp, vp]
        L.verifier_train_step8.restype = i32
        L.verifier_train_step8.argtypes = [vp, vp, i64, i32, vp, vp, vp, i32] + [C.c_double] * 4 + [vp, vp, sz, vp]
        L.spr_test_verifier_train_step8.restype = i32
        L.spr_test_verifier_train_step8.argtypes = L.verifier_train_step8.argtypes + [i32, C.c_uint]
        L.spr_test_pair_kernels.restype = None
        L.spr_test_pair_kernels.argtypes = [i32, C.c_uint]
        L.cache_append.restype = i32
        L.cache_append.argtypes = [vp, i64, vp, i64, vp, i64] + [i32] * 6 + [vp] * 5 + [i32, i32, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        L.tree_attention.restype = i32
        L.tree_attention.argtypes = [vp] * 3 + [i32] * 6 + [vp] * 4 + [i32] * 3 + [f32, vp, vp, sz, vp]
        L.logits_rules.restype = i32
        L.logits_rules.argtypes = [vp, i64, i32, i32, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp, vp, i32, vp, i64, i32, vp, vp, i64, vp, sz, vp]
        L.spr_draft_pass_call.restype = i32
        L.spr_draft_pass_call.argtypes = [i32, C.c_char_p]
        L.spr_test_tree_attention.restype = None
        L.spr_test_tree_attention.argtypes = [i32, C.c_uint]
        L.spr_host_arena_bytes.restype = sz
        L.spr_host_arena_bytes.argtypes = [i32, i32, i32, i32, i64, i32, i32, i32]
        L.sprinter_verify_host.restype = i32
        L.sprinter_verify_host.argtypes = [vp, vp, vp, vp, vp, f32, i32, i32, i32, i32, i32, i32,
                                           vp, vp, vp, vp, sz, vp, sz, vp]
        L.replace_sample_host.restype = i32
        L.replace_sample_host.argtypes = [vp, i64, i32, i64, vp, vp, i32, i32, i32, vp, i32, vp,
                                          vp, sz, vp, sz, vp]
        L.sd_verify_host.restype = i32
        L.sd_verify_host.argtypes = [vp, vp, i64, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                     vp, vp, sz, vp, sz, vp]
        L.replace_sample_static.restype = i32
        L.replace_sample_static.argtypes = [vp, i64, i32, i64, vp, vp, i32, i32, i32, vp, i32, vp, vp]
        L.spr_set_stage_events.restype = None
        L.spr_set_stage_events.argtypes = [vp, vp]
        L.spr_device_status.restype = i32
        L.spr_device_status.argtypes = [vp, vp]
        L.spr_status_string.restype = C.c_char_p
        L.spr_status_string.argtypes = [i32]
        L.spr_last_cuda_error.restype = C.c_char_p
        L.spr_last_cuda_error.argtypes = []
        L.spr_version.restype = i32
        L.spr_version.argtypes = []
        L.spr_sd_verify_launches.restype = i32
        L.spr_sd_verify_launches.argtypes = [i32, i32, i32, i32]
        _lib = L
    return _lib


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported element type {t.dtype}")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(fn: str, rc: int):
    if rc != 0:
        raise SprinterError(fn, rc)


def _dev(t: torch.Tensor, dtype=None, name="tensor"):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    return t


def _selectors(rows, first_reject, n: int):
    """The optional int32 [n] row selectors of a replacement draw: the kernel reads n entries of
    each, as 32-bit integers, so anything else is refused here."""
    for name, t in (("rows", rows), ("first_reject", first_reject)):
        if t is None:
            continue
        if t.dtype != torch.int32:
            raise TypeError(f"{name} must be torch.int32, got {t.dtype}")
        if t.numel() != n:
            raise ValueError(f"{name} must have one entry per draw ({n}), got {t.numel()}")
        _dev(t, torch.int32, name)


def sd_verify_launches(B: int, K: int, V: int, dt: int = BF16) -> int:
    """Kernels one sd_verify call launches for this shape."""
    return int(lib().spr_sd_verify_launches(B, K, V, dt))


def workspace_bytes(op: int, B: int, K: int = 1, V: int = 1, d: int = 1, h: int = 0, dt: int = BF16) -> int:
    return int(lib().spr_workspace_bytes(op, B, K, V, d, h, dt))


class Workspace:
    """Device scratch for the library calls, cleared once at creation."""

    def __init__(self, nbytes: int, device="cuda"):
        nbytes = max(int(nbytes), 256)
        self.buf = torch.empty((nbytes + 255) // 256 * 256, dtype=torch.uint8, device=device)
        assert self.buf.data_ptr() % 256 == 0
        _check("spr_workspace_init", lib().spr_workspace_init(_ptr(self.buf), self.buf.numel(), _stream()))

    @property
    def nbytes(self) -> int:
        return self.buf.numel()

    def device_status(self) -> int:
        """Synchronises the current stream; returns and clears the sticky device status."""
        return int(lib().spr_device_status(_ptr(self.buf), _stream()))

    @classmethod
    def for_problem(cls, B: int, K: int, V: int, d: int, h: int, dt: int, device="cuda"):
        n = max(workspace_bytes(OP_SPRINTER_VERIFY, B, K, V, d, h, dt),
                workspace_bytes(OP_REPLACE_SAMPLE, B, K, V, d, h, dt),
                workspace_bytes(OP_SD_VERIFY, B, K, V, d, h, dt),
                workspace_bytes(OP_SPRINTER_STEP, B, K, V, d, h, dt))
        return cls(n, device)


def sprinter_verify(hidden, W1, b1, W2, b2, threshold: float, ws: Workspace, path: int = PATH_AUTO,
                    want_scores: bool = True, out=None):
    """hidden [B,K,d]; W1 [h,d], b1 [h], W2 [h], b2 [1] (or W1 [d], b1 = W2 = None).

    Returns (scores f32 [B,K] or None, accept u8 [B,K], first_reject i32 [B])."""
    _dev(hidden, name="hidden")
    B, K, d = hidden.shape
    dt = _dt(hidden)
    _dev(W1, hidden.dtype, "W1")
    h = 0 if W1.dim() == 1 else W1.shape[0]
    if W1.shape[-1] != d:
        raise ValueError("W1 inner dimension must equal d")
    _dev(b2, torch.float32, "b2")
    if h:
        _dev(b1, torch.float32, "b1")
        _dev(W2, hidden.dtype, "W2")
        if b1.numel() != h or W2.numel() != h:
            raise ValueError("b1 and W2 must have h entries")
    else:
        b1 = W2 = None
    if out is None:
        scores = torch.empty((B, K), dtype=torch.float32, device=hidden.device) if want_scores else None
        accept = torch.empty((B, K), dtype=torch.uint8, device=hidden.device)
        first_reject = torch.empty((B,), dtype=torch.int32, device=hidden.device)
    else:
        scores, accept, first_reject = out
    rc = lib().sprinter_verify(_ptr(hidden), _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2), float(threshold),
                               B, K, d, h, dt, path, _ptr(scores), _ptr(accept), _ptr(first_reject),
                               _ptr(ws.buf), ws.nbytes, _stream())
    _check("sprinter_verify", rc)
    return scores, accept, first_reject


def sprinter_verify_shaped(hidden, W1, b1, W2, b2, threshold: float, ws: Workspace, bm: int = 0, bn: int = 0,
                           splits: int = 0, cluster_n: int = 0, flags: int = 0, spin_limit: int = 0, out=None):
    """Test hook (spr_test_sprinter_verify): the tensor-core verifier with a forced launch shape."""
    _dev(hidden, torch.bfloat16, "hidden")
    B, K, d = hidden.shape
    h = W1.shape[0]
    for t, ty, nm in ((W1, torch.bfloat16, "W1"), (b1, torch.float32, "b1"), (W2, torch.bfloat16, "W2"),
                      (b2, torch.float32, "b2")):
        _dev(t, ty, nm)
    if W1.shape[-1] != d or b1.numel() != h or W2.numel() != h:
        raise ValueError("W1 must be [h, d]; b1 and W2 must have h entries")
    if out is None:
        scores = torch.empty((B, K), dtype=torch.float32, device=hidden.device)
        accept = torch.empty((B, K), dtype=torch.uint8, device=hidden.device)
        first_reject = torch.empty((B,), dtype=torch.int32, device=hidden.device)
    else:
        scores, accept, first_reject = out
    rc = lib().spr_test_sprinter_verify(_ptr(hidden), _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2), float(threshold),
                                        B, K, d, h, BF16, _ptr(scores), _ptr(accept), _ptr(first_reject),
                                        _ptr(ws.buf), ws.nbytes, _stream(), bm, bn, splits, cluster_n, flags,
                                        spin_limit)
    _check("spr_test_sprinter_verify", rc)
    return scores, accept, first_reject


def sprinter_step(hidden, W1, b1, W2, b2, threshold: float, target_logits, V: int, uniforms,
                  ws: Workspace, path: int = PATH_AUTO, want_scores: bool = True, out=None):
    """sprinter_verify followed by the gated replace_sample, as one library call.

    target_logits [B, seq_stride, ldv]; uniforms f32 [B].
    Returns (scores or None, accept u8 [B,K], first_reject i32 [B], tokens i32 [B])."""
    _dev(hidden, name="hidden")
    B, K, d = hidden.shape
    dt = _dt(hidden)
    _dev(W1, hidden.dtype, "W1")
    h = 0 if W1.dim() == 1 else W1.shape[0]
    _dev(b2, torch.float32, "b2")
    if h:
        _dev(b1, torch.float32, "b1")
        _dev(W2, hidden.dtype, "W2")
    else:
        b1 = W2 = None
    _dev(target_logits, hidden.dtype, "target_logits")
    if target_logits.dim() != 3 or target_logits.shape[0] != B:
        raise ValueError("target_logits must be [B, seq_stride, ldv]")
    seq_stride, ldv = target_logits.shape[1], target_logits.shape[2]
    _dev(uniforms, torch.float32, "uniforms")
    if uniforms.numel() != B:
        raise ValueError("uniforms must have one entry per sequence")
    if out is None:
        dev = hidden.device
        scores = torch.empty((B, K), dtype=torch.float32, device=dev) if want_scores else None
        accept = torch.empty((B, K), dtype=torch.uint8, device=dev)
        first_reject = torch.empty((B,), dtype=torch.int32, device=dev)
        tokens = torch.empty((B,), dtype=torch.int32, device=dev)
    else:
        scores, accept, first_reject, tokens = out
    rc = lib().sprinter_step(_ptr(hidden), _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2), float(threshold),
                             B, K, d, h, _ptr(target_logits), ldv, V, seq_stride, _ptr(uniforms), dt, path,
                             _ptr(scores), _ptr(accept), _ptr(first_reject), _ptr(tokens),
                             _ptr(ws.buf), ws.nbytes, _stream())
    _check("sprinter_step", rc)
    return scores, accept, first_reject, tokens


def replace_sample(target_logits, V: int, uniforms, ws: Workspace, rows=None, first_reject=None,
                   K: int = 0, seq_stride: int = 1, out=None):
    """target_logits [R, ldv] (any leading shape is flattened to rows); returns tokens i32 [n]."""
    _dev(target_logits, name="target_logits")
    ldv = target_logits.shape[-1]
    R = target_logits.numel() // ldv
    _dev(uniforms, torch.float32, "uniforms")
    n = uniforms.numel()
    _selectors(rows, first_reject, n)
    tokens = torch.empty((n,), dtype=torch.int32, device=target_logits.device) if out is None else out
    if tokens.numel() != n:
        raise ValueError("tokens must have one entry per uniform")
    rc = lib().replace_sample(_ptr(target_logits), ldv, V, R, _ptr(rows), _ptr(first_reject), K,
                              seq_stride, n, _ptr(uniforms), _dt(target_logits), _ptr(tokens),
                              _ptr(ws.buf), ws.nbytes, _stream())
    _check("replace_sample", rc)
    return tokens


def sd_verify(p_logits, q_logits, V: int, draft_tokens, uniforms, ws: Workspace, extras: bool = True,
              out=None):
    """p_logits [B,Kp,ldv], q_logits [B,K,ldv], draft_tokens i32 [B,K], uniforms f32 [B,K+1].

    Returns dict(accepted_len, correction_token[, accept, p_tok, q_tok, residual_mass])."""
    _dev(p_logits, name="p_logits")
    _dev(q_logits, p_logits.dtype, "q_logits")
    B, Kp, ldv = p_logits.shape
    K = q_logits.shape[1]
    if q_logits.shape[0] != B or q_logits.shape[2] != ldv:
        raise ValueError("p_logits and q_logits disagree in batch or row stride")
    _dev(draft_tokens, torch.int32, "draft_tokens")
    _dev(uniforms, torch.float32, "uniforms")
    if tuple(draft_tokens.shape) != (B, K) or tuple(uniforms.shape) != (B, K + 1):
        raise ValueError("draft_tokens must be [B,K] and uniforms [B,K+1]")
    dev = p_logits.device
    if out is None:
        out = dict(accepted_len=torch.empty((B,), dtype=torch.int32, device=dev),
                   correction_token=torch.empty((B,), dtype=torch.int32, device=dev))
        if extras:
            out.update(accept=torch.empty((B, K), dtype=torch.uint8, device=dev),
                       p_tok=torch.empty((B, K), dtype=torch.float32, device=dev),
                       q_tok=torch.empty((B, K), dtype=torch.float32, device=dev),
                       residual_mass=torch.empty((B,), dtype=torch.float32, device=dev))
    rc = lib().sd_verify(_ptr(p_logits), _ptr(q_logits), ldv, _ptr(draft_tokens), _ptr(uniforms),
                         B, K, Kp, V, _dt(p_logits), _ptr(out["accepted_len"]),
                         _ptr(out["correction_token"]), _ptr(out.get("accept")), _ptr(out.get("p_tok")),
                         _ptr(out.get("q_tok")), _ptr(out.get("residual_mass")),
                         _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_verify", rc)
    return out


# ---------------------------------------------------------------------------- vocabulary shards


def _shard(t: torch.Tensor, dtype=None, name="tensor"):
    """A [*, rows, Vs] view whose last dimension is dense; rows may be strided (a column slice
    of a wider tensor).  Returns the row stride in elements."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    B, R, Vs = t.shape
    ldv = t.stride(1)
    if t.stride(2) != 1 or ldv < Vs or (B > 1 and t.stride(0) != R * ldv):
        raise ValueError(f"{name}: rows must be dense and equally spaced")
    return ldv


def sd_shard_stats(p_shard, q_shard, v0: int, draft_tokens, ws: Workspace, out=None):
    """Pass 1 of the vocabulary-sharded sd_verify: this shard's row statistics [B*Kp, 6] f32."""
    ldv = _shard(p_shard, name="p_shard")
    if _shard(q_shard, p_shard.dtype, "q_shard") != ldv:
        raise ValueError("p_shard and q_shard must have the same row stride")
    B, Kp, Vs = p_shard.shape
    K = q_shard.shape[1]
    _dev(draft_tokens, torch.int32, "draft_tokens")
    if out is None:
        out = torch.empty((B * Kp, 6), dtype=torch.float32, device=p_shard.device)
    rc = lib().sd_shard_stats(_ptr(p_shard), _ptr(q_shard), ldv, Vs, v0, _ptr(draft_tokens), B, K, Kp,
                              _dt(p_shard), _ptr(out), _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_shard_stats", rc)
    return out


def sd_shard_decide(all_stats, draft_tokens, uniforms, V: int, Vs: int, Kp: int, dt: int, ws: Workspace,
                    extras: bool = True, out=None):
    """Pass 2: all_stats [G, B*Kp, 6] (rank order) -> accepted_len (and accept, p_tok, q_tok)."""
    _dev(all_stats, torch.float32, "all_stats")
    _dev(draft_tokens, torch.int32, "draft_tokens")
    _dev(uniforms, torch.float32, "uniforms")
    B, K = draft_tokens.shape
    G = all_stats.shape[0]
    if tuple(all_stats.shape) != (G, B * Kp, 6) or tuple(uniforms.shape) != (B, K + 1):
        raise ValueError("all_stats must be [G,B*Kp,6] and uniforms [B,K+1]")
    dev = all_stats.device
    if out is None:
        out = dict(accepted_len=torch.empty((B,), dtype=torch.int32, device=dev))
        if extras:
            out.update(accept=torch.empty((B, K), dtype=torch.uint8, device=dev),
                       p_tok=torch.empty((B, K), dtype=torch.float32, device=dev),
                       q_tok=torch.empty((B, K), dtype=torch.float32, device=dev))
    rc = lib().sd_shard_decide(_ptr(all_stats), G, _ptr(draft_tokens), _ptr(uniforms), B, K, Kp, V, Vs, dt,
                               _ptr(out["accepted_len"]), _ptr(out.get("accept")), _ptr(out.get("p_tok")),
                               _ptr(out.get("q_tok")), _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_shard_decide", rc)
    return out


def sd_shard_weights(p_shard, q_shard, accepted_len, uniforms, ws: Workspace, out=None):
    """Pass 3: this shard's share [B, 2] f64 of every sequence's correction draw."""
    ldv = _shard(p_shard, name="p_shard")
    _shard(q_shard, p_shard.dtype, "q_shard")
    B, Kp, Vs = p_shard.shape
    K = q_shard.shape[1]
    _dev(accepted_len, torch.int32, "accepted_len")
    _dev(uniforms, torch.float32, "uniforms")
    if out is None:
        out = torch.empty((B, 2), dtype=torch.float64, device=p_shard.device)
    rc = lib().sd_shard_weights(_ptr(p_shard), _ptr(q_shard), ldv, Vs, _ptr(accepted_len), _ptr(uniforms),
                                B, K, Kp, _dt(p_shard), _ptr(out), _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_shard_weights", rc)
    return out


def sd_shard_decide_weights(p_shard, q_shard, all_stats, draft_tokens, uniforms, V: int, ws: Workspace,
                            extras: bool = True):
    """Passes 2 and 3 in one launch.  Returns (dict(accepted_len[, accept, p_tok, q_tok]), weights [B,2] f64)."""
    ldv = _shard(p_shard, name="p_shard")
    _shard(q_shard, p_shard.dtype, "q_shard")
    B, Kp, Vs = p_shard.shape
    K = q_shard.shape[1]
    _dev(all_stats, torch.float32, "all_stats")
    _dev(draft_tokens, torch.int32, "draft_tokens")
    _dev(uniforms, torch.float32, "uniforms")
    G = all_stats.shape[0]
    if tuple(all_stats.shape) != (G, B * Kp, 6) or tuple(uniforms.shape) != (B, K + 1) or \
            tuple(draft_tokens.shape) != (B, K):
        raise ValueError("all_stats must be [G,B*Kp,6], draft_tokens [B,K] and uniforms [B,K+1]")
    dev = p_shard.device
    out = dict(accepted_len=torch.empty((B,), dtype=torch.int32, device=dev))
    if extras:
        out.update(accept=torch.empty((B, K), dtype=torch.uint8, device=dev),
                   p_tok=torch.empty((B, K), dtype=torch.float32, device=dev),
                   q_tok=torch.empty((B, K), dtype=torch.float32, device=dev))
    weights = torch.empty((B, 2), dtype=torch.float64, device=dev)
    rc = lib().sd_shard_decide_weights(_ptr(p_shard), _ptr(q_shard), ldv, Vs, _ptr(all_stats), G, _ptr(draft_tokens),
                                       _ptr(uniforms), B, K, Kp, V, _dt(p_shard), _ptr(out["accepted_len"]),
                                       _ptr(out.get("accept")), _ptr(out.get("p_tok")), _ptr(out.get("q_tok")),
                                       _ptr(weights), _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_shard_decide_weights", rc)
    return out, weights


def sd_shard_draw(p_shard, q_shard, v0: int, all_weights, all_stats, rank: int, accepted_len, uniforms,
                  ws: Workspace, extras: bool = True, out=None):
    """Pass 4: correction_token [B] (-1 unless this shard holds the token) and residual_mass."""
    ldv = _shard(p_shard, name="p_shard")
    _shard(q_shard, p_shard.dtype, "q_shard")
    B, Kp, Vs = p_shard.shape
    K = q_shard.shape[1]
    _dev(all_weights, torch.float64, "all_weights")
    _dev(all_stats, torch.float32, "all_stats")
    G = all_weights.shape[0]
    if tuple(all_weights.shape) != (G, B, 2) or tuple(all_stats.shape) != (G, B * Kp, 6):
        raise ValueError("all_weights must be [G,B,2] and all_stats [G,B*Kp,6]")
    dev = p_shard.device
    if out is None:
        out = dict(correction_token=torch.empty((B,), dtype=torch.int32, device=dev))
        if extras:
            out["residual_mass"] = torch.empty((B,), dtype=torch.float32, device=dev)
    rc = lib().sd_shard_draw(_ptr(p_shard), _ptr(q_shard), ldv, Vs, v0, _ptr(all_weights), _ptr(all_stats),
                             G, rank, _ptr(accepted_len), _ptr(uniforms), B, K, Kp, _dt(p_shard),
                             _ptr(out["correction_token"]), _ptr(out.get("residual_mass")),
                             _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_shard_draw", rc)
    return out


# ---------------------------------------------------------------------------- fitting the verifier


def verifier_labels(p_logits, q_logits, V: int, draft_tokens, lambdas, ws: Workspace, want_ratio: bool = True):
    """p_logits [B,Kp,ldv], q_logits [B,K,ldv], draft_tokens i32 [B,K]; lambdas: up to 8 floats.

    Returns (labels u8 [len(lambdas),B,K], ratio f32 [B,K] or None) with ratio = q(x)/p(x)."""
    _dev(p_logits, name="p_logits")
    _dev(q_logits, p_logits.dtype, "q_logits")
    B, Kp, ldv = p_logits.shape
    K = q_logits.shape[1]
    _dev(draft_tokens, torch.int32, "draft_tokens")
    if q_logits.shape[0] != B or q_logits.shape[2] != ldv or tuple(draft_tokens.shape) != (B, K):
        raise ValueError("shapes of p_logits, q_logits and draft_tokens disagree")
    lam = (C.c_float * len(lambdas))(*[float(x) for x in lambdas])
    dev = p_logits.device
    labels = torch.empty((len(lambdas), B, K), dtype=torch.uint8, device=dev)
    ratio = torch.empty((B, K), dtype=torch.float32, device=dev) if want_ratio else None
    rc = lib().verifier_labels(_ptr(p_logits), _ptr(q_logits), ldv, _ptr(draft_tokens), B, K, Kp, V,
                               _dt(p_logits), C.cast(lam, C.c_void_p), len(lambdas), _ptr(labels), _ptr(ratio),
                               _ptr(ws.buf), ws.nbytes, _stream())
    _check("verifier_labels", rc)
    return labels, ratio


def verifier_train_step(hidden, labels, theta, adam_m, adam_v, t: int, lr: float, ws: Workspace,
                        beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, loss=None,
                        test_flags: int = 0, spin_limit: int = 0):
    """One Adam step on the mean BCE loss of sigmoid(b + w.s): hidden [N,d], labels u8 [N], theta /
    adam_m / adam_v f32 [d+1] (updated in place).  Returns the loss before the step (f32 [1]).
    test_flags / spin_limit: the test hook spr_test_verifier_train_step instead of the public call."""
    _dev(hidden, name="hidden")
    N, d = hidden.shape
    _dev(labels, torch.uint8, "labels")
    for name, a in (("theta", theta), ("adam_m", adam_m), ("adam_v", adam_v)):
        _dev(a, torch.float32, name)
        if a.numel() != d + 1:
            raise ValueError(f"{name} must have d + 1 entries")
    if labels.numel() != N:
        raise ValueError("labels must have one entry per hidden state")
    if loss is None:
        loss = torch.empty((1,), dtype=torch.float32, device=hidden.device)
    if test_flags or spin_limit:
        rc = lib().spr_test_verifier_train_step(_ptr(hidden), _ptr(labels), N, d, _dt(hidden), _ptr(theta),
                                                _ptr(adam_m), _ptr(adam_v), t, lr, beta1, beta2, eps, _ptr(loss),
                                                _ptr(ws.buf), ws.nbytes, _stream(), test_flags, spin_limit)
    else:
        rc = lib().verifier_train_step(_ptr(hidden), _ptr(labels), N, d, _dt(hidden), _ptr(theta), _ptr(adam_m),
                                       _ptr(adam_v), t, lr, beta1, beta2, eps, _ptr(loss), _ptr(ws.buf), ws.nbytes,
                                       _stream())
    _check("verifier_train_step", rc)
    return loss


# ---------------------------------------------------------------------------- heads and 8-bit states
#
# These calls may take a few microseconds on the GPU, so their checks are kept short: addresses are passed as
# plain integers, and devices are compared by index.


_INT_MAX = 0x7fffffff
_PACK8_MOST = 1 << 20          # elements of a packed row


def _on(device: int, dtype, name: str, t: torch.Tensor) -> int:
    """Address of a contiguous tensor of this type on this device."""
    if t.get_device() == device and t.dtype == dtype and t.is_contiguous():
        return t.data_ptr()
    if t.get_device() != device:
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the current device is cuda:{device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    raise ValueError(f"{name} must be contiguous")


def _result(device: int, t, shape, dtype, name: str):
    """An output tensor and its address: the caller's, checked, or a new one."""
    if t is None:
        t = torch.empty(shape, dtype=dtype, device=torch.device("cuda", device))
        return t, t.data_ptr()
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    return t, _on(device, dtype, name, t)


def _ws(device: int, ws: "Workspace"):
    if ws.buf.get_device() != device:
        raise ValueError(f"the workspace is on cuda:{ws.buf.get_device()}, the current device is cuda:{device}")
    return ws.buf.data_ptr(), ws.buf.numel()


def _raw_stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _head(device, hidden, W, tokens, name="hidden", W_name="W", token_name="targets"):
    """Checks hidden [N,d], W [V,d] and int32 tokens [N]; returns (N, d, V, their addresses, dt)."""
    dtype = hidden.dtype
    dt = _dt(hidden)
    h, w = _on(device, dtype, name, hidden), _on(device, dtype, W_name, W)
    t = _on(device, torch.int32, token_name, tokens)
    if hidden.dim() != 2 or W.dim() != 2 or W.shape[1] != hidden.shape[1]:
        raise ValueError(f"{name} must be [N,d] and {W_name} [V,d]")
    N, d = hidden.shape
    if tokens.numel() != N:
        raise ValueError(f"{token_name} must have one entry per hidden state")
    V = W.shape[0]
    if N > _INT_MAX or d > _INT_MAX or V > _INT_MAX:      # ctypes would cut them to 32 bits
        raise ValueError(f"{name} [N,d] and {W_name} [V,d] must have N, d and V below 2^31")
    return N, d, V, h, w, t, dt


def head_loss(hidden, W, targets, ws: Workspace, want_lse: bool = True, out=None):
    """Softmax cross entropy of hidden [N,d] under the head W [V,d]; targets i32 [N], negative = padding.

    Returns (loss f32 [N], lse f32 [N] or None); out: the same two tensors.  No autograd graph is recorded, whether or not
    hidden and W require gradients: those come from head_loss_grad."""
    dev = torch.cuda.current_device()
    N, d, V, h, w, t, dt = _head(dev, hidden, W, targets)
    loss, lse = (None, None) if out is None else out
    loss, a = _result(dev, loss, (N,), torch.float32, "loss")
    lse, b = _result(dev, lse, (N,), torch.float32, "lse") if want_lse or lse is not None else (None, None)
    p, n = _ws(dev, ws)
    rc = lib().head_loss(h, w, t, N, d, V, dt, a, b, p, n, _raw_stream(dev))
    if rc != 0:
        _check("head_loss", rc)
    return loss, lse


def head_loss_grad(hidden, W, targets, lse, grad_loss, ws: Workspace, want_hidden: bool = True, want_W: bool = True,
                   out=None):
    """Gradient of sum(grad_loss * loss) of head_loss; lse as head_loss returned it, grad_loss f32 [N].

    Returns (d_hidden [N,d] or None, d_W [V,d] or None) in the operands' type; out: the same two tensors.  They are returned,
    not added to hidden.grad and W.grad."""
    dev = torch.cuda.current_device()
    N, d, V, h, w, t, dt = _head(dev, hidden, W, targets)
    z, g = _on(dev, torch.float32, "lse", lse), _on(dev, torch.float32, "grad_loss", grad_loss)
    if lse.numel() != N or grad_loss.numel() != N:
        raise ValueError("lse and grad_loss must have one entry per hidden state")
    d_hidden, d_W = (None, None) if out is None else out
    d_hidden, a = _result(dev, d_hidden, (N, d), hidden.dtype, "d_hidden") if want_hidden else (None, None)
    d_W, b = _result(dev, d_W, (V, d), hidden.dtype, "d_W") if want_W else (None, None)
    if d_hidden is None and d_W is None:
        raise ValueError("at least one of the two gradients must be wanted")
    if N == 0 and d_W is None:
        return d_hidden, None
    p, n = _ws(dev, ws)
    rc = lib().head_loss_grad(h, w, t, z, g, N, d, V, dt, a, b, p, n, _raw_stream(dev))
    if rc != 0:
        _check("head_loss_grad", rc)
    return d_hidden, d_W


def verifier_labels_head(p_hidden, p_W, q_hidden, q_W, draft_tokens, lambdas, ws: Workspace, want_ratio: bool = True):
    """verifier_labels from hidden states and heads: p_hidden [N,dp], p_W [V,dp] of the target, q_hidden
    [N,dq], q_W [V,dq] of the draft; draft_tokens i32 [N]; lambdas: up to 8 floats.

    Returns (labels u8 [len(lambdas),N], ratio f32 [N] or None) with ratio = q(x)/p(x)."""
    dev = torch.cuda.current_device()
    N, dp, V, ph, pw, x, dt = _head(dev, p_hidden, p_W, draft_tokens, "p_hidden", "p_W", "draft_tokens")
    _, dq, Vq, qh, qw, _, dtq = _head(dev, q_hidden, q_W, draft_tokens, "q_hidden", "q_W", "draft_tokens")
    if V != Vq:
        raise ValueError("the two heads must have one vocabulary")
    if dt != dtq:
        raise TypeError("p_hidden and q_hidden must have one type")
    lam = (C.c_float * len(lambdas))(*lambdas)
    labels, a = _result(dev, None, (len(lambdas), N), torch.uint8, "labels")
    ratio, b = _result(dev, None, (N,), torch.float32, "ratio") if want_ratio else (None, None)
    p, n = _ws(dev, ws)
    rc = lib().verifier_labels_head(ph, pw, dp, qh, qw, dq, x, N, V, dt, lam, len(lambdas), a, b, p, n,
                                    _raw_stream(dev))
    if rc != 0:
        _check("verifier_labels_head", rc)
    return labels, ratio


def pack8_pitch(d: int) -> int:
    """Bytes of a packed row of d elements."""
    return int(lib().spr_pack8_pitch(d))


def _packed(device: int, packed, d: int):
    p = _on(device, torch.uint8, "packed", packed)
    if d > _PACK8_MOST:
        raise ValueError(f"packed rows have at most 2^20 elements, got {d}")
    if d <= 0 or packed.dim() != 2 or packed.shape[1] != (d + (d + 31) // 32 + 15) // 16 * 16:
        raise ValueError(f"packed must be [N, {pack8_pitch(d)}] for d = {d}, got {tuple(packed.shape)}")
    return packed.shape[0], p


def _rows(hidden):
    N, d = hidden.shape
    if d > _PACK8_MOST:            # ctypes would cut it to 32 bits
        raise ValueError(f"packed rows have at most 2^20 elements, got {d}")
    return N, d


def hidden_pack8(hidden, out=None):
    """hidden [N,d] in 8 bits with an exponent per 32 elements: u8 [N, pack8_pitch(d)]."""
    dev = torch.cuda.current_device()
    dt = _dt(hidden)
    h = _on(dev, hidden.dtype, "hidden", hidden)
    N, d = _rows(hidden)
    packed, p = _result(dev, out, (N, (d + (d + 31) // 32 + 15) // 16 * 16), torch.uint8, "packed")
    rc = lib().hidden_pack8(h, N, d, dt, p, _raw_stream(dev))
    if rc != 0:
        _check("hidden_pack8", rc)
    return packed


def hidden_unpack8(packed, d: int, dtype=torch.bfloat16, out=None):
    """The values [N,d] that packed rows stand for (exact in bf16 and fp32)."""
    dev = torch.cuda.current_device()
    N, p = _packed(dev, packed, d)
    hidden, h = _result(dev, out, (N, d), dtype, "hidden")
    rc = lib().hidden_unpack8(p, N, d, _dt(hidden), h, _raw_stream(dev))
    if rc != 0:
        _check("hidden_unpack8", rc)
    return hidden


def verifier_train_step8(packed, d: int, labels, theta, adam_m, adam_v, t: int, lr: float, ws: Workspace,
                         beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, loss=None,
                         test_flags: int = 0, spin_limit: int = 0):
    """verifier_train_step on hidden states kept in 8 bits: packed u8 [N, pack8_pitch(d)].
    test_flags / spin_limit: the test hook spr_test_verifier_train_step8 instead of the public call."""
    dev = torch.cuda.current_device()
    N, p = _packed(dev, packed, d)
    y = _on(dev, torch.uint8, "labels", labels)
    w, m, v = (_on(dev, torch.float32, name, a) for name, a in (("theta", theta), ("adam_m", adam_m), ("adam_v", adam_v)))
    if theta.numel() != d + 1 or adam_m.numel() != d + 1 or adam_v.numel() != d + 1:
        raise ValueError("theta, adam_m and adam_v must have d + 1 entries")
    if labels.numel() != N:
        raise ValueError("labels must have one entry per hidden state")
    loss, a = _result(dev, loss, (1,), torch.float32, "loss")
    wsp, n = _ws(dev, ws)
    args = (p, y, N, d, w, m, v, t, lr, beta1, beta2, eps, a, wsp, n, _raw_stream(dev))
    if test_flags or spin_limit:
        rc = lib().spr_test_verifier_train_step8(*args, test_flags, spin_limit)
    else:
        rc = lib().verifier_train_step8(*args)
    if rc != 0:
        _check("verifier_train_step8", rc)
    return loss


# ---------------------------------------------------------------------------- the target's pass over drafted tokens


# arguments of the three calls of a draft pass, 64 bits each
_APPEND_ARGS, _ATTENTION_ARGS, _RULES_ARGS = struct.Struct("29q").pack, struct.Struct("16qd4q").pack, struct.Struct("25q").pack


def _optional(device: int, t, dtype, shape, name: str):
    """Address of an optional tensor of this shape, or 0."""
    if t is None:
        return 0
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    return _on(device, dtype, name, t)


def _caches(device: int, k_cache, v_cache, page_table, dtype, B: int, D: int):
    """(addresses, Hkv, page_size, num_pages, max_pages) of paged caches [num_pages, Hkv, page_size, D]."""
    shape, pages = k_cache.shape, page_table.shape
    if len(shape) != 4 or shape != v_cache.shape or shape[3] != D:
        raise ValueError(f"k_cache and v_cache must be [num_pages, Hkv, page_size, {D}]")
    if len(pages) != 2 or pages[0] != B:
        raise ValueError(f"page_table must be [{B}, max_pages]")
    k, v = _on(device, dtype, "k_cache", k_cache), _on(device, dtype, "v_cache", v_cache)
    table = _on(device, torch.int32, "page_table", page_table)
    num_pages, Hkv, page_size, _ = shape
    max_pages = pages[1]
    if (num_pages | Hkv | page_size | max_pages) > _INT_MAX:
        raise ValueError("caches and page_table must have sizes below 2^31")
    return k, v, table, Hkv, page_size, num_pages, max_pages


def _node_rows(device: int, t, dtype, shape, name: str):
    """Address and distance between nodes (in elements) of [B,T,H,D], dense but for that distance: a projection that gives
    queries, keys and values side by side is read where it is."""
    if t.shape != shape:
        raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    B, T, H, D = shape
    if t.is_contiguous():
        return _on(device, dtype, name, t), H * D
    b, n, h, d = t.stride()
    stride = n if T > 1 else b if B > 1 else H * D
    if (d != 1 and D > 1) or (h != D and H > 1) or stride < H * D or (T > 1 and B > 1 and b != T * n):
        raise ValueError(f"{name} must have dense heads and one distance between nodes, got strides {t.stride()}")
    if t.get_device() != device or t.dtype != dtype:
        _on(device, dtype, name, t)             # (says which)
    return t.data_ptr(), stride


def cache_append(k, v, k_cache, v_cache, page_table, lens, ws: Workspace, q=None, inv_freq=None, interleaved: bool = False,
                 counts=None, parents=None, slots=None, q_out=None):
    """Puts the keys and values k, v [B,T,Hkv,D] of T nodes per sequence into a paged cache, keys (and the queries
    q [B,T,Hq,D]) rotated by their positions.

    k_cache, v_cache [num_pages,Hkv,page_size,D]; page_table i32 [B,max_pages]; lens i32 [B] tokens in the cache before;
    inv_freq f32 [rot/2] (None: no rotation); counts i32 [B], parents i32 [B,T] (None: a chain), slots i32 [B,T]: see
    include/sprinter.h.  q, k, v may be parts of one tensor [B,T,Hq+2*Hkv,D].  Returns q_out, or None without q."""
    dev = torch.cuda.current_device()
    dtype, dt = k.dtype, _dt(k)
    if k.dim() != 4:
        raise ValueError("k must be [B,T,Hkv,D]")
    B, T, Hkv, D = shape = tuple(k.shape)
    if (B | T | Hkv | D) > _INT_MAX:
        raise ValueError("k [B,T,Hkv,D] must have sizes below 2^31")
    kc, vc, table, heads, page_size, num_pages, max_pages = _caches(dev, k_cache, v_cache, page_table, dtype, B, D)
    if heads != Hkv:
        raise ValueError(f"the caches have {heads} heads, k has {Hkv}")
    ka, ks = _node_rows(dev, k, dtype, shape, "k")
    va, vs = _node_rows(dev, v, dtype, shape, "v")
    qa, qs, Hq, oa = 0, 0, 0, 0
    if q is not None:
        if q.dim() != 4 or q.shape[2] > _INT_MAX:
            raise ValueError("q must be [B,T,Hq,D]")
        Hq = q.shape[2]
        qa, qs = _node_rows(dev, q, dtype, (B, T, Hq, D), "q")
    elif q_out is not None:
        raise ValueError("q_out needs q")
    rot, fa = 0, 0
    if inv_freq is not None:
        fa, rot = _on(dev, torch.float32, "inv_freq", inv_freq), 2 * inv_freq.numel()
        if rot > D:
            raise ValueError(f"inv_freq must have at most D / 2 = {D // 2} entries, got {inv_freq.numel()}")
    n = _optional(dev, lens, torch.int32, (B,), "lens")
    c = _optional(dev, counts, torch.int32, (B,), "counts")
    par = _optional(dev, parents, torch.int32, (B, T), "parents")
    sl = _optional(dev, slots, torch.int32, (B, T), "slots")
    p, size = _ws(dev, ws)
    if q is not None:
        q_out, oa = _result(dev, q_out, (B, T, Hq, D), dtype, "q_out")
    rc = lib().spr_draft_pass_call(OP_CACHE_APPEND, _APPEND_ARGS(
        qa, qs, ka, ks, va, vs, B, T, Hq, Hkv, D, dt, n, c, par, sl, fa, rot, bool(interleaved), table, max_pages, num_pages, page_size,
        kc, vc, oa, p, size, _raw_stream(dev)))
    if rc != 0:
        _check("cache_append", rc)
    return q_out


def tree_attention(q, k_cache, v_cache, page_table, lens, ws: Workspace, scale=None, counts=None, parents=None, out=None):
    """Attention of q [B,T,Hq,D], T nodes per sequence, over the paged cache that cache_append has put them into: each
    sees the lens[b] tokens before the pass and the nodes on its path.  scale: 1 / sqrt(D) unless given.

    counts i32 [B] and parents i32 [B,T] as for cache_append.  Returns out [B,T,Hq,D]; out may be q."""
    dev = torch.cuda.current_device()
    dtype, dt = q.dtype, _dt(q)
    if q.dim() != 4:
        raise ValueError("q must be [B,T,Hq,D]")
    B, T, Hq, D = shape = tuple(q.shape)
    if (B | T | Hq | D) > _INT_MAX:
        raise ValueError("q [B,T,Hq,D] must have sizes below 2^31")
    qa = _on(dev, dtype, "q", q)
    kc, vc, table, Hkv, page_size, num_pages, max_pages = _caches(dev, k_cache, v_cache, page_table, dtype, B, D)
    n = _optional(dev, lens, torch.int32, (B,), "lens")
    c = _optional(dev, counts, torch.int32, (B,), "counts")
    par = _optional(dev, parents, torch.int32, (B, T), "parents")
    p, size = _ws(dev, ws)
    if out is None:
        out = torch.empty_like(q)
        oa = out.data_ptr()
    else:
        out, oa = _result(dev, out, shape, dtype, "out")
    rc = lib().spr_draft_pass_call(OP_TREE_ATTENTION, _ATTENTION_ARGS(
        qa, kc, vc, B, T, Hq, Hkv, D, dt, n, c, par, table, max_pages, num_pages, page_size, (D or 1) ** -0.5 if scale is None else scale, oa, p,
        size, _raw_stream(dev)))
    if rc != 0:
        _check("tree_attention", rc)
    return out


def logits_rules(logits, V: int, ws: Workspace, history=None, history_len=None, tokens=None, parents=None, counts=None,
                 penalties=None, bias_tokens=None, bias_values=None, masks=None, mask_rows=None, out=None):
    """Penalties for repeated tokens, biases and grammar masks on logits [B,T,ldv], row i of a sequence being what the
    model says after node i.

    history i32 [B,L] with history_len i32 [B], tokens i32 [B,T] (the nodes' own), parents and counts as for
    cache_append; penalties f32 [B,3]: repetition, frequency, presence; bias_tokens i32 [B,n] with bias_values f32 [B,n];
    masks i32 [M,words], a bit per token, with mask_rows i32 [B,T], negative: none.  Returns out [B,T,ld_out] (new
    rows have ldv entries, those behind V not written); out may be logits."""
    dev = torch.cuda.current_device()
    dtype, dt = logits.dtype, _dt(logits)
    if logits.dim() != 3:
        raise ValueError("logits must be [B,T,ldv]")
    B, T, ldv = logits.shape
    if (B | T) > _INT_MAX or V > _INT_MAX:
        raise ValueError("logits [B,T,ldv] and V must be below 2^31")
    la = _on(dev, dtype, "logits", logits)
    if (history is None) != (history_len is None):
        raise ValueError("history and history_len go together")
    L, ha = 0, 0
    if history is not None:
        if history.dim() != 2 or history.shape[0] != B:
            raise ValueError(f"history must be [{B}, L]")
        ha, L = _on(dev, torch.int32, "history", history), history.shape[1]
    hl = _optional(dev, history_len, torch.int32, (B,), "history_len")
    ta = _optional(dev, tokens, torch.int32, (B, T), "tokens")
    c = _optional(dev, counts, torch.int32, (B,), "counts")
    par = _optional(dev, parents, torch.int32, (B, T), "parents")
    pa = _optional(dev, penalties, torch.float32, (B, 3), "penalties")
    if (bias_tokens is None) != (bias_values is None):
        raise ValueError("bias_tokens and bias_values go together")
    nb, ba, bv = 0, 0, 0
    if bias_tokens is not None:
        if bias_tokens.dim() != 2 or bias_tokens.shape[0] != B or bias_tokens.shape[1] > _INT_MAX:
            raise ValueError(f"bias_tokens must be [{B}, n]")
        nb = bias_tokens.shape[1]
        ba = _on(dev, torch.int32, "bias_tokens", bias_tokens)
        bv = _optional(dev, bias_values, torch.float32, (B, nb), "bias_values")
    if (masks is None) != (mask_rows is None):
        raise ValueError("masks and mask_rows go together")
    ma, ld_mask, num_masks, mr = 0, 0, 0, 0
    if masks is not None:
        if masks.dim() != 2 or not 0 < masks.shape[0] <= _INT_MAX:
            raise ValueError("masks must be [M, words] with M >= 1")
        num_masks, ld_mask = masks.shape
        ma = _on(dev, torch.int32, "masks", masks)
        mr = _optional(dev, mask_rows, torch.int32, (B, T), "mask_rows")
    p, size = _ws(dev, ws)
    if out is None:
        out, ld_out = torch.empty_like(logits), ldv
        oa = out.data_ptr()
    else:
        if out.dim() != 3 or out.shape[0] != B or out.shape[1] != T:
            raise ValueError(f"out must be [{B}, {T}, ld_out]")
        oa, ld_out = _on(dev, dtype, "out", out), out.shape[2]
    rc = lib().spr_draft_pass_call(OP_LOGITS_RULES, _RULES_ARGS(
        la, ldv, V, B, T, dt, ha, L, hl, ta, par, c, pa, ba, bv, nb, ma, ld_mask, num_masks, mr, oa, ld_out, p, size, _raw_stream(dev)))
    if rc != 0:
        _check("logits_rules", rc)
    return out


# ---------------------------------------------------------------------------- host buffers


def _host(t: torch.Tensor, dtype=None, name="tensor"):
    if t.is_cuda:
        raise ValueError(f"{name} must be a host tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    return t


def host_arena_bytes(op: int, B: int, K: int = 1, Kp: int = 1, ldv: int = 0, d: int = 0, h: int = 0,
                     dt: int = BF16) -> int:
    return int(lib().spr_host_arena_bytes(op, B, K, Kp, ldv, d, h, dt))


class Arena:
    """Device staging memory for the host-buffer calls."""

    def __init__(self, nbytes: int, device="cuda"):
        self.buf = torch.empty((max(int(nbytes), 256) + 255) // 256 * 256, dtype=torch.uint8, device=device)

    @property
    def nbytes(self) -> int:
        return self.buf.numel()


def sprinter_verify_host(hidden, W1, b1, W2, b2, threshold: float, arena: Arena, ws: Workspace,
                         path: int = PATH_AUTO, want_scores: bool = True, out=None):
    """Host tensors in, host tensors out (pinned memory recommended); synchronises."""
    _host(hidden, name="hidden")
    B, K, d = hidden.shape
    h = 0 if W1.dim() == 1 else W1.shape[0]
    _host(W1, hidden.dtype, "W1")
    _host(b2, torch.float32, "b2")
    if h:
        _host(b1, torch.float32, "b1")
        _host(W2, hidden.dtype, "W2")
    else:
        b1 = W2 = None
    if out is None:
        scores = torch.empty((B, K), dtype=torch.float32) if want_scores else None
        accept = torch.empty((B, K), dtype=torch.uint8)
        first_reject = torch.empty((B,), dtype=torch.int32)
    else:
        scores, accept, first_reject = out
    rc = lib().sprinter_verify_host(_ptr(hidden), _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2),
                                    float(threshold), B, K, d, h, _dt(hidden), path, _ptr(scores),
                                    _ptr(accept), _ptr(first_reject), _ptr(arena.buf), arena.nbytes,
                                    _ptr(ws.buf), ws.nbytes, _stream())
    _check("sprinter_verify_host", rc)
    return scores, accept, first_reject


def replace_sample_host(target_logits, V: int, uniforms, arena: Arena, ws: Workspace, rows=None,
                        first_reject=None, K: int = 0, seq_stride: int = 1, out=None):
    _host(target_logits, name="target_logits")
    ldv = target_logits.shape[-1]
    R = target_logits.numel() // ldv
    _host(uniforms, torch.float32, "uniforms")
    n = uniforms.numel()
    if rows is not None:
        _host(rows, torch.int32, "rows")
    if first_reject is not None:
        _host(first_reject, torch.int32, "first_reject")
    tokens = torch.empty((n,), dtype=torch.int32) if out is None else out
    rc = lib().replace_sample_host(_ptr(target_logits), ldv, V, R, _ptr(rows), _ptr(first_reject), K,
                                   seq_stride, n, _ptr(uniforms), _dt(target_logits), _ptr(tokens),
                                   _ptr(arena.buf), arena.nbytes, _ptr(ws.buf), ws.nbytes, _stream())
    _check("replace_sample_host", rc)
    return tokens


def sd_verify_host(p_logits, q_logits, V: int, draft_tokens, uniforms, arena: Arena, ws: Workspace,
                   extras: bool = False, out=None):
    _host(p_logits, name="p_logits")
    _host(q_logits, p_logits.dtype, "q_logits")
    B, Kp, ldv = p_logits.shape
    K = q_logits.shape[1]
    _host(draft_tokens, torch.int32, "draft_tokens")
    _host(uniforms, torch.float32, "uniforms")
    if out is None:
        out = dict(accepted_len=torch.empty((B,), dtype=torch.int32),
                   correction_token=torch.empty((B,), dtype=torch.int32))
        if extras:
            out.update(accept=torch.empty((B, K), dtype=torch.uint8),
                       p_tok=torch.empty((B, K), dtype=torch.float32),
                       q_tok=torch.empty((B, K), dtype=torch.float32),
                       residual_mass=torch.empty((B,), dtype=torch.float32))
    rc = lib().sd_verify_host(_ptr(p_logits), _ptr(q_logits), ldv, _ptr(draft_tokens), _ptr(uniforms),
                              B, K, Kp, V, _dt(p_logits), _ptr(out["accepted_len"]),
                              _ptr(out["correction_token"]), _ptr(out.get("accept")),
                              _ptr(out.get("p_tok")), _ptr(out.get("q_tok")),
                              _ptr(out.get("residual_mass")), _ptr(arena.buf), arena.nbytes,
                              _ptr(ws.buf), ws.nbytes, _stream())
    _check("sd_verify_host", rc)
    return out


def set_stage_events(before=None, after=None):
    """torch.cuda.Event pair (created with enable_timing=True and recorded once so that the
    handles exist) that sd_verify records around its row-statistics kernel; None to stop."""
    lib().spr_set_stage_events(None if before is None else C.c_void_p(before.cuda_event),
                               None if after is None else C.c_void_p(after.cuda_event))


def replace_sample_static(target_logits, V: int, uniforms, tokens, rows=None, first_reject=None,
                          K: int = 0, seq_stride: int = 1):
    """replace_sample on the library's built-in scratch: no workspace argument, and nothing is
    allocated here either - the caller passes the output tensor `tokens` (int32 [n]).  For
    code that must not allocate device memory around the call; limited to
    n <= 1024 draws and n * steps <= 65536 (see include/sprinter.h).  Calls that may overlap
    on one GPU race on the shared scratch: keep them on one stream."""
    _dev(target_logits, name="target_logits")
    ldv = target_logits.shape[-1]
    R = target_logits.numel() // ldv
    _dev(uniforms, torch.float32, "uniforms")
    _dev(tokens, torch.int32, "tokens")
    n = uniforms.numel()
    if tokens.numel() != n:
        raise ValueError("tokens must have one entry per uniform")
    _selectors(rows, first_reject, n)
    rc = lib().replace_sample_static(_ptr(target_logits), ldv, V, R, _ptr(rows), _ptr(first_reject), K,
                                     seq_stride, n, _ptr(uniforms), _dt(target_logits), _ptr(tokens),
                                     _stream())
    _check("replace_sample_static", rc)
    return tokens


def sprinter_simulate(seed: int, runs: int, r: int, eta_tp: float, eta_fp: float, max_tokens: int,
                      first_run: int = 0, want_runs: bool = True, device="cuda"):
    """Run lengths of an i.i.d. verifier (Theorems 2 and 3).

    Returns (n_accepted int32 [runs] or None, histogram int64 [max_tokens + 1])."""
    n = torch.empty((runs,), dtype=torch.int32, device=device) if want_runs else None
    hist = torch.empty((max_tokens + 1,), dtype=torch.int64, device=device)
    rc = lib().sprinter_simulate(int(seed), int(first_run), int(runs), int(r), float(eta_tp), float(eta_fp),
                                 int(max_tokens), _ptr(n), _ptr(hist), _stream())
    _check("sprinter_simulate", rc)
    return n, hist
