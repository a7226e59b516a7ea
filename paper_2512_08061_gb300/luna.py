"""Thin Python binding of the C ABI in include/luna.h (argument marshalling only).

Every function here has the name of the C entry point it calls and does no
arithmetic of its own: tensors are passed as device pointers, the stream as
torch's current CUDA stream.  PyTorch provides device memory and streams.
If the compiled library is missing this module raises at import time; there
is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

LUNA_OK = 0
STATUS_NAMES = {0: "LUNA_OK", 1: "LUNA_ERR_INVALID_ARG", 2: "LUNA_ERR_UNSUPPORTED", 3: "LUNA_ERR_WORKSPACE",
                4: "LUNA_ERR_CUDA", 5: "LUNA_ERR_DEVICE_TIMEOUT"}
LUNA_F32, LUNA_BF16 = 0, 1
_DTYPES = {torch.float32: LUNA_F32, torch.bfloat16: LUNA_BF16}
# names of the tensor-core kernels accepted by luna_profile_start
TC_KERNELS: list[str] = ["tile_split", "tc_keys", "tc_query", "tc_bwd_query", "tc_bwd_key", "tc_causal", "seg_scan",
                         "tcc_query", "tcc_dstats", "seg_rscan", "tcc_key", "tc_phi_bwd"]


class LunaError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")
        self.status = status


class PhiDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int), ("L", ctypes.c_int), ("hidden", ctypes.c_int), ("shared_channels", ctypes.c_int),
                ("ch_rms_target", ctypes.c_float), ("signed_outputs", ctypes.c_int),
                ("param_head_stride", ctypes.c_int64), ("act", ctypes.c_int), ("envelope", ctypes.c_int),
                ("bank_coef", ctypes.c_int)]


PARAM_KEYS = ("W", "b", "w1", "b1", "w2", "b2", "We", "be", "coef")
GRAD_KEYS = tuple("d" + k for k in PARAM_KEYS)
ACTS = {"relu": 0, "gelu": 1, "silu": 2, "tanh": 3}  # luna_act


class PhiParams(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in PARAM_KEYS]


class PhiGrads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in GRAD_KEYS]


class AttnDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("H", ctypes.c_int), ("n", ctypes.c_int), ("d", ctypes.c_int),
                ("dv", ctypes.c_int), ("causal", ctypes.c_int), ("chunk", ctypes.c_int), ("eps", ctypes.c_float),
                ("io", ctypes.c_int)]


class Strides(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("t", ctypes.c_int64)]


class DecayDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int), ("n", ctypes.c_int),
                ("d", ctypes.c_int), ("dv", ctypes.c_int), ("scale", ctypes.c_float), ("io", ctypes.c_int),
                *[(k, Strides) for k in ("q", "k", "v", "o", "gq", "gk", "gv", "go")]]


class DeltaDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("H", ctypes.c_int), ("Hk", ctypes.c_int), ("n", ctypes.c_int),
                ("d", ctypes.c_int), ("dv", ctypes.c_int), ("scale", ctypes.c_float), ("io", ctypes.c_int),
                *[(k, Strides) for k in ("q", "k", "v", "o", "g", "beta", "gq", "gk", "gv", "go", "gg", "gbeta")]]


class BeamDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("K", ctypes.c_int), ("V", ctypes.c_int), ("io", ctypes.c_int),
                ("ld", ctypes.c_int64), ("end", ctypes.c_int)]


class NormDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int), ("groups", ctypes.c_int), ("kind", ctypes.c_int),
                ("gate", ctypes.c_int), ("alpha", ctypes.c_float), ("eps", ctypes.c_float), ("io", ctypes.c_int),
                *[(k, ctypes.c_int64) for k in ("ldx", "ldy", "ldgate", "ldX", "ldH", "lddX", "lddH", "lddx", "lddy",
                                                "lddgate")]]


NORM_KINDS = {"rms": 0, "layer": 1}  # luna_norm_kind
GATES = {"none": 0, "sigmoid": 1, "silu": 2}  # luna_gate


class LinearDesc(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("n", ctypes.c_int), ("k", ctypes.c_int), ("act", ctypes.c_int),
                ("io", ctypes.c_int), *[(k, ctypes.c_int64) for k in ("ldx", "ldw", "ldy", "ldr", "ldz", "lddy", "lddx")]]


LINEAR_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}  # luna_linear_act


def library_path() -> str:
    return _build.LIB


def _load():
    path = library_path()
    if not os.path.exists(path):
        raise ImportError(f"LUNA CUDA library not built ({path}); run paper_2512_08061_gb300.build.build()")
    lib = ctypes.CDLL(path)
    P, S, I, I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64
    pd, ad = ctypes.POINTER(PhiDesc), ctypes.POINTER(AttnDesc)
    dd, nd, ld = ctypes.POINTER(DecayDesc), ctypes.POINTER(NormDesc), ctypes.POINTER(LinearDesc)
    td, bd = ctypes.POINTER(DeltaDesc), ctypes.POINTER(BeamDesc)
    sig = {
        "luna_status_string": ([I], ctypes.c_char_p),
        "luna_version": ([], I),
        "luna_phi_table_size": ([pd, I, ctypes.POINTER(S)], I),
        "luna_phi_prepare": ([pd, I, ctypes.POINTER(PhiParams), P, S, P], I),
        "luna_featmap": ([pd, I, P, P, I, I64, P, P], I),
        "luna_workspace_size": ([ad, pd, I, ctypes.POINTER(S)], I),
        "luna_state_size": ([ad, pd, ctypes.POINTER(S)], I),
        "luna_attn_fwd": ([ad, pd, P, P, P, P, P, P, P, P, S, P], I),
        "luna_attn_bwd": ([ad, pd, P, P, P, P, P, P, P, P, P, P, ctypes.POINTER(PhiGrads), P, S, P], I),
        "luna_device_status": ([P, P], I),
        "luna_profile_start": ([ctypes.c_char_p], I),
        "luna_profile_stop": ([ctypes.POINTER(ctypes.c_double), ctypes.POINTER(I)], I),
        "luna_launch_count": ([], ctypes.c_uint64),
        "luna_attn_fwd_noalloc": ([ad, pd, P, P, P, P, P, P, P], I),
        "luna_state_final": ([ad, pd, P, ctypes.POINTER(P), ctypes.POINTER(I64), ctypes.POINTER(P),
                              ctypes.POINTER(I64)], I),
        "luna_attn_decode": ([ad, pd, P, P, P, P, P, P, I64, P, I64, P], I),
        "luna_selftest_wait": ([P, I64, P], I),
        "luna_noalloc_scratch": ([ctypes.POINTER(P), ctypes.POINTER(S)], I),
        "luna_attn_weights": ([ad, pd, P, P, P, P, I, I, I, P, P], I),
        "luna_decay_workspace_size": ([dd, I, ctypes.POINTER(S)], I),
        "luna_decay_fwd": ([dd, P, P, P, P, P, P, P, P, P, S, P], I),
        "luna_decay_bwd": ([dd, P, P, P, P, P, P, P, P, P, P, P, P, P, S, P], I),
        "luna_decay_step": ([dd, P, P, P, P, P, I, P, P, P], I),
        "luna_delta_workspace_size": ([td, I, ctypes.POINTER(S)], I),
        "luna_delta_fwd": ([td] + [P] * 10 + [S, P], I),
        "luna_delta_bwd": ([td] + [P] * 16 + [S, P], I),
        "luna_delta_step": ([td, P, P, P, P, P, P, I, P, P, P], I),
        "luna_beam_workspace_size": ([bd, ctypes.POINTER(S)], I),
        "luna_beam_select": ([bd] + [P] * 8 + [S, P], I),
        "luna_beam_reorder": ([bd, P, P, I, P, S, P, P], I),
        "luna_norm_workspace_size": ([nd, ctypes.POINTER(S)], I),
        "luna_norm_fwd": ([nd] + [P] * 10, I),
        "luna_norm_bwd": ([nd] + [P] * 16 + [S, P], I),
        "luna_linear_workspace_size": ([ld, I, ctypes.POINTER(S)], I),
        "luna_linear_fwd": ([ld] + [P] * 7 + [S, P], I),
        "luna_linear_bwd": ([ld] + [P] * 8 + [S, P], I),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


_lib = _load()
EXPORTED = ("luna_status_string", "luna_version", "luna_phi_table_size", "luna_phi_prepare", "luna_featmap",
            "luna_workspace_size", "luna_state_size", "luna_attn_fwd", "luna_attn_bwd", "luna_device_status",
            "luna_profile_start", "luna_profile_stop", "luna_launch_count", "luna_attn_fwd_noalloc",
            "luna_state_final", "luna_attn_decode", "luna_selftest_wait", "luna_noalloc_scratch",
            "luna_attn_weights",
            "luna_decay_workspace_size", "luna_decay_fwd", "luna_decay_bwd", "luna_decay_step",
            "luna_delta_workspace_size", "luna_delta_fwd", "luna_delta_bwd", "luna_delta_step",
            "luna_beam_workspace_size", "luna_beam_select", "luna_beam_reorder",
            "luna_norm_workspace_size", "luna_norm_fwd", "luna_norm_bwd",
            "luna_linear_workspace_size", "luna_linear_fwd", "luna_linear_bwd")


def _ptr(t):
    """Device address of a tensor, or a raw address given as an int."""
    if t is None:
        return None
    if isinstance(t, int):
        return ctypes.c_void_p(t)
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check(st: int, where: str) -> None:
    if st != LUNA_OK:
        raise LunaError(st, where)


def _io_code(t: torch.Tensor) -> int:
    if t.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return _DTYPES[t.dtype]


def phi_desc(M: int, L: int, hidden: int, shared: bool = False, ch_rms_target: float = 0.0,
             signed: bool = False, param_head_stride: int = 0, act: str = "relu", envelope: bool = False,
             bank_coef: bool = False) -> PhiDesc:
    return PhiDesc(M, L, hidden, int(bool(shared)), float(ch_rms_target), int(bool(signed)), int(param_head_stride),
                   ACTS[act], int(bool(envelope)), int(bool(bank_coef)))


def attn_desc(B, H, n, d, dv, causal=False, chunk=0, eps=1e-6, io=LUNA_BF16) -> AttnDesc:
    return AttnDesc(B, H, n, d, dv, int(bool(causal)), chunk, eps, io)


def luna_status_string(status: int) -> str:
    return _lib.luna_status_string(status).decode()


def luna_version() -> int:
    return _lib.luna_version()


def luna_phi_table_size(pd: PhiDesc, d: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_phi_table_size(ctypes.byref(pd), d, ctypes.byref(out)), "luna_phi_table_size")
    return out.value


def luna_phi_prepare(pd: PhiDesc, d: int, params: dict, table: torch.Tensor, stream=None) -> None:
    pp = PhiParams(*[_ptr(params.get(k)) for k in PARAM_KEYS])
    _check(_lib.luna_phi_prepare(ctypes.byref(pd), d, ctypes.byref(pp), _ptr(table), table.numel() * table.element_size(),
                                 _stream(stream)), "luna_phi_prepare")


def luna_featmap(pd: PhiDesc, d: int, table: torch.Tensor, X: torch.Tensor, Phi: torch.Tensor, stream=None) -> None:
    rows = X.numel() // d if d else 0
    _check(_lib.luna_featmap(ctypes.byref(pd), d, _ptr(table), _ptr(X), _io_code(X), rows, _ptr(Phi), _stream(stream)),
           "luna_featmap")


def luna_workspace_size(ad: AttnDesc, pd: PhiDesc, backward: bool) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_workspace_size(ctypes.byref(ad), ctypes.byref(pd), int(bool(backward)), ctypes.byref(out)),
           "luna_workspace_size")
    return out.value


def luna_state_size(ad: AttnDesc, pd: PhiDesc) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_state_size(ctypes.byref(ad), ctypes.byref(pd), ctypes.byref(out)), "luna_state_size")
    return out.value


def luna_attn_fwd(ad, pd, table, Q, K, V, lengths, O, state, workspace, stream=None) -> None:
    _check(_lib.luna_attn_fwd(ctypes.byref(ad), ctypes.byref(pd), _ptr(table), _ptr(Q), _ptr(K), _ptr(V),
                              _ptr(lengths), _ptr(O), _ptr(state), _ptr(workspace),
                              workspace.numel() * workspace.element_size(), _stream(stream)), "luna_attn_fwd")


def luna_attn_bwd(ad, pd, table, Q, K, V, dO, lengths, state, dQ, dK, dV, grads: dict, workspace, stream=None) -> None:
    pg = PhiGrads(*[_ptr(grads.get(k)) for k in GRAD_KEYS])
    _check(_lib.luna_attn_bwd(ctypes.byref(ad), ctypes.byref(pd), _ptr(table), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO),
                              _ptr(lengths), _ptr(state), _ptr(dQ), _ptr(dK), _ptr(dV), ctypes.byref(pg),
                              _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "luna_attn_bwd")


def luna_attn_fwd_noalloc(ad, pd, table, Q, K, V, lengths, O, stream=None) -> None:
    _check(_lib.luna_attn_fwd_noalloc(ctypes.byref(ad), ctypes.byref(pd), _ptr(table), _ptr(Q), _ptr(K), _ptr(V),
                                      _ptr(lengths), _ptr(O), _stream(stream)), "luna_attn_fwd_noalloc")


NOALLOC_SCRATCH_BYTES = 16 << 20


def luna_attn_weights(ad, pd, table, Q, K, lengths, row0: int, rows: int, teacher: bool, A: torch.Tensor,
                      stream=None) -> None:
    _check(_lib.luna_attn_weights(ctypes.byref(ad), ctypes.byref(pd), _ptr(table), _ptr(Q), _ptr(K), _ptr(lengths),
                                  int(row0), int(rows), int(bool(teacher)), _ptr(A), _stream(stream)),
           "luna_attn_weights")


def luna_state_final(ad, pd, state) -> tuple[int, int, int, int]:
    """(S address, S stride, z address, z stride) of the final causal state inside `state` (floats)."""
    S, Ss, z, zs = ctypes.c_void_p(), ctypes.c_int64(), ctypes.c_void_p(), ctypes.c_int64()
    _check(_lib.luna_state_final(ctypes.byref(ad), ctypes.byref(pd), _ptr(state), ctypes.byref(S), ctypes.byref(Ss),
                                 ctypes.byref(z), ctypes.byref(zs)), "luna_state_final")
    return S.value, Ss.value, z.value, zs.value


def luna_attn_decode(ad, pd, table, q, k, v, o, S, S_stride, z, z_stride, stream=None) -> None:
    """S, z: tensors (their data pointers are used) or raw device addresses."""
    sp = _ptr(S) if isinstance(S, torch.Tensor) else ctypes.c_void_p(S)
    zp = _ptr(z) if isinstance(z, torch.Tensor) else ctypes.c_void_p(z)
    _check(_lib.luna_attn_decode(ctypes.byref(ad), ctypes.byref(pd), _ptr(table), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                 sp, S_stride, zp, z_stride, _stream(stream)), "luna_attn_decode")


# ---------------------------------------------------------------------------
# linear attention with a decay for each head

def decay_desc(B, H, n, d, dv, Hkv=None, scale=None, io=LUNA_BF16) -> DecayDesc:
    """Contiguous tensors; set the strides q, k, v, o (gq, gk, gv, go) for views."""
    return DecayDesc(B, H, H if Hkv is None else Hkv, n, d, dv,
                     max(d, 1) ** -0.5 if scale is None else scale, io)


def luna_decay_workspace_size(dd: DecayDesc, backward: bool) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_decay_workspace_size(ctypes.byref(dd), int(bool(backward)), ctypes.byref(out)),
           "luna_decay_workspace_size")
    return out.value


def luna_decay_fwd(dd, log_decay, Q, K, V, lengths, S0, O, S1, workspace, stream=None) -> None:
    _check(_lib.luna_decay_fwd(ctypes.byref(dd), _ptr(log_decay), _ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(S0),
                               _ptr(O), _ptr(S1), _ptr(workspace), workspace.numel() * workspace.element_size(),
                               _stream(stream)), "luna_decay_fwd")


def luna_decay_bwd(dd, log_decay, Q, K, V, dO, lengths, S0, dS1, dQ, dK, dV, dS0, workspace, stream=None) -> None:
    _check(_lib.luna_decay_bwd(ctypes.byref(dd), _ptr(log_decay), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(lengths),
                               _ptr(S0), _ptr(dS1), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dS0), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream(stream)), "luna_decay_bwd")


def luna_decay_step(dd, log_decay, q, k, v, slots, nslots: int, S, o, stream=None) -> None:
    _check(_lib.luna_decay_step(ctypes.byref(dd), _ptr(log_decay), _ptr(q), _ptr(k), _ptr(v), _ptr(slots), nslots,
                                _ptr(S), _ptr(o), _stream(stream)), "luna_decay_step")


# ---------------------------------------------------------------------------
# the gated delta rule

def delta_desc(B, H, n, d, dv, Hk=None, scale=None, io=LUNA_BF16) -> DeltaDesc:
    """Contiguous tensors; set the strides q, k, v, o, g, beta (gq, gk, gv, go, gg, gbeta) for views."""
    return DeltaDesc(B, H, H if Hk is None else Hk, n, d, dv, max(d, 1) ** -0.5 if scale is None else scale, io)


def luna_delta_workspace_size(dd: DeltaDesc, backward: bool) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_delta_workspace_size(ctypes.byref(dd), int(bool(backward)), ctypes.byref(out)),
           "luna_delta_workspace_size")
    return out.value


def luna_delta_fwd(dd, log_decay, beta, Q, K, V, lengths, S0, O, S1, workspace, stream=None) -> None:
    _check(_lib.luna_delta_fwd(ctypes.byref(dd), _ptr(log_decay), _ptr(beta), _ptr(Q), _ptr(K), _ptr(V), _ptr(lengths),
                               _ptr(S0), _ptr(O), _ptr(S1), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream(stream)), "luna_delta_fwd")


def luna_delta_bwd(dd, log_decay, beta, Q, K, V, dO, lengths, S0, dS1, dQ, dK, dV, dlog_decay, dbeta, dS0, workspace,
                   stream=None) -> None:
    _check(_lib.luna_delta_bwd(ctypes.byref(dd), _ptr(log_decay), _ptr(beta), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO),
                               _ptr(lengths), _ptr(S0), _ptr(dS1), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dlog_decay),
                               _ptr(dbeta), _ptr(dS0), _ptr(workspace), workspace.numel() * workspace.element_size(),
                               _stream(stream)), "luna_delta_bwd")


def luna_delta_step(dd, log_decay, beta, q, k, v, slots, nslots: int, S, o, stream=None) -> None:
    _check(_lib.luna_delta_step(ctypes.byref(dd), _ptr(log_decay), _ptr(beta), _ptr(q), _ptr(k), _ptr(v), _ptr(slots),
                                nslots, _ptr(S), _ptr(o), _stream(stream)), "luna_delta_step")


# ---------------------------------------------------------------------------
# beam search over recurrent states

def beam_desc(B, K, V=0, end=-1, io=LUNA_BF16) -> BeamDesc:
    return BeamDesc(B, K, V, io, 0, end)


def luna_beam_workspace_size(bd: BeamDesc) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_beam_workspace_size(ctypes.byref(bd), ctypes.byref(out)), "luna_beam_workspace_size")
    return out.value


def luna_beam_select(bd, logits, scores, done, scores_out, tokens, parents, done_out, workspace, stream=None) -> None:
    _check(_lib.luna_beam_select(ctypes.byref(bd), _ptr(logits), _ptr(scores), _ptr(done), _ptr(scores_out),
                                 _ptr(tokens), _ptr(parents), _ptr(done_out), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "luna_beam_select")


def luna_beam_reorder(bd, parents, slots, nslots: int, pool, slot_bytes: int, new_slots, stream=None) -> None:
    _check(_lib.luna_beam_reorder(ctypes.byref(bd), _ptr(parents), _ptr(slots), nslots, _ptr(pool), slot_bytes,
                                  _ptr(new_slots), _stream(stream)), "luna_beam_reorder")


# ---------------------------------------------------------------------------
# norms after and before a block, with its gate and residual scale

def norm_desc(rows, cols, groups=1, kind="rms", gate="none", res_scale=1.0, eps=1e-6, io=LUNA_BF16) -> NormDesc:
    return NormDesc(rows, cols, groups, NORM_KINDS[kind], GATES[gate], res_scale, eps, io)


def luna_norm_workspace_size(nd: NormDesc) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_norm_workspace_size(ctypes.byref(nd), ctypes.byref(out)), "luna_norm_workspace_size")
    return out.value


def luna_norm_fwd(nd, x, y, gate, w_post, b_post, w_pre, b_pre, X, H, stream=None) -> None:
    _check(_lib.luna_norm_fwd(ctypes.byref(nd), _ptr(x), _ptr(y), _ptr(gate), _ptr(w_post), _ptr(b_post), _ptr(w_pre),
                              _ptr(b_pre), _ptr(X), _ptr(H), _stream(stream)), "luna_norm_fwd")


def luna_norm_bwd(nd, x, y, gate, w_post, b_post, w_pre, dX, dH, dx, dy, dgate, dw_post, db_post, dw_pre, db_pre,
                  workspace, stream=None) -> None:
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.luna_norm_bwd(ctypes.byref(nd), _ptr(x), _ptr(y), _ptr(gate), _ptr(w_post), _ptr(b_post), _ptr(w_pre),
                              _ptr(dX), _ptr(dH), _ptr(dx), _ptr(dy), _ptr(dgate), _ptr(dw_post), _ptr(db_post),
                              _ptr(dw_pre), _ptr(db_pre), _ptr(workspace), nbytes, _stream(stream)), "luna_norm_bwd")


# ---------------------------------------------------------------------------
# linear layers

def linear_desc(m, n, k, act="none", io=LUNA_BF16) -> LinearDesc:
    return LinearDesc(m, n, k, LINEAR_ACTS[act], io)


def luna_linear_workspace_size(ld: LinearDesc, backward: bool) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.luna_linear_workspace_size(ctypes.byref(ld), int(bool(backward)), ctypes.byref(out)),
           "luna_linear_workspace_size")
    return out.value


def luna_linear_fwd(ld, X, W, bias, R, Y, Z, workspace, stream=None) -> None:
    _check(_lib.luna_linear_fwd(ctypes.byref(ld), _ptr(X), _ptr(W), _ptr(bias), _ptr(R), _ptr(Y), _ptr(Z),
                                _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "luna_linear_fwd")


def luna_linear_bwd(ld, X, W, Z, dY, dX, dW, db, workspace, stream=None) -> None:
    _check(_lib.luna_linear_bwd(ctypes.byref(ld), _ptr(X), _ptr(W), _ptr(Z), _ptr(dY), _ptr(dX), _ptr(dW), _ptr(db),
                                _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "luna_linear_bwd")


def luna_device_status(workspace: torch.Tensor, stream=None) -> int:
    return _lib.luna_device_status(_ptr(workspace), _stream(stream))


def luna_noalloc_scratch() -> tuple[int, int]:
    """(device address, bytes) of the no-allocation entry point's scratch array on the current device."""
    p, n = ctypes.c_void_p(), ctypes.c_size_t(0)
    _check(_lib.luna_noalloc_scratch(ctypes.byref(p), ctypes.byref(n)), "luna_noalloc_scratch")
    return p.value, n.value


def luna_selftest_wait(workspace: torch.Tensor, limit_ns: int, stream=None) -> None:
    _check(_lib.luna_selftest_wait(_ptr(workspace), int(limit_ns), _stream(stream)), "luna_selftest_wait")


def luna_profile_start(kernel: str) -> None:
    _check(_lib.luna_profile_start(kernel.encode()), "luna_profile_start")


def luna_profile_stop() -> tuple[float, int]:
    ms, n = ctypes.c_double(0.0), ctypes.c_int(0)
    _check(_lib.luna_profile_stop(ctypes.byref(ms), ctypes.byref(n)), "luna_profile_stop")
    return ms.value, n.value


def luna_launch_count() -> int:
    return int(_lib.luna_launch_count())


# ---------------------------------------------------------------------------
# convenience: buffers sized by the library, allocated with torch

def alloc_bytes(nbytes: int, device) -> torch.Tensor:
    """A 256-byte aligned uint8 device buffer (torch's caching allocator aligns to 512)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


class Luna:
    """Owns the table, workspace and state buffers of one problem shape."""

    def __init__(self, B, H, n, d, dv, M, L, hidden=64, causal=False, eps=1e-6, io=torch.bfloat16, chunk=0,
                 device="cuda", shared=False, ch_rms_target=0.0, signed=False, per_head=False, act="relu",
                 envelope=False, bank_coef=False):
        self.pd = phi_desc(M, L, hidden, shared, ch_rms_target, signed, 0, act, envelope, bank_coef)
        self.ad = attn_desc(B, H, n, d, dv, causal, chunk, eps, _DTYPES[io])
        self.d = d
        self.device = torch.device(device)
        tb = luna_phi_table_size(self.pd, d)
        self.heads = H if per_head else 0  # per-head parameters: one table per head, tb bytes apart
        if per_head:
            self.pd.param_head_stride = tb
        self.table = alloc_bytes(tb * max(1, self.heads), self.device)
        self.ws = alloc_bytes(max(luna_workspace_size(self.ad, self.pd, False),
                                  luna_workspace_size(self.ad, self.pd, True)), self.device)
        self.state = alloc_bytes(luna_state_size(self.ad, self.pd), self.device)

    def prepare(self, params: dict, stream=None):
        """params: W, b, w1, b1, w2, b2 device tensors (with a leading head axis for per-head parameters),
        and We, be (envelope) or coef (Bank+Coef) with those variants."""
        if not self.heads:
            luna_phi_prepare(self.pd, self.d, params, self.table, stream)
            return
        tb = self.pd.param_head_stride
        for h in range(self.heads):
            luna_phi_prepare(self.pd, self.d, {k: v[h] for k, v in params.items()}, self.table[h * tb:(h + 1) * tb],
                             stream)

    def forward(self, Q, K, V, lengths=None, O=None, save_state=True, stream=None):
        if O is None:
            O = torch.empty(Q.shape[:-1] + (self.ad.dv,), dtype=Q.dtype, device=Q.device)
        luna_attn_fwd(self.ad, self.pd, self.table, Q, K, V, lengths, O, self.state if save_state else None,
                      self.ws, stream)
        return O

    def backward(self, Q, K, V, dO, lengths=None, use_state=True, out=None, stream=None):
        if out is None:
            M, L, hid = self.pd.M, self.pd.L, self.pd.hidden
            f32 = dict(dtype=torch.float32, device=Q.device)
            fc1 = (hid,) if self.pd.shared_channels else (L, hid)
            g = (self.heads,) if self.heads else ()
            out = {"dQ": torch.empty_like(Q), "dK": torch.empty_like(K), "dV": torch.empty_like(V),
                   "dW": torch.empty(g + (M, self.d), **f32), "db": torch.empty(g + (M,), **f32),
                   "dw1": torch.empty(g + fc1, **f32), "db1": torch.empty(g + fc1, **f32),
                   "dw2": torch.empty(g + (L, hid), **f32), "db2": torch.empty(g + (L,), **f32)}
            if self.pd.envelope:
                out.update(dWe=torch.empty((L, self.d), **f32), dbe=torch.empty((L,), **f32))
            if self.pd.bank_coef:
                out["dcoef"] = torch.empty((L,), **f32)
        luna_attn_bwd(self.ad, self.pd, self.table, Q, K, V, dO, lengths, self.state if use_state else None,
                      out["dQ"], out["dK"], out["dV"], out, self.ws, stream)
        return out

    def decode(self, q, k, v, o=None, stream=None):
        """One streaming-form step per (b, h) from the final state of the last causal forward
        (saved with save_state=True), which it advances in place.  q, k: (B, H, d); v: (B, H, dv)."""
        if o is None:
            o = torch.empty(q.shape[:-1] + (self.ad.dv,), dtype=q.dtype, device=q.device)
        S, Ss, z, zs = luna_state_final(self.ad, self.pd, self.state)
        luna_attn_decode(self.ad, self.pd, self.table, q, k, v, o, S, Ss, z, zs, stream)
        return o


def _want(name: str, t, shape, dtype, device) -> None:
    """An argument's shape, type and place, before its address goes to the library."""
    if t is None:
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {t.dtype}, expected {dtype}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")


def _place(device) -> torch.device:
    """A device with its number: "cuda" is the GPU that is current now, and tensors of another one are refused."""
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        return torch.device("cuda", torch.cuda.current_device())
    return device


def _dense(name: str, t) -> None:
    if t is not None and not t.is_contiguous():
        raise ValueError(f"{name}: not contiguous")


def _layout(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.device)


def _addr(t):
    return None if t is None else t.data_ptr()


# the current stream's handle without the stream object around it, where torch offers that (a single
# token's kernels take less time than the object does)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _handle(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _new(stream, make=torch.empty):
    """torch.empty (or what `make` is) for a call on `stream` (None: the current one), from that stream's memory: the
    allocator may hand it out again only behind the call's kernels."""
    if stream is None:
        return make

    def on_stream(*args, **kwargs):
        with torch.cuda.stream(stream):
            return make(*args, **kwargs)

    return on_stream


class _Checked:
    """Calls of one problem shape.  The arguments' shapes, strides, types and devices are looked at in full
    when they differ from those of the last call of the same kind, and their strides put into that
    kind's descriptor."""

    def __init__(self, desc):
        self._desc = {kind: type(desc).from_buffer_copy(desc) for kind in ("forward", "backward", "step")}
        self._ref = {kind: ctypes.byref(d) for kind, d in self._desc.items()}
        self._seen = {}
        self.ws, self._ws, self._streams = None, (None, 0), set()

    def _workspace(self, nbytes: int) -> None:
        self.ws = alloc_bytes(nbytes, self.device)
        self._ws = (self.ws.data_ptr(), self.ws.numel())
        if self.device.type == "cuda":
            self._streams = {_handle(None)}

    def _on(self, stream):
        """The handle of the stream of a call; the workspace stays until what is queued there is done."""
        if stream is None and _raw_stream is not None:  # (as _handle, without its call)
            handle = _raw_stream(torch.cuda.current_device())
        else:
            handle = _handle(stream)
        if handle not in self._streams and self.ws is not None:
            self.ws.record_stream(torch.cuda.current_stream() if stream is None else stream)
            self._streams.add(handle)
        return handle

    def _looked_at(self, kind: str, *tensors) -> bool:
        """Whether these layouts are the last call's; the caller checks and fills in the descriptor if not."""
        layouts = [_layout(t) for t in tensors]
        if self._seen.get(kind) == layouts:
            return True
        self._seen[kind] = None
        self._pending = (kind, layouts)
        return False

    def _accept(self) -> None:
        kind, layouts = self._pending
        self._seen[kind] = layouts


class Decay(_Checked):
    """Linear attention with a decay for each head at one problem shape; owns the workspace, so its calls
    belong on one stream at a time.  Q: (B, H, n, d), K: (B, Hkv, n, d), V: (B, Hkv, n, dv), any strides
    with a contiguous last dimension; log_decay: (H,) fp32; lengths: (B,) int32 or None; states:
    (B, H, d, dv) fp32."""

    def __init__(self, B, H, n, d, dv, Hkv=None, scale=None, io=torch.bfloat16, device="cuda", backward=False):
        self.dd = decay_desc(B, H, n, d, dv, Hkv, scale, _DTYPES[io])
        super().__init__(self.dd)
        self.io, self.device = io, _place(device)
        self._workspace(luna_decay_workspace_size(self.dd, backward))
        self.shapes = {"q": (B, H, n, d), "k": (B, self.dd.Hkv, n, d), "v": (B, self.dd.Hkv, n, dv), "o": (B, H, n, dv)}
        self.state_shape = (B, H, d, dv)

    def _view(self, kind: str, field: str, t) -> None:
        """Checks a tensor of rows (of single rows for a step) and notes its strides."""
        shape = self.shapes[field[-1]]
        if kind == "step":
            shape = shape[:2] + shape[3:]
        _want(field, t, shape, self.io, self.device)
        s = t.stride()
        if s[-1] != 1 and t.shape[-1] != 1:
            raise ValueError(f"{field}: the last dimension is not contiguous")
        if not any(s[:-1]) and t[..., 0].numel() > 1:
            raise ValueError(f"{field}: one row repeated")
        setattr(self._desc[kind], field, Strides(s[0], s[1], s[2] if kind != "step" else 0))

    def _vectors(self, log_decay, lengths, name="lengths") -> None:
        B, H = self.state_shape[:2]
        _want("log_decay", log_decay, (H,), torch.float32, self.device)
        _want(name, lengths, (B,), torch.int32, self.device)
        _dense("log_decay", log_decay)
        _dense(name, lengths)

    def _states(self, **states) -> None:
        for name, t in states.items():
            _want(name, t, self.state_shape, torch.float32, self.device)
            _dense(name, t)

    def forward(self, Q, K, V, log_decay, lengths=None, S0=None, want_state=False, O=None, S1=None, stream=None):
        """O, or (O, S1) with want_state."""
        if not self._looked_at("forward", Q, K, V, log_decay, lengths, S0, O, S1):
            for field, t in (("q", Q), ("k", K), ("v", V)):
                self._view("forward", field, t)
            self._vectors(log_decay, lengths)
            self._states(S0=S0, S1=S1)
            # a new output lies as V does, or Q
            self._like = next((tuple(torch.empty_like(t).stride()) for t in (V, Q) if t.shape == self.shapes["o"]), None)
            self._view("forward", "o", self._new_output(Q, stream) if O is None else O)
            self._accept()
        if O is None:
            O = self._new_output(Q, stream)
        if want_state and S1 is None:
            S1 = _new(stream)(self.state_shape, dtype=torch.float32, device=Q.device)
        _check(_lib.luna_decay_fwd(self._ref["forward"], log_decay.data_ptr(), Q.data_ptr(), K.data_ptr(), V.data_ptr(),
                                   _addr(lengths), _addr(S0), O.data_ptr(), _addr(S1), *self._ws, self._on(stream)),
               "luna_decay_fwd")
        return (O, S1) if want_state else O

    def _new_output(self, Q, stream):
        shape = self.shapes["o"]
        if self._like is None:
            return _new(stream)(shape, dtype=self.io, device=Q.device)
        return _new(stream, torch.empty_strided)(shape, self._like, dtype=self.io, device=Q.device)

    def backward(self, Q, K, V, dO, log_decay, lengths=None, S0=None, dS1=None, out=None, stream=None):
        """dQ, dK, dV, and dS0 where S0 is given (or `out` holds it), of forward on the same inputs."""
        if out is None:
            out = {"d" + k: _new(stream, torch.empty_like)(t) for k, t in (("Q", Q), ("K", K), ("V", V))}
            if S0 is not None:
                out["dS0"] = _new(stream)(self.state_shape, dtype=torch.float32, device=Q.device)
        dQ, dK, dV, dS0 = out["dQ"], out["dK"], out["dV"], out.get("dS0")
        if not self._looked_at("backward", Q, K, V, dO, log_decay, lengths, S0, dS1, dQ, dK, dV, dS0):
            for field, t in (("q", Q), ("k", K), ("v", V), ("go", dO), ("gq", dQ), ("gk", dK), ("gv", dV)):
                self._view("backward", field, t)
            self._vectors(log_decay, lengths)
            self._states(S0=S0, dS1=dS1, dS0=dS0)
            self._accept()
        _check(_lib.luna_decay_bwd(self._ref["backward"], log_decay.data_ptr(), Q.data_ptr(), K.data_ptr(), V.data_ptr(),
                                   dO.data_ptr(), _addr(lengths), _addr(S0), _addr(dS1), dQ.data_ptr(), dK.data_ptr(),
                                   dV.data_ptr(), _addr(dS0), *self._ws, self._on(stream)), "luna_decay_bwd")
        return out

    def step(self, q, k, v, log_decay, S, slots=None, o=None, stream=None):
        """One token: q (B, H, d), k (B, Hkv, d), v (B, Hkv, dv); S (nslots, H, d, dv) is advanced in place."""
        if o is None:
            o = _new(stream)(self.state_shape[:2] + self.state_shape[3:], dtype=self.io, device=q.device)
        if not self._looked_at("step", q, k, v, log_decay, S, slots, o):
            for field, t in (("q", q), ("k", k), ("v", v), ("o", o)):
                self._view("step", field, t)
            _want("S", S, (S.shape[0],) + self.state_shape[1:], torch.float32, self.device)
            _dense("S", S)
            self._vectors(log_decay, slots, "slots")
            self._accept()
        _check(_lib.luna_decay_step(self._ref["step"], log_decay.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                    _addr(slots), S.shape[0], S.data_ptr(), o.data_ptr(), self._on(stream)),
               "luna_decay_step")
        return o


class Delta(_Checked):
    """The gated delta rule at one problem shape; owns the workspace, so its calls belong on one stream at a time.
    Q, K: (B, Hk, n, d), V: (B, H, n, dv), any strides with a contiguous last dimension; log_decay, beta: (B, H, n) of
    the tensors' type, any strides; lengths: (B,) int32 or None; states: (B, H, d, dv) fp32."""

    def __init__(self, B, H, n, d, dv, Hk=None, scale=None, io=torch.bfloat16, device="cuda", backward=False):
        self.td = delta_desc(B, H, n, d, dv, Hk, scale, _DTYPES[io])
        super().__init__(self.td)
        self.io, self.device = io, _place(device)
        self._workspace(max(luna_delta_workspace_size(self.td, b) for b in ((False, True) if backward else (False,))))
        qk, vo, gate = (B, self.td.Hk, n, d), (B, H, n, dv), (B, H, n)
        self.shapes = {"q": qk, "k": qk, "v": vo, "o": vo, "g": gate, "beta": gate}
        self.state_shape = (B, H, d, dv)

    def _view(self, kind: str, field: str, name: str, t) -> None:
        """Checks a tensor of rows or gates (of single ones for a step) and notes its strides."""
        shape = self.shapes[field if field in self.shapes else field[1:]]
        rows = len(shape) == 4
        if kind == "step":
            shape = shape[:2] + shape[3:]
        _want(name, t, shape, self.io, self.device)
        s = t.stride()
        if rows and s[-1] != 1 and t.shape[-1] != 1:
            raise ValueError(f"{name}: the last dimension is not contiguous")
        if not any(s[:-1] if rows else s) and (t[..., 0] if rows and t.shape[-1] else t).numel() > 1:
            raise ValueError(f"{name}: one {'row' if rows else 'value'} repeated")
        setattr(self._desc[kind], field, Strides(s[0], s[1], s[2] if kind != "step" else 0))

    def _vector(self, name: str, t) -> None:
        _want(name, t, self.state_shape[:1], torch.int32, self.device)
        _dense(name, t)

    def _states(self, **states) -> None:
        for name, t in states.items():
            _want(name, t, self.state_shape, torch.float32, self.device)
            _dense(name, t)

    def forward(self, Q, K, V, log_decay, beta, lengths=None, S0=None, want_state=False, O=None, S1=None, stream=None):
        """O, or (O, S1) with want_state."""
        given = O  # (a new output lies as V does: not to be looked at again)
        if O is None:
            O = _new(stream, torch.empty_like)(V)
        if not self._looked_at("forward", Q, K, V, log_decay, beta, lengths, S0, given, S1):
            for field, name, t in (("q", "Q", Q), ("k", "K", K), ("v", "V", V), ("g", "log_decay", log_decay),
                                   ("beta", "beta", beta), ("o", "O", O)):
                self._view("forward", field, name, t)
            self._vector("lengths", lengths)
            self._states(S0=S0, S1=S1)
            self._accept()
        if want_state and S1 is None:
            S1 = _new(stream)(self.state_shape, dtype=torch.float32, device=self.device)
        _check(_lib.luna_delta_fwd(self._ref["forward"], log_decay.data_ptr(), beta.data_ptr(), Q.data_ptr(), K.data_ptr(),
                                   V.data_ptr(), _addr(lengths), _addr(S0), O.data_ptr(), _addr(S1), *self._ws,
                                   self._on(stream)), "luna_delta_fwd")
        return (O, S1) if want_state else O

    def backward(self, Q, K, V, dO, log_decay, beta, lengths=None, S0=None, dS1=None, out=None, stream=None):
        """dQ, dK, dV, dlog_decay, dbeta, and dS0 where S0 is given (or `out` holds it), of forward on the same inputs."""
        new = out is None  # (new gradients lie as what they are gradients of)
        if new:
            out = {"d" + k: _new(stream, torch.empty_like)(t)
                   for k, t in (("Q", Q), ("K", K), ("V", V), ("log_decay", log_decay), ("beta", beta))}
            if S0 is not None:
                out["dS0"] = _new(stream)(self.state_shape, dtype=torch.float32, device=self.device)
        dQ, dK, dV, dg, db, dS0 = (out.get("d" + k) for k in ("Q", "K", "V", "log_decay", "beta", "S0"))
        given = (None,) * 6 if new else (dQ, dK, dV, dg, db, dS0)
        if not self._looked_at("backward", Q, K, V, dO, log_decay, beta, lengths, S0, dS1, *given):
            for field, name, t in (("q", "Q", Q), ("k", "K", K), ("v", "V", V), ("g", "log_decay", log_decay),
                                   ("beta", "beta", beta), ("go", "dO", dO), ("gq", "dQ", dQ), ("gk", "dK", dK),
                                   ("gv", "dV", dV), ("gg", "dlog_decay", dg), ("gbeta", "dbeta", db)):
                self._view("backward", field, name, t)
            self._vector("lengths", lengths)
            self._states(S0=S0, dS1=dS1, dS0=dS0)
            self._accept()
        _check(_lib.luna_delta_bwd(self._ref["backward"], log_decay.data_ptr(), beta.data_ptr(), Q.data_ptr(), K.data_ptr(),
                                   V.data_ptr(), dO.data_ptr(), _addr(lengths), _addr(S0), _addr(dS1), dQ.data_ptr(),
                                   dK.data_ptr(), dV.data_ptr(), dg.data_ptr(), db.data_ptr(), _addr(dS0), *self._ws,
                                   self._on(stream)), "luna_delta_bwd")
        return out

    def step(self, q, k, v, log_decay, beta, S, slots=None, o=None, stream=None):
        """One token: q, k (B, Hk, d), v (B, H, dv), log_decay, beta (B, H); S (nslots, H, d, dv) is advanced in place."""
        given = o  # (a new output is contiguous)
        if o is None:
            o = _new(stream)(self.state_shape[:2] + self.state_shape[3:], dtype=self.io, device=self.device)
        if not self._looked_at("step", q, k, v, log_decay, beta, S, slots, given):
            for field, name, t in (("q", "q", q), ("k", "k", k), ("v", "v", v), ("g", "log_decay", log_decay),
                                   ("beta", "beta", beta), ("o", "o", o)):
                self._view("step", field, name, t)
            _want("S", S, (S.shape[0],) + self.state_shape[1:], torch.float32, self.device)
            _dense("S", S)
            self._vector("slots", slots)
            self._accept()
        _check(_lib.luna_delta_step(self._ref["step"], log_decay.data_ptr(), beta.data_ptr(), q.data_ptr(), k.data_ptr(),
                                    v.data_ptr(), _addr(slots), S.shape[0], S.data_ptr(), o.data_ptr(),
                                    self._on(stream)), "luna_delta_step")
        return o


class Beam(_Checked):
    """Beam search over recurrent states: `beams` beams of each of B sequences.  Owns the workspace of select, whose
    calls belong on one stream at a time.  vocab is not needed for reorder; end: the token that ends a sequence, or -1."""

    def __init__(self, B, beams, vocab=0, end=-1, io=torch.bfloat16, device="cuda"):
        self.bd = beam_desc(B, beams, vocab, end, _DTYPES[io])
        super().__init__(self.bd)
        self.io, self.device, self.shape = io, _place(device), (B, beams)
        self._workspace(luna_beam_workspace_size(self.bd))

    def _beams(self, dtype, **tensors) -> None:
        for name, t in tensors.items():
            _want(name, t, self.shape, dtype, self.device)
            _dense(name, t)

    def select(self, logits, scores, done=None, out=None, stream=None):
        """The best continuations of every sequence from logits (B * beams, vocab), running log-probabilities scores
        (B, beams) fp32 and, with an end token, done (B, beams) bool: {"scores", "tokens", "parents"} and with an end
        token "done", each (B, beams), best first.  `out` may hold scores and done themselves."""
        given = (None,) * 4  # (new outputs are as they have to be)
        if out is None:
            new, at, shape = _new(stream), self.device, self.shape
            out = {"scores": new(shape, dtype=torch.float32, device=at), "tokens": new(shape, dtype=torch.int32, device=at),
                   "parents": new(shape, dtype=torch.int32, device=at)}
            if self.bd.end >= 0:
                out["done"] = new(shape, dtype=torch.bool, device=at)
            to = [out["scores"], out["tokens"], out["parents"], out.get("done")]
        else:
            given = to = [out.get(k) for k in ("scores", "tokens", "parents", "done")]
        if not self._looked_at("select", logits, scores, done, *given):
            _set_rows(self._desc["forward"], "ld", "logits", logits, (self.shape[0] * self.shape[1], self.bd.V), self.io,
                      self.device)
            if any(t is None for t in to[:3]):
                raise ValueError("out: needs scores, tokens and parents")
            self._beams(torch.float32, scores=scores, scores_out=to[0])
            self._beams(torch.int32, tokens=to[1], parents=to[2])
            self._beams(torch.bool, done=done, done_out=to[3])
            self._accept()
        _check(_lib.luna_beam_select(self._ref["forward"], logits.data_ptr(), scores.data_ptr(), _addr(done),
                                     *[_addr(t) for t in to], *self._ws, self._on(stream)), "luna_beam_select")
        return out

    def reorder(self, parents, slots, *pools, out=None, stream=None):
        """The states in `pools` (each (nslots, ...), contiguous) follow their beams in place; returns the new beams'
        slots (B, beams), for slots (B, beams) int32 of the old ones."""
        given = out
        if out is None:
            out = _new(stream)(self.shape, dtype=torch.int32, device=self.device)
        if not self._looked_at("reorder", parents, slots, given, *pools):
            self._beams(torch.int32, parents=parents, slots=slots, out=out)
            for i, t in enumerate(pools):
                _want(f"pools[{i}]", t, t.shape, t.dtype, self.device)
                if t.dim() < 1:
                    raise ValueError(f"pools[{i}]: no slots")
                _dense(f"pools[{i}]", t)
            self._accept()
        handle = self._on(stream)
        for at, n, size in [(t.data_ptr(), t.shape[0], t.nbytes // t.shape[0] if t.shape[0] else 0) for t in pools] or [(None, 0, 0)]:
            _check(_lib.luna_beam_reorder(self._ref["forward"], parents.data_ptr(), slots.data_ptr(), n, at, size,
                                          out.data_ptr(), handle), "luna_beam_reorder")
        return out


def _set_rows(desc, field: str, name: str, t, shape, dtype, device) -> None:
    """Checks a matrix of contiguous rows and puts the distance of its rows into a descriptor."""
    if t is None:
        setattr(desc, field, 0)
        return
    _want(name, t, shape, dtype, device)
    if (t.stride(1) != 1 and t.shape[1] > 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{name}: rows are not contiguous")
    setattr(desc, field, t.stride(0) if t.shape[0] > 1 else 0)


class BlockNorm(_Checked):
    """The norms after and before a block with its gate and residual scale, over (rows, cols) matrices
    whose rows may be strided; weights are (cols,) fp32.  Owns the workspace of the backward pass, whose
    calls belong on one stream at a time."""

    def __init__(self, rows, cols, groups=1, kind="rms", gate="none", res_scale=1.0, eps=1e-6, io=torch.bfloat16,
                 device="cuda", backward=False):
        self.nd = norm_desc(rows, cols, groups, kind, gate, res_scale, eps, _DTYPES[io])
        super().__init__(self.nd)
        self.io, self.device, self.shape = io, _place(device), (rows, cols)
        if backward:
            self._workspace(luna_norm_workspace_size(self.nd))

    def _rows(self, kind: str, **matrices) -> None:
        for name, t in matrices.items():
            _set_rows(self._desc[kind], "ld" + name, name, t, self.shape, self.io, self.device)

    def _weights(self, **weights) -> None:
        for name, t in weights.items():
            _want(name, t, self.shape[1:], torch.float32, self.device)
            _dense(name, t)

    def forward(self, x, y, gate=None, w_post=None, w_pre=None, b_post=None, b_pre=None, X=None, H=None, stream=None):
        """{"X": x'} where there is a residual or no second norm (or X is given), {"H": h} with w_pre."""
        if X is None and ((x is not None and y is not None) or w_pre is None):
            X = _new(stream)(self.shape, dtype=self.io, device=(y if x is None else x).device)
        if H is None and w_pre is not None:
            H = _new(stream)(self.shape, dtype=self.io, device=(y if x is None else x).device)
        if not self._looked_at("forward", x, y, gate, w_post, w_pre, b_post, b_pre, X, H):
            self._rows("forward", x=x, y=y, gate=gate, X=X, H=H)
            self._weights(w_post=w_post, w_pre=w_pre, b_post=b_post, b_pre=b_pre)
            self._accept()
        _check(_lib.luna_norm_fwd(self._ref["forward"], _addr(x), _addr(y), _addr(gate), _addr(w_post), _addr(b_post),
                                  _addr(w_pre), _addr(b_pre), _addr(X), _addr(H), self._on(stream)), "luna_norm_fwd")
        if X is None:
            return {"H": H}
        return {"X": X} if H is None else {"X": X, "H": H}

    def backward(self, x, y, gate, w_post, w_pre, dX, dH, b_post=None, b_pre=None, out=None, stream=None):
        """dx, dy, dgate, dw_post, dw_pre of what forward was given, and db_post, db_pre of given biases."""
        if out is None:
            out = {k: _new(stream)(self.shape, dtype=self.io, device=t.device)
                   for k, t in (("dx", x), ("dy", y), ("dgate", gate)) if t is not None}
            out.update({k: _new(stream, torch.empty_like)(t)
                        for k, t in (("dw_post", w_post), ("dw_pre", w_pre), ("db_post", b_post), ("db_pre", b_pre))
                        if t is not None})
        g = [out.get(k) for k in ("dx", "dy", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")]
        if not self._looked_at("backward", x, y, gate, w_post, w_pre, dX, dH, b_post, b_pre, *g):
            self._rows("backward", x=x, y=y, gate=gate, dX=dX, dH=dH, dx=g[0], dy=g[1], dgate=g[2])
            self._weights(w_post=w_post, w_pre=w_pre, b_post=b_post, b_pre=b_pre, dw_post=g[3], db_post=g[4],
                          dw_pre=g[5], db_pre=g[6])
            self._accept()
        _check(_lib.luna_norm_bwd(self._ref["backward"], _addr(x), _addr(y), _addr(gate), _addr(w_post), _addr(b_post),
                                  _addr(w_pre), _addr(dX), _addr(dH), *[_addr(t) for t in g], *self._ws,
                                  self._on(stream)), "luna_norm_bwd")
        return out


class Linear(_Checked):
    """Y = act(X W^T + bias) + R for X (m, k), W (n, k), rows strided or not; owns the workspace, so its
    calls belong on one stream at a time."""

    def __init__(self, m, n, k, act="none", io=torch.bfloat16, device="cuda", backward=False):
        self.ld = linear_desc(m, n, k, act, _DTYPES[io])
        super().__init__(self.ld)
        self.io, self.device, self.m, self.n, self.k = io, _place(device), m, n, k
        self._workspace(max(luna_linear_workspace_size(self.ld, b) for b in ((False, True) if backward else (False,))))

    def _rows(self, kind: str, **matrices) -> None:
        shapes = {"x": (self.m, self.k), "dx": (self.m, self.k), "w": (self.n, self.k)}
        for name, t in matrices.items():
            _set_rows(self._desc[kind], "ld" + name, name, t, shapes.get(name, (self.m, self.n)), self.io, self.device)

    def _vector(self, name: str, t, shape) -> None:
        _want(name, t, shape, self.io, self.device)
        _dense(name, t)

    def forward(self, x, W, bias=None, r=None, save_z=False, Y=None, Z=None, stream=None):
        """Y, or (Y, z) with save_z."""
        if Y is None:
            Y = _new(stream)((self.m, self.n), dtype=self.io, device=x.device)
        if save_z and Z is None:
            Z = _new(stream)((self.m, self.n), dtype=self.io, device=x.device)
        if not self._looked_at("forward", x, W, bias, r, Y, Z):
            self._rows("forward", x=x, w=W, r=r, y=Y, z=Z)
            self._vector("bias", bias, (self.n,))
            self._accept()
        _check(_lib.luna_linear_fwd(self._ref["forward"], x.data_ptr(), W.data_ptr(), _addr(bias), _addr(r), Y.data_ptr(),
                                    _addr(Z), *self._ws, self._on(stream)), "luna_linear_fwd")
        return (Y, Z) if save_z else Y

    def backward(self, x, W, dY, Z=None, bias=False, out=None, stream=None):
        """dX, dW and with `bias` db; Z is forward's z (needed with an activation)."""
        if out is None:
            out = {"dX": _new(stream)((self.m, self.k), dtype=self.io, device=dY.device),
                   "dW": _new(stream)((self.n, self.k), dtype=self.io, device=dY.device)}
            if bias:
                out["db"] = _new(stream)(self.n, dtype=self.io, device=dY.device)
        dX, dW, db = out.get("dX"), out.get("dW"), out.get("db")
        if not self._looked_at("backward", x, W, Z, dY, dX, dW, db):
            self._rows("backward", x=x, w=W, z=Z, dy=dY, dx=dX)
            self._vector("dW", dW, (self.n, self.k))
            self._vector("db", db, (self.n,))
            self._accept()
        _check(_lib.luna_linear_bwd(self._ref["backward"], x.data_ptr(), W.data_ptr(), _addr(Z), dY.data_ptr(), _addr(dX),
                                    _addr(dW), _addr(db), *self._ws, self._on(stream)), "luna_linear_bwd")
        return out
