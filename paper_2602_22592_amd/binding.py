"""Thin ctypes binding over libpquant.so: argument marshalling only.

Every computation runs in the HIP kernels behind the C ABI (include/pquant.h).  PyTorch is used for
device memory and the current stream.  There is no CPU fallback: if the library has not been
built, the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpquant.so")

PQ_F32, PQ_BF16 = 0, 1
PQ_W_MASTER, PQ_W_PACKED = 0, 1
PQ_STE_IDENTITY, PQ_STE_CLIP = 0, 1
PQ_HP_LOWRANK_BF16, PQ_HP_LOWRANK_INT8 = 0, 1
PQ_PACKED_ROWMAJOR, PQ_PACKED_TILED64 = 0, 1
PQ_KV_BF16, PQ_KV_INT8 = 0, 1
PQ_ROPE_HALF, PQ_ROPE_PAIRS = 0, 1
PQ_STATE_F32, PQ_STATE_8BIT = 0, 1

EXPORTS = [
    "pq_version", "pq_last_error_string", "pq_quant_act", "pq_pack_workspace_bytes", "pq_pack_sign",
    "pq_router_topk", "pq_onebit_acc", "pq_linear_ctx_bytes", "pq_linear_workspace_bytes",
    "pq_linear_fwd", "pq_linear_bwd", "pq_prof_enable", "pq_prof_count", "pq_prof_label", "pq_prof_read",
    "pq_prof_reset", "pq_decode_workspace_bytes", "pq_decode_gemv", "pq_pack_tiled64_bytes", "pq_pack_retile64", "pq_ffn_ctx_bytes", "pq_ffn_workspace_bytes",
    "pq_ffn_fwd", "pq_ffn_bwd", "pq_glue_lincomb", "pq_glue_gather_rows",
    "pq_rmsnorm_quant_fwd", "pq_rmsnorm_bwd_workspace_bytes", "pq_rmsnorm_bwd",
    "pq_linear_norm_ctx_bytes", "pq_linear_norm_workspace_bytes", "pq_linear_norm_fwd", "pq_linear_norm_bwd",
    "pq_hp_int8_ctx_bytes", "pq_hp_int8_workspace_bytes", "pq_hp_int8_fwd", "pq_hp_int8_bwd", "pq_decode_gemv_int8",
    "pq_decode_ffn_workspace_bytes", "pq_decode_ffn", "pq_rmsnorm_bwd_static_max_bytes", "pq_rmsnorm_bwd_static",
    "pq_groupwise_workspace_bytes", "pq_groupwise_fwd", "pq_ffn_ctx_section",
    "pq_kv_cache_bytes", "pq_kv_write", "pq_kv_read", "pq_attn_decode_workspace_bytes", "pq_attn_decode", "pq_attn_prefill",
    "pq_rope", "pq_self_attn_fwd", "pq_self_attn_bwd_workspace_bytes", "pq_self_attn_bwd",
    "pq_adamw_plan_bytes", "pq_adamw_plan", "pq_adamw_step", "pq_adamw_read",
]


class LinearDesc(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32), ("hp_rank", C.c_int32),
                ("n_experts", C.c_int32), ("top_k", C.c_int32), ("io_dtype", C.c_int32), ("w_kind", C.c_int32),
                ("ste_mode", C.c_int32), ("ste_tau", C.c_float), ("alpha", C.c_float), ("beta", C.c_float),
                ("hp_kind", C.c_int32)]


class DecodeDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32), ("hp_rank", C.c_int32),
                ("n_experts", C.c_int32), ("top_k", C.c_int32), ("n_layers", C.c_int32),
                ("packed_layout", C.c_int32), ("alpha", C.c_float)]


class FFNDesc(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("d_model", C.c_int32), ("d_ffn", C.c_int32), ("hp_rank", C.c_int32),
                ("n_experts", C.c_int32), ("top_k", C.c_int32), ("io_dtype", C.c_int32), ("alpha", C.c_float),
                ("beta", C.c_float), ("hp_kind", C.c_int32)]


class DecodeFFNDesc(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("d_ffn", C.c_int32), ("hp_rank", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("n_layers", C.c_int32), ("alpha", C.c_float), ("batch", C.c_int32)]


class KVDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kv_kind", "n_kv_heads", "d_head", "page_tokens", "n_pages", "n_seqs", "max_pages")]


class AttnDesc(C.Structure):
    _fields_ = [("kv", KVDesc), ("n_heads", C.c_int32), ("causal", C.c_int32), ("window", C.c_int32), ("max_len", C.c_int32),
                ("scale", C.c_float)]


class RopeDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "n_kv_heads", "d_head", "rot_dim", "layout", "inverse", "n_seqs")] + [("scale", C.c_float)]


class SelfAttnDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "n_kv_heads", "d_head", "n_seqs", "causal", "window")] + [("scale", C.c_float)]


class AdamWTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "master", "m", "v", "steps", "m_values", "v_values")] + [("n", C.c_int64)]


class AdamWDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_tensors", "param_dtype", "grad_dtype", "state_kind", "has_masters", "has_values")] + [
        (n, C.c_double) for n in ("beta1", "beta2", "eps")]


class PQError(RuntimeError):
    pass


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_22592_amd.build` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        L.pq_last_error_string.restype = C.c_char_p
        L.pq_prof_label.restype = C.c_char_p
        for name in ("pq_pack_workspace_bytes", "pq_linear_ctx_bytes", "pq_linear_workspace_bytes",
                     "pq_decode_workspace_bytes", "pq_pack_tiled64_bytes", "pq_ffn_ctx_bytes",
                     "pq_ffn_workspace_bytes", "pq_rmsnorm_bwd_workspace_bytes", "pq_linear_norm_ctx_bytes",
                     "pq_linear_norm_workspace_bytes", "pq_hp_int8_ctx_bytes", "pq_hp_int8_workspace_bytes",
                     "pq_decode_ffn_workspace_bytes", "pq_rmsnorm_bwd_static_max_bytes", "pq_kv_cache_bytes",
                     "pq_attn_decode_workspace_bytes", "pq_self_attn_bwd_workspace_bytes", "pq_adamw_plan_bytes"):
            getattr(L, name).restype = C.c_size_t
        p, i, l, n = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        kv, attn = C.POINTER(KVDesc), C.POINTER(AttnDesc)
        L.pq_kv_write.argtypes = [kv, p, p, i, i, l, l, p, p, p, p, n, p]
        L.pq_kv_read.argtypes = [kv, p, n, p, p, p, i, p, p, i, l, l, p]
        L.pq_attn_decode.argtypes = [attn, p, l, p, n, p, p, p, p, p, n, p]
        L.pq_attn_prefill.argtypes = [attn, p, l, i, p, p, n, p, p, p, p, p]
        rope, self_attn, adamw = C.POINTER(RopeDesc), C.POINTER(SelfAttnDesc), C.POINTER(AdamWDesc)
        L.pq_rope.argtypes = [rope, p, l, p, l, i, i, p, p, p, p, l, p, l, p]
        L.pq_self_attn_fwd.argtypes = [self_attn, p, l, p, l, p, l, i, p, p, p, p]
        L.pq_self_attn_bwd_workspace_bytes.argtypes = [self_attn, i]
        L.pq_self_attn_bwd.argtypes = [self_attn, p, p, l, p, l, p, l, p, p, i, p, p, l, p, l, p, l, p, n, p]
        L.pq_adamw_plan_bytes.argtypes = [adamw, C.POINTER(AdamWTensor)]
        L.pq_adamw_plan.argtypes = [adamw, C.POINTER(AdamWTensor), p, n]
        L.pq_adamw_step.argtypes = [adamw, p, n, p, p]
        L.pq_adamw_read.argtypes = [adamw, p, n, p]
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise PQError(f"libpquant error {rc}: {lib().pq_last_error_string().decode()}")


def _p(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dt(t):
    if t.dtype == torch.float32:
        return PQ_F32
    if t.dtype == torch.bfloat16:
        return PQ_BF16
    raise PQError(f"unsupported dtype {t.dtype}")


def _bytes(n, device):
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)


def version():
    return lib().pq_version()


def quant_act(X):
    T, K = X.shape
    Xq = torch.empty((T, K), dtype=torch.int8, device=X.device)
    gamma = torch.empty((T,), dtype=torch.float32, device=X.device)
    _check(lib().pq_quant_act(_p(X), _dt(X), T, K, _p(Xq), _p(gamma), _stream()))
    return Xq, gamma


def quant_act_into(X, Xq, gamma):
    T, K = X.shape
    _check(lib().pq_quant_act(_p(X), _dt(X), T, K, _p(Xq), _p(gamma), _stream()))


def rmsnorm_quant_fwd_into(X, gain, eps, Xn, Xq, gamma, Xt, rstd):
    """Same call as rmsnorm_quant_fwd, writing into buffers the caller holds (any of Xn, Xt, rstd may be None)."""
    T, K = X.shape
    _check(lib().pq_rmsnorm_quant_fwd(_p(X), _p(gain), _dt(X), T, K, C.c_float(eps), _p(Xn), _p(Xq), _p(gamma), _p(Xt),
                                      _p(rstd), _stream()))


def rmsnorm_bwd_into(dXn, X, gain, rstd, dX, dgain, ws):
    T, K = X.shape
    _check(lib().pq_rmsnorm_bwd(_p(dXn), _p(X), _p(gain), _p(rstd), _dt(X), T, K, _p(dX), _p(dgain), _p(ws),
                                C.c_size_t(ws.numel()), _stream()))


def rmsnorm_bwd_static_into(dXn, X, gain, rstd, dX, dgain):
    """pq_rmsnorm_bwd_static: no workspace argument, nothing allocated by the call."""
    T, K = X.shape
    _check(lib().pq_rmsnorm_bwd_static(_p(dXn), _p(X), _p(gain), _p(rstd), _dt(X), T, K, _p(dX), _p(dgain), _stream()))


def rmsnorm_bwd_static_max_bytes():
    return lib().pq_rmsnorm_bwd_static_max_bytes()


def rmsnorm_quant_fwd(X, gain, eps, want_xn=True, want_xt=True, want_rstd=True):
    """Returns (Xn, Xq, gamma, Xt, rstd); entries not asked for are None."""
    T, K = X.shape
    Xq = torch.empty((T, K), dtype=torch.int8, device=X.device)
    gamma = torch.empty((T,), dtype=torch.float32, device=X.device)
    Xn = torch.empty_like(X) if want_xn else None
    Xt = torch.empty((T, K), dtype=torch.bfloat16, device=X.device) if want_xt else None
    rstd = torch.empty((T,), dtype=torch.float32, device=X.device) if want_rstd else None
    _check(lib().pq_rmsnorm_quant_fwd(_p(X), _p(gain), _dt(X), T, K, C.c_float(eps), _p(Xn), _p(Xq), _p(gamma), _p(Xt),
                                      _p(rstd), _stream()))
    return Xn, Xq, gamma, Xt, rstd


def rmsnorm_bwd(dXn, X, gain, rstd, ws=None):
    """Returns (dX, dgain)."""
    T, K = X.shape
    dX = torch.empty_like(X)
    dgain = torch.empty((K,), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = _bytes(lib().pq_rmsnorm_bwd_workspace_bytes(T, K), X.device)
    _check(lib().pq_rmsnorm_bwd(_p(dXn), _p(X), _p(gain), _p(rstd), _dt(X), T, K, _p(dX), _p(dgain), _p(ws),
                                C.c_size_t(ws.numel()), _stream()))
    return dX, dgain


def pack_sign(W, transposed=False):
    N, K = W.shape
    P = torch.empty((N, (K + 31) // 32), dtype=torch.int32, device=W.device)
    Pt = torch.empty((K, (N + 31) // 32), dtype=torch.int32, device=W.device) if transposed else None
    ml = torch.empty((2,), dtype=torch.float32, device=W.device)
    nws = lib().pq_pack_workspace_bytes(N, K)
    ws = _bytes(nws, W.device)
    _check(lib().pq_pack_sign(_p(W), _dt(W), N, K, _p(P), _p(Pt), _p(ml), _p(ws), C.c_size_t(ws.numel()), _stream()))
    return P, Pt, ml


def router_topk(X, Wr, k, want_probs=True):
    T, K = X.shape
    E = Wr.shape[0]
    idx = torch.empty((T, k), dtype=torch.int32, device=X.device)
    gate = torch.empty((T, k), dtype=torch.float32, device=X.device)
    probs = torch.empty((T, E), dtype=torch.float32, device=X.device) if want_probs else None
    _check(lib().pq_router_topk(_p(X), _p(Wr), _dt(X), T, K, E, k, _p(idx), _p(gate), _p(probs), _stream()))
    return idx, gate, probs


def onebit_acc(Xq, P, N):
    T, K = Xq.shape
    acc = torch.empty((T, N), dtype=torch.int32, device=Xq.device)
    _check(lib().pq_onebit_acc(_p(Xq), _p(P), T, K, N, _p(acc), _stream()))
    return acc


def make_desc(tokens, d_in, d_out, hp_rank=0, n_experts=1, top_k=1, io_dtype=PQ_BF16, w_kind=PQ_W_MASTER,
              ste_mode=PQ_STE_IDENTITY, ste_tau=0.0, alpha=2.0, beta=0.2, hp_kind=PQ_HP_LOWRANK_BF16):
    return LinearDesc(tokens, d_in, d_out, hp_rank, n_experts, top_k, io_dtype, w_kind, ste_mode, ste_tau,
                      alpha, beta, hp_kind)


class LinearBuffers:
    """Caller-owned ctx / workspace for one descriptor (allocated once, reused across steps)."""

    def __init__(self, desc, device="cuda", ws=None):
        nctx = lib().pq_linear_ctx_bytes(C.byref(desc))
        nws = lib().pq_linear_workspace_bytes(C.byref(desc))
        if nctx == 0 or nws == 0:
            raise PQError(f"bad descriptor: {lib().pq_last_error_string().decode()}")
        self.ctx = _bytes(nctx, device)
        self.ws = ws if ws is not None else _bytes(nws, device)   # scratch may be shared between layers


def linear_fwd(desc, X, W, Y, bufs, A=None, B=None, Wr=None, mu_lambda=None, save=True):
    ctx = bufs.ctx if save else None
    _check(lib().pq_linear_fwd(C.byref(desc), _p(X), _p(W), _p(mu_lambda), _p(A), _p(B), _p(Wr), _p(Y),
                               _p(ctx), C.c_size_t(0 if ctx is None else ctx.numel()),
                               _p(bufs.ws), C.c_size_t(bufs.ws.numel()), _stream()))
    return Y


def linear_bwd(desc, dY, X, W, bufs, dX, dW, d_ab, A=None, B=None, Wr=None, dA=None, dB=None, dWr=None):
    _check(lib().pq_linear_bwd(C.byref(desc), _p(dY), _p(X), _p(W), _p(A), _p(B), _p(Wr),
                               _p(bufs.ctx), C.c_size_t(bufs.ctx.numel()), _p(dX), _p(dW), _p(dA), _p(dB),
                               _p(dWr), _p(d_ab), _p(bufs.ws), C.c_size_t(bufs.ws.numel()), _stream()))
    return dX, dW, d_ab


class LinearNormBuffers:
    """ctx / workspace of the linear with its normalisation in front."""

    def __init__(self, desc, device="cuda"):
        nctx = lib().pq_linear_norm_ctx_bytes(C.byref(desc))
        nws = lib().pq_linear_norm_workspace_bytes(C.byref(desc))
        if nctx == 0 or nws == 0:
            raise PQError(f"bad descriptor: {lib().pq_last_error_string().decode()}")
        self.ctx = _bytes(nctx, device)
        self.ws = _bytes(nws, device)


def linear_norm_fwd(desc, X, gain, eps, W, Y, bufs, A=None, B=None, Wr=None):
    _check(lib().pq_linear_norm_fwd(C.byref(desc), _p(X), _p(gain), C.c_float(eps), _p(W), _p(A), _p(B), _p(Wr), _p(Y),
                                    _p(bufs.ctx), C.c_size_t(bufs.ctx.numel()), _p(bufs.ws), C.c_size_t(bufs.ws.numel()),
                                    _stream()))
    return Y


def linear_norm_bwd(desc, dY, X, gain, W, bufs, dX, dgain, dW, d_ab, A=None, B=None, Wr=None, dA=None, dB=None, dWr=None):
    _check(lib().pq_linear_norm_bwd(C.byref(desc), _p(dY), _p(X), _p(gain), _p(W), _p(A), _p(B), _p(Wr), _p(bufs.ctx),
                                    C.c_size_t(bufs.ctx.numel()), _p(dX), _p(dgain), _p(dW), _p(dA), _p(dB), _p(dWr), _p(d_ab),
                                    _p(bufs.ws), C.c_size_t(bufs.ws.numel()), _stream()))
    return dX, dgain, dW, d_ab


class HpInt8Buffers:
    """ctx and workspace of the INT8 high-precision branch, with views of what the forward saved."""

    def __init__(self, T, K, N, r, device="cuda"):
        self.shape = (T, K, N, r)
        self.ctx = _bytes(lib().pq_hp_int8_ctx_bytes(T, K, N, r), device)
        self.ws = _bytes(lib().pq_hp_int8_workspace_bytes(T, K, N, r), device)

    def views(self):
        """(q_a, g_a, q_b, g_b, H, q_h, g_h) as tensors over ctx (same order and 256-byte rounding as the library)."""
        T, K, N, r = self.shape
        off = 0

        def take(nbytes, dtype, shape):
            nonlocal off
            v = self.ctx[off:off + nbytes].view(dtype).view(shape)
            off += (nbytes + 255) // 256 * 256
            return v
        q_a = take(r * K, torch.int8, (r, K)); g_a = take(r * 4, torch.float32, (r,)); take(r * K * 2, torch.bfloat16, (r, K))
        q_b = take(N * r, torch.int8, (N, r)); g_b = take(N * 4, torch.float32, (N,)); take(N * r * 2, torch.bfloat16, (N, r))
        H = take(T * r * 2, torch.bfloat16, (T, r)); q_h = take(T * r, torch.int8, (T, r)); g_h = take(T * 4, torch.float32, (T,))
        return q_a, g_a, q_b, g_b, H, q_h, g_h


def hp_int8_fwd(Xq, gamma_x, A, B, alpha, Y, bufs, accumulate=False):
    T, K, N, r = bufs.shape
    _check(lib().pq_hp_int8_fwd(_p(Xq), _p(gamma_x), _p(A), _p(B), _dt(A), T, K, N, r, C.c_float(alpha), _p(Y),
                                int(accumulate), _p(bufs.ctx), C.c_size_t(bufs.ctx.numel()), _p(bufs.ws),
                                C.c_size_t(bufs.ws.numel()), _stream()))


def hp_int8_bwd(dY, Xt, alpha, bufs, dX, dA, dB, accumulate_dX=False):
    T, K, N, r = bufs.shape
    _check(lib().pq_hp_int8_bwd(_p(dY), _p(Xt), _dt(dY), T, K, N, r, C.c_float(alpha), _p(bufs.ctx),
                                C.c_size_t(bufs.ctx.numel()), _p(dX), int(accumulate_dX), _p(dA), _p(dB), _p(bufs.ws),
                                C.c_size_t(bufs.ws.numel()), _stream()))


def groupwise_fwd(X, W, beta, group=64, Y=None, ws=None):
    """Sec. 4.6 contrast: the 1-bit forward with one fp16 scale per 64 weights (group=64) or the per-tensor scale in the
    same kernel (group=0).  X [T][K], W [N][K] bf16 on the device; returns Y [T][N] fp32."""
    import torch
    T, K = X.shape
    N = W.shape[0]
    lib().pq_groupwise_workspace_bytes.restype = C.c_size_t
    nbytes = lib().pq_groupwise_workspace_bytes(T, K, N)
    if ws is None:
        ws = torch.empty((max(int(nbytes), 256),), dtype=torch.uint8, device=X.device)
    if Y is None:
        Y = torch.empty((T, N), dtype=torch.float32, device=X.device)
    _check(lib().pq_groupwise_fwd(_p(X), _p(W), _dt(X), T, K, N, int(group), C.c_float(beta), _p(Y), _p(ws),
                                  C.c_size_t(ws.numel()), _stream()))
    return Y


def prof_enable(on=True):
    _check(lib().pq_prof_enable(1 if on else 0))


def prof_reset():
    _check(lib().pq_prof_reset())


def prof_read():
    """{label: (total_ms, launches)} for every kernel label with at least one recorded launch."""
    out = {}
    for i in range(lib().pq_prof_count()):
        ms, n = C.c_double(0), C.c_int(0)
        _check(lib().pq_prof_read(i, C.byref(ms), C.byref(n)))
        if n.value:
            out[lib().pq_prof_label(i).decode()] = (ms.value, n.value)
    return out


def decode_workspace(desc, device="cuda"):
    n = lib().pq_decode_workspace_bytes(C.byref(desc))
    if n == 0:
        raise PQError(f"bad decode descriptor: {lib().pq_last_error_string().decode()}")
    return _bytes(n, device)


def decode_gemv(desc, X, packed, scale_fp16, Y, ws, A=None, B=None, Wr=None, acc_out=None):
    """scale_fp16: int16/uint16 tensor [L] holding the fp16 bits of beta*lambda per layer."""
    _check(lib().pq_decode_gemv(C.byref(desc), _p(X), _p(packed), _p(scale_fp16), _p(A), _p(B), _p(Wr), _p(Y),
                                _p(acc_out), _p(ws), C.c_size_t(ws.numel()), _stream()))
    return Y


def quant_rows(W):
    """AbsMax INT8 codes and gammas of the rows of the last axis of a bf16 / fp32 tensor (the activation quantiser
    applied to weight rows): returns (codes of W's shape, gammas of W's shape without the last axis)."""
    K = W.shape[-1]
    q, g = quant_act(W.reshape(-1, K).contiguous())
    return q.view(W.shape), g.view(W.shape[:-1])


def decode_gemv_int8(desc, X, packed, scale_fp16, Y, ws, Aq, gA, Bq, gB, Wr, acc_out=None):
    _check(lib().pq_decode_gemv_int8(C.byref(desc), _p(X), _p(packed), _p(scale_fp16), _p(Aq), _p(gA), _p(Bq), _p(gB),
                                     _p(Wr), _p(Y), _p(acc_out), _p(ws), C.c_size_t(ws.numel()), _stream()))
    return Y


def decode_ws_hidden(desc, ws):
    """The expert hidden states [L][B][top_k][r] (fp32) inside a decode workspace (same section order and 256-byte
    rounding as the library: codes, bit planes, row sums, gammas, indices, gates, hidden states)."""
    L, B, K, k, r = desc.n_layers, desc.batch, desc.d_in, desc.top_k, desc.hp_rank
    off = 0
    for nbytes in (L * B * K, L * B * 8 * (K // 32) * 4, L * B * 4, L * B * 4, L * B * k * 4, L * B * k * 4):
        off = (off + nbytes + 255) // 256 * 256
    return ws[off:off + L * B * k * r * 4].view(torch.float32).view(L, B, k, r)


def decode_ws_idx(desc, ws):
    """The selected expert indices [L][B][top_k] (int32) inside a decode workspace (section order as in decode_ws_hidden)."""
    L, B, K, k = desc.n_layers, desc.batch, desc.d_in, desc.top_k
    off = 0
    for nbytes in (L * B * K, L * B * 8 * (K // 32) * 4, L * B * 4, L * B * 4):
        off = (off + nbytes + 255) // 256 * 256
    return ws[off:off + L * B * k * 4].view(torch.int32).view(L, B, k)


def decode_ffn_workspace(desc, device="cuda"):
    n = lib().pq_decode_ffn_workspace_bytes(C.byref(desc))
    if n == 0:
        raise PQError(f"bad decode FFN descriptor: {lib().pq_last_error_string().decode()}")
    return _bytes(n, device)


def decode_ffn(desc, X, packed_upgate, scale_upgate, packed_down, scale_down, UpGate, Down, Wr, Y, ws, acc_upgate=None):
    _check(lib().pq_decode_ffn(C.byref(desc), _p(X), _p(packed_upgate), _p(scale_upgate), _p(packed_down), _p(scale_down),
                               _p(UpGate), _p(Down), _p(Wr), _p(Y), _p(acc_upgate), _p(ws), C.c_size_t(ws.numel()), _stream()))
    return Y


def pack_retile64(P, K):
    """Row-major packed words [N][K/32] -> the row-interleaved order used by batch-1 decode."""
    N = P.shape[0]
    n = lib().pq_pack_tiled64_bytes(N, K)
    if n == 0:
        raise PQError("pq_pack_tiled64_bytes: bad shape")
    T = torch.empty((n // 4,), dtype=torch.int32, device=P.device)
    _check(lib().pq_pack_retile64(_p(P), N, K, _p(T), _stream()))
    return T


class FFNBuffers:
    def __init__(self, desc, device="cuda", ws=None):
        nctx = lib().pq_ffn_ctx_bytes(C.byref(desc))
        nws = lib().pq_ffn_workspace_bytes(C.byref(desc))
        if nctx == 0 or nws == 0:
            raise PQError(f"bad FFN descriptor: {lib().pq_last_error_string().decode()}")
        self.ctx = _bytes(nctx, device)
        self.ws = ws if ws is not None else _bytes(nws, device)


FFN_CTX_XQ, FFN_CTX_GAMMA_X, FFN_CTX_U, FFN_CTX_G, FFN_CTX_HQ, FFN_CTX_GAMMA_H = range(6)


def ffn_ctx_section(desc, bufs, section):
    """The bytes of one stored intermediate of pq_ffn_fwd inside bufs.ctx (a uint8 view)."""
    off, n = C.c_size_t(0), C.c_size_t(0)
    _check(lib().pq_ffn_ctx_section(C.byref(desc), int(section), C.byref(off), C.byref(n)))
    return bufs.ctx[off.value:off.value + n.value]


def ffn_fwd(desc, X, W_up, W_gate, W_down, Up, Gate, Down, Wr, Y, bufs):
    _check(lib().pq_ffn_fwd(C.byref(desc), _p(X), _p(W_up), _p(W_gate), _p(W_down), _p(Up), _p(Gate), _p(Down), _p(Wr),
                            _p(Y), _p(bufs.ctx), C.c_size_t(bufs.ctx.numel()), _p(bufs.ws), C.c_size_t(bufs.ws.numel()),
                            _stream()))
    return Y


def ffn_bwd(desc, dY, X, Up, Gate, Down, Wr, bufs, dX, dW_up, dW_gate, dW_down, dUp, dGate, dDown, dWr, d_ab):
    _check(lib().pq_ffn_bwd(C.byref(desc), _p(dY), _p(X), _p(Up), _p(Gate), _p(Down), _p(Wr), _p(bufs.ctx),
                            C.c_size_t(bufs.ctx.numel()), _p(dX), _p(dW_up), _p(dW_gate), _p(dW_down), _p(dUp),
                            _p(dGate), _p(dDown), _p(dWr), _p(d_ab), _p(bufs.ws), C.c_size_t(bufs.ws.numel()), _stream()))


def make_kv_desc(kv_kind, n_kv_heads, d_head, page_tokens, n_pages, n_seqs, max_pages):
    return KVDesc(kv_kind, n_kv_heads, d_head, page_tokens, n_pages, n_seqs, max_pages)


def make_attn_desc(kv, n_heads, scale=None, causal=True, window=0, max_len=0):
    """scale: 1 / sqrt(d_head) unless given.  max_len: an upper bound of the sequences' lengths (0: what the page table can hold)."""
    return AttnDesc(kv, n_heads, int(causal), window, max_len, kv.d_head ** -0.5 if scale is None else scale)


def kv_cache(desc, device="cuda"):
    n = lib().pq_kv_cache_bytes(C.byref(desc))
    if n == 0:
        raise PQError(f"bad cache descriptor: {lib().pq_last_error_string().decode()}")
    return _bytes(n, device)


def attn_decode_workspace(desc, device="cuda"):
    n = lib().pq_attn_decode_workspace_bytes(C.byref(desc))
    if n == 0:
        raise PQError(f"bad attention descriptor: {lib().pq_last_error_string().decode()}")
    return _bytes(n, device)


# the current stream of a device as an integer, and the current device; the public calls build a Stream object and look whether the runtime
# is up, which takes as long as half a launch
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _kv_check(kv, cache, lens, page_table, row_start):
    """What the C side of a cache call cannot see: devices, types and sizes of the tensors.  Returns the cache's device, whose current
    stream the call goes to, whichever device is current."""
    dev, i32, B = cache.get_device(), torch.int32, kv.n_seqs              # (-1: not on a GPU; a device object takes four times as long)
    if (lens.dtype is not i32 or page_table.dtype is not i32 or lens.get_device() != dev or page_table.get_device() != dev
            or not lens.is_contiguous() or not page_table.is_contiguous()):
        raise PQError("lens, page_table and row_start are contiguous int32 tensors on the cache's device")
    if lens.numel() < B or page_table.numel() < B * kv.max_pages:
        raise PQError("lens, page_table or row_start is smaller than the descriptor says")
    if B > 1 and page_table.dim() > 1 and page_table.shape[-1] != kv.max_pages:   # (its rows would be read one behind the other)
        raise PQError(f"rows of {page_table.shape[-1]} pages in page_table, {kv.max_pages} in the descriptor")
    if row_start is not None:
        if row_start.dtype is not i32 or row_start.get_device() != dev or not row_start.is_contiguous():
            raise PQError("lens, page_table and row_start are contiguous int32 tensors on the cache's device")
        if row_start.numel() < B + 1:
            raise PQError("lens, page_table or row_start is smaller than the descriptor says")
    if dev < 0 or cache.dtype is not torch.uint8 or not cache.is_contiguous():
        raise PQError("the cache is a contiguous uint8 tensor on a GPU")
    return dev


def _rows(t, heads, d):
    """Rows of a [T][heads][d] tensor whose rows are contiguous, and their stride."""
    s = t.shape
    if len(s) != 3:
        raise PQError(f"a tensor of shape {tuple(s)}: [rows, {heads}, {d}] is wanted")
    T, h, n = s
    if h != heads or n != d:
        raise PQError(f"a tensor of shape {tuple(s)}: [rows, {heads}, {d}] is wanted")
    if t.is_contiguous():
        return T, heads * d
    row, head, one = t.stride()
    if one != 1 or (heads > 1 and head != d):
        raise PQError("the heads of a row must be contiguous")
    return T, row if T > 1 else heads * d


_KV_DT = {torch.float32: PQ_F32, torch.bfloat16: PQ_BF16}


def kv_write(desc, K, V, cache, lens, page_table, row_start=None):
    """K, V [T, n_kv_heads, d_head] (bf16 or fp32, any even row stride) into the cache at the last positions of their sequences."""
    dev, heads, d = _kv_check(desc, cache, lens, page_table, row_start), desc.n_kv_heads, desc.d_head
    (T, ks), (Tv, vs), dt = _rows(K, heads, d), _rows(V, heads, d), _KV_DT.get(K.dtype)
    if K.dtype is not V.dtype or T != Tv or dt is None:
        raise PQError("K and V differ in type or rows, or are neither fp32 nor bf16")
    if K.get_device() != dev or V.get_device() != dev:
        raise PQError("K and V are on the cache's device")
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return kv_write(desc, K, V, cache, lens, page_table, row_start)
    rc = lib().pq_kv_write(C.byref(desc), K.data_ptr(), V.data_ptr(), dt, T, ks, vs, None if row_start is None else row_start.data_ptr(),
                           lens.data_ptr(), page_table.data_ptr(), cache.data_ptr(), cache.numel(), _raw_stream(dev))
    if rc:
        _check(rc)
    return cache


def kv_read(desc, cache, lens, page_table, K, V, row_start=None):
    """The inverse of kv_write, into K and V (either may be None)."""
    dev, heads, d = _kv_check(desc, cache, lens, page_table, row_start), desc.n_kv_heads, desc.d_head
    X = V if K is None else K
    if X is None:
        raise PQError("neither keys nor values are asked for")
    (T, ks), dt = _rows(X, heads, d), _KV_DT.get(X.dtype)
    Tv, vs = (T, ks) if V is None or V is X else _rows(V, heads, d)
    if dt is None or T != Tv or (V is not None and V.dtype is not X.dtype):
        raise PQError("K and V differ in type or rows, or are neither fp32 nor bf16")
    if X.get_device() != dev or (V is not None and V.get_device() != dev):
        raise PQError("K and V are on the cache's device")
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return kv_read(desc, cache, lens, page_table, K, V, row_start)
    rc = lib().pq_kv_read(C.byref(desc), cache.data_ptr(), cache.numel(), None if row_start is None else row_start.data_ptr(), lens.data_ptr(),
                          page_table.data_ptr(), T, None if K is None else K.data_ptr(), None if V is None else V.data_ptr(), dt, ks, vs,
                          _raw_stream(dev))
    if rc:
        _check(rc)
    return K, V


def _attn_rows(desc, Q, O, lse):
    H, d = desc.n_heads, desc.kv.d_head
    T, qs = _rows(Q, H, d)
    if Q.dtype is not torch.bfloat16 or O.dtype is not torch.bfloat16:
        raise PQError("Q and O are bf16")
    if O.numel() != T * H * d or not O.is_contiguous():
        raise PQError("O is contiguous and of Q's size")
    dev = Q.get_device()
    if O.get_device() != dev or (lse is not None and lse.get_device() != dev):
        raise PQError("Q, O and lse are on one device")
    if lse is not None and (lse.dtype is not torch.float32 or lse.numel() != T * H or not lse.is_contiguous()):
        raise PQError("lse is a contiguous fp32 tensor of one value per row and head")
    return T, qs


def attn_decode(desc, Q, cache, lens, page_table, O, ws, lse=None):
    """Q [n_seqs, n_heads, d_head] bf16: the last token of every sequence over its whole cache."""
    kv = desc.kv
    dev, (T, qs) = _kv_check(kv, cache, lens, page_table, None), _attn_rows(desc, Q, O, lse)
    if T != kv.n_seqs:
        raise PQError(f"{T} rows for {kv.n_seqs} sequences")
    if Q.get_device() != dev or ws.get_device() != dev or ws.dtype is not torch.uint8 or not ws.is_contiguous():
        raise PQError("the rows and the workspace, a contiguous uint8 tensor, are on the cache's device")
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return attn_decode(desc, Q, cache, lens, page_table, O, ws, lse)
    rc = lib().pq_attn_decode(C.byref(desc), Q.data_ptr(), qs, cache.data_ptr(), cache.numel(), lens.data_ptr(), page_table.data_ptr(),
                              O.data_ptr(), None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.numel(), _raw_stream(dev))
    if rc:
        _check(rc)
    return O


def attn_prefill(desc, Q, cache, lens, page_table, row_start, O, lse=None):
    """Q [T, n_heads, d_head] bf16: the rows of prompts, sequence by sequence (row_start [n_seqs + 1])."""
    dev, (T, qs) = _kv_check(desc.kv, cache, lens, page_table, row_start), _attn_rows(desc, Q, O, lse)
    if Q.get_device() != dev:
        raise PQError("the rows are on the cache's device")
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return attn_prefill(desc, Q, cache, lens, page_table, row_start, O, lse)
    rc = lib().pq_attn_prefill(C.byref(desc), Q.data_ptr(), qs, T, None if row_start is None else row_start.data_ptr(), cache.data_ptr(),
                               cache.numel(), lens.data_ptr(), page_table.data_ptr(), O.data_ptr(), None if lse is None else lse.data_ptr(),
                               _raw_stream(dev))
    if rc:
        _check(rc)
    return O


def make_rope_desc(n_heads, n_kv_heads, d_head, n_seqs, rot_dim=0, layout=PQ_ROPE_HALF, inverse=False, scale=1.0):
    """rot_dim: elements of a head that turn (0: all of them).  n_kv_heads 0: calls have no keys."""
    return RopeDesc(n_heads, n_kv_heads, d_head, rot_dim or d_head, layout, int(inverse), n_seqs, scale)


def rope_freqs(rot_dim, base=10000.0, factor=1.0, original_len=0, low=1.0, high=32.0, device="cuda"):
    """Turns per position of every pair [rot_dim / 2], fp64: base^(-2 i / rot_dim) / (2 pi).

    factor > 1 stretches them for contexts that many times longer: all of them by the factor (original_len 0), or by parts: of the pairs that turn r
    times within original_len tokens those with r >= high are left as they are, those with r <= low are slowed down by the factor, a ramp between."""
    if rot_dim < 2 or rot_dim % 2 or base <= 0 or factor <= 0 or not low < high:
        raise PQError(f"rope_freqs: rot_dim={rot_dim} is even, base={base} and factor={factor} are positive, low={low} is below high={high}")
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    f = base ** (-2.0 * i / rot_dim) / 6.283185307179586
    keep = ((original_len * f - low) / (high - low)).clamp(0.0, 1.0) if original_len else torch.zeros_like(f)
    return (f * (keep + (1.0 - keep) / factor)).to(device)


def _index_check(dev, what, t, n):
    if t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous():
        raise PQError(f"{what} is a contiguous int32 tensor on the rows' device")
    if t.numel() < n:
        raise PQError(f"{what}: {t.numel()} entries where the descriptor asks for {n}")


def rope(desc, Q, K, freqs, Qr, Kr, row_start=None, lens=None):
    """Q [T, n_heads, d_head] and K [T, n_kv_heads, d_head] (or None) turned into Qr and Kr, which may be Q and K themselves."""
    d, B, Hk, dtype, dev = desc.d_head, desc.n_seqs, desc.n_kv_heads, Q.dtype, Q.get_device()
    dt = _KV_DT.get(dtype)
    T, qs = _rows(Q, desc.n_heads, d)
    Tr, qrs = _rows(Qr, desc.n_heads, d)
    if dev < 0 or dt is None or Qr.dtype is not dtype or T != Tr or Qr.get_device() != dev:
        raise PQError("Q and Qr are fp32 or bf16 tensors of as many rows on one GPU")
    k = kr = None
    ks = krs = 0
    if Hk:
        if K is None or Kr is None:
            raise PQError("the descriptor has key heads: K and Kr are wanted")
        Tk, ks = _rows(K, Hk, d)
        Tkr, krs = _rows(Kr, Hk, d)
        if Tk != T or Tkr != T or K.dtype is not dtype or Kr.dtype is not dtype or K.get_device() != dev or Kr.get_device() != dev:
            raise PQError("K and Kr have Q's rows, type and device")
        k, kr = K.data_ptr(), Kr.data_ptr()
    elif K is not None or Kr is not None:
        raise PQError("the descriptor has no key heads")
    if freqs.dtype is not torch.float64 or freqs.get_device() != dev or not freqs.is_contiguous() or freqs.numel() != desc.rot_dim // 2:
        raise PQError(f"freqs is a contiguous fp64 tensor of rot_dim / 2 = {desc.rot_dim // 2} values on Q's device")
    rs = ln = None
    if row_start is not None:
        _index_check(dev, "row_start", row_start, B + 1)
        rs = row_start.data_ptr()
    if lens is not None:
        _index_check(dev, "lens", lens, B)
        ln = lens.data_ptr()
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return rope(desc, Q, K, freqs, Qr, Kr, row_start, lens)
    rc = lib().pq_rope(C.byref(desc), Q.data_ptr(), qs, k, ks, dt, T, freqs.data_ptr(), rs, ln, Qr.data_ptr(), qrs, kr, krs, _raw_stream(dev))
    if rc:
        _check(rc)
    return Qr, Kr


def make_self_attn_desc(n_heads, n_kv_heads, d_head, n_seqs, scale=None, causal=True, window=0):
    """scale: 1 / sqrt(d_head) unless given."""
    return SelfAttnDesc(n_heads, n_kv_heads, d_head, n_seqs, int(causal), window, d_head ** -0.5 if scale is None else scale)


def self_attn_bwd_workspace(desc, T, device="cuda"):
    n = lib().pq_self_attn_bwd_workspace_bytes(C.byref(desc), T)
    if n == 0:
        raise PQError(f"bad attention descriptor: {lib().pq_last_error_string().decode()}")
    return _bytes(n, device)


def _self_attn_check(desc, Q, K, V, row_start, O, lse):
    """What the C side of a call cannot see.  Returns the rows, the strides of Q, K and V, and the device."""
    H, Hk, d, bf, dev = desc.n_heads, desc.n_kv_heads, desc.d_head, torch.bfloat16, Q.get_device()
    (T, qs), (Tk, ks), (Tv, vs) = _rows(Q, H, d), _rows(K, Hk, d), _rows(V, Hk, d)
    if Tk != T or Tv != T or Q.dtype is not bf or K.dtype is not bf or V.dtype is not bf:
        raise PQError("Q, K and V are bf16 and have as many rows")
    if O.dtype is not bf or O.numel() != T * H * d or not O.is_contiguous():
        raise PQError("O and dO are contiguous bf16 tensors of Q's size")
    if lse.dtype is not torch.float32 or lse.numel() != T * H or not lse.is_contiguous():
        raise PQError("lse is a contiguous fp32 tensor of one value per row and head")
    if dev < 0 or K.get_device() != dev or V.get_device() != dev or O.get_device() != dev or lse.get_device() != dev:
        raise PQError("Q, K, V, O and lse are on one GPU")
    _index_check(dev, "row_start", row_start, desc.n_seqs + 1)
    return T, qs, ks, vs, dev


def self_attn_fwd(desc, Q, K, V, row_start, O, lse):
    """Q [T, n_heads, d_head], K, V [T, n_kv_heads, d_head] bf16, sequences packed row by row (row_start [n_seqs + 1] int32)."""
    T, qs, ks, vs, dev = _self_attn_check(desc, Q, K, V, row_start, O, lse)
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return self_attn_fwd(desc, Q, K, V, row_start, O, lse)
    rc = lib().pq_self_attn_fwd(C.byref(desc), Q.data_ptr(), qs, K.data_ptr(), ks, V.data_ptr(), vs, T, row_start.data_ptr(), O.data_ptr(),
                                lse.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)
    return O, lse


def self_attn_bwd(desc, dO, Q, K, V, O, lse, row_start, dQ, dK, dV, ws):
    """The gradients of self_attn_fwd's inputs, from what it was given and left."""
    T, qs, ks, vs, dev = _self_attn_check(desc, Q, K, V, row_start, O, lse)
    H, Hk, d, bf = desc.n_heads, desc.n_kv_heads, desc.d_head, torch.bfloat16
    (Tq, dqs), (Tk, dks), (Tv, dvs) = _rows(dQ, H, d), _rows(dK, Hk, d), _rows(dV, Hk, d)
    if Tq != T or Tk != T or Tv != T or dQ.dtype is not bf or dK.dtype is not bf or dV.dtype is not bf:
        raise PQError("dQ, dK and dV are bf16 and have Q's rows")
    if dO.dtype is not bf or dO.numel() != T * H * d or not dO.is_contiguous():
        raise PQError("O and dO are contiguous bf16 tensors of Q's size")
    if (dO.get_device() != dev or dQ.get_device() != dev or dK.get_device() != dev or dV.get_device() != dev or ws.get_device() != dev
            or ws.dtype is not torch.uint8 or not ws.is_contiguous()):
        raise PQError("the gradients and the workspace, a contiguous uint8 tensor, are on Q's device")
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return self_attn_bwd(desc, dO, Q, K, V, O, lse, row_start, dQ, dK, dV, ws)
    rc = lib().pq_self_attn_bwd(C.byref(desc), dO.data_ptr(), Q.data_ptr(), qs, K.data_ptr(), ks, V.data_ptr(), vs, O.data_ptr(), lse.data_ptr(), T,
                                row_start.data_ptr(), dQ.data_ptr(), dqs, dK.data_ptr(), dks, dV.data_ptr(), dvs, ws.data_ptr(), ws.numel(),
                                _raw_stream(dev))
    if rc:
        _check(rc)
    return dQ, dK, dV


class AdamWTensors:
    """The tensors of an AdamW step and their states, laid out once for adamw_step and adamw_read.

    params: contiguous tensors of one type, fp32 or bf16, on one GPU; grads: of the same sizes, fp32 or bf16, read anew by every step; masters: fp32, of bf16
    params, or None.  States m and v that are not given are made here and begin at zero, of `state` (PQ_STATE_F32 or PQ_STATE_8BIT: int8 m, uint8 v and
    steps [ceil(n / 256), 2] fp32); those that are given say by their type which it is.  m_values, v_values: fp32, where adamw_read writes 8-bit
    states as the values they stand for, or None.  The tensors must stay where they are: gradients too, which are written into the same memory by every
    backward.  (Laying out fifty tensors anew takes 190 us, seventy 260, many times a small step.)"""

    def __init__(self, params, grads, m=None, v=None, steps=None, masters=None, m_values=None, v_values=None, beta1=0.9, beta2=0.999, eps=1e-8,
                 state=PQ_STATE_F32):
        params, grads = list(params), list(grads)
        if not params:
            raise PQError("an optimizer step without tensors")
        dev = params[0].get_device()
        if (m is None) != (v is None):
            raise PQError("m and v are given together")
        if m is not None:
            m, v = list(m), list(v)
            state = PQ_STATE_8BIT if m and m[0].dtype is torch.int8 else PQ_STATE_F32
        if state not in (PQ_STATE_F32, PQ_STATE_8BIT):
            raise PQError(f"unknown state {state}")
        eight = state == PQ_STATE_8BIT
        zeros = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=params[0].device)
        if m is None:
            m = [zeros(p.shape, torch.int8 if eight else torch.float32) for p in params]
            v = [zeros(p.shape, torch.uint8 if eight else torch.float32) for p in params]
        if eight and steps is None:
            if any(bool(x.any()) for x in m + v):
                raise PQError("8-bit states that are not zero have steps")
            steps = [zeros((-(-p.numel() // 256), 2), torch.float32) for p in params]
        if not eight and steps is not None:
            raise PQError("steps belong to 8-bit states")
        f32 = torch.float32
        kinds = [("params", params, params[0].dtype), ("grads", grads, grads[0].dtype if grads else f32), ("masters", masters, f32),
                 ("m", m, torch.int8 if eight else f32), ("v", v, torch.uint8 if eight else f32), ("steps", steps, f32),
                 ("m_values", m_values, f32), ("v_values", v_values, f32)]
        written = []
        for name, ts, dtype in kinds:
            if ts is None:
                continue
            if len(ts) != len(params):
                raise PQError(f"{len(ts)} {name} for {len(params)} params")
            for t, p in zip(ts, params):
                n = -(-p.numel() // 256) * 2 if name == "steps" else p.numel()
                if t.dtype is not dtype or t.get_device() != dev or dev < 0 or not t.is_contiguous() or t.numel() != n:
                    raise PQError(f"{name}: contiguous {dtype} tensors of their params' sizes on one GPU are wanted"
                                  + (" (steps: [ceil(n / 256), 2])" if name == "steps" else ""))
                if n:
                    written.append((t.data_ptr(), t.data_ptr() + n * t.element_size(), name))
        written.sort()                                                  # (gradients are only read and may share memory among themselves)
        reach = {True: (0, ""), False: (0, "")}
        for begin, end, name in written:
            for read_only, (to, other) in reach.items():
                if begin < to and not (read_only and name == "grads"):
                    raise PQError(f"{other} and {name} overlap")
            reach[name == "grads"] = max(reach[name == "grads"], (end, name))
        self.desc = AdamWDesc(len(params), _dt(params[0]), _dt(grads[0]), state, int(masters is not None), int(m_values is not None), beta1, beta2, eps)
        lists = [params, grads, masters, m, v, steps, m_values, v_values]
        self.params, self.grads, self.masters, self.m, self.v, self.steps, self.m_values, self.v_values = lists
        arr = (AdamWTensor * len(params))(*[AdamWTensor(*[ts[i].data_ptr() if ts is not None else None for ts in lists], params[i].numel())
                                            for i in range(len(params))])
        n = lib().pq_adamw_plan_bytes(C.byref(self.desc), arr)
        if n == 0:
            raise PQError(f"bad optimizer tensors: {lib().pq_last_error_string().decode()}")
        host = torch.empty(n, dtype=torch.uint8)
        _check(lib().pq_adamw_plan(C.byref(self.desc), arr, host.data_ptr(), n))
        self.plan, self.device, self._bytes = host.to(params[0].device), dev, n


def adamw_scalars(tensors, step, lr, weight_decay=0.0, grad_scale=1.0, out=None):
    """What changes from step to step (counted from 1), as the device tensor that adamw_step reads; `out`: into that tensor, for steps that are captured.
    Formed on the host and copied by a transfer that the host waits for, on the current stream behind all that is there: about 16 us of every step that
    takes new ones, and no run-ahead of the host across it."""
    if step < 1 or lr < 0.0 or weight_decay < 0.0:
        raise PQError(f"step={step} counts from 1, lr={lr} and weight_decay={weight_decay} are not negative")
    d = tensors.desc
    x = torch.tensor([1.0 - lr * weight_decay, lr / (1.0 - d.beta1 ** step), (1.0 - d.beta2 ** step) ** -0.5, grad_scale], dtype=torch.float64).float()
    if out is None:
        return x.to(tensors.plan.device)
    if out.dtype is not torch.float32 or out.numel() != 4 or not out.is_contiguous() or out.get_device() != tensors.device:
        raise PQError("scalars are a contiguous fp32 tensor of four values on the tensors' device")
    return out.copy_(x)


def adamw_step(tensors, scalars):
    """One step of all tensors, with the gradients as they are now."""
    dev = tensors.device
    if scalars.dtype is not torch.float32 or scalars.numel() != 4 or not scalars.is_contiguous() or scalars.get_device() != dev:
        raise PQError("scalars are a contiguous fp32 tensor of four values on the tensors' device")
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return adamw_step(tensors, scalars)
    rc = lib().pq_adamw_step(C.byref(tensors.desc), tensors.plan.data_ptr(), tensors._bytes, scalars.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)


def adamw_read(tensors):
    """8-bit states as the values they stand for, into m_values and v_values."""
    dev = tensors.device
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return adamw_read(tensors)
    rc = lib().pq_adamw_read(C.byref(tensors.desc), tensors.plan.data_ptr(), tensors._bytes, _raw_stream(dev))
    if rc:
        _check(rc)
    return tensors.m_values, tensors.v_values


def glue_lincomb(out, xs, cs):
    xs = list(xs) + [None] * (4 - len(xs))
    cs = list(cs) + [0.0] * (4 - len(cs))
    _check(lib().pq_glue_lincomb(_p(out), _p(xs[0]), _p(xs[1]), _p(xs[2]), _p(xs[3]), C.c_float(cs[0]), C.c_float(cs[1]),
                                 C.c_float(cs[2]), C.c_float(cs[3]), C.c_size_t(out.numel()), _stream()))
    return out


def glue_gather_rows(table, ids, out):
    _check(lib().pq_glue_gather_rows(_p(table), _p(ids), ids.numel(), table.shape[1], _p(out), _stream()))
    return out
