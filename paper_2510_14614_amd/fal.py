"""Thin ctypes binding of libfal.so (the C ABI in include/fal.h).

Everything here is argument marshalling: flattening parameter dicts into the
library's layout, device buffers owned by PyTorch, and status checking.  All
computation of the training step happens in the library's HIP kernels.  If
libfal.so is missing the import of :func:`lib` raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_void_p
from typing import NamedTuple

import numpy as np

from .config import Config
from .synth import BLOCK_NAMES, GLOBAL_NAMES

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfal.so")

FAL_OK, FAL_ERR_INVALID_ARG, FAL_ERR_UNSUPPORTED, FAL_ERR_WORKSPACE, FAL_ERR_HIP, FAL_ERR_STATE = range(6)

# Order of the FAL_P_* and FAL_B_* enums in include/fal.h.
GLOBAL_TENSORS = GLOBAL_NAMES
BLOCK_TENSORS = BLOCK_NAMES

ABI_FUNCTIONS = (
    "fal_validate_config", "fal_param_layout", "fal_workspace_bytes", "fal_init", "fal_destroy",
    "fal_block_fwd", "fal_block_bwd", "fal_model_step", "fal_stack_step", "fal_residual_out",
    "fal_profile_enable", "fal_profile_read", "fal_status_string", "fal_last_error", "fal_adamw_step",
    "fal_model_forward", "fal_stack_forward", "fal_adamw_step_noalloc",
    "fal_window_attention_workspace_bytes", "fal_window_attention_fwd", "fal_window_attention_bwd",
    "fal_set_attention_window", "fal_token_logprobs", "fal_logit_loss_workspace_bytes", "fal_policy_loss",
    "fal_preference_loss", "fal_model_logprobs", "fal_policy_step", "fal_preference_step",
)
PROF_GEMM, PROF_ATTN_FWD, PROF_ATTN_BWD, PROF_NORM, PROF_CE, PROF_EMBED, PROF_BIAS, PROF_OPTIM = range(8)
PROF_NAMES = {PROF_GEMM: "gemm", PROF_ATTN_FWD: "attn_fwd", PROF_ATTN_BWD: "attn_bwd", PROF_NORM: "norm",
              PROF_CE: "cross_entropy", PROF_EMBED: "embedding", PROF_BIAS: "bias_grad", PROF_OPTIM: "optimizer"}

# AdamW settings of the paper's training setups (appendix: lr 1e-4, weight
# decay 0.001, clip-grad-norm 1) with the usual beta and eps defaults.
ADAMW_PAPER = {"lr": 1e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 1e-3,
               "max_grad_norm": 1.0}


class fal_config_t(ctypes.Structure):
    _fields_ = [
        ("n_layer", c_int32), ("d_model", c_int32), ("n_head", c_int32), ("head_dim", c_int32),
        ("d_ff", c_int32), ("vocab", c_int32), ("seq_len", c_int32), ("batch", c_int32),
        ("arch", c_int32), ("dtype", c_int32), ("sched", c_int32), ("ln_eps", c_float),
        ("gelu_tanh", c_int32), ("has_embed_head", c_int32), ("fal_block1_mode", c_int32),
        ("bidirectional", c_int32), ("n_kv_head", c_int32),
    ]


class fal_adamw_t(ctypes.Structure):
    _fields_ = [("lr", c_float), ("beta1", c_float), ("beta2", c_float), ("eps", c_float),
                ("weight_decay", c_float), ("max_grad_norm", c_float)]


def adamw_params(**hp) -> fal_adamw_t:
    v = dict(ADAMW_PAPER)
    v.update(hp)
    return fal_adamw_t(**{k: float(v[k]) for k in ADAMW_PAPER})


class fal_window_attention_t(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("seq_len", c_int32), ("n_head", c_int32), ("n_kv_head", c_int32),
                ("head_dim", c_int32), ("dtype", c_int32), ("window", c_int32), ("sinks", c_int32),
                ("ld_qkv", c_int64), ("ld_out", c_int64)]


class fal_logit_rows_t(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("seq_len", c_int32), ("vocab", c_int32), ("dtype", c_int32),
                ("ld_logits", c_int64), ("ld_targets", c_int64), ("ld_dlogits", c_int64), ("dlogits_cols", c_int32),
                ("temperature", c_float)]


class fal_policy_t(ctypes.Structure):
    _fields_ = [("clip_low", c_float), ("clip_high", c_float), ("kl_coef", c_float), ("sequence_mean", c_int32)]


class fal_preference_t(ctypes.Structure):
    _fields_ = [("beta", c_float), ("label_smoothing", c_float), ("ipo", c_int32), ("length_mean", c_int32)]


class PolicyLoss(NamedTuple):
    stats: object    # fp32 [4]: loss, its policy part, KL mean, share of rows whose ratio the clip holds
    logp: object     # fp32 [B, T]
    dlogits: object  # gradient of the loss, in the logits' dtype


class PreferenceLoss(NamedTuple):
    loss: object      # fp32 [1]
    seq_logp: object  # fp32 [B]
    dlogits: object


class FalError(RuntimeError):
    def __init__(self, status, msg=""):
        self.status = status
        super().__init__(f"libfal status {status}: {msg}")


_LIB = None


def lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise FalError(-1, f"{LIB_PATH} is not built (python -m paper_2510_14614_amd.build)")
        L = ctypes.CDLL(LIB_PATH)
        cfgp = POINTER(fal_config_t)
        L.fal_validate_config.argtypes = [cfgp]
        L.fal_param_layout.argtypes = [cfgp, POINTER(c_int64), POINTER(c_int64), POINTER(c_int64),
                                       POINTER(c_int64), POINTER(c_int64)]
        L.fal_workspace_bytes.argtypes = [cfgp, POINTER(c_size_t)]
        L.fal_init.argtypes = [cfgp, c_void_p, c_size_t, c_void_p, c_void_p, POINTER(c_void_p)]
        L.fal_destroy.argtypes = [c_void_p]
        L.fal_block_fwd.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]
        L.fal_block_bwd.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_void_p, c_void_p, c_void_p]
        L.fal_model_step.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        L.fal_stack_step.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        L.fal_model_forward.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        L.fal_stack_forward.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p]
        L.fal_residual_out.argtypes = [c_void_p, POINTER(c_void_p)]
        L.fal_profile_enable.argtypes = [c_void_p, c_int32]
        L.fal_profile_read.argtypes = [c_void_p, c_int32, POINTER(c_int64), POINTER(c_double),
                                       POINTER(c_double), POINTER(c_double)]
        L.fal_adamw_step.argtypes = [c_void_p, POINTER(fal_adamw_t), c_int64, c_int64, c_void_p, c_void_p,
                                     c_void_p, c_void_p, c_void_p, c_void_p]
        L.fal_adamw_step_noalloc.argtypes = [POINTER(fal_adamw_t), c_int64, c_int64, c_int32, c_void_p, c_void_p,
                                             c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        attnp, rowsp = POINTER(fal_window_attention_t), POINTER(fal_logit_rows_t)
        L.fal_window_attention_workspace_bytes.argtypes = [attnp, POINTER(c_size_t)]
        L.fal_window_attention_fwd.argtypes = [attnp] + [c_void_p] * 5
        L.fal_window_attention_bwd.argtypes = ([attnp] + [c_void_p] * 6 + [c_int64, c_void_p, c_size_t, c_void_p])
        L.fal_set_attention_window.argtypes = [c_void_p, c_int32, c_int32]
        L.fal_token_logprobs.argtypes = [rowsp] + [c_void_p] * 6
        L.fal_logit_loss_workspace_bytes.argtypes = [rowsp, POINTER(c_size_t)]
        L.fal_policy_loss.argtypes = [rowsp, POINTER(fal_policy_t)] + [c_void_p] * 10 + [c_size_t, c_void_p]
        L.fal_preference_loss.argtypes = [rowsp, POINTER(fal_preference_t)] + [c_void_p] * 8 + [c_size_t, c_void_p]
        L.fal_model_logprobs.argtypes = [c_void_p] * 4 + [c_float] + [c_void_p] * 2
        L.fal_policy_step.argtypes = ([c_void_p] * 2 + [POINTER(fal_policy_t)] + [c_void_p] * 2 + [c_float] +
                                      [c_void_p] * 6)
        L.fal_preference_step.argtypes = ([c_void_p] * 2 + [POINTER(fal_preference_t)] + [c_void_p] * 2 + [c_float] +
                                          [c_void_p] * 4)
        L.fal_status_string.argtypes = [c_int32]
        L.fal_status_string.restype = c_char_p
        L.fal_last_error.argtypes = [c_void_p]
        L.fal_last_error.restype = c_char_p
        for name in ABI_FUNCTIONS:
            if name not in ("fal_status_string", "fal_last_error"):
                getattr(L, name).restype = c_int32
        _LIB = L
    return _LIB


def to_c(cfg: Config) -> fal_config_t:
    return fal_config_t(cfg.n_layer, cfg.d_model, cfg.n_head, cfg.head_dim, cfg.d_ff, cfg.vocab,
                        cfg.seq_len, cfg.batch, cfg.arch, cfg.dtype, cfg.sched, cfg.ln_eps,
                        cfg.gelu_tanh, cfg.has_embed_head, cfg.fal_block1_mode, cfg.bidirectional,
                        cfg.n_kv_head)


def _check(status, ctx=None):
    if status != FAL_OK:
        L = lib()
        msg = L.fal_last_error(ctx).decode() if ctx else ""
        name = L.fal_status_string(status).decode()
        raise FalError(status, f"{name}: {msg}")


def validate_config(cfg: Config) -> int:
    c = to_c(cfg)
    return lib().fal_validate_config(byref(c))


def param_layout(cfg: Config) -> dict:
    c = to_c(cfg)
    g = (c_int64 * 4)()
    b = (c_int64 * 14)()
    base, stride, total = c_int64(), c_int64(), c_int64()
    _check(lib().fal_param_layout(byref(c), g, b, byref(base), byref(stride), byref(total)))
    return {"global": list(g), "block": list(b), "block_base": base.value,
            "block_stride": stride.value, "total": total.value}


def workspace_bytes(cfg: Config) -> int:
    c = to_c(cfg)
    n = c_size_t()
    _check(lib().fal_workspace_bytes(byref(c), byref(n)))
    return n.value


def flatten_params(cfg: Config, gparams: dict, blocks: list, layout: dict | None = None) -> np.ndarray:
    """Host float32 flat buffer in the library's parameter layout."""
    lay = layout or param_layout(cfg)
    flat = np.zeros(lay["total"], dtype=np.float32)
    if cfg.has_embed_head:
        for k, name in enumerate(GLOBAL_TENSORS):
            a = np.asarray(gparams[name], dtype=np.float32).reshape(-1)
            flat[lay["global"][k]:lay["global"][k] + a.size] = a
    for i, blk in enumerate(blocks):
        base = lay["block_base"] + i * lay["block_stride"]
        for k, name in enumerate(BLOCK_TENSORS):
            a = np.asarray(blk[name], dtype=np.float32).reshape(-1)
            o = base + lay["block"][k]
            flat[o:o + a.size] = a
    return flat


def unflatten(cfg: Config, flat: np.ndarray, gshapes: dict, bshapes: dict, layout: dict | None = None):
    """Inverse of flatten_params for a host float32 buffer (gradients)."""
    lay = layout or param_layout(cfg)
    g = {}
    if cfg.has_embed_head:
        for k, name in enumerate(GLOBAL_TENSORS):
            n = int(np.prod(gshapes[name]))
            g[name] = flat[lay["global"][k]:lay["global"][k] + n].reshape(gshapes[name]).copy()
    blocks = []
    for i in range(cfg.n_layer):
        base = lay["block_base"] + i * lay["block_stride"]
        d = {}
        for k, name in enumerate(BLOCK_TENSORS):
            n = int(np.prod(bshapes[name]))
            o = base + lay["block"][k]
            d[name] = flat[o:o + n].reshape(bshapes[name]).copy()
        blocks.append(d)
    return g, blocks


def adamw_step_noalloc(hp: fal_adamw_t, step: int, n: int, dtype: int, master, params, grads, m, v,
                       grad_norm=None, stream=None):
    """fal_adamw_step_noalloc on torch device tensors (no context, no
    allocation): one AdamW update of n elements on `stream` (a torch stream;
    None: the current stream)."""
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    ptr = lambda t: c_void_p(t.data_ptr()) if t is not None else None  # noqa: E731
    st = lib().fal_adamw_step_noalloc(byref(hp), step, n, dtype, ptr(master), ptr(params), ptr(grads), ptr(m), ptr(v),
                                      ptr(grad_norm), c_void_p(s.cuda_stream))
    if st != FAL_OK:
        L = lib()
        raise FalError(st, f"{L.fal_status_string(st).decode()}: {L.fal_last_error(None).decode()}")


# ------------------------------------------- operators without a context --
# Each takes torch device tensors, runs on the current stream of their device
# and returns without waiting.  Outputs that are not given are allocated, as is
# the workspace, so calls on different streams or in different captured graphs
# share nothing.  ValueError: a tensor is not what the call needs; FalError:
# the library refused the call.
# A small call's time is the host's, so the checks read each attribute once and
# format messages only to raise them.
def _refuse(what):
    raise ValueError(what)


def _dtype_code(t, name):
    import torch
    if t.dtype is torch.bfloat16:
        return 1
    if t.dtype is not torch.float32:
        _refuse(f"{name} must be bfloat16 or float32")
    return 0


def _dense(t, name, shape, dtypes, device):
    """Checks a contiguous tensor of the given shape on a device."""
    if t.dtype not in dtypes:
        _refuse(f"{name} must be {' or '.join(str(d) for d in dtypes)}")
    if t.shape != shape:
        _refuse(f"{name} must have shape {shape}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        _refuse(f"{name} must be contiguous")
    if t.device != device:
        _refuse(f"{name} must be on {device}")


def _row_stride(t, name):
    """Row stride of a [B, T, width] tensor whose rows are equally spaced."""
    B, T, width = t.shape
    sb, st, sw = t.stride()
    if width > 1 and sw != 1:
        _refuse(f"{name} must be contiguous in its last dimension")
    ld = st if T > 1 else sb if B > 1 else width
    if B > 1 and sb != T * ld:
        _refuse(f"the sequences of {name} must follow each other at seq_len rows")
    return ld


def _ptr(t):
    return None if t is None else t.data_ptr()


class _call:
    """The device guard and the stream of one library call."""
    __slots__ = ("device", "guard")

    def __init__(self, device):
        import torch
        if device.type != "cuda":
            _refuse("tensors must be on a GPU")
        self.device = device
        self.guard = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        import torch
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _check_noctx(status):
    if status != FAL_OK:
        L = lib()
        raise FalError(status, f"{L.fal_status_string(status).decode()}: {L.fal_last_error(None).decode()}")


@functools.lru_cache(maxsize=1024)
def _window_workspace(*shape):
    n = c_size_t()
    _check_noctx(lib().fal_window_attention_workspace_bytes(byref(fal_window_attention_t(*shape)), byref(n)))
    return n.value


@functools.lru_cache(maxsize=1024)
def _loss_workspace(B, T):
    n = c_size_t()
    r = fal_logit_rows_t(B, T, 1, 0, 1, T, 1, 1, 1.0)
    _check_noctx(lib().fal_logit_loss_workspace_bytes(byref(r), byref(n)))
    return n.value


def _clamp32(n):
    # past 32 bits every window is the whole sequence, and every number of
    # sinks and size of an array too many
    return n if -1 <= n <= 2147483647 else max(-1, min(n, 2147483647))


def _window_shape(qkv, n_head, n_kv_head, window, sinks, lens):
    """The call's shape, with dense rows of out."""
    import torch
    if qkv.dim() != 3:
        _refuse("qkv must be [B, T, (n_head + 2 n_kv_head) * head_dim]")
    B, T, width = qkv.shape
    heads = n_head + 2 * (n_kv_head or n_head)
    if n_head < 1 or n_kv_head < 0 or width % heads:
        _refuse("qkv's last dimension must be (n_head + 2 n_kv_head) * head_dim")
    hd = width // heads
    code = _dtype_code(qkv, "qkv")
    if lens is not None:
        _dense(lens, "lens", (B,), (torch.int32,), qkv.device)
    return (B, T, n_head, n_kv_head, hd, code, _clamp32(window), _clamp32(sinks), _row_stride(qkv, "qkv"),
            n_head * hd)


def _window_rows(t, name, like, shape):
    if t.dtype is not like.dtype or t.device != like.device:
        _refuse(f"{name} must have qkv's dtype and device")
    if t.shape != shape:
        _refuse(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    return _row_stride(t, name)


def window_attention_fwd(qkv, n_head, window, sinks=0, n_kv_head=0, lens=None, out=None, lse=None):
    """Causal attention over a sliding window: query t sees the keys j <= t
    with t - j < window or j < sinks (fal_window_attention_fwd).

    qkv: [B, T, (n_head + 2 n_kv_head) * head_dim], bfloat16 or float32, rows
    [Q | K | V] at any equal spacing; lens: int32 [B] or None.  Returns out
    [B, T, n_head * head_dim] (rows at any equal spacing if given) and the
    log-sum-exp, float32 [B, n_head, T]."""
    import torch
    shape = _window_shape(qkv, n_head, n_kv_head, window, sinks, lens)
    B, T = shape[:2]
    device = qkv.device
    a = fal_window_attention_t(*shape)
    with _call(device) as stream:
        if out is None:
            out = torch.empty((B, T, shape[9]), dtype=qkv.dtype, device=device)
        else:
            a.ld_out = _window_rows(out, "out", qkv, (B, T, shape[9]))
        if lse is None:
            lse = torch.empty((B, n_head, T), dtype=torch.float32, device=device)
        else:
            _dense(lse, "lse", (B, n_head, T), (torch.float32,), device)
        _check_noctx(lib().fal_window_attention_fwd(byref(a), qkv.data_ptr(), _ptr(lens), out.data_ptr(),
                                                    lse.data_ptr(), stream))
    return out, lse


def window_attention_bwd(qkv, out, dout, lse, n_head, window, sinks=0, n_kv_head=0, lens=None, dqkv=None):
    """Gradient of window_attention_fwd with respect to qkv, from the out and
    lse it returned and the gradient of out (rows spaced as out's).  dqkv, if
    given, has rows at any equal spacing; returned."""
    import torch
    shape = _window_shape(qkv, n_head, n_kv_head, window, sinks, lens)
    B, T = shape[:2]
    device = qkv.device
    a = fal_window_attention_t(*shape)
    a.ld_out = ld = _window_rows(out, "out", qkv, (B, T, shape[9]))
    if _window_rows(dout, "dout", qkv, (B, T, shape[9])) != ld:
        _refuse(f"dout must have out's row stride of {ld} elements")
    _dense(lse, "lse", (B, n_head, T), (torch.float32,), device)
    with _call(device) as stream:
        if dqkv is None:
            dqkv = torch.empty(qkv.shape, dtype=qkv.dtype, device=device)
        ld = _window_rows(dqkv, "dqkv", qkv, qkv.shape)
        n = _window_workspace(*shape)
        # allocations of the caching allocator start at multiples of 512 bytes
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        _check_noctx(lib().fal_window_attention_bwd(byref(a), qkv.data_ptr(), _ptr(lens), out.data_ptr(),
                                                    dout.data_ptr(), lse.data_ptr(), dqkv.data_ptr(), ld,
                                                    ws.data_ptr(), n, stream))
    return dqkv


def _logit_rows(logits, targets, mask, vocab, temperature):
    import torch
    if logits.dim() != 3:
        _refuse("logits must be [B, T, vocab]")
    B, T, width = logits.shape
    V = width if vocab is None else vocab
    if not 1 <= V <= width:
        _refuse("vocab must lie in [1, logits' last dimension]")
    code = _dtype_code(logits, "logits")
    if targets.dtype is not torch.int32 or targets.shape != (B, T) or targets.device != logits.device:
        _refuse("targets must be int32 [B, T] on the logits' device")
    sb, st = targets.stride()
    if T > 1 and st != 1:
        _refuse("targets must be contiguous in their last dimension")
    if mask is not None:
        _dense(mask, "mask", (B, T), (torch.bool, torch.uint8), logits.device)
    ld = _row_stride(logits, "logits")
    return fal_logit_rows_t(_clamp32(B), _clamp32(T), _clamp32(V), code, ld, sb if B > 1 else T, ld, _clamp32(width),
                            temperature)


def token_logprobs(logits, targets, mask=None, vocab=None, temperature=1.0, entropy=False):
    """Log-probability of targets (int32 [B, T]) under softmax(logits /
    temperature), float32 [B, T], zero where mask (bool or uint8 [B, T]) is
    zero; with entropy=True also the entropy of each row's softmax
    (fal_token_logprobs).  logits: [B, T, >= vocab], bfloat16 or float32."""
    import torch
    r = _logit_rows(logits, targets, mask, vocab, temperature)
    with _call(logits.device) as stream:
        logp = torch.empty(targets.shape, dtype=torch.float32, device=logits.device)
        ent = torch.empty_like(logp) if entropy else None
        _check_noctx(lib().fal_token_logprobs(byref(r), logits.data_ptr(), targets.data_ptr(), _ptr(mask),
                                              logp.data_ptr(), _ptr(ent), stream))
    return (logp, ent) if entropy else logp


def _gradient_rows(r, logits, dlogits):
    """The gradient's buffer: as wide as the logits and spaced as they are."""
    import torch
    if r.dlogits_cols > 1 << 30:
        _refuse("logits of a gradient must have at most 2^30 columns")
    if dlogits is None:
        ld = r.ld_logits if r.ld_logits < r.dlogits_cols + 64 else r.dlogits_cols
        dlogits = torch.empty((r.batch, r.seq_len, ld), dtype=logits.dtype, device=logits.device)
        dlogits = dlogits[:, :, :r.dlogits_cols]
    elif dlogits.dtype is not logits.dtype or dlogits.device != logits.device or dlogits.shape != logits.shape:
        _refuse("dlogits must have the logits' shape, dtype and device")
    r.ld_dlogits = _row_stride(dlogits, "dlogits")
    return dlogits


def policy_loss(logits, targets, old_logp, advantages, ref_logp=None, mask=None, vocab=None, dlogits=None, *,
                clip_low=0.2, clip_high=0.2, kl_coef=0.0, sequence_mean=False, temperature=1.0):
    """Clipped policy loss with a KL term, and its gradient with respect to
    the logits (fal_policy_loss): old_logp, advantages and ref_logp are float32
    [B, T].  The gradient has the logits' shape, zero in the columns past vocab
    and in rows that do not count; dlogits may be the logits themselves."""
    import torch
    r = _logit_rows(logits, targets, mask, vocab, temperature)
    shape, device, f32 = targets.shape, logits.device, (torch.float32,)
    _dense(old_logp, "old_logp", shape, f32, device)
    _dense(advantages, "advantages", shape, f32, device)
    if ref_logp is not None:
        _dense(ref_logp, "ref_logp", shape, f32, device)
    hp = fal_policy_t(clip_low, clip_high, kl_coef, int(sequence_mean))
    with _call(device) as stream:
        dlogits = _gradient_rows(r, logits, dlogits)
        stats = torch.empty(4, dtype=torch.float32, device=device)
        logp = torch.empty(shape, dtype=torch.float32, device=device)
        n = _loss_workspace(*shape)
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        _check_noctx(lib().fal_policy_loss(byref(r), byref(hp), logits.data_ptr(), targets.data_ptr(), _ptr(mask),
                                           old_logp.data_ptr(), _ptr(ref_logp), advantages.data_ptr(),
                                           stats.data_ptr(), logp.data_ptr(), dlogits.data_ptr(), ws.data_ptr(), n,
                                           stream))
    return PolicyLoss(stats, logp, dlogits)


def preference_loss(logits, targets, ref_logp, mask=None, vocab=None, dlogits=None, *, beta=0.1, label_smoothing=0.0,
                    ipo=False, length_mean=False, temperature=1.0):
    """Preference loss over the pairs (b, b + B/2) of which the first is
    preferred, and its gradient with respect to the logits
    (fal_preference_loss): ref_logp is float32 [B], the reference model's
    log-probability of each sequence."""
    import torch
    r = _logit_rows(logits, targets, mask, vocab, temperature)
    device = logits.device
    B, T = targets.shape
    _dense(ref_logp, "ref_logp", (B,), (torch.float32,), device)
    hp = fal_preference_t(beta, label_smoothing, int(ipo), int(length_mean))
    with _call(device) as stream:
        dlogits = _gradient_rows(r, logits, dlogits)
        loss = torch.empty(1, dtype=torch.float32, device=device)
        seq_logp = torch.empty(B, dtype=torch.float32, device=device)
        n = _loss_workspace(B, T)
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        _check_noctx(lib().fal_preference_loss(byref(r), byref(hp), logits.data_ptr(), targets.data_ptr(), _ptr(mask),
                                               ref_logp.data_ptr(), loss.data_ptr(), seq_logp.data_ptr(),
                                               dlogits.data_ptr(), ws.data_ptr(), n, stream))
    return PreferenceLoss(loss, seq_logp, dlogits)


class Fal:
    """A libfal context with PyTorch-owned device buffers on the current GPU.

    Calls run on stream_main (the current stream of the constructor unless
    given).  A caller on another stream orders the two itself, inputs before the
    call and results after it, as between any two streams; the memory of token
    arrays and of results is kept until both are done with it."""

    def __init__(self, cfg: Config, stream_main=None, stream_aux=None):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.layout = param_layout(cfg)
        self.ws_bytes = workspace_bytes(cfg)
        dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        self._ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=dev)
        ptr = self._ws.data_ptr()
        self.ws_ptr = (ptr + 255) // 256 * 256
        self.stream_main = stream_main if stream_main is not None else torch.cuda.current_stream(dev)
        self.stream_aux = stream_aux if stream_aux is not None else torch.cuda.Stream(dev)
        self.pdtype = torch.bfloat16 if cfg.dtype == 1 else torch.float32
        self.params = torch.zeros(self.layout["total"], dtype=self.pdtype, device=dev)
        self.grads = torch.zeros(self.layout["total"], dtype=torch.float32, device=dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        c = to_c(cfg)
        self._ccfg = c
        ctx = c_void_p()
        _check(lib().fal_init(byref(c), c_void_p(self.ws_ptr), self.ws_bytes,
                              c_void_p(self.stream_main.cuda_stream), c_void_p(self.stream_aux.cuda_stream),
                              byref(ctx)))
        self.ctx = ctx

    def close(self):
        if getattr(self, "ctx", None):
            lib().fal_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -------------------------------------------------------------- params --
    def load_params(self, gparams: dict, blocks: list):
        flat = flatten_params(self.cfg, gparams, blocks, self.layout)
        t = self.torch.from_numpy(flat).to(self.pdtype)
        self.params.copy_(t.to(self.device))

    def block_param_ptr(self, i: int) -> int:
        es = self.params.element_size()
        return self.params.data_ptr() + (self.layout["block_base"] + i * self.layout["block_stride"]) * es

    def block_grad_ptr(self, i: int) -> int:
        return self.grads.data_ptr() + (self.layout["block_base"] + i * self.layout["block_stride"]) * 4

    def grads_numpy(self):
        from .synth import block_shapes, global_shapes
        flat = self.grads.detach().cpu().numpy()
        return unflatten(self.cfg, flat, global_shapes(self.cfg), block_shapes(self.cfg), self.layout)

    # ---------------------------------------------------------------- calls --
    def _share(self, *tensors, result=False):
        """Tells the allocator of the second stream that uses a tensor: the
        context's reads the caller's, the caller's the results."""
        current = self.torch.cuda.current_stream(self.device)
        if current != self.stream_main:
            for t in tensors:
                if t is not None:
                    t.record_stream(current if result else self.stream_main)

    def model_step(self, tokens, logits=None):
        """tokens: int32 device tensor [B, T+1]; logits: optional fp32 device
        tensor [B*T, V].  Returns the loss tensor (device, shape [1])."""
        assert tokens.dtype == self.torch.int32 and tokens.is_cuda and tokens.is_contiguous()
        lp = c_void_p(logits.data_ptr()) if logits is not None else None
        _check(lib().fal_model_step(self.ctx, c_void_p(self.params.data_ptr()), c_void_p(tokens.data_ptr()),
                                    c_void_p(self.loss.data_ptr()), lp, c_void_p(self.grads.data_ptr())),
               self.ctx)
        self._share(tokens, logits)
        return self.loss

    def model_forward(self, tokens, logits=None, loss=True):
        """Forward only (no gradients).  Returns the loss tensor (device [1])
        when loss is True, else None."""
        assert tokens.dtype == self.torch.int32 and tokens.is_cuda and tokens.is_contiguous()
        lp = c_void_p(logits.data_ptr()) if logits is not None else None
        _check(lib().fal_model_forward(self.ctx, c_void_p(self.params.data_ptr()), c_void_p(tokens.data_ptr()),
                                       c_void_p(self.loss.data_ptr()) if loss else None, lp), self.ctx)
        self._share(tokens, logits)
        return self.loss if loss else None

    def stack_forward(self, x_in, x_out=None):
        _check(lib().fal_stack_forward(self.ctx, c_void_p(self.params.data_ptr()), c_void_p(x_in.data_ptr()),
                                       c_void_p(x_out.data_ptr()) if x_out is not None else None), self.ctx)

    def stack_step(self, x_in, dy, dx_in=None):
        _check(lib().fal_stack_step(self.ctx, c_void_p(self.params.data_ptr()), c_void_p(x_in.data_ptr()),
                                    c_void_p(dy.data_ptr()), c_void_p(self.loss.data_ptr()),
                                    c_void_p(self.grads.data_ptr()),
                                    c_void_p(dx_in.data_ptr()) if dx_in is not None else None), self.ctx)
        return self.loss

    def block_fwd(self, layer, x_in, x_out, first):
        _check(lib().fal_block_fwd(self.ctx, layer, c_void_p(self.block_param_ptr(layer)),
                                   c_void_p(x_in.data_ptr()), c_void_p(x_out.data_ptr()),
                                   c_void_p(first.data_ptr()) if first is not None else None), self.ctx)

    def block_bwd(self, layer, x_in, first, dx_out, dx_in, dfirst):
        _check(lib().fal_block_bwd(self.ctx, layer, c_void_p(self.block_param_ptr(layer)),
                                   c_void_p(x_in.data_ptr()),
                                   c_void_p(first.data_ptr()) if first is not None else None,
                                   c_void_p(dx_out.data_ptr()),
                                   c_void_p(dx_in.data_ptr()),
                                   c_void_p(dfirst.data_ptr()) if dfirst is not None else None,
                                   c_void_p(self.block_grad_ptr(layer))), self.ctx)

    # ------------------------------------------- window, tuning losses --
    def set_attention_window(self, window, sinks=0):
        """Every later forward and backward attends causally over the last
        `window` keys and the first `sinks`; window 0 restores the full mask."""
        _check(lib().fal_set_attention_window(self.ctx, _clamp32(window), _clamp32(sinks)), self.ctx)

    def _empty(self, *shape):
        """An fp32 result, allocated on the stream that will write it."""
        with self.torch.cuda.stream(self.stream_main):
            t = self.torch.empty(shape, dtype=self.torch.float32, device=self.device)
        self._share(t, result=True)
        return t

    def _token_arrays(self, tokens, mask, **arrays):
        torch = self.torch
        B, T = self.cfg.batch, self.cfg.seq_len
        _dense(tokens, "tokens", (B, T + 1), (torch.int32,), self.device)
        if mask is not None:
            _dense(mask, "mask", (B, T), (torch.bool, torch.uint8), self.device)
        for name, t in arrays.items():
            if t is not None:
                _dense(t, name, (B,) if name == "ref_seq_logp" else (B, T), (torch.float32,), self.device)
        self._share(tokens, mask, *arrays.values())

    def model_logprobs(self, tokens, mask=None, temperature=1.0, entropy=False):
        """Log-probabilities of tokens[:, 1:] under the model, float32 [B, T]
        (zero where mask, over the T predicted tokens, is zero); with
        entropy=True also the entropies."""
        self._token_arrays(tokens, mask)
        logp = self._empty(self.cfg.batch, self.cfg.seq_len)
        ent = self._empty(self.cfg.batch, self.cfg.seq_len) if entropy else None
        _check(lib().fal_model_logprobs(self.ctx, self.params.data_ptr(), tokens.data_ptr(), _ptr(mask), temperature,
                                        logp.data_ptr(), _ptr(ent)), self.ctx)
        return (logp, ent) if entropy else logp

    def policy_step(self, tokens, old_logp, advantages, ref_logp=None, mask=None, *, clip_low=0.2, clip_high=0.2,
                    kl_coef=0.0, sequence_mean=False, temperature=1.0):
        """Forward, clipped policy loss over tokens[:, 1:] and backward: fills
        self.grads and returns the stats of policy_loss (float32 [4]) and the
        log-probabilities (float32 [B, T])."""
        self._token_arrays(tokens, mask, old_logp=old_logp, advantages=advantages, ref_logp=ref_logp)
        hp = fal_policy_t(clip_low, clip_high, kl_coef, int(sequence_mean))
        stats, logp = self._empty(4), self._empty(self.cfg.batch, self.cfg.seq_len)
        _check(lib().fal_policy_step(self.ctx, self.params.data_ptr(), byref(hp), tokens.data_ptr(), _ptr(mask),
                                     temperature, _ptr(old_logp), _ptr(ref_logp), _ptr(advantages), stats.data_ptr(),
                                     logp.data_ptr(), self.grads.data_ptr()), self.ctx)
        return stats, logp

    def preference_step(self, tokens, ref_logp, mask=None, *, beta=0.1, label_smoothing=0.0, ipo=False,
                        length_mean=False, temperature=1.0):
        """Forward, preference loss over the pairs (b, b + B/2) of tokens[:,
        1:] and backward: fills self.grads and returns the loss (self.loss)
        and the sequences' log-probabilities (float32 [B])."""
        self._token_arrays(tokens, mask, ref_seq_logp=ref_logp)
        hp = fal_preference_t(beta, label_smoothing, int(ipo), int(length_mean))
        seq_logp = self._empty(self.cfg.batch)
        _check(lib().fal_preference_step(self.ctx, self.params.data_ptr(), byref(hp), tokens.data_ptr(), _ptr(mask),
                                         temperature, _ptr(ref_logp), self.loss.data_ptr(), seq_logp.data_ptr(),
                                         self.grads.data_ptr()), self.ctx)
        return self.loss, seq_logp

    # ----------------------------------------------------------- optimizer --
    def init_optimizer(self):
        """fp32 master weights (copied from the current parameters) and zero
        AdamW moments, all in the flat parameter layout."""
        torch = self.torch
        self.master = self.params.float().clone() if self.cfg.dtype == 1 else self.params
        self.m = torch.zeros_like(self.grads)
        self.v = torch.zeros_like(self.grads)
        self.grad_norm = torch.zeros(1, dtype=torch.float32, device=self.device)
        self.opt_step = 0

    def adamw_step(self, **hp):
        """One AdamW update of every parameter from self.grads (defaults: the
        paper's lr 1e-4, weight decay 0.001, clip 1).  Returns the pre-clip
        gradient norm (device tensor [1])."""
        if getattr(self, "master", None) is None:
            self.init_optimizer()
        self.opt_step += 1
        p = adamw_params(**hp)
        lp = c_void_p(self.params.data_ptr()) if self.cfg.dtype == 1 else None
        _check(lib().fal_adamw_step(self.ctx, byref(p), self.opt_step, self.layout["total"],
                                    c_void_p(self.master.data_ptr()), lp, c_void_p(self.grads.data_ptr()),
                                    c_void_p(self.m.data_ptr()), c_void_p(self.v.data_ptr()),
                                    c_void_p(self.grad_norm.data_ptr())), self.ctx)
        return self.grad_norm

    def train_step(self, tokens, **hp):
        """Forward + backward (fal_model_step) and one AdamW update; returns
        the loss of the batch before the update (device tensor [1])."""
        self.model_step(tokens)
        self.adamw_step(**hp)
        return self.loss

    def profile_enable(self, on: bool = True):
        _check(lib().fal_profile_enable(self.ctx, 1 if on else 0), self.ctx)

    def profile_read(self) -> dict:
        out = {}
        for cls, name in PROF_NAMES.items():
            n, ms, fl, by = c_int64(), c_double(), c_double(), c_double()
            _check(lib().fal_profile_read(self.ctx, cls, byref(n), byref(ms), byref(fl), byref(by)), self.ctx)
            out[name] = {"launches": n.value, "ms": ms.value, "flops": fl.value, "bytes": by.value}
        return out

    def residual_out(self):
        p = c_void_p()
        _check(lib().fal_residual_out(self.ctx, byref(p)))
        return p.value
