"""ctypes binding of libwino.so - argument marshalling only.

Every function here has the name of the C entry point it calls and forwards
plain pointers, sizes and a stream handle.  torch tensors are accepted where a
device pointer is expected (their data_ptr() is passed after a device / dtype /
contiguity check).  All computation happens in the HIP library; if it is not
built, importing this module fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libwino.so")


class WinoError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        msg = f"{where}: {status_string(status)} ({status})"
        if detail:
            msg += f": {detail}"
        super().__init__(msg)


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"libwino.so not found at {_LIB_PATH}; build it with "
            "`python paper_2605_16941_amd/build.py` (hipcc, gfx950)")
    # The library must run on the HIP runtime that allocates the device memory
    # it is handed.  torch ships its own copy of that runtime: loaded first,
    # it satisfies the library's runtime dependency; loaded after the library,
    # it joins the system copy the library pulled in, and pointers of one copy
    # are unknown to the other (wino_create then fails with WINO_ERR_HIP).
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    return C.CDLL(_LIB_PATH)


lib = _load()

N_KERNEL_CLASSES = 13
WINO_FLAG_NO_FORCE_TOP1 = 0x1
WINO_FLAG_NO_CAP_FILL = 0x2
KEEP, DRAFT, REMASK, FORCED, CAPFILL = 0, 1, 2, 3, 4
STATUS = {0: "WINO_OK", -1: "WINO_ERR_INVALID_ARG", -2: "WINO_ERR_SHAPE", -3: "WINO_ERR_HIP",
          -4: "WINO_ERR_NO_MEMORY", -5: "WINO_ERR_STEP_CAP", -6: "WINO_ERR_UNSUPPORTED"}


class wino_model_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("head_dim", C.c_int32), ("d_ff", C.c_int32), ("vocab", C.c_int32),
                ("rope_theta", C.c_float), ("rms_eps", C.c_float), ("act_precision", C.c_int32)]


ACT_BF16, ACT_FP16 = 0, 1


class wino_weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("attn_norm", C.POINTER(C.c_void_p)),
                ("w_qkv", C.POINTER(C.c_void_p)), ("w_o", C.POINTER(C.c_void_p)),
                ("ffn_norm", C.POINTER(C.c_void_p)), ("w_gate_up", C.POINTER(C.c_void_p)),
                ("w_down", C.POINTER(C.c_void_p)), ("final_norm", C.c_void_p),
                ("lm_head", C.c_void_p), ("lm_bias", C.c_void_p)]


class wino_params(C.Structure):
    _fields_ = [("batch", C.c_int32), ("prompt_len", C.c_int32), ("gen_len", C.c_int32),
                ("block_len", C.c_int32), ("mask_id", C.c_int32), ("tau1", C.c_float),
                ("tau2", C.c_float), ("max_steps", C.c_int32), ("flags", C.c_uint32),
                ("tokens_per_step", C.c_int32)]


class wino_row_stats(C.Structure):
    _fields_ = [("m_all", C.c_float), ("sumexp", C.c_float), ("z_best", C.c_float),
                ("z_target", C.c_float), ("argmax", C.c_int32), ("row_kind", C.c_int32)]


ROW_STATS_BYTES = C.sizeof(wino_row_stats)


class wino_row_loss(C.Structure):
    _fields_ = [("entropy", C.c_float), ("nll", C.c_float), ("conf", C.c_float), ("argmax", C.c_int32)]


ROW_LOSS_BYTES = C.sizeof(wino_row_loss)

ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_BASE, ROPE_SCALE_PARTS = 0, 1, 2, 3
MASK_FULL, MASK_CAUSAL, MASK_SHADOW = 0, 1, 2


class wino_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class wino_kv_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class wino_rope_params(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("dtype", C.c_int32),
                ("inverse", C.c_int32), ("magnitude", C.c_float)]


class wino_rope_config(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("scaling", C.c_int32), ("theta", C.c_double), ("factor", C.c_double),
                ("orig_len", C.c_double), ("turns_fast", C.c_double), ("turns_slow", C.c_double)]


class wino_attn_params(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("mask", C.c_int32), ("block_len", C.c_int32), ("scale", C.c_float)]

_vp, _i32, _u32, _sz, _i64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_size_t, C.c_int64
_P = C.POINTER
_protos = {
    "wino_create": (_i32, [_P(wino_model_config), _P(wino_weights), _i32, _i32, _P(_vp)]),
    "wino_destroy": (_i32, [_vp]),
    "wino_workspace_bytes": (_sz, [_P(wino_model_config), _i32, _i32]),
    "wino_step": (_i32, [_vp, _P(wino_params), _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "wino_decode_block": (_i32, [_vp, _P(wino_params), _vp, _vp, _vp, _P(_i32), _vp]),
    "wino_decode": (_i32, [_vp, _P(wino_params), _vp, _vp, _vp, _vp, _i32, _P(_i32), _P(_i32), _vp]),
    "wino_epilogue_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "wino_epilogue": (_i32, [_P(wino_params), _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "wino_epilogue_noalloc": (_i32, [_P(wino_params), _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "wino_row_losses": (_i32, [_vp, _P(wino_params), _vp, _vp, _vp, _vp]),
    "wino_rope_frequencies": (_i32, [_P(wino_rope_config), _P(C.c_double), _P(C.c_float)]),
    "wino_rope": (_i32, [_P(wino_rope_params), _i64, _i32, _vp, _vp, _P(wino_heads), _P(wino_heads), _vp]),
    "wino_rope_append": (_i32, [_P(wino_rope_params), _P(wino_kv_cache), _i64, _i32, _vp, _vp, _vp] +
                         [_P(wino_heads)] * 4 + [_vp]),
    "wino_attention_workspace_bytes": (_sz, [_P(wino_attn_params), _i32, _i32, _i32]),
    "wino_paged_attention": (_i32, [_P(wino_attn_params), _P(wino_kv_cache), _i32, _i32, _i32, _vp, _vp, _vp, _i64,
                                    _i32, _vp, _P(wino_heads), _P(wino_heads), _vp, _vp, _sz, _vp]),
    "wino_packed_attention": (_i32, [_P(wino_attn_params), _i32, _i32, _i32, _i32, _vp, _vp, _vp] +
                              [_P(wino_heads)] * 4 + [_vp, _vp, _sz, _vp]),
    "wino_debug_logits": (_i32, [_vp, _P(wino_params), _vp, _vp, _vp, _vp]),
    "wino_debug_forward": (_i32, [_vp, _P(wino_params), _vp, _vp, _i32, _vp, _vp]),
    "wino_debug_gemm": (_i32, [_vp, _vp, _i32, _i32, _i32, _vp, _vp]),
    "wino_profile": (_i32, [_vp, _u32]),
    "wino_profile_read": (_i32, [_vp, _P(C.c_int64), _P(C.c_double), _P(C.c_double), _P(C.c_double)]),
    "wino_kernel_class_name": (C.c_char_p, [_i32]),
    "wino_status_string": (C.c_char_p, [_i32]),
    "wino_last_error": (C.c_char_p, [_vp]),
}
for _name, (_res, _args) in _protos.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTED = tuple(_protos)


# ------------------------------------------------------------------ helpers
# The binding's own time counts where a call's kernels take a few microseconds
# (one block's epilogue: 10 us of kernels), so nothing is imported or looked up per
# call and the current stream is read as a raw handle (no Stream object).
try:
    import torch as _torch
    _Tensor, _i32_t, _u8_t = _torch.Tensor, _torch.int32, _torch.uint8
    _f32_t, _bf16_t = _torch.float32, _torch.bfloat16
    _i64_t, _f64_t = _torch.int64, _torch.float64
    _act_t = (_bf16_t, _torch.float16)  # by activation type
    _get_device = getattr(_torch._C, "_cuda_getDevice", None)
except ImportError:  # int pointers only
    _torch = _Tensor = _i32_t = _u8_t = _f32_t = _bf16_t = _i64_t = _f64_t = _get_device = None
    _act_t = (None, None)
_raw_stream = getattr(_torch._C, "_cuda_getCurrentRawStream", None) if _torch else None


def _ptr(x, dtype=None, name="tensor"):
    """Device pointer of a torch tensor (checked), an int, or None."""
    if x is None or isinstance(x, int):
        return x
    if _Tensor is None or not isinstance(x, _Tensor):
        raise TypeError(f"{name}: expected a torch tensor, int pointer or None")
    if not x.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    if dtype is not None and x.dtype != dtype:
        raise TypeError(f"{name}: dtype {x.dtype}, expected {dtype}")
    if not x.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _torch.cuda.is_initialized():
            return _raw_stream(_torch._C._cuda_getDevice())
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def status_string(s: int) -> str:
    return lib.wino_status_string(int(s)).decode()


def _check(status, where, ctx=None):
    if status != 0:
        detail = lib.wino_last_error(ctx).decode() if ctx else ""
        raise WinoError(status, where, detail)


def make_params(batch, prompt_len, gen_len, block_len, mask_id, tau1=0.7, tau2=0.9,
                max_steps=0, flags=0, tokens_per_step=0) -> wino_params:
    return wino_params(batch, prompt_len, gen_len, block_len, mask_id, tau1, tau2, max_steps, flags,
                       tokens_per_step)


# ------------------------------------------------------------------ entry points
def wino_workspace_bytes(cfg: wino_model_config, max_batch: int, max_seq: int) -> int:
    return int(lib.wino_workspace_bytes(C.byref(cfg), max_batch, max_seq))


def wino_create(cfg: wino_model_config, weights: wino_weights, max_batch: int, max_seq: int) -> int:
    out = C.c_void_p()
    s = lib.wino_create(C.byref(cfg), C.byref(weights), max_batch, max_seq, C.byref(out))
    if s != 0:
        raise WinoError(s, "wino_create", lib.wino_last_error(None).decode())
    return out.value


def wino_destroy(ctx: int) -> None:
    _check(lib.wino_destroy(ctx), "wino_destroy")


def wino_step(ctx, p: wino_params, tokens, block_start, block_steps=None, flags=None,
              n_masked=None, stats=None, stream=None) -> None:
    _check(lib.wino_step(ctx, C.byref(p), _ptr(tokens, _i32_t, "tokens"),
                         _ptr(block_start, _i32_t, "block_start"),
                         _ptr(block_steps, _i32_t, "block_steps"),
                         _ptr(flags, _u8_t, "flags"), _ptr(n_masked, _i32_t, "n_masked"),
                         _ptr(stats, None, "stats"), _stream(stream)), "wino_step", ctx)


def wino_decode_block(ctx, p: wino_params, tokens, block_start, final_step=None, stream=None):
    """Returns the per-sequence steps.  final_step as in wino_decode."""
    steps = (C.c_int32 * p.batch)()
    fs = _ptr(final_step, _i32_t, "final_step") if final_step is not None else None
    _check(lib.wino_decode_block(ctx, C.byref(p), _ptr(tokens, _i32_t, "tokens"),
                                 _ptr(block_start, _i32_t, "block_start"), fs, steps,
                                 _stream(stream)), "wino_decode_block", ctx)
    return list(steps)


def wino_decode(ctx, p: wino_params, tokens, block_start, final_step=None, stream=None,
                block_steps=None, max_forwards=0):
    """Returns (per-sequence steps, batched forward passes).  final_step: int32
    [batch, gen_len] device tensor for the finalization steps, or None;
    block_steps: int32 [batch] device tensor (in/out) of steps already taken
    in each current block, or None; max_forwards > 0 stops early with a
    resumable state."""
    steps = (C.c_int32 * p.batch)()
    fw = C.c_int32(0)
    fs = _ptr(final_step, _i32_t, "final_step") if final_step is not None else None
    _check(lib.wino_decode(ctx, C.byref(p), _ptr(tokens, _i32_t, "tokens"),
                           _ptr(block_start, _i32_t, "block_start"),
                           _ptr(block_steps, _i32_t, "block_steps"), fs, int(max_forwards), steps,
                           C.byref(fw), _stream(stream)), "wino_decode", ctx)
    return list(steps), fw.value


def wino_row_losses(ctx, p: wino_params, tokens, targets, out, stream=None) -> None:
    """WINO+ per-row quantities of training states (Sec. 5.2-5.3).  tokens int32
    [B, P+G], targets int32 [B, G], out: device buffer of B*G wino_row_loss
    (16 bytes each: entropy, nll, conf float32; argmax int32)."""
    _check(lib.wino_row_losses(ctx, C.byref(p), _ptr(tokens, _i32_t, "tokens"),
                               _ptr(targets, _i32_t, "targets"), _ptr(out, None, "out"),
                               _stream(stream)), "wino_row_losses", ctx)


def wino_epilogue_workspace_bytes(batch: int, block_len: int, vocab: int) -> int:
    return int(lib.wino_epilogue_workspace_bytes(batch, block_len, vocab))


def wino_epilogue(p: wino_params, vocab: int, logits, cur_tokens, mask_bitmap, flags=None,
                  stats=None, workspace=None, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(lib.wino_epilogue(C.byref(p), vocab, _ptr(logits, _bf16_t, "logits"),
                             _ptr(cur_tokens, _i32_t, "cur_tokens"),
                             _ptr(mask_bitmap, _u8_t, "mask_bitmap"),
                             _ptr(flags, _u8_t, "flags"), _ptr(stats, None, "stats"),
                             _ptr(workspace, None, "workspace"), workspace_bytes,
                             _stream(stream)), "wino_epilogue")


EPILOGUE_NOALLOC_MAX_BYTES = 2 << 20


def wino_epilogue_noalloc(p: wino_params, vocab: int, logits, cur_tokens, mask_bitmap, flags=None,
                          stats=None, stream=None) -> None:
    """wino_epilogue with the library's own per-GPU scratch (no workspace)."""
    _check(lib.wino_epilogue_noalloc(C.byref(p), vocab, _ptr(logits, _bf16_t, "logits"),
                                     _ptr(cur_tokens, _i32_t, "cur_tokens"),
                                     _ptr(mask_bitmap, _u8_t, "mask_bitmap"),
                                     _ptr(flags, _u8_t, "flags"), _ptr(stats, None, "stats"),
                                     _stream(stream)), "wino_epilogue_noalloc")


# ------------------------------------------------------------------ operators on the caller's tensors
def _fit(n):
    """n for a 32-bit argument, of which ctypes would take the lower bits: the nearest number that fits, which every
    limit refuses (counts of keys and pages, which 32-bit offsets and ids index, have none and need no more)."""
    return n if -0x80000000 <= n <= 0x7FFFFFFF else (0x7FFFFFFF if n > 0 else -0x80000000)


def _current_device():
    try:
        return _get_device() if _get_device else _torch.cuda.current_device()
    except Exception:  # no device: there is no device tensor either
        return None


def _stream_on(stream, dev):
    """_stream, with the current device known."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(dev)
    return _stream(stream)


def _wrong_device(x, dev, name):
    if not x.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    raise ValueError(f"{name}: on device {x.get_device()}, the current device is {dev}")


def _op_ptr(x, dtype, name, dev, numel=None):
    """Device pointer of a contiguous tensor of device `dev` (the current one), with at least `numel` elements."""
    if not isinstance(x, _Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if x.get_device() != dev:
        _wrong_device(x, dev, name)
    if dtype is not None and x.dtype is not dtype:
        raise TypeError(f"{name}: dtype {x.dtype}, expected {dtype}")
    if not x.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if numel is not None and x.numel() < numel:
        raise ValueError(f"{name}: {x.numel()} elements, {numel} needed")
    return x.data_ptr() or 16  # an empty tensor has no address


def _heads(x, act, n_heads, head_dim, name, dev, n_tokens) -> wino_heads:
    """Rows of heads [tokens, heads, head_dim] with any token and head strides."""
    if not isinstance(x, _Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if x.dtype is not _act_t[act]:
        raise TypeError(f"{name}: dtype {x.dtype}, expected {_act_t[act]}")
    if x.get_device() != dev:
        _wrong_device(x, dev, name)
    if x.shape != (n_tokens, n_heads, head_dim):
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {(n_tokens, n_heads, head_dim)}")
    ts, hs, es = x.stride()
    if es != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    # the stride of an axis of length one says nothing, and an empty tensor has no address
    return wino_heads(x.data_ptr() or 16, ts if n_tokens > 1 else n_heads * head_dim, hs if n_heads > 1 else head_dim)


def _table(x, batch, dev):
    """Address, row stride and width of a page table: int32 [batch, width], the entries of a row side by side."""
    if not isinstance(x, _Tensor):
        raise TypeError("page_table: expected a torch tensor")
    if x.get_device() != dev:
        _wrong_device(x, dev, "page_table")
    if x.dtype is not _i32_t:
        raise TypeError(f"page_table: dtype {x.dtype}, expected {_i32_t}")
    if x.dim() != 2 or x.shape[0] != batch:
        raise ValueError(f"page_table: shape {tuple(x.shape)}, expected [{batch}, width]")
    width = x.shape[1]
    if width > 1 and x.stride(1) != 1:
        raise ValueError("page_table: the last axis must be contiguous")
    return x.data_ptr() or 16, x.stride(0) if batch > 1 else width, width


def make_rope_params(head_dim, rotary_dim=None, layout=ROPE_HALF, dtype=ACT_BF16, magnitude=1.0,
                     inverse=False) -> wino_rope_params:
    return wino_rope_params(_fit(head_dim), _fit(head_dim if rotary_dim is None else rotary_dim), _fit(layout),
                            _fit(dtype), int(bool(inverse)), magnitude)


def make_attn_params(n_heads, n_kv_heads, head_dim, dtype=ACT_BF16, mask=MASK_FULL, block_len=0,
                     scale=None) -> wino_attn_params:
    """scale: of the scores, 1/sqrt(head_dim) by default."""
    return wino_attn_params(_fit(n_heads), _fit(n_kv_heads), _fit(head_dim), _fit(dtype), _fit(mask), _fit(block_len),
                            head_dim ** -0.5 if scale is None else scale)


def make_kv_cache(k, v) -> wino_kv_cache:
    """The cache held by k and v, device tensors [pages, page_size, kv_heads, head_dim] of the same strides
    (a [pages, kv_heads, page_size, head_dim] cache: its transpose(1, 2)), which stay alive with it."""
    for x, name in ((k, "k"), (v, "v")):
        if not isinstance(x, _Tensor) or x.dim() != 4:
            raise TypeError(f"{name}: expected a tensor [pages, page_size, kv_heads, head_dim]")
        if x.dtype not in _act_t:
            raise TypeError(f"{name}: dtype {x.dtype}, expected bfloat16 or float16")
        if not x.is_cuda:
            raise ValueError(f"{name}: must be a device tensor")
        if x.stride(3) != 1:
            raise ValueError(f"{name}: the last axis must be contiguous")
    if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device:
        raise ValueError("k and v must have the same shape, strides, type and device")
    n, page, heads, hd = k.shape
    sp, st, sh, _ = k.stride()
    c = wino_kv_cache(k.data_ptr(), v.data_ptr(), sp if n > 1 else page * heads * hd, st, sh if heads > 1 else hd,
                      _fit(n), _fit(page), _fit(heads), _fit(hd), _act_t.index(k.dtype))
    c.tensors = (k, v)
    c.device = k.get_device()
    return c


def _check_cache(cache, dev):
    if not isinstance(cache, wino_kv_cache):
        raise TypeError("cache: expected the result of make_kv_cache")
    if cache.device != dev:
        raise ValueError(f"cache: on device {cache.device}, the current device is {dev}")
    return cache


def wino_rope_frequencies(rotary_dim, theta, scaling=ROPE_SCALE_NONE, factor=1.0, orig_len=4096, turns_fast=32.0,
                          turns_slow=1.0):
    """(frequencies in radians per position, a list of rotary_dim/2 floats; the magnitude that goes with them)."""
    rotary_dim = _fit(rotary_dim)
    # (no more than 65536 is accepted)
    out, mag = (C.c_double * min(max(rotary_dim // 2, 1), 32768))(), C.c_float()
    c = wino_rope_config(rotary_dim, _fit(scaling), theta, factor, orig_len, turns_fast, turns_slow)
    _check(lib.wino_rope_frequencies(C.byref(c), out, C.byref(mag)), "wino_rope_frequencies")
    return list(out), mag.value


def wino_rope(p: wino_rope_params, freq, pos, x, out, stream=None) -> None:
    """out = x rotated to positions pos (int32 [tokens]); x and out [tokens, heads, head_dim], out may be x;
    freq float64 [rotary_dim/2] on the device."""
    dev, a, hd = _current_device(), p.dtype, p.head_dim
    n, h, _ = x.shape
    xs, os_ = _heads(x, a, h, hd, "x", dev, n), _heads(out, a, h, hd, "out", dev, n)
    _check(lib.wino_rope(p, n, h, _op_ptr(freq, _f64_t, "freq", dev, p.rotary_dim // 2),
                         _op_ptr(pos, _i32_t, "pos", dev, n), xs, os_, _stream_on(stream, dev)), "wino_rope")


def wino_rope_append(p: wino_rope_params, cache: wino_kv_cache, freq, pos, slot, q, k, v, q_out, stream=None) -> None:
    """q_out = q rotated, and k (rotated) and v into the cache at rows slot (int64 [tokens], outside the cache: not
    written).  q and q_out [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim]."""
    dev, a, hd = _current_device(), p.dtype, p.head_dim
    hk = _check_cache(cache, dev).n_kv_heads
    n, h, _ = q.shape
    qs, ks = _heads(q, a, h, hd, "q", dev, n), _heads(k, a, hk, hd, "k", dev, n)
    vs, os_ = _heads(v, a, hk, hd, "v", dev, n), _heads(q_out, a, h, hd, "q_out", dev, n)
    _check(lib.wino_rope_append(p, cache, n, h, _op_ptr(freq, _f64_t, "freq", dev, p.rotary_dim // 2),
                                _op_ptr(pos, _i32_t, "pos", dev, n), _op_ptr(slot, _i64_t, "slot", dev, n), qs, ks, vs,
                                os_, _stream_on(stream, dev)), "wino_rope_append")


def wino_attention_workspace_bytes(p: wino_attn_params, batch: int, total_q: int, max_kv_len: int) -> int:
    return int(lib.wino_attention_workspace_bytes(p, _fit(batch), _fit(total_q), _fit(max_kv_len)))


def wino_paged_attention(p: wino_attn_params, cache: wino_kv_cache, q, out, cu_q, kv_len, page_table, max_kv_len,
                         cur_start=None, lse=None, workspace=None, stream=None) -> None:
    """Attention of the rows q [total_q, heads, head_dim] (sequence b: rows cu_q[b]..cu_q[b+1]) over the cache's pages
    page_table int32 [batch, width] (rows may be part of wider ones), kv_len int32 [batch] keys each, at most
    max_kv_len.  lse: float32 [total_q, heads] or None; workspace: of wino_attention_workspace_bytes for these sizes or
    larger ones, None if that is 0."""
    dev, a, h, hd = _current_device(), p.dtype, p.n_heads, p.head_dim
    _check_cache(cache, dev)
    n, batch = q.shape[0], kv_len.shape[0]
    table, table_stride, width = _table(page_table, batch, dev)
    qs, os_ = _heads(q, a, h, hd, "q", dev, n), _heads(out, a, h, hd, "out", dev, n)
    _check(lib.wino_paged_attention(
        p, cache, _fit(batch), _fit(n), _fit(max_kv_len), _op_ptr(cu_q, _i32_t, "cu_q", dev, batch + 1),
        _op_ptr(kv_len, _i32_t, "kv_len", dev), table, table_stride, _fit(width),
        None if cur_start is None else _op_ptr(cur_start, _i32_t, "cur_start", dev, batch), qs, os_,
        None if lse is None else _op_ptr(lse, _f32_t, "lse", dev, n * h),
        None if workspace is None else _op_ptr(workspace, None, "workspace", dev),
        0 if workspace is None else workspace.nbytes, _stream_on(stream, dev)), "wino_paged_attention")


def wino_packed_attention(p: wino_attn_params, q, k, v, out, cu_q, cu_k, max_kv_len, cur_start=None, lse=None,
                          workspace=None, stream=None) -> None:
    """Attention of the rows q [total_q, heads, head_dim] over keys and values [total_k, kv_heads, head_dim], sequence b
    owning rows cu_q[b]..cu_q[b+1] and keys cu_k[b]..cu_k[b+1] (int32 [batch + 1]), at most max_kv_len keys each.
    lse and workspace as for wino_paged_attention."""
    dev, a, h, hk, hd = _current_device(), p.dtype, p.n_heads, p.n_kv_heads, p.head_dim
    n, nk, batch = q.shape[0], k.shape[0], cu_q.shape[0] - 1
    qs, os_ = _heads(q, a, h, hd, "q", dev, n), _heads(out, a, h, hd, "out", dev, n)
    ks, vs = _heads(k, a, hk, hd, "k", dev, nk), _heads(v, a, hk, hd, "v", dev, nk)
    _check(lib.wino_packed_attention(
        p, _fit(batch), _fit(n), _fit(nk), _fit(max_kv_len), _op_ptr(cu_q, _i32_t, "cu_q", dev),
        _op_ptr(cu_k, _i32_t, "cu_k", dev, batch + 1),
        None if cur_start is None else _op_ptr(cur_start, _i32_t, "cur_start", dev, batch), qs, ks, vs, os_,
        None if lse is None else _op_ptr(lse, _f32_t, "lse", dev, n * h),
        None if workspace is None else _op_ptr(workspace, None, "workspace", dev),
        0 if workspace is None else workspace.nbytes, _stream_on(stream, dev)), "wino_packed_attention")


def wino_debug_logits(ctx, p: wino_params, tokens, block_start, logits, stream=None) -> None:
    _check(lib.wino_debug_logits(ctx, C.byref(p), _ptr(tokens, _i32_t, "tokens"),
                                 _ptr(block_start, _i32_t, "block_start"),
                                 _ptr(logits, _f32_t, "logits"), _stream(stream)),
           "wino_debug_logits", ctx)


def wino_debug_forward(ctx, p: wino_params, tokens, block_start, n_sublayers, out, stream=None) -> None:
    _check(lib.wino_debug_forward(ctx, C.byref(p), _ptr(tokens, _i32_t, "tokens"),
                                  _ptr(block_start, _i32_t, "block_start"), n_sublayers,
                                  _ptr(out, _f32_t, "out"), _stream(stream)),
           "wino_debug_forward", ctx)


def wino_debug_gemm(A, W, out, stream=None) -> None:
    """out = A W^T (fp32) with the backbone GEMM kernel; A [M,K], W [N,K] bf16."""
    M, K = A.shape
    N = W.shape[0]
    if W.shape[1] != K or tuple(out.shape) != (M, N):
        raise ValueError("wino_debug_gemm: shape mismatch")
    _check(lib.wino_debug_gemm(_ptr(A, _bf16_t, "A"), _ptr(W, _bf16_t, "W"), M, N, K,
                               _ptr(out, _f32_t, "out"), _stream(stream)), "wino_debug_gemm")


def wino_profile(ctx, class_mask: int) -> None:
    _check(lib.wino_profile(ctx, class_mask), "wino_profile", ctx)


def wino_profile_read(ctx) -> dict:
    n = N_KERNEL_CLASSES
    la, ms, fl, by = (C.c_int64 * n)(), (C.c_double * n)(), (C.c_double * n)(), (C.c_double * n)()
    _check(lib.wino_profile_read(ctx, la, ms, fl, by), "wino_profile_read", ctx)
    return {wino_kernel_class_name(i): {"launches": la[i], "ms": ms[i], "flops": fl[i], "bytes": by[i]}
            for i in range(n)}


def wino_kernel_class_name(cls: int) -> str:
    return lib.wino_kernel_class_name(cls).decode()


def wino_status_string(s: int) -> str:
    return status_string(s)


def wino_last_error(ctx) -> str:
    return lib.wino_last_error(ctx).decode()
