"""ctypes binding of include/moe355.h -- argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

MOE_F32, MOE_BF16, MOE_E4M3 = 0, 1, 2
_TORCH = {MOE_F32: torch.float32, MOE_BF16: torch.bfloat16, MOE_E4M3: torch.float8_e4m3fn}
_CODE = {"f32": MOE_F32, "bf16": MOE_BF16, "e4m3": MOE_E4M3}
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB: Optional[C.CDLL] = None
_ARGS = None
_FN = {}            # addresses of the library's functions for _args, the marshalling in C++ of the calls that are over in microseconds


class MoeError(RuntimeError):
    pass


class MoeCfg(C.Structure):
    _fields_ = [("T", C.c_int32), ("d", C.c_int32), ("f", C.c_int32), ("E", C.c_int32), ("k", C.c_int32),
                ("dtype", C.c_int32), ("renorm", C.c_int32), ("act", C.c_int32), ("gate", C.c_int32),
                ("gate_packed", C.c_int32)]

    @classmethod
    def make(cls, T, d, f, E, k=1, dtype="bf16", renorm=1, act=0, gate=0, gate_packed=0) -> "MoeCfg":
        code = {"bf16": MOE_BF16, "f32": MOE_F32}[dtype] if isinstance(dtype, str) else int(dtype)
        return cls(T, d, f, E, k, code, renorm, act, gate, gate_packed)

    def with_packed_gate(self, on: bool = True) -> "MoeCfg":
        """A copy of this cfg whose W_g arguments are (or are not) the block written by moe_pack_gate."""
        return MoeCfg(self.T, self.d, self.f, self.E, self.k, self.dtype, self.renorm, self.act, self.gate, 1 if on else 0)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == MOE_BF16 else torch.float32


class NormCfg(C.Structure):
    """moe_norm_cfg: rows, columns and types of moe_add_norm."""
    _fields_ = [("T", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32), ("q_group", C.c_int32), ("eps", C.c_float)]

    @classmethod
    def make(cls, T, d, dtype="bf16", eps=1e-6, q_group=0) -> "NormCfg":
        return cls(T, d, _CODE[dtype] if isinstance(dtype, str) else int(dtype), q_group, eps)


class KvCfg(C.Structure):
    """moe_kv_cfg: a paged cache of keys and values."""
    _fields_ = [("pages", C.c_int32), ("page_size", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("cache_dtype", C.c_int32)]

    @classmethod
    def make(cls, pages, page_size, heads, head_dim, dtype="bf16", cache_dtype=None) -> "KvCfg":
        code = _CODE[dtype] if isinstance(dtype, str) else int(dtype)
        cache = code if cache_dtype is None else _CODE[cache_dtype] if isinstance(cache_dtype, str) else int(cache_dtype)
        return cls(pages, page_size, heads, head_dim, code, cache)

    def empty(self, device="cuda"):
        """(k_pages, v_pages, k_scales, v_scales) of this cache, not filled; the scales are None unless it is an e4m3 cache."""
        shape = (self.pages, self.heads, self.page_size, self.head_dim)
        k, v = (torch.empty(shape, dtype=_TORCH[self.cache_dtype], device=device) for _ in range(2))
        if self.cache_dtype != MOE_E4M3:
            return k, v, None, None
        return (k, v, *(torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in range(2)))


class AttnCfg(C.Structure):
    """moe_attn_cfg: the sequences and query heads of one moe_attn_decode."""
    _fields_ = [("B", C.c_int32), ("q_heads", C.c_int32), ("table_pages", C.c_int32), ("window", C.c_int32), ("scale", C.c_float)]

    @classmethod
    def make(cls, B, q_heads, table_pages, scale=0.0, window=0) -> "AttnCfg":
        return cls(B, q_heads, table_pages, window, scale)


class ScoresCfg(C.Structure):
    """moe_scores_cfg: scores capped by a tanh or biased by distance."""
    _fields_ = [("cap", C.c_float), ("back", C.c_int32), ("ahead", C.c_int32)]

    @classmethod
    def make(cls, cap=0.0, back=0, ahead=0) -> "ScoresCfg":
        return cls(cap, back, ahead)


class PromptCfg(C.Structure):
    """moe_prompt_cfg: the tokens, sequences and query heads of one moe_attn_prompt."""
    _fields_ = [("tokens", C.c_int32), ("B", C.c_int32), ("q_heads", C.c_int32), ("table_pages", C.c_int32), ("window", C.c_int32),
                ("scale", C.c_float)]

    @classmethod
    def make(cls, tokens, B, q_heads, table_pages, scale=0.0, window=0) -> "PromptCfg":
        return cls(tokens, B, q_heads, table_pages, window, scale)


_PAIRS = {"half": 0, "neighbours": 1}
_SCALING = {"none": 0, "linear": 1, "base": 2, "parts": 3}


class RopeCfg(C.Structure):
    """moe_rope_cfg: heads, columns, pairs and frequencies of moe_rope."""
    _fields_ = [("q_heads", C.c_int32), ("k_heads", C.c_int32), ("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("dtype", C.c_int32),
                ("pairs", C.c_int32), ("scaling", C.c_int32), ("original", C.c_int32), ("base", C.c_float), ("factor", C.c_float),
                ("slow", C.c_float), ("fast", C.c_float), ("amplitude", C.c_float)]

    @classmethod
    def make(cls, q_heads, k_heads, head_dim, rot_dim=None, dtype="bf16", pairs="half", base=10000.0, scaling="none", factor=1.0,
             original=0, slow=1.0, fast=32.0, amplitude=1.0) -> "RopeCfg":
        code = _CODE[dtype] if isinstance(dtype, str) else int(dtype)
        return cls(q_heads, k_heads, head_dim, head_dim if rot_dim is None else rot_dim, code, _PAIRS[pairs] if isinstance(pairs, str) else int(pairs),
                   _SCALING[scaling] if isinstance(scaling, str) else int(scaling), original, base, factor, slow, fast, amplitude)


def lib_path() -> str:
    """The library next to this file, or the build named by the environment variable MOE355_LIB."""
    return os.environ.get("MOE355_LIB") or os.path.join(_HERE, "libmoe355.so")


def lib() -> C.CDLL:
    """The loaded library; raises if it was never built (python -m paper_2106_10715_amd.build)."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise MoeError(f"{path} is missing: build it with `python paper_2106_10715_amd/build.py`; "
                           "there is no non-HIP fallback")
        L = C.CDLL(path)
        p, i32p, f32p, cfgp = C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(MoeCfg)
        L.moe_last_error.restype = C.c_char_p
        L.moe_last_error.argtypes = []
        sigs = {
            "moe_workspace_bytes": [cfgp, C.POINTER(C.c_size_t)],
            "moe_expert_bytes": [cfgp, C.POINTER(C.c_size_t)],
            "moe_pack_weights": [cfgp, p, p, p, p, p],
            "moe_gate_bytes": [cfgp, C.POINTER(C.c_size_t)],
            "moe_pack_gate": [cfgp, p, p, p],
            "moe_route": [cfgp, p, p, f32p, i32p, f32p, p, p],
            "moe_permute": [cfgp, p, i32p, i32p, i32p, i32p, i32p, p, p, p],
            "moe_permute_static": [cfgp, p, i32p, i32p, i32p, i32p, i32p, p, p],
            "moe_expert_ffn": [cfgp, p, i32p, p, p, p, p],
            "moe_combine": [cfgp, p, i32p, f32p, p, p],
            "moe_layer_forward": [cfgp, p, p, f32p, p, p, p, p, p],
            "moe_stream_ctx_create": [cfgp, p, C.c_size_t, p, C.c_int32, C.POINTER(C.c_void_p)],
            "moe_stream_ctx_destroy": [p],
            "moe_stream_ctx_stats": [p, C.POINTER(C.c_int32), C.POINTER(C.c_size_t), C.POINTER(C.c_float)],
            "moe_schedule_order": [C.POINTER(C.c_int32), C.c_int32, C.c_double, C.c_int32, C.POINTER(C.c_int32),
                                   C.POINTER(C.c_int32), C.POINTER(C.c_int32)],
            "moe_stream_ctx_set_order": [p, C.c_int32, C.c_double, C.c_int32],
            "moe_stream_ctx_last_order": [p, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32)],
            "moe_stream_slots_that_fit": [C.POINTER(MoeCfg), C.c_size_t, C.POINTER(C.c_int32)],
            "moe_stream_ctx_keep_experts": [p, C.c_int32],
            "moe_stream_ctx_prefetch": [p, C.c_int32],
            "moe_stream_ctx_share_loader": [p, p],
            "moe_plan_slots": [C.POINTER(C.c_int32), C.c_int32, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int64),
                               C.POINTER(C.c_int64), C.POINTER(C.c_int32), C.POINTER(C.c_int32)],
            "moe_timer_create": [C.c_int32, C.c_int32, C.POINTER(C.c_void_p)],
            "moe_timer_destroy": [p],
            "moe_timer_reset": [p],
            "moe_timer_read": [p, C.POINTER(C.c_float), C.c_int32, C.POINTER(C.c_int32)],
            "moe_layer_forward_timed": [cfgp, p, p, f32p, p, p, p, p, p],
            "moe_add_norm": [p] * 9,
            "moe_kv_write": [p, C.c_int32, p, C.c_int64, p, C.c_int64, p, p, p, p, p, p],
            "moe_kv_read": [p, C.c_int32, p, p, p, p, p, p, C.c_int64, p, C.c_int64, p],
            "moe_attn_workspace_bytes": [p, p, C.POINTER(C.c_size_t)],
            "moe_attn_decode": [p, p, p, C.c_int64, p, p, p, p, p, p, p, p, p, p],
            "moe_attn_decode_scored": [p, p, p, p, C.c_int64, *[p] * 12],
            "moe_attn_prompt_workspace_bytes": [p, p, C.POINTER(C.c_size_t)],
            "moe_attn_prompt": [p, p, p, p, C.c_int64, *[p] * 15],
            "moe_rope_frequencies": [p, p],
            "moe_rope": [p, C.c_int32, p, p, p, C.c_int64, p, C.c_int64, p, C.c_int64, p, C.c_int64, p],
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.restype = C.c_int
            fn.argtypes = args
            _FN[name] = C.cast(fn, p).value
        _LIB = L
    return _LIB


def _check(rc: int) -> None:
    if rc != 0:
        raise MoeError(f"moe355 error {rc}: {lib().moe_last_error().decode()}")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise MoeError("tensors passed to moe355 must be contiguous")
    return C.c_void_p(t.data_ptr())


# The current stream's handle without a Stream object around it (about a microsecond a call), where this torch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream: Optional[torch.cuda.Stream]):
    return stream.cuda_stream if stream is not None else _raw_stream(torch.cuda.current_device())


_SIZES = {"attn_prompt": "moe_attn_prompt_workspace_bytes"}     # what says how large a call's workspace is; else moe_attn_workspace_bytes


def _native(name: str, *args, stream=None) -> bool:
    """The call through _args.  False where an argument is not as it has to be: the caller then says which and why, and calls nothing."""
    global _ARGS
    if _LIB is None or _ARGS is None:
        lib()
        try:
            from . import _args
        except ImportError as e:
            raise MoeError(f"_args is not built: run python -m paper_2106_10715_amd.build ({e})")
        _ARGS = _args
    rc = getattr(_ARGS, name)(_FN["moe_" + name], _FN[_SIZES.get(name, "moe_attn_workspace_bytes")], *args, None if stream is None else stream.cuda_stream)
    if rc is None:
        return False
    _check(rc)
    return True


def moe_workspace_bytes(cfg: MoeCfg) -> int:
    n = C.c_size_t(0)
    _check(lib().moe_workspace_bytes(C.byref(cfg), C.byref(n)))
    return n.value


def moe_expert_bytes(cfg: MoeCfg) -> int:
    n = C.c_size_t(0)
    _check(lib().moe_expert_bytes(C.byref(cfg), C.byref(n)))
    return n.value


def moe_pack_weights(cfg, W_in_e, W_gate_e, W_out_e, packed_e, stream=None) -> None:
    _check(lib().moe_pack_weights(C.byref(cfg), _ptr(W_in_e), _ptr(W_gate_e), _ptr(W_out_e), _ptr(packed_e),
                                  _stream(stream)))


def moe_gate_bytes(cfg: MoeCfg) -> int:
    n = C.c_size_t(0)
    _check(lib().moe_gate_bytes(C.byref(cfg), C.byref(n)))
    return n.value


def moe_pack_gate(cfg, W_g, gate_packed, stream=None) -> None:
    _check(lib().moe_pack_gate(C.byref(cfg), _ptr(W_g), _ptr(gate_packed), _stream(stream)))


def moe_route(cfg, x, W_g, gate_bias, idx, w, ws, stream=None) -> None:
    _check(lib().moe_route(C.byref(cfg), _ptr(x), _ptr(W_g), _ptr(gate_bias), _ptr(idx), _ptr(w), _ptr(ws),
                           _stream(stream)))


def moe_permute(cfg, x, idx, counts, offsets, perm, inv, Xp, ws, stream=None) -> None:
    _check(lib().moe_permute(C.byref(cfg), _ptr(x), _ptr(idx), _ptr(counts), _ptr(offsets), _ptr(perm), _ptr(inv),
                             _ptr(Xp), _ptr(ws), _stream(stream)))


def moe_permute_static(cfg, x, idx, counts, offsets, perm, inv, Xp, stream=None) -> None:
    _check(lib().moe_permute_static(C.byref(cfg), _ptr(x), _ptr(idx), _ptr(counts), _ptr(offsets), _ptr(perm), _ptr(inv),
                                    _ptr(Xp), _stream(stream)))


def moe_expert_ffn(cfg, Xp, offsets, W_packed, Yp, ws, stream=None) -> None:
    _check(lib().moe_expert_ffn(C.byref(cfg), _ptr(Xp), _ptr(offsets), _ptr(W_packed), _ptr(Yp), _ptr(ws),
                                _stream(stream)))


def moe_combine(cfg, Yp, inv, w, y, stream=None) -> None:
    _check(lib().moe_combine(C.byref(cfg), _ptr(Yp), _ptr(inv), _ptr(w), _ptr(y), _stream(stream)))


class StreamCtx:
    """Host-streamed expert mode: experts in pinned host memory, K device slots, a copy stream."""

    def __init__(self, cfg: MoeCfg, host_experts: torch.Tensor, dev_slots: torch.Tensor, K: int = 2):
        if not host_experts.is_pinned():
            raise MoeError("host_experts must be pinned host memory")
        self._keep = (host_experts, dev_slots)
        self._h = C.c_void_p(None)
        _check(lib().moe_stream_ctx_create(C.byref(cfg), _ptr(host_experts), moe_expert_bytes(cfg), _ptr(dev_slots),
                                           K, C.byref(self._h)))

    @property
    def handle(self):
        return self._h

    def stats(self):
        n, b, ms = C.c_int32(0), C.c_size_t(0), C.c_float(0)
        _check(lib().moe_stream_ctx_stats(self._h, C.byref(n), C.byref(b), C.byref(ms)))
        return {"n_loaded": n.value, "bytes": b.value, "copy_ms": ms.value}

    def set_order(self, policy: int, tokens_per_load: float = 1.0, K: int = 0) -> None:
        _check(lib().moe_stream_ctx_set_order(self._h, policy, tokens_per_load, K))

    def keep_experts(self, on: bool = True) -> None:
        _check(lib().moe_stream_ctx_keep_experts(self._h, 1 if on else 0))

    def share_loader(self, owner: "StreamCtx") -> None:
        _check(lib().moe_stream_ctx_share_loader(self._h, owner.handle))
        self._owner = owner                      # the owner's stream must outlive this context

    def prefetch(self, expert: int) -> None:
        _check(lib().moe_stream_ctx_prefetch(self._h, int(expert)))

    def last_order(self):
        order = (C.c_int32 * 256)()
        n, ok = C.c_int32(0), C.c_int32(0)
        _check(lib().moe_stream_ctx_last_order(self._h, order, C.byref(n), C.byref(ok)))
        return list(order[:n.value]), bool(ok.value)

    def close(self):
        if self._h:
            lib().moe_stream_ctx_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def moe_layer_forward(cfg, x, W_g, gate_bias, W_packed, sctx: Optional[StreamCtx], y, ws, stream=None) -> None:
    _check(lib().moe_layer_forward(C.byref(cfg), _ptr(x), _ptr(W_g), _ptr(gate_bias), _ptr(W_packed),
                                   sctx.handle if sctx is not None else None, _ptr(y), _ptr(ws), _stream(stream)))


ORDER_ASCENDING, ORDER_GREEDY = 0, 1
GATE_TOPK, GATE_HASH = 0, 1


def moe_schedule_order(counts, tokens_per_load: float, K: int):
    """(order of the non-empty experts, satisfiable) for host token counts; argument marshalling only."""
    E = len(counts)
    c = (C.c_int32 * E)(*[int(v) for v in counts])
    order = (C.c_int32 * E)()
    n, ok = C.c_int32(0), C.c_int32(0)
    _check(lib().moe_schedule_order(c, E, float(tokens_per_load), int(K), order, C.byref(n), C.byref(ok)))
    return list(order[:n.value]), bool(ok.value)


def moe_plan_slots(order, slot_expert, slot_tick, tick: int):
    """(slot_of, load, slot_expert_after, slot_tick_after, tick_after); argument marshalling only."""
    n, K = len(order), len(slot_expert)
    o = (C.c_int32 * max(n, 1))(*[int(v) for v in order])
    se = (C.c_int32 * K)(*[int(v) for v in slot_expert])
    st = (C.c_int64 * K)(*[int(v) for v in slot_tick])
    tk = C.c_int64(int(tick))
    so, ld = (C.c_int32 * max(n, 1))(), (C.c_int32 * max(n, 1))()
    _check(lib().moe_plan_slots(o, n, K, se, st, C.byref(tk), so, ld))
    return list(so[:n]), [bool(v) for v in ld[:n]], list(se), list(st), tk.value


def moe_stream_slots_that_fit(cfg: MoeCfg, reserve_bytes: int = 0) -> int:
    K = C.c_int32(0)
    _check(lib().moe_stream_slots_that_fit(C.byref(cfg), int(reserve_bytes), C.byref(K)))
    return K.value


STAGES = ("route", "permute", "ffn_up", "ffn_down", "combine")
TIME_STAGES, TIME_UP_KERNEL = 0, 1


class Timer:
    """Event timing of resident layer calls (moe_timer_* of the library): all five stages, or the expert
    up-projection kernel alone."""

    def __init__(self, max_calls: int, mode: int = TIME_STAGES):
        self._h = C.c_void_p(None)
        self.mode = mode
        self.max_calls = max_calls
        _check(lib().moe_timer_create(max_calls, mode, C.byref(self._h)))

    @property
    def handle(self):
        return self._h

    def reset(self) -> None:
        _check(lib().moe_timer_reset(self._h))

    def read(self):
        """Per recorded call: {stage: ms} (all stages) or the kernel's ms (up-projection kernel alone)."""
        width = len(STAGES) if self.mode == TIME_STAGES else 1
        buf = (C.c_float * (self.max_calls * width))()
        n = C.c_int32(0)
        _check(lib().moe_timer_read(self._h, buf, self.max_calls, C.byref(n)))
        got = min(n.value, self.max_calls)
        if self.mode == TIME_STAGES:
            return [{s: buf[c * width + i] for i, s in enumerate(STAGES)} for c in range(got)]
        return [buf[c] for c in range(got)]

    def close(self) -> None:
        if self._h:
            lib().moe_timer_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def moe_layer_forward_timed(cfg, x, W_g, gate_bias, W_packed, y, ws, timer: Timer, stream=None) -> None:
    _check(lib().moe_layer_forward_timed(C.byref(cfg), _ptr(x), _ptr(W_g), _ptr(gate_bias), _ptr(W_packed), _ptr(y),
                                         _ptr(ws), _stream(stream), timer.handle))


def _tensor(t, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor):
        raise MoeError(f"{name} must be a tensor (got {type(t).__name__})")
    return t


def _description(cfg, kind, name: str = "cfg"):
    """The description, whose types have to be ones there are."""
    if not isinstance(cfg, kind):
        raise MoeError(f"{name} must be {'an' if kind is AttnCfg else 'a'} {kind.__name__} (got {type(cfg).__name__})")
    for field in ("dtype", "cache_dtype"):
        if getattr(cfg, field, MOE_F32) not in _TORCH:
            raise MoeError(f"{field} must be MOE_F32, MOE_BF16 or MOE_E4M3 (got {getattr(cfg, field)})")
    return cfg


def _array(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, numel: int) -> None:
    """Refuses what is not a contiguous device tensor of this type and size (None is for the library to refuse)."""
    if t is None:
        return
    _tensor(t, name)
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous():
        raise MoeError(f"{name} must be a contiguous {dtype} tensor of {numel} elements (got {t.dtype}, shape {tuple(t.shape)}, "
                       f"strides {t.stride()})")
    if not t.is_cuda:
        raise MoeError(f"{name} must be in device memory")


def _head_rows(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, n: int, heads: int, dim: int) -> None:
    """Refuses what is not [n, heads, dim] in device memory, whose rows may be part of wider ones, each row contiguous."""
    if t is None:
        return
    _tensor(t, name)
    if t.dtype is not dtype or t.shape != (n, heads, dim) or n > 0 and (t.stride(2) != 1 or t.stride(1) != dim and heads != 1):
        raise MoeError(f"{name} must be a {dtype} tensor [{n}, {heads}, {dim}] with contiguous rows (got {t.dtype}, shape "
                       f"{tuple(t.shape)}, strides {t.stride()})")
    if not t.is_cuda:
        raise MoeError(f"{name} must be in device memory")


def _cache(cfg: KvCfg, k_pages, v_pages, k_scales, v_scales) -> None:
    dt, rows = _TORCH[cfg.cache_dtype], cfg.pages * cfg.heads * cfg.page_size
    for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
        _array(t, name, dt, rows * cfg.head_dim)
    for t, name in ((k_scales, "k_scales"), (v_scales, "v_scales")):
        _array(t, name, torch.float32, rows)


def _tokens(slots) -> int:
    if slots is None:
        raise MoeError("slots is NULL")
    return _tensor(slots, "slots").numel()


def _refused(name: str):
    raise MoeError(f"{name}: an argument is not as its description says")


def moe_add_norm(cfg: NormCfg, x, residual, weight, sum, y, q=None, q_scale=None, stream=None) -> None:
    if _native("add_norm", cfg, x, residual, weight, sum, y, q, q_scale, stream=stream):
        return
    dt, n = _TORCH[_description(cfg, NormCfg).dtype], cfg.T * cfg.d
    for t, name, numel in ((x, "x", n), (residual, "residual", n), (weight, "weight", cfg.d), (sum, "sum", n), (y, "y", n)):
        _array(t, name, dt, numel)
    _array(q, "q", torch.float8_e4m3fn, n)
    _array(q_scale, "q_scale", torch.float32, cfg.T * (cfg.d // cfg.q_group if cfg.q_group > 0 else 1))
    _refused("moe_add_norm")


def _kv_refused(name: str, cfg: KvCfg, k, v, slots, cache) -> None:
    dt, n = _TORCH[_description(cfg, KvCfg).dtype], _tokens(slots)
    _head_rows(k, "k", dt, n, cfg.heads, cfg.head_dim)
    _head_rows(v, "v", dt, n, cfg.heads, cfg.head_dim)
    _cache(cfg, *cache)
    _array(slots, "slots", torch.int32, n)
    _refused(name)


def moe_kv_write(cfg: KvCfg, k, v, slots, k_pages, v_pages, k_scales=None, v_scales=None, stream=None) -> None:
    if not _native("kv_write", cfg, k, v, slots, k_pages, v_pages, k_scales, v_scales, stream=stream):
        _kv_refused("moe_kv_write", cfg, k, v, slots, (k_pages, v_pages, k_scales, v_scales))


def moe_kv_read(cfg: KvCfg, k_pages, v_pages, k_scales, v_scales, slots, k, v, stream=None) -> None:
    if not _native("kv_read", cfg, k_pages, v_pages, k_scales, v_scales, slots, k, v, stream=stream):
        _kv_refused("moe_kv_read", cfg, k, v, slots, (k_pages, v_pages, k_scales, v_scales))


def moe_attn_workspace_bytes(cfg: KvCfg, attn: AttnCfg) -> int:
    n = C.c_size_t(0)
    _check(lib().moe_attn_workspace_bytes(C.addressof(cfg), C.addressof(attn), C.byref(n)))
    return n.value


def moe_attn_decode(cfg: KvCfg, attn: AttnCfg, q, k_pages, v_pages, k_scales, v_scales, table, lens, out, lse, ws, stream=None) -> None:
    if _native("attn_decode", cfg, attn, q, k_pages, v_pages, k_scales, v_scales, table, lens, out, lse, ws,
               stream=stream):
        return
    dt = _TORCH[_description(cfg, KvCfg).dtype]
    B, heads = _description(attn, AttnCfg, "attn").B, attn.q_heads
    _head_rows(q, "q", dt, B, heads, cfg.head_dim)
    _workspace(ws, lambda: moe_attn_workspace_bytes(cfg, attn), "moe_attn_workspace_bytes")
    _cache(cfg, k_pages, v_pages, k_scales, v_scales)
    _array(table, "table", torch.int32, B * attn.table_pages)
    _array(lens, "lens", torch.int32, B)
    _array(out, "out", dt, B * heads * cfg.head_dim)
    _array(lse, "lse", torch.float32, B * heads)
    _refused("moe_attn_decode")


def _workspace(ws, need, what: str) -> None:
    if ws is None:
        return
    if _tensor(ws, "ws").nbytes < need():
        raise MoeError(f"ws is smaller than {what}")
    if not ws.is_contiguous():
        raise MoeError("ws must be contiguous")
    if not ws.is_cuda:
        raise MoeError("ws must be in device memory")


def _scores(scores: Optional[ScoresCfg], heads: int, slopes, bias) -> None:
    if scores is not None:
        _description(scores, ScoresCfg, "scores")
    distances = 1 if scores is None else scores.back + scores.ahead + 1
    _array(slopes, "slopes", torch.float32, heads)
    _array(bias, "bias", torch.float32, heads * distances)


def _here(*tensors) -> None:
    """Refuses tensors of another device than the current one, whose stream the call is put on."""
    for t in tensors:
        if t is not None and t.is_cuda and t.device.index != torch.cuda.current_device():
            raise MoeError(f"a tensor is on {t.device}, the current device is {torch.cuda.current_device()}")


def moe_attn_decode_scored(cfg: KvCfg, attn: AttnCfg, scores: Optional[ScoresCfg], q, k_pages, v_pages, k_scales, v_scales, table, lens, slopes,
                           bias, out, lse, ws, stream=None) -> None:
    if _native("attn_decode_scored", cfg, attn, scores, q, k_pages, v_pages, k_scales, v_scales, table, lens, slopes, bias, out, lse, ws,
               stream=stream):
        return
    dt = _TORCH[_description(cfg, KvCfg).dtype]
    B, heads = _description(attn, AttnCfg, "attn").B, attn.q_heads
    _scores(scores, heads, slopes, bias)
    _head_rows(q, "q", dt, B, heads, cfg.head_dim)
    _workspace(ws, lambda: moe_attn_workspace_bytes(cfg, attn), "moe_attn_workspace_bytes")
    _cache(cfg, k_pages, v_pages, k_scales, v_scales)
    _array(table, "table", torch.int32, B * attn.table_pages)
    _array(lens, "lens", torch.int32, B)
    _array(out, "out", dt, B * heads * cfg.head_dim)
    _array(lse, "lse", torch.float32, B * heads)
    _here(q, k_pages, v_pages, k_scales, v_scales, table, lens, slopes, bias, out, lse, ws)
    _refused("moe_attn_decode_scored")


def moe_attn_prompt_workspace_bytes(cfg: KvCfg, prompt: PromptCfg) -> int:
    n = C.c_size_t(0)
    _check(lib().moe_attn_prompt_workspace_bytes(C.addressof(cfg), C.addressof(prompt), C.byref(n)))
    return n.value


def moe_attn_prompt(cfg: KvCfg, prompt: PromptCfg, scores: Optional[ScoresCfg], q, k_pages, v_pages, k_scales, v_scales, table, lens, starts,
                    first, end, slopes, bias, out, lse, ws, stream=None) -> None:
    if _native("attn_prompt", cfg, prompt, scores, q, k_pages, v_pages, k_scales, v_scales, table, lens, starts, first, end, slopes, bias, out, lse,
               ws, stream=stream):
        return
    dt = _TORCH[_description(cfg, KvCfg).dtype]
    n, heads = _description(prompt, PromptCfg, "prompt").tokens, prompt.q_heads
    _scores(scores, heads, slopes, bias)
    _head_rows(q, "q", dt, n, heads, cfg.head_dim)
    _workspace(ws, lambda: moe_attn_prompt_workspace_bytes(cfg, prompt), "moe_attn_prompt_workspace_bytes")
    _cache(cfg, k_pages, v_pages, k_scales, v_scales)
    for t, name, numel in ((table, "table", prompt.B * prompt.table_pages), (lens, "lens", prompt.B), (starts, "starts", prompt.B + 1),
                           (first, "first", n), (end, "end", n)):
        _array(t, name, torch.int32, numel)
    _array(out, "out", dt, n * heads * cfg.head_dim)
    _array(lse, "lse", torch.float32, n * heads)
    _here(q, k_pages, v_pages, k_scales, v_scales, table, lens, starts, first, end, slopes, bias, out, lse, ws)
    _refused("moe_attn_prompt")


def moe_rope_frequencies(cfg: RopeCfg) -> torch.Tensor:
    """Radians per position of each pair, fp64, in host memory; moe_rope takes them from device memory."""
    freqs = torch.empty(max(_description(cfg, RopeCfg).rot_dim, 0) // 2, dtype=torch.float64)
    _check(lib().moe_rope_frequencies(C.addressof(cfg), freqs.data_ptr()))
    return freqs


def moe_rope(cfg: RopeCfg, positions, freqs, q, q_out, k=None, k_out=None, stream=None) -> None:
    if _native("rope", cfg, positions, freqs, q, q_out, k, k_out, stream=stream):
        return
    dt = _TORCH[_description(cfg, RopeCfg).dtype]
    if positions is None:
        raise MoeError("positions is NULL")
    n = _tensor(positions, "positions").numel()
    for t, name, heads in ((q, "q", cfg.q_heads), (q_out, "q_out", cfg.q_heads), (k, "k", cfg.k_heads), (k_out, "k_out", cfg.k_heads)):
        _head_rows(t, name, dt, n, heads, cfg.head_dim)
    _array(freqs, "freqs", torch.float64, cfg.rot_dim // 2)
    _array(positions, "positions", torch.int32, n)
    _here(positions, freqs, q, q_out, k, k_out)
    _refused("moe_rope")
