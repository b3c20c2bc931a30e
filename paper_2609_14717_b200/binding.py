"""ctypes binding of libcod.so (the C ABI declared in include/cod.h).

Argument marshalling only: every step of the round runs in the library's CUDA kernels.
torch is used for device memory and the current stream.  If the compiled library is
missing the import of this module fails — there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcod.so")

COD_F32, COD_BF16 = 0, 1
COD_CARRY, COD_BASELINE = 0, 1
COD_F_HIDDEN_NORM = 1
COD_F_NO_TENSOR_CORES = 2
COD_F_ATTN_ONE_ITEM_CTAS = 32
COD_F_ATTN_PERSISTENT = 64
COD_F_QK_NORM = 4
COD_F_NO_CARRY_EMBED = 8
COD_F_REJ_PROJECTOR = 16
COD_F_KV8 = 128
DEV_BAD_TOKEN, DEV_PAGE_OVERFLOW, DEV_BAD_PAGE, DEV_TIMEOUT, DEV_BAD_LEN = 1, 2, 4, 8, 16
DEV_NO_PAGES, DEV_BAD_SLOT = 32, 64

EXPORTS = ("cod_create", "cod_destroy", "cod_set_weights", "cod_verify_accept", "cod_project_kv",
           "cod_scatter_kv", "cod_block_attn", "cod_lm_head_argmax", "cod_lm_head_argmax_static",
           "cod_draft_round", "cod_reconvergence_count", "cod_verify_accept_stochastic",
           "cod_draft_round_stochastic", "cod_lm_head_sample", "cod_lm_head_rank",
           "cod_kv_append", "cod_pages_reserve", "cod_pages_release",
           "cod_poll_status", "cod_set_wait_limit", "cod_selftest_expire_wait",
           "cod_profile_enable", "cod_profile_read", "cod_launch_count",
           "cod_workspace_bytes", "cod_error_string")
KERNEL_CLASSES = ("verify", "fc", "kv", "qkv", "attn", "oproj", "lmhead", "rowops", "mlp")


class CodConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "d_target", "n_cap", "d_model", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "vocab",
        "mask_token_id", "block", "page_size", "max_batch", "max_pages_per_seq", "n_pages", "dtype")] + [
        ("flags", C.c_uint32), ("rope_theta", C.c_float), ("rms_eps", C.c_float),
        ("attn_split_len", C.c_int32), ("d_ff", C.c_int32), ("carry_rounds", C.c_int32)]


_WEIGHT_FIELDS = ("fc", "e_carry", "g_hidden", "wk", "wv", "wq", "wo", "g_attn", "g_final", "emb",
                  "w_gate", "w_up", "w_down", "g_mlp", "g_qnorm", "g_knorm",   # these six: complete layer only
                  "fc_rej")                                                     # separate-projector variant only
_SPLIT_FIELDS = ("accept_len", "bonus", "row_pos", "commit_slot", "carry_slot", "acc_rows", "acc_off",
                 "rej_rows", "rej_off")
_STATE_FIELDS = ("kv_pool", "block_table", "committed_len", "carry_kv", "carry_len", "carry_hist", "kv_scale")
_PAGES_FIELDS = ("free_list", "n_free", "held")
_PLAN_FIELDS = ("row_off", "slot", "row_pos", "row_seq")
_TAP_FIELDS = ("z", "attn_out", "x_final", "top_logit", "carry_mass")


class CodWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _WEIGHT_FIELDS]


class CodState(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _STATE_FIELDS]


class CodSplit(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _SPLIT_FIELDS]


class CodPages(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _PAGES_FIELDS]


class CodRowPlan(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _PLAN_FIELDS] + [("max_rows", C.c_int32)]


class CodTaps(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _TAP_FIELDS]


def load_library() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
    lib.cod_create.argtypes = [C.POINTER(CodConfig), C.POINTER(vp)]
    lib.cod_destroy.argtypes = [vp]
    lib.cod_set_weights.argtypes = [vp, C.POINTER(CodWeights), vp]
    lib.cod_verify_accept.argtypes = [vp, vp, vp, i32, i32, C.POINTER(CodState), C.POINTER(CodSplit), vp]
    lib.cod_project_kv.argtypes = [vp, vp, C.POINTER(CodSplit), i32, i32, vp, vp]
    lib.cod_scatter_kv.argtypes = [vp, vp, C.POINTER(CodSplit), i32, i32, C.POINTER(CodState), vp]
    lib.cod_block_attn.argtypes = [vp, i32, vp, vp, vp, C.POINTER(CodState), i32, i32, vp, vp, vp]
    lib.cod_lm_head_argmax.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.cod_lm_head_argmax_static.argtypes = [vp, vp, vp, i32, i32, i32, i32, C.c_float, vp, vp, vp]
    lib.cod_draft_round.argtypes = [vp, vp, vp, vp, i32, i32, i32, C.POINTER(CodState), C.POINTER(CodSplit),
                                    vp, C.POINTER(CodTaps), vp]
    lib.cod_reconvergence_count.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.cod_lm_head_sample.argtypes = [vp, vp, i32, C.c_uint64, C.c_uint32, vp, vp, vp, vp]
    lib.cod_lm_head_rank.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    lib.cod_verify_accept_stochastic.argtypes = [vp, vp, vp, vp, vp, i32, i32, C.POINTER(CodState), C.POINTER(CodSplit), vp]
    lib.cod_draft_round_stochastic.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, C.POINTER(CodState),
                                               C.POINTER(CodSplit), vp, C.POINTER(CodTaps), vp, C.c_uint64,
                                               C.c_uint32, vp]
    lib.cod_kv_append.argtypes = [vp, vp, vp, i32, C.POINTER(CodState), vp]
    lib.cod_pages_reserve.argtypes = [vp, C.POINTER(CodPages), vp, i32, C.POINTER(CodState), C.POINTER(CodRowPlan), i32, vp]
    lib.cod_pages_release.argtypes = [vp, C.POINTER(CodPages), vp, i32, C.POINTER(CodState), vp]
    lib.cod_poll_status.argtypes = [vp, C.POINTER(C.c_uint32), i32, vp]
    lib.cod_profile_enable.argtypes = [vp, C.c_uint32]
    lib.cod_profile_read.argtypes = [vp, i32, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.cod_launch_count.argtypes = [vp]
    lib.cod_launch_count.restype = i64
    lib.cod_workspace_bytes.argtypes = [vp]
    lib.cod_workspace_bytes.restype = i64
    lib.cod_error_string.argtypes = [i32]
    lib.cod_error_string.restype = C.c_char_p
    for name in EXPORTS[:-3]:
        getattr(lib, name).restype = i32
    return lib


_LIB: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    global _LIB
    if _LIB is None:
        _LIB = load_library()
    return _LIB


class CodError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {lib().cod_error_string(status).decode()} ({status})")


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise CodError(fn, status)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    return t.data_ptr()


def _want(name: str, t: torch.Tensor, dtype: str, shape) -> None:
    """The library sees only an address: a tensor of another type or size must not get that far."""
    td = torch.int32 if dtype == "i32" else torch_dtype(dtype)
    if t.dtype != td or t.shape != shape:
        raise ValueError(f"{name}: expected {td} {shape}, got {t.dtype} {tuple(t.shape)}")


def _arg(name: str, t: Optional[torch.Tensor], n: int, dtype: torch.dtype, device: int) -> Optional[int]:
    """Address of a tensor that holds at least the n elements which the call reaches, on the context's device."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected at least {n} contiguous elements of {dtype} on device {device}, "
                         f"got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


_I32 = torch.int32


class _Sizes:
    """What a configuration says about its tensors, as plain numbers (a ctypes field costs a call of a few us 0.1 us per read)."""
    __slots__ = ("device", "batch", "width", "rounds", "n_pages", "pool", "pool_dtype", "scales")

    def __init__(self, cfg: CodConfig, device: int):
        self.device, self.batch, self.width, self.n_pages = device, cfg.max_batch, cfg.max_pages_per_seq, cfg.n_pages
        self.rounds = max(1, cfg.carry_rounds)
        self.scales = cfg.n_layers * cfg.n_pages * cfg.n_kv_heads * 2
        self.pool = self.scales * cfg.page_size * cfg.head_dim
        self.pool_dtype = (torch.float8_e4m3fn if cfg.flags & COD_F_KV8 else torch.bfloat16 if cfg.dtype == COD_BF16 else torch.float32)


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def torch_dtype(dtype: str):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def to_device(a: np.ndarray, dtype: str, device="cuda") -> torch.Tensor:
    """Host float32 array (already holding storage-exact values) -> device tensor of the storage type."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=torch_dtype(dtype))


class Split:
    """Device arrays cod_verify_accept fills."""

    def __init__(self, S: int, W: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.accept_len = torch.zeros(S, **i32)
        self.bonus = torch.zeros(S, **i32)
        self.row_pos = torch.zeros(S * W, **i32)
        self.commit_slot = torch.zeros(S * W, **i32)
        self.carry_slot = torch.zeros(S * W, **i32)
        self.acc_rows = torch.zeros(S * W, **i32)
        self.acc_off = torch.zeros(S + 1, **i32)
        self.rej_rows = torch.zeros(S * W, **i32)
        self.rej_off = torch.zeros(S + 1, **i32)

    def struct(self) -> CodSplit:
        return CodSplit(*[_ptr(getattr(self, n)) for n in _SPLIT_FIELDS])

    def to_host(self) -> Dict[str, np.ndarray]:
        return {n: getattr(self, n).cpu().numpy() for n in _SPLIT_FIELDS}


class State:
    """Paged committed KV, block table, carry slot and lengths of one batch (device tensors).

    block_table and committed_len: host arrays, or device tensors, which are used as they are. Tensors that the caller has
    already (a pool, scales, carry slots) are used in the place of new ones, which start as zeros."""

    def __init__(self, cfg: CodConfig, dtype: str, S: int, block_table, committed_len, device="cuda",
                 kv_pool: Optional[torch.Tensor] = None, kv_scale: Optional[torch.Tensor] = None,
                 carry_kv: Optional[torch.Tensor] = None, carry_len: Optional[torch.Tensor] = None,
                 carry_hist: Optional[torch.Tensor] = None):
        td = torch_dtype(dtype)
        self.S = S
        kv8 = bool(cfg.flags & COD_F_KV8)                       # committed cache in e4m3 with one scale per page, head, K|V
        k = max(1, int(cfg.carry_rounds))                       # rounds of rejected rows the carry slot holds

        def take(name, given, shape, dt):
            if given is None:
                return torch.zeros(shape, dtype=dt, device=device)
            if given.dtype != dt or given.shape != shape:
                raise ValueError(f"{name}: expected {dt} {shape}, got {given.dtype} {tuple(given.shape)}")
            return given

        def table(name, a, shape):
            if isinstance(a, torch.Tensor) and a.is_cuda:
                return take(name, a, shape, torch.int32)
            return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(device)

        self.kv_pool = take("kv_pool", kv_pool, (cfg.n_layers, cfg.n_pages, cfg.n_kv_heads, 2, cfg.page_size, cfg.head_dim),
                            torch.float8_e4m3fn if kv8 else td)
        self.kv_scale = take("kv_scale", kv_scale, (cfg.n_layers, cfg.n_pages, cfg.n_kv_heads, 2), torch.float32) if kv8 else None
        self.block_table = table("block_table", block_table, (S, cfg.max_pages_per_seq))
        self.committed_len = table("committed_len", committed_len, (S,))
        self.carry_kv = take("carry_kv", carry_kv, (cfg.n_layers, cfg.max_batch, cfg.n_kv_heads, 2, k * cfg.block, cfg.head_dim), td)
        self.carry_len = take("carry_len", carry_len, (S,), torch.int32)
        self.carry_hist = take("carry_hist", carry_hist, (S, k), torch.int32) if k > 1 else None

    def struct(self) -> CodState:
        return CodState(*[_ptr(getattr(self, n)) for n in _STATE_FIELDS])

    def cache_struct(self, sizes: _Sizes) -> CodState:
        """The fields that cod_kv_append reads (marshalling a tensor costs the host some 0.4 us, a small append's kernel takes 4)."""
        return CodState(_arg("kv_pool", self.kv_pool, sizes.pool, sizes.pool_dtype, sizes.device), None, None, None, None, None,
                        _arg("kv_scale", self.kv_scale, sizes.scales, torch.float32, sizes.device))

    def table_struct(self, sizes: _Sizes, S: int) -> CodState:
        """The fields that cod_pages_reserve and cod_pages_release read and write."""
        dev, width = sizes.device, sizes.width
        if self.block_table.shape[-1] != width:
            raise ValueError(f"block_table: expected rows of {width}, got {tuple(self.block_table.shape)}")
        return CodState(None, _arg("block_table", self.block_table, S * width, _I32, dev), _arg("committed_len", self.committed_len, S, _I32, dev),
                        None, _arg("carry_len", self.carry_len, S, _I32, dev), _arg("carry_hist", self.carry_hist, S * sizes.rounds, _I32, dev))


class Pages:
    """Free list of the pool's pages and pages held per sequence (device). Without arguments: everything is free."""

    def __init__(self, cfg: CodConfig, S: int, free_list: Optional[torch.Tensor] = None,
                 n_free: Optional[torch.Tensor] = None, held: Optional[torch.Tensor] = None, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.free_list = free_list if free_list is not None else torch.arange(cfg.n_pages - 1, -1, -1, **i32)
        self.n_free = n_free if n_free is not None else torch.full((1,), cfg.n_pages, **i32)
        self.held = held if held is not None else torch.zeros(S, **i32)

    def struct(self, sizes: _Sizes, S: int) -> CodPages:
        dev = sizes.device
        return CodPages(_arg("free_list", self.free_list, sizes.n_pages, _I32, dev), _arg("n_free", self.n_free, 1, _I32, dev),
                        _arg("held", self.held, S, _I32, dev))


class RowPlan:
    """Slots, positions and sequences of a step's new rows, filled by Context.pages_reserve (device)."""

    def __init__(self, S: int, max_rows: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.max_rows = max_rows
        self.row_off = torch.zeros(S + 1, **i32)
        self.slot = torch.full((max_rows,), -1, **i32)
        self.row_pos = torch.full((max_rows,), -1, **i32)
        self.row_seq = torch.full((max_rows,), -1, **i32)

    def struct(self, sizes: _Sizes, S: int) -> CodRowPlan:
        dev, n = sizes.device, self.max_rows
        return CodRowPlan(_arg("row_off", self.row_off, S + 1, _I32, dev), _arg("slot", self.slot, n, _I32, dev),
                          _arg("row_pos", self.row_pos, n, _I32, dev), _arg("row_seq", self.row_seq, n, _I32, dev), n)


class Taps:
    def __init__(self, cfg: CodConfig, S: int, device="cuda"):
        R = S * cfg.block
        f32 = dict(dtype=torch.float32, device=device)
        self.z = torch.zeros((R, cfg.d_model), **f32)
        self.attn_out = torch.zeros((cfg.n_layers, R, cfg.n_q_heads * cfg.head_dim), **f32)
        self.x_final = torch.zeros((R, cfg.d_model), **f32)
        self.top_logit = torch.zeros(R, **f32)
        self.carry_mass = torch.zeros((cfg.n_layers, S, cfg.block, cfg.n_q_heads), **f32)

    def struct(self) -> CodTaps:
        return CodTaps(*[_ptr(getattr(self, n)) for n in _TAP_FIELDS])


class Context:
    """Owns a cod_ctx on the current CUDA device; methods mirror the C entry points."""

    def __init__(self, cfg: CodConfig):
        if not torch.cuda.is_available():
            raise RuntimeError("the Carryover drafting library needs a CUDA device (no CPU fallback)")
        torch.cuda.init()
        torch.zeros(1, device="cuda")          # make sure the primary context exists
        self.cfg = cfg
        self.dtype = "bf16" if cfg.dtype == COD_BF16 else "f32"
        self._sizes = _Sizes(cfg, torch.cuda.current_device())
        self._h = C.c_void_p()
        _check("cod_create", lib().cod_create(C.byref(cfg), C.byref(self._h)))
        self._weights = None

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().cod_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- set-up
    def set_weights(self, w: Dict[str, torch.Tensor]) -> None:
        self._weights = {k: w[k] for k in _WEIGHT_FIELDS if k in w}      # keep the tensors alive
        ws = CodWeights(*[_ptr(self._weights.get(k)) for k in _WEIGHT_FIELDS])
        _check("cod_set_weights", lib().cod_set_weights(self._h, C.byref(ws), _stream()))

    # ---- the five parts
    def verify_accept(self, draft, target, S, n_forced, state: State, split: Split) -> None:
        st, sp = state.struct(), split.struct()
        _check("cod_verify_accept", lib().cod_verify_accept(self._h, _ptr(draft), _ptr(target), S, n_forced,
                                                            C.byref(st), C.byref(sp), _stream()))

    def project_kv(self, H, split: Split, S, mode, J) -> None:
        sp = split.struct()
        _check("cod_project_kv", lib().cod_project_kv(self._h, _ptr(H), C.byref(sp), S, mode, _ptr(J), _stream()))

    def scatter_kv(self, J, split: Split, S, mode, state: State) -> None:
        st, sp = state.struct(), split.struct()
        _check("cod_scatter_kv", lib().cod_scatter_kv(self._h, _ptr(J), C.byref(sp), S, mode, C.byref(st), _stream()))

    def kv_append(self, J, slot, state: State) -> None:
        """J [Ld, n_rows, 2, n_kv, hd] into the committed cache at slot [n_rows] (-1: nowhere)."""
        sz, n = self._sizes, slot.numel()
        _want("J", J, self.dtype, (self.cfg.n_layers, n, 2, self.cfg.n_kv_heads, self.cfg.head_dim))
        _check("cod_kv_append", lib().cod_kv_append(self._h, _arg("J", J, 0, J.dtype, sz.device), _arg("slot", slot, n, _I32, sz.device), n,
                                                    state.cache_struct(sz), _stream()))

    def pages_reserve(self, pages: Pages, n_new, state: State, S, plan: Optional[RowPlan] = None,
                      advance: bool = False) -> None:
        """Pages for n_new [S] more tokens per sequence; plan: where their rows go; advance: the lengths grow too."""
        sz = self._sizes
        n = S if S <= sz.batch else sz.batch                    # (a larger S is refused by the library)
        if n_new.numel() != S:
            raise ValueError(f"n_new: expected {S} elements, got {tuple(n_new.shape)}")
        _check("cod_pages_reserve", lib().cod_pages_reserve(
            self._h, pages.struct(sz, n), _arg("n_new", n_new, S, _I32, sz.device), S, state.table_struct(sz, n),
            plan.struct(sz, n) if plan is not None else None, int(advance), _stream()))

    def pages_release(self, pages: Pages, keep, state: State, S) -> None:
        """Pages behind the first keep [S] tokens back to the free list (keep None: behind the committed ones)."""
        sz = self._sizes
        n = S if S <= sz.batch else sz.batch
        if keep is not None and keep.numel() != S:
            raise ValueError(f"keep: expected {S} elements, got {tuple(keep.shape)}")
        _check("cod_pages_release", lib().cod_pages_release(
            self._h, pages.struct(sz, n), _arg("keep", keep, S, _I32, sz.device), S, state.table_struct(sz, n), _stream()))

    def block_attn(self, layer, q, k_blk, v_blk, state: State, S, use_carry, out, carry_mass=None) -> None:
        st = state.struct()
        _check("cod_block_attn", lib().cod_block_attn(self._h, layer, _ptr(q), _ptr(k_blk), _ptr(v_blk), C.byref(st),
                                                      S, int(use_carry), _ptr(out), _ptr(carry_mass), _stream()))

    def lm_head_argmax(self, x, n_rows, tok, top_logit=None) -> None:
        _check("cod_lm_head_argmax", lib().cod_lm_head_argmax(self._h, _ptr(x), n_rows, _ptr(tok), _ptr(top_logit),
                                                              _stream()))

    def draft_round(self, draft, target, H, S, n_forced, mode, state: State, split: Optional[Split], next_draft,
                    taps: Optional[Taps] = None) -> None:
        st = state.struct()
        sp = split.struct() if split is not None else None
        tp = taps.struct() if taps is not None else None
        _check("cod_draft_round", lib().cod_draft_round(
            self._h, _ptr(draft), _ptr(target), _ptr(H), S, n_forced, mode, C.byref(st),
            C.byref(sp) if sp is not None else None, _ptr(next_draft),
            C.byref(tp) if tp is not None else None, _stream()))

    def verify_accept_stochastic(self, target, p_tok, q_tok, u, S, n_forced, state: State, split: Split) -> None:
        st, sp = state.struct(), split.struct()
        _check("cod_verify_accept_stochastic", lib().cod_verify_accept_stochastic(
            self._h, _ptr(target), _ptr(p_tok), _ptr(q_tok), _ptr(u), S, n_forced, C.byref(st), C.byref(sp), _stream()))

    def draft_round_stochastic(self, target, p_tok, q_tok, u, H, S, n_forced, mode, state: State,
                               split: Optional[Split], next_draft, taps: Optional[Taps] = None,
                               q_next=None, seed: int = 0, step: int = 0) -> None:
        st = state.struct()
        sp = split.struct() if split is not None else None
        tp = taps.struct() if taps is not None else None
        _check("cod_draft_round_stochastic", lib().cod_draft_round_stochastic(
            self._h, _ptr(target), _ptr(p_tok), _ptr(q_tok), _ptr(u), _ptr(H), S, n_forced, mode, C.byref(st),
            C.byref(sp) if sp is not None else None, _ptr(next_draft),
            C.byref(tp) if tp is not None else None, _ptr(q_next), seed, step, _stream()))

    def lm_head_sample(self, x, n_rows, seed, step, tok, q_tok=None, lse=None) -> None:
        _check("cod_lm_head_sample", lib().cod_lm_head_sample(
            self._h, _ptr(x), n_rows, seed, step, _ptr(tok), _ptr(q_tok), _ptr(lse), _stream()))

    def lm_head_rank(self, x, n_rows, ref_tok, rank, ref_logit=None) -> None:
        _check("cod_lm_head_rank", lib().cod_lm_head_rank(
            self._h, _ptr(x), n_rows, _ptr(ref_tok), _ptr(rank), _ptr(ref_logit), _stream()))

    def reconvergence_count(self, z, y, length, S, out) -> None:
        _check("cod_reconvergence_count", lib().cod_reconvergence_count(
            self._h, _ptr(z), _ptr(y), _ptr(length), S, _ptr(out), _stream()))

    # ---- bookkeeping
    def poll_status(self, clear: bool = True) -> int:
        flags = C.c_uint32(0)
        _check("cod_poll_status", lib().cod_poll_status(self._h, C.byref(flags), int(clear), _stream()))
        return int(flags.value)

    def set_wait_limit(self, sm_cycles: int) -> None:
        """Bound of the device-side waits of the weight-streaming contraction, in SM cycles (0: built-in)."""
        _check("cod_set_wait_limit", lib().cod_set_wait_limit(self._h, C.c_longlong(sm_cycles)))

    def selftest_expire_wait(self, on: bool) -> None:
        """While on, that kernel requests no operands: its waits run out and raise COD_DEV_TIMEOUT."""
        _check("cod_selftest_expire_wait", lib().cod_selftest_expire_wait(self._h, int(bool(on))))

    def profile_enable(self, classes=()) -> None:
        mask = 0
        for k in classes:
            mask |= 1 << KERNEL_CLASSES.index(k)
        _check("cod_profile_enable", lib().cod_profile_enable(self._h, mask))

    def profile_read(self, klass: str):
        ms, n = C.c_float(0), C.c_int32(0)
        _check("cod_profile_read", lib().cod_profile_read(self._h, KERNEL_CLASSES.index(klass), C.byref(ms), C.byref(n)))
        return float(ms.value), int(n.value)

    def launch_count(self) -> int:
        return int(lib().cod_launch_count(self._h))

    def workspace_bytes(self) -> int:
        return int(lib().cod_workspace_bytes(self._h))


def lm_head_argmax_static(emb: torch.Tensor, g_final: torch.Tensor, x: torch.Tensor, tok: torch.Tensor,
                          top_logit: Optional[torch.Tensor], rms_eps: float) -> None:
    """cod_lm_head_argmax_static: the LM-head argmax for callers that may not allocate device memory.

    Needs no Context. The scratch is a fixed array inside the library (rows <= 64, width <= 8192);
    calls that overlap on the GPU race on it, and the first call on a device should precede any
    stream capture."""
    n_rows, d_model = x.shape
    dtype = COD_BF16 if emb.dtype == torch.bfloat16 else COD_F32
    _check("cod_lm_head_argmax_static", lib().cod_lm_head_argmax_static(
        _ptr(emb), _ptr(g_final), _ptr(x), n_rows, d_model, emb.shape[0], dtype, C.c_float(rms_eps),
        _ptr(tok), _ptr(top_logit), _stream()))


def make_config(sh, max_batch: int, max_pages_per_seq: int, n_pages: int, attn_split_len: int = 0,
                no_tensor_cores: bool = False, extra_flags: int = 0) -> CodConfig:
    """cod_config from a synthetic DrafterShape."""
    return CodConfig(
        d_target=sh.d_target, n_cap=sh.n_cap, d_model=sh.d_model, n_layers=sh.n_layers, n_q_heads=sh.n_q,
        n_kv_heads=sh.n_kv, head_dim=sh.hd, vocab=sh.vocab, mask_token_id=sh.mask_token_id, block=sh.W,
        page_size=sh.page, max_batch=max_batch, max_pages_per_seq=max_pages_per_seq, n_pages=n_pages,
        dtype=COD_BF16 if sh.dtype == "bf16" else COD_F32,
        flags=extra_flags | (COD_F_HIDDEN_NORM if sh.hidden_norm else 0) | (COD_F_NO_TENSOR_CORES if no_tensor_cores else 0)
        | (COD_F_QK_NORM if sh.qk_norm else 0) | (COD_F_KV8 if sh.kv8 else 0)
        | {"embedding": 0, "none": COD_F_NO_CARRY_EMBED, "projector": COD_F_REJ_PROJECTOR}[sh.carry_variant],
        rope_theta=sh.rope_theta, rms_eps=sh.rms_eps,
        attn_split_len=attn_split_len, d_ff=sh.d_ff, carry_rounds=sh.carry_rounds)


def weights_to_device(w: Dict[str, np.ndarray], dtype: str) -> Dict[str, torch.Tensor]:
    return {k: to_device(v, dtype) for k, v in w.items()}
