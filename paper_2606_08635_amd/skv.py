"""ctypes binding over ``libskv.so`` (the C ABI of ``include/skv.h``).

Argument marshalling only: every function checks that the torch tensors it is
given have the dtype, device and size the configuration implies (the C library
cannot see device buffer sizes), passes their ``data_ptr()`` and the current
HIP stream, and raises ``SkvError`` on a nonzero status.  All work, the codec's and
that of the attention and page operators (``attn_*``, ``pages_*``), runs in the
library's HIP kernels; there is no fallback.  If ``libskv.so`` has not
been built, the first call raises.
"""
import ctypes
import os
import struct
from typing import Optional

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libskv.so")

OK, ERR_INVALID_ARG, ERR_BUDGET, ERR_CAPACITY, ERR_FORMAT, ERR_DEVICE = range(6)
FP16, INT8, INT4, DROP = 0, 1, 2, 3
KVNORM, ATTN, RECENCY = 0, 1, 2
UPGRADE_FP16, UPGRADE_RESIDUAL8 = 0, 1
GROUP_TOKEN, GROUP_LAYER, GROUP_HEAD = 0, 1, 2
QUANT_GROUP64, QUANT_GROUP32, QUANT_ASYM, QUANT_FP16, QUANT_CHANNEL = 1, 2, 4, 8, 16
ABI_VERSION = 2
STATIC_SCRATCH_BYTES = 48 << 20  # SKV_STATIC_SCRATCH_BYTES

EXPORTED = ("skv_abi_version", "skv_status_string", "skv_plan_tiers", "skv_payload_size",
            "skv_workspace_size", "skv_prepare", "skv_score", "skv_score_static", "skv_assign_tiers", "skv_pack",
            "skv_unpack", "skv_pack_batch", "skv_unpack_batch", "skv_link", "skv_upgrade_size",
            "skv_pack_upgrade", "skv_unpack_upgrade", "skv_group_count", "skv_plan_groups",
            "skv_grouped_payload_size", "skv_group_workspace_size", "skv_prepare_groups", "skv_score_groups",
            "skv_assign_groups", "skv_pack_groups", "skv_unpack_groups", "skv_batch_workspace_size",
            "skv_score_batch", "skv_assign_batch", "skv_attn_prompt_workspace_size", "skv_attn_prompt",
            "skv_attn_decode_workspace_size", "skv_attn_decode", "skv_pages_workspace_size", "skv_pages_reserve",
            "skv_pages_fork", "skv_pages_compact", "skv_pages_free", "skv_pages_copy")
DTYPE_F16, DTYPE_BF16 = 0, 1


class SkvError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} (status {status})")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("num_tokens", ctypes.c_int32),
                ("budget", ctypes.c_float), ("first_ratio", ctypes.c_float),
                ("num_sink", ctypes.c_int32), ("decay", ctypes.c_float),
                ("num_tiers", ctypes.c_int32), ("score_mode", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("obs_window", ctypes.c_int32),
                ("quant_int8", ctypes.c_int32), ("quant_int4", ctypes.c_int32)]


class Request(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("tier", ctypes.c_void_p), ("payload", ctypes.c_void_p),
                ("payload_bytes", ctypes.c_uint64), ("block_table", ctypes.c_void_p),
                ("dev_status", ctypes.c_void_p)]


class ScoreRequest(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("score", ctypes.c_void_p), ("tier", ctypes.c_void_p)]


class GroupSpec(ctypes.Structure):
    _fields_ = [("granularity", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("budgets", ctypes.POINTER(ctypes.c_float))]


class Plan(ctypes.Structure):
    _fields_ = [("n_sink", ctypes.c_int32), ("n_fp16", ctypes.c_int32),
                ("n_int8", ctypes.c_int32), ("n_int4", ctypes.c_int32),
                ("n_drop", ctypes.c_int32), ("budget_units", ctypes.c_int64),
                ("used_units", ctypes.c_int64)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(the codec has no non-HIP fallback)")
        L = ctypes.CDLL(LIB_PATH)
        P, vp, u64, i32 = ctypes.POINTER, ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int32
        cfgp = P(Config)
        sigs = {
            "skv_abi_version": (i32, []),
            "skv_status_string": (ctypes.c_char_p, [ctypes.c_int]),
            "skv_plan_tiers": (ctypes.c_int, [cfgp, P(Plan)]),
            "skv_payload_size": (ctypes.c_int, [cfgp, P(u64)]),
            "skv_workspace_size": (ctypes.c_int, [cfgp, P(u64)]),
            "skv_prepare": (ctypes.c_int, [cfgp, vp, vp]),
            "skv_score": (ctypes.c_int, [cfgp, vp, vp, vp, vp, vp, vp]),
            "skv_score_static": (ctypes.c_int, [cfgp, vp, vp, vp, vp, vp]),
            "skv_assign_tiers": (ctypes.c_int, [cfgp, vp, vp, vp, vp]),
            "skv_pack": (ctypes.c_int, [cfgp, vp, vp, vp, vp, u64, vp, vp]),
            "skv_unpack": (ctypes.c_int, [cfgp, vp, u64, vp, vp, vp, i32, i32, vp, vp]),
            "skv_link": (ctypes.c_int, [vp, vp, u64, vp, vp]),
            "skv_pack_batch": (ctypes.c_int, [cfgp, P(Request), i32, i32, i32, vp]),
            "skv_unpack_batch": (ctypes.c_int, [cfgp, P(Request), i32, vp, vp, i32, i32, i32, i32, vp]),
            "skv_upgrade_size": (ctypes.c_int, [cfgp, i32, i32, P(u64)]),
            "skv_group_count": (ctypes.c_int, [cfgp, P(GroupSpec), P(i32)]),
            "skv_plan_groups": (ctypes.c_int, [cfgp, P(GroupSpec), P(Plan)]),
            "skv_grouped_payload_size": (ctypes.c_int, [cfgp, P(GroupSpec), P(u64)]),
            "skv_group_workspace_size": (ctypes.c_int, [cfgp, P(GroupSpec), P(u64)]),
            "skv_prepare_groups": (ctypes.c_int, [cfgp, P(GroupSpec), vp, vp]),
            "skv_score_groups": (ctypes.c_int, [cfgp, P(GroupSpec), vp, vp, vp, vp, vp, vp]),
            "skv_assign_groups": (ctypes.c_int, [cfgp, P(GroupSpec), vp, vp, vp, vp]),
            "skv_pack_groups": (ctypes.c_int, [cfgp, P(GroupSpec), vp, vp, vp, vp, vp, u64, vp, vp]),
            "skv_unpack_groups": (ctypes.c_int, [cfgp, P(GroupSpec), vp, vp, u64, vp, vp, vp, i32, i32, vp, vp]),
            "skv_pack_upgrade": (ctypes.c_int, [cfgp, vp, vp, vp, vp, i32, i32, vp, u64, vp, vp]),
            "skv_unpack_upgrade": (ctypes.c_int, [cfgp, vp, u64, i32, i32, vp, vp, vp, i32, i32, vp, vp]),
            "skv_batch_workspace_size": (ctypes.c_int, [cfgp, P(ScoreRequest), i32, P(u64)]),
            "skv_score_batch": (ctypes.c_int, [cfgp, P(ScoreRequest), i32, vp, vp]),
            "skv_assign_batch": (ctypes.c_int, [cfgp, P(ScoreRequest), i32, vp, vp]),
            "skv_attn_prompt_workspace_size": (ctypes.c_int, [vp, vp, i32, P(u64)]),
            "skv_attn_decode_workspace_size": (ctypes.c_int, [vp, P(u64)]),
            "skv_attn_decode": (ctypes.c_int, [vp] + [vp] * 10 + [u64, vp]),
            "skv_pages_workspace_size": (ctypes.c_int, [i32, i32, i32, P(u64)]),
            "skv_pages_reserve": (ctypes.c_int, [vp, vp, i32, vp, vp, i32, vp, vp, u64, vp]),
            "skv_pages_fork": (ctypes.c_int, [vp, vp, i32, vp, i32, vp, i32, vp, i32, vp, vp, vp, u64, vp]),
            "skv_pages_compact": (ctypes.c_int, [vp, vp, i32, vp, i32, vp, i32, ctypes.c_int64, vp, i32, vp,
                                                 vp, vp, u64, vp]),
            "skv_pages_free": (ctypes.c_int, [vp, vp, i32, vp, i32, vp, vp]),
            "skv_pages_copy": (ctypes.c_int, [vp, vp, vp, vp, i32, vp, vp]),
            "skv_attn_prompt": (ctypes.c_int, [vp, vp, i32, vp, u64, vp]),
        }
        for name, (res, args) in sigs.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().skv_status_string(int(status)).decode()


def config(num_layers, num_kv_heads, head_dim, num_tokens, budget, first_ratio=0.02, num_sink=-1,
           decay=0.005, num_tiers=3, score_mode=KVNORM, num_q_heads=0, obs_window=0, quant_int8=0,
           quant_int4=0) -> Config:
    return Config(num_layers, num_kv_heads, head_dim, num_tokens, budget, first_ratio, num_sink,
                  decay, num_tiers, score_mode, num_q_heads, obs_window, quant_int8, quant_int4)


def _check(status: int, what: str):
    if status != OK:
        raise SkvError(status, what)


# Small requests are bound by the host: their six launches take less time on
# the GPU than the calls that issue them.  The checks below run without a Stream
# object or a ctypes wrapper per argument (1 x 2 x 64 x 512, encode and decode:
# 46 -> 36 us; the calls of a seven-step pipeline 264 -> 186 us).


def _stream(stream) -> int:
    if stream is None:  # the handle alone, without a Stream object
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _dev(t: Optional[torch.Tensor], dtype, numel: int, name: str) -> int:
    """Device pointer of a contiguous tensor holding at least `numel` elements of `dtype`."""
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs {numel}")
    return t.data_ptr()


def _cache_blocks(cfg: Config, k_cache: torch.Tensor, v_cache: torch.Tensor, block_size: int) -> int:
    """Blocks of a paged cache pair of the configuration's shape."""
    shape = k_cache.shape
    if len(shape) != 5 or shape[2] != block_size or shape != v_cache.shape:
        raise ValueError("caches must be [L][num_blocks][block_size][H][d] and alike")
    L, nb, _, H, d = shape
    if (L, H, d) != (cfg.num_layers, cfg.num_kv_heads, cfg.head_dim):
        raise ValueError("cache shape does not match the configuration")
    return nb


def plan_tiers(cfg: Config) -> dict:
    p = Plan()
    _check(lib().skv_plan_tiers(ctypes.byref(cfg), ctypes.byref(p)), "skv_plan_tiers")
    return {f: getattr(p, f) for f, _ in Plan._fields_}


def payload_size(cfg: Config) -> int:
    out = ctypes.c_uint64()
    _check(lib().skv_payload_size(ctypes.byref(cfg), ctypes.byref(out)), "skv_payload_size")
    return out.value


def workspace_size(cfg: Config) -> int:
    out = ctypes.c_uint64()
    _check(lib().skv_workspace_size(ctypes.byref(cfg), ctypes.byref(out)), "skv_workspace_size")
    return out.value


def _kv_numel(cfg: Config) -> int:
    return cfg.num_layers * cfg.num_kv_heads * cfg.num_tokens * cfg.head_dim


def prepare(cfg: Config, ws: torch.Tensor, stream=None):
    _check(lib().skv_prepare(ctypes.byref(cfg), _dev(ws, torch.uint8, workspace_size(cfg), "ws"),
                             _stream(stream)), "skv_prepare")


def score(cfg: Config, k: torch.Tensor, v: torch.Tensor, q_obs: Optional[torch.Tensor],
          out: torch.Tensor, ws: torch.Tensor, stream=None):
    n = _kv_numel(cfg)
    kp = _dev(k, torch.float16, n, "k")
    vp = _dev(v, torch.float16, n, "v") if cfg.score_mode != ATTN else None
    qp = None
    if cfg.score_mode == ATTN:
        qn = cfg.num_layers * cfg.num_q_heads * cfg.obs_window * cfg.head_dim
        qp = _dev(q_obs, torch.float16, qn, "q_obs")
    _check(lib().skv_score(ctypes.byref(cfg), kp, vp, qp, _dev(out, torch.float64, cfg.num_tokens, "score"),
                           _dev(ws, torch.uint8, workspace_size(cfg), "ws"), _stream(stream)), "skv_score")


def score_static(cfg: Config, k: torch.Tensor, v: torch.Tensor, q_obs: Optional[torch.Tensor],
                 out: torch.Tensor, stream=None):
    """skv_score_static: skv_score with the library's own scratch (no workspace)."""
    n = _kv_numel(cfg)
    kp = _dev(k, torch.float16, n, "k") if cfg.score_mode != RECENCY else None
    vp = _dev(v, torch.float16, n, "v") if cfg.score_mode == KVNORM else None
    qp = None
    if cfg.score_mode == ATTN:
        qn = cfg.num_layers * cfg.num_q_heads * cfg.obs_window * cfg.head_dim
        qp = _dev(q_obs, torch.float16, qn, "q_obs")
    _check(lib().skv_score_static(ctypes.byref(cfg), kp, vp, qp, _dev(out, torch.float64, cfg.num_tokens, "score"),
                                  _stream(stream)), "skv_score_static")


def assign_tiers(cfg: Config, scores: torch.Tensor, tier: torch.Tensor, stream=None,
                 ws: Optional[torch.Tensor] = None):
    """ws: the request's workspace (workspace_size bytes), or None; with it,
    rows past 32768 non-sink tokens are cut by the split form."""
    wsp = None if ws is None else _dev(ws, torch.uint8, workspace_size(cfg), "ws")
    _check(lib().skv_assign_tiers(ctypes.byref(cfg), _dev(scores, torch.float64, cfg.num_tokens, "score"),
                                  _dev(tier, torch.uint8, cfg.num_tokens, "tier"), wsp,
                                  _stream(stream)), "skv_assign_tiers")


def pack(cfg: Config, k: torch.Tensor, v: torch.Tensor, tier: torch.Tensor, payload: torch.Tensor,
         dev_status: Optional[torch.Tensor] = None, stream=None):
    n = _kv_numel(cfg)
    st = None if dev_status is None else _dev(dev_status, torch.int32, 1, "dev_status")
    _check(lib().skv_pack(ctypes.byref(cfg), _dev(k, torch.float16, n, "k"), _dev(v, torch.float16, n, "v"),
                          _dev(tier, torch.uint8, cfg.num_tokens, "tier"),
                          _dev(payload, torch.uint8, 0, "payload"), payload.numel(), st,
                          _stream(stream)), "skv_pack")


def unpack(cfg: Config, payload: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
           block_table: torch.Tensor, block_size: int, dev_status: torch.Tensor, stream=None):
    """k_cache/v_cache: float16 [L][num_blocks][block_size][H][d]."""
    nb = _cache_blocks(cfg, k_cache, v_cache, block_size)
    nbt = -(-cfg.num_tokens // block_size)
    _check(lib().skv_unpack(ctypes.byref(cfg), _dev(payload, torch.uint8, 0, "payload"), payload.numel(),
                            _dev(k_cache, torch.float16, k_cache.numel(), "k_cache"),
                            _dev(v_cache, torch.float16, v_cache.numel(), "v_cache"),
                            _dev(block_table, torch.int32, nbt, "block_table"), nb, block_size,
                            _dev(dev_status, torch.int32, 1, "dev_status"), _stream(stream)), "skv_unpack")


def upgrade_size(cfg: Config, m: int, mode: int) -> int:
    out = ctypes.c_uint64()
    _check(lib().skv_upgrade_size(ctypes.byref(cfg), m, mode, ctypes.byref(out)), "skv_upgrade_size")
    return out.value


def pack_upgrade(cfg: Config, k: torch.Tensor, v: torch.Tensor, tier: torch.Tensor, tokens: torch.Tensor,
                 mode: int, out: torch.Tensor, dev_status: Optional[torch.Tensor] = None, stream=None):
    """Upgrade payload for the listed tokens (int32, strictly ascending)."""
    n = _kv_numel(cfg)
    m = tokens.numel()
    st = None if dev_status is None else _dev(dev_status, torch.int32, 1, "dev_status")
    _check(lib().skv_pack_upgrade(ctypes.byref(cfg), _dev(k, torch.float16, n, "k"), _dev(v, torch.float16, n, "v"),
                                  _dev(tier, torch.uint8, cfg.num_tokens, "tier"),
                                  _dev(tokens, torch.int32, m, "tokens"), m, mode,
                                  _dev(out, torch.uint8, 0, "out"), out.numel(), st, _stream(stream)),
           "skv_pack_upgrade")


def unpack_upgrade(cfg: Config, upgrade: torch.Tensor, m: int, mode: int, k_cache: torch.Tensor,
                   v_cache: torch.Tensor, block_table: torch.Tensor, block_size: int, dev_status: torch.Tensor,
                   stream=None):
    """Applies an upgrade payload in place to caches filled by unpack."""
    nb = _cache_blocks(cfg, k_cache, v_cache, block_size)
    nbt = -(-cfg.num_tokens // block_size)
    _check(lib().skv_unpack_upgrade(ctypes.byref(cfg), _dev(upgrade, torch.uint8, 0, "upgrade"), upgrade.numel(),
                                    m, mode, _dev(k_cache, torch.float16, k_cache.numel(), "k_cache"),
                                    _dev(v_cache, torch.float16, v_cache.numel(), "v_cache"),
                                    _dev(block_table, torch.int32, nbt, "block_table"), nb, block_size,
                                    _dev(dev_status, torch.int32, 1, "dev_status"), _stream(stream)),
           "skv_unpack_upgrade")


class Groups:
    """A granularity and optional per-group budgets (host float32 array of G
    entries in (0, 1]) for the grouped calls; keeps the budget array alive."""

    def __init__(self, granularity: int, budgets=None):
        import numpy as np

        self.budgets = None if budgets is None else np.ascontiguousarray(budgets, np.float32)
        ptr = None if self.budgets is None else self.budgets.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
        self.spec = GroupSpec(granularity, 0, ptr)

    @property
    def ref(self):
        return ctypes.byref(self.spec)


def group_count(cfg: Config, groups: Groups) -> int:
    out = ctypes.c_int32()
    _check(lib().skv_group_count(ctypes.byref(cfg), groups.ref, ctypes.byref(out)), "skv_group_count")
    return out.value


def plan_groups(cfg: Config, groups: Groups) -> list:
    G = group_count(cfg, groups)
    plans = (Plan * G)()
    _check(lib().skv_plan_groups(ctypes.byref(cfg), groups.ref, plans), "skv_plan_groups")
    return [{f: getattr(p, f) for f, _ in Plan._fields_} for p in plans]


def grouped_payload_size(cfg: Config, groups: Groups) -> int:
    out = ctypes.c_uint64()
    _check(lib().skv_grouped_payload_size(ctypes.byref(cfg), groups.ref, ctypes.byref(out)),
           "skv_grouped_payload_size")
    return out.value


def group_workspace_size(cfg: Config, groups: Groups) -> int:
    out = ctypes.c_uint64()
    _check(lib().skv_group_workspace_size(ctypes.byref(cfg), groups.ref, ctypes.byref(out)),
           "skv_group_workspace_size")
    return out.value


def prepare_groups(cfg: Config, groups: Groups, ws: torch.Tensor, stream=None):
    _check(lib().skv_prepare_groups(ctypes.byref(cfg), groups.ref,
                                    _dev(ws, torch.uint8, group_workspace_size(cfg, groups), "ws"),
                                    _stream(stream)), "skv_prepare_groups")


def score_groups(cfg: Config, groups: Groups, k: torch.Tensor, v: Optional[torch.Tensor],
                 q_obs: Optional[torch.Tensor], out: torch.Tensor, ws: torch.Tensor, stream=None):
    n = _kv_numel(cfg)
    G = group_count(cfg, groups)
    kp = _dev(k, torch.float16, n, "k")
    vp = _dev(v, torch.float16, n, "v") if cfg.score_mode != ATTN else None
    qp = None
    if cfg.score_mode == ATTN:
        qp = _dev(q_obs, torch.float16, cfg.num_layers * cfg.num_q_heads * cfg.obs_window * cfg.head_dim, "q_obs")
    _check(lib().skv_score_groups(ctypes.byref(cfg), groups.ref, kp, vp, qp,
                                  _dev(out, torch.float64, G * cfg.num_tokens, "score"),
                                  _dev(ws, torch.uint8, group_workspace_size(cfg, groups), "ws"), _stream(stream)),
           "skv_score_groups")


def assign_groups(cfg: Config, groups: Groups, scores: torch.Tensor, tier: torch.Tensor, ws: torch.Tensor,
                  stream=None):
    G = group_count(cfg, groups)
    _check(lib().skv_assign_groups(ctypes.byref(cfg), groups.ref,
                                   _dev(scores, torch.float64, G * cfg.num_tokens, "score"),
                                   _dev(tier, torch.uint8, G * cfg.num_tokens, "tier"),
                                   _dev(ws, torch.uint8, group_workspace_size(cfg, groups), "ws"),
                                   _stream(stream)), "skv_assign_groups")


def pack_groups(cfg: Config, groups: Groups, k: torch.Tensor, v: torch.Tensor, tier: torch.Tensor,
                ws: torch.Tensor, payload: torch.Tensor, dev_status: Optional[torch.Tensor] = None, stream=None):
    n = _kv_numel(cfg)
    G = group_count(cfg, groups)
    st = None if dev_status is None else _dev(dev_status, torch.int32, 1, "dev_status")
    _check(lib().skv_pack_groups(ctypes.byref(cfg), groups.ref, _dev(k, torch.float16, n, "k"),
                                 _dev(v, torch.float16, n, "v"), _dev(tier, torch.uint8, G * cfg.num_tokens, "tier"),
                                 _dev(ws, torch.uint8, group_workspace_size(cfg, groups), "ws"),
                                 _dev(payload, torch.uint8, 0, "payload"), payload.numel(), st, _stream(stream)),
           "skv_pack_groups")


def unpack_groups(cfg: Config, groups: Groups, ws: torch.Tensor, payload: torch.Tensor, k_cache: torch.Tensor,
                  v_cache: torch.Tensor, block_table: torch.Tensor, block_size: int, dev_status: torch.Tensor,
                  stream=None):
    nb = _cache_blocks(cfg, k_cache, v_cache, block_size)
    nbt = -(-cfg.num_tokens // block_size)
    _check(lib().skv_unpack_groups(ctypes.byref(cfg), groups.ref,
                                   _dev(ws, torch.uint8, group_workspace_size(cfg, groups), "ws"),
                                   _dev(payload, torch.uint8, 0, "payload"), payload.numel(),
                                   _dev(k_cache, torch.float16, k_cache.numel(), "k_cache"),
                                   _dev(v_cache, torch.float16, v_cache.numel(), "v_cache"),
                                   _dev(block_table, torch.int32, nbt, "block_table"), nb, block_size,
                                   _dev(dev_status, torch.int32, 1, "dev_status"), _stream(stream)),
           "skv_unpack_groups")


def _per_token(cfg: Config) -> int:
    return cfg.num_layers * cfg.num_kv_heads * cfg.head_dim


def pack_batch(cfg: Config, ks, vs, tiers, payloads, statuses=None, layer_begin=0, layer_count=None,
               stream=None):
    """Packs len(ks) requests (n taken from each tier map's length) in batched launches."""
    count = len(ks)
    per_token = _per_token(cfg)
    reqs = (Request * count)()
    for i in range(count):
        n = tiers[i].numel()
        r = reqs[i]
        kv_n = per_token * n
        r.num_tokens = n
        r.k = _dev(ks[i], torch.float16, kv_n, "k")
        r.v = _dev(vs[i], torch.float16, kv_n, "v")
        r.tier = _dev(tiers[i], torch.uint8, n, "tier")
        r.payload = _dev(payloads[i], torch.uint8, 0, "payload")
        r.payload_bytes = payloads[i].numel()
        if statuses is not None:
            r.dev_status = _dev(statuses[i], torch.int32, 1, "dev_status")
    lc = cfg.num_layers - layer_begin if layer_count is None else layer_count
    _check(lib().skv_pack_batch(ctypes.byref(cfg), reqs, count, layer_begin, lc, _stream(stream)),
           "skv_pack_batch")


def _score_requests(cfg: Config, scores, ks=None, vs=None, tiers=None):
    count = len(scores)
    per_token = _per_token(cfg)
    reqs = (ScoreRequest * count)()
    for i in range(count):
        n = scores[i].numel()
        r = reqs[i]
        r.num_tokens = n
        r.score = _dev(scores[i], torch.float64, n, "score")
        if ks is not None and cfg.score_mode == KVNORM:
            kv_n = per_token * n
            r.k = _dev(ks[i], torch.float16, kv_n, "k")
            r.v = _dev(vs[i], torch.float16, kv_n, "v")
        if tiers is not None:
            r.tier = _dev(tiers[i], torch.uint8, n, "tier")
    return reqs, count


def batch_workspace_size(cfg: Config, scores) -> int:
    """Workspace bytes of score_batch and assign_batch for requests of these
    lengths (cfg.num_tokens >= every n)."""
    count = len(scores)
    reqs = (ScoreRequest * count)()
    for i in range(count):
        r = reqs[i]
        r.num_tokens = scores[i].numel()
        r.score = 256  # sizes only: the pointers are not dereferenced
        r.k = r.v = 256
    out = ctypes.c_uint64()
    _check(lib().skv_batch_workspace_size(ctypes.byref(cfg), reqs, count, ctypes.byref(out)),
           "skv_batch_workspace_size")
    return out.value


def score_batch(cfg: Config, ks, vs, scores, ws: torch.Tensor, stream=None):
    """Scores len(scores) requests (n = each score buffer's length) in batched
    launches; ws prepared by prepare(cfg, ws) with cfg.num_tokens >= every n."""
    reqs, count = _score_requests(cfg, scores, ks, vs)
    _check(lib().skv_score_batch(ctypes.byref(cfg), reqs, count,
                                 _dev(ws, torch.uint8, batch_workspace_size(cfg, scores), "ws"), _stream(stream)),
           "skv_score_batch")


def assign_batch(cfg: Config, scores, tiers, stream=None, ws=None):
    """Assigns the tiers of len(scores) requests: one workgroup per request of
    at most 32768 non-sink tokens; longer requests split over the GPU when ws
    (batch_workspace_size bytes) is given, else one workgroup each."""
    reqs, count = _score_requests(cfg, scores, tiers=tiers)
    w = None if ws is None else _dev(ws, torch.uint8, batch_workspace_size(cfg, scores), "ws")
    _check(lib().skv_assign_batch(ctypes.byref(cfg), reqs, count, w, _stream(stream)), "skv_assign_batch")


def unpack_batch(cfg: Config, payloads, token_counts, block_tables, k_cache: torch.Tensor,
                 v_cache: torch.Tensor, block_size: int, statuses, layer_begin=0, layer_count=None,
                 stream=None):
    """Unpacks len(payloads) requests into one shared paged cache in batched launches."""
    nb = _cache_blocks(cfg, k_cache, v_cache, block_size)
    count = len(payloads)
    reqs = (Request * count)()
    for i in range(count):
        n = int(token_counts[i])
        r = reqs[i]
        r.num_tokens = n
        r.payload = _dev(payloads[i], torch.uint8, 0, "payload")
        r.payload_bytes = payloads[i].numel()
        r.block_table = _dev(block_tables[i], torch.int32, -(-n // block_size), "block_table")
        r.dev_status = _dev(statuses[i], torch.int32, 1, "dev_status")
    lc = cfg.num_layers - layer_begin if layer_count is None else layer_count
    _check(lib().skv_unpack_batch(ctypes.byref(cfg), reqs, count,
                                  _dev(k_cache, torch.float16, k_cache.numel(), "k_cache"),
                                  _dev(v_cache, torch.float16, v_cache.numel(), "v_cache"), nb, block_size,
                                  layer_begin, lc, _stream(stream)), "skv_unpack_batch")


# The structures of the attention and page calls, packed at once: building a ctypes
# structure field by field takes several times as long as the call (a small prompt's
# call 11 -> 6 us).
_ATTN_TYPES = {torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16}
_ATTN_CONFIG = struct.Struct("@5if4q")      # skv_attn_config
_ATTN_REQUEST = struct.Struct("@2i5P2q")    # skv_attn_request
_DECODE_CONFIG = struct.Struct("@12if9q")   # skv_decode_config
_PAGE_POOL = struct.Struct("@4i3P")         # skv_page_pool


def _stream_on(device: int, stream) -> int:
    """The raw stream of a call on tensors of `device`, which must be the current
    one: the library launches there."""
    if device != torch.cuda.current_device() or (stream is not None and stream.device_index != device):
        raise ValueError("the tensors (and the stream) must be on the current device")
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _strided(t: Optional[torch.Tensor], dtype, device: int, shape, name: str):
    """Device pointer and strides of a tensor of this dtype, device and shape
    whose last axis is contiguous."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name} must be a device tensor, all of them on one device")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    st = t.stride()
    if st[-1] != 1 and t.numel():
        raise ValueError(f"{name}'s last axis must be contiguous")
    return t.data_ptr(), st


def _flat(t: Optional[torch.Tensor], dtype, device: int, numel: int, name: str) -> int:
    """Device pointer of a contiguous tensor on `device` holding at least `numel`
    elements of `dtype`."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name} must be a device tensor, all of them on one device")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs {numel}")
    return t.data_ptr()


def _steps(strides, shape):
    """Strides with those of single-place axes (torch gives any number there) as packing would have them."""
    if 1 in shape or 0 in shape:
        return tuple(s if n > 1 else shape[-1] for s, n in zip(strides, shape))
    return strides


def attn_prompt_workspace_size(q_lens, kv_lens, num_q_heads: int, num_kv_heads: int, head_dim: int,
                               causal: bool = True) -> int:
    """Workspace bytes with which attn_prompt splits these sequences' keys over the GPU (0: it would not)."""
    count = len(q_lens)
    if len(kv_lens) != count:
        raise ValueError("q_lens and kv_lens differ in length")
    cfg = _ATTN_CONFIG.pack(DTYPE_F16, num_q_heads, num_kv_heads, head_dim, bool(causal), 1.0, 0, 0, 0, 0)
    reqs = b"".join(_ATTN_REQUEST.pack(nq, nk, 0, 0, 0, 0, 0, 0, 0) for nq, nk in zip(q_lens, kv_lens))
    out = ctypes.c_uint64()
    _check(lib().skv_attn_prompt_workspace_size(cfg, reqs, count, ctypes.byref(out)), "skv_attn_prompt_workspace_size")
    return out.value


def attn_prompt(q: torch.Tensor, k, v, out: torch.Tensor, q_lens=None, kv_lens=None, causal: bool = True,
                scale: Optional[float] = None, lse: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None, stream=None):
    """Attention of packed sequences: q and out [sum(q_lens)][Hq][d] (float16
    or bfloat16, any token and head strides), sequence after sequence.  k, v:
    packed the same way, [sum(kv_lens)][H][d], or a list with each sequence's
    [H][n][d] (a layer of the codec's K and V).  q_lens defaults to one
    sequence, kv_lens to the lists' lengths, or (packed) to one sequence of all
    keys, else to q_lens; causal query i sees keys j <= i + n_keys - n_queries.
    scale defaults to 1/sqrt(d).  lse: float32 [sum(q_lens)][Hq], written when
    given.  ws: attn_prompt_workspace_size bytes, or None (no splitting of the
    keys: few queries over many keys then take several times as long)."""
    dtype, device = q.dtype, q.get_device()
    if dtype not in _ATTN_TYPES:
        raise TypeError(f"q must be float16 or bfloat16, got {dtype}")
    if q.dim() != 3:
        raise ValueError("q must be [tokens][heads][d]")
    shape = q.shape
    total, Hq, d = shape
    lists = isinstance(k, (list, tuple))
    if lists != isinstance(v, (list, tuple)) or (lists and len(k) != len(v)):
        raise ValueError("k and v must both be packed tensors or lists of one length")
    if kv_lens is None:
        kv_lens = [x.shape[1] for x in k] if lists else [k.shape[0]] if q_lens is None else q_lens
    if q_lens is None:
        q_lens = [total]
    count = len(q_lens)
    if len(kv_lens) != count or (lists and len(k) != count):
        raise ValueError("q_lens, kv_lens and the lists of k and v differ in length")
    if min(q_lens, default=0) < 0 or min(kv_lens, default=0) < 0 or sum(q_lens) != total:
        raise ValueError("q_lens must be non-negative and add up to q's tokens")
    qp, qs = _strided(q, dtype, device, shape, "q")
    op, os_ = _strided(out, dtype, device, shape, "out")
    qs, os_ = _steps(qs, shape), _steps(os_, shape)
    lp = 0 if lse is None else _flat(lse, torch.float32, device, total * Hq, "lse")
    lstep = 4 * Hq if lp else 0
    reqs = []
    if lists:
        H = k[0].shape[0] if count else 1
        for nq, nk, ki, vi in zip(q_lens, kv_lens, k, v):
            want = (H, nk, d)
            kp, ks = _strided(ki, dtype, device, want, "k")
            vp, vs = _strided(vi, dtype, device, want, "v")
            ks = _steps(ks, want)
            if ks != _steps(vs, want):
                raise ValueError("k and v must have the same strides")
            reqs.append(_ATTN_REQUEST.pack(nq, nk, qp, kp, vp, op, lp, ks[1], ks[0]))
            qp, op, lp = qp + 2 * qs[0] * nq, op + 2 * os_[0] * nq, lp + lstep * nq
    else:
        if k.dim() != 3 or sum(kv_lens) != k.shape[0]:
            raise ValueError("k must be [tokens][heads][d], kv_lens adding up to its tokens")
        H = k.shape[1]
        want = (k.shape[0], H, d)
        kp, ks = _strided(k, dtype, device, want, "k")
        vp, vs = _strided(v, dtype, device, want, "v")
        ks = _steps(ks, want)
        if ks != _steps(vs, want):
            raise ValueError("k and v must have the same strides")
        kstep = 2 * ks[0]
        for nq, nk in zip(q_lens, kv_lens):
            reqs.append(_ATTN_REQUEST.pack(nq, nk, qp, kp, vp, op, lp, ks[0], ks[1]))
            qp, op, lp = qp + 2 * qs[0] * nq, op + 2 * os_[0] * nq, lp + lstep * nq
            kp, vp = kp + kstep * nk, vp + kstep * nk
    cfg = _ATTN_CONFIG.pack(_ATTN_TYPES[dtype], Hq, H, d, bool(causal), d ** -0.5 if scale is None else scale,
                            qs[0], qs[1], os_[0], os_[1])
    size = 0 if ws is None else ws.numel()
    wsp = _flat(ws, torch.uint8, device, 0, "ws") if size else None
    _check(lib().skv_attn_prompt(cfg, b"".join(reqs), count, wsp, size, _stream_on(device, stream)), "skv_attn_prompt")


def attn_decode_workspace_size(num_requests: int, num_queries: int, num_q_heads: int, num_kv_heads: int, head_dim: int,
                               max_len: int, prefix_len: int = 0) -> int:
    """Workspace bytes of attn_decode with these arguments."""
    cfg = _DECODE_CONFIG.pack(DTYPE_F16, num_requests, num_queries, num_q_heads, num_kv_heads, head_dim, 1, 1, 0, max_len,
                              prefix_len, 0, 1.0, *[0] * 9)
    out = ctypes.c_uint64()
    _check(lib().skv_attn_decode_workspace_size(cfg, ctypes.byref(out)), "skv_attn_decode_workspace_size")
    return out.value


def attn_decode(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_tables: torch.Tensor,
                lens: torch.Tensor, out: torch.Tensor, ws: Optional[torch.Tensor], max_len: int, prefix_len: int = 0,
                tiers: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                lse: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None, stream=None):
    """Attention of each request's newest tokens over one layer of a paged
    cache.  q, out: [B][Lq][Hq][d] (any strides, last axis contiguous); k_cache,
    v_cache: [num_blocks][block_size][H][d] (k_cache[layer] of what unpack
    fills); block_tables: int32 [B][width]; lens: int32 [B], tokens in the cache,
    the Lq newest among them.  max_len: about the longest length (sizes the
    launch).  prefix_len: leading tokens that every request shares, a multiple
    of the block size (their table entries and tiers are request 0's).  tiers:
    uint8 [tier_len], [B][tier_len] or [B][H][tier_len] (expanded axes may
    have stride 0); DROP tokens are masked, tokens past tier_len kept.  lse:
    float32 [B][Lq][Hq].  ws: attn_decode_workspace_size bytes.  dev_status:
    int32[1], set on a bad table entry or length, never cleared."""
    dtype, device = q.dtype, q.get_device()
    if dtype not in _ATTN_TYPES:
        raise TypeError(f"q must be float16 or bfloat16, got {dtype}")
    if q.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("q must be [B][Lq][Hq][d] and the caches [num_blocks][block_size][H][d]")
    shape = q.shape
    B, Lq, Hq, d = shape
    nb, bs, H, dk = k_cache.shape
    if dk != d or k_cache.shape != v_cache.shape:
        raise ValueError("caches must be [num_blocks][block_size][H][d] of q's d and alike")
    if block_tables.dim() != 2 or block_tables.shape[0] != B:
        raise ValueError("block_tables must be [B][width]")
    qp, qs = _strided(q, dtype, device, shape, "q")
    op, os_ = _strided(out, dtype, device, shape, "out")
    qs, os_ = _steps(qs, shape), _steps(os_, shape)
    cells = nb * bs * H * d
    kp, vp = _flat(k_cache, dtype, device, cells, "k_cache"), _flat(v_cache, dtype, device, cells, "v_cache")
    tp, width = _flat(block_tables, torch.int32, device, 0, "block_tables"), block_tables.shape[1]
    tier_p, tier_len, per_request, per_head = None, 0, 0, 0
    if tiers is not None:
        ts, tier_len = tiers.stride(), tiers.shape[-1] if tiers.dim() else 0
        if tiers.shape == (tier_len,):
            pass
        elif tiers.shape == (B, tier_len):
            per_request = ts[0]
        elif tiers.shape == (B, H, tier_len):
            per_request, per_head = ts[0], ts[1]
        else:
            raise ValueError("tiers must be [tier_len], [B][tier_len] or [B][H][tier_len]")
        if tiers.dtype != torch.uint8 or tiers.get_device() != device:
            raise TypeError("tiers must be a uint8 tensor on q's device")
        if tier_len > 1 and ts[-1] != 1:
            raise ValueError("tiers' last axis must be contiguous")
        tier_p = tiers.data_ptr()
    cfg = _DECODE_CONFIG.pack(_ATTN_TYPES[dtype], B, Lq, Hq, H, d, nb, bs, width, max_len, prefix_len, tier_len,
                              d ** -0.5 if scale is None else scale, qs[0], qs[1], qs[2], os_[0], os_[1], os_[2], width,
                              per_request, per_head)
    size = 0 if ws is None else ws.numel()
    _check(lib().skv_attn_decode(
        cfg, qp, kp, vp, tp, _flat(lens, torch.int32, device, B, "lens"), tier_p, op,
        None if lse is None else _flat(lse, torch.float32, device, B * Lq * Hq, "lse"),
        None if dev_status is None else _flat(dev_status, torch.int32, device, 1, "dev_status"),
        _flat(ws, torch.uint8, device, 0, "ws") if size else None, size, _stream_on(device, stream)), "skv_attn_decode")


def _pool(k_cache: torch.Tensor, v_cache: torch.Tensor, refs: Optional[torch.Tensor], device: int) -> bytes:
    """The pool of a 16-bit paged cache pair [L][num_blocks][block_size][H][d]."""
    shape, dtype = k_cache.shape, k_cache.dtype
    if len(shape) != 5 or shape != v_cache.shape:
        raise ValueError("caches must be [L][num_blocks][block_size][H][d] and alike")
    if dtype not in _ATTN_TYPES:
        raise TypeError(f"caches must be float16 or bfloat16, got {dtype}")
    L, nb, bs, H, d = shape
    if refs is not None and refs.numel() != nb:
        raise ValueError(f"refs must hold one count per page, {nb}, got {refs.numel()}")
    return _PAGE_POOL.pack(L, nb, bs, 2 * H * d, _flat(k_cache, dtype, device, 0, "k_cache"),
                           _flat(v_cache, dtype, device, 0, "v_cache"),
                           0 if refs is None else _flat(refs, torch.int32, device, nb, "refs"))


def _tables(tables: torch.Tensor, rows: int, device: int, name: str):
    """Pointer and width of contiguous block tables int32 [rows][width]."""
    if tables.dim() != 2 or tables.shape[0] != rows:
        raise ValueError(f"{name} must be [{rows}][width]")
    return _flat(tables, torch.int32, device, 0, name), tables.shape[1]


def pages_workspace_size(num_requests: int, num_blocks: int, max_len: int) -> int:
    """Workspace bytes of pages_reserve, pages_fork and pages_compact with up to
    num_requests output rows of up to max_len tokens (table width * block size)."""
    out = ctypes.c_uint64()
    _check(lib().skv_pages_workspace_size(num_requests, num_blocks, max_len, ctypes.byref(out)),
           "skv_pages_workspace_size")
    return out.value


def pages_reserve(refs: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, new_lens: torch.Tensor,
                  block_size: int, ws: torch.Tensor, dev_status: torch.Tensor, stream=None):
    """Gives each request the pages to grow from lens to new_lens tokens: the
    lowest free ones (refs 0), written into tables (int32 [B][width])."""
    B, device = lens.numel(), refs.get_device()
    pool = _PAGE_POOL.pack(1, refs.numel(), block_size, 16, 0, 0, _flat(refs, torch.int32, device, 0, "refs"))
    tp, width = _tables(tables, B, device, "tables")
    _check(lib().skv_pages_reserve(pool, tp, width, _flat(lens, torch.int32, device, B, "lens"),
                                   _flat(new_lens, torch.int32, device, B, "new_lens"), B,
                                   _flat(dev_status, torch.int32, device, 1, "dev_status"),
                                   _flat(ws, torch.uint8, device, 0, "ws"), ws.numel(), _stream_on(device, stream)),
           "skv_pages_reserve")


def pages_fork(k_cache: torch.Tensor, v_cache: torch.Tensor, refs: torch.Tensor, tables: torch.Tensor,
               lens: torch.Tensor, parents: torch.Tensor, out_tables: torch.Tensor, out_lens: torch.Tensor,
               ws: torch.Tensor, dev_status: torch.Tensor, stream=None):
    """Child c becomes a copy of request parents[c]: full pages shared, a partly
    filled last page copied.  Writes out_tables [children][width] and out_lens,
    which may not be the inputs."""
    B, N, device = lens.numel(), parents.numel(), refs.get_device()
    pool = _pool(k_cache, v_cache, refs, device)
    tp, width = _tables(tables, B, device, "tables")
    op, out_width = _tables(out_tables, N, device, "out_tables")
    _check(lib().skv_pages_fork(pool, tp, width, _flat(lens, torch.int32, device, B, "lens"), B,
                                _flat(parents, torch.int32, device, N, "parents"), N, op, out_width,
                                _flat(out_lens, torch.int32, device, N, "out_lens"),
                                _flat(dev_status, torch.int32, device, 1, "dev_status"),
                                _flat(ws, torch.uint8, device, 0, "ws"), ws.numel(), _stream_on(device, stream)),
           "skv_pages_fork")


def pages_compact(k_cache: torch.Tensor, v_cache: torch.Tensor, refs: torch.Tensor, tables: torch.Tensor,
                  lens: torch.Tensor, tiers: torch.Tensor, out_tables: torch.Tensor, out_lens: torch.Tensor,
                  ws: torch.Tensor, dev_status: torch.Tensor, stream=None):
    """Copies of the requests without their DROP tokens (tiers: uint8
    [B][tier_len], any request stride; tokens past tier_len are kept): full
    pages before the first dropped token shared, the other rows gathered into
    new pages.  out_tables and out_lens may not be the inputs."""
    B, device = lens.numel(), refs.get_device()
    pool = _pool(k_cache, v_cache, refs, device)
    tp, width = _tables(tables, B, device, "tables")
    op, out_width = _tables(out_tables, B, device, "out_tables")
    if tiers.get_device() != device or tiers.dtype != torch.uint8:
        raise TypeError("tiers must be a uint8 tensor on the pool's device")
    if tiers.dim() != 2 or tiers.shape[0] != B or (tiers.shape[1] > 1 and tiers.stride(1) != 1):
        raise ValueError("tiers must be [requests][tier_len], its last axis contiguous")
    _check(lib().skv_pages_compact(pool, tp, width, _flat(lens, torch.int32, device, B, "lens"), B,
                                   tiers.data_ptr(), tiers.shape[1], tiers.stride(0), op, out_width,
                                   _flat(out_lens, torch.int32, device, B, "out_lens"),
                                   _flat(dev_status, torch.int32, device, 1, "dev_status"),
                                   _flat(ws, torch.uint8, device, 0, "ws"), ws.numel(), _stream_on(device, stream)),
           "skv_pages_compact")


def pages_free(refs: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, block_size: int,
               dev_status: torch.Tensor, stream=None):
    """Releases requests: the count of every page they hold goes down by one."""
    B, device = lens.numel(), refs.get_device()
    pool = _PAGE_POOL.pack(1, refs.numel(), block_size, 16, 0, 0, _flat(refs, torch.int32, device, 0, "refs"))
    tp, width = _tables(tables, B, device, "tables")
    _check(lib().skv_pages_free(pool, tp, width, _flat(lens, torch.int32, device, B, "lens"), B,
                                _flat(dev_status, torch.int32, device, 1, "dev_status"), _stream_on(device, stream)),
           "skv_pages_free")


def pages_copy(src_k: torch.Tensor, src_v: torch.Tensor, dst_k: torch.Tensor, dst_v: torch.Tensor,
               src_pages: torch.Tensor, dst_pages: torch.Tensor, dev_status: torch.Tensor, stream=None):
    """Copies page src_pages[i] of one cache pair to page dst_pages[i] of another
    in every layer."""
    device = src_k.get_device()
    src, dst = _pool(src_k, src_v, None, device), _pool(dst_k, dst_v, None, device)
    if src_k.shape[2:] != dst_k.shape[2:] or src_k.shape[0] != dst_k.shape[0] or src_k.dtype != dst_k.dtype:
        raise ValueError("the caches must agree in layers, block size, heads, dimension and type")
    n = src_pages.numel()
    _check(lib().skv_pages_copy(src, dst, _flat(src_pages, torch.int32, device, n, "src_pages"),
                                _flat(dst_pages, torch.int32, device, n, "dst_pages"), n,
                                _flat(dev_status, torch.int32, device, 1, "dev_status"), _stream_on(device, stream)),
           "skv_pages_copy")


def link(dst: torch.Tensor, src: torch.Tensor, nbytes: int, host_staging: Optional[torch.Tensor] = None,
         stream=None):
    """Emulated transfer of nbytes (device to device, or through pinned host memory)."""
    if dst.numel() * dst.element_size() < nbytes or src.numel() * src.element_size() < nbytes:
        raise ValueError("link buffers smaller than nbytes")
    hs = None
    if host_staging is not None:
        if host_staging.is_cuda or not host_staging.is_pinned() or host_staging.numel() * host_staging.element_size() < nbytes:
            raise ValueError("host_staging must be pinned host memory of at least nbytes")
        hs = host_staging.data_ptr()
    _check(lib().skv_link(dst.data_ptr(), src.data_ptr(), nbytes, hs,
                          _stream(stream)), "skv_link")


class Codec:
    """Device buffers for one request shape: workspace (prepared), scores,
    tier map, payload and status words, plus the encode/decode sequence."""

    def __init__(self, cfg: Config, device="cuda"):
        self.cfg = cfg
        self.device = torch.device(device)
        self.plan = plan_tiers(cfg)
        self.payload_bytes = payload_size(cfg)
        self.ws = torch.empty(workspace_size(cfg), dtype=torch.uint8, device=self.device)
        self.scores = torch.empty(cfg.num_tokens, dtype=torch.float64, device=self.device)
        self.tier = torch.empty(cfg.num_tokens, dtype=torch.uint8, device=self.device)
        self.payload = torch.empty(self.payload_bytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(2, dtype=torch.int32, device=self.device)
        prepare(cfg, self.ws)

    def encode(self, k, v, q_obs=None, stream=None):
        score(self.cfg, k, v, q_obs, self.scores, self.ws, stream)
        assign_tiers(self.cfg, self.scores, self.tier, stream, ws=self.ws)
        pack(self.cfg, k, v, self.tier, self.payload, self.status[0:1], stream)
        return self.payload

    def decode(self, payload, k_cache, v_cache, block_table, block_size=16, stream=None):
        unpack(self.cfg, payload, k_cache, v_cache, block_table, block_size, self.status[1:2], stream)
