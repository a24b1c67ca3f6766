"""Python binding of the DualMap routing engine (libdualmap.so, gfx950).

Argument marshalling only: every step of routing, rebalancing and scaling
runs in the HIP kernels behind the C ABI declared in include/dualmap.h.
PyTorch supplies device memory and the stream.  The module refuses to load
if the library has not been built (run __graft_entry__.build() or
python -m paper_2602_06502_amd._build); there is no CPU fallback.

Functions with the C names (dm_create, dm_build_rings, dm_index_insert,
dm_route_batch, dm_rebalance, dm_scale, ...) take raw device pointers; the
DualMap class wraps them for torch tensors.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdualmap.so")

DM_OK, DM_EINVAL, DM_ENOMEM, DM_EFULL, DM_ESTATE, DM_EDEVICE = range(6)
_NAMES = {0: "DM_OK", 1: "DM_EINVAL", 2: "DM_ENOMEM", 3: "DM_EFULL", 4: "DM_ESTATE",
          5: "DM_EDEVICE"}

EXPORTS = ("dm_create", "dm_destroy", "dm_build_rings", "dm_ring_export", "dm_index_insert",
           "dm_index_erase", "dm_index_clear", "dm_index_size", "dm_route_batch",
           "dm_route_batch_noalloc",
           "dm_rebalance", "dm_scale", "dm_set_timing", "dm_route_stage_ms",
           "dm_kv_save", "dm_queue_append", "dm_queue_migrate", "dm_queue_drain", "dm_queue_reprobe",
           "dm_set_pipelining", "dm_set_policy", "dm_keylen_enable",
           "dm_keylen_window",
           "dm_keylen_export", "dm_pages_fork", "dm_pages_compact", "dm_pages_copy", "dm_kv_append",
           "dm_attn_plan_bytes", "dm_attn_plan", "dm_attn", "dm_sync", "dm_last_error")


class DMError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_NAMES.get(status, status)}: {msg}")
        self.status = status


class dm_config(C.Structure):
    _fields_ = [("block_size", C.c_uint32), ("key_blocks", C.c_uint32),
                ("seed", C.c_uint64 * 2), ("vnodes", C.c_uint32), ("max_slots", C.c_uint32),
                ("index_log2_slots", C.c_uint32), ("reserved", C.c_uint32),
                ("ttft_base_us", C.c_int64), ("ttft_per_token_us", C.c_int64),
                ("queue_div", C.c_int64), ("slo_us", C.c_int64)]


class dm_route_out(C.Structure):
    _fields_ = [("key", C.c_void_p), ("cand", C.c_void_p), ("match", C.c_void_p),
                ("chosen", C.c_void_p), ("ttft_us", C.c_void_p), ("flags", C.c_void_p),
                ("block_keys", C.c_void_p), ("key_len", C.c_void_p)]


class dm_queues(C.Structure):
    _fields_ = [("qoff", C.c_void_p), ("rec_id", C.c_void_p), ("unc_here", C.c_void_p),
                ("alt", C.c_void_p), ("unc_alt", C.c_void_p), ("base_work", C.c_void_p),
                ("prefill_interval", C.c_void_p), ("decode_threshold_us", C.c_int64)]


class dm_queue_out(C.Structure):
    _fields_ = [("qoff", C.c_void_p), ("rec_id", C.c_void_p), ("unc_here", C.c_void_p),
                ("alt", C.c_void_p), ("unc_alt", C.c_void_p), ("base_work", C.c_void_p),
                ("cap", C.c_uint64)]


class dm_migrations(C.Structure):
    _fields_ = [("rec_id", C.c_void_p), ("from_", C.c_void_p), ("to", C.c_void_p),
                ("benefit_us", C.c_void_p), ("ttft_to_us", C.c_void_p), ("count", C.c_void_p)]


class dm_kv_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64),
                ("layers", C.c_uint32), ("n_pages", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("dtype", C.c_uint32), ("reserved", C.c_uint32)]


class dm_page_tables(C.Structure):
    _fields_ = [("off", C.c_void_p), ("page", C.c_void_p), ("len", C.c_void_p), ("n", C.c_uint64),
                ("entries", C.c_uint64)]


class dm_pages_out(C.Structure):
    _fields_ = [("off", C.c_void_p), ("page", C.c_void_p), ("len", C.c_void_p), ("cap", C.c_uint64),
                ("ref", C.c_void_p), ("move_src", C.c_void_p), ("move_dst", C.c_void_p),
                ("move_cap", C.c_uint64), ("moves", C.c_void_p), ("live", C.c_void_p)]


class dm_token_batch(C.Structure):
    _fields_ = [("tables", dm_page_tables), ("q_off", C.c_void_p), ("q_tokens", C.c_uint64),
                ("group_off", C.c_void_p), ("groups", C.c_uint64)]


class dm_append_args(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64),
                ("k_stride", C.c_int64), ("v_stride", C.c_int64), ("q_out", C.c_void_p),
                ("q_out_stride", C.c_int64), ("q_norm", C.c_void_p), ("k_norm", C.c_void_p),
                ("cos", C.c_void_p), ("sin", C.c_void_p), ("max_pos", C.c_uint64),
                ("q_heads", C.c_uint32), ("rot_dim", C.c_uint32), ("interleaved", C.c_uint32),
                ("eps", C.c_float)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libdualmap.so (raises if it is missing: no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"libdualmap.so not built at {path}; run __graft_entry__.build()")
    L = C.CDLL(path)
    P, u32, u64, i32 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int
    sig = {
        "dm_create": (i32, [P, P, P]),
        "dm_destroy": (None, [P]),
        "dm_build_rings": (i32, [P, P, u32]),
        "dm_ring_export": (i32, [P, i32, P, P, u64, P]),
        "dm_index_insert": (i32, [P, u32, P, u64]),
        "dm_index_erase": (i32, [P, u32, P, u64]),
        "dm_index_clear": (i32, [P, u32]),
        "dm_index_size": (i32, [P, u32, P]),
        "dm_route_batch": (i32, [P, P, u64, P, u64, P, P]),
        "dm_route_batch_noalloc": (i32, [P, P, u64, P, u64, P, P]),
        "dm_rebalance": (i32, [P, P, P, P, u64]),
        "dm_scale": (i32, [P, P, u32, P, u32, P, u64, P, P, P, P]),
        "dm_set_timing": (i32, [P, i32]),
        "dm_route_stage_ms": (i32, [P, P, i32]),
        "dm_set_pipelining": (i32, [P, i32]),
        "dm_set_policy": (i32, [P, i32]),
        "dm_kv_save": (i32, [P, P, u64, P, P, u64, u64, P, P]),
        "dm_queue_append": (i32, [P, P, P, u64, P, u64, P]),
        "dm_queue_migrate": (i32, [P, P, P, P, P, u64, P]),
        "dm_queue_drain": (i32, [P, P, P, P]),
        "dm_queue_reprobe": (i32, [P, P, P, P, u64, P, u64, P]),
        "dm_keylen_enable": (i32, [P, u64, u64]),
        "dm_keylen_window": (i32, [P]),
        "dm_keylen_export": (i32, [P, P, u64, P]),
        "dm_pages_fork": (i32, [P, P, P, u32, P, P, P, u64, P]),
        "dm_pages_compact": (i32, [P, P, P, u32, P]),
        "dm_pages_copy": (i32, [P, P, P, P, P, u64]),
        "dm_kv_append": (i32, [P, P, u32, P, P]),
        "dm_attn_plan_bytes": (u64, [u64, u64]),
        "dm_attn_plan": (i32, [P, P, P, u32, P, u64]),
        "dm_attn": (i32, [P, P, P, u32, P, u32, P, C.c_int64, C.c_float, P, C.c_int64, P]),
        "dm_sync": (i32, [P]),
        "dm_last_error": (C.c_char_p, [P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def __getattr__(name):
    # dm_* names resolve to the C functions
    if name in EXPORTS:
        return getattr(load_library(), name)
    raise AttributeError(name)


def make_config(cfg: Dict) -> dm_config:
    c = dm_config()
    c.block_size = cfg["block"]
    c.key_blocks = cfg["key_blocks"]
    c.seed[0], c.seed[1] = cfg["seeds"]
    c.vnodes = cfg["vnodes"]
    c.max_slots = cfg["max_slots"]
    c.index_log2_slots = cfg.get("index_log2_slots", 16)
    c.reserved = 0
    c.ttft_base_us = cfg.get("ttft_base_us", 2000)
    c.ttft_per_token_us = cfg.get("ttft_per_token_us", 3)
    c.queue_div = cfg.get("queue_div", 4)
    c.slo_us = cfg.get("slo_us", 400_000)
    return c


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


# dm_page_tables, dm_token_batch, dm_pages_out and dm_append_args as bytes: a decode step makes these calls for every
# layer, and packing takes a fraction of the time of filling a ctypes structure
_PACK_TABLES = struct.Struct("=5Q").pack
_PACK_BATCH = struct.Struct("=9Q").pack
_PACK_OUT = struct.Struct("=10Q").pack
_PACK_APPEND = struct.Struct("=3Q3qQq5Q3If").pack


class KVPages:
    """A store of KV pages (see dm_kv_pages): keys and values, torch tensors
    [layers, pages, kv_heads, block, head_dim] of one shape, bfloat16 or
    float16, each layer contiguous."""

    def __init__(self, k, v):
        import torch
        types = {torch.bfloat16: 0, torch.float16: 1}
        if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in types \
                or k.device != v.device:
            raise ValueError("k and v must be bfloat16 or float16 tensors of one shape "
                             "[layers, pages, kv_heads, block, head_dim] on one device")
        if k.shape[0] < 1 or k.shape[1] < 1 or k.stride() != v.stride() or not k[0].is_contiguous():
            raise ValueError("k and v need a layer and a page, the same strides and contiguous layers")
        self.k, self.v = k, v
        self.layers, self.pages, self.kv_heads, self.block, self.head_dim = k.shape
        self.dtype, self.index = k.dtype, k.get_device()
        stride = k.stride(0) if self.layers > 1 else k[0].numel()
        self.struct = dm_kv_pages(k.data_ptr(), v.data_ptr(), stride, self.layers, self.pages,
                                  self.kv_heads, self.head_dim, types[k.dtype], 0)
        self._ref = C.byref(self.struct)


class AttnPlan:
    """A plan of DualMap.attn_plan: the batch that it was made for."""

    def __init__(self, batch, q_tokens, kv, q_heads, buf, keep):
        self.batch, self.q_tokens, self.kv, self.q_heads, self.buf = batch, q_tokens, kv, q_heads, buf
        self._keep = keep  # the batch's tensors


def _current_stream(index):
    """The current stream's handle, by torch's short way where it has one."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw else torch.cuda.current_stream(index).cuda_stream


class DualMap:
    """A routing engine context on one GPU (torch tensors in and out)."""

    def __init__(self, cfg: Dict, device=None, stream=None):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.device = torch.device("cuda", torch.cuda.current_device() if device is None
                                   else torch.device(device).index or 0)
        self._index = self.device.index
        self.cfg = dict(cfg)
        self.max_slots = cfg["max_slots"]
        self.block = cfg["block"]
        with torch.cuda.device(self.device):
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            self._raw_stream = self.stream.cuda_stream
            h = C.c_void_p()
            st = self.lib.dm_create(C.byref(make_config(cfg)), C.c_void_p(self.stream.cuda_stream),
                                    C.byref(h))
        if st != DM_OK:
            raise DMError(st, "dm_create rejected the configuration %r" % (cfg,))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            self.lib.dm_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers ----------------------------------------------------------
    def _check(self, st: int, what: str):
        if st != DM_OK:
            raise DMError(st, f"{what}: {self.lib.dm_last_error(self._h).decode()}")

    def _dev(self, t, dtype, name):
        try:
            ok = t.dtype is dtype and t.get_device() == self._index and t.is_contiguous()
        except AttributeError:  # no tensor
            ok = False
        if not ok:
            raise ValueError(f"{name} must be a contiguous {dtype} tensor on {self.device}")
        return t

    def _empty(self, n, dtype):
        return self.torch.empty(max(int(n), 0), dtype=dtype, device=self.device)

    # -- C ABI mirrors --------------------------------------------------------
    def set_timing(self, on: bool) -> None:
        self._check(self.lib.dm_set_timing(self._h, 1 if on else 0), "dm_set_timing")

    def set_pipelining(self, on: bool) -> None:
        """Overlap each batch's selection with the next batch's hashing and
        probing (see dm_set_pipelining): consecutive batches need distinct
        output buffers, and results are final after sync()."""
        self._check(self.lib.dm_set_pipelining(self._h, 1 if on else 0), "dm_set_pipelining")

    POLICIES = {"slo_aware": 0, "cache_affinity": 1, "least_loaded": 2, "min_ttft": 3}

    def set_policy(self, policy) -> None:
        """Selection rule of later batches (see dm_set_policy): a name of
        POLICIES or its number."""
        p = self.POLICIES[policy] if isinstance(policy, str) else int(policy)
        self._check(self.lib.dm_set_policy(self._h, p), "dm_set_policy")

    def stage_ms(self):
        """(hash, lookup+match, selection, block offsets) ms, averaged over the
        batches routed since timing was turned on (the last 64 at most)."""
        ms = (C.c_float * 4)()
        self._check(self.lib.dm_route_stage_ms(self._h, ms, 4), "dm_route_stage_ms")
        return tuple(float(x) for x in ms)

    def sync(self) -> None:
        self._check(self.lib.dm_sync(self._h), "dm_sync")

    def build_rings(self, ids: Sequence[int]) -> None:
        arr = (C.c_uint32 * len(ids))(*[int(i) for i in ids])
        self._check(self.lib.dm_build_rings(self._h, arr, len(ids)), "dm_build_rings")

    def ring(self, s: int):
        import numpy as np
        n = C.c_uint64()
        self._check(self.lib.dm_ring_export(self._h, s, None, None, 0, C.byref(n)), "dm_ring_export")
        pos = np.zeros(n.value, np.uint64)
        ids = np.zeros(n.value, np.uint32)
        self._check(self.lib.dm_ring_export(self._h, s, pos.ctypes.data_as(C.c_void_p),
                                            ids.ctypes.data_as(C.c_void_p), n.value, C.byref(n)),
                    "dm_ring_export")
        return pos, ids

    def index_insert(self, inst: int, keys) -> None:
        keys = self._dev(keys, self.torch.uint64, "keys")
        self._check(self.lib.dm_index_insert(self._h, inst, _ptr(keys), keys.numel()),
                    "dm_index_insert")

    def index_erase(self, inst: int, keys) -> None:
        keys = self._dev(keys, self.torch.uint64, "keys")
        self._check(self.lib.dm_index_erase(self._h, inst, _ptr(keys), keys.numel()),
                    "dm_index_erase")

    def index_clear(self, inst: int) -> None:
        self._check(self.lib.dm_index_clear(self._h, inst), "dm_index_clear")

    def index_size(self, inst: int) -> int:
        n = C.c_uint64()
        self._check(self.lib.dm_index_size(self._h, inst, C.byref(n)), "dm_index_size")
        return int(n.value)

    def route_into(self, tokens, offsets, loads, out: Dict, noalloc: bool = False) -> None:
        """dm_route_batch into preallocated outputs; with noalloc,
        dm_route_batch_noalloc (work arrays from the library's static area)."""
        n = offsets.numel() - 1
        ro = dm_route_out(_ptr(out["key"]), _ptr(out["cand"]), _ptr(out["match"]),
                          _ptr(out["chosen"]), _ptr(out["ttft"]), _ptr(out["flags"]),
                          _ptr(out.get("block_keys")), _ptr(out.get("key_len")))
        fn = self.lib.dm_route_batch_noalloc if noalloc else self.lib.dm_route_batch
        name = "dm_route_batch_noalloc" if noalloc else "dm_route_batch"
        self._check(fn(self._h, _ptr(tokens), tokens.numel(), _ptr(offsets), n, _ptr(loads),
                       C.byref(ro)), name)

    def alloc_route_out(self, n: int, n_blocks: Optional[int] = None,
                        key_len: bool = False) -> Dict:
        t = self.torch
        out = dict(key=self._empty(2 * n, t.uint64), cand=self._empty(2 * n, t.uint32),
                   match=self._empty(2 * n, t.uint32), chosen=self._empty(n, t.uint32),
                   ttft=self._empty(n, t.int64), flags=self._empty(n, t.uint8))
        if n_blocks is not None:
            out["block_keys"] = self._empty(max(n_blocks, 1), t.uint64)
        if key_len:
            out["key_len"] = self._empty(max(n, 1), t.uint32)
        return out

    def kv_save(self, offsets, block_keys, inst, clock: int, cap: int):
        """Save a served batch's blocks with LRU eviction (see dm_kv_save);
        returns (keys added, keys removed)."""
        t = self.torch
        offsets = self._dev(offsets, t.int64, "offsets")
        block_keys = self._dev(block_keys, t.uint64, "block_keys")
        inst = self._dev(inst, t.uint32, "inst")
        a, r = C.c_uint64(), C.c_uint64()
        self._check(self.lib.dm_kv_save(self._h, _ptr(offsets), offsets.numel() - 1,
                                        _ptr(block_keys), _ptr(inst), int(clock), int(cap),
                                        C.byref(a), C.byref(r)), "dm_kv_save")
        return int(a.value), int(r.value)

    # -- queued requests on the device: tuples (qoff, rec_id, unc_here, alt,
    # unc_alt, base_work) of device tensors
    def _qin(self, q):
        t = self.torch
        qoff, rec, here, alt, there, base = q
        return (self._dev(qoff, t.int64, "qoff"), self._dev(rec, t.uint64, "rec_id"),
                self._dev(here, t.uint32, "unc_here"), self._dev(alt, t.uint32, "alt"),
                self._dev(there, t.uint32, "unc_alt"), self._dev(base, t.int64, "base_work"))

    def _qnew(self, cap: int):
        t = self.torch
        c = max(int(cap), 1)
        return (self._empty(self.max_slots + 1, t.int64), self._empty(c, t.uint64),
                self._empty(c, t.uint32), self._empty(c, t.uint32), self._empty(c, t.uint32),
                self._empty(self.max_slots, t.int64))

    @staticmethod
    def _qstructs(qi, qo, cap):
        qs = dm_queues(*[_ptr(x) for x in qi], None, 0)
        qd = dm_queue_out(*[_ptr(x) for x in qo], int(cap))
        return qs, qd

    def _qtrim(self, qo):
        n = int(qo[0][-1].item())
        return (qo[0], qo[1][:n], qo[2][:n], qo[3][:n], qo[4][:n], qo[5])

    def queue_append(self, q, offsets, routed: Dict, rec_base: int):
        """A routed batch joins the queues (see dm_queue_append)."""
        qi = self._qin(q)
        offsets = self._dev(offsets, self.torch.int64, "offsets")
        n = offsets.numel() - 1
        cap = qi[1].numel() + n
        qo = self._qnew(cap)
        qs, qd = self._qstructs(qi, qo, cap)
        ro = dm_route_out(_ptr(routed["key"]), _ptr(routed["cand"]), _ptr(routed["match"]),
                          _ptr(routed["chosen"]), _ptr(routed["ttft"]), _ptr(routed["flags"]),
                          None, None)
        self._check(self.lib.dm_queue_append(self._h, C.byref(qs), _ptr(offsets), n,
                                             C.byref(ro), int(rec_base), C.byref(qd)),
                    "dm_queue_append")
        return self._qtrim(qo)

    def queue_migrate(self, q, rec_id, src, dst):
        """A migration list applied to the queues (see dm_queue_migrate)."""
        t = self.torch
        qi = self._qin(q)
        rec_id = self._dev(rec_id, t.uint64, "rec_id")
        src = self._dev(src, t.uint32, "from")
        dst = self._dev(dst, t.uint32, "to")
        cap = qi[1].numel()
        qo = self._qnew(cap)
        qs, qd = self._qstructs(qi, qo, cap)
        self._check(self.lib.dm_queue_migrate(self._h, C.byref(qs), _ptr(rec_id), _ptr(src),
                                              _ptr(dst), rec_id.numel(), C.byref(qd)),
                    "dm_queue_migrate")
        return self._qtrim(qo)

    def queue_drain(self, q, units):
        """units[i] of service per instance (see dm_queue_drain)."""
        qi = self._qin(q)
        units = self._dev(units, self.torch.int64, "units")
        cap = qi[1].numel()
        qo = self._qnew(cap)
        qs, qd = self._qstructs(qi, qo, cap)
        self._check(self.lib.dm_queue_drain(self._h, C.byref(qs), _ptr(units), C.byref(qd)),
                    "dm_queue_drain")
        return self._qtrim(qo)

    def queue_reprobe(self, q, chain_off, chain_keys, prompt_len):
        """Queued records re-priced against the current caches (see
        dm_queue_reprobe): record id r's chain chain_keys[chain_off[r]:
        chain_off[r+1]], its prompt prompt_len[r] tokens."""
        t = self.torch
        qi = self._qin(q)
        chain_off = self._dev(chain_off, t.int64, "chain_off")
        chain_keys = self._dev(chain_keys, t.uint64, "chain_keys")
        prompt_len = self._dev(prompt_len, t.int64, "prompt_len")
        if chain_off.numel() != prompt_len.numel() + 1:
            raise ValueError("chain_off needs one entry more than prompt_len")
        cap = qi[1].numel()
        qo = self._qnew(cap)
        qs, qd = self._qstructs(qi, qo, cap)
        self._check(self.lib.dm_queue_reprobe(self._h, C.byref(qs), _ptr(chain_off),
                                              _ptr(chain_keys), chain_keys.numel(),
                                              _ptr(prompt_len), prompt_len.numel(), C.byref(qd)),
                    "dm_queue_reprobe")
        return self._qtrim(qo)

    def keylen_enable(self, max_nodes: int, max_window_blocks: int = 1 << 24) -> None:
        """Adaptive hash-key length (see dm_keylen_enable): an empty prefix
        hotness tree with room for max_nodes extended prefixes and a window
        record of max_window_blocks prefixes; max_nodes = 0 turns it off."""
        self._check(self.lib.dm_keylen_enable(self._h, int(max_nodes), int(max_window_blocks)),
                    "dm_keylen_enable")

    def keylen_window(self) -> None:
        """Close the hotness window: hot leaves extend, cold nodes shrink."""
        self._check(self.lib.dm_keylen_window(self._h), "dm_keylen_window")

    def keylen_tree(self):
        """The extended prefixes (canonical f1 keys), ascending, as numpy."""
        import numpy as np
        n = C.c_uint64()
        self._check(self.lib.dm_keylen_export(self._h, None, 0, C.byref(n)), "dm_keylen_export")
        a = np.zeros(max(int(n.value), 1), np.uint64)
        self._check(self.lib.dm_keylen_export(self._h, a.ctypes.data_as(C.c_void_p), len(a),
                                              C.byref(n)), "dm_keylen_export")
        return a[:int(n.value)]

    def route(self, tokens, offsets, loads, block_keys: bool = False) -> Dict:
        """Route a batch; loads (int64 [max_slots]) are updated in place."""
        t = self.torch
        tokens = self._dev(tokens, t.int32, "tokens")
        offsets = self._dev(offsets, t.int64, "offsets")
        loads = self._dev(loads, t.int64, "loads")
        if loads.numel() != self.max_slots:
            raise ValueError("loads must have max_slots entries")
        n = offsets.numel() - 1
        nb = None
        if block_keys:
            nb = int(((offsets[1:] - offsets[:-1]).clamp(min=0) // self.block).sum().item())
        out = self.alloc_route_out(n, nb, key_len=True)
        self.route_into(tokens, offsets, loads, out)
        return out

    def rebalance(self, qoff, rec_id, unc_here, alt, unc_alt, base_work, cap: Optional[int] = None,
                  prefill_interval=None, decode_threshold_us: int = 3_000_000):
        t = self.torch
        qoff = self._dev(qoff, t.int64, "qoff")
        rec_id = self._dev(rec_id, t.uint64, "rec_id")
        unc_here = self._dev(unc_here, t.uint32, "unc_here")
        alt = self._dev(alt, t.uint32, "alt")
        unc_alt = self._dev(unc_alt, t.uint32, "unc_alt")
        base_work = self._dev(base_work, t.int64, "base_work")
        if qoff.numel() != self.max_slots + 1 or base_work.numel() != self.max_slots:
            raise ValueError("qoff needs max_slots + 1 entries and base_work max_slots")
        if prefill_interval is not None:
            prefill_interval = self._dev(prefill_interval, t.int64, "prefill_interval")
            if prefill_interval.numel() != self.max_slots:
                raise ValueError("prefill_interval needs max_slots entries")
        cap = rec_id.numel() if cap is None else cap
        m = dict(rec=self._empty(max(cap, 1), t.uint64), src=self._empty(max(cap, 1), t.uint32),
                 dst=self._empty(max(cap, 1), t.uint32), benefit=self._empty(max(cap, 1), t.int64),
                 ttft_to=self._empty(max(cap, 1), t.int64), count=self._empty(1, t.uint64))
        loads = self._empty(self.max_slots, t.int64)
        q = dm_queues(_ptr(qoff), _ptr(rec_id), _ptr(unc_here), _ptr(alt), _ptr(unc_alt),
                      _ptr(base_work),
                      _ptr(prefill_interval), int(decode_threshold_us))
        mg = dm_migrations(_ptr(m["rec"]), _ptr(m["src"]), _ptr(m["dst"]), _ptr(m["benefit"]),
                           _ptr(m["ttft_to"]), _ptr(m["count"]))
        self._check(self.lib.dm_rebalance(self._h, C.byref(q), _ptr(loads), C.byref(mg), cap),
                    "dm_rebalance")
        m["loads"] = loads
        return m

    def scale(self, add: Sequence[int], rm: Sequence[int], keys) -> Dict:
        t = self.torch
        keys = self._dev(keys, t.uint64, "keys")
        n = keys.numel() // 2
        a = (C.c_uint32 * max(len(add), 1))(*[int(i) for i in add])
        r = (C.c_uint32 * max(len(rm), 1))(*[int(i) for i in rm])
        out = dict(old=self._empty(2 * n, t.uint32), new=self._empty(2 * n, t.uint32),
                   moved=self._empty(2, t.uint64), violations=self._empty(1, t.uint64))
        self._check(self.lib.dm_scale(self._h, a, len(add), r, len(rm), _ptr(keys), n,
                                      _ptr(out["old"]), _ptr(out["new"]), _ptr(out["moved"]),
                                      _ptr(out["violations"])), "dm_scale")
        return out

    # -- KV pages and attention over them: tables are tuples (off, page, len)
    # of device tensors (int64 [n + 1], int32, int64 [n])
    def _tables(self, tables):
        """dm_page_tables' fields."""
        t = self.torch
        off, page, length = tables
        self._dev(off, t.int64, "off")
        self._dev(page, t.int32, "page")
        self._dev(length, t.int64, "len")
        n = length.numel()
        if off.numel() != n + 1:
            raise ValueError("off needs one entry more than len")
        return off.data_ptr(), page.data_ptr(), length.data_ptr(), n, page.numel()

    def _kv(self, kv):
        if kv.index != self._index or kv.block != self.block:
            raise ValueError("pages must be on %s and hold %d tokens" % (self.device, self.block))
        return kv

    def _pages_out(self, out, n_pages, m=None):
        dev, i32, i64 = self._dev, self.torch.int32, self.torch.int64
        page, ref = dev(out["page"], i32, "page"), dev(out["ref"], i32, "ref")
        src, dst = dev(out["move_src"], i32, "move_src"), dev(out["move_dst"], i32, "move_dst")
        moves = dev(out["moves"], i64, "moves")
        off = length = live = 0
        cap, room = page.numel(), src.numel()
        ok = ref.numel() == n_pages and moves.numel() == 1 and dst.numel() == room
        if m is not None:
            off, length = dev(out["off"], i64, "off"), dev(out["len"], i64, "len")
            ok = ok and off.numel() == m + 1 and length.numel() == m
            off, length = off.data_ptr(), length.data_ptr()
        else:
            live = dev(out["live"], i64, "live")
            ok = ok and live.numel() == 1
            live = live.data_ptr()
        if not ok:
            raise ValueError("an output has the wrong size")
        return _PACK_OUT(off, page.data_ptr(), length, cap, ref.data_ptr(), src.data_ptr(),
                         dst.data_ptr(), room, moves.data_ptr(), live), cap

    def alloc_pages_out(self, n_pages: int, m: int, cap: int) -> Dict:
        """Outputs of pages_fork_into for m sequences and cap entries (and, with cap the
        tables' entries, of pages_compact_into)."""
        t = self.torch
        moves = max(m, n_pages // 2 + 1)
        return dict(off=self._empty(m + 1, t.int64), page=self._empty(cap, t.int32),
                    len=self._empty(m, t.int64), ref=self._empty(n_pages, t.int32),
                    move_src=self._empty(moves, t.int32), move_dst=self._empty(moves, t.int32),
                    moves=self._empty(1, t.int64), live=self._empty(1, t.int64))

    def pages_fork_into(self, tables, ref, src, keep, grow, out: Dict) -> None:
        """The tables of the next step (see dm_pages_fork) into preallocated
        outputs: sequence j holds the first keep[j] tokens of src[j] and room
        for grow[j] more.  out["move_src"], out["move_dst"] and out["moves"]
        are pages_copy's list."""
        t = self.torch
        tb = self._tables(tables)
        ref = self._dev(ref, t.int32, "ref")
        src = self._dev(src, t.int32, "src")
        keep = self._dev(keep, t.int64, "keep")
        grow = self._dev(grow, t.int64, "grow")
        m = src.numel()
        if keep.numel() != m or grow.numel() != m:
            raise ValueError("src, keep and grow must have one length")
        o, _ = self._pages_out(out, ref.numel(), m)
        self._check(self.lib.dm_pages_fork(self._h, _PACK_TABLES(*tb), ref.data_ptr(), ref.numel(),
                                           src.data_ptr(), keep.data_ptr(), grow.data_ptr(), m, o),
                    "dm_pages_fork")

    def pages_fork(self, tables, ref, src, keep, grow, cap: int) -> Dict:
        """pages_fork_into with outputs of its own (cap entries); page is cut
        to the entries there are, which waits for the device."""
        out = self.alloc_pages_out(ref.numel(), src.numel(), cap)
        self.pages_fork_into(tables, ref, src, keep, grow, out)
        self.sync()
        out["page"] = out["page"][:int(out["off"][-1].item())]
        return out

    def pages_compact_into(self, tables, ref, out: Dict) -> None:
        """Live pages moved together (see dm_pages_compact): out["page"], out["ref"],
        out["live"] and the list of moves for pages_copy."""
        tb = self._tables(tables)
        ref = self._dev(ref, self.torch.int32, "ref")
        o, cap = self._pages_out(out, ref.numel())
        if cap < tb[4]:
            raise ValueError("page needs room for the tables' entries")
        self._check(self.lib.dm_pages_compact(self._h, _PACK_TABLES(*tb), ref.data_ptr(), ref.numel(), o),
                    "dm_pages_compact")

    def pages_copy(self, kv: KVPages, moves: Dict) -> None:
        """Page data moved by a list of pages_fork or pages_compact (see dm_pages_copy)."""
        t = self.torch
        self._kv(kv)
        src = self._dev(moves["move_src"], t.int32, "move_src")
        dst = self._dev(moves["move_dst"], t.int32, "move_dst")
        count = self._dev(moves["moves"], t.int64, "moves")
        if src.numel() != dst.numel() or count.numel() != 1:
            raise ValueError("move_src and move_dst must have one length, moves one entry")
        self._check(self.lib.dm_pages_copy(self._h, kv._ref, src.data_ptr(), dst.data_ptr(),
                                           count.data_ptr(), src.numel()), "dm_pages_copy")

    def _batch(self, tables, q_off, q_tokens, groups=None):
        """dm_token_batch's fields."""
        i64 = self.torch.int64
        tb = self._tables(tables)
        if self._dev(q_off, i64, "q_off").numel() != tb[3] + 1:
            raise ValueError("q_off needs one entry more than len")
        if not 0 <= q_tokens < 1 << 31:
            raise ValueError("q_tokens must be at least 0 and below 2^31")
        if groups is None:
            return tb + (q_off.data_ptr(), q_tokens, 0, 0)
        if self._dev(groups, i64, "groups").numel() < 1:
            raise ValueError("groups needs one entry more than there are runs")
        return tb + (q_off.data_ptr(), q_tokens, groups.data_ptr(), groups.numel() - 1)

    def _rows(self, x, name, heads, dim, tokens, dtype):
        """Address and row stride of [tokens, heads, dim] with contiguous heads."""
        if x.dtype is not dtype or x.shape != (tokens, heads, dim) or x.get_device() != self._index:
            raise ValueError(f"{name} must be a {dtype} tensor {(tokens, heads, dim)} on {self.device}")
        a, b, c = x.stride()
        if tokens and (c != 1 or (heads > 1 and b != dim)):
            raise ValueError(f"{name}'s heads must be contiguous")
        return x.data_ptr(), a if tokens > 1 else heads * dim

    def kv_append(self, kv: KVPages, layer: int, tables, q_off, q, k, v, q_out, q_norm=None,
                  k_norm=None, eps: float = 1e-6, cos=None, sin=None, interleaved: bool = False) -> None:
        """New tokens' queries and keys normed per head and rotated, keys and
        values written to layer's pages (see dm_kv_append).  q, q_out: [tokens,
        q_heads, head_dim]; k, v: [tokens, kv_heads, head_dim]; cos, sin: float32
        [positions, rot_dim / 2]."""
        self._kv(kv)
        T, D, dt = q.shape[0], kv.head_dim, kv.dtype
        heads = q.shape[1]
        b = self._batch(tables, q_off, T)
        qp, qs = self._rows(q, "q", heads, D, T, dt)
        kp, ks = self._rows(k, "k", kv.kv_heads, D, T, dt)
        vp, vs = self._rows(v, "v", kv.kv_heads, D, T, dt)
        op, os_ = self._rows(q_out, "q_out", heads, D, T, dt)
        wq = wk = cp = sp = rot = rows = 0
        if q_norm is not None:
            wq = self._dev(q_norm, dt, "q_norm").data_ptr()
        if k_norm is not None:
            wk = self._dev(k_norm, dt, "k_norm").data_ptr()
        if (q_norm is not None and q_norm.numel() != D) or (k_norm is not None and k_norm.numel() != D):
            raise ValueError("q_norm and k_norm need head_dim weights")
        if cos is not None or sin is not None:
            f32 = self.torch.float32
            cp, sp = self._dev(cos, f32, "cos").data_ptr(), self._dev(sin, f32, "sin").data_ptr()
            if cos.dim() != 2 or cos.shape != sin.shape:
                raise ValueError("cos and sin must be [positions, rot_dim / 2]")
            rows, rot = cos.shape
            rot *= 2
        a = _PACK_APPEND(qp, kp, vp, qs, ks, vs, op, os_, wq, wk, cp, sp, rows, heads, rot,
                         1 if interleaved else 0, eps)
        self._check(self.lib.dm_kv_append(self._h, kv._ref, layer, _PACK_BATCH(*b), a), "dm_kv_append")

    def attn_plan(self, kv: KVPages, tables, q_off, q_tokens: int, q_heads: int, groups=None) -> AttnPlan:
        """The work of attn for a batch (see dm_attn_plan), once for all layers.
        groups: int64 [runs + 1], the runs of sequences that may share a prefix."""
        self._kv(kv)
        b = self._batch(tables, q_off, q_tokens, groups)
        need = self.lib.dm_attn_plan_bytes(b[3], b[8])
        # of the context's stream, whose work is all that the memory has to outlive
        torch = self.torch
        if _current_stream(self._index) == self._raw_stream:
            buf = torch.empty(need, dtype=torch.uint8, device=self.device)
        else:
            with torch.cuda.stream(self.stream):
                buf = torch.empty(need, dtype=torch.uint8, device=self.device)
        batch = _PACK_BATCH(*b)
        self._check(self.lib.dm_attn_plan(self._h, batch, kv._ref, q_heads, buf.data_ptr(), need),
                    "dm_attn_plan")
        return AttnPlan(batch, q_tokens, kv, q_heads, buf, (tables, q_off, groups))

    def attn(self, plan: AttnPlan, layer: int, q, scale: float, out, lse=None) -> None:
        """Attention of a batch's new tokens over layer's pages (see dm_attn): q
        and out [tokens, q_heads, head_dim], lse float32 [tokens, q_heads]."""
        kv, T, heads = plan.kv, plan.q_tokens, plan.q_heads
        qp, qs = self._rows(q, "q", heads, kv.head_dim, T, kv.dtype)
        op, os_ = self._rows(out, "out", heads, kv.head_dim, T, kv.dtype)
        lp = None
        if lse is not None:
            lp = self._dev(lse, self.torch.float32, "lse").data_ptr()
            if lse.shape != (T, heads):
                raise ValueError("lse must be [tokens, q_heads]")
        self._check(self.lib.dm_attn(self._h, plan.batch, kv._ref, heads, plan.buf.data_ptr(), layer, qp,
                                     qs, scale, op, os_, lp), "dm_attn")
