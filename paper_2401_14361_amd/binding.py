"""ctypes binding of libmoei.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/moei.h) and
takes torch CUDA tensors for device buffers; outputs are allocated with torch
(device memory plumbing) and filled by the library's kernels.  A missing library
is an error: there is no CPU fallback.

With `stream=` a call's work is queued there, and the tensors that it allocates belong to that stream, as those of any
torch operation under torch.cuda.stream(stream) do.  Ordering is the caller's: `stream` waits for whoever wrote the inputs, and
whoever uses the outputs waits for `stream` (events, wait_stream; record_stream for tensors given up while another stream uses them).
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

__all__ = [
    "MoeiError", "ModelDesc", "lib", "lib_path", "Eamc", "Cache",
    "moe_route_topk", "eam_update", "eamc_match", "eamc_match_topm", "expert_priority", "expert_ffn_gemv",
    "expert_ffn_gemv_static",
    "moe_decode_layer", "moe_prefill_layer", "expert_ffn_grouped", "WDTYPE_FP32", "WDTYPE_BF16", "EXPORTS", "expert_pack", "profile_enable", "profile_disable", "profile_read", "profile_samples",
    "Kv", "KvDesc", "KvPages", "kv_append", "kv_append_norm", "kv_attend", "kv_attend_blocks", "kv_attend_shared", "kv_attend_weights", "kv_evict", "KVDTYPE_FP8",
]

WDTYPE_FP32, WDTYPE_BF16 = 0, 1
KVDTYPE_FP8 = 2
_HERE = os.path.dirname(os.path.abspath(__file__))

EXPORTS = [
    "moei_last_error", "moei_version",
    "moei_eamc_create", "moei_eamc_load", "moei_eamc_insert", "moei_eamc_export", "moei_eamc_save", "moei_eamc_restore", "moei_eamc_size", "moei_eamc_destroy",
    "moe_route_topk", "eam_update", "eamc_match", "eamc_match_topm", "expert_priority",
    "moei_cache_create", "moei_cache_destroy", "moei_expert_pack", "moei_cache_reset", "moei_cache_slot_ptr", "moei_cache_slot_table",
    "moei_cache_get_slots", "moei_cache_retrieve", "expert_ffn_gemv", "expert_ffn_gemv_static", "expert_ffn_grouped", "moei_cache_error_flags",
    "moe_decode_layer", "moei_cache_last_step", "moei_cache_last_heads", "moei_cache_join", "moei_cache_sync",
    "moei_cache_set_match_count", "moei_cache_last_matches",
    "moe_prefill_layer", "moei_cache_set_policy", "moei_cache_prefetch", "moei_cache_set_prefetch", "moei_cache_last_prefetch",
    "moei_kv_create", "moei_kv_destroy", "moei_kv_error_flags", "moei_kv_set_weights", "moei_kv_set_shared",
    "kv_append", "kv_append_norm", "kv_attend", "kv_attend_blocks", "kv_attend_shared", "kv_attend_weights", "kv_evict",
    "moei_profile_enable", "moei_profile_disable", "moei_profile_kernels", "moei_profile_kernel_name",
    "moei_profile_read", "moei_profile_samples",
]


class MoeiError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"moei error {code}: {msg}")
        self.code = code


class ModelDesc(C.Structure):
    _fields_ = [("L", C.c_int32), ("E", C.c_int32), ("k", C.c_int32), ("n_shared", C.c_int32),
                ("H", C.c_int32), ("I", C.c_int32), ("wdtype", C.c_int32), ("renorm_topk", C.c_int32),
                ("eps", C.c_float)]

    @classmethod
    def from_config(cls, cfg, eps: float = 2.0 ** -20) -> "ModelDesc":
        return cls(cfg.L, cfg.E, cfg.k, cfg.n_shared, cfg.H, cfg.I,
                   WDTYPE_FP32 if cfg.wdtype == "fp32" else WDTYPE_BF16, int(cfg.renorm), eps)


def lib_path() -> str:
    return os.path.join(_HERE, "libmoei.so")


_lib = None


def lib() -> C.CDLL:
    """The loaded HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        p = lib_path()
        if not os.path.exists(p):
            raise FileNotFoundError(f"{p} is missing: run `python -m paper_2401_14361_amd.build` "
                                    "(or __graft_entry__.build()) first; there is no CPU fallback")
        L = C.CDLL(p)
        L.moei_last_error.restype = C.c_char_p
        L.moei_version.restype = C.c_char_p
        for name in EXPORTS[2:]:
            getattr(L, name).restype = C.c_int
        L.moei_profile_kernel_name.restype = C.c_char_p
        P, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        L.kv_append.argtypes = [P, P, P, i32, i32, P, P, i32, P, i64, P, i64, P, i64, P, i32, i32, P, P]
        L.moei_kv_set_weights.argtypes = [P, i64]
        L.moei_kv_set_shared.argtypes = [P, i32]
        L.kv_attend_shared.argtypes = [P, P, P, i32, P, i32, P, P, i32, P, i64, f32, P, P, P]
        L.kv_attend_weights.argtypes = [P, P, P, i32, P, i32, P, i64, f32, i32, P, i64, P, P, P]
        L.kv_evict.argtypes = [P, P, P, i32, P, i32, P, i64, i32, i32, i32, P, i32, P, P, i64, P, P]
        L.kv_append_norm.argtypes = [P, P, P, i32, i32, P, P, P, i32, P, i64, P, i64, P, i64, P, P, i32, f32, P, i32, i32, P, P]
        L.kv_attend.argtypes = [P, P, P, i32, P, i32, P, i64, f32, i32, P, P, P]
        L.kv_attend_blocks.argtypes = [P, P, P, i32, P, i32, P, i64, f32, i32, i32, i32, P, P, P, P]
        _lib = L
    return _lib


def _check(rc: int) -> int:
    if rc < 0:
        raise MoeiError(rc, lib().moei_last_error().decode())
    return rc


def _p(t) -> C.c_void_p:
    if t is None:
        return C.c_void_p(0)
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous(), "tensors handed to the library must be contiguous"
        return C.c_void_p(t.data_ptr())
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"]
        return C.c_void_p(t.ctypes.data)
    return C.c_void_p(int(t))


def _stream(stream=None) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _elsewhere(stream, device: int):
    """The torch stream that `stream` (a torch stream or a handle) names, None if it is the device's current one."""
    if stream is None:
        return None
    at = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if at == torch._C._cuda_getCurrentRawStream(device):
        return None
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(at, device=device) if at else torch.cuda.default_stream(device)


def _new(shape, dtype, device: torch.device, stream) -> torch.Tensor:
    """A tensor that the call on `stream` fills: from that stream's memory, which nothing queued on another one still uses."""
    on = _elsewhere(stream, device.index)
    if on is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(on):
        return torch.empty(shape, dtype=dtype, device=device)


def _dev(t: torch.Tensor, dtype) -> torch.Tensor:
    assert t.is_cuda and t.dtype == dtype and t.is_contiguous(), (t.device, t.dtype, dtype)
    return t


# ---------------------------------------------------------------------------- objects
class Eamc:
    """Owner of a moei_eamc handle."""

    def __init__(self, desc: ModelDesc, n_cap: int, cell_bytes: int = 4):
        self.desc, self.n_cap, self.cell_bytes = desc, n_cap, cell_bytes
        self.h = C.c_void_p(0)
        _check(lib().moei_eamc_create(C.byref(desc), n_cap, cell_bytes, C.byref(self.h)))

    def load(self, traces: np.ndarray) -> None:
        traces = np.ascontiguousarray(traces, dtype=np.int32)
        N = traces.shape[0]
        assert traces.shape[1:] == (self.desc.L, self.desc.E) or N == 0
        _check(lib().moei_eamc_load(self.h, _p(traces), N))

    def insert(self, eam: np.ndarray, victim: int = -1) -> None:
        eam = np.ascontiguousarray(eam, dtype=np.int32)
        assert eam.shape == (self.desc.L, self.desc.E)
        _check(lib().moei_eamc_insert(self.h, _p(eam), victim))

    def export(self) -> np.ndarray:
        out = np.zeros((self.size, self.desc.L, self.desc.E), dtype=np.int32)
        _check(lib().moei_eamc_export(self.h, _p(out), out.shape[0]))
        return out

    def save(self, path: str) -> None:
        """Checkpoint file of the collection (failure recovery)."""
        _check(lib().moei_eamc_save(self.h, os.fsencode(path)))

    def restore(self, path: str) -> None:
        _check(lib().moei_eamc_restore(self.h, os.fsencode(path)))

    @property
    def size(self) -> int:
        return _check(lib().moei_eamc_size(self.h))

    def close(self) -> None:
        if self.h:
            lib().moei_eamc_destroy(self.h)
            self.h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache:
    """Owner of a moei_cache handle (slot pool, slot table, per-layer scratch)."""

    def __init__(self, desc: ModelDesc, n_slots: int, h_experts: torch.Tensor | np.ndarray | None = None,
                 h_shared: torch.Tensor | np.ndarray | None = None):
        self.desc, self.n_slots = desc, n_slots
        self._keep = (h_experts, h_shared)      # the library reads the host copy on every miss
        n_host = 0 if h_experts is None else int(h_experts.shape[0])
        self.h = C.c_void_p(0)
        _check(lib().moei_cache_create(C.byref(desc), n_slots, _p(h_experts), n_host, _p(h_shared), C.byref(self.h)))
        self.slot_elems = 3 * desc.H * desc.I

    def reset(self, n_resident: int) -> None:
        _check(lib().moei_cache_reset(self.h, n_resident))

    def slot_ptr(self, slot: int) -> int:
        out = C.c_void_p(0)
        _check(lib().moei_cache_slot_ptr(self.h, slot, C.byref(out)))
        return out.value

    def slot_tensor(self, slot: int) -> torch.Tensor:
        """A torch view of one slot's weights on the device (no copy, no ownership)."""
        fp32 = self.desc.wdtype == WDTYPE_FP32

        class _View:
            pass

        v = _View()
        v.__cuda_array_interface__ = {"shape": (self.slot_elems,), "typestr": "<f4" if fp32 else "<i2",
                                      "data": (self.slot_ptr(slot), False), "version": 2}
        t = torch.as_tensor(v, device="cuda")
        return t if fp32 else t.view(torch.bfloat16)

    def slot_table(self) -> int:
        out = C.c_void_p(0)
        _check(lib().moei_cache_slot_table(self.h, C.byref(out)))
        return out.value

    def get_slots(self) -> np.ndarray:
        out = np.empty(self.desc.L * self.desc.E, dtype=np.int32)
        _check(lib().moei_cache_get_slots(self.h, _p(out)))
        return out

    def retrieve(self, layer: int, idx, ev_order, stream=None):
        idx = np.ascontiguousarray(idx, dtype=np.int32)
        ev = np.ascontiguousarray(ev_order, dtype=np.int32)
        n = idx.shape[0]
        slots = np.empty(n, dtype=np.int32)
        victims = np.empty(n, dtype=np.int32)
        n_miss = C.c_int32(0)
        _check(lib().moei_cache_retrieve(self.h, layer, _p(idx), n, _p(ev), ev.shape[0], _p(slots), _p(victims),
                                         C.byref(n_miss), _stream(stream)))
        return slots, victims, n_miss.value

    def error_flags(self, stream=None) -> int:
        f = C.c_int32(0)
        _check(lib().moei_cache_error_flags(self.h, C.byref(f), _stream(stream)))
        return f.value

    def join(self, stream=None) -> None:
        _check(lib().moei_cache_join(self.h, _stream(stream)))

    def sync(self) -> None:
        _check(lib().moei_cache_sync(self.h))

    def last_heads(self, stream=None):
        """(pf_head, ev_head): the leading entries of the two orders as the last layer step selected them."""
        pf = np.empty(64, dtype=np.int32)
        ev = np.empty(128, dtype=np.int32)
        n_pf, n_ev = C.c_int32(0), C.c_int32(0)
        _check(lib().moei_cache_last_heads(self.h, _p(pf), pf.size, C.byref(n_pf), _p(ev), ev.size, C.byref(n_ev),
                                           _stream(stream)))
        return pf[:n_pf.value].copy(), ev[:n_ev.value].copy()

    def last_step(self, stream=None) -> dict:
        LE, k = self.desc.L * self.desc.E, self.desc.k
        w = np.empty(k, dtype=np.float32)
        sim = C.c_float(0)
        P = np.empty(LE, dtype=np.float32)
        V = np.empty(LE, dtype=np.float32)
        pf = np.empty(LE, dtype=np.int32)
        ev = np.empty(LE, dtype=np.int32)
        n_pf, n_ev = C.c_int32(0), C.c_int32(0)
        _check(lib().moei_cache_last_step(self.h, _p(w), C.byref(sim), _p(P), _p(V), _p(pf), C.byref(n_pf), _p(ev),
                                          C.byref(n_ev), _stream(stream)))
        return dict(w=w, sim=sim.value, P=P.reshape(self.desc.L, self.desc.E), V=V.reshape(self.desc.L, self.desc.E),
                    pf_order=pf[:n_pf.value].copy(), ev_order=ev[:n_ev.value].copy())

    POLICIES = {"eam": 0, "lru": 1, "count": 2}

    def set_policy(self, policy: str) -> None:
        """Eviction rule: "eam" (Alg. 1, default), "lru" or "count" (the comparison rules)."""
        _check(lib().moei_cache_set_policy(self.h, self.POLICIES[policy]))

    def set_prefetch(self, depth: int) -> None:
        """Prefetch candidates considered after each synchronous layer step (0 = off)."""
        _check(lib().moei_cache_set_prefetch(self.h, int(depth)))

    def prefetch(self, pf_order, ev_order, V, depth: int, protect=(), stream=None):
        """Sec. 4.6 prefetch step from host-side orders and fp32 scores -> list of (fid, victim, slot)."""
        pf = np.ascontiguousarray(np.asarray(pf_order, dtype=np.int32).reshape(-1))
        ev = np.ascontiguousarray(np.asarray(ev_order, dtype=np.int32).reshape(-1))
        Vf = np.ascontiguousarray(np.asarray(V, dtype=np.float32).reshape(-1))
        assert Vf.size == self.desc.L * self.desc.E
        pr = np.ascontiguousarray(np.asarray(list(protect), dtype=np.int32).reshape(-1))
        n = max(int(depth), 1)
        fids, vic, slots = (np.empty(n, dtype=np.int32) for _ in range(3))
        issued = C.c_int32(0)
        _check(lib().moei_cache_prefetch(self.h, _p(pf) if pf.size else None, pf.size, _p(ev) if ev.size else None,
                                         ev.size, _p(Vf), int(depth), _p(pr) if pr.size else None, pr.size,
                                         _p(fids), _p(vic), _p(slots), C.byref(issued), _stream(stream)))
        m = issued.value
        return [(int(fids[i]), int(vic[i]), int(slots[i])) for i in range(m)]

    def last_prefetch(self):
        fids, vic = np.empty(32, dtype=np.int32), np.empty(32, dtype=np.int32)
        n = C.c_int32(0)
        _check(lib().moei_cache_last_prefetch(self.h, _p(fids), _p(vic), 32, C.byref(n)))
        return [(int(fids[i]), int(vic[i])) for i in range(n.value)]

    def set_match_count(self, m: int) -> None:
        """Traces aggregated by the layer step's prediction (Sec. 4.5 step 2); default 1."""
        _check(lib().moei_cache_set_match_count(self.h, int(m)))

    def last_matches(self, stream=None):
        """(trace indices, similarities) matched by the last layer step, most similar first."""
        top = np.empty(16, dtype=np.int32)
        sim = np.empty(16, dtype=np.float32)
        m = C.c_int32(0)
        _check(lib().moei_cache_last_matches(self.h, _p(top), _p(sim), 16, C.byref(m), _stream(stream)))
        return top[:m.value].copy(), sim[:m.value].copy()

    def close(self) -> None:
        if self.h:
            lib().moei_cache_destroy(self.h)
            self.h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------------------------ entry points
def expert_pack(desc: ModelDesc, w_gate: np.ndarray, w_up: np.ndarray, w_down: np.ndarray,
                out: np.ndarray | None = None) -> np.ndarray:
    """W_gate [I][H], W_up [I][H], W_down [H][I] (host arrays in the storage dtype) -> one
    expert in slot layout, flat [3*H*I].  Data movement only."""
    H, I = desc.H, desc.I
    dt = np.float32 if desc.wdtype == WDTYPE_FP32 else np.uint16
    g = np.ascontiguousarray(w_gate, dtype=dt)
    u = np.ascontiguousarray(w_up, dtype=dt)
    d = np.ascontiguousarray(w_down, dtype=dt)
    assert g.shape == (I, H) and u.shape == (I, H) and d.shape == (H, I)
    if out is None:
        out = np.empty(3 * H * I, dtype=dt)
    assert out.dtype == dt and out.size == 3 * H * I and out.flags["C_CONTIGUOUS"]
    _check(lib().moei_expert_pack(C.byref(desc), _p(g), _p(u), _p(d), _p(out)))
    return out



def moe_route_topk(logits: torch.Tensor, k: int, renorm: bool, stream=None):
    """logits [B][E] fp32 (device) -> (idx [B][k] int32, w [B][k] fp32) on the device."""
    _dev(logits, torch.float32)
    B, E = logits.shape
    idx = _new((B, k), torch.int32, logits.device, stream)
    w = _new((B, k), torch.float32, logits.device, stream)
    _check(lib().moe_route_topk(_p(logits), B, E, k, int(renorm), _p(idx), _p(w), _stream(stream)))
    return idx, w


def eam_update(eam: torch.Tensor, layer: int, idx: torch.Tensor, stream=None) -> None:
    """eam [B][L][E] int32 (device), updated in place with the picks idx [B][k]."""
    _dev(eam, torch.int32)
    _dev(idx, torch.int32)
    if eam.dim() == 2:
        eam = eam.unsqueeze(0)
    B, L, E = eam.shape
    assert idx.shape[0] == B
    _check(lib().eam_update(_p(eam), B, L, E, layer, _p(idx), idx.shape[1], _stream(stream)))


def eamc_match(eamc: Eamc, eam: torch.Tensor, layer_hi: int | None = None, want_sims: bool = False, stream=None):
    """eam [B][L][E] int32 (device) -> (best [B] int32, best_sim [B] fp32, sims [B][N] fp32 or None)."""
    _dev(eam, torch.int32)
    if eam.dim() == 2:
        eam = eam.unsqueeze(0)
    B = eam.shape[0]
    assert tuple(eam.shape[1:]) == (eamc.desc.L, eamc.desc.E)
    best = _new(B, torch.int32, eam.device, stream)
    sim = _new(B, torch.float32, eam.device, stream)
    sims = _new((B, eamc.size), torch.float32, eam.device, stream) if want_sims else None
    lh = eamc.desc.L - 1 if layer_hi is None else layer_hi
    _check(lib().eamc_match(eamc.h, _p(eam), B, lh, _p(best), _p(sim), _p(sims), _stream(stream)))
    return best, sim, sims


def eamc_match_topm(eamc: Eamc, eam: torch.Tensor, m: int, layer_hi: int | None = None, want_sims: bool = False,
                    stream=None):
    """eam [L][E] int32 (device) -> (top [m] int32, top_sim [m] fp32, sims [N] fp32 or None): the m most
    similar traces, most similar first; entries beyond the stored traces are -1."""
    _dev(eam, torch.int32)
    assert tuple(eam.shape) == (eamc.desc.L, eamc.desc.E)
    n = max(int(m), 1)
    top = _new(n, torch.int32, eam.device, stream)
    sim = _new(n, torch.float32, eam.device, stream)
    sims = _new(eamc.size, torch.float32, eam.device, stream) if want_sims else None
    lh = eamc.desc.L - 1 if layer_hi is None else layer_hi
    _check(lib().eamc_match_topm(eamc.h, _p(eam), lh, int(m), _p(top), _p(sim), _p(sims), _stream(stream)))
    return top, sim, sims


def expert_priority(eamc: Eamc, best: torch.Tensor, cur_layer: int, slot_of, eps: float,
                    cur_idx: torch.Tensor | None = None, stream=None):
    """-> (P [L][E] fp32, V [L][E] fp32, pf_order, n_pf, ev_order, n_ev), all device tensors.
    slot_of: device int32 tensor [L*E] or a raw device address (Cache.slot_table())."""
    _dev(best, torch.int32)
    L, E = eamc.desc.L, eamc.desc.E
    dev = best.device
    P = _new((L, E), torch.float32, dev, stream)
    V = _new((L, E), torch.float32, dev, stream)
    pf = _new(L * E, torch.int32, dev, stream)
    ev = _new(L * E, torch.int32, dev, stream)
    n_pf = _new(1, torch.int32, dev, stream)  # (the kernel writes both counts: no launches to clear them)
    n_ev = _new(1, torch.int32, dev, stream)
    k = 0
    if cur_idx is not None:
        _dev(cur_idx, torch.int32)
        k = cur_idx.numel()
    _check(lib().expert_priority(eamc.h, _p(best), best.shape[0], cur_layer, _p(slot_of), C.c_float(eps),
                                 _p(cur_idx), k, _p(P), _p(V), _p(pf), _p(n_pf), _p(ev), _p(n_ev), _stream(stream)))
    return P, V, pf, n_pf, ev, n_ev


def expert_ffn_gemv(cache: Cache, slot_ids: torch.Tensor, gate_w: torch.Tensor, x: torch.Tensor, stream=None,
                    out: torch.Tensor | None = None) -> torch.Tensor:
    """x [H] in the weight dtype (device) -> y [H] fp32 over the given slots."""
    _dev(slot_ids, torch.int32)
    _dev(gate_w, torch.float32)
    assert x.is_cuda and x.is_contiguous() and x.numel() == cache.desc.H
    y = out if out is not None else _new(cache.desc.H, torch.float32, x.device, stream)
    _check(lib().expert_ffn_gemv(cache.h, _p(slot_ids), _p(gate_w), slot_ids.numel(), _p(x), _p(y), _stream(stream)))
    return y


def expert_ffn_gemv_static(cache: Cache, slot_ids: torch.Tensor, gate_w: torch.Tensor, x: torch.Tensor, out: torch.Tensor,
                           stream=None) -> torch.Tensor:
    """expert_ffn_gemv with its scratch in the library's static device array: allocates nothing,
    so the output tensor is the caller's."""
    _dev(slot_ids, torch.int32)
    _dev(gate_w, torch.float32)
    _dev(out, torch.float32)
    assert x.is_cuda and x.is_contiguous() and x.numel() == cache.desc.H and out.numel() == cache.desc.H
    _check(lib().expert_ffn_gemv_static(cache.h, _p(slot_ids), _p(gate_w), slot_ids.numel(), _p(x), _p(out),
                                        _stream(stream)))
    return out


def expert_ffn_grouped(cache: Cache, layer: int, idx: torch.Tensor, w: torch.Tensor, x: torch.Tensor,
                       stream=None) -> torch.Tensor:
    """Decode batch: idx [B][k] int32, w [B][k] fp32, x [B][H] weight dtype (device) -> y [B][H] fp32."""
    _dev(idx, torch.int32)
    _dev(w, torch.float32)
    B = idx.shape[0]
    assert x.is_cuda and x.is_contiguous() and x.numel() == B * cache.desc.H
    y = _new((B, cache.desc.H), torch.float32, x.device, stream)
    _check(lib().expert_ffn_grouped(cache.h, layer, _p(idx), _p(w), B, _p(x), _p(y), _stream(stream)))
    return y


def moe_decode_layer(cache: Cache, eamc: Eamc, eam: torch.Tensor, layer: int, router_w: torch.Tensor,
                     router_bias: torch.Tensor | None, x: torch.Tensor, y: torch.Tensor, sync: bool = True,
                     stream=None):
    """One fused layer step. sync=True returns (topk_idx [k] np.int32, best, n_miss); else None."""
    _dev(eam, torch.int32)
    assert router_w.is_cuda and x.is_cuda and y.is_cuda and y.dtype == torch.float32
    if not sync:
        _check(lib().moe_decode_layer(cache.h, eamc.h, _p(eam), layer, _p(router_w), _p(router_bias), _p(x), _p(y),
                                      None, None, None, _stream(stream)))
        return None
    idx = np.empty(cache.desc.k, dtype=np.int32)
    best, n_miss = C.c_int32(0), C.c_int32(0)
    _check(lib().moe_decode_layer(cache.h, eamc.h, _p(eam), layer, _p(router_w), _p(router_bias), _p(x), _p(y),
                                  _p(idx), C.byref(best), C.byref(n_miss), _stream(stream)))
    return idx, best.value, n_miss.value


# -------------------------------------------------------------------- KV cache and attention
class KvDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "k_dim", "v_dim", "page_size", "dtype",
                                         "max_batch", "max_pages", "max_sel")]


class _KvPages(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("n_pages", C.c_int32), ("d_k_scale", C.c_void_p), ("d_v_scale", C.c_void_p),
                ("d_k_min", C.c_void_p), ("d_k_max", C.c_void_p)]


class Kv:
    """Owner of a moei_kv handle: shapes, scratch and error flags of a paged KV cache (the pages are the caller's).

    max_sel, the largest n_sel of kv_attend_blocks (None: 256 or max_pages), costs scratch: 12 bytes for each of max_pages pages of each
    key/value head of each of max_batch sequences, 25 MB for the defaults and eight heads.  0 where pages are never selected: none.
    shared: there is scratch for kv_attend_shared; max_weight_tokens, tokens (sequences times the table's) of a kv_attend_weights call, costs 4 bytes for each
    query head of each of them.  set_shared and set_weights change these later: graphs that hold such calls are replayed no more, unless nothing changes."""

    DTYPES = {"fp32": WDTYPE_FP32, "bf16": WDTYPE_BF16, "fp8": KVDTYPE_FP8}
    _PAGE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}

    def __init__(self, n_q_heads: int, n_kv_heads: int, k_dim: int, v_dim: int, page_size: int, dtype: str = "bf16",
                 max_batch: int = 64, max_pages: int = 4096, max_sel: int | None = None, shared: bool = False, max_weight_tokens: int = 0):
        max_sel = min(256, max_pages) if max_sel is None else max_sel
        self.desc = KvDesc(n_q_heads, n_kv_heads, k_dim, v_dim, page_size, self.DTYPES[dtype], max_batch, max_pages, max_sel)
        self.max_batch, self.max_pages = max_batch, max_pages
        self.h = C.c_void_p(0)
        _check(lib().moei_kv_create(C.byref(self.desc), C.byref(self.h)))
        self.index = torch.cuda.current_device()
        self.device = torch.device("cuda", self.index)
        self.page_dtype = self._PAGE[dtype]
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16  # of queries, new keys and values, outputs, summaries
        self.k_page = (n_kv_heads, page_size, k_dim)
        self.v_page = (n_kv_heads, page_size, v_dim)
        self.heads, self.k_heads, self.v_heads = (n_q_heads, k_dim), (n_kv_heads, k_dim), (n_kv_heads, v_dim)
        self.out_heads = (n_q_heads, v_dim)
        self.layout = (self.k_page, self.v_page, self.page_dtype, self.index)
        self.max_weight_tokens = 0
        if shared:
            self.set_shared(True)
        if max_weight_tokens:
            self.set_weights(max_weight_tokens)

    def set_shared(self, on: bool) -> None:
        _check(lib().moei_kv_set_shared(self.h, on))

    def set_weights(self, max_tokens: int) -> None:
        _check(lib().moei_kv_set_weights(self.h, max_tokens))
        self.max_weight_tokens = max_tokens

    def error_flags(self, stream=None) -> int:
        f = C.c_int32(0)
        _check(lib().moei_kv_error_flags(self.h, C.byref(f), _stream(stream)))
        return f.value

    def close(self) -> None:
        if self.h:
            lib().moei_kv_destroy(self.h)
            self.h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _pages(kv: Kv, t: torch.Tensor, shape: tuple) -> int:
    """Checks a pool of pages (each page dense) and returns the elements between pages."""
    assert t.device == kv.device and t.dtype == kv.page_dtype and tuple(t.shape[1:]) == shape, (t.device, t.dtype, t.shape, shape)
    assert t[:1].is_contiguous() and (t.shape[0] <= 1 or t.stride(0) > 0), "a page must be dense, and pages lie apart"
    return t.stride(0) if t.shape[0] > 1 else 0


class KvPages:
    """One layer's pages: k [n_pages][Hkv][page][k_dim], v likewise with v_dim (pages may lie apart: any stride between them);
    8-bit pages with k_scale, v_scale [Hkv] fp32; k_min, k_max [n_pages][Hkv][k_dim] for kv_attend_blocks."""

    def __init__(self, kv: Kv, k: torch.Tensor, v: torch.Tensor, k_min: torch.Tensor | None = None, k_max: torch.Tensor | None = None,
                 k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None):
        ks, vs = _pages(kv, k, kv.k_page), _pages(kv, v, kv.v_page)
        n = k.shape[0]
        assert v.shape[0] == n
        for t in (k_scale, v_scale):
            assert t is None or (t.numel() == kv.k_page[0] and t.device == kv.device and _dev(t, torch.float32) is t)
        for t in (k_min, k_max):
            assert t is None or (tuple(t.shape) == (n, kv.k_page[0], kv.k_page[2]) and t.device == kv.device and _dev(t, kv.dtype) is t)
        self.layout = kv.layout
        self._keep = (k, v, k_min, k_max, k_scale, v_scale)
        ptr = [None if t is None else t.data_ptr() for t in self._keep]
        self.c = _KvPages(ptr[0], ptr[1], ks, vs, n, ptr[4], ptr[5], ptr[2], ptr[3])
        self.ref = C.addressof(self.c)


def _kv_stream(kv: Kv, stream) -> int:
    """The raw stream of a call: the device's current one by its number alone (a Stream object costs 3 us)."""
    return torch._C._cuda_getCurrentRawStream(kv.index) if stream is None else _stream(stream).value


def _rows(kv: Kv, t: torch.Tensor, n: int, heads: tuple) -> int:
    """Checks n tokens' heads - a contiguous tensor of as many elements, or [n][heads][width] with dense tokens - and returns the
    elements between tokens (0: dense)."""
    assert t.dtype is kv.dtype and t.get_device() == kv.index, (t.device, t.dtype)
    if t.is_contiguous() and t.numel() == n * heads[0] * heads[1]:
        return 0
    s = t.stride()
    assert t.shape == (n, *heads) and (s[2] == 1 or heads[1] == 1) and (s[1] == heads[1] or heads[0] == 1), (t.shape, s, (n, *heads))
    assert n <= 1 or s[0] > 0, "an expanded tensor: the tokens must lie apart"  # (a stride of 0 would be taken for dense)
    return s[0] if n > 1 else 0


def _ints(kv: Kv, t: torch.Tensor) -> int:
    assert t.dtype is torch.int32 and t.get_device() == kv.index and t.is_contiguous(), (t.device, t.dtype)
    return t.data_ptr()


def _given(kv: Kv, t: torch.Tensor, n: int, heads: tuple, dtype=None) -> int:
    """Checks a caller's output [n][heads][width] and returns its address."""
    assert t.dtype is (dtype or kv.dtype) and t.get_device() == kv.index and t.is_contiguous() and t.numel() == n * heads[0] * heads[1], (t.device, t.dtype, t.shape)
    return t.data_ptr()


def kv_append(kv: Kv, pages: KvPages, table: torch.Tensor, pos: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
              inv_freq: torch.Tensor | None, seq: torch.Tensor | None = None, interleaved: bool = False,
              q_out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """q [T][Hq][k_dim], k [T][Hkv][k_dim], v [T][Hkv][v_dim] of the tokens at pos [T] of sequences seq [T] (None: token t is of
    sequence t) -> rotated queries; keys and values go into the pages that table [B][width] names.  inv_freq [rot_dim / 2] fp32."""
    assert pages.layout == kv.layout, (pages.layout, kv.layout)
    T = pos.numel()
    B, width = table.shape
    if q_out is None:
        q_out = _new((T, *kv.heads), kv.dtype, kv.device, stream)
    assert inv_freq is None or (inv_freq.dtype is torch.float32 and inv_freq.get_device() == kv.index and inv_freq.is_contiguous()), (inv_freq.device, inv_freq.dtype)
    assert seq is None or seq.numel() == T
    _check(lib().kv_append(kv.h, pages.ref, _ints(kv, table), width, B, None if seq is None else _ints(kv, seq), _ints(kv, pos), T,
                           q.data_ptr(), _rows(kv, q, T, kv.heads), k.data_ptr(), _rows(kv, k, T, kv.k_heads),
                           v.data_ptr(), _rows(kv, v, T, kv.v_heads),
                           None if inv_freq is None else inv_freq.data_ptr(), 0 if inv_freq is None else 2 * inv_freq.numel(),
                           interleaved, _given(kv, q_out, T, kv.heads), _kv_stream(kv, stream)))
    return q_out


def kv_append_norm(kv: Kv, pages: KvPages, table: torch.Tensor, pos: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                   q_weight: torch.Tensor, k_weight: torch.Tensor, inv_freq: torch.Tensor | None, eps: float = 1e-6,
                   seq: torch.Tensor | None = None, turn: torch.Tensor | None = None, interleaved: bool = False,
                   q_out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """kv_append of queries and keys that are normed for each head before the rotation, with fp32 weights [k_dim], or [Hq][k_dim] and
    [Hkv][k_dim].  turn [T]: positions to rotate by, where they are not the tokens' places pos [T]."""
    assert pages.layout == kv.layout, (pages.layout, kv.layout)
    T = pos.numel()
    B, width = table.shape
    if q_out is None:
        q_out = _new((T, *kv.heads), kv.dtype, kv.device, stream)
    assert inv_freq is None or (inv_freq.dtype is torch.float32 and inv_freq.get_device() == kv.index and inv_freq.is_contiguous()), (inv_freq.device, inv_freq.dtype)
    assert (seq is None or seq.numel() == T) and (turn is None or turn.numel() == T)
    each = q_weight.dim() == 2
    assert q_weight.shape == (kv.heads if each else kv.heads[1:]) and k_weight.shape == (kv.k_heads if each else kv.heads[1:]), (q_weight.shape, k_weight.shape)
    for w in (q_weight, k_weight):
        assert w.dtype is torch.float32 and w.get_device() == kv.index and w.is_contiguous(), (w.device, w.dtype)
    _check(lib().kv_append_norm(kv.h, pages.ref, _ints(kv, table), width, B, None if seq is None else _ints(kv, seq), _ints(kv, pos),
                                None if turn is None else _ints(kv, turn), T,
                                q.data_ptr(), _rows(kv, q, T, kv.heads), k.data_ptr(), _rows(kv, k, T, kv.k_heads),
                                v.data_ptr(), _rows(kv, v, T, kv.v_heads), q_weight.data_ptr(), k_weight.data_ptr(), each, eps,
                                None if inv_freq is None else inv_freq.data_ptr(), 0 if inv_freq is None else 2 * inv_freq.numel(),
                                interleaved, _given(kv, q_out, T, kv.heads), _kv_stream(kv, stream)))
    return q_out


def _attend_args(kv: Kv, pages: KvPages, table, lens, q, out, want_lse, lse):
    """Checks what kv_attend and kv_attend_blocks have in common, once: their library call takes as long as these lines."""
    assert pages.layout == kv.layout, (pages.layout, kv.layout)
    B, width = table.shape
    at, i32 = kv.index, torch.int32
    assert table.dtype is i32 and lens.dtype is i32 and table.get_device() == at and lens.get_device() == at, (table.device, table.dtype, lens.device, lens.dtype)
    assert table.is_contiguous() and lens.is_contiguous() and lens.numel() == B, (table.shape, lens.shape)
    stride = _rows(kv, q, B, kv.heads)
    if out is None:
        if kv.out_heads != kv.heads or q.shape[1:] != kv.heads:
            out = q.new_empty((B, *kv.out_heads))
        else:
            out = torch.empty_like(q) if stride == 0 else torch.empty_like(q, memory_format=torch.contiguous_format)
        to = out.data_ptr()
    else:
        to = _given(kv, out, B, kv.out_heads)
    if lse is not None:
        lse_to = _given(kv, lse, B, (kv.heads[0], 1), torch.float32)
    else:
        lse = q.new_empty((B, kv.heads[0]), dtype=torch.float32) if want_lse else None
        lse_to = lse.data_ptr() if want_lse else None
    return B, width, table.data_ptr(), lens.data_ptr(), stride, out, to, lse, lse_to


def kv_attend(kv: Kv, pages: KvPages, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, scale: float, window: int = 0,
              out: torch.Tensor | None = None, want_lse: bool = False, stream=None, lse: torch.Tensor | None = None):
    """q [B][Hq][k_dim] (any stride between sequences) over the first lens [B] tokens of each sequence, or the last `window` of them
    -> out [B][Hq][v_dim], or (out, lse [B][Hq] fp32) with want_lse or where lse is given."""
    if stream is not None and (on := _elsewhere(stream, kv.index)) is not None:
        with torch.cuda.stream(on):
            return kv_attend(kv, pages, table, lens, q, scale, window, out, want_lse, None, lse)
    B, width, table_at, lens_at, stride, out, out_at, lse, lse_at = _attend_args(kv, pages, table, lens, q, out, want_lse, lse)
    _check(lib().kv_attend(kv.h, pages.ref, table_at, width, lens_at, B, q.data_ptr(), stride, scale, window, out_at, lse_at, _kv_stream(kv, None)))
    return out if lse is None else (out, lse)


def kv_attend_blocks(kv: Kv, pages: KvPages, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, scale: float, n_sel: int,
                     keep_first: int = 1, keep_last: int = 1, out: torch.Tensor | None = None, want_lse: bool = False,
                     want_blocks: bool = False, stream=None, lse: torch.Tensor | None = None, blocks: torch.Tensor | None = None):
    """kv_attend over at most n_sel pages a sequence and key/value head: the first keep_first, the last keep_last and those whose
    logits have the highest bounds.  Returns out, or a tuple with lse [B][Hq] and blocks [B][Hkv][n_sel] int32 as wanted or given."""
    if stream is not None and (on := _elsewhere(stream, kv.index)) is not None:
        with torch.cuda.stream(on):
            return kv_attend_blocks(kv, pages, table, lens, q, scale, n_sel, keep_first, keep_last, out, want_lse, want_blocks, None, lse, blocks)
    B, width, table_at, lens_at, stride, out, out_at, lse, lse_at = _attend_args(kv, pages, table, lens, q, out, want_lse, lse)
    if blocks is not None:
        blocks_at = _given(kv, blocks, B, (kv.k_page[0], n_sel), torch.int32)
    else:
        blocks = torch.empty((B, kv.k_page[0], max(n_sel, 0)), dtype=torch.int32, device=kv.device) if want_blocks else None
        blocks_at = blocks.data_ptr() if want_blocks else None
    _check(lib().kv_attend_blocks(kv.h, pages.ref, table_at, width, lens_at, B, q.data_ptr(), stride, scale, n_sel, keep_first, keep_last,
                                  out_at, lse_at, blocks_at, _kv_stream(kv, None)))
    got = (out,) + (() if lse is None else (lse,)) + (() if blocks is None else (blocks,))
    return got if len(got) > 1 else out


def kv_attend_shared(kv: Kv, pages: KvPages, table: torch.Tensor, lens: torch.Tensor, starts: torch.Tensor, prefix: torch.Tensor,
                     q: torch.Tensor, scale: float, out: torch.Tensor | None = None, want_lse: bool = False, stream=None,
                     lse: torch.Tensor | None = None):
    """kv_attend of a batch whose sequences starts[g] to starts[g + 1] (starts [groups + 1] int32) share their first prefix[g] tokens, which are
    read once for all of them.  The handle is made with shared=True."""
    if stream is not None and (on := _elsewhere(stream, kv.index)) is not None:
        with torch.cuda.stream(on):
            return kv_attend_shared(kv, pages, table, lens, starts, prefix, q, scale, out, want_lse, None, lse)
    B, width, table_at, lens_at, stride, out, out_at, lse, lse_at = _attend_args(kv, pages, table, lens, q, out, want_lse, lse)
    n = prefix.numel()
    assert starts.numel() == n + 1, (starts.shape, prefix.shape)
    _check(lib().kv_attend_shared(kv.h, pages.ref, table_at, width, lens_at, B, _ints(kv, starts), _ints(kv, prefix), n, q.data_ptr(), stride, scale,
                                  out_at, lse_at, _kv_stream(kv, None)))
    return out if lse is None else (out, lse)


def _weight_rows(kv: Kv, w: torch.Tensor, B: int, tokens: int) -> int:
    """Checks weights [B][Hkv][tokens or more] fp32, contiguous, and returns the elements between rows."""
    assert w.dtype is torch.float32 and w.get_device() == kv.index and w.is_contiguous() and w.dim() == 3, (w.device, w.dtype, w.shape)
    assert w.shape[:2] == (B, kv.k_page[0]) and w.shape[2] >= max(tokens, 1), (w.shape, (B, kv.k_page[0], tokens))
    return w.shape[2]


def kv_attend_weights(kv: Kv, pages: KvPages, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, scale: float, weights: torch.Tensor,
                      window: int = 0, out: torch.Tensor | None = None, want_lse: bool = False, stream=None, lse: torch.Tensor | None = None):
    """kv_attend that adds to weights [B][Hkv][tokens] fp32 what the heads of each group give to every token of the sequence (a row holds as many
    tokens as the table, or more).  The handle is made with max_weight_tokens."""
    if stream is not None and (on := _elsewhere(stream, kv.index)) is not None:
        with torch.cuda.stream(on):
            return kv_attend_weights(kv, pages, table, lens, q, scale, weights, window, out, want_lse, None, lse)
    B, width, table_at, lens_at, stride, out, out_at, lse, lse_at = _attend_args(kv, pages, table, lens, q, out, want_lse, lse)
    _check(lib().kv_attend_weights(kv.h, pages.ref, table_at, width, lens_at, B, q.data_ptr(), stride, scale, window, weights.data_ptr(),
                                   _weight_rows(kv, weights, B, width * kv.k_page[1]), out_at, lse_at, _kv_stream(kv, None)))
    return out if lse is None else (out, lse)


def kv_evict(kv: Kv, pages: KvPages, table: torch.Tensor, lens: torch.Tensor, weights: torch.Tensor, n_keep: int, to_table: torch.Tensor,
             to_weights: torch.Tensor | None = None, keep_first: int = 0, keep_last: int = 1, to_lens: torch.Tensor | None = None,
             kept: torch.Tensor | None = None, stream=None):
    """Moves n_keep tokens of each sequence and key/value head - the first, the last and those with the largest weights [B][Hkv][tokens] - to the
    pages of to_table [B][pages], and their weights to to_weights -> (to_lens [B], kept [B][Hkv][n_keep] int32, -1 behind the last)."""
    if stream is not None and (on := _elsewhere(stream, kv.index)) is not None:
        with torch.cuda.stream(on):
            return kv_evict(kv, pages, table, lens, weights, n_keep, to_table, to_weights, keep_first, keep_last, to_lens, kept, None)
    assert pages.layout == kv.layout, (pages.layout, kv.layout)
    B, width = table.shape
    assert lens.numel() == B and to_table.dim() == 2 and to_table.shape[0] == B, (lens.shape, to_table.shape)
    row, to_row = _weight_rows(kv, weights, B, width * kv.k_page[1]), 0 if to_weights is None else _weight_rows(kv, to_weights, B, n_keep)
    if to_lens is None:
        to_lens = torch.empty((B,), dtype=torch.int32, device=kv.device)
    if kept is None:
        kept = torch.empty((B, kv.k_page[0], max(n_keep, 0)), dtype=torch.int32, device=kv.device)
    _check(lib().kv_evict(kv.h, pages.ref, _ints(kv, table), width, _ints(kv, lens), B, weights.data_ptr(), row, n_keep, keep_first, keep_last,
                          _ints(kv, to_table), to_table.shape[1], _given(kv, to_lens, B, (1, 1), torch.int32),
                          None if to_weights is None else to_weights.data_ptr(), to_row, _given(kv, kept, B, (kv.k_page[0], n_keep), torch.int32),
                          _kv_stream(kv, None)))
    return to_lens, kept


# -------------------------------------------------------------------- kernel timing
def moe_prefill_layer(cache: Cache, eam: torch.Tensor, layer: int, router_w: torch.Tensor, router_bias,
                      X: torch.Tensor, Y: torch.Tensor | None = None, want_picks: bool = False, stream=None):
    """Prefill iteration of one layer: X [n][H] (bf16 bits) -> Y [n][H] fp32; eam [L][E] int32 updated in
    place.  Returns Y, or (Y, idx [n][k], w [n][k]) with want_picks."""
    _dev(eam, torch.int32)
    n, H = X.shape
    assert H == cache.desc.H and X.is_contiguous()
    if Y is None:
        Y = _new((n, H), torch.float32, X.device, stream)
    idx = _new((n, cache.desc.k), torch.int32, X.device, stream) if want_picks else None
    w = _new((n, cache.desc.k), torch.float32, X.device, stream) if want_picks else None
    _check(lib().moe_prefill_layer(cache.h, _p(eam), layer, _p(router_w), _p(router_bias), _p(X), n, _p(Y),
                                   _p(idx), _p(w), _stream(stream)))
    return (Y, idx, w) if want_picks else Y


def profile_enable(max_samples: int) -> None:
    _check(lib().moei_profile_enable(max_samples))


def profile_disable() -> None:
    _check(lib().moei_profile_disable())


def profile_samples(name: str) -> np.ndarray:
    """Durations (microseconds) of the recorded launches of one kernel, in launch order."""
    for i in range(lib().moei_profile_kernels()):
        if lib().moei_profile_kernel_name(i).decode() == name:
            n = C.c_int32(0)
            _check(lib().moei_profile_samples(i, None, 0, C.byref(n)))
            out = np.empty(max(n.value, 1), dtype=np.float32)
            _check(lib().moei_profile_samples(i, _p(out), n.value, C.byref(n)))
            return out[:n.value].astype(np.float64) * 1e3
    raise KeyError(name)


def profile_read() -> dict:
    """{kernel name: (launches recorded, total milliseconds between their event brackets)}"""
    out = {}
    for i in range(lib().moei_profile_kernels()):
        t, n = C.c_double(0), C.c_int32(0)
        _check(lib().moei_profile_read(i, C.byref(t), C.byref(n)))
        out[lib().moei_profile_kernel_name(i).decode()] = (n.value, t.value)
    return out
