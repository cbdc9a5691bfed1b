"""ctypes binding of libhg.so with the same entry-point names as include/hg.h.

Argument marshalling only: torch tensors provide device memory and the
current stream; every step of the computation runs in the library's HIP
kernels.  If libhg.so is missing this module raises on first use -- there
is no fallback implementation.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass, field
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhg.so")

HG_OK = 0
HG_ERR_ARG = -1
HG_ERR_RANGE = -2
HG_ERR_CAPACITY = -3
HG_ERR_HIP = -4
HG_ERR_UNSUPPORTED = -5
HG_KEY_OUTDEG = 0
HG_KEY_HINDEX = 1
HG_KEYDIR_OUT = 0
HG_THETA_NONE = 2**31 - 1
HG_DTYPE_F32 = 0
HG_DTYPE_BF16 = 1
HG_ACT_NONE = 0
HG_ACT_RELU = 1
HG_ACT_SILU = 2
HG_ACT_GELU = 3
HG_MAX_REL = 255
HG_MAX_NTYPE = 255
HG_MAX_PARTS = 64

EXPORTS = [
    "hg_plan_size", "hg_build_csr_workspace_size", "hg_build_csr", "hg_node_keys_workspace_size", "hg_node_keys",
    "hg_layer_saved_size", "hg_layer_fwd_workspace_size", "hg_layer_bwd_workspace_size",
    "hg_layer_fwd", "hg_layer_bwd", "hg_hgt_saved_size", "hg_hgt_fwd_workspace_size",
    "hg_hgt_bwd_workspace_size", "hg_hgt_fwd", "hg_hgt_bwd", "hg_align_workspace_size", "hg_align_loss_fwd_bwd", "hg_align_noalloc_scratch_size",
    "hg_align_loss_fwd_bwd_noalloc",
    "hg_mlp_bce_workspace_size", "hg_mlp_bce_fwd_bwd", "hg_adam_step",
    "hg_temporal_fwd", "hg_temporal_bwd_workspace_size", "hg_temporal_bwd",
    "hg_mean_agg_fwd", "hg_mean_agg_bwd", "hg_home_gather",
    "hg_linear_fwd_workspace_size", "hg_linear_bwd_workspace_size", "hg_linear_fwd", "hg_linear_bwd",
    "hg_glu_fwd_workspace_size", "hg_glu_bwd_workspace_size", "hg_glu_fwd", "hg_glu_bwd",
    "hg_rope_table", "hg_qk_norm_rope_fwd", "hg_qk_norm_rope_bwd_workspace_size", "hg_qk_norm_rope_bwd",
    "hg_linattn_fwd_workspace_size", "hg_linattn_bwd_workspace_size", "hg_linattn_fwd", "hg_linattn_bwd",
    "hg_linattn_step",
    "hg_recur_fwd_workspace_size", "hg_recur_bwd_workspace_size", "hg_recur_fwd", "hg_recur_bwd", "hg_recur_step",
    "hg_group_norm_fwd_workspace_size", "hg_group_norm_bwd_workspace_size", "hg_group_norm_fwd", "hg_group_norm_bwd",
    "hg_muon_workspace_size", "hg_muon_step",
    "hg_status_string", "hg_last_error_detail", "hg_timing_enable", "hg_timing_collect",
]


class HgError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: {status_string(status)} ({detail})")
        self.status = status


class GraphDesc(C.Structure):
    _fields_ = [("n_nodes", C.c_int64), ("n_edges", C.c_int64), ("n_rel", C.c_int32),
                ("n_ntype", C.c_int32), ("src", C.c_void_p), ("dst", C.c_void_p),
                ("rel", C.c_void_p), ("ntype", C.c_void_p), ("part", C.c_void_p),
                ("k", C.c_int32), ("edge_w", C.c_void_p), ("edge_ts", C.c_void_p), ("t_cut", C.c_int32),
                ("reserved", C.c_int32)]


class OverlapDesc(C.Structure):
    _fields_ = [("budget_M", C.c_int64), ("key", C.c_int32), ("key_dir", C.c_int32),
                ("theta", C.c_int32), ("reserved", C.c_int32), ("seed", C.c_uint64), ("node_key", C.c_void_p)]


class SubgraphStruct(C.Structure):
    _fields_ = [("local2global", C.c_void_p), ("global2local", C.c_void_p),
                ("type_off", C.c_void_p), ("overlap", C.c_void_p), ("overlap_home", C.c_void_p),
                ("overlap_rel", C.c_void_p), ("csr_ptr", C.c_void_p), ("csr_col", C.c_void_p),
                ("csr_eid", C.c_void_p), ("csc_ptr", C.c_void_p), ("csc_row", C.c_void_p),
                ("csc_scale", C.c_void_p), ("csr_w", C.c_void_p), ("plan", C.c_void_p),
                ("plan_bytes", C.c_size_t),
                ("n_nodes", C.c_int64), ("n_edges", C.c_int64), ("n_sub", C.c_int64),
                ("e_sub", C.c_int64), ("m_sel", C.c_int64), ("n_rel", C.c_int32),
                ("n_ntype", C.c_int32), ("type_off_host", C.c_int64 * (HG_MAX_NTYPE + 1)),
                ("n_active", C.c_int64 * HG_MAX_REL), ("plan_items", C.c_int64),
                ("plan_heavy", C.c_int64), ("plan_partials", C.c_int64),
                ("plan_fwd_heavy", C.c_int64), ("plan_fwd_parts", C.c_int64), ("plan_slot_rows", C.c_int64),
                ("weighted", C.c_int64)]


class LayerDesc(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("dtype", C.c_int32),
                ("relu", C.c_int32), ("residual", C.c_int32)]


HGT_PARAMS = ("W_K", "b_K", "W_Q", "b_Q", "W_V", "b_V", "W_att", "W_msg", "mu", "W_agg", "b_agg")


class HgtDesc(C.Structure):
    _fields_ = [("d", C.c_int32), ("heads", C.c_int32), ("dtype", C.c_int32), ("relu", C.c_int32),
                ("residual", C.c_int32), ("lean", C.c_int32)]


class HgtWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in HGT_PARAMS]


TEMPORAL_PARAMS = ("Q", "r", "Wi", "bi", "Wh", "bh")


class TemporalWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in TEMPORAL_PARAMS]


class LinearDesc(C.Structure):
    _fields_ = [("n", C.c_int64), ("d_in", C.c_int32), ("d_out", C.c_int32), ("dtype", C.c_int32),
                ("act", C.c_int32), ("ld_x", C.c_int64), ("ld_y", C.c_int64), ("ld_r", C.c_int64)]


class GluDesc(C.Structure):
    _fields_ = [("n", C.c_int64), ("d", C.c_int32), ("f", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32),
                ("ld_x", C.c_int64), ("ld_h", C.c_int64), ("ld_dx", C.c_int64)]


class Heads(C.Structure):
    _fields_ = [("p", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class RopeDesc(C.Structure):
    _fields_ = [("n", C.c_int64), ("n_pos", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("d", C.c_int32), ("rot", C.c_int32), ("interleaved", C.c_int32), ("dtype", C.c_int32),
                ("eps", C.c_float), ("reserved", C.c_int32)]


class LinattnDesc(C.Structure):
    _fields_ = [("t", C.c_int64), ("batch", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("d", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


class RecurDesc(C.Structure):
    _fields_ = [("t", C.c_int64), ("batch", C.c_int32), ("width", C.c_int32), ("dtype", C.c_int32),
                ("rate", C.c_float)]


class GroupNormDesc(C.Structure):
    _fields_ = [("t", C.c_int64), ("batch", C.c_int32), ("width", C.c_int32), ("groups", C.c_int32),
                ("dtype", C.c_int32), ("act", C.c_int32), ("eps", C.c_float)]


class MuonDesc(C.Structure):
    _fields_ = [("count", C.c_int32), ("rows", C.c_int32), ("cols", C.c_int32), ("dtype", C.c_int32),
                ("steps", C.c_int32), ("nesterov", C.c_int32), ("lr", C.c_float), ("mu", C.c_float),
                ("weight_decay", C.c_float), ("scale", C.c_float), ("eps", C.c_float), ("reserved", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """Load libhg.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run __graft_entry__.build() "
                          "(python -m paper_2608_02168_amd.build)")
    L = C.CDLL(LIB_PATH)
    vp, sz, i64, i32, f32 = C.c_void_p, C.c_size_t, C.c_int64, C.c_int32, C.c_float
    sig = {
        "hg_plan_size": (sz, [i64, i64, i32]),
        "hg_node_keys_workspace_size": (sz, [vp, i32]),
        "hg_node_keys": (C.c_int, [vp, i32, vp, vp, sz, vp]),
        "hg_build_csr_workspace_size": (sz, [vp, vp]),
        "hg_build_csr": (C.c_int, [vp, vp, vp, vp, sz, vp]),
        "hg_layer_saved_size": (sz, [vp, vp]),
        "hg_layer_fwd_workspace_size": (sz, [vp, vp]),
        "hg_layer_bwd_workspace_size": (sz, [vp, vp]),
        "hg_layer_fwd": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "hg_layer_bwd": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]),
        "hg_hgt_saved_size": (sz, [vp, vp]),
        "hg_hgt_fwd_workspace_size": (sz, [vp, vp]),
        "hg_hgt_bwd_workspace_size": (sz, [vp, vp]),
        "hg_hgt_fwd": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "hg_hgt_bwd": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]),
        "hg_align_workspace_size": (sz, [i64, i32]),
        "hg_align_loss_fwd_bwd": (C.c_int, [i64, i32, i32, i64, vp, vp, vp, vp, f32, f32, f32,
                                            i32, vp, vp, vp, vp, vp, sz, vp]),
        "hg_align_noalloc_scratch_size": (sz, []),
        "hg_align_loss_fwd_bwd_noalloc": (C.c_int, [i64, i32, i32, i64, vp, vp, vp, vp, f32, f32, f32,
                                                    i32, vp, vp, vp, vp, vp]),
        "hg_mlp_bce_workspace_size": (sz, [i64, i32, i32]),
        "hg_mlp_bce_fwd_bwd": (C.c_int, [i64, i32, i32] + [vp] * 7 + [i64] + [vp] * 8 + [sz, vp]),
        "hg_adam_step": (C.c_int, [i64, vp, vp, vp, vp, i64, f32, f32, f32, f32, f32, vp]),
        "hg_temporal_fwd": (C.c_int, [i64, i32, i32, i32, vp, vp, vp, vp, vp]),
        "hg_temporal_bwd_workspace_size": (sz, [i64, i32, i32]),
        "hg_temporal_bwd": (C.c_int, [i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]),
        "hg_mean_agg_fwd": (C.c_int, [i64, i32, i32, i32, vp, vp, vp, vp, vp]),
        "hg_mean_agg_bwd": (C.c_int, [i64, i32, i32, vp, vp, vp, vp, i32, vp]),
        "hg_home_gather": (C.c_int, [i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]),
        "hg_linear_fwd_workspace_size": (sz, [vp]),
        "hg_linear_bwd_workspace_size": (sz, [vp]),
        "hg_linear_fwd": (C.c_int, [vp] * 7 + [sz, vp]),
        "hg_linear_bwd": (C.c_int, [vp] * 8 + [i32, vp, sz, vp]),
        "hg_glu_fwd_workspace_size": (sz, [vp]),
        "hg_glu_bwd_workspace_size": (sz, [vp]),
        "hg_glu_fwd": (C.c_int, [vp] * 6 + [sz, vp]),
        "hg_glu_bwd": (C.c_int, [vp] * 8 + [i32, vp, sz, vp]),
        "hg_rope_table": (C.c_int, [i64, i32, C.c_double, C.c_double, vp, vp]),
        "hg_qk_norm_rope_fwd": (C.c_int, [vp] * 10),
        "hg_qk_norm_rope_bwd_workspace_size": (sz, [vp]),
        "hg_qk_norm_rope_bwd": (C.c_int, [vp] * 13 + [i32, vp, sz, vp]),
        "hg_linattn_fwd_workspace_size": (sz, [vp]),
        "hg_linattn_bwd_workspace_size": (sz, [vp]),
        "hg_linattn_fwd": (C.c_int, [vp] * 10 + [sz, vp]),
        "hg_linattn_bwd": (C.c_int, [vp] * 14 + [sz, vp]),
        "hg_linattn_step": (C.c_int, [vp] * 7 + [i64, vp, vp]),
        "hg_recur_fwd_workspace_size": (sz, [vp]),
        "hg_recur_bwd_workspace_size": (sz, [vp]),
        "hg_recur_fwd": (C.c_int, [vp] * 10 + [sz, vp]),
        "hg_recur_bwd": (C.c_int, [vp] * 15 + [i32, vp, sz, vp]),
        "hg_recur_step": (C.c_int, [vp] * 7 + [i64, vp, vp]),
        "hg_group_norm_fwd_workspace_size": (sz, [vp]),
        "hg_group_norm_bwd_workspace_size": (sz, [vp]),
        "hg_group_norm_fwd": (C.c_int, [vp] * 8 + [sz, vp]),
        "hg_group_norm_bwd": (C.c_int, [vp] * 10 + [i32, vp, sz, vp]),
        "hg_muon_workspace_size": (sz, [vp]),
        "hg_muon_step": (C.c_int, [vp] * 5 + [sz, vp]),
        "hg_status_string": (C.c_char_p, [C.c_int]),
        "hg_last_error_detail": (C.c_char_p, []),
        "hg_timing_enable": (C.c_int, [C.c_int]),
        "hg_timing_collect": (C.c_int, [vp, vp, vp, C.c_int]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().hg_status_string(status).decode()


def last_error_detail() -> str:
    return lib().hg_last_error_detail().decode()


def _check(status: int, where: str):
    if status != HG_OK:
        raise HgError(status, where, last_error_detail())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(1, int(nbytes)), dtype=torch.uint8, device=device)


@dataclass
class Subgraph:
    """Device arrays of hg_subgraph plus the host counts the build returned."""
    c: SubgraphStruct
    device: torch.device
    arrays: dict = field(default_factory=dict)

    @property
    def n_sub(self) -> int:
        return int(self.c.n_sub)

    @property
    def e_sub(self) -> int:
        return int(self.c.e_sub)

    @property
    def m_sel(self) -> int:
        return int(self.c.m_sel)

    @property
    def n_rel(self) -> int:
        return int(self.c.n_rel)

    @property
    def n_ntype(self) -> int:
        return int(self.c.n_ntype)

    def view(self, name: str) -> torch.Tensor:
        """The valid prefix of one output array."""
        n_ptr = self.n_sub * self.n_rel + 1
        length = {"local2global": self.n_sub, "global2local": int(self.c.n_nodes),
                  "type_off": self.n_ntype + 1, "overlap": self.m_sel,
                  "overlap_home": self.m_sel, "overlap_rel": self.m_sel, "csr_ptr": n_ptr,
                  "csc_ptr": n_ptr, "csr_col": self.e_sub, "csr_eid": self.e_sub,
                  "csc_row": self.e_sub, "csc_scale": self.e_sub, "csr_w": self.e_sub}[name]
        return self.arrays[name][:length]

    def n_active(self):
        return [int(self.c.n_active[r]) for r in range(self.n_rel)]

    def type_off_host(self):
        return [int(self.c.type_off_host[t]) for t in range(self.n_ntype + 1)]


def hg_plan_size(n_nodes: int, n_edges: int, n_rel: int) -> int:
    return int(lib().hg_plan_size(n_nodes, n_edges, n_rel))


def hg_build_csr(src, dst, rel, ntype, part, k: int, n_rel: int, n_ntype: int, budget_M: int,
                 key: int = HG_KEY_OUTDEG, theta: int = HG_THETA_NONE, seed: int = 0,
                 want_eid: bool = True, stream=None, ws: Optional[torch.Tensor] = None,
                 out: Optional[Subgraph] = None, edge_ts=None, t_cut: int = 0, node_key=None,
                 edge_w=None) -> Subgraph:
    """Overlapping-subgraph construction; inputs are device tensors
    (src/dst/part int32, rel/ntype uint8, edge_ts int32 or None, edge_w
    float32 or None).  Synchronous.  ``out`` reuses the arrays of an earlier
    build of the same input sizes.  With edge_ts, the snapshot that keeps the
    induced edges with edge_ts <= t_cut.  node_key: the graph's keys from
    hg_node_keys (same key kind), or None to compute them inside the build.
    edge_w: message weights of the edges (csr_w is then allocated)."""
    dev = ntype.device
    n, e = int(ntype.shape[0]), int(src.shape[0])
    g = GraphDesc(n, e, n_rel, n_ntype, _ptr(src), _ptr(dst), _ptr(rel), _ptr(ntype), _ptr(part),
                  k, _ptr(edge_w), _ptr(edge_ts), int(t_cut), 0)
    o = OverlapDesc(budget_M, key, HG_KEYDIR_OUT, theta, 0, seed, _ptr(node_key))
    L = lib()
    if out is not None:
        if ws is None:
            ws = out.arrays.get("ws")
        if ws is None:
            ws = _ws(int(L.hg_build_csr_workspace_size(C.byref(g), C.byref(o))), dev)
        _check(L.hg_build_csr(C.byref(g), C.byref(o), C.byref(out.c), _ptr(ws), ws.numel(),
                              _stream(stream)), "hg_build_csr")
        return out
    i32 = dict(dtype=torch.int32, device=dev)
    m_cap = max(1, min(budget_M, n))
    nq = n * n_rel + 1
    arrays = {
        "local2global": torch.empty(n, **i32), "global2local": torch.empty(n, **i32),
        "type_off": torch.empty(n_ntype + 1, **i32), "overlap": torch.empty(m_cap, **i32),
        "overlap_home": torch.empty(m_cap, **i32),
        "overlap_rel": torch.empty(m_cap, dtype=torch.uint8, device=dev),
        "csr_ptr": torch.empty(nq, **i32), "csr_col": torch.empty(max(1, e), **i32),
        "csr_eid": torch.empty(max(1, e), **i32) if want_eid else None,
        "csc_ptr": torch.empty(nq, **i32), "csc_row": torch.empty(max(1, e), **i32),
        "csc_scale": torch.empty(max(1, e), dtype=torch.float32, device=dev),
        "csr_w": torch.empty(max(1, e), dtype=torch.float32, device=dev) if edge_w is not None else None,
    }
    plan_bytes = hg_plan_size(n, e, n_rel)
    arrays["plan"] = _ws(plan_bytes, dev)
    s = SubgraphStruct()
    for name in ("local2global", "global2local", "type_off", "overlap", "overlap_home",
                 "overlap_rel", "csr_ptr", "csr_col", "csr_eid", "csc_ptr", "csc_row",
                 "csc_scale", "csr_w", "plan"):
        setattr(s, name, _ptr(arrays[name]))
    s.plan_bytes = plan_bytes
    need = int(L.hg_build_csr_workspace_size(C.byref(g), C.byref(o)))
    if need == 0:
        _check(L.hg_build_csr(C.byref(g), C.byref(o), C.byref(s), None, 0, _stream(stream)),
               "hg_build_csr")
    if ws is None or ws.numel() < need:
        ws = _ws(need, dev)
    _check(L.hg_build_csr(C.byref(g), C.byref(o), C.byref(s), _ptr(ws), ws.numel(),
                          _stream(stream)), "hg_build_csr")
    arrays["ws"] = ws
    return Subgraph(s, dev, arrays)


def _layer_desc(d: int, dtype, relu: bool, residual: bool) -> LayerDesc:
    code = HG_DTYPE_BF16 if dtype == torch.bfloat16 else HG_DTYPE_F32
    return LayerDesc(d, d, code, int(relu), int(residual))


def hg_layer_saved_size(sub: Subgraph, d: int, dtype=torch.float32) -> int:
    desc = _layer_desc(d, dtype, True, True)
    return int(lib().hg_layer_saved_size(C.byref(sub.c), C.byref(desc)))


def hg_layer_fwd_workspace_size(sub: Subgraph, d: int, dtype=torch.float32) -> int:
    desc = _layer_desc(d, dtype, True, True)
    return int(lib().hg_layer_fwd_workspace_size(C.byref(sub.c), C.byref(desc)))


def hg_layer_bwd_workspace_size(sub: Subgraph, d: int, dtype=torch.float32) -> int:
    desc = _layer_desc(d, dtype, True, True)
    return int(lib().hg_layer_bwd_workspace_size(C.byref(sub.c), C.byref(desc)))


def hg_layer_fwd(sub: Subgraph, H_in, W_rel, W_self, bias=None, relu=True, residual=True,
                 H_out=None, saved=None, ws=None, stream=None):
    """Returns (H_out, saved); saved is the ReLU bitmask [n_sub, d/32] int32."""
    d = int(H_in.shape[1])
    desc = _layer_desc(d, H_in.dtype, relu, residual)
    L = lib()
    if H_out is None:
        H_out = torch.empty_like(H_in)
    if saved is None:
        saved = torch.empty((max(1, sub.n_sub), (d + 31) // 32), dtype=torch.int32, device=H_in.device)
    if ws is None:
        need = int(L.hg_layer_fwd_workspace_size(C.byref(sub.c), C.byref(desc)))
        ws = _ws(need, H_in.device)
    _check(L.hg_layer_fwd(C.byref(sub.c), C.byref(desc), _ptr(H_in), _ptr(W_rel), _ptr(W_self),
                          _ptr(bias), _ptr(H_out), _ptr(saved), _ptr(ws), ws.numel(),
                          _stream(stream)), "hg_layer_fwd")
    return H_out, saved


def hg_layer_bwd(sub: Subgraph, H_in, W_rel, W_self, saved, dH_out, relu=True, residual=True,
                 dH_in=None, dW_rel=None, dW_self=None, dbias=None, want_dbias=True, accumulate=False,
                 ws=None, stream=None):
    """Returns (dH_in, dW_rel, dW_self, dbias); with accumulate the weight
    gradients are added into the given buffers."""
    d = int(H_in.shape[1])
    desc = _layer_desc(d, H_in.dtype, relu, residual)
    L = lib()
    dev = H_in.device
    if dH_in is None:
        dH_in = torch.empty_like(H_in)
    if dW_rel is None:
        dW_rel = torch.empty_like(W_rel)
    if dW_self is None:
        dW_self = torch.empty_like(W_self)
    if dbias is None and want_dbias:
        dbias = torch.empty((W_self.shape[0], d), dtype=torch.float32, device=dev)
    if ws is None:
        need = int(L.hg_layer_bwd_workspace_size(C.byref(sub.c), C.byref(desc)))
        ws = _ws(need, dev)
    _check(L.hg_layer_bwd(C.byref(sub.c), C.byref(desc), _ptr(H_in), _ptr(W_rel), _ptr(W_self),
                          _ptr(saved), _ptr(dH_out), _ptr(dH_in), _ptr(dW_rel), _ptr(dW_self),
                          _ptr(dbias), int(bool(accumulate)), _ptr(ws), ws.numel(), _stream(stream)),
           "hg_layer_bwd")
    return dH_in, dW_rel, dW_self, dbias


def _hgt_desc(d: int, heads: int, relu: bool, residual: bool, lean: bool = False) -> HgtDesc:
    return HgtDesc(d, heads, HG_DTYPE_F32, int(relu), int(residual), int(lean))


def _hgt_struct(weights: dict) -> HgtWeights:
    """weights: name -> device float32 tensor (biases may be missing or None)."""
    return HgtWeights(*[_ptr(weights.get(n)) for n in HGT_PARAMS])


def hg_hgt_saved_size(sub: Subgraph, d: int, heads: int, lean: bool = False) -> int:
    desc = _hgt_desc(d, heads, True, True, lean)
    return int(lib().hg_hgt_saved_size(C.byref(sub.c), C.byref(desc)))


def hg_hgt_fwd_workspace_size(sub: Subgraph, d: int, heads: int, lean: bool = False) -> int:
    desc = _hgt_desc(d, heads, True, True, lean)
    return int(lib().hg_hgt_fwd_workspace_size(C.byref(sub.c), C.byref(desc)))


def hg_hgt_bwd_workspace_size(sub: Subgraph, d: int, heads: int, lean: bool = False) -> int:
    desc = _hgt_desc(d, heads, True, True, lean)
    return int(lib().hg_hgt_bwd_workspace_size(C.byref(sub.c), C.byref(desc)))


def hg_hgt_fwd(sub: Subgraph, H_in, weights: dict, heads: int, relu=True, residual=True, H_out=None,
               mask=None, saved=None, ws=None, stream=None, lean=False):
    """Attention layer forward; returns (H_out, mask, saved): mask is the ReLU
    bitmask [n_sub, d/32] int32, saved a uint8 buffer for the backward (lean:
    without the relation transforms, which the backward computes again)."""
    d = int(H_in.shape[1])
    desc = _hgt_desc(d, heads, relu, residual, lean)
    L = lib()
    if H_out is None:
        H_out = torch.empty_like(H_in)
    if mask is None:
        mask = torch.empty((max(1, sub.n_sub), d // 32), dtype=torch.int32, device=H_in.device)
    if saved is None:
        saved = _ws(int(L.hg_hgt_saved_size(C.byref(sub.c), C.byref(desc))), H_in.device)
    if ws is None:
        ws = _ws(int(L.hg_hgt_fwd_workspace_size(C.byref(sub.c), C.byref(desc))), H_in.device)
    W = _hgt_struct(weights)
    _check(L.hg_hgt_fwd(C.byref(sub.c), C.byref(desc), _ptr(H_in), C.byref(W), _ptr(H_out), _ptr(mask),
                        _ptr(saved), _ptr(ws), ws.numel(), _stream(stream)), "hg_hgt_fwd")
    return H_out, mask, saved


def hg_hgt_bwd(sub: Subgraph, H_in, weights: dict, heads: int, mask, saved, dH_out, relu=True, residual=True,
               dH_in=None, grads: Optional[dict] = None, accumulate: bool = False, ws=None, stream=None, lean=False):
    """Attention layer backward; returns (dH_in, grads) with grads a dict of
    the same names as the weights (bias gradients for the biases given),
    overwritten, or added into when accumulate.  lean as in the forward."""
    d = int(H_in.shape[1])
    desc = _hgt_desc(d, heads, relu, residual, lean)
    L = lib()
    if dH_in is None:
        dH_in = torch.empty_like(H_in)
    if grads is None:
        grads = {n: torch.empty_like(w) for n, w in weights.items() if w is not None}
    if ws is None:
        ws = _ws(int(L.hg_hgt_bwd_workspace_size(C.byref(sub.c), C.byref(desc))), H_in.device)
    G = _hgt_struct(grads)
    W = _hgt_struct(weights)
    _check(L.hg_hgt_bwd(C.byref(sub.c), C.byref(desc), _ptr(H_in), C.byref(W), _ptr(mask), _ptr(saved),
                        _ptr(dH_out), _ptr(dH_in), C.byref(G), int(accumulate), _ptr(ws), ws.numel(),
                        _stream(stream)), "hg_hgt_bwd")
    return dH_in, grads


def hg_mlp_bce_workspace_size(n_rows: int, d: int) -> int:
    return int(lib().hg_mlp_bce_workspace_size(n_rows, d, d))


def hg_mlp_bce_fwd_bwd(H, W1, b1, W2, b2, labels, dH=None, grads: Optional[dict] = None, loss=None, prob=None,
                       ws=None, stream=None, rows=None):
    """Prediction head + masked BCE: returns (loss [1], dH, grads) with grads
    {W1, b1, W2, b2}; dH is overwritten with dL_BCE/dH.  rows: int32 list
    of rows holding every labelled one (only those go through the head)."""
    n, d = int(H.shape[0]), int(H.shape[1])
    L = lib()
    if dH is None:
        dH = torch.empty_like(H)
    if grads is None:
        grads = {"W1": torch.empty_like(W1), "b1": torch.empty_like(b1), "W2": torch.empty_like(W2),
                 "b2": torch.empty_like(b2)}
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=H.device)
    if ws is None:
        ws = _ws(int(L.hg_mlp_bce_workspace_size(n, d, d)), H.device)
    n_list = 0 if rows is None else int(rows.shape[0])
    _check(L.hg_mlp_bce_fwd_bwd(n, d, d, _ptr(H), _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2), _ptr(labels), _ptr(rows),
                                n_list, _ptr(loss),
                                _ptr(prob), _ptr(dH), _ptr(grads["W1"]), _ptr(grads.get("b1")), _ptr(grads["W2"]),
                                _ptr(grads.get("b2")), _ptr(ws), ws.numel(), _stream(stream)), "hg_mlp_bce_fwd_bwd")
    return loss, dH, grads


def hg_adam_step(param, grad, m, v, step: int, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=1e-5,
                 stream=None):
    """In-place Adam update of one float32 tensor."""
    _check(lib().hg_adam_step(param.numel(), _ptr(param), _ptr(grad), _ptr(m), _ptr(v), step, lr, beta1, beta2, eps,
                              weight_decay, _stream(stream)), "hg_adam_step")


def _host_ptrs(tensors):
    """A host array of device pointers (None entries stay NULL)."""
    arr = (C.c_void_p * max(1, len(tensors)))(*[None if t is None else t.data_ptr() for t in tensors])
    return arr


def _dtype_code(t) -> int:
    return HG_DTYPE_BF16 if t.dtype == torch.bfloat16 else HG_DTYPE_F32


def hg_temporal_fwd(h, states, weights: dict, H=None, stream=None):
    """Temporal module forward: h [n, d] and the w context states (oldest
    first, each [n, d], same dtype); returns H."""
    n, d = int(h.shape[0]), int(h.shape[1])
    if H is None:
        H = torch.empty_like(h)
    ctx = _host_ptrs(states)
    W = TemporalWeights(*[_ptr(weights.get(k)) for k in TEMPORAL_PARAMS])
    _check(lib().hg_temporal_fwd(n, d, len(states), _dtype_code(h), _ptr(h), C.cast(ctx, C.c_void_p), C.byref(W),
                                 _ptr(H), _stream(stream)), "hg_temporal_fwd")
    return H


def hg_temporal_bwd_workspace_size(n: int, d: int, w: int) -> int:
    return int(lib().hg_temporal_bwd_workspace_size(n, d, w))


def hg_temporal_bwd(h, states, weights: dict, dH, dh=None, dstates=None, grads: Optional[dict] = None,
                    accumulate: bool = False, ws=None, stream=None):
    """Temporal module backward: returns (dh, grads).  dL/dc_k is ADDED into
    dstates[k] (a list of tensors or None entries; None = no state
    gradients); grads are overwritten, or added into when accumulate."""
    n, d = int(h.shape[0]), int(h.shape[1])
    w = len(states)
    L = lib()
    if dh is None:
        dh = torch.empty_like(h)
    if grads is None:
        grads = {k: torch.empty_like(v) for k, v in weights.items() if v is not None}
    if ws is None:
        ws = _ws(int(L.hg_temporal_bwd_workspace_size(n, d, w)), h.device)
    ctx = _host_ptrs(states)
    darr = None if dstates is None else _host_ptrs(dstates)  # kept alive through the call
    dctx = None if darr is None else C.cast(darr, C.c_void_p)
    W = TemporalWeights(*[_ptr(weights.get(k)) for k in TEMPORAL_PARAMS])
    G = TemporalWeights(*[_ptr(grads.get(k)) for k in TEMPORAL_PARAMS])
    _check(L.hg_temporal_bwd(n, d, w, _dtype_code(h), _ptr(h), C.cast(ctx, C.c_void_p), C.byref(W), _ptr(dH),
                             _ptr(dh), dctx, int(accumulate), C.byref(G), _ptr(ws), ws.numel(), _stream(stream)),
           "hg_temporal_bwd")
    return dh, grads


def hg_node_keys(src, dst, rel, n_nodes: int, n_rel: int, key: int = HG_KEY_OUTDEG, keys=None, ws=None,
                 stream=None):
    """Key of every node (out-degree or out-neighbour h-index), int32
    [n_nodes] on the device.  Synchronous."""
    dev = src.device
    g = GraphDesc(n_nodes, int(src.shape[0]), n_rel, 1, _ptr(src), _ptr(dst), _ptr(rel), None, None, 0, None, None,
                  0, 0)
    L = lib()
    if keys is None:
        keys = torch.empty(n_nodes, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _ws(int(L.hg_node_keys_workspace_size(C.byref(g), key)), dev)
    _check(L.hg_node_keys(C.byref(g), key, _ptr(keys), _ptr(ws), ws.numel(), _stream(stream)), "hg_node_keys")
    return keys


def hg_node_keys_workspace_size(n_nodes: int, n_edges: int, n_rel: int, key: int = HG_KEY_OUTDEG) -> int:
    g = GraphDesc(n_nodes, n_edges, n_rel, 1, None, C.c_void_p(8), C.c_void_p(8), None, None, 0, None, None, 0, 0)
    g.src = C.c_void_p(8)
    return int(lib().hg_node_keys_workspace_size(C.byref(g), key))


def hg_mean_agg_fwd(g2l: list, h_parts: list, H=None, cnt=None, stream=None):
    """MeanAgg over K subgraphs: g2l[k] (int32 [n_nodes]) and h_parts[k]
    ([n_sub_k, d]) of subgraph k; returns (H [n_nodes, d], cnt int32 [n_nodes])."""
    n, d = int(g2l[0].shape[0]), int(h_parts[0].shape[1])
    if H is None:
        H = torch.empty((n, d), dtype=h_parts[0].dtype, device=h_parts[0].device)
    if cnt is None:
        cnt = torch.empty(n, dtype=torch.int32, device=h_parts[0].device)
    ga, ha = _host_ptrs(g2l), _host_ptrs(h_parts)
    _check(lib().hg_mean_agg_fwd(n, d, _dtype_code(h_parts[0]), len(h_parts), C.cast(ga, C.c_void_p),
                                 C.cast(ha, C.c_void_p), _ptr(H), _ptr(cnt), _stream(stream)), "hg_mean_agg_fwd")
    return H, cnt


def hg_mean_agg_bwd(l2g, cnt, dH, dh_part=None, accumulate=False, stream=None):
    """dh_part[i] = dH[l2g[i]] / cnt[l2g[i]] (added into dh_part when accumulate)."""
    n_sub, d = int(l2g.shape[0]), int(dH.shape[1])
    if dh_part is None:
        dh_part = torch.empty((n_sub, d), dtype=dH.dtype, device=dH.device)
    _check(lib().hg_mean_agg_bwd(n_sub, d, _dtype_code(dH), _ptr(l2g), _ptr(cnt), _ptr(dH), _ptr(dh_part),
                                 int(bool(accumulate)), _stream(stream)), "hg_mean_agg_bwd")
    return dh_part


def hg_home_gather(overlap, l2g, home, g2l: list, h_parts: list, Y=None, stream=None):
    """Home copies of one subgraph's overlap rows: Y [m, d]."""
    m, d = int(overlap.shape[0]), int(h_parts[0].shape[1])
    if Y is None:
        Y = torch.empty((m, d), dtype=h_parts[0].dtype, device=h_parts[0].device)
    ga, ha = _host_ptrs(g2l), _host_ptrs(h_parts)
    _check(lib().hg_home_gather(m, d, _dtype_code(h_parts[0]), len(h_parts), _ptr(overlap), _ptr(l2g), _ptr(home),
                                C.cast(ga, C.c_void_p), C.cast(ha, C.c_void_p), _ptr(Y), _stream(stream)),
           "hg_home_gather")
    return Y


def hg_align_workspace_size(M: int, d: int) -> int:
    return int(lib().hg_align_workspace_size(M, d))


def hg_align_loss_fwd_bwd(H, overlap, H_ref, dH, w=None, lambda_n=2e-4, scale=0.1, eps=1e-5,
                          ddof=0, dH_ref=None, loss3=None, ws=None, stream=None, dH_base=None):
    """CCA alignment: returns loss3 (device float32 [3] = L_inv, L_dec, L);
    dH[overlap] = dH_base[overlap] + scale * dL/dX (dH_base = dH when None:
    the gradient is added into dH) and overwrites dH_ref if given."""
    M = int(overlap.shape[0])
    d = int(H.shape[1])
    L = lib()
    code = HG_DTYPE_BF16 if H.dtype == torch.bfloat16 else HG_DTYPE_F32
    if loss3 is None:
        loss3 = torch.empty(3, dtype=torch.float32, device=H.device)
    if ws is None:
        ws = _ws(int(L.hg_align_workspace_size(M, d)), H.device)
    _check(L.hg_align_loss_fwd_bwd(M, d, code, int(H.shape[0]), _ptr(H), _ptr(overlap), _ptr(H_ref),
                                   _ptr(w), lambda_n, scale, eps, ddof, _ptr(loss3), _ptr(dH), _ptr(dH_base),
                                   _ptr(dH_ref), _ptr(ws), ws.numel(), _stream(stream)),
           "hg_align_loss_fwd_bwd")
    return loss3


def hg_align_noalloc_scratch_size() -> int:
    return int(lib().hg_align_noalloc_scratch_size())


def hg_align_loss_fwd_bwd_noalloc(H, overlap, H_ref, dH, loss3, w=None, lambda_n=2e-4, scale=0.1, eps=1e-5,
                                  ddof=0, dH_ref=None, stream=None, dH_base=None):
    """hg_align_loss_fwd_bwd with the library's static scratch instead of a
    workspace: allocates nothing (loss3 is the caller's device float32 [3])."""
    code = HG_DTYPE_BF16 if H.dtype == torch.bfloat16 else HG_DTYPE_F32
    _check(lib().hg_align_loss_fwd_bwd_noalloc(int(overlap.shape[0]), int(H.shape[1]), code, int(H.shape[0]),
                                               _ptr(H), _ptr(overlap), _ptr(H_ref), _ptr(w), lambda_n, scale, eps,
                                               ddof, _ptr(loss3), _ptr(dH), _ptr(dH_base), _ptr(dH_ref),
                                               _stream(stream)),
           "hg_align_loss_fwd_bwd_noalloc")
    return loss3


# ---- sequence encoder -------------------------------------------------------
# These calls are made for single tokens too, so their marshalling is kept
# short: descriptors are packed bytes (the layouts of LinearDesc, GluDesc,
# RopeDesc, LinattnDesc, RecurDesc, GroupNormDesc, MuonDesc and Heads), devices
# are compared by index.

_pack_linear = struct.Struct("@qiiiiqqq").pack
_pack_glu = struct.Struct("@qiiiiqqq").pack
_pack_rope = struct.Struct("@qqiiiiiifi").pack
_pack_linattn = struct.Struct("@qiiiiif").pack
_pack_heads = struct.Struct("@Pqqq").pack
_pack_recur = struct.Struct("@qiiif").pack
_pack_group_norm = struct.Struct("@qiiiiif").pack
_pack_muon = struct.Struct("@iiiiiifffffi").pack
_DTYPES = {torch.float32: HG_DTYPE_F32, torch.bfloat16: HG_DTYPE_BF16}


def _float_code(where: str, t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{where}: {t.dtype} is neither float32 nor bfloat16")
    return code


def _same(where: str, t, *others):
    """Every given tensor has the first one's type and device, which is a GPU."""
    dtype, dev = t.dtype, t.get_device()
    _on_gpu(where, t)
    for o in others:
        if o is not None and (o.dtype is not dtype or o.get_device() != dev):
            raise TypeError(f"{where}: {o.dtype} on {o.device} beside {t.dtype} on {t.device}")


def _on_gpu(where: str, t):
    """The library takes device addresses only: a host address would fault in a kernel."""
    if t.get_device() < 0:
        raise TypeError(f"{where}: a tensor on {t.device}, expected one on a GPU")


def _vector(where: str, t, n: int, like, dtype=torch.float32):
    """A contiguous vector of n values on like's device, or None; its address."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or t.get_device() != like.get_device() or not t.is_contiguous():
        raise ValueError(f"{where}: expected {n} contiguous {dtype} on {like.device}, got {tuple(t.shape)} {t.dtype} on "
                         f"{t.device}")
    return t.data_ptr()


def _rows(where: str, t, n: int, width: int) -> int:
    """Checks an [n, width] matrix whose rows are contiguous; returns their distance."""
    s = t.stride()
    if t.shape != (n, width) or (s[1] != 1 and width > 1 and n > 0):
        raise ValueError(f"{where}: expected rows [{n}, {width}] with unit column stride, got {tuple(t.shape)} strides {s}")
    return s[0] if n > 1 else width


def _matrix(where: str, t, rows: int, cols: int):
    if t.shape != (rows, cols) or not t.is_contiguous():
        raise ValueError(f"{where}: expected a contiguous [{rows}, {cols}], got {tuple(t.shape)} strides {t.stride()}")


def _heads(where: str, name: str, t, shape, single=False) -> bytes:
    """hg_heads of a [tokens, heads, d] or [batch, tokens, heads, d] tensor.  The
    stride of a dimension with one entry is never walked."""
    s = t.stride()
    if t.shape != shape or (s[-1] != 1 and t.numel()):
        raise ValueError(f"{where}: expected {name} {tuple(shape)} with unit stride in a head, got {tuple(t.shape)} "
                         f"strides {s}")
    if len(s) == 3:  # tokens, or with `single` sequences of one token
        n, h, _ = shape
        st, sh = s[0] if n > 1 else 0, s[1] if h > 1 else 0
        return _pack_heads(t.data_ptr(), st, 0, sh) if single else _pack_heads(t.data_ptr(), 0, st, sh)
    b, n, h, _ = shape
    return _pack_heads(t.data_ptr(), s[0] if b > 1 else 0, s[1] if n > 1 else 0, s[2] if h > 1 else 0)


def _addr(t):
    return None if t is None else t.data_ptr()


def _workspace(where: str, ws, need: int, like):
    """(buffer kept alive by the caller, its address, its size)"""
    if ws is None:
        if not need:
            return None, None, 0
        ws = torch.empty(need, dtype=torch.uint8, device=like.device)
    elif ws.get_device() != like.get_device() or not ws.is_contiguous():
        raise ValueError(f"{where}: expected a contiguous workspace on {like.device}, got strides {ws.stride()} on {ws.device}")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def _raw_stream(like):
    """The current stream of the tensor's device.  The calls below that take a
    stream make it the current one first, so that what they allocate is that
    stream's too."""
    return torch.cuda.current_stream(like.device).cuda_stream if _current_raw is None else _current_raw(like.get_device())


_current_raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _linear_sizes(where, x, W):
    n, d = x.shape
    m = W.shape[1]
    _matrix(where, W, d, m)
    return n, d, m


def hg_linear_fwd_workspace_size(n: int, d_in: int, d_out: int, dtype=torch.float32, act: int = HG_ACT_NONE,
                                 ld_x: Optional[int] = None) -> int:
    return int(lib().hg_linear_fwd_workspace_size(_pack_linear(
        n, d_in, d_out, _DTYPES[dtype], act, d_in if ld_x is None else ld_x, d_out, d_out)))


def hg_linear_bwd_workspace_size(n: int, d_in: int, d_out: int, dtype=torch.float32, act: int = HG_ACT_NONE,
                                 ld_x: Optional[int] = None, ld_dy: Optional[int] = None) -> int:
    return int(lib().hg_linear_bwd_workspace_size(_pack_linear(
        n, d_in, d_out, _DTYPES[dtype], act, d_in if ld_x is None else ld_x, d_out if ld_dy is None else ld_dy, d_in)))


def hg_linear_fwd(x, W, bias=None, residual=None, act: int = HG_ACT_NONE, y=None, ws=None, stream=None):
    """y = act(x W + bias) + residual: x [n, d_in], W [d_in, d_out], bias
    float32 [d_out], residual and y [n, d_out] (y may be the residual); rows
    may be strided, W is contiguous."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_linear_fwd(x, W, bias, residual, act, y, ws)
    where = "hg_linear_fwd"
    L = lib()
    n, d, m = _linear_sizes(where, x, W)
    if y is None:
        y = torch.empty((n, m), dtype=x.dtype, device=x.device)
        ld_y = m
    else:
        ld_y = _rows(where, y, n, m)
    _same(where, x, W, y, residual)
    desc = _pack_linear(n, d, m, _float_code(where, x), act, _rows(where, x, n, d), ld_y,
                        m if residual is None else _rows(where, residual, n, m))
    ws, wp, wn = _workspace(where, ws, L.hg_linear_fwd_workspace_size(desc), x)
    st = L.hg_linear_fwd(desc, x.data_ptr(), W.data_ptr(), _vector(where, bias, m, x), _addr(residual), y.data_ptr(), wp,
                         wn, _raw_stream(x))
    if st:
        _check(st, where)
    return y


def hg_linear_bwd(x, W, bias, dy, act: int = HG_ACT_NONE, dx=None, dW=None, dbias=None, accumulate: bool = False,
                  want=(True, True, True), ws=None, stream=None):
    """Returns (dx, dW, dbias) of hg_linear_fwd for dy = dL/dy (the residual's
    gradient is dy itself); dbias only with a bias.  With accumulate, dW and
    dbias are added into the given buffers.  want: which of the three to
    compute where no buffer is given."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_linear_bwd(x, W, bias, dy, act, dx, dW, dbias, accumulate, want, ws)
    where = "hg_linear_bwd"
    L = lib()
    n, d, m = _linear_sizes(where, x, W)
    dx, dW, dbias = _linear_grads(where, x, W, bias, dx, dW, dbias, accumulate, want)
    _same(where, x, W, dy, dx, dW)
    desc = _pack_linear(n, d, m, _float_code(where, x), act, _rows(where, x, n, d), _rows(where, dy, n, m),
                        d if dx is None else _rows(where, dx, n, d))
    ws, wp, wn = _workspace(where, ws, L.hg_linear_bwd_workspace_size(desc), x)
    st = L.hg_linear_bwd(desc, x.data_ptr(), W.data_ptr(), _addr(bias), dy.data_ptr(), _addr(dx), _addr(dW), _addr(dbias),
                         1 if accumulate else 0, wp, wn, _raw_stream(x))
    if st:
        _check(st, where)
    return dx, dW, dbias


def _linear_grads(where, x, W, bias, dx, dW, dbias, accumulate, want):
    if accumulate and ((dW is None and want[1]) or (dbias is None and want[2] and bias is not None)):
        raise ValueError(f"{where}: accumulate needs the buffers to add into")
    if dx is None and want[0]:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if dW is None and want[1]:
        dW = torch.empty(W.shape, dtype=W.dtype, device=W.device)
    elif dW is not None:
        _matrix(where, dW, *W.shape)
    _vector(where, bias, W.shape[1], x)
    if dbias is None and want[2] and bias is not None:
        dbias = torch.empty_like(bias)
    _vector(where, dbias, W.shape[1], x)
    return dx, dW, dbias


def _glu_sizes(where, x, W):
    n, d = x.shape
    if W.dim() != 2 or W.shape[1] % 2:
        raise ValueError(f"{where}: W is [d, 2 f], got {tuple(W.shape)}")
    _matrix(where, W, d, W.shape[1])
    return n, d, W.shape[1] // 2


def hg_glu_fwd_workspace_size(n: int, d: int, f: int, dtype=torch.float32, ld_x: Optional[int] = None) -> int:
    return int(lib().hg_glu_fwd_workspace_size(_pack_glu(n, d, f, _DTYPES[dtype], HG_ACT_SILU,
                                                         d if ld_x is None else ld_x, f, d)))


def hg_glu_bwd_workspace_size(n: int, d: int, f: int, dtype=torch.float32, ld_x: Optional[int] = None) -> int:
    return int(lib().hg_glu_bwd_workspace_size(_pack_glu(n, d, f, _DTYPES[dtype], HG_ACT_SILU,
                                                         d if ld_x is None else ld_x, f, d)))


def hg_glu_fwd(x, W, bias=None, act: int = HG_ACT_SILU, h=None, ws=None, stream=None):
    """h = act(a) * u with [a u] = x W + bias: x [n, d], W [d, 2 f] (the gate's
    columns first), bias float32 [2 f], h [n, f]."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_glu_fwd(x, W, bias, act, h, ws)
    where = "hg_glu_fwd"
    L = lib()
    n, d, f = _glu_sizes(where, x, W)
    if h is None:
        h = torch.empty((n, f), dtype=x.dtype, device=x.device)
        ld_h = f
    else:
        ld_h = _rows(where, h, n, f)
    _same(where, x, W, h)
    desc = _pack_glu(n, d, f, _float_code(where, x), act, _rows(where, x, n, d), ld_h, d)
    ws, wp, wn = _workspace(where, ws, L.hg_glu_fwd_workspace_size(desc), x)
    st = L.hg_glu_fwd(desc, x.data_ptr(), W.data_ptr(), _vector(where, bias, 2 * f, x), h.data_ptr(), wp, wn,
                      _raw_stream(x))
    if st:
        _check(st, where)
    return h


def hg_glu_bwd(x, W, bias, dh, act: int = HG_ACT_SILU, dx=None, dW=None, dbias=None, accumulate: bool = False,
               want=(True, True, True), ws=None, stream=None):
    """Returns (dx, dW, dbias) of hg_glu_fwd for dh = dL/dh, as hg_linear_bwd does."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_glu_bwd(x, W, bias, dh, act, dx, dW, dbias, accumulate, want, ws)
    where = "hg_glu_bwd"
    L = lib()
    n, d, f = _glu_sizes(where, x, W)
    dx, dW, dbias = _linear_grads(where, x, W, bias, dx, dW, dbias, accumulate, want)
    _same(where, x, W, dh, dx, dW)
    desc = _pack_glu(n, d, f, _float_code(where, x), act, _rows(where, x, n, d), _rows(where, dh, n, f),
                     d if dx is None else _rows(where, dx, n, d))
    ws, wp, wn = _workspace(where, ws, L.hg_glu_bwd_workspace_size(desc), x)
    st = L.hg_glu_bwd(desc, x.data_ptr(), W.data_ptr(), _addr(bias), dh.data_ptr(), _addr(dx), _addr(dW), _addr(dbias),
                      1 if accumulate else 0, wp, wn, _raw_stream(x))
    if st:
        _check(st, where)
    return dx, dW, dbias


def hg_rope_table(n_pos: int, rot: int, base: float = 10000.0, step: float = 1.0, table=None, device="cuda",
                  stream=None):
    """Cosines and sines [n_pos, rot] of position * step * base^(-2 p / rot)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_rope_table(n_pos, rot, base, step, table, device)
    if table is None:
        table = torch.empty((n_pos, rot), dtype=torch.float32, device=device)
    elif tuple(table.shape) != (n_pos, rot) or table.dtype != torch.float32 or not table.is_contiguous():
        raise ValueError(f"hg_rope_table: expected a contiguous float32 [{n_pos}, {rot}], got {tuple(table.shape)}")
    _on_gpu("hg_rope_table", table)
    _check(lib().hg_rope_table(n_pos, rot, base, step, table.data_ptr(), _raw_stream(table)), "hg_rope_table")
    return table


def _rope_desc(where, q, k, table, eps, interleaved):
    n, hq, d = q.shape
    hk = 0 if k is None else k.shape[1]
    if (table.dim() != 2 or table.dtype is not torch.float32 or table.get_device() != q.get_device()
            or not table.is_contiguous()):
        raise ValueError(f"{where}: expected a contiguous float32 table [positions, rot], got {tuple(table.shape)}")
    n_pos, rot = table.shape
    return _pack_rope(n, n_pos, hq, hk, d, rot, 1 if interleaved else 0, _float_code(where, q), eps, 0), \
        (n, hq, d), (n, hk, d)


def hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos, eps: float = 1e-6, interleaved: bool = False, q_out=None,
                        k_out=None, stream=None):
    """Per-head norm and position rotation: q [n, heads, d], k [n, kv_heads, d]
    or None (views of a packed projection are used where they lie), wq, wk
    float32 [d] or None, table [positions, rot] from hg_rope_table, pos int32
    [n].  Returns (q_out, k_out); they may be q and k themselves."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos, eps, interleaved, q_out, k_out)
    where = "hg_qk_norm_rope_fwd"
    desc, qs, ks = _rope_desc(where, q, k, table, eps, interleaved)
    if q_out is None:
        q_out = torch.empty(qs, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = torch.empty(ks, dtype=q.dtype, device=q.device)
    _same(where, q, k, q_out, k_out)
    hk, hl = (None, None) if k is None else (_heads(where, "k", k, ks), _heads(where, "k_out", k_out, ks))
    st = lib().hg_qk_norm_rope_fwd(desc, _heads(where, "q", q, qs), hk, _vector(where, wq, qs[2], q),
                                   _vector(where, wk, qs[2], q), table.data_ptr(),
                                   _vector(where, pos, qs[0], q, torch.int32), _heads(where, "q_out", q_out, qs), hl,
                                   _raw_stream(q))
    if st:
        _check(st, where)
    return q_out, k_out


def hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, dq_out, dk_out, eps: float = 1e-6, interleaved: bool = False,
                        dq=None, dk=None, dwq=None, dwk=None, accumulate: bool = False, ws=None, stream=None):
    """Returns (dq, dk, dwq, dwk) of hg_qk_norm_rope_fwd (q and k as it read
    them); dwq and dwk for the weights given, added into when accumulate."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, dq_out, dk_out, eps, interleaved, dq,
                                       dk, dwq, dwk, accumulate, ws)
    where = "hg_qk_norm_rope_bwd"
    L = lib()
    desc, qs, ks = _rope_desc(where, q, k, table, eps, interleaved)
    if accumulate and ((wq is not None and dwq is None) or (wk is not None and dwk is None)):
        raise ValueError(f"{where}: accumulate needs the buffers to add into")
    if dq is None:
        dq = torch.empty(qs, dtype=q.dtype, device=q.device)
    if k is not None and dk is None:
        dk = torch.empty(ks, dtype=q.dtype, device=q.device)
    if dwq is None and wq is not None:
        dwq = torch.empty_like(wq)
    if dwk is None and wk is not None:
        dwk = torch.empty_like(wk)
    _same(where, q, k, dq_out, dk_out, dq, dk)
    h = [_heads(where, n, t, qs) for n, t in (("q", q), ("dq_out", dq_out), ("dq", dq))]
    g = [None if k is None else _heads(where, n, t, ks) for n, t in (("k", k), ("dk_out", dk_out), ("dk", dk))]
    ws, wp, wn = _workspace(where, ws, L.hg_qk_norm_rope_bwd_workspace_size(desc), q)
    d = qs[2]
    st = L.hg_qk_norm_rope_bwd(desc, h[0], g[0], _vector(where, wq, d, q), _vector(where, wk, d, q), table.data_ptr(),
                               _vector(where, pos, qs[0], q, torch.int32), h[1], g[1], h[2], g[2],
                               _vector(where, dwq, d, q), _vector(where, dwk, d, q), 1 if accumulate else 0, wp, wn,
                               _raw_stream(q))
    if st:
        _check(st, where)
    return dq, dk, dwq, dwk


def _state(where, s, shape, like):
    if s is None:
        return None
    if s.shape != shape or s.dtype is not torch.float32 or s.get_device() != like.get_device() or not s.is_contiguous():
        raise ValueError(f"{where}: expected a contiguous float32 state {tuple(shape)}, got {tuple(s.shape)} {s.dtype}")
    return s.data_ptr()


def hg_linattn_fwd_workspace_size(batch: int, t: int, heads: int, kv_heads: int, d: int, dtype=torch.float32) -> int:
    return int(lib().hg_linattn_fwd_workspace_size(_pack_linattn(t, batch, heads, kv_heads, d, _DTYPES[dtype], 1.0)))


def hg_linattn_bwd_workspace_size(batch: int, t: int, heads: int, kv_heads: int, d: int, dtype=torch.float32) -> int:
    return int(lib().hg_linattn_bwd_workspace_size(_pack_linattn(t, batch, heads, kv_heads, d, _DTYPES[dtype], 1.0)))


def hg_linattn_fwd(q, k, v, log_decay, scale: float = 1.0, lens=None, state=None, o=None, state_out=None,
                   want_state: bool = False, ws=None, stream=None):
    """Linear attention with a decay for each head: q [b, t, heads, d], k, v
    [b, t, kv_heads, d], log_decay float32 [heads], lens int32 [b] or None,
    state float32 [b, heads, d, d] or None.  Returns (o, state_out); state_out
    is None unless given or wanted."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_linattn_fwd(q, k, v, log_decay, scale, lens, state, o, state_out, want_state, ws)
    where = "hg_linattn_fwd"
    L = lib()
    qs = q.shape
    b, t, h, d = qs
    if state_out is None and want_state:
        state_out = torch.empty((b, h, d, d), dtype=torch.float32, device=q.device)
    if o is None:
        o = torch.empty(qs, dtype=q.dtype, device=q.device)
    _same(where, q, k, v, o)
    kv = (b, t, k.shape[2], d)
    desc = _pack_linattn(t, b, h, kv[2], d, _float_code(where, q), scale)
    ws, wp, wn = _workspace(where, ws, L.hg_linattn_fwd_workspace_size(desc), q)
    st = L.hg_linattn_fwd(desc, _heads(where, "q", q, qs), _heads(where, "k", k, kv), _heads(where, "v", v, kv),
                          _vector(where, log_decay, h, q), _vector(where, lens, b, q, torch.int32),
                          _state(where, state, (b, h, d, d), q), _heads(where, "o", o, qs),
                          _state(where, state_out, (b, h, d, d), q), wp, wn, _raw_stream(q))
    if st:
        _check(st, where)
    return o, state_out


def hg_linattn_bwd(q, k, v, log_decay, do, scale: float = 1.0, lens=None, state=None, dstate_out=None, dq=None,
                   dk=None, dv=None, dstate=None, ws=None, stream=None):
    """Returns (dq, dk, dv, dstate) of hg_linattn_fwd for do = dL/do and
    dstate_out = dL/dstate_out (or None); dstate is None unless a state or a
    buffer is given."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_linattn_bwd(q, k, v, log_decay, do, scale, lens, state, dstate_out, dq, dk, dv, dstate, ws)
    where = "hg_linattn_bwd"
    L = lib()
    qs = q.shape
    b, t, h, d = qs
    s = (b, h, d, d)
    kv = (b, t, k.shape[2], d)
    if dstate is None and state is not None:
        dstate = torch.empty(s, dtype=torch.float32, device=q.device)
    dq = torch.empty(qs, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(kv, dtype=q.dtype, device=q.device) if dk is None else dk
    dv = torch.empty(kv, dtype=q.dtype, device=q.device) if dv is None else dv
    _same(where, q, k, v, do, dq, dk, dv)
    desc = _pack_linattn(t, b, h, kv[2], d, _float_code(where, q), scale)
    ws, wp, wn = _workspace(where, ws, L.hg_linattn_bwd_workspace_size(desc), q)
    st = L.hg_linattn_bwd(desc, _heads(where, "q", q, qs), _heads(where, "k", k, kv), _heads(where, "v", v, kv),
                          _vector(where, log_decay, h, q), _vector(where, lens, b, q, torch.int32),
                          _state(where, state, s, q), _heads(where, "do", do, qs), _state(where, dstate_out, s, q),
                          _heads(where, "dq", dq, qs), _heads(where, "dk", dk, kv), _heads(where, "dv", dv, kv),
                          _state(where, dstate, s, q), wp, wn, _raw_stream(q))
    if st:
        _check(st, where)
    return dq, dk, dv, dstate


def hg_linattn_step(q, k, v, log_decay, states, slots=None, scale: float = 1.0, o=None, stream=None):
    """One token for each row: q [b, heads, d], k, v [b, kv_heads, d], states
    float32 [n, heads, d, d] updated in place, slots int32 [b] (None: row b
    has state b; a slot outside the states: an idle row).  Returns o."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_linattn_step(q, k, v, log_decay, states, slots, scale, o)
    where = "hg_linattn_step"
    b, h, d = q.shape
    hk = k.shape[1]
    if o is None:
        o = torch.empty((b, h, d), dtype=q.dtype, device=q.device)
    _same(where, q, k, v, o)
    n = states.shape[0]
    qs, ks = (b, h, d), (b, hk, d)
    st = lib().hg_linattn_step(_pack_linattn(1, b, h, hk, d, _float_code(where, q), scale),
                               _heads(where, "q", q, qs, True), _heads(where, "k", k, ks, True),
                               _heads(where, "v", v, ks, True), _vector(where, log_decay, h, q),
                               _state(where, states, (n, h, d, d), q), _vector(where, slots, b, q, torch.int32), n,
                               _heads(where, "o", o, qs, True), _raw_stream(q))
    if st:
        _check(st, where)
    return o


# ---- recurrent block and its training -----------------------------------------

def _channels(where: str, name: str, t, shape) -> bytes:
    """hg_heads of [batch, tokens, width] rows, or of [n, width] ones (a token
    each).  The stride of a dimension with one entry is never walked."""
    s = t.stride()
    if t.shape != shape or (s[-1] != 1 and shape[-1] > 1 and t.numel()):
        raise ValueError(f"{where}: expected {name} {tuple(shape)} with unit column stride, got {tuple(t.shape)} strides {s}")
    if len(s) == 2:
        return _pack_heads(t.data_ptr(), s[0] if shape[0] > 1 else 0, 0, 0)
    return _pack_heads(t.data_ptr(), s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, 0)


def hg_recur_fwd_workspace_size(batch: int, t: int, width: int, dtype=torch.float32) -> int:
    return int(lib().hg_recur_fwd_workspace_size(_pack_recur(t, batch, width, _DTYPES[dtype], 1.0)))


def hg_recur_bwd_workspace_size(batch: int, t: int, width: int, dtype=torch.float32) -> int:
    return int(lib().hg_recur_bwd_workspace_size(_pack_recur(t, batch, width, _DTYPES[dtype], 1.0)))


def hg_recur_fwd(x, r, i, decay, rate: float = 8.0, lens=None, state=None, h=None, state_out=None,
                 want_state: bool = False, ws=None, stream=None):
    """Gated linear recurrence: x and its gates r and i [b, t, width] (views of a
    packed projection are used where they lie), decay float32 [width], lens int32
    [b] or None, state float32 [b, width] or None.  Returns (h, state_out);
    state_out is None unless given or wanted."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_recur_fwd(x, r, i, decay, rate, lens, state, h, state_out, want_state, ws)
    where = "hg_recur_fwd"
    L = lib()
    xs = x.shape
    b, t, w = xs
    if state_out is None and want_state:
        state_out = torch.empty((b, w), dtype=torch.float32, device=x.device)
    if h is None:
        h = torch.empty(xs, dtype=x.dtype, device=x.device)
    _same(where, x, r, i, h)
    desc = _pack_recur(t, b, w, _float_code(where, x), rate)
    ws, wp, wn = _workspace(where, ws, L.hg_recur_fwd_workspace_size(desc), x)
    st = L.hg_recur_fwd(desc, _channels(where, "x", x, xs), _channels(where, "r", r, xs), _channels(where, "i", i, xs),
                        _vector(where, decay, w, x), _vector(where, lens, b, x, torch.int32),
                        _state(where, state, (b, w), x), _channels(where, "h", h, xs),
                        _state(where, state_out, (b, w), x), wp, wn, _raw_stream(x))
    if st:
        _check(st, where)
    return h, state_out


def hg_recur_bwd(x, r, i, decay, h, dh, rate: float = 8.0, lens=None, state=None, dstate_out=None, dx=None, dr=None,
                 di=None, ddecay=None, dstate=None, accumulate: bool = False, ws=None, stream=None):
    """Returns (dx, dr, di, ddecay, dstate) of hg_recur_fwd, whose output h was,
    for dh = dL/dh and dstate_out = dL/dstate_out (or None); ddecay is added into
    the given buffer when accumulate; dstate is None unless a state or a buffer
    is given."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_recur_bwd(x, r, i, decay, h, dh, rate, lens, state, dstate_out, dx, dr, di, ddecay, dstate,
                                accumulate, ws)
    where = "hg_recur_bwd"
    L = lib()
    xs = x.shape
    b, t, w = xs
    if accumulate and ddecay is None:
        raise ValueError(f"{where}: accumulate needs the buffer to add into")
    if dstate is None and state is not None:
        dstate = torch.empty((b, w), dtype=torch.float32, device=x.device)
    dx, dr, di = (torch.empty(xs, dtype=x.dtype, device=x.device) if g is None else g for g in (dx, dr, di))
    if ddecay is None:
        ddecay = torch.empty_like(decay)
    _same(where, x, r, i, h, dh, dx, dr, di)
    desc = _pack_recur(t, b, w, _float_code(where, x), rate)
    ws, wp, wn = _workspace(where, ws, L.hg_recur_bwd_workspace_size(desc), x)
    ch = [_channels(where, n, v, xs) for n, v in (("x", x), ("r", r), ("i", i), ("h", h), ("dh", dh), ("dx", dx),
                                                  ("dr", dr), ("di", di))]
    st = L.hg_recur_bwd(desc, *ch[:3], _vector(where, decay, w, x), _vector(where, lens, b, x, torch.int32),
                        _state(where, state, (b, w), x), *ch[3:5], _state(where, dstate_out, (b, w), x), *ch[5:],
                        _vector(where, ddecay, w, x), _state(where, dstate, (b, w), x), 1 if accumulate else 0, wp, wn,
                        _raw_stream(x))
    if st:
        _check(st, where)
    return dx, dr, di, ddecay, dstate


def hg_recur_step(x, r, i, decay, states, slots=None, rate: float = 8.0, h=None, stream=None):
    """One token for each row: x, r, i [b, width], states float32 [n, width]
    updated in place, slots int32 [b] (None: row b has state b; a slot outside
    the states: an idle row).  Returns h."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_recur_step(x, r, i, decay, states, slots, rate, h)
    where = "hg_recur_step"
    xs = x.shape
    b, w = xs
    if h is None:
        h = torch.empty(xs, dtype=x.dtype, device=x.device)
    _same(where, x, r, i, h)
    n = states.shape[0]
    st = lib().hg_recur_step(_pack_recur(1, b, w, _float_code(where, x), rate), _channels(where, "x", x, xs),
                             _channels(where, "r", r, xs), _channels(where, "i", i, xs), _vector(where, decay, w, x),
                             _state(where, states, (n, w), x), _vector(where, slots, b, x, torch.int32), n,
                             _channels(where, "h", h, xs), _raw_stream(x))
    if st:
        _check(st, where)
    return h


def hg_group_norm_fwd_workspace_size(batch: int, t: int, width: int, groups: int, dtype=torch.float32) -> int:
    return int(lib().hg_group_norm_fwd_workspace_size(_pack_group_norm(t, batch, width, groups, _DTYPES[dtype], 0, 1.0)))


def hg_group_norm_bwd_workspace_size(batch: int, t: int, width: int, groups: int, dtype=torch.float32) -> int:
    return int(lib().hg_group_norm_bwd_workspace_size(_pack_group_norm(t, batch, width, groups, _DTYPES[dtype], 0, 1.0)))


def _group_norm_desc(where, x, groups, act, eps):
    if x.dim() not in (2, 3):
        raise ValueError(f"{where}: rows are [batch, t, width] or [n, width], got {tuple(x.shape)}")
    b, w = x.shape[0], x.shape[-1]
    return _pack_group_norm(x.shape[1] if x.dim() == 3 else 1, b, w, groups, _float_code(where, x), act, eps), b, w


def hg_group_norm_fwd(x, groups: int, w=None, b=None, act: int = HG_ACT_NONE, eps: float = 1e-5, lens=None, y=None,
                      stats=None, want_stats: bool = False, ws=None, stream=None):
    """act(w (x - mean) / sqrt(var + eps) + b) over the tokens and the channels of
    each group: x [batch, t, width], or [n, width] for every row by itself; w, b
    float32 [width] or None, lens int32 [batch] or None.  Returns (y, stats):
    stats float32 [batch, groups, 2] for the backward, None unless given or
    wanted."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_group_norm_fwd(x, groups, w, b, act, eps, lens, y, stats, want_stats, ws)
    where = "hg_group_norm_fwd"
    L = lib()
    desc, n, width = _group_norm_desc(where, x, groups, act, eps)
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if stats is None and want_stats:
        stats = torch.empty((n, groups, 2), dtype=torch.float32, device=x.device)
    _same(where, x, y)
    ws, wp, wn = _workspace(where, ws, L.hg_group_norm_fwd_workspace_size(desc), x)
    st = L.hg_group_norm_fwd(desc, _channels(where, "x", x, x.shape), _vector(where, w, width, x),
                             _vector(where, b, width, x), _vector(where, lens, n, x, torch.int32),
                             _channels(where, "y", y, x.shape), _state(where, stats, (n, groups, 2), x), wp, wn,
                             _raw_stream(x))
    if st:
        _check(st, where)
    return y, stats


def hg_group_norm_bwd(x, groups: int, w, b, stats, dy, act: int = HG_ACT_NONE, eps: float = 1e-5, lens=None, dx=None,
                      dw=None, db=None, accumulate: bool = False, ws=None, stream=None):
    """Returns (dx, dw, db) of hg_group_norm_fwd, whose stats these are, for dy =
    dL/dy; dw and db for the vectors given, added into when accumulate."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_group_norm_bwd(x, groups, w, b, stats, dy, act, eps, lens, dx, dw, db, accumulate, ws)
    where = "hg_group_norm_bwd"
    L = lib()
    desc, n, width = _group_norm_desc(where, x, groups, act, eps)
    if accumulate and ((w is not None and dw is None) or (b is not None and db is None)):
        raise ValueError(f"{where}: accumulate needs the buffers to add into")
    if dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if dw is None and w is not None:
        dw = torch.empty_like(w)
    if db is None and b is not None:
        db = torch.empty_like(b)
    _same(where, x, dy, dx)
    ws, wp, wn = _workspace(where, ws, L.hg_group_norm_bwd_workspace_size(desc), x)
    st = L.hg_group_norm_bwd(desc, _channels(where, "x", x, x.shape), _vector(where, w, width, x),
                             _vector(where, b, width, x), _vector(where, lens, n, x, torch.int32),
                             _state(where, stats, (n, groups, 2), x), _channels(where, "dy", dy, x.shape),
                             _channels(where, "dx", dx, x.shape), _vector(where, dw, width, x),
                             _vector(where, db, width, x), 1 if accumulate else 0, wp, wn, _raw_stream(x))
    if st:
        _check(st, where)
    return dx, dw, db


def hg_muon_workspace_size(count: int, rows: int, cols: int, dtype=torch.float32, steps: int = 5) -> int:
    return int(lib().hg_muon_workspace_size(_pack_muon(count, rows, cols, _DTYPES[dtype], steps, 1, 0.0, 0.0, 0.0, 1.0,
                                                       1.0, 0)))


def hg_muon_step(param, grad, momentum, lr: float, mu: float = 0.95, weight_decay: float = 0.0, nesterov: bool = True,
                 steps: int = 5, scale: Optional[float] = None, eps: float = 1e-7, ws=None, stream=None):
    """One update of matrices along their orthogonalised momentum, in place on
    param and momentum: param and grad [rows, cols] or [count, rows, cols],
    float32 or bfloat16, momentum float32.  scale None: sqrt(max(1, rows / cols)), the
    published factor for weights stored [outputs, inputs]; the weights of
    hg_linear_fwd and hg_glu_fwd are [inputs, outputs], for which it is
    sqrt(max(1, cols / rows)): give it as scale (as encoder.train does)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hg_muon_step(param, grad, momentum, lr, mu, weight_decay, nesterov, steps, scale, eps, ws)
    where = "hg_muon_step"
    L = lib()
    shape = param.shape
    if param.dim() not in (2, 3):
        raise ValueError(f"{where}: matrices are [rows, cols] or [count, rows, cols], got {tuple(shape)}")
    _same(where, param, grad)
    if grad.shape != shape or not grad.is_contiguous() or not param.is_contiguous():
        raise ValueError(f"{where}: expected contiguous {tuple(shape)}, got param strides {param.stride()}, grad "
                         f"{tuple(grad.shape)} strides {grad.stride()}")
    count = shape[0] if len(shape) == 3 else 1
    rows, cols = shape[-2:]
    if scale is None:
        scale = max(1.0, rows / max(1, cols)) ** 0.5
    desc = _pack_muon(count, rows, cols, _float_code(where, param), steps, 1 if nesterov else 0, lr, mu, weight_decay,
                      scale, eps, 0)
    ws, wp, wn = _workspace(where, ws, L.hg_muon_workspace_size(desc), param)
    st = L.hg_muon_step(desc, param.data_ptr(), grad.data_ptr(), _state(where, momentum, shape, param), wp, wn,
                        _raw_stream(param))
    if st:
        _check(st, where)


def hg_timing_enable(on: bool = True):
    _check(lib().hg_timing_enable(int(on)), "hg_timing_enable")


def hg_timing_collect(cap: int = 256) -> dict:
    """{kernel name: (launches, total_ms)} since the last collect."""
    names = (C.c_char * 64 * cap)()
    launches = (C.c_int64 * cap)()
    total = (C.c_double * cap)()
    n = lib().hg_timing_collect(names, launches, total, cap)
    if n < 0:
        _check(n, "hg_timing_collect")
    out = {}
    for i in range(min(n, cap)):
        out[bytes(names[i]).split(b"\0", 1)[0].decode()] = (int(launches[i]), float(total[i]))
    return out
