"""Thin ctypes binding of libgdp (the C ABI in include/gdp.h).

Only argument marshalling happens here: torch tensors provide device memory
and the current HIP stream; every step of the forward pass runs in the
library's HIP kernels.  Importing this module fails loudly when libgdp.so has
not been built -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_uint64, c_void_p
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgdp.so")

GDP_OK = 0
GDP_E_INVALID_ARG = -1
GDP_E_BAD_GRAPH = -2
GDP_E_UNSUPPORTED = -3
GDP_E_WORKSPACE = -4
GDP_E_HIP = -5
GDP_F32 = 0
GDP_BF16 = 1
GDP_TOPO_IDS = 1
GDP_MAX_GRAPHS = 128
GDP_NOALLOC_SCRATCH_BYTES = 4 << 20

KERNEL_KINDS = ["graph_prep", "nbr_sample", "gemm_pool_sigmoid", "gather_max", "gemm_update_relu",
                "meanpool", "film", "pre_layer", "seg_attention", "post_attn",
                "head_lse", "gumbel_sample", "logp_reduce", "mlp_placer", "ppo_grad", "head_backward", "advantages",
                "evaluate", "train_forward", "backward", "adam", "log_prob", "gemm_update_pool", "layer_norm",
                "layer_norm_backward", "fc", "fc_backward", "rel_attention", "rel_attention_backward"]
K_COUNT = len(KERNEL_KINDS)


class GdpError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libgdp error {code}: {msg}")
        self.code = code


class GdpGraph(ctypes.Structure):
    _fields_ = [("n_graphs", c_int32), ("graph_ptr_h", POINTER(c_int32)), ("n_nodes", c_int32),
                ("row_ptr", c_void_p), ("col_idx", c_void_p), ("n_edges", c_int64), ("x", c_void_p),
                ("feat_dim", c_int32), ("dtype", c_int32), ("flags", c_uint32)]


class GdpGnnLayer(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("w_pool", "b_pool", "w_self", "w_neigh", "b_upd")]


class GdpGnn(ctypes.Structure):
    _fields_ = [("n_layers", c_int32), ("in_dim", c_int32), ("hidden", c_int32), ("fanout", c_int32),
                ("nbr_seed", c_uint64), ("layers", POINTER(GdpGnnLayer))]


PLACER_LAYER_FIELDS = ("film_wg", "film_bg", "film_wb", "film_bb", "w_qkv", "b_qkv", "w_o", "b_o",
                       "ln1_g", "ln1_b", "w_1", "b_1", "w_2", "b_2", "ln2_g", "ln2_b")


class GdpPlacerLayer(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in PLACER_LAYER_FIELDS]


class GdpPlacer(ctypes.Structure):
    _fields_ = [("n_layers", c_int32), ("d_model", c_int32), ("n_heads", c_int32), ("d_ff", c_int32),
                ("seg_len", c_int32), ("mem_len", c_int32), ("n_devices", c_int32), ("film", c_int32),
                ("attention", c_int32),
                ("layers", POINTER(GdpPlacerLayer)), ("w_out", c_void_p), ("b_out", c_void_p)]


class GdpGnnLayerGrad(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("w_pool", "b_pool", "w_self", "w_neigh", "b_upd")]


class GdpPlacerLayerGrad(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in PLACER_LAYER_FIELDS]


class GdpGrads(ctypes.Structure):
    _fields_ = [("gnn", POINTER(GdpGnnLayerGrad)), ("placer", POINTER(GdpPlacerLayerGrad)), ("w_out", c_void_p),
                ("b_out", c_void_p)]


class GdpAdamTensor(ctypes.Structure):
    _fields_ = [("param", c_void_p), ("master", c_void_p), ("grad", c_void_p), ("m", c_void_p), ("v", c_void_p),
                ("n", c_int64)]


class GdpFcLayer(ctypes.Structure):
    _fields_ = [("rows", c_int64), ("in_dim", c_int32), ("out_dim", c_int32), ("dtype", c_int32), ("act", c_int32)] + \
               [(n, c_int64) for n in ("ld_x", "ld_y", "ld_res", "ld_act", "ld_dy", "ld_dx", "ld_dx_add")]


class GdpRelAttn(ctypes.Structure):
    _fields_ = [("n_graphs", c_int32), ("key_start_h", POINTER(c_int32)), ("len_h", POINTER(c_int32)),
                ("n_query_h", POINTER(c_int32)), ("n_heads", c_int32), ("n_kv_heads", c_int32),
                ("head_dim", c_int32), ("seg_len", c_int32), ("mem_len", c_int32), ("causal", c_int32),
                ("n_bounds", c_int32), ("bounds_h", POINTER(c_int32)), ("dtype", c_int32), ("scale", c_float)] + \
               [(n, c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_o", "ld_do", "ld_dq", "ld_dk", "ld_dv")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1910_01578_amd.build_lib` "
                          "(there is no fallback path)")
    # torch ships its own HIP runtime under the same soname (libamdhip64.so.7).
    # Loading torch first makes libgdp bind to that copy; loaded the other way
    # round the process would hold two runtimes, and pointers and streams from
    # torch would not be valid in the one libgdp calls.
    import torch  # noqa: F401
    lib = ctypes.CDLL(LIB_PATH)
    sig = {
        "gdp_workspace_bytes": (c_size_t, [POINTER(GdpGraph), POINTER(GdpGnn), POINTER(GdpPlacer), c_int32]),
        "gdp_embed": (c_int32, [POINTER(GdpGraph), POINTER(GdpGnn), c_void_p, c_void_p, c_void_p, c_size_t,
                                c_void_p]),
        "gdp_place": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, POINTER(GdpPlacer), c_void_p, c_void_p,
                                c_void_p, c_size_t, c_void_p]),
        "gdp_sample": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, c_int32, c_int32, c_uint64, c_void_p,
                                 c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
        "gdp_place_sample": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, POINTER(GdpPlacer), c_void_p,
                                       c_void_p, c_int32, c_uint64, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_size_t, c_void_p]),
        "gdp_sample_noalloc": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, c_int32, c_int32, c_uint64,
                                         c_void_p, c_void_p, c_void_p, c_void_p]),
        "gdp_evaluate_workspace_bytes": (c_size_t, [POINTER(GdpGraph), c_int32, c_int32]),
        "gdp_evaluate": (c_int32, [POINTER(GdpGraph), c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                   POINTER(c_int64), c_double, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                   c_void_p]),
        "gdp_train_sizes": (c_int32, [POINTER(GdpGraph), POINTER(GdpGnn), POINTER(GdpPlacer), POINTER(c_size_t),
                                      POINTER(c_size_t)]),
        "gdp_forward_train": (c_int32, [POINTER(GdpGraph), POINTER(GdpGnn), POINTER(GdpPlacer), c_void_p, c_size_t,
                                        c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
        "gdp_backward": (c_int32, [POINTER(GdpGraph), POINTER(GdpGnn), POINTER(GdpPlacer), c_void_p, c_size_t,
                                   c_void_p, POINTER(GdpGrads), c_void_p, c_size_t, c_void_p]),
        "gdp_log_prob": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p,
                                   c_void_p, c_size_t, c_void_p]),
        "gdp_adam_step": (c_int32, [c_int32, POINTER(GdpAdamTensor), c_int32, c_float, c_float, c_float, c_float,
                                    c_int64, c_void_p]),
        "gdp_debug_train_tensor": (c_int32, [POINTER(GdpGraph), POINTER(GdpGnn), POINTER(GdpPlacer), c_void_p,
                                             c_size_t, c_int32, c_int32, c_void_p, c_size_t, c_void_p]),
        "gdp_validate_graph_host": (c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_int64, c_uint32]),
        "gdp_last_error": (c_char_p, []),
        "gdp_abi_version": (c_int32, []),
        "gdp_advantages": (c_int32, [c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                     c_void_p]),
        "gdp_place_train": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, POINTER(GdpPlacer), c_void_p, c_void_p,
                                      c_void_p, c_void_p, c_size_t, c_void_p]),
        "gdp_head_backward": (c_int32, [POINTER(GdpGraph), POINTER(GdpPlacer), c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_void_p, c_size_t, c_void_p]),
        "gdp_ppo_grad": (c_int32, [POINTER(GdpGraph), c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_float, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
        "gdp_debug_uniforms": (c_int32, [c_uint64, c_int32, c_int32, c_int32, c_void_p, c_void_p]),
        "gdp_debug_neighbors": (c_int32, [POINTER(GdpGraph), POINTER(GdpGnn), c_void_p, c_void_p, c_int64,
                                          c_void_p, c_size_t, c_void_p]),
        "gdp_layer_norm": (c_int32, [c_int64, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                     c_void_p, c_float, c_void_p, c_int64, c_void_p, c_int64, c_void_p]),
        "gdp_layer_norm_workspace_bytes": (c_size_t, [c_int64, c_int32]),
        "gdp_layer_norm_backward": (c_int32, [c_int64, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_float,
                                              c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                              c_void_p, c_void_p, c_size_t, c_void_p]),
        "gdp_fc": (c_int32, [POINTER(GdpFcLayer)] + [c_void_p] * 7),
        "gdp_fc_workspace_bytes": (c_size_t, [POINTER(GdpFcLayer)]),
        "gdp_fc_backward": (c_int32, [POINTER(GdpFcLayer)] + [c_void_p] * 9 + [c_size_t, c_void_p]),
        "gdp_rel_attention_workspace_bytes": (c_size_t, [POINTER(GdpRelAttn), c_int32]),
        "gdp_rel_attention": (c_int32, [POINTER(GdpRelAttn)] + [c_void_p] * 8 + [c_size_t, c_void_p]),
        "gdp_rel_attention_backward": (c_int32, [POINTER(GdpRelAttn)] + [c_void_p] * 13 + [c_size_t, c_void_p]),
        "gdp_set_place_streams": (c_int32, [c_int32]),
        "gdp_timer_begin": (c_int32, [c_uint32]),
        "gdp_timer_end": (c_int32, [POINTER(c_double), POINTER(c_int64)]),
        "gdp_kernel_kind_name": (c_char_p, [c_int32]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


lib = _load()


def last_error() -> str:
    return lib.gdp_last_error().decode()


def check(code: int):
    if code != GDP_OK:
        raise GdpError(code, last_error())


def abi_version() -> int:
    return lib.gdp_abi_version()


def validate_graph_host(graph_ptr, row_ptr, col_idx, flags: int = GDP_TOPO_IDS) -> int:
    gp = np.ascontiguousarray(graph_ptr, np.int32)
    rp = np.ascontiguousarray(row_ptr, np.int32)
    ci = np.ascontiguousarray(col_idx, np.int32)
    return lib.gdp_validate_graph_host(gp.ctypes.data, gp.size - 1, rp.ctypes.data, rp.size - 1,
                                       ci.ctypes.data if ci.size else None, ci.size, flags)


# ----------------------------------------------------------------------------
# torch-facing helpers: device memory and the current stream only.
# ----------------------------------------------------------------------------

def _torch():
    import torch
    return torch


def _stream_handle(stream=None) -> int:
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def to_device(arr: np.ndarray, dtype: str, device="cuda"):
    """Upload a float32 array (dtype "f32") or uint16 bf16 bit patterns ("bf16")."""
    torch = _torch()
    a = np.ascontiguousarray(arr)
    if dtype == "bf16":
        assert a.dtype == np.uint16
        return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16).to(device)
    assert a.dtype == np.float32
    return torch.from_numpy(a).to(device)


class DeviceGraph:
    """A graph batch resident in device memory plus its C descriptor."""

    def __init__(self, graph, dtype: str, device="cuda", flags: int = GDP_TOPO_IDS):
        torch = _torch()
        self.dtype = dtype
        self.graph_ptr = np.ascontiguousarray(graph.graph_ptr, np.int32)
        self.row_ptr = torch.from_numpy(np.ascontiguousarray(graph.row_ptr, np.int32)).to(device)
        ci = np.ascontiguousarray(graph.col_idx, np.int32)
        self.col_idx = torch.from_numpy(ci if ci.size else np.zeros(1, np.int32)).to(device)
        self.x = to_device(graph.x_dev, dtype, device)
        self.n_nodes = int(graph.row_ptr.size - 1)
        self.n_edges = int(ci.size)
        self.feat_dim = int(graph.x_dev.shape[1])
        self.n_graphs = int(self.graph_ptr.size - 1)
        self.c = GdpGraph(self.n_graphs, self.graph_ptr.ctypes.data_as(POINTER(c_int32)), self.n_nodes,
                          self.row_ptr.data_ptr(), self.col_idx.data_ptr(), self.n_edges, self.x.data_ptr(),
                          self.feat_dim, GDP_BF16 if dtype == "bf16" else GDP_F32, flags)


class DevicePolicy:
    """Policy weights resident in device memory plus the C descriptors."""

    def __init__(self, cfg, weights, device="cuda", film: Optional[bool] = None,
                 attention: Optional[bool] = None):
        self.cfg = cfg
        dt = cfg.dtype
        up = lambda pair: to_device(pair[1], dt, device)
        self.gnn_t = [{k: up(v) for k, v in l.items()} for l in weights.gnn]
        self.placer_t = [{k: up(v) for k, v in l.items()} for l in weights.placer]
        self.head_t = {k: up(v) for k, v in weights.head.items()}
        L = len(self.gnn_t)
        self._gl = (GdpGnnLayer * L)(*[GdpGnnLayer(*[l[k].data_ptr() for k in ("w_pool", "b_pool", "w_self",
                                                                              "w_neigh", "b_upd")])
                                       for l in self.gnn_t])
        self.gnn = GdpGnn(L, cfg.feat_dim, cfg.hidden, cfg.fanout, cfg.nb_seed, self._gl)
        P = len(self.placer_t)
        self._pl = (GdpPlacerLayer * P)(*[GdpPlacerLayer(*[l[k].data_ptr() for k in PLACER_LAYER_FIELDS])
                                          for l in self.placer_t])
        use_film = cfg.film if film is None else film
        use_attention = cfg.attention if attention is None else attention
        self.placer = GdpPlacer(P, cfg.d_model, cfg.heads, cfg.d_ff, cfg.seg_len, cfg.mem_len, cfg.n_devices,
                                1 if use_film else 0, 1 if use_attention else 0, self._pl,
                                self.head_t["w_out"].data_ptr(), self.head_t["b_out"].data_ptr())


class Runner:
    """Owns the outputs and the workspace of one (graph, policy, K) problem."""

    def __init__(self, graph: DeviceGraph, policy: DevicePolicy, k_samples: int, device="cuda"):
        torch = _torch()
        self.graph, self.policy, self.k = graph, policy, int(k_samples)
        cfg = policy.cfg
        tdt = torch.bfloat16 if graph.dtype == "bf16" else torch.float32
        N, G, H, D = graph.n_nodes, graph.n_graphs, cfg.hidden, cfg.n_devices
        self.ws_bytes = lib.gdp_workspace_bytes(ctypes.byref(graph.c), ctypes.byref(policy.gnn),
                                                ctypes.byref(policy.placer), self.k)
        if self.ws_bytes == 0:
            raise GdpError(GDP_E_INVALID_ARG, last_error())
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.node_emb = torch.empty((N, H), dtype=tdt, device=device)
        self.graph_emb = torch.empty((G, H), dtype=torch.float32, device=device)
        self.logits = torch.empty((N, D), dtype=torch.float32, device=device)
        self.lse = torch.empty((N,), dtype=torch.float32, device=device)
        self.placements = torch.empty((self.k, N), dtype=torch.int32, device=device)
        self.logp = torch.empty((G, self.k), dtype=torch.float32, device=device)

    def embed(self, stream=None):
        check(lib.gdp_embed(ctypes.byref(self.graph.c), ctypes.byref(self.policy.gnn), self.node_emb.data_ptr(),
                            self.graph_emb.data_ptr(), self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))

    def place(self, stream=None):
        check(lib.gdp_place(ctypes.byref(self.graph.c), self.node_emb.data_ptr(), self.graph_emb.data_ptr(),
                            ctypes.byref(self.policy.placer), self.logits.data_ptr(), self.lse.data_ptr(),
                            self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))

    def place_train(self, stream=None):
        """place() that also keeps the placement network's output X [N, d] (fp32),
        the head's input, for head_backward(); returns X."""
        torch = _torch()
        x = torch.empty((self.graph.n_nodes, self.policy.cfg.d_model), dtype=torch.float32, device=self.ws.device)
        check(lib.gdp_place_train(ctypes.byref(self.graph.c), self.node_emb.data_ptr(), self.graph_emb.data_ptr(),
                                  ctypes.byref(self.policy.placer), self.logits.data_ptr(), self.lse.data_ptr(),
                                  x.data_ptr(), self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))
        return x

    def head_backward(self, x, dlogits, stream=None):
        """The head's backward pass for dL/dlogits: returns (dx, dw_out, db_out), fp32."""
        torch = _torch()
        N, d, D = self.graph.n_nodes, self.policy.cfg.d_model, self.policy.cfg.n_devices
        dev = self.ws.device
        dx = torch.empty((N, d), dtype=torch.float32, device=dev)
        dw = torch.empty((D, d), dtype=torch.float32, device=dev)
        db = torch.empty((D,), dtype=torch.float32, device=dev)
        check(lib.gdp_head_backward(ctypes.byref(self.graph.c), ctypes.byref(self.policy.placer), x.data_ptr(),
                                    dlogits.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(),
                                    self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))
        return dx, dw, db

    def sample(self, seed: int, uniforms=None, use_lse: bool = True, stream=None):
        check(lib.gdp_sample(ctypes.byref(self.graph.c), self.logits.data_ptr(),
                             self.lse.data_ptr() if use_lse else None, self.policy.cfg.n_devices, self.k, seed,
                             None if uniforms is None else uniforms.data_ptr(), self.placements.data_ptr(),
                             self.logp.data_ptr(), self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))

    def sample_noalloc(self, seed: int, placements=None, logp=None, uniforms=None, use_lse: bool = True,
                       stream=None):
        """sample() through gdp_sample_noalloc (no workspace: the library's own
        per-device scratch array); writes into the given or the runner's outputs."""
        placements = self.placements if placements is None else placements
        logp = self.logp if logp is None else logp
        check(lib.gdp_sample_noalloc(ctypes.byref(self.graph.c), self.logits.data_ptr(),
                                     self.lse.data_ptr() if use_lse else None, self.policy.cfg.n_devices,
                                     int(placements.shape[0]), seed,
                                     None if uniforms is None else uniforms.data_ptr(), placements.data_ptr(),
                                     logp.data_ptr(), _stream_handle(stream)))

    def place_sample(self, seed: int, uniforms=None, use_lse: bool = True, stream=None):
        """place() then sample() as one call (gdp_place_sample); with use_lse
        False the placer writes no lse and the sampling forms it."""
        check(lib.gdp_place_sample(ctypes.byref(self.graph.c), self.node_emb.data_ptr(), self.graph_emb.data_ptr(),
                                   ctypes.byref(self.policy.placer), self.logits.data_ptr(),
                                   self.lse.data_ptr() if use_lse else None, self.k, seed,
                                   None if uniforms is None else uniforms.data_ptr(), self.placements.data_ptr(),
                                   self.logp.data_ptr(), self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))

    def forward(self, seed: int, stream=None):
        """One pass of the hot path: embed -> place -> sample (the last two as one call)."""
        self.embed(stream)
        self.place_sample(seed, stream=stream)

    def ppo_grad(self, logp_old, advantages, clip_eps: float = 0.2, use_lse: bool = True, stream=None):
        """PPO's clipped surrogate per graph and its gradient with respect to the
        logits, for the placements and log-probs of the last sample() call."""
        torch = _torch()
        G, N, D = self.graph.n_graphs, self.graph.n_nodes, self.policy.cfg.n_devices
        loss = torch.empty((G,), dtype=torch.float32, device=self.ws.device)
        dlogits = torch.empty((N, D), dtype=torch.float32, device=self.ws.device)
        check(lib.gdp_ppo_grad(ctypes.byref(self.graph.c), self.logits.data_ptr(),
                               self.lse.data_ptr() if use_lse else None, D, self.k, self.placements.data_ptr(),
                               self.logp.data_ptr(), logp_old.data_ptr(), advantages.data_ptr(), float(clip_eps),
                               loss.data_ptr(), dlogits.data_ptr(), self.ws.data_ptr(), self.ws_bytes,
                               _stream_handle(stream)))
        return loss, dlogits

    def neighbors(self, stream=None):
        torch = _torch()
        n = self.graph.n_nodes
        cap = max(1, min(2 * self.graph.n_edges, n * self.policy.cfg.fanout))
        s_ptr = torch.empty(n + 1, dtype=torch.int32, device=self.ws.device)
        s_idx = torch.empty(cap, dtype=torch.int32, device=self.ws.device)
        check(lib.gdp_debug_neighbors(ctypes.byref(self.graph.c), ctypes.byref(self.policy.gnn), s_ptr.data_ptr(),
                                      s_idx.data_ptr(), cap, self.ws.data_ptr(), self.ws_bytes,
                                      _stream_handle(stream)))
        return s_ptr, s_idx


class Evaluator:
    """Simulated run time and validity of sampled placements (gdp_evaluate) for
    one graph batch: per-op costs in device memory, the workspace, the outputs."""

    def __init__(self, graph: DeviceGraph, n_devices: int, k_samples: int, costs, device="cuda"):
        torch = _torch()
        self.graph, self.D, self.k = graph, int(n_devices), int(k_samples)
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(device)
        self.op_cost, self.out_xfer, self.op_mem = up(costs.op_cost), up(costs.out_xfer), up(costs.op_mem)
        self.mem_cap = np.ascontiguousarray(costs.mem_cap, np.int64)
        self.ws_bytes = lib.gdp_evaluate_workspace_bytes(ctypes.byref(graph.c), self.D, self.k)
        if self.ws_bytes == 0:
            raise GdpError(GDP_E_INVALID_ARG, last_error())
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        G = graph.n_graphs
        self.makespan = torch.empty((G, self.k), dtype=torch.int64, device=device)
        self.valid = torch.empty((G, self.k), dtype=torch.uint8, device=device)
        self.run_time = torch.empty((G, self.k), dtype=torch.float32, device=device)

    def evaluate(self, placements, time_unit: float = 1e-6, stream=None):
        """placements [K, N] int32 (device); returns (makespan, valid, run_time)."""
        assert tuple(placements.shape) == (self.k, self.graph.n_nodes)
        check(lib.gdp_evaluate(ctypes.byref(self.graph.c), self.D, self.k, placements.data_ptr(),
                               self.op_cost.data_ptr(), self.out_xfer.data_ptr(), self.op_mem.data_ptr(),
                               self.mem_cap.ctypes.data_as(POINTER(c_int64)), float(time_unit),
                               self.makespan.data_ptr(), self.valid.data_ptr(), self.run_time.data_ptr(),
                               self.ws.data_ptr(), self.ws_bytes, _stream_handle(stream)))
        return self.makespan, self.valid, self.run_time


class Trainer:
    """The update step of a policy on one graph batch (Section 3, PPO): the
    training forward that keeps every intermediate in a store, the log-probs of
    given placements, the backward pass into fp32 gradients shaped like the
    weights, and Adam on fp32 master copies (the policy's own device weights,
    in its dtype, are rewritten after every step)."""

    def __init__(self, graph: DeviceGraph, policy: DevicePolicy, k_samples: int, device="cuda"):
        torch = _torch()
        self.graph, self.policy, self.k = graph, policy, int(k_samples)
        sb, wb = c_size_t(0), c_size_t(0)
        check(lib.gdp_train_sizes(ctypes.byref(graph.c), ctypes.byref(policy.gnn), ctypes.byref(policy.placer),
                                  ctypes.byref(sb), ctypes.byref(wb)))
        self.store_bytes, self.ws_bytes = sb.value, wb.value
        self.store = torch.empty(self.store_bytes, dtype=torch.uint8, device=device)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.sample_ws_bytes = lib.gdp_workspace_bytes(ctypes.byref(graph.c), None, None, self.k)
        self.sample_ws = torch.empty(max(1, self.sample_ws_bytes), dtype=torch.uint8, device=device)
        N, G, D = graph.n_nodes, graph.n_graphs, policy.cfg.n_devices
        self.logits = torch.empty((N, D), dtype=torch.float32, device=device)
        self.lse = torch.empty((N,), dtype=torch.float32, device=device)
        z = lambda t: torch.zeros(t.shape, dtype=torch.float32, device=device)
        self.grad_gnn = [{k: z(v) for k, v in l.items()} for l in policy.gnn_t]
        self.grad_placer = [{k: z(v) for k, v in l.items()} for l in policy.placer_t]
        self.grad_head = {k: z(v) for k, v in policy.head_t.items()}
        self._gg = (GdpGnnLayerGrad * len(self.grad_gnn))(
            *[GdpGnnLayerGrad(*[l[k].data_ptr() for k in ("w_pool", "b_pool", "w_self", "w_neigh", "b_upd")])
              for l in self.grad_gnn])
        self._gp = (GdpPlacerLayerGrad * len(self.grad_placer))(
            *[GdpPlacerLayerGrad(*[l[k].data_ptr() for k in PLACER_LAYER_FIELDS]) for l in self.grad_placer])
        self.grads = GdpGrads(self._gg, self._gp, self.grad_head["w_out"].data_ptr(),
                              self.grad_head["b_out"].data_ptr())
        # Adam: master copies and moments of every weight, in one list
        pairs = []
        for lw, lg in zip(policy.gnn_t, self.grad_gnn):
            pairs += [(lw[k], lg[k]) for k in lw]
        for lw, lg in zip(policy.placer_t, self.grad_placer):
            pairs += [(lw[k], lg[k]) for k in lw]
        pairs += [(policy.head_t[k], self.grad_head[k]) for k in policy.head_t]
        self._adam = []
        for prm, grd in pairs:
            master = prm.float().clone()
            self._adam.append((prm, master, grd, torch.zeros_like(master), torch.zeros_like(master)))
        self._adam_c = (GdpAdamTensor * len(self._adam))(
            *[GdpAdamTensor(prm.data_ptr(), ms.data_ptr(), grd.data_ptr(), m.data_ptr(), v.data_ptr(), prm.numel())
              for prm, ms, grd, m, v in self._adam])
        self.step_count = 0

    def forward(self, stream=None):
        """The training forward; returns (logits, lse) of the current weights."""
        check(lib.gdp_forward_train(ctypes.byref(self.graph.c), ctypes.byref(self.policy.gnn),
                                    ctypes.byref(self.policy.placer), self.store.data_ptr(), self.store_bytes,
                                    self.logits.data_ptr(), self.lse.data_ptr(), self.ws.data_ptr(), self.ws_bytes,
                                    _stream_handle(stream)))
        return self.logits, self.lse

    def log_prob(self, placements, stream=None):
        """log pi(placements) [G, K] under the last forward's logits."""
        torch = _torch()
        logp = torch.empty((self.graph.n_graphs, int(placements.shape[0])), dtype=torch.float32,
                           device=self.logits.device)
        check(lib.gdp_log_prob(ctypes.byref(self.graph.c), self.logits.data_ptr(), self.lse.data_ptr(),
                               self.policy.cfg.n_devices, int(placements.shape[0]), placements.data_ptr(),
                               logp.data_ptr(), self.sample_ws.data_ptr(), self.sample_ws_bytes,
                               _stream_handle(stream)))
        return logp

    def ppo_grad(self, placements, logp, logp_old, advantages, clip_eps=0.2, stream=None):
        """PPO's clipped surrogate and dL/dlogits at the last forward's logits."""
        torch = _torch()
        G, N, D = self.graph.n_graphs, self.graph.n_nodes, self.policy.cfg.n_devices
        K = int(placements.shape[0])
        loss = torch.empty((G,), dtype=torch.float32, device=self.logits.device)
        dlogits = torch.empty((N, D), dtype=torch.float32, device=self.logits.device)
        check(lib.gdp_ppo_grad(ctypes.byref(self.graph.c), self.logits.data_ptr(), self.lse.data_ptr(), D, K,
                               placements.data_ptr(), logp.data_ptr(), logp_old.data_ptr(), advantages.data_ptr(),
                               float(clip_eps), loss.data_ptr(), dlogits.data_ptr(), self.sample_ws.data_ptr(),
                               self.sample_ws_bytes, _stream_handle(stream)))
        return loss, dlogits

    def backward(self, dlogits, stream=None):
        """Gradients of sum(dlogits * logits) into grad_gnn / grad_placer / grad_head."""
        check(lib.gdp_backward(ctypes.byref(self.graph.c), ctypes.byref(self.policy.gnn),
                               ctypes.byref(self.policy.placer), self.store.data_ptr(), self.store_bytes,
                               dlogits.data_ptr(), ctypes.byref(self.grads), self.ws.data_ptr(), self.ws_bytes,
                               _stream_handle(stream)))

    def decisions(self, stream=None):
        """The last forward's discrete choices, for comparisons that take them the
        same way: {"gnn": [(winning neighbour [N, H], ReLU sign [N, H])] per GNN
        layer, "ffn": [ReLU sign [N, d_ff]] per placer layer} (numpy)."""
        torch = _torch()
        N, H, dff = self.graph.n_nodes, self.policy.cfg.hidden, self.policy.cfg.d_ff
        dev = self.store.device

        def get(which, layer, shape, dtype):
            out = torch.empty(shape, dtype=dtype, device=dev)
            check(lib.gdp_debug_train_tensor(ctypes.byref(self.graph.c), ctypes.byref(self.policy.gnn),
                                             ctypes.byref(self.policy.placer), self.store.data_ptr(), self.store_bytes,
                                             which, layer, out.data_ptr(), out.numel() * out.element_size(),
                                             _stream_handle(stream)))
            return out
        gnn = []
        for l in range(len(self.policy.gnn_t)):
            arg = get(2, l, (N, H), torch.int32).cpu().numpy()
            sign = (get(1, l, (N, H), torch.float32) > 0).cpu().numpy()
            gnn.append((arg, sign))
        ffn = [(get(0, l, (N, dff), torch.float32) > 0).cpu().numpy() for l in range(len(self.policy.placer_t))]
        return {"gnn": gnn, "ffn": ffn}

    def adam(self, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, stream=None):
        """One Adam step on every weight (master copies in fp32)."""
        self.step_count += 1
        dt = GDP_BF16 if self.graph.dtype == "bf16" else GDP_F32
        check(lib.gdp_adam_step(len(self._adam), self._adam_c, dt, float(lr), float(beta1), float(beta2), float(eps),
                                self.step_count, _stream_handle(stream)))


class RewardBaseline:
    """Section 4's reward and advantage with the running average of previous
    trials as the bias, one state per graph (device fp64 sums, int64 counts)."""

    def __init__(self, n_graphs: int, device="cuda"):
        torch = _torch()
        self.reward_sum = torch.zeros(n_graphs, dtype=torch.float64, device=device)
        self.trial_count = torch.zeros(n_graphs, dtype=torch.int64, device=device)

    def advantages(self, run_time, valid=None, stream=None):
        """run_time [G, K] fp32 (device), valid [G, K] uint8 or None; returns
        (reward, advantage), both [G, K] fp32, and advances the state."""
        torch = _torch()
        G, K = run_time.shape
        reward = torch.empty_like(run_time)
        adv = torch.empty_like(run_time)
        check(lib.gdp_advantages(G, K, run_time.data_ptr(), None if valid is None else valid.data_ptr(),
                                 self.reward_sum.data_ptr(), self.trial_count.data_ptr(), reward.data_ptr(),
                                 adv.data_ptr(), _stream_handle(stream)))
        return reward, adv


# ----------------------------------------------------------------------------
# Layer operators: the parts of a placement layer as calls of their own, forward
# and backward.  Tensors are float32 or bfloat16 matrices on one GPU whose last
# dimension is contiguous (any row stride); they run on that GPU's current
# stream, or on `stream`, where outputs and workspaces are allocated too.
# ----------------------------------------------------------------------------

_t = _torch()
_ACTS = {"none": 0, "relu": 1}
_DTYPES = {_t.float32: GDP_F32, _t.bfloat16: GDP_BF16}
# the current stream's handle without a Stream object around it (2.6 us a call less)
_raw_stream = getattr(_t._C, "_cuda_getCurrentRawStream", None) or (lambda d: _t.cuda.current_stream(d).cuda_stream)


def _bad(msg: str):
    raise GdpError(GDP_E_INVALID_ARG, msg)


def _placed(x, stream, call):
    """call(the stream's handle) with x's GPU as the current one and `stream`, if given, as its current stream."""
    d = x.get_device()
    if stream is None and (d < 0 or d == _t.cuda.current_device()):
        return call(_raw_stream(d) if d >= 0 else 0)
    with _t.cuda.device(d), _t.cuda.stream(stream):
        return call(_raw_stream(d))


def _dtype_of(name, t) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        _bad(f"{name} is {t.dtype}, not float32 or bfloat16")
    return dt


def _need(name, t, like, shape, dtype=None):
    """t has this shape, like's device, like's dtype (or the given one) and a contiguous last dimension."""
    dtype = dtype or like.dtype
    d = like.get_device()
    if t.shape == shape and t.dtype is dtype and t.get_device() == d >= 0 and t.is_contiguous():
        return
    if t.get_device() != d or d < 0:
        _bad(f"{name} is on {t.device}, not on {like.device}" if t.device != like.device else f"{name} is not on a GPU")
    if t.dtype is not dtype:
        _bad(f"{name} is {t.dtype}, not {dtype}")
    if t.shape != shape:
        _bad(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _bad(f"{name}'s last dimension is not contiguous")
    if len(shape) == 2 and shape[0] > 1 and t.stride(0) < shape[1]:
        _bad(f"{name}'s rows overlap")


def _matrix(name, t):
    if t.dim() != 2:
        _bad(f"{name} is not a matrix")
    return t.shape


def _ld(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _dense(name, t):
    if not t.is_contiguous():
        _bad(f"{name} is not contiguous")


def _ptr(t):
    return None if t is None else t.data_ptr()


def layer_norm(x, gamma, beta, residual=None, eps: float = 1e-5, keep_sum: bool = False, stream=None):
    """LayerNorm of x (+ residual), [rows, width]; with keep_sum (y, sum), the sum being layer_norm_backward's h."""
    dt = _dtype_of("x", x)
    rows, width = shape = _matrix("x", x)
    _need("x", x, x, shape)
    _need("gamma", gamma, x, (width,))
    _need("beta", beta, x, (width,))
    if residual is not None:
        _need("residual", residual, x, shape)

    def call(st):
        y = _t.empty(shape, dtype=x.dtype, device=x.device)
        s = _t.empty_like(y) if keep_sum else None
        check(lib.gdp_layer_norm(rows, width, dt, x.data_ptr(), _ld(x), _ptr(residual),
                                 0 if residual is None else _ld(residual), gamma.data_ptr(), beta.data_ptr(), eps,
                                 y.data_ptr(), width, _ptr(s), width, st))
        return (y, s) if keep_sum else y
    return _placed(x, stream, call)


def layer_norm_backward(h, gamma, dy, dsum=None, eps: float = 1e-5, stream=None):
    """The gradients of layer_norm at h (x, or the sum it kept): (dh, dgamma, dbeta), the last two fp32.  dsum: the
    gradient that reaches h past the LayerNorm, added to dh (the gradient of x and of residual)."""
    dt = _dtype_of("h", h)
    rows, width = shape = _matrix("h", h)
    _need("h", h, h, shape)
    _need("gamma", gamma, h, (width,))
    _need("dy", dy, h, shape)
    if dsum is not None:
        _need("dsum", dsum, h, shape)

    def call(st):
        dh = _t.empty(shape, dtype=h.dtype, device=h.device)
        dg = _t.empty(width, dtype=_t.float32, device=h.device)
        db = _t.empty_like(dg)
        need = lib.gdp_layer_norm_workspace_bytes(rows, width)
        if need == 0:
            raise GdpError(GDP_E_INVALID_ARG, last_error())
        ws = _t.empty(need, dtype=_t.uint8, device=h.device)
        check(lib.gdp_layer_norm_backward(rows, width, dt, h.data_ptr(), _ld(h), gamma.data_ptr(), eps, dy.data_ptr(),
                                          _ld(dy), _ptr(dsum), 0 if dsum is None else _ld(dsum), dh.data_ptr(), width,
                                          dg.data_ptr(), db.data_ptr(), ws.data_ptr(), need, st))
        return dh, dg, db
    return _placed(h, stream, call)


def _fc_shapes(x, w, act):
    dt = _dtype_of("x", x)
    if act not in _ACTS:
        _bad(f"act {act!r} is not one of {sorted(_ACTS)}")
    rows, k = _matrix("x", x)
    n = _matrix("w", w)[0]
    _need("x", x, x, (rows, k))
    _need("w", w, x, (n, k))
    _dense("w", w)
    return dt, rows, k, n


def fc(x, w, b=None, act: str = "none", residual=None, keep_act: bool = False, stream=None):
    """act(x w^T + b) + residual for x [rows, K], w [N, K], act "none" or "relu"; with keep_act (y, a), a the
    activation's output before the residual, for fc_backward (without residual that is y)."""
    dt, rows, k, n = _fc_shapes(x, w, act)
    if b is not None:
        _need("b", b, x, (n,))
    if residual is not None:
        _need("residual", residual, x, (rows, n))

    def call(st):
        y = _t.empty((rows, n), dtype=x.dtype, device=x.device)
        a = _t.empty_like(y) if keep_act else None
        f = GdpFcLayer(rows, k, n, dt, _ACTS[act], _ld(x), n, 0 if residual is None else _ld(residual), n)
        check(lib.gdp_fc(ctypes.byref(f), x.data_ptr(), w.data_ptr(), _ptr(b), _ptr(residual), y.data_ptr(), _ptr(a), st))
        return (y, a) if keep_act else y
    return _placed(x, stream, call)


def fc_backward(dy, x, w, act: str = "none", act_out=None, dx_add=None, need_dx: bool = True, stream=None):
    """The gradients of fc: (dx or None, dw, db), the last two fp32; act_out: the activation's output (with "relu");
    dx_add: what reaches x on another path, added to dx.  The residual's gradient is dy itself."""
    dt, rows, k, n = _fc_shapes(x, w, act)
    _need("dy", dy, x, (rows, n))
    if act == "relu":
        if act_out is None:
            _bad("act_out is needed with relu")
        _need("act_out", act_out, x, (rows, n))
    else:
        act_out = None
    if dx_add is not None:
        _need("dx_add", dx_add, x, (rows, k))

    def call(st):
        dx = _t.empty((rows, k), dtype=x.dtype, device=x.device) if need_dx else None
        dw = _t.empty((n, k), dtype=_t.float32, device=x.device)
        db = _t.empty(n, dtype=_t.float32, device=x.device)
        f = GdpFcLayer(rows, k, n, dt, _ACTS[act], _ld(x), 0, 0, 0 if act_out is None else _ld(act_out), _ld(dy), k,
                       0 if dx_add is None else _ld(dx_add))
        need = lib.gdp_fc_workspace_bytes(ctypes.byref(f))
        if need == 0:
            raise GdpError(GDP_E_INVALID_ARG, last_error())
        ws = _t.empty(need, dtype=_t.uint8, device=x.device)
        check(lib.gdp_fc_backward(ctypes.byref(f), dy.data_ptr(), x.data_ptr(), w.data_ptr(), _ptr(act_out),
                                  _ptr(dx_add), _ptr(dx), dw.data_ptr(), db.data_ptr(), ws.data_ptr(), need, st))
        return dx, dw, db
    return _placed(x, stream, call)


def rel_bounds(n_buckets: int, reach: int):
    """Bucket bounds for n_buckets buckets of a distance: one bucket a distance up to half of them, the rest
    spread evenly over the logarithm up to `reach`, from where on the last bucket holds everything."""
    n = int(n_buckets) - 1
    if n < 0:
        _bad(f"n_buckets = {n_buckets} < 1")
    near = min(n, max(1, int(n_buckets) // 2))
    out = list(range(1, near + 1))
    for i in range(n - near):
        out.append(max(out[-1] + 1, int(round(near * (reach / near) ** ((i + 1) / (n - near))))))
    return out


class RelAttention:
    """Segment attention with a learned relative position bias by buckets (gdp_rel_attention) over a batch of
    graphs.  Graph g has lengths[g] positions, whose keys and values are rows from starts[g] on (default: one graph
    after another); queries: how many of each graph's last positions are queries (default: all; 1 for one op
    appended to a graph whose keys and values are kept).  bounds: ascending distances at which a bucket begins.
    The plan holds host data only: calls may run at once, on any stream or GPU."""

    def __init__(self, lengths, heads: int, d_head: int, bounds, kv_heads: Optional[int] = None,
                 seg_len: Optional[int] = None, mem_len: int = 0, causal: bool = False, queries=None, starts=None,
                 scale: Optional[float] = None):
        i32 = lambda a: np.array(list(a), np.int32)
        self.lengths = i32(lengths)
        self.starts = i32(np.cumsum(self.lengths) - self.lengths) if starts is None else i32(starts)
        self.queries = None if queries is None else i32(queries)
        self.bounds = i32(bounds)
        G = self.lengths.size
        if self.starts.size != G or (self.queries is not None and self.queries.size != G):
            _bad("lengths, starts and queries differ in length")
        self.heads, self.d_head = int(heads), int(d_head)
        self.kv_heads = self.heads if kv_heads is None else int(kv_heads)
        self.n_queries = int((self.lengths if self.queries is None else self.queries).sum())
        self.n_buckets = (self.bounds.size + 1) * (1 if causal else 2)
        # rows that k and v need; whether the graphs' rows cover all of them
        self.n_rows = int((self.starts + self.lengths)[self.lengths > 0].max(initial=0))
        self.n_keys = int(self.lengths.sum())
        seg = max(1, int(self.lengths.max(initial=1))) if seg_len is None else int(seg_len)
        ptr = lambda a: None if a is None else a.ctypes.data_as(POINTER(c_int32))
        self._c = GdpRelAttn(G, ptr(self.starts), ptr(self.lengths), ptr(self.queries), self.heads, self.kv_heads,
                             self.d_head, seg, int(mem_len), 1 if causal else 0, self.bounds.size, ptr(self.bounds),
                             GDP_F32, self.d_head ** -0.5 if scale is None else float(scale))
        wq, wk = self.heads * self.d_head, self.kv_heads * self.d_head
        self._widths = (wq, wk)
        for n, w in (("ld_q", wq), ("ld_k", wk), ("ld_v", wk), ("ld_o", wq), ("ld_do", wq), ("ld_dq", wq),
                     ("ld_dk", wk), ("ld_dv", wk)):
            setattr(self._c, n, w)
        self._ws = lib.gdp_rel_attention_workspace_bytes(ctypes.byref(self._c), 0)   # the same for both types
        if self._ws == 0:
            raise GdpError(GDP_E_INVALID_ARG, last_error())

    def _call(self, q, k, v, table, key_mask):
        """The arrays checked; a descriptor of this call's own."""
        wq, wk = self._widths
        dt = _dtype_of("q", q)
        rows = k.shape[0] if k.dim() == 2 else 0
        if rows < self.n_rows:
            _bad(f"k has shape {tuple(k.shape)}, not at least {self.n_rows} rows of {wk}")
        _need("q", q, q, (self.n_queries, wq))
        _need("k", k, q, (rows, wk))
        _need("v", v, q, (rows, wk))
        _need("table", table, q, (self.heads, self.n_buckets))
        _dense("table", table)
        if key_mask is not None:
            _need("key_mask", key_mask, q, (rows,), _t.uint8)
        c = GdpRelAttn.from_buffer_copy(self._c)
        c.dtype, c.ld_q, c.ld_k, c.ld_v = dt, _ld(q), _ld(k), _ld(v)
        return c

    def forward(self, q, k, v, table, key_mask=None, stream=None):
        """q [queries, heads * d_head]; k, v [rows, kv_heads * d_head]; table [heads, buckets]; key_mask [rows]
        uint8.  Returns (o like q, lse [queries, heads] fp32 in base 2, for backward)."""
        c = self._call(q, k, v, table, key_mask)

        def call(st):
            o = _t.empty((self.n_queries, self._widths[0]), dtype=q.dtype, device=q.device)
            lse = _t.empty((self.n_queries, self.heads), dtype=_t.float32, device=q.device)
            ws = _t.empty(self._ws, dtype=_t.uint8, device=q.device)
            check(lib.gdp_rel_attention(ctypes.byref(c), q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(),
                                        _ptr(key_mask), o.data_ptr(), lse.data_ptr(), ws.data_ptr(), self._ws, st))
            return o, lse
        return _placed(q, stream, call)

    def backward(self, dout, q, k, v, table, o, lse, key_mask=None, out=None, stream=None):
        """(dq, dk, dv, dtable) for dL/do, from the forward's inputs and results; dtable is fp32, rows of k and v
        that belong to no graph get zeros.  out: the arrays for dq, dk and dv (e.g. columns of one matrix), whose
        rows of no graph are left as they are."""
        c = self._call(q, k, v, table, key_mask)
        wq, wk = self._widths
        _need("dout", dout, q, (self.n_queries, wq))
        _need("o", o, q, (self.n_queries, wq))
        _need("lse", lse, q, (self.n_queries, self.heads), _t.float32)
        _dense("lse", lse)
        if out is not None:
            for n, t, like in zip(("dq", "dk", "dv"), out, (q, k, v)):
                _need(n, t, q, like.shape)
        c.ld_do, c.ld_o = _ld(dout), _ld(o)

        def call(st):
            if out is None:
                make = _t.empty if self.n_keys == k.shape[0] else _t.zeros
                dq = _t.empty((self.n_queries, wq), dtype=q.dtype, device=q.device)
                dk, dv = (make((k.shape[0], wk), dtype=q.dtype, device=q.device) for _ in range(2))
            else:
                dq, dk, dv = out
                c.ld_dq, c.ld_dk, c.ld_dv = _ld(dq), _ld(dk), _ld(dv)
            dtable = _t.empty((self.heads, self.n_buckets), dtype=_t.float32, device=q.device)
            need = lib.gdp_rel_attention_workspace_bytes(ctypes.byref(c), 1)
            if need == 0:
                raise GdpError(GDP_E_INVALID_ARG, last_error())
            ws = _t.empty(need, dtype=_t.uint8, device=q.device)
            check(lib.gdp_rel_attention_backward(ctypes.byref(c), dout.data_ptr(), q.data_ptr(), k.data_ptr(),
                                                 v.data_ptr(), table.data_ptr(), _ptr(key_mask), o.data_ptr(),
                                                 lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                                 dtable.data_ptr(), ws.data_ptr(), need, st))
            return dq, dk, dv, dtable
        return _placed(q, stream, call)


def debug_uniforms(seed: int, n: int, k: int, d: int, device="cuda", stream=None):
    torch = _torch()
    out = torch.empty((k, n, d), dtype=torch.float32, device=device)
    check(lib.gdp_debug_uniforms(seed, n, k, d, out.data_ptr(), _stream_handle(stream)))
    return out


def set_place_streams(n: int) -> None:
    """gdp_place's stream schedule for this thread: 2 (the default) splits a
    large placer pass into two row parts on two streams, 1 keeps every launch
    on the caller's stream.  The results are the same bit for bit."""
    check(lib.gdp_set_place_streams(int(n)))


def timer_begin(kinds) -> None:
    mask = 0
    for k in kinds:
        mask |= 1 << (KERNEL_KINDS.index(k) if isinstance(k, str) else int(k))
    check(lib.gdp_timer_begin(mask))


def timer_end() -> Dict[str, Dict[str, float]]:
    ms = (c_double * K_COUNT)()
    cnt = (c_int64 * K_COUNT)()
    check(lib.gdp_timer_end(ms, cnt))
    return {KERNEL_KINDS[i]: {"ms": ms[i], "launches": int(cnt[i])} for i in range(K_COUNT) if cnt[i]}
