"""ctypes binding of libace (include/ace.h).

Argument marshalling only: torch supplies device memory and the current HIP
stream; every step of the computation runs in the library's HIP kernels.
Importing this module loads libace.so and raises if it is missing -- there is
no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libace.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libace.so not found at {LIB_PATH}; build it with "
                      "`python -m paper_2609_06072_amd.build`")
_lib = ctypes.CDLL(LIB_PATH)

ACE_OK, ACE_ERR_INVALID_ARG, ACE_ERR_UNSUPPORTED, ACE_ERR_WORKSPACE, ACE_ERR_HIP = 0, -1, -2, -3, -4
ACE_F32, ACE_BF16 = 0, 1
ACE_ROWS_GROUP_DEDUP, ACE_ROWS_GROUP_PAIRS, ACE_ROWS_EXPERT = 0, 1, 2
ACE_INPUT_SHARED, ACE_INPUT_PER_PAIR, ACE_INPUT_COMBINED = 0, 1, 2
ACE_OP_PERMUTE, ACE_OP_FWD, ACE_OP_BWD, ACE_OP_CKA, ACE_OP_MOE_DX = 0, 1, 2, 3, 4

EXPORTS = ("ace_group_permute", "ace_group_expert_permute", "ace_grouped_lora_fwd", "ace_grouped_lora_bwd",
           "ace_expertwise_lora_fwd", "ace_expertwise_lora_bwd", "ace_workspace_bytes",
           "ace_routing_check", "ace_last_error", "ace_pairwise_cka", "ace_similarity_graph",
           "ace_louvain", "ace_group_anchors", "ace_consolidate_adapters", "ace_moe_lora_fwd",
           "ace_group_permute_noalloc", "ace_moe_dx", "ace_moe_combine_fwd", "ace_moe_combine_bwd",
           "ace_act_pack", "ace_act_unpack", "ace_swiglu_fwd", "ace_swiglu_bwd")
ACE_PERMUTE_SCRATCH_BYTES = 4 << 20


class AceRouting(ctypes.Structure):
    _fields_ = [("counts", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("row_token", ctypes.c_void_p), ("row_slots", ctypes.c_void_p),
                ("pair_row", ctypes.c_void_p), ("n_dropped", ctypes.c_void_p),
                ("row_pair", ctypes.c_void_p), ("pair_list", ctypes.c_void_p),
                ("n_keys", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("T", ctypes.c_int32), ("k", ctypes.c_int32)]


class AcePackedAct(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("exps", ctypes.c_void_p)]


_i32, _f32, _vp, _sz = ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
_R = ctypes.POINTER(AceRouting)
_lib.ace_group_permute.argtypes = [_vp, _i32, _i32, _i32, _vp, _i32, _i32, _R, _vp, _sz, _vp]
_lib.ace_group_permute.restype = _i32
_lib.ace_group_permute_noalloc.argtypes = [_vp, _i32, _i32, _i32, _vp, _i32, _i32, _R, _vp]
_lib.ace_group_permute_noalloc.restype = _i32
_lib.ace_group_expert_permute.argtypes = [_vp, _i32, _i32, _i32, _vp, _i32, _i32, _R, _R, _vp, _sz,
                                          _vp]
_lib.ace_group_expert_permute.restype = _i32
_FWD = [_i32, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _f32, _vp, _vp, _vp, _vp, _R, _vp, _vp, _sz, _vp]
_BWD = [_i32, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _f32, _vp, _vp, _vp, _vp, _R, _vp, _vp, _vp,
        _vp, _vp, _vp, _sz, _vp]
_lib.ace_grouped_lora_fwd.argtypes = _FWD
_lib.ace_grouped_lora_fwd.restype = _i32
_lib.ace_grouped_lora_bwd.argtypes = _BWD
_lib.ace_grouped_lora_bwd.restype = _i32
_EFWD = list(_FWD)
_EFWD[7] = _i32          # rank instead of group_rank pointer
_EBWD = list(_BWD)
_EBWD[7] = _i32
_lib.ace_expertwise_lora_fwd.argtypes = _EFWD
_lib.ace_expertwise_lora_fwd.restype = _i32
_lib.ace_expertwise_lora_bwd.argtypes = _EBWD
_lib.ace_expertwise_lora_bwd.restype = _i32
_lib.ace_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32, _i32, _i32]
_lib.ace_workspace_bytes.restype = _sz
_lib.ace_routing_check.argtypes = [_R, ctypes.POINTER(ctypes.c_int32), _vp]
_lib.ace_routing_check.restype = _i32
_lib.ace_pairwise_cka.argtypes = [_i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _sz,
                                  _vp]
_lib.ace_pairwise_cka.restype = _i32
_lib.ace_similarity_graph.argtypes = [_vp, _i32, _vp]
_lib.ace_similarity_graph.restype = _i32
_lib.ace_louvain.argtypes = [_vp, _i32, ctypes.c_double, _vp, ctypes.POINTER(ctypes.c_int32)]
_lib.ace_louvain.restype = _i32
_lib.ace_group_anchors.argtypes = [_vp, _i32, _vp, _i32, _vp]
_lib.ace_group_anchors.restype = _i32
_lib.ace_consolidate_adapters.argtypes = [_i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _i32, _vp,
                                          _vp, _vp, _vp, _vp, _vp]
_lib.ace_consolidate_adapters.restype = _i32
_lib.ace_moe_lora_fwd.argtypes = [_i32, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _R, _i32, _vp,
                                  _vp, _f32, _vp, _vp, _R, _vp, _vp, _sz, _vp]
_lib.ace_moe_lora_fwd.restype = _i32
_i64, _K = ctypes.c_int64, ctypes.POINTER(AcePackedAct)
_lib.ace_moe_dx.argtypes = [_i32, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _R, _i32, _vp, _vp,
                            _sz, _vp]
_lib.ace_moe_dx.restype = _i32
_lib.ace_moe_combine_fwd.argtypes = [_i32, _i32, _i32, _i32, _vp, _vp, _R, _vp, _vp]
_lib.ace_moe_combine_fwd.restype = _i32
_lib.ace_moe_combine_bwd.argtypes = [_i32, _i32, _i32, _i32, _vp, _vp, _vp, _R, _vp, _vp, _vp]
_lib.ace_moe_combine_bwd.restype = _i32
_lib.ace_act_pack.argtypes = [_i32, _i64, _i32, _vp, _K, _vp]
_lib.ace_act_pack.restype = _i32
_lib.ace_act_unpack.argtypes = [_i32, _i64, _i32, _K, _vp, _vp]
_lib.ace_act_unpack.restype = _i32
_lib.ace_swiglu_fwd.argtypes = [_i32, _i64, _i32, _vp, _vp, _vp, _K, _K, _vp]
_lib.ace_swiglu_fwd.restype = _i32
_lib.ace_swiglu_bwd.argtypes = [_i32, _i64, _i32, _vp, _vp, _vp, _K, _K, _vp, _vp, _vp]
_lib.ace_swiglu_bwd.restype = _i32
_lib.ace_last_error.argtypes = []
_lib.ace_last_error.restype = ctypes.c_char_p


class AceError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where} failed with status {status}: {ace_last_error()}")


def ace_last_error() -> str:
    return _lib.ace_last_error().decode()


def _check(status: int, where: str) -> None:
    if status != ACE_OK:
        raise AceError(status, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libace must be contiguous")
    return t.data_ptr() or None


# the current stream's handle without building a Stream object (2.8 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device()) or None
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return ACE_BF16
    if t.dtype == torch.float32:
        return ACE_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _want(name: str, t, numel: Optional[int] = None, dtype=None, device=None,
          optional: bool = False) -> None:
    """Host-side shape/type check of one argument before the call (the
    library sees only pointers): numel, dtype and device must match."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


def _check_lora_args(x, A, B, R: int, n_keys: int, routing: "Routing", d_out: int,
                     input_mode: int, pair_w, y=None, dy=None, dx=None, dA=None, dB=None) -> None:
    """R: total rank of the call's n_keys adapters."""
    T, k = routing.c.T, routing.c.k
    dt, dev = A.dtype, A.device
    if A.dim() != 2 or A.shape[0] != R:
        raise ValueError(f"A must be [R={R}, d_in], got {tuple(A.shape)}")
    d_in = A.shape[1]
    rows_in = T if input_mode == ACE_INPUT_SHARED else T * k
    rows_out = T if input_mode == ACE_INPUT_COMBINED else T * k
    _want("x", x, rows_in * d_in, dt, dev)
    _want("B", B, R * d_out, dt, dev)
    _want("pair_w", pair_w, T * k, torch.float32, dev, optional=True)
    if y is not None:
        _want("y", y, rows_out * d_out, dt, dev)
    if dy is not None:
        _want("dy", dy, rows_out * d_out, dt, dev)
        _want("dx", dx, rows_in * d_in, dt, dev)
        _want("dA", dA, R * d_in, torch.float32, dev)
        _want("dB", dB, R * d_out, torch.float32, dev)
    if routing.n_keys != n_keys:
        raise ValueError(f"routing has {routing.n_keys} keys, the call has {n_keys}")


def ace_workspace_bytes(op: int, T: int, k: int, d_in: int, d_out: int, n_keys: int,
                        r_max: int) -> int:
    n = _lib.ace_workspace_bytes(op, T, k, d_in, d_out, n_keys, r_max)
    if n == ctypes.c_size_t(-1).value:
        raise AceError(ACE_ERR_INVALID_ARG, "ace_workspace_bytes")
    return int(n)


class Routing:
    """Owns the device arrays of an ace_routing (sized for T*k pairs)."""

    def __init__(self, T: int, k: int, n_keys: int, device="cuda"):
        P = max(1, T * k)
        i32 = dict(dtype=torch.int32, device=device)
        self.counts = torch.zeros(n_keys, **i32)
        self.offsets = torch.zeros(n_keys + 1, **i32)
        self.row_token = torch.zeros(P, **i32)
        self.row_slots = torch.zeros(P, **i32)
        self.pair_row = torch.zeros(P, **i32)
        self.n_dropped = torch.zeros(1, **i32)
        self.row_pair = torch.zeros(P + 1, **i32)
        self.pair_list = torch.zeros(P, **i32)
        self.c = AceRouting(self.counts.data_ptr(), self.offsets.data_ptr(),
                            self.row_token.data_ptr(), self.row_slots.data_ptr(),
                            self.pair_row.data_ptr(), self.n_dropped.data_ptr(),
                            self.row_pair.data_ptr(), self.pair_list.data_ptr(), n_keys, -1, T, k)

    def check_capacity(self, T: int, k: int, n_keys: int) -> None:
        """The arrays must hold a permutation of T*k pairs over n_keys keys."""
        P = max(1, T * k)
        if self.row_token.numel() < P or self.row_pair.numel() < P + 1:
            raise ValueError(f"routing holds {self.row_token.numel()} pairs, the call needs {P}")
        if self.counts.numel() != n_keys:
            raise ValueError(f"routing has room for {self.counts.numel()} keys, the call has {n_keys}")

    @property
    def n_keys(self) -> int:
        return self.c.n_keys

    @property
    def mode(self) -> int:
        return self.c.mode


def ace_group_permute(topk_ids: torch.Tensor, E: int, expert_to_group: Optional[torch.Tensor],
                      G: int, mode: int, routing: Optional[Routing] = None,
                      ws: Optional[torch.Tensor] = None, stream=None) -> Routing:
    T, k = topk_ids.shape
    n_keys = E if mode == ACE_ROWS_EXPERT else G
    _want("topk_ids", topk_ids, dtype=torch.int32)
    _want("expert_to_group", expert_to_group, E, torch.int32, topk_ids.device, optional=True)
    if routing is None:
        routing = Routing(T, k, n_keys, device=topk_ids.device)
    routing.check_capacity(T, k, n_keys)
    need = ace_workspace_bytes(ACE_OP_PERMUTE, T, k, 0, 0, n_keys, 0)
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=topk_ids.device)
    _check(_lib.ace_group_permute(_ptr(topk_ids), T, k, E, _ptr(expert_to_group), G, mode,
                                  ctypes.byref(routing.c), _ptr(ws), ws.numel(), _stream(stream)),
           "ace_group_permute")
    return routing


def ace_group_permute_noalloc(topk_ids: torch.Tensor, E: int,
                              expert_to_group: Optional[torch.Tensor], G: int, mode: int,
                              routing: Routing, stream=None) -> Routing:
    """ace_group_permute with the library's static scratch instead of a
    workspace: allocates nothing (the caller passes the routing arrays)."""
    T, k = topk_ids.shape
    n_keys = E if mode == ACE_ROWS_EXPERT else G
    _want("topk_ids", topk_ids, dtype=torch.int32)
    _want("expert_to_group", expert_to_group, E, torch.int32, topk_ids.device, optional=True)
    routing.check_capacity(T, k, n_keys)
    _check(_lib.ace_group_permute_noalloc(_ptr(topk_ids), T, k, E, _ptr(expert_to_group), G,
                                          mode, ctypes.byref(routing.c), _stream(stream)),
           "ace_group_permute_noalloc")
    return routing


def ace_group_expert_permute(topk_ids: torch.Tensor, E: int, expert_to_group: torch.Tensor,
                             G: int, group_mode: int = ACE_ROWS_GROUP_DEDUP,
                             group_routing: Optional[Routing] = None,
                             expert_routing: Optional[Routing] = None,
                             ws: Optional[torch.Tensor] = None, stream=None):
    """Group-keyed and expert-keyed routings from one pass over topk_ids."""
    T, k = topk_ids.shape
    _want("topk_ids", topk_ids, dtype=torch.int32)
    _want("expert_to_group", expert_to_group, E, torch.int32, topk_ids.device)
    if group_routing is None:
        group_routing = Routing(T, k, G, device=topk_ids.device)
    if expert_routing is None:
        expert_routing = Routing(T, k, E, device=topk_ids.device)
    group_routing.check_capacity(T, k, G)
    expert_routing.check_capacity(T, k, E)
    need = (ace_workspace_bytes(ACE_OP_PERMUTE, T, k, 0, 0, G, 0)
            + ace_workspace_bytes(ACE_OP_PERMUTE, T, k, 0, 0, E, 0))
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=topk_ids.device)
    _check(_lib.ace_group_expert_permute(_ptr(topk_ids), T, k, E, _ptr(expert_to_group), G,
                                         group_mode, ctypes.byref(group_routing.c),
                                         ctypes.byref(expert_routing.c), _ptr(ws), ws.numel(),
                                         _stream(stream)),
           "ace_group_expert_permute")
    return group_routing, expert_routing


def ace_routing_check(routing: Routing, stream=None) -> int:
    n = ctypes.c_int32(0)
    _check(_lib.ace_routing_check(ctypes.byref(routing.c), ctypes.byref(n), _stream(stream)),
           "ace_routing_check")
    return int(n.value)


@functools.lru_cache(maxsize=256)
def _rank_table(ranks: tuple):
    """(C array, total, largest) of a rank list, kept by value: a layer passes
    the same few lists on every call, and the library only reads them."""
    return (ctypes.c_int32 * len(ranks))(*ranks), sum(ranks), max(ranks, default=0)


def _fwd_ws(ws, T, k, d_in, d_out, n_keys, r_max, device):
    if ws is not None:
        return ws
    need = ace_workspace_bytes(ACE_OP_FWD, T, k, d_in, d_out, n_keys, r_max)
    return torch.empty(max(need, 256), dtype=torch.uint8, device=device)


def ace_grouped_lora_fwd(x, A, B, group_rank: Sequence[int], alpha: float, routing: Routing,
                         y, pair_w=None, input_mode: int = ACE_INPUT_SHARED, ws=None,
                         stream=None) -> None:
    T, k = routing.c.T, routing.c.k
    d_in, d_out = A.shape[1], y.shape[1]
    ranks, R, r_max = _rank_table(tuple(map(int, group_rank)))
    _check_lora_args(x, A, B, R, len(group_rank), routing, d_out, input_mode, pair_w, y=y)
    ws = _fwd_ws(ws, T, k, d_in, d_out, len(group_rank), r_max, A.device)
    _check(_lib.ace_grouped_lora_fwd(_dtype(x), input_mode, T, k, d_in, d_out, len(group_rank),
                                     ranks, alpha, _ptr(x), _ptr(A), _ptr(B), _ptr(pair_w),
                                     ctypes.byref(routing.c), _ptr(y), _ptr(ws),
                                     0 if ws is None else ws.numel(), _stream(stream)),
           "ace_grouped_lora_fwd")


def ace_grouped_lora_bwd(x, A, B, group_rank: Sequence[int], alpha: float, routing: Routing,
                         dy, dx, dA, dB, pair_w=None, input_mode: int = ACE_INPUT_SHARED,
                         ws=None, stream=None, h_fwd=None) -> None:
    """h_fwd: None, or the workspace of the forward call with the same arguments
    (the backward then reuses the forward's h instead of recomputing it)."""
    T, k = routing.c.T, routing.c.k
    d_in, d_out = A.shape[1], dy.shape[1]
    ranks, R, r_max = _rank_table(tuple(map(int, group_rank)))
    _check_lora_args(x, A, B, R, len(group_rank), routing, d_out, input_mode, pair_w, dy=dy, dx=dx,
                     dA=dA, dB=dB)
    if ws is None:
        need = ace_workspace_bytes(ACE_OP_BWD, T, k, d_in, d_out, len(group_rank), r_max)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=A.device)
    _check(_lib.ace_grouped_lora_bwd(_dtype(A), input_mode, T, k, d_in, d_out, len(group_rank),
                                     ranks, alpha, _ptr(x), _ptr(A), _ptr(B), _ptr(pair_w),
                                     ctypes.byref(routing.c), _ptr(h_fwd), _ptr(dy), _ptr(dx),
                                     _ptr(dA), _ptr(dB), _ptr(ws), ws.numel(), _stream(stream)),
           "ace_grouped_lora_bwd")


def ace_expertwise_lora_fwd(x, A, B, E: int, rank: int, alpha: float, routing: Routing, y,
                            pair_w=None, input_mode: int = ACE_INPUT_SHARED, ws=None,
                            stream=None) -> None:
    T, k = routing.c.T, routing.c.k
    d_in, d_out = A.shape[1], y.shape[1]
    _check_lora_args(x, A, B, int(rank) * E, E, routing, d_out, input_mode, pair_w, y=y)
    ws = _fwd_ws(ws, T, k, d_in, d_out, E, rank, A.device)
    _check(_lib.ace_expertwise_lora_fwd(_dtype(x), input_mode, T, k, d_in, d_out, E, rank, alpha,
                                        _ptr(x), _ptr(A), _ptr(B), _ptr(pair_w),
                                        ctypes.byref(routing.c), _ptr(y), _ptr(ws),
                                        0 if ws is None else ws.numel(), _stream(stream)),
           "ace_expertwise_lora_fwd")


def ace_expertwise_lora_bwd(x, A, B, E: int, rank: int, alpha: float, routing: Routing, dy, dx,
                            dA, dB, pair_w=None, input_mode: int = ACE_INPUT_SHARED, ws=None,
                            stream=None, h_fwd=None) -> None:
    T, k = routing.c.T, routing.c.k
    d_in, d_out = A.shape[1], dy.shape[1]
    _check_lora_args(x, A, B, int(rank) * E, E, routing, d_out, input_mode, pair_w, dy=dy, dx=dx,
                     dA=dA, dB=dB)
    if ws is None:
        need = ace_workspace_bytes(ACE_OP_BWD, T, k, d_in, d_out, E, rank)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=A.device)
    _check(_lib.ace_expertwise_lora_bwd(_dtype(A), input_mode, T, k, d_in, d_out, E, rank, alpha,
                                        _ptr(x), _ptr(A), _ptr(B), _ptr(pair_w),
                                        ctypes.byref(routing.c), _ptr(h_fwd), _ptr(dy), _ptr(dx),
                                        _ptr(dA), _ptr(dB), _ptr(ws), ws.numel(),
                                        _stream(stream)),
           "ace_expertwise_lora_bwd")


def ace_pairwise_cka(X, A, B, E: int, rank: int, S=None, ws=None, stream=None) -> torch.Tensor:
    """Pairwise linear CKA [E, E] (fp32) of the expert adapters A, B (packed,
    E keys of rank `rank`) on the probe rows X [N, d_in]."""
    N, d_in = X.shape
    d_out = B.numel() // (E * rank)
    if S is None:
        S = torch.empty(E, E, dtype=torch.float32, device=A.device)
    if ws is None:
        need = ace_workspace_bytes(ACE_OP_CKA, N, 1, d_in, d_out, E, rank)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=A.device)
    _check(_lib.ace_pairwise_cka(_dtype(A), N, d_in, d_out, E, rank, _ptr(X), _ptr(A), _ptr(B),
                                 _ptr(S), _ptr(ws), ws.numel(), _stream(stream)),
           "ace_pairwise_cka")
    return S


def _host(a, dtype):
    import numpy as np
    return np.ascontiguousarray(a, dtype=dtype)


def ace_similarity_graph(S):
    """W [E, E] (float64, numpy) from the similarity matrix S [E, E] (host)."""
    import numpy as np
    S = _host(S, np.float32)
    E = S.shape[0]
    W = np.empty((E, E), dtype=np.float64)
    _check(_lib.ace_similarity_graph(S.ctypes.data, E, W.ctypes.data), "ace_similarity_graph")
    return W


def ace_louvain(W, gamma: float = 0.8):
    """(groups int32 [E], G) from the graph W [E, E] (host, float64)."""
    import numpy as np
    W = _host(W, np.float64)
    E = W.shape[0]
    groups = np.empty(E, dtype=np.int32)
    G = ctypes.c_int32(0)
    _check(_lib.ace_louvain(W.ctypes.data, E, float(gamma), groups.ctypes.data, ctypes.byref(G)),
           "ace_louvain")
    return groups, int(G.value)


def ace_group_anchors(S, expert_to_group, G: int):
    """CKA centre of every group (int32 [G])."""
    import numpy as np
    S = _host(S, np.float32)
    e2g = _host(expert_to_group, np.int32)
    anchors = np.empty(G, dtype=np.int32)
    _check(_lib.ace_group_anchors(S.ctypes.data, S.shape[0], e2g.ctypes.data, G,
                                  anchors.ctypes.data), "ace_group_anchors")
    return anchors


def ace_consolidate_adapters(A, B, E: int, rank: int, expert_to_group, G: int, anchors, A_init,
                             A_g=None, B_g=None, stream=None):
    """Group adapters (A_g, B_g, group ranks) from the expert adapters A, B
    (device); the library returns the group ranks.  A_g, B_g hold E * rank
    ranks in total (the unchanged budget)."""
    import numpy as np
    e2g = _host(expert_to_group, np.int32)
    anc = _host(anchors, np.int32)
    d_in = A.shape[1]
    d_out = B.numel() // (E * rank)
    if A_g is None:
        A_g = torch.empty(E * rank, d_in, dtype=A.dtype, device=A.device)
    if B_g is None:
        B_g = torch.empty(E * rank * d_out, dtype=B.dtype, device=B.device)
    for t, n in ((A_g, E * rank * d_in), (B_g, E * rank * d_out)):
        if t.numel() != n or t.dtype != A.dtype or t.device != A.device:
            raise ValueError("A_g / B_g must hold E * rank ranks in A's dtype and device")
    ranks = np.zeros(G, dtype=np.int32)
    _check(_lib.ace_consolidate_adapters(_dtype(A), d_in, d_out, E, rank, _ptr(A), _ptr(B),
                                         e2g.ctypes.data, G, anc.ctypes.data, _ptr(A_init),
                                         _ptr(A_g), _ptr(B_g), ranks.ctypes.data,
                                         _stream(stream)),
           "ace_consolidate_adapters")
    return A_g, B_g, [int(r) for r in ranks]


def raw_lib() -> ctypes.CDLL:
    """The loaded library (tests check exports and host-side validation)."""
    return _lib


def ace_moe_lora_fwd(x, W, expert_routing: Routing, y, key_rank: Optional[Sequence[int]] = None,
                     expert_key: Optional[Sequence[int]] = None, alpha: float = 16.0, A=None,
                     B=None, adapter_routing: Optional[Routing] = None,
                     input_mode: int = ACE_INPUT_SHARED, ws=None, stream=None) -> None:
    """y[t*k + j] = W_e xin(t, j) + s_q B_q (A_q xin(t, j)) (include/ace.h).
    key_rank None runs the plain expert projection."""
    T, k = expert_routing.c.T, expert_routing.c.k
    E, d_out, d_in = W.shape
    n_keys = 0 if key_rank is None else len(key_rank)
    ranks = ekey = None
    if n_keys:
        ranks, _, r_max = _rank_table(tuple(map(int, key_rank)))
        ekey = (ctypes.c_int32 * E)(*[int(v) for v in expert_key])
        ws = _fwd_ws(ws, T, k, d_in, d_out, n_keys, r_max, x.device)
    _check(_lib.ace_moe_lora_fwd(_dtype(x), input_mode, T, k, d_in, d_out, E, _ptr(x), _ptr(W),
                                 ctypes.byref(expert_routing.c), n_keys, ranks, ekey, alpha,
                                 _ptr(A), _ptr(B),
                                 ctypes.byref(adapter_routing.c) if adapter_routing else None,
                                 _ptr(y), _ptr(ws), 0 if ws is None else ws.numel(),
                                 _stream(stream)),
           "ace_moe_lora_fwd")


# The calls below check each tensor in one function (a call of a few microseconds
# is bound by the host), and refuse tensors of another device than the current one:
# the library launches on the current device's stream.
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on_device(t: torch.Tensor) -> int:
    """Index of the tensor's device, which must be the current one."""
    index = t.get_device()
    if index < 0 or index != _get_device():
        raise ValueError(f"tensors are on {t.device}, which is not the current GPU")
    return index


def _arg(name: str, t, numel: int, dtype, index: int) -> Optional[int]:
    """Pointer of a tensor argument of the given size, type and device."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{index}")
    if not t.is_contiguous():
        raise ValueError("tensors passed to libace must be contiguous")
    return t.data_ptr() or None


def _opt(name: str, t, numel: int, dtype, index: int) -> Optional[int]:
    return None if t is None else _arg(name, t, numel, dtype, index)


def _stream_on(index: int, stream) -> Optional[int]:
    if stream is None and _raw_stream is not None:
        return _raw_stream(index) or None
    return _stream(stream)


def _alloc(make, stream, *shape, **kw):
    """A tensor that belongs to the call's stream: filled there, and given out
    again only behind the work queued there."""
    if stream is None:
        return make(*shape, **kw)
    with torch.cuda.stream(stream):
        return make(*shape, **kw)


def _width(name: str, n: int) -> int:
    """A row length as the library's 32-bit argument (a longer one would wrap)."""
    if n >= 1 << 31:
        raise ValueError(f"{name} has {n} columns, more than 2^31 - 1")
    return n


def _check_routing(routing: Routing, T: int, k: int, index: int) -> None:
    if (routing.c.T, routing.c.k) != (T, k):
        raise ValueError(f"routing was built for T={routing.c.T} k={routing.c.k}, the call has "
                         f"T={T} k={k}")
    if routing.pair_row.get_device() != index:
        raise ValueError(f"routing is on {routing.pair_row.device}, expected cuda:{index}")


# a per-pair input gradient without a workspace computes the same sums in one piece;
# calls up to this size are given one
_DX_SPLIT_ELEMS = 1 << 22


def ace_moe_dx(dy, W, expert_routing: Routing, dx=None, input_mode: int = ACE_INPUT_SHARED,
               accumulate: bool = False, ws=None, stream=None) -> torch.Tensor:
    """Input gradient of the frozen expert projection (include/ace.h): per pair
    dx[t*k + j] = W_e^T dy[t*k + j], shared their sum over a token's slots.
    dx None allocates it (per pair: zeros, so that dropped pairs give 0)."""
    T, k = expert_routing.c.T, expert_routing.c.k
    dev = _on_device(W)
    if W.dim() != 3:
        raise ValueError(f"W must be [E, d_out, d_in], got {tuple(W.shape)}")
    E, d_out, d_in = W.shape
    _width("dx", d_in)
    _width("dy", d_out)
    dt = W.dtype
    _check_routing(expert_routing, T, k, dev)
    shared = input_mode == ACE_INPUT_SHARED
    rows = T if shared else T * k
    if dx is None:
        if accumulate:
            raise ValueError("accumulate needs dx")
        dx = _alloc(torch.empty if shared else torch.zeros, stream, rows, d_in, dtype=dt,
                    device=W.device)
    if ws is None and (shared or accumulate or T * k * d_in <= _DX_SPLIT_ELEMS):
        need = ace_workspace_bytes(ACE_OP_MOE_DX, T, k, d_in, d_out, E, 0)
        ws = _alloc(torch.empty, stream, max(need, 256), dtype=torch.uint8, device=W.device)
    ws_bytes = 0 if ws is None else ws.numel()
    _check(_lib.ace_moe_dx(_dtype(W), input_mode, T, k, d_in, d_out, E,
                           _arg("dy", dy, T * k * d_out, dt, dev),
                           _arg("W", W, E * d_out * d_in, dt, dev), ctypes.byref(expert_routing.c),
                           int(accumulate), _arg("dx", dx, rows * d_in, dt, dev),
                           _opt("ws", ws, ws_bytes, torch.uint8, dev), ws_bytes,
                           _stream_on(dev, stream)), "ace_moe_dx")
    return dx


def ace_moe_combine_fwd(y, routing: Routing, out=None, pair_w=None, stream=None) -> torch.Tensor:
    """out[t] = sum over the routed slots j of pair_w[t, j] y[t*k + j]."""
    T, k = routing.c.T, routing.c.k
    dev = _on_device(y)
    if y.dim() != 2 or y.shape[0] != T * k:
        raise ValueError(f"y must be [T*k={T * k}, d], got {tuple(y.shape)}")
    d, dt = _width("y", y.shape[1]), y.dtype
    _check_routing(routing, T, k, dev)
    if out is None:
        out = _alloc(torch.empty, stream, T, d, dtype=dt, device=y.device)
    _check(_lib.ace_moe_combine_fwd(_dtype(y), T, k, d, _arg("y", y, T * k * d, dt, dev),
                                    _opt("pair_w", pair_w, T * k, torch.float32, dev),
                                    ctypes.byref(routing.c), _arg("out", out, T * d, dt, dev),
                                    _stream_on(dev, stream)), "ace_moe_combine_fwd")
    return out


def ace_moe_combine_bwd(dout, routing: Routing, dy=None, pair_w=None, y=None, dw=None,
                        stream=None) -> torch.Tensor:
    """dy[t*k + j] = pair_w[t, j] dout[t]; with dw also dw[t, j] = <dout[t], y[t*k + j]>.
    dy None allocates it (zeros, so that dropped pairs give 0)."""
    T, k = routing.c.T, routing.c.k
    dev = _on_device(dout)
    if dout.dim() != 2 or dout.shape[0] != T:
        raise ValueError(f"dout must be [T={T}, d], got {tuple(dout.shape)}")
    d, dt = _width("dout", dout.shape[1]), dout.dtype
    _check_routing(routing, T, k, dev)
    if dy is None:
        dy = _alloc(torch.zeros, stream, T * k, d, dtype=dt, device=dout.device)
    yp = _opt("y", y, T * k * d, dt, dev) if dw is None else _arg("y", y, T * k * d, dt, dev)
    _check(_lib.ace_moe_combine_bwd(_dtype(dout), T, k, d, _arg("dout", dout, T * d, dt, dev), yp,
                                    _opt("pair_w", pair_w, T * k, torch.float32, dev),
                                    ctypes.byref(routing.c), _arg("dy", dy, T * k * d, dt, dev),
                                    _opt("dw", dw, T * k, torch.float32, dev),
                                    _stream_on(dev, stream)), "ace_moe_combine_bwd")
    return dy


class PackedAct:
    """Owns the device arrays of an ace_packed_act: activation rows [rows, d]
    at 8.25 bits per element."""

    def __init__(self, rows: int, d: int, device="cuda"):
        self.rows, self.d = int(rows), int(d)
        self.codes = torch.empty(self.rows, self.d, dtype=torch.int8, device=device)
        self.exps = torch.empty(self.rows, -(-self.d // 32), dtype=torch.uint8, device=device)
        self.c = AcePackedAct(self.codes.data_ptr() or None, self.exps.data_ptr() or None)


def _packed(name: str, c: PackedAct, rows: int, d: int, index: int):
    """Checkpoint argument of the given shape and device."""
    if not isinstance(c, PackedAct):
        raise TypeError(f"{name} must be a PackedAct")
    if c.rows != rows or c.d != d:
        raise ValueError(f"{name} holds [{c.rows}, {c.d}], expected [{rows}, {d}]")
    if c.codes.get_device() != index:
        raise ValueError(f"{name} is on {c.codes.device}, expected cuda:{index}")
    return ctypes.byref(c.c)


def _rows(name: str, t: torch.Tensor):
    if t.dim() != 2:
        raise ValueError(f"{name} must be [rows, d], got {tuple(t.shape)}")
    _width(name, t.shape[1])
    return t.shape


def ace_act_pack(x, packed: Optional[PackedAct] = None, stream=None) -> PackedAct:
    """8-bit checkpoint of the rows x [rows, d] (include/ace.h)."""
    dev = _on_device(x)
    rows, d = _rows("x", x)
    if packed is None:
        packed = _alloc(PackedAct, stream, rows, d, device=x.device)
    _check(_lib.ace_act_pack(_dtype(x), rows, d, _arg("x", x, rows * d, x.dtype, dev),
                             _packed("packed", packed, rows, d, dev), _stream_on(dev, stream)),
           "ace_act_pack")
    return packed


def ace_act_unpack(packed: PackedAct, x=None, dtype=None, stream=None) -> torch.Tensor:
    """The rows that a checkpoint stands for: into x, or a new tensor of dtype
    (bf16 by default; the values are exact in both types)."""
    dev = _on_device(packed.codes)
    rows, d = packed.rows, _width("packed", packed.d)
    if x is None:
        x = _alloc(torch.empty, stream, rows, d, dtype=dtype or torch.bfloat16,
                   device=packed.codes.device)
    _check(_lib.ace_act_unpack(_dtype(x), rows, d, _packed("packed", packed, rows, d, dev),
                               _arg("x", x, rows * d, dtype or x.dtype, dev),
                               _stream_on(dev, stream)), "ace_act_unpack")
    return x


def _gate_up(g, u, rows: int, d: int, dtype, index: int):
    """(g, u, g_packed, u_packed) as the library takes them: pointers of the
    tensors, or None and the checkpoints."""
    if isinstance(g, PackedAct) != isinstance(u, PackedAct):
        raise TypeError("g and u must both be tensors or both be PackedAct")
    if isinstance(g, PackedAct):
        return None, None, _packed("g", g, rows, d, index), _packed("u", u, rows, d, index)
    n = rows * d
    return _arg("g", g, n, dtype, index), _arg("u", u, n, dtype, index), None, None


def ace_swiglu_fwd(g, u, a=None, g_packed: Optional[PackedAct] = None,
                   u_packed: Optional[PackedAct] = None, dtype=None, stream=None) -> torch.Tensor:
    """a = g sigmoid(g) u per row.  g and u are tensors (with g_packed and
    u_packed their 8-bit checkpoints are written in the same pass) or both
    PackedAct (then a, or dtype, tells the type: bf16 by default)."""
    held = isinstance(g, PackedAct)
    src = g.codes if held else g
    dev = _on_device(src)
    rows, d = _rows("g", src)
    if held and (g_packed is not None or u_packed is not None):
        raise ValueError("g and u are checkpoints already")
    if dtype is None:
        dtype = g.dtype if not held else a.dtype if a is not None else torch.bfloat16
    gp, up, g8, u8 = _gate_up(g, u, rows, d, dtype, dev)
    if a is None:
        a = _alloc(torch.empty, stream, rows, d, dtype=dtype, device=src.device)
    if g_packed is not None:
        g8 = _packed("g_packed", g_packed, rows, d, dev)
    if u_packed is not None:
        u8 = _packed("u_packed", u_packed, rows, d, dev)
    _check(_lib.ace_swiglu_fwd(_dtype(a), rows, d, gp, up, _arg("a", a, rows * d, dtype, dev), g8,
                               u8, _stream_on(dev, stream)), "ace_swiglu_fwd")
    return a


def ace_swiglu_bwd(da, g, u, dg=None, du=None, stream=None):
    """(dg, du) of ace_swiglu_fwd; g and u are the forward's tensors or, both,
    their checkpoints (PackedAct)."""
    dev = _on_device(da)
    rows, d = _rows("da", da)
    dt = da.dtype
    gp, up, g8, u8 = _gate_up(g, u, rows, d, dt, dev)
    if dg is None:
        dg = _alloc(torch.empty, stream, rows, d, dtype=dt, device=da.device)
    if du is None:
        du = _alloc(torch.empty, stream, rows, d, dtype=dt, device=da.device)
    n = rows * d
    _check(_lib.ace_swiglu_bwd(_dtype(da), rows, d, _arg("da", da, n, dt, dev), gp, up, g8, u8,
                               _arg("dg", dg, n, dt, dev), _arg("du", du, n, dt, dev),
                               _stream_on(dev, stream)), "ace_swiglu_bwd")
    return dg, du
