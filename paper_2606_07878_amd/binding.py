"""ctypes binding of libstill.so (include/still.h).

Argument marshalling only: torch tensors supply device pointers and the
current HIP stream; every step of the compaction runs in the library's HIP
kernels.  There is no fallback: if the library is missing or fails to load,
every entry point raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence

from . import configs

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libstill.so")

STILL_OK = 0
STATUS = {0: "STILL_OK", -1: "STILL_E_INVAL", -2: "STILL_E_SHAPE", -3: "STILL_E_DTYPE",
          -4: "STILL_E_WORKSPACE", -5: "STILL_E_UNSUPPORTED", -6: "STILL_E_HIP"}
STILL_F_REROTATE = 1


class StillError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS.get(status, status)}: {detail}")
        self.status = status


class still_config(ctypes.Structure):
    _fields_ = [("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("latent_dim", ctypes.c_int32), ("n_blocks", ctypes.c_int32),
                ("cross_every_block", ctypes.c_int32), ("n_cross_heads", ctypes.c_int32),
                ("cross_head_dim", ctypes.c_int32), ("n_self_heads", ctypes.c_int32),
                ("self_head_dim", ctypes.c_int32), ("ffn_kind", ctypes.c_int32),
                ("ffn_hidden", ctypes.c_int32), ("final_norm", ctypes.c_int32),
                ("logit_scale_cross", ctypes.c_float), ("logit_scale_self", ctypes.c_float),
                ("compactor_rope_base", ctypes.c_double), ("rms_eps", ctypes.c_float),
                ("l2_eps", ctypes.c_float), ("mode", ctypes.c_int32)]


_BLOCK_FIELDS = ["ca_wq", "ca_bq", "ca_wk", "ca_bk", "ca_wv", "ca_wo",
                 "sa_wq", "sa_bq", "sa_wk", "sa_bk", "sa_wv", "sa_wo",
                 "ffn_wg", "ffn_wu", "ffn_wd"]


class still_block_weights(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in _BLOCK_FIELDS]


class still_layer_weights(ctypes.Structure):
    _fields_ = [("latents", ctypes.c_void_p), ("t_bank", ctypes.c_int32),
                ("blocks", ctypes.POINTER(still_block_weights)),
                ("w_key", ctypes.c_void_p), ("w_val", ctypes.c_void_p)]


class still_beta_opts(ctypes.Structure):
    _fields_ = [("beta_max", ctypes.c_float), ("mass_alpha", ctypes.c_float), ("log_x", ctypes.c_float)]


class still_attend_config(ctypes.Structure):
    _fields_ = [("n_kv_heads", ctypes.c_int32), ("group", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_queries", ctypes.c_int32), ("t", ctypes.c_int32), ("n_suffix", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("scale", ctypes.c_float), ("mode", ctypes.c_int32),
                ("rope_theta", ctypes.c_double)]


class still_paged_cache(ctypes.Structure):
    _fields_ = [("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("mode", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("beta", ctypes.c_void_p)]


class still_paged8_cache(ctypes.Structure):
    _fields_ = [("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("mode", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("beta", ctypes.c_void_p)]


class still_paged_seqs(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p)]


class still_paged_tokens(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_token_stride", ctypes.c_int64), ("k_head_stride", ctypes.c_int64),
                ("v_token_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64),
                ("beta", ctypes.c_void_p), ("beta_token_stride", ctypes.c_int64),
                ("beta_head_stride", ctypes.c_int64), ("offsets", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("rope_theta", ctypes.c_double)]


class still_paged_attend_config(ctypes.Structure):
    _fields_ = [("group", ctypes.c_int32), ("n_queries", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float), ("rope_theta", ctypes.c_double), ("q_stride", ctypes.c_int64)]


class still_paged_evict_config(ctypes.Structure):
    _fields_ = [("keep", ctypes.c_int32), ("first", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("shared", ctypes.c_int32)]


_lib = None


def lib():
    """Load libstill.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2606_07878_amd.build` (no CPU fallback exists)")
        L = ctypes.CDLL(_LIB_PATH)
        L.still_workspace_size.argtypes = [ctypes.POINTER(still_config), ctypes.c_int64, ctypes.c_int32,
                                           ctypes.c_int32]
        L.still_workspace_size.restype = ctypes.c_size_t
        common = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_double, ctypes.c_int32, ctypes.c_uint32]
        L.still_compact_layer.argtypes = [ctypes.POINTER(still_config), ctypes.POINTER(still_layer_weights),
                                          ctypes.c_void_p, ctypes.c_void_p, *common,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.still_compact_layer.restype = ctypes.c_int32
        L.still_compact_model.argtypes = [ctypes.POINTER(still_config), ctypes.c_int32,
                                          ctypes.POINTER(still_layer_weights),
                                          ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                                          *common,
                                          ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.still_compact_model.restype = ctypes.c_int32
        L.still_compact_model_beta.argtypes = [*L.still_compact_model.argtypes[:13],
                                               ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(still_beta_opts),
                                               ctypes.POINTER(ctypes.c_void_p),
                                               ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.still_compact_model_beta.restype = ctypes.c_int32
        L.still_attend_workspace_size.argtypes = [ctypes.POINTER(still_attend_config)]
        L.still_attend_workspace_size.restype = ctypes.c_size_t
        L.still_attend.argtypes = [ctypes.POINTER(still_attend_config), *[ctypes.c_void_p] * 9, ctypes.c_size_t,
                                   ctypes.c_void_p]
        L.still_attend.restype = ctypes.c_int32
        L.still_backward_workspace_size.argtypes = [ctypes.POINTER(still_config), ctypes.c_int64, ctypes.c_int32]
        L.still_backward_workspace_size.restype = ctypes.c_size_t
        L.still_compact_layer_backward.argtypes = [ctypes.POINTER(still_config),
                                                   ctypes.POINTER(still_layer_weights), ctypes.c_void_p,
                                                   ctypes.c_void_p, *common, ctypes.c_void_p, ctypes.c_void_p,
                                                   ctypes.POINTER(still_layer_weights), ctypes.c_void_p,
                                                   ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                   ctypes.c_void_p]
        L.still_compact_layer_backward.restype = ctypes.c_int32
        L.still_attend_scratch.argtypes = [ctypes.POINTER(still_attend_config), *[ctypes.c_void_p] * 9]
        L.still_attend_scratch.restype = ctypes.c_int32
        cache, seqs = ctypes.POINTER(still_paged_cache), ctypes.POINTER(still_paged_seqs)
        L.still_paged_append.argtypes = [cache, seqs, ctypes.POINTER(still_paged_tokens), ctypes.c_void_p]
        L.still_paged_append.restype = ctypes.c_int32
        L.still_paged_gather.argtypes = [cache, seqs, *[ctypes.c_int32] * 3, *[ctypes.c_void_p] * 4]
        L.still_paged_gather.restype = ctypes.c_int32
        L.still_paged_attend_workspace_size.argtypes = [cache, ctypes.POINTER(still_paged_attend_config)]
        L.still_paged_attend_workspace_size.restype = ctypes.c_size_t
        L.still_paged_attend.argtypes = [cache, seqs, ctypes.POINTER(still_paged_attend_config),
                                         *[ctypes.c_void_p] * 4, ctypes.c_size_t, ctypes.c_void_p]
        L.still_paged_attend.restype = ctypes.c_int32
        L.still_paged_attend_lse.argtypes = [cache, seqs, ctypes.POINTER(still_paged_attend_config),
                                             *[ctypes.c_void_p] * 5, ctypes.c_size_t, ctypes.c_void_p]
        L.still_paged_attend_lse.restype = ctypes.c_int32
        cache8 = ctypes.POINTER(still_paged8_cache)
        for plain, eight in ((L.still_paged_append, L.still_paged8_append), (L.still_paged_gather, L.still_paged8_gather),
                             (L.still_paged_attend_workspace_size, L.still_paged8_attend_workspace_size),
                             (L.still_paged_attend_lse, L.still_paged8_attend)):
            eight.argtypes = [cache8, *plain.argtypes[1:]]
            eight.restype = plain.restype
        for kind, score, evict in ((cache, L.still_paged_score, L.still_paged_evict),
                                   (cache8, L.still_paged8_score, L.still_paged8_evict)):
            score.argtypes = [kind, seqs, ctypes.POINTER(still_paged_attend_config), *[ctypes.c_void_p] * 6]
            evict.argtypes = [kind, seqs, ctypes.POINTER(still_paged_evict_config), *[ctypes.c_void_p] * 4, ctypes.c_size_t,
                              ctypes.c_void_p]
            score.restype = evict.restype = ctypes.c_int32
        L.still_paged_evict_workspace_size.argtypes = [cache, seqs, ctypes.POINTER(still_paged_evict_config)]
        L.still_paged_evict_workspace_size.restype = ctypes.c_size_t
        L.still_status_string.argtypes = [ctypes.c_int32]
        L.still_status_string.restype = ctypes.c_char_p
        L.still_last_error.argtypes = []
        L.still_last_error.restype = ctypes.c_char_p
        L.still_version.argtypes = []
        L.still_version.restype = ctypes.c_char_p
        L.still_timing_enable.argtypes = [ctypes.c_int32]
        L.still_timing_enable.restype = ctypes.c_int32
        L.still_timing_reset.argtypes = []
        L.still_timing_reset.restype = ctypes.c_int32
        L.still_timing_read.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_int64)]
        L.still_timing_read.restype = ctypes.c_int32
        _lib = L
    return _lib


def make_config(cfg: configs.CompactorConfig, mode: int = configs.MODE_BF16) -> still_config:
    return still_config(cfg.n_kv_heads, cfg.head_dim, cfg.latent_dim, cfg.n_blocks, cfg.cross_every_block,
                        cfg.n_cross_heads, cfg.cross_head_dim, cfg.n_self_heads, cfg.self_head_dim,
                        cfg.ffn_kind, cfg.ffn_hidden, cfg.final_norm, cfg.logit_scale_cross,
                        cfg.logit_scale_self, cfg.compactor_rope_base, cfg.rms_eps, cfg.l2_eps, mode)


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    return x.data_ptr() if hasattr(x, "data_ptr") else int(x)


class LayerWeights:
    """still_layer_weights built from a dict of device tensors keyed like
    ``configs.layer_shapes`` (keeps the tensors alive)."""

    def __init__(self, cfg: configs.CompactorConfig, tensors: Dict[str, object]):
        self.tensors = tensors
        nb = cfg.n_blocks
        self._blocks = (still_block_weights * nb)()
        for b in range(nb):
            for f in _BLOCK_FIELDS:
                setattr(self._blocks[b], f, _ptr(tensors.get(f"b{b}.{f}")))
        lat = tensors["latents"]
        self.struct = still_layer_weights(_ptr(lat), int(lat.shape[1]), self._blocks,
                                          _ptr(tensors["w_key"]), _ptr(tensors["w_val"]))


def _check(status: int):
    if status != STILL_OK:
        raise StillError(status, lib().still_last_error().decode())


def still_workspace_size(cfg: still_config, N: int, t: int, n_layers: int = 1) -> int:
    return int(lib().still_workspace_size(ctypes.byref(cfg), N, t, n_layers))


def still_compact_layer(cfg: still_config, w: LayerWeights, K, V, positions, N: int, rope_theta: float,
                        t: int, flags: int, C_k, C_v, out_positions, workspace, workspace_bytes: int,
                        stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_compact_layer(ctypes.byref(cfg), ctypes.byref(w.struct), _ptr(K), _ptr(V),
                                     _ptr(positions), N, rope_theta, t, flags, _ptr(C_k), _ptr(C_v),
                                     _ptr(out_positions), _ptr(workspace), workspace_bytes, _ptr(stream))


def still_compact_model(cfg: still_config, ws: Sequence[LayerWeights], K: Sequence, V: Sequence, positions,
                        N: int, rope_theta: float, t: int, flags: int, C_k: Sequence, C_v: Sequence,
                        out_positions, workspace, workspace_bytes: int, stream) -> int:
    L = len(ws)
    wa = (still_layer_weights * L)(*[w.struct for w in ws])
    arr = lambda xs: (ctypes.c_void_p * L)(*[_ptr(x) for x in xs])  # noqa: E731
    return lib().still_compact_model(ctypes.byref(cfg), L, wa, arr(K), arr(V), _ptr(positions), N,
                                     rope_theta, t, flags, arr(C_k), arr(C_v), _ptr(out_positions),
                                     _ptr(workspace), workspace_bytes, _ptr(stream))


def still_compact_model_beta(cfg: still_config, ws: Sequence[LayerWeights], K: Sequence, V: Sequence, positions,
                             N: int, rope_theta: float, t: int, flags: int, C_k: Sequence, C_v: Sequence,
                             out_positions, w_beta: Sequence, beta_opts: Optional[still_beta_opts],
                             beta: Sequence, workspace, workspace_bytes: int, stream) -> int:
    L = len(ws)
    wa = (still_layer_weights * L)(*[w.struct for w in ws])
    arr = lambda xs: (ctypes.c_void_p * L)(*[_ptr(x) for x in xs])  # noqa: E731
    return lib().still_compact_model_beta(ctypes.byref(cfg), L, wa, arr(K), arr(V), _ptr(positions), N,
                                          rope_theta, t, flags, arr(C_k), arr(C_v), _ptr(out_positions),
                                          arr(w_beta), ctypes.byref(beta_opts) if beta_opts is not None else None,
                                          arr(beta), _ptr(workspace), workspace_bytes, _ptr(stream))


def still_attend_workspace_size(cfg: still_attend_config) -> int:
    return int(lib().still_attend_workspace_size(ctypes.byref(cfg)))


def still_attend(cfg: still_attend_config, q, q_positions, C_k, C_v, beta, K, V, out, workspace,
                 workspace_bytes: int, stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_attend(ctypes.byref(cfg), _ptr(q), _ptr(q_positions), _ptr(C_k), _ptr(C_v), _ptr(beta),
                              _ptr(K), _ptr(V), _ptr(out), _ptr(workspace), workspace_bytes, _ptr(stream))


def still_attend_scratch(cfg: still_attend_config, q, q_positions, C_k, C_v, beta, K, V, out, stream) -> int:
    """Raw entry point of the allocation-free attention (no workspace argument);
    returns the status code."""
    return lib().still_attend_scratch(ctypes.byref(cfg), _ptr(q), _ptr(q_positions), _ptr(C_k), _ptr(C_v),
                                      _ptr(beta), _ptr(K), _ptr(V), _ptr(out), _ptr(stream))


STILL_ATTEND_SCRATCH_BYTES = 68 << 20


def still_paged_append(cache: still_paged_cache, seqs: still_paged_seqs, tokens: still_paged_tokens, stream) -> int:
    """Raw entry point; returns the status code."""
    return lib().still_paged_append(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(tokens), _ptr(stream))


def still_paged_gather(cache: still_paged_cache, seqs: still_paged_seqs, seq: int, start: int, n: int, K, V, beta,
                       stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_paged_gather(ctypes.byref(cache), ctypes.byref(seqs), seq, start, n, _ptr(K), _ptr(V),
                                    _ptr(beta), _ptr(stream))


def still_paged_attend_workspace_size(cache: still_paged_cache, cfg: still_paged_attend_config) -> int:
    return int(lib().still_paged_attend_workspace_size(ctypes.byref(cache), ctypes.byref(cfg)))


def still_paged_attend(cache: still_paged_cache, seqs: still_paged_seqs, cfg: still_paged_attend_config, q,
                       q_positions, out, workspace, workspace_bytes: int, stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_paged_attend(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), _ptr(q),
                                    _ptr(q_positions), _ptr(out), _ptr(workspace), workspace_bytes, _ptr(stream))


def still_paged_attend_lse(cache: still_paged_cache, seqs: still_paged_seqs, cfg: still_paged_attend_config, q,
                           q_positions, out, lse, workspace, workspace_bytes: int, stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_paged_attend_lse(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), _ptr(q),
                                        _ptr(q_positions), _ptr(out), _ptr(lse), _ptr(workspace), workspace_bytes,
                                        _ptr(stream))


def still_paged8_append(cache: still_paged8_cache, seqs: still_paged_seqs, tokens: still_paged_tokens, stream) -> int:
    """Raw entry point; returns the status code."""
    return lib().still_paged8_append(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(tokens), _ptr(stream))


def still_paged8_gather(cache: still_paged8_cache, seqs: still_paged_seqs, seq: int, start: int, n: int, K, V, beta,
                        stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_paged8_gather(ctypes.byref(cache), ctypes.byref(seqs), seq, start, n, _ptr(K), _ptr(V),
                                     _ptr(beta), _ptr(stream))


def still_paged8_attend_workspace_size(cache: still_paged8_cache, cfg: still_paged_attend_config) -> int:
    return int(lib().still_paged8_attend_workspace_size(ctypes.byref(cache), ctypes.byref(cfg)))


def still_paged8_attend(cache: still_paged8_cache, seqs: still_paged_seqs, cfg: still_paged_attend_config, q,
                        q_positions, out, lse, workspace, workspace_bytes: int, stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_paged8_attend(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), _ptr(q),
                                     _ptr(q_positions), _ptr(out), _ptr(lse), _ptr(workspace), workspace_bytes,
                                     _ptr(stream))


def still_paged_score(cache, seqs: still_paged_seqs, cfg: still_paged_attend_config, q, q_positions, lse, known, scores,
                      stream) -> int:
    """Raw entry points still_paged_score and, for a still_paged8_cache, still_paged8_score (pointers or
    tensors); returns the status code."""
    call = lib().still_paged8_score if isinstance(cache, still_paged8_cache) else lib().still_paged_score
    return call(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), _ptr(q), _ptr(q_positions), _ptr(lse),
                _ptr(known), _ptr(scores), _ptr(stream))


def still_paged_evict_workspace_size(cache: still_paged_cache, seqs: still_paged_seqs, cfg: still_paged_evict_config) -> int:
    return int(lib().still_paged_evict_workspace_size(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg)))


def still_paged_evict(cache, seqs: still_paged_seqs, cfg: still_paged_evict_config, scores, kept, new_lens, workspace,
                      workspace_bytes: int, stream) -> int:
    """Raw entry points still_paged_evict and, for a still_paged8_cache, still_paged8_evict (pointers or
    tensors); returns the status code."""
    call = lib().still_paged8_evict if isinstance(cache, still_paged8_cache) else lib().still_paged_evict
    return call(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), _ptr(scores), _ptr(kept), _ptr(new_lens),
                _ptr(workspace), workspace_bytes, _ptr(stream))


STILL_PAGED_WORKSPACE_BYTES = 17 << 20


def still_status_string(status: int) -> str:
    return lib().still_status_string(status).decode()


def still_last_error() -> str:
    return lib().still_last_error().decode()


def still_version() -> str:
    return lib().still_version().decode()


# kernel classes of the timing facility (still.h)
KERNEL_CLASSES = {"cross_attn": 0, "kproj": 1, "qproj": 2, "refine": 3, "latent": 4, "other": 5, "attend": 6,
                  "stage": 7}


def still_timing_enable(class_mask: int) -> None:
    """Record hipEvent pairs around launches of the classes in class_mask (0 = off)."""
    _check(lib().still_timing_enable(int(class_mask)))


def still_timing_reset() -> None:
    _check(lib().still_timing_reset())


def still_timing_read(kernel_class: int):
    """(total ms, launches) of one kernel class since the last reset."""
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    _check(lib().still_timing_read(kernel_class, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


# ----------------------------------------------------------------------------
# torch conveniences (allocation of outputs / workspace on the caller's device)
# ----------------------------------------------------------------------------

def _torch():
    import torch
    return torch


def compact_model(cfg: configs.CompactorConfig, weights: List[Dict[str, object]], K: List, V: List, positions,
                  rope_theta: float, t: int, rerotate: bool = True, mode: int = configs.MODE_BF16,
                  workspace=None, outputs=None):
    """Compact L layers on the current stream; returns ([C_k], [C_v], out_positions)."""
    torch = _torch()
    dev = K[0].device
    ccfg = make_config(cfg, mode)
    N = int(K[0].shape[1])
    L = len(K)
    need = still_workspace_size(ccfg, N, t, L)
    if need == 0:
        raise StillError(-5, "configuration rejected by still_workspace_size")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    dt = K[0].dtype
    if outputs is None:
        Ck = [torch.empty(cfg.n_kv_heads, t, cfg.head_dim, dtype=dt, device=dev) for _ in range(L)]
        Cv = [torch.empty(cfg.n_kv_heads, t, cfg.head_dim, dtype=dt, device=dev) for _ in range(L)]
    else:
        Ck, Cv = outputs
    outp = torch.empty(t, dtype=torch.float64, device=dev)
    lw = [w if isinstance(w, LayerWeights) else LayerWeights(cfg, w) for w in weights]
    stream = torch.cuda.current_stream(dev).cuda_stream
    _check(still_compact_model(ccfg, lw, K, V, positions, N, rope_theta, t,
                               STILL_F_REROTATE if rerotate else 0, Ck, Cv, outp, workspace,
                               workspace.numel(), stream))
    return Ck, Cv, outp


def compact_layer(cfg: configs.CompactorConfig, weights: Dict[str, object], K, V, positions, rope_theta: float,
                  t: int, rerotate: bool = True, mode: int = configs.MODE_BF16, workspace=None):
    """Compact one layer through still_compact_layer; returns (C_k, C_v, out_positions)."""
    torch = _torch()
    dev = K.device
    ccfg = make_config(cfg, mode)
    N = int(K.shape[1])
    need = still_workspace_size(ccfg, N, t, 1)
    if need == 0:
        raise StillError(-5, "configuration rejected by still_workspace_size")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    Ck = torch.empty(cfg.n_kv_heads, t, cfg.head_dim, dtype=K.dtype, device=dev)
    Cv = torch.empty_like(Ck)
    outp = torch.empty(t, dtype=torch.float64, device=dev)
    lw = weights if isinstance(weights, LayerWeights) else LayerWeights(cfg, weights)
    stream = torch.cuda.current_stream(dev).cuda_stream
    _check(still_compact_layer(ccfg, lw, K, V, positions, N, rope_theta, t,
                               STILL_F_REROTATE if rerotate else 0, Ck, Cv, outp, workspace,
                               workspace.numel(), stream))
    return Ck, Cv, outp


def still_backward_workspace_size(cfg: still_config, N: int, t: int) -> int:
    return int(lib().still_backward_workspace_size(ctypes.byref(cfg), N, t))


def still_compact_layer_backward(cfg: still_config, w: LayerWeights, K, V, positions, N: int, rope_theta: float,
                                 t: int, flags: int, dC_k, dC_v, grad: LayerWeights, C_k, C_v, workspace,
                                 workspace_bytes: int, stream) -> int:
    """Raw entry point (pointers or tensors); returns the status code."""
    return lib().still_compact_layer_backward(ctypes.byref(cfg), ctypes.byref(w.struct), _ptr(K), _ptr(V),
                                              _ptr(positions), N, rope_theta, t, flags, _ptr(dC_k), _ptr(dC_v),
                                              ctypes.byref(grad.struct), _ptr(C_k), _ptr(C_v), _ptr(workspace),
                                              workspace_bytes, _ptr(stream))


def compact_layer_backward(cfg: configs.CompactorConfig, weights: Dict[str, object], K, V, positions,
                           rope_theta: float, t: int, dC_k, dC_v, rerotate: bool = True, workspace=None):
    """Gradients of <dC_k, C_k> + <dC_v, C_v> w.r.t. every compactor tensor
    (fp32 mode) through still_compact_layer_backward; returns (grads dict
    keyed like ``weights``, C_k, C_v) as float32 tensors on K's device."""
    torch = _torch()
    dev = K.device
    ccfg = make_config(cfg, configs.MODE_FP32)
    N = int(K.shape[1])
    need = still_backward_workspace_size(ccfg, N, t)
    if need == 0:
        raise StillError(-5, "configuration rejected by still_backward_workspace_size")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    grads = {k: torch.empty(tuple(v.shape), dtype=torch.float32, device=dev) for k, v in weights.items()}
    Ck = torch.empty(cfg.n_kv_heads, t, cfg.head_dim, dtype=torch.float32, device=dev)
    Cv = torch.empty_like(Ck)
    lw = weights if isinstance(weights, LayerWeights) else LayerWeights(cfg, weights)
    gw = LayerWeights(cfg, grads)
    stream = torch.cuda.current_stream(dev).cuda_stream
    _check(still_compact_layer_backward(ccfg, lw, K, V, positions, N, rope_theta, t,
                                        STILL_F_REROTATE if rerotate else 0, dC_k, dC_v, gw, Ck, Cv, workspace,
                                        workspace.numel(), stream))
    return grads, Ck, Cv


def compact_subrange(cfg: configs.CompactorConfig, weights: Dict[str, object], K, V, positions, rope_theta: float,
                     t: int, start: int, end: int, rerotate: bool = True, mode: int = configs.MODE_BF16):
    """Compact only the cache entries [start, end) of one layer (to t) and
    splice the preserved prefix and suffix back around them: returns
    (K', V', positions') with N - (end - start) + t entries.  The compaction
    runs through still_compact_layer; slicing and concatenation are copies."""
    torch = _torch()
    N = int(K.shape[1])
    if not (0 <= start < end <= N):
        raise StillError(-1, f"subrange [{start}, {end}) outside [0, {N})")
    Ck, Cv, pq = compact_layer(cfg, weights, K[:, start:end].contiguous(), V[:, start:end].contiguous(),
                               positions[start:end].contiguous(), rope_theta, t, rerotate=rerotate, mode=mode)
    return (torch.cat([K[:, :start], Ck, K[:, end:]], dim=1), torch.cat([V[:, :start], Cv, V[:, end:]], dim=1),
            torch.cat([positions[:start], pq, positions[end:]]))


def compact_chunks(cfg: configs.CompactorConfig, weights: Dict[str, object], K, V, positions, rope_theta: float,
                   t: int, chunk: int, rerotate: bool = True, mode: int = configs.MODE_BF16):
    """Independent chunk compaction: consecutive chunks of `chunk` entries (the
    last may be shorter) are each compacted to t by still_compact_layer and
    the compact chunks concatenated in order."""
    torch = _torch()
    N = int(K.shape[1])
    if chunk < 1:
        raise StillError(-1, "chunk must be >= 1")
    lw = weights if isinstance(weights, LayerWeights) else LayerWeights(cfg, weights)
    need = still_workspace_size(make_config(cfg, mode), min(chunk, N), t, 1)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=K.device)   # shared by the chunks (one stream)
    outs = [compact_layer(cfg, lw, K[:, a:a + chunk].contiguous(), V[:, a:a + chunk].contiguous(),
                          positions[a:a + chunk].contiguous(), rope_theta, t, rerotate=rerotate, mode=mode,
                          workspace=ws)
            for a in range(0, N, chunk)]
    return (torch.cat([o[0] for o in outs], dim=1), torch.cat([o[1] for o in outs], dim=1),
            torch.cat([o[2] for o in outs]))


def compact_model_beta(cfg: configs.CompactorConfig, weights: List[Dict[str, object]], K: List, V: List,
                       positions, rope_theta: float, t: int, w_beta: List, beta_max: float = 0.0,
                       mass_alpha: float = 0.0, log_x: float = 0.0, rerotate: bool = True,
                       mode: int = configs.MODE_BF16, workspace=None):
    """compact_model plus the bias head: returns ([C_k], [C_v], out_positions, [beta [H, t] float32])."""
    torch = _torch()
    dev = K[0].device
    ccfg = make_config(cfg, mode)
    N = int(K[0].shape[1])
    L = len(K)
    need = still_workspace_size(ccfg, N, t, L)
    if need == 0:
        raise StillError(-5, "configuration rejected by still_workspace_size")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    dt = K[0].dtype
    Ck = [torch.empty(cfg.n_kv_heads, t, cfg.head_dim, dtype=dt, device=dev) for _ in range(L)]
    Cv = [torch.empty(cfg.n_kv_heads, t, cfg.head_dim, dtype=dt, device=dev) for _ in range(L)]
    betas = [torch.empty(cfg.n_kv_heads, t, dtype=torch.float32, device=dev) for _ in range(L)]
    outp = torch.empty(t, dtype=torch.float64, device=dev)
    lw = [w if isinstance(w, LayerWeights) else LayerWeights(cfg, w) for w in weights]
    stream = torch.cuda.current_stream(dev).cuda_stream
    _check(still_compact_model_beta(ccfg, lw, K, V, positions, N, rope_theta, t,
                                    STILL_F_REROTATE if rerotate else 0, Ck, Cv, outp, w_beta,
                                    still_beta_opts(beta_max, mass_alpha, log_x), betas, workspace,
                                    workspace.numel(), stream))
    return Ck, Cv, outp, betas


def attend(q, C_k, C_v, beta, K, V, group: int = 1, causal: bool = False, scale: float = 0.0, workspace=None,
           out=None, q_positions=None, rope_theta: float = 0.0):
    """Attention of q [H*group, n_q, d] over [C_k; K] with bias [beta; 0]
    through still_attend on the current stream; returns out like q.  C_k/C_v
    [H, t, d] and K/V [H, S, d] may be None for t = 0 / S = 0; beta [H, t]
    float32 or None.  ``out`` (like q) and ``workspace`` may be given, so that
    the call allocates nothing (graph capture).  With ``q_positions`` (float64
    [n_q] device tensor of logical positions) and ``rope_theta`` the kernel
    rotates q there first."""
    torch = _torch()
    Hq, nq, d = (int(x) for x in q.shape)
    H = Hq // group
    t = int(C_k.shape[1]) if C_k is not None else 0
    S = int(K.shape[1]) if K is not None else 0
    mode = configs.MODE_FP32 if q.dtype == torch.float32 else configs.MODE_BF16
    acfg = still_attend_config(H, group, d, nq, t, S, int(causal), float(scale), mode,
                               float(rope_theta) if q_positions is not None else 0.0)
    need = still_attend_workspace_size(acfg)
    if need == 0:
        _check(lib().still_attend(ctypes.byref(acfg), *[None] * 9, 0, None))   # raises with the reason
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty_like(q)
    stream = torch.cuda.current_stream(q.device).cuda_stream
    _check(still_attend(acfg, q, q_positions, C_k, C_v, beta, K, V, out, workspace, workspace.numel(), stream))
    return out


# ----------------------------------------------------------------------------
# Paged cache
# ----------------------------------------------------------------------------

def _refuse(status: int, detail: str):
    raise StillError(status, detail)


def _want(x, name: str, dtype, shape, dev: int) -> None:
    """x is a contiguous tensor of this type and shape on GPU dev (-1: none)."""
    if x.dtype == dtype and x.shape == shape and x.is_contiguous() and x.get_device() == dev:
        return
    if x.dtype != dtype:
        _refuse(-3, f"{name} is {x.dtype}, not {dtype}")
    if x.shape != shape:
        _refuse(-2, f"{name} has shape {tuple(x.shape)}, not {tuple(shape)}")
    if x.get_device() != dev:
        _refuse(-1, f"{name} is on {x.device}, the pages on GPU {dev}")
    _refuse(-1, f"{name} is not contiguous")


def _want_rows(x, name: str, pages, shape, dtype=None) -> None:
    """x is a tensor of the pages' type (or the one given) with this shape and whole rows, on their GPU."""
    dtype = dtype or pages.dtype
    if x.dtype == dtype and x.shape == shape and x.stride(2) == 1 and x.get_device() == pages.get_device():
        return
    if x.dtype != dtype:
        _refuse(-3, f"{name} is {x.dtype}, the pages {dtype}" if dtype == pages.dtype else f"{name} is {x.dtype}, not {dtype}")
    if x.shape != shape:
        _refuse(-2, f"{name} has shape {tuple(x.shape)}, not {tuple(shape)}")
    if x.get_device() != pages.get_device():
        _refuse(-1, f"{name} is on {x.device}, the pages on {pages.device}")
    _refuse(-1, f"{name}'s rows are not contiguous")


def _refuse_paged(torch, k_pages, v_pages, beta_pages, table, lens, dtypes=None) -> None:
    """Says what is wrong with a paged cache or its sequences."""
    shape, dt, dev = k_pages.shape, k_pages.dtype, k_pages.get_device()
    if len(shape) != 4:
        _refuse(-2, f"k_pages has {len(shape)} dimensions, not [n_pages, H, page_size, d]")
    if dt not in (dtypes or (torch.bfloat16, torch.float32)):
        _refuse(-3, f"pages of {dt}: bfloat16 and float32 are supported")
    if not k_pages.is_contiguous():
        _refuse(-1, "k_pages is not contiguous")
    _want(v_pages, "v_pages", dt, shape, dev)
    if beta_pages is not None:
        _want(beta_pages, "beta_pages", torch.float32, shape[:3], dev)
    if table.dim() != 2 or table.dtype != torch.int32 or (table.stride(1) != 1 and table.shape[1] > 1):
        _refuse(-2, "table is no int32 tensor [n_seqs, pages] with contiguous rows")
    if table.shape[0] > 1 and table.stride(0) >= 1 << 31:
        _refuse(-2, f"table rows {table.stride(0)} entries apart")
    if max(table.shape) >= 1 << 31:
        _refuse(-2, f"a table of {table.shape[0]} x {table.shape[1]} entries")
    if table.get_device() != dev:
        _refuse(-1, f"table is on {table.device}, the pages on {k_pages.device}")
    _want(lens, "lens", torch.int32, table.shape[:1], dev)
    _refuse(-1, f"the pages are on {k_pages.device}: a GPU is needed")


def _paged(torch, k_pages, v_pages, beta_pages, table, lens):
    """(C view of a paged cache, C view of its sequences, GPU), checked."""
    shape, dt, dev, size = k_pages.shape, k_pages.dtype, k_pages.get_device(), table.shape
    i32, fp32 = torch.int32, dt is torch.float32
    # one expression: this runs before every call of a decode step
    if not (dev >= 0 and len(shape) == 4 and (fp32 or dt is torch.bfloat16) and v_pages.dtype is dt
            and v_pages.shape == shape and k_pages.is_contiguous() and v_pages.is_contiguous()
            and v_pages.get_device() == dev and table.dtype is i32 and len(size) == 2 and lens.dtype is i32
            and lens.shape == size[:1] and lens.is_contiguous() and lens.get_device() == dev
            and table.get_device() == dev and (table.stride(1) == 1 or size[1] <= 1) and (size[0] <= 1 or table.stride(0) < 1 << 31)
            and size[0] < 1 << 31 and size[1] < 1 << 31
            and (beta_pages is None or beta_pages.dtype is torch.float32 and beta_pages.shape == shape[:3]
                 and beta_pages.is_contiguous() and beta_pages.get_device() == dev)):
        _refuse_paged(torch, k_pages, v_pages, beta_pages, table, lens)
    n_pages, H, P, d = shape
    n, width = size
    return (still_paged_cache(H, d, P, n_pages, fp32, k_pages.data_ptr(), v_pages.data_ptr(),
                              None if beta_pages is None else beta_pages.data_ptr()),
            still_paged_seqs(n, width, table.stride(0) if n > 1 else width, table.data_ptr(), lens.data_ptr()), dev)


def _on(torch, dev: int, call, *args) -> None:
    """call(*args, current stream of GPU dev) with that GPU current; raises if it fails."""
    if torch.cuda.current_device() == dev:
        status = call(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            status = call(*args, torch._C._cuda_getCurrentRawStream(dev))
    if status != STILL_OK:
        _check(status)


def _tokens(torch, k, v, k_pages, dtype, cache, seqs, dev, offsets, positions, rope_theta, beta):
    """C view of rows k, v of this type to append, checked."""
    size = k.shape
    if len(size) != 3:
        _refuse(-2, f"k has {k.dim()} dimensions, not [n_tokens, H, d]")
    n = size[0]
    if n >= 1 << 31:
        _refuse(-2, f"{n} tokens given")
    shape = (n, cache.n_kv_heads, cache.head_dim)
    # one expression, as before every call of a decode step
    if not (size == shape and v.shape == size and k.dtype is dtype and v.dtype is dtype and k.stride(2) == 1
            and v.stride(2) == 1 and k.get_device() == dev and v.get_device() == dev):
        _want_rows(k, "k", k_pages, shape, dtype)
        _want_rows(v, "v", k_pages, shape, dtype)
    off = pos = b = None
    if offsets is not None:
        _want(offsets, "offsets", torch.int32, (seqs.n_seqs + 1,), dev)
        off = offsets.data_ptr()
    if positions is not None:
        _want(positions, "positions", torch.float64, (n,), dev)
        pos = positions.data_ptr()
    ts = hs = 0
    if beta is not None:
        if beta.dtype != torch.float32 or beta.shape != shape[:2] or beta.get_device() != dev:
            _refuse(-2, "beta is no float32 tensor [n_tokens, H] on the pages' device")
        ts, hs = beta.stride()
        b = beta.data_ptr()
    kt, kh, _ = k.stride()
    vt, vh, _ = v.stride()
    if n == 1:                       # strides of dimensions of one address nothing and may be any number
        kt = vt = 0
    if shape[1] == 1:
        kh = vh = 0
    return still_paged_tokens(n, k.data_ptr(), v.data_ptr(), kt, kh, vt, vh, b, ts, hs, off, pos, rope_theta)


def paged_append(k, v, k_pages, v_pages, table, lens, offsets=None, positions=None, rope_theta: float = 0.0,
                 beta=None, beta_pages=None) -> None:
    """Append rows k, v [n_tokens, H, d] to the pages [n_pages, H, P, d] of
    their sequences on the current stream (still_paged_append).  table
    [n_seqs, pages] and lens [n_seqs] are int32 device tensors; lens counts the
    new entries already.  Sequence s's tokens are offsets[s] .. offsets[s + 1] - 1
    (int32 [n_seqs + 1]); without offsets every sequence has n_tokens / n_seqs.
    With ``positions`` (float64 [n_tokens] logical positions) and
    ``rope_theta`` the keys are rotated there first.  k and v may be strided
    views with contiguous rows (slices of a fused projection, transposed [H, t, d]
    outputs of the compactor).  A cache that keeps bias passes ``beta_pages``
    [n_pages, H, P] float32 always, and the entries' ``beta`` [n_tokens, H]
    float32 where it is not zero."""
    torch = _torch()
    cache, seqs, dev = _paged(torch, k_pages, v_pages, beta_pages, table, lens)
    tokens = _tokens(torch, k, v, k_pages, k_pages.dtype, cache, seqs, dev, offsets, positions, rope_theta, beta)
    _on(torch, dev, (_lib or lib()).still_paged_append, ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(tokens))


def _dense(torch, k_pages, dtype, cache, dev, seq, start, n, beta_pages, out):
    """(seq, start, n, (K, V) or (K, V, beta) of this type to fill), checked."""
    seq, start, n = int(seq), int(start), int(n)
    if max(abs(seq), abs(start), abs(n)) >= 1 << 31:
        _refuse(-2, f"entries [{start}, {start + n}) of sequence {seq} asked for")
    shape = (cache.n_kv_heads, n, cache.head_dim)
    if out is None:
        if n < 0:
            _refuse(-2, f"{n} entries asked for")
        out = tuple(torch.empty(shape, dtype=dtype, device=k_pages.device) for _ in range(2))
        if beta_pages is not None:
            out += (torch.empty(shape[:2], dtype=torch.float32, device=k_pages.device),)
    elif len(out) != (2 if beta_pages is None else 3):
        _refuse(-2, "out holds K, V and, with beta_pages, beta")
    else:
        _want(out[0], "out[0]", dtype, shape, dev)
        _want(out[1], "out[1]", dtype, shape, dev)
        if beta_pages is not None:
            _want(out[2], "out[2]", torch.float32, shape[:2], dev)
    return seq, start, n, out


def paged_gather(k_pages, v_pages, table, lens, seq: int, n: int, start: int = 0, beta_pages=None, out=None):
    """Entries [start, start + n) of sequence ``seq`` as dense (K, V) [H, n, d],
    with ``beta_pages`` (K, V, beta [H, n]), through still_paged_gather on the
    current stream; into ``out`` (such a tuple) where given."""
    torch = _torch()
    cache, seqs, dev = _paged(torch, k_pages, v_pages, beta_pages, table, lens)
    seq, start, n, out = _dense(torch, k_pages, k_pages.dtype, cache, dev, seq, start, n, beta_pages, out)
    _on(torch, dev, (_lib or lib()).still_paged_gather, ctypes.byref(cache), ctypes.byref(seqs), seq, start, n,
        out[0].data_ptr(), out[1].data_ptr(), None if beta_pages is None else out[2].data_ptr())
    return out


def _queries(torch, q, k_pages, dtype, cache, seqs, dev, causal, scale, q_positions, rope_theta):
    """(C view of how the newest tokens q of this type attend, their positions' address), checked."""
    shape = q.shape
    if len(shape) != 3:
        _refuse(-2, f"q has {len(shape)} dimensions, not [n_seqs * n_queries, H * group, d]")
    tokens, Hq, d = shape
    H, n = cache.n_kv_heads, seqs.n_seqs
    if n < 1 or H < 1 or d != cache.head_dim or Hq < H or Hq % H or tokens < n or tokens % n:
        _refuse(-2, f"q {tuple(shape)} does not fit {n} sequences and pages {tuple(k_pages.shape)}")
    qs = q.stride()
    if not (q.dtype is dtype and qs[2] == 1 and q.get_device() == dev):
        _want_rows(q, "q", k_pages, shape, dtype)
    if (qs[1] != d and Hq > 1) or (qs[0] == 0 and tokens > 1):   # (a stride of 0 means dense tokens to the C call)
        _refuse(-1, "q's tokens are not contiguous, or the same one")
    pos = None
    if q_positions is not None:
        _want(q_positions, "q_positions", torch.float64, (tokens,), dev)
        pos = q_positions.data_ptr()
    return still_paged_attend_config(Hq // H, tokens // n, causal, scale, rope_theta, qs[0] if tokens > 1 else 0), pos


def _attend(torch, q, k_pages, cache, seqs, dev, causal, scale, q_positions, rope_theta, workspace, out, lse):
    """Attention over checked pages, of 8 bits or of q's type."""
    eight = type(cache) is still_paged8_cache
    cfg, pos = _queries(torch, q, k_pages, q.dtype if eight else k_pages.dtype, cache, seqs, dev, causal, scale, q_positions,
                        rope_theta)
    shape = q.shape
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=q.device)
    elif not (out.dtype is q.dtype and out.shape == shape and out.is_contiguous() and out.get_device() == dev):
        _want(out, "out", q.dtype, shape, dev)
    if lse is not None:
        _want(lse, "lse", torch.float32, shape[:2], dev)
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        _refuse(-1, f"workspace is on {workspace.device}, the pages on {k_pages.device}, or it is not contiguous")
    room = 0 if workspace is None else workspace.numel()
    if room < STILL_PAGED_WORKSPACE_BYTES:
        need = (still_paged8_attend_workspace_size if eight else still_paged_attend_workspace_size)(cache, cfg)
        if room < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            room = need
    call = (_lib or lib()).still_paged8_attend if eight else (_lib or lib()).still_paged_attend_lse
    _on(torch, dev, call, ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), q.data_ptr(), pos, out.data_ptr(),
        None if lse is None else lse.data_ptr(), _ptr(workspace), room)
    return out


def paged_attend(q, k_pages, v_pages, table, lens, causal: bool = False, scale: float = 0.0, beta_pages=None,
                 q_positions=None, rope_theta: float = 0.0, workspace=None, out=None, lse=None):
    """Attention of the newest tokens q [n_seqs * n_queries, H * group, d]
    (sequence by sequence) over their sequences' pages through
    still_paged_attend on the current stream; returns out, contiguous, like q.
    q may be a strided view with contiguous tokens.  With ``q_positions``
    (float64, one per token) and ``rope_theta`` the kernel rotates q first.
    ``out`` and ``workspace`` (STILL_PAGED_WORKSPACE_BYTES serve every call)
    may be given, so that the call allocates nothing (graph capture).  ``lse``
    (float32 [n_seqs * n_queries, H * group], contiguous) is filled with the log of each row's
    sum of exponentials, minus infinity for a row that sees nothing."""
    torch = _torch()
    cache, seqs, dev = _paged(torch, k_pages, v_pages, beta_pages, table, lens)
    return _attend(torch, q, k_pages, cache, seqs, dev, causal, scale, q_positions, rope_theta, workspace, out, lse)


# ---- pages of 8 bits

def _refuse_paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, dtype) -> None:
    """Says what is wrong with a paged cache in 8 bits or its sequences."""
    shape, dev = k_pages.shape, k_pages.get_device()
    if len(shape) != 4:
        _refuse(-2, f"k_pages has {len(shape)} dimensions, not [n_pages, H, page_size, d]")
    if k_pages.dtype != torch.float8_e4m3fn:
        _refuse(-3, f"pages of {k_pages.dtype}, not float8_e4m3fn")
    if dtype != torch.bfloat16 and dtype != torch.float32:
        _refuse(-3, f"rows of {dtype}: bfloat16 and float32 are supported")
    blocks = (shape[0], shape[1], shape[2] // 16)
    _want(v_pages, "v_pages", k_pages.dtype, shape, dev)
    _want(k_scales, "k_scales", torch.float32, blocks, dev)
    _want(v_scales, "v_scales", torch.float32, blocks, dev)
    _refuse_paged(torch, k_pages, v_pages, beta_pages, table, lens, (torch.float8_e4m3fn,))


def _paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, dtype):
    """(C view of a paged cache in 8 bits with rows of this type, C view of its sequences, GPU), checked."""
    shape, dt, dev, size = k_pages.shape, k_pages.dtype, k_pages.get_device(), table.shape
    i32, f32 = torch.int32, torch.float32
    # one expression: this runs before every call of a decode step
    if not (dev >= 0 and len(shape) == 4 and dt is torch.float8_e4m3fn and (dtype is f32 or dtype is torch.bfloat16)
            and v_pages.dtype is dt and v_pages.shape == shape and k_pages.is_contiguous() and v_pages.is_contiguous()
            and v_pages.get_device() == dev and table.dtype is i32 and len(size) == 2 and lens.dtype is i32
            and k_scales.dtype is f32 and v_scales.dtype is f32
            and k_scales.shape == v_scales.shape == (shape[0], shape[1], shape[2] >> 4)
            and k_scales.is_contiguous() and v_scales.is_contiguous()
            and k_scales.get_device() == dev and v_scales.get_device() == dev
            and lens.shape == size[:1] and lens.is_contiguous() and lens.get_device() == dev
            and table.get_device() == dev and (table.stride(1) == 1 or size[1] <= 1) and (size[0] <= 1 or table.stride(0) < 1 << 31)
            and size[0] < 1 << 31 and size[1] < 1 << 31
            and (beta_pages is None or beta_pages.dtype is f32 and beta_pages.shape == shape[:3]
                 and beta_pages.is_contiguous() and beta_pages.get_device() == dev)):
        _refuse_paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, dtype)
    n_pages, H, P, d = shape
    n, width = size
    return (still_paged8_cache(H, d, P, n_pages, dtype is f32, k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(),
                               v_scales.data_ptr(), None if beta_pages is None else beta_pages.data_ptr()),
            still_paged_seqs(n, width, table.stride(0) if n > 1 else width, table.data_ptr(), lens.data_ptr()), dev)


def paged8_append(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, offsets=None, positions=None,
                  rope_theta: float = 0.0, beta=None, beta_pages=None) -> None:
    """paged_append into pages of 8 bits (still_paged8_append): k_pages, v_pages
    [n_pages, H, P, d] float8_e4m3fn and their scales [n_pages, H, P // 16] float32, one
    for each block of 16 entries and head, which the call sets: powers of two, that grow
    with what their blocks get.  k and v [n_tokens, H, d] are bfloat16 or float32."""
    torch = _torch()
    cache, seqs, dev = _paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, k.dtype)
    tokens = _tokens(torch, k, v, k_pages, k.dtype, cache, seqs, dev, offsets, positions, rope_theta, beta)
    _on(torch, dev, (_lib or lib()).still_paged8_append, ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(tokens))


def paged8_gather(k_pages, v_pages, k_scales, v_scales, table, lens, seq: int, n: int, start: int = 0, dtype=None,
                  beta_pages=None, out=None):
    """paged_gather from pages of 8 bits (still_paged8_gather): the rows that entries
    [start, start + n) stand for, of ``dtype`` (bfloat16, or out's type)."""
    torch = _torch()
    dtype = dtype or (out[0].dtype if out else torch.bfloat16)
    cache, seqs, dev = _paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, dtype)
    seq, start, n, out = _dense(torch, k_pages, dtype, cache, dev, seq, start, n, beta_pages, out)
    _on(torch, dev, (_lib or lib()).still_paged8_gather, ctypes.byref(cache), ctypes.byref(seqs), seq, start, n,
        out[0].data_ptr(), out[1].data_ptr(), None if beta_pages is None else out[2].data_ptr())
    return out


def paged8_attend(q, k_pages, v_pages, k_scales, v_scales, table, lens, causal: bool = False, scale: float = 0.0,
                  beta_pages=None, q_positions=None, rope_theta: float = 0.0, workspace=None, out=None, lse=None):
    """paged_attend over pages of 8 bits (still_paged8_attend); q and out are
    bfloat16 or float32."""
    torch = _torch()
    cache, seqs, dev = _paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, q.dtype)
    return _attend(torch, q, k_pages, cache, seqs, dev, causal, scale, q_positions, rope_theta, workspace, out, lse)


# ---- what entries are worth, and eviction by it

def _cache(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, dtype):
    """_paged or, for pages of 8 bits, _paged8 with rows of this type."""
    if k_pages.dtype is torch.float8_e4m3fn and k_scales is not None and v_scales is not None:
        return _paged8(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, dtype)
    if k_scales is not None or v_scales is not None:
        _refuse(-1, f"scales given to pages of {k_pages.dtype}, or to keys or values alone")
    return _paged(torch, k_pages, v_pages, beta_pages, table, lens)


def paged_score(q, lse, k_pages, scores, table, lens, causal: bool = False, scale: float = 0.0, k_scales=None,
                beta_pages=None, known=None, q_positions=None, rope_theta: float = 0.0) -> None:
    """Add the attention weights of the newest tokens q, summed over the rows of each
    KV head, to the entries' scores [n_pages, H, P] float32 on the current stream
    (still_paged_score; still_paged8_score for pages of 8 bits, with ``k_scales``).
    Arguments as in paged_attend, whose ``lse`` of the same rows the call takes.
    Entries from ``known`` on (int32 [n_seqs]: the lengths at the call before) get the
    weights in place of their slots' old scores.  More than 32 rows of a KV head (a prompt's
    last tokens) go in several calls, the oldest first, with ``lens`` up to each call's last token."""
    torch = _torch()
    cache, seqs, dev = _cache(torch, k_pages, k_pages, k_scales, k_scales, beta_pages, table, lens, q.dtype)
    cfg, pos = _queries(torch, q, k_pages, k_pages.dtype if k_scales is None else q.dtype, cache, seqs, dev, causal, scale,
                        q_positions, rope_theta)
    _want(lse, "lse", torch.float32, q.shape[:2], dev)
    _want(scores, "scores", torch.float32, k_pages.shape[:3], dev)
    if known is not None:
        _want(known, "known", torch.int32, table.shape[:1], dev)
    call = (_lib or lib()).still_paged_score if k_scales is None else (_lib or lib()).still_paged8_score
    _on(torch, dev, call, ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), q.data_ptr(), pos, lse.data_ptr(),
        None if known is None else known.data_ptr(), scores.data_ptr())


def paged_evict(k_pages, v_pages, table, lens, scores, keep: int, first: int = 0, recent: int = 0, shared: bool = False,
                k_scales=None, v_scales=None, beta_pages=None, kept=None, new_lens=None, workspace=None):
    """Cut every sequence to its ``keep`` entries of largest score inside its pages, on
    the current stream (still_paged_evict; still_paged8_evict with ``k_scales`` and
    ``v_scales``): the ``first`` and the ``recent`` ones always stay.  Each KV head
    keeps entries of its own or, with ``shared``, all the same by the sum of their
    scores: then an entry still has one position, and compact_paged can take the
    sequence with ``positions[kept]``.  Returns (kept [n_seqs, H or 1, keep] int32: the entries that
    stay, rising, -1 behind them; new lengths [n_seqs] int32), into ``kept`` and
    ``new_lens`` where given; ``new_lens`` may be ``lens`` (of several layers that share it, in the
    last one's call).  The dropped entries are lost, those
    behind the new lengths too: of 8 bits, their block's scale may have changed.  ``workspace`` (96 MiB serve every
    call, none is needed for tables of up to 8192 entries) may be given too."""
    torch = _torch()
    cache, seqs, dev = _cache(torch, k_pages, v_pages, k_scales, v_scales, beta_pages, table, lens, torch.bfloat16)
    keep, first, recent = int(keep), int(first), int(recent)
    if max(abs(keep), abs(first), abs(recent)) >= 1 << 31:
        _refuse(-2, f"{keep} entries to keep, {first} first and {recent} recent ones")
    _want(scores, "scores", torch.float32, k_pages.shape[:3], dev)
    shape = (seqs.n_seqs, 1 if shared else cache.n_kv_heads, keep)
    if kept is None:
        if keep < 1:
            _refuse(-2, f"{keep} entries to keep")
        kept = torch.empty(shape, dtype=torch.int32, device=k_pages.device)
    else:
        _want(kept, "kept", torch.int32, shape, dev)
    if new_lens is None:
        new_lens = torch.empty(seqs.n_seqs, dtype=torch.int32, device=k_pages.device)
    else:
        _want(new_lens, "new_lens", torch.int32, table.shape[:1], dev)
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        _refuse(-1, f"workspace is on {workspace.device}, the pages on {k_pages.device}, or it is not contiguous")
    cfg = still_paged_evict_config(keep, first, recent, bool(shared))
    need, room = 0, 0 if workspace is None else workspace.numel() * workspace.element_size()
    if seqs.max_pages * k_pages.shape[2] > 8192:
        plain = cache if k_scales is None else still_paged_cache(cache.n_kv_heads, cache.head_dim, cache.page_size,
                                                                        cache.n_pages, cache.mode, cache.k, cache.v)
        need = still_paged_evict_workspace_size(plain, seqs, cfg)
    if room < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=k_pages.device)
        room = need
    call = (_lib or lib()).still_paged_evict if k_scales is None else (_lib or lib()).still_paged8_evict
    _on(torch, dev, call, ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(cfg), scores.data_ptr(), kept.data_ptr(),
        new_lens.data_ptr(), _ptr(workspace), room)
    return kept, new_lens


def compact_paged(cfg: configs.CompactorConfig, weights: List[Dict[str, object]], k_pages: List, v_pages: List,
                  table, lens, seq: int, n: int, positions, rope_theta: float, t: int, start: int = 0,
                  end: Optional[int] = None, w_beta: Optional[List] = None, beta_pages: Optional[List] = None,
                  beta_max: float = 0.0, mass_alpha: float = 0.0, log_x: float = 0.0, rerotate: bool = True,
                  drop_bias: bool = True, scales: Optional[List] = None):
    """Compact entries [start, end) (default: all) of sequence ``seq``, which
    holds n entries, to t inside its pages, layer by layer (lists of L layers'
    weights and pages, one table): they are read out, compacted
    (still_compact_layer, or still_compact_model_beta with ``w_beta``) and
    written back behind the preserved prefix, and the entries behind them move
    up with their bias.  ``positions`` [n] are the entries' float64 logical
    positions; lens[seq] holds n, and the pages up to the new length are there.
    Sets lens[seq] on the current stream and returns the new positions
    [n - (end - start) + t]; pages behind the new length are free.  A page that
    another sequence's table names too changes for that one as well.
    A cache that keeps bias passes ``beta_pages``; new entries without
    ``w_beta`` get bias 0.  The compactor reads keys and values only: bias that
    entries [start, end) carry (those of an earlier compaction) is not taken in
    and is lost, each counting as one entry without bias.  To keep it, start
    behind them; ``drop_bias=False`` waits for the GPU and refuses a range that
    carries any, before anything changes.
    Pages of 8 bits pass ``scales``, a (k_scales, v_scales) for each layer; the
    compactor then works in bfloat16."""
    torch = _torch()
    end = n if end is None else end
    if not (0 <= start < end <= n):
        _refuse(-1, f"subrange [{start}, {end}) outside [0, {n})")
    L = len(k_pages)
    if L < 1 or len(v_pages) != L or len(weights) != L or any(x is not None and len(x) != L for x in (w_beta, beta_pages, scales)):
        _refuse(-2, "lists of different numbers of layers")
    if scales is not None and any(x is None or len(x) != 2 for x in scales):
        _refuse(-1, "scales hold a (k_scales, v_scales) for each layer")
    if w_beta is not None and beta_pages is None:
        _refuse(-1, "w_beta given to a cache without beta")
    length = n - (end - start) + t
    if table.dim() != 2:
        _refuse(-2, f"table has {table.dim()} dimensions, not [n_seqs, pages]")
    if not 0 <= seq < table.shape[0]:
        _refuse(-2, f"sequence {seq} outside [0, {table.shape[0]})")
    for i in range(L):
        if tuple(k_pages[i].shape[1::2]) != (cfg.n_kv_heads, cfg.head_dim):
            _refuse(-2, f"layer {i}: pages {tuple(k_pages[i].shape)} for a compactor of {cfg.n_kv_heads} heads of width "
                        f"{cfg.head_dim}")
        if k_pages[i].dtype != k_pages[0].dtype:
            _refuse(-3, f"layer {i}: pages of {k_pages[i].dtype}, layer 0's of {k_pages[0].dtype}")
        if max(n, length) > table.shape[1] * k_pages[i].shape[2]:
            _refuse(-2, f"{max(n, length)} entries do not fit the sequence's {table.shape[1]} pages")
        if w_beta is not None and beta_pages[i] is None:
            _refuse(-1, f"layer {i}: w_beta given to a cache without beta")
    _want(positions, "positions", torch.float64, (n,), k_pages[0].get_device())
    def read(i, count, at, bias, out=None):
        if scales is None:
            return paged_gather(k_pages[i], v_pages[i], table, lens, seq, count, at, beta_pages=bias, out=out)
        return paged8_gather(k_pages[i], v_pages[i], *scales[i], table, lens, seq, count, at, beta_pages=bias, out=out)

    def write(i, k, v, row, to, beta, bias):
        if scales is None:
            return paged_append(k, v, k_pages[i], v_pages[i], row, to, beta=beta, beta_pages=bias)
        return paged8_append(k, v, k_pages[i], v_pages[i], *scales[i], row, to, beta=beta, beta_pages=bias)

    for i in range(L):   # (no entry read: the C call's checks, pointers among them)
        read(i, 0, 0, None if beta_pages is None else beta_pages[i])
    with torch.cuda.device(k_pages[0].device):
        return _compact_paged(cfg, weights, read, write, k_pages[0].device,
                              k_pages[0].dtype if scales is None else torch.bfloat16, L, table, lens, seq, n, positions,
                              rope_theta, t, start, end, w_beta, beta_pages, beta_max, mass_alpha, log_x, rerotate, drop_bias)


def _compact_paged(cfg, weights, read, write, dev, dtype, L, table, lens, seq, n, positions, rope_theta, t, start, end,
                   w_beta, beta_pages, beta_max, mass_alpha, log_x, rerotate, drop_bias):
    """compact_paged behind its checks, with the pages' GPU current: read(layer, n, start, bias pages, out)
    and write(layer, k, v, table, lens, beta, bias pages) as dense rows of this type."""
    torch = _torch()
    length = n - (end - start) + t
    mode = configs.MODE_FP32 if dtype == torch.float32 else configs.MODE_BF16
    row = table[seq:seq + 1]
    to = [torch.full((1,), x, dtype=torch.int32, device=dev) for x in (start + t, length)]
    inside = positions[start:end].contiguous()
    ws = torch.empty(max(still_workspace_size(make_config(cfg, mode), end - start, t, 1), 1), dtype=torch.uint8,
                     device=dev)                                     # shared by the layers (one stream)
    # every layer is compacted, and what the second loop needs allocated, before the first one's
    # pages change: a refusal, or memory that runs out, leaves them as they were
    new = []
    for i in range(L):
        K, V, *carried = read(i, end - start, start, None if drop_bias or beta_pages is None else beta_pages[i])
        if carried and bool((carried[0] != 0).any()):
            _refuse(-5, f"layer {i}: entries [{start}, {end}) carry bias, which a compaction does not take in")
        if w_beta is None:
            Ck, Cv, pq = compact_layer(cfg, weights[i], K, V, inside, rope_theta, t, rerotate=rerotate, mode=mode,
                                       workspace=ws)
            beta = None
        else:
            (Ck,), (Cv,), pq, (beta,) = compact_model_beta(cfg, [weights[i]], [K], [V], inside, rope_theta, t,
                                                           [w_beta[i]], beta_max, mass_alpha, log_x, rerotate, mode, ws)
            beta = beta.t()
        new.append((Ck.transpose(0, 1), Cv.transpose(0, 1), beta))
    now_at = torch.cat([positions[:start], pq, positions[end:]])
    rest = [torch.empty(cfg.n_kv_heads, n - end, cfg.head_dim, dtype=dtype, device=dev) for _ in range(2)]
    if beta_pages is not None:
        rest.append(torch.empty(cfg.n_kv_heads, n - end, dtype=torch.float32, device=dev))
    for i, (Ck, Cv, beta) in enumerate(new):
        bp = None if beta_pages is None else beta_pages[i]
        read(i, n - end, end, bp, rest[:2] if bp is None else rest)
        write(i, Ck, Cv, row, to[0], beta, bp)
        write(i, rest[0].transpose(0, 1), rest[1].transpose(0, 1), row, to[1], None if bp is None else rest[2].t(), bp)
    lens[seq:seq + 1].fill_(length)
    return now_at
