"""ctypes binding over libcfdetr.so (argument marshalling only).

The functions ``cfdetr_*`` mirror the C ABI declared in include/cfdetr.h one to
one and take raw device addresses.  ``Encoder`` is a small convenience wrapper
that keeps the weights on the device as torch tensors and passes their
addresses; every step of the computation runs in the library's HIP kernels.
PyTorch is used for device memory and streams only.

There is no fallback: if the shared library has not been built, importing any
entry point raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcfdetr.so")

CFDETR_OK, CFDETR_EINVAL, CFDETR_ESHAPE, CFDETR_ECAPACITY, CFDETR_ENOMEM, CFDETR_EDEVICE = range(6)
CFDETR_BF16, CFDETR_FP32 = 0, 1
CFDETR_MAX_LEVELS = 3
CFDETR_MAX_AXES = 4
KERNEL_NAMES = ["select", "plan", "embed", "gather", "layernorm", "qkv", "attention",
                "out_proj", "ffn1", "ffn2", "roi", "dec"]
CFDETR_K_COUNT = len(KERNEL_NAMES)
STATUS_NAMES = ["OK", "EINVAL", "ESHAPE", "ECAPACITY", "ENOMEM", "EDEVICE"]

EXPORTS = [
    "cfdetr_create", "cfdetr_destroy", "cfdetr_last_error", "cfdetr_workspace_bytes",
    "cfdetr_sync_status", "cfdetr_coarse_encode", "cfdetr_propose_rois", "cfdetr_select_fine",
    "cfdetr_select_fine_hard", "cfdetr_select_fine_static",
    "cfdetr_fine_encode", "cfdetr_fine_encode_padded",
    "cfdetr_multilevel_batch", "cfdetr_profile_begin", "cfdetr_profile_end",
    "cfdetr_sched_response_times", "cfdetr_sched_coarse_batch", "cfdetr_sched_fine_batches",
    "cfdetr_sched_decide", "cfdetr_decoder_attach", "cfdetr_decode", "cfdetr_merge_detections",
    "cfdetr_rotary_frequencies", "cfdetr_rotary", "cfdetr_diff_attention", "cfdetr_norm_residual",
    "cfdetr_differential_attach",
    "cfdetr_memory_attach", "cfdetr_memory_advance", "cfdetr_memory_append", "cfdetr_memory_attention",
    "cfdetr_rotary_axes_table", "cfdetr_rotary_axes",
]
POLICIES = {"C": 0, "CF": 1, "[C]F": 2, "C[F]": 3, "[C][F]": 4}
SCHED_ACTIONS = ["idle", "coarse", "fine"]


class CfdetrConfig(ctypes.Structure):
    _fields_ = [
        ("n_levels", ctypes.c_int32),
        ("patch", ctypes.c_int32 * CFDETR_MAX_LEVELS),
        ("img_h", ctypes.c_int32), ("img_w", ctypes.c_int32),
        ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
        ("n_layers", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
        ("max_batch", ctypes.c_int32), ("max_tokens_total", ctypes.c_int32),
        ("image_dtype", ctypes.c_int), ("act_dtype", ctypes.c_int),
        ("ln_eps", ctypes.c_float),
    ]


class CfdetrRoiParams(ctypes.Structure):
    _fields_ = [("tau_hi", ctypes.c_float), ("tau_lo", ctypes.c_float),
                ("scale", ctypes.c_float), ("min_side", ctypes.c_float),
                ("tier", ctypes.c_int32)]


class CfdetrWeights(ctypes.Structure):
    _fields_ = [
        ("w_embed", ctypes.c_void_p * CFDETR_MAX_LEVELS),
        ("b_embed", ctypes.c_void_p * CFDETR_MAX_LEVELS),
        ("ln1_g", ctypes.c_void_p), ("ln1_b", ctypes.c_void_p),
        ("w_qkv", ctypes.c_void_p), ("b_qkv", ctypes.c_void_p),
        ("w_o", ctypes.c_void_p), ("b_o", ctypes.c_void_p),
        ("ln2_g", ctypes.c_void_p), ("ln2_b", ctypes.c_void_p),
        ("w_ff1", ctypes.c_void_p), ("b_ff1", ctypes.c_void_p),
        ("w_ff2", ctypes.c_void_p), ("b_ff2", ctypes.c_void_p),
        ("lnf_g", ctypes.c_void_p), ("lnf_b", ctypes.c_void_p),
    ]


DECODER_MATRICES = ("w_qkv", "w_o", "w_q", "w_kv", "w_o2", "w_ff1", "w_ff2", "w_cls", "w_box1",
                    "w_box2", "w_box3")
DECODER_FIELDS = ("query_embed", "ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b",
                  "w_q", "b_q", "w_kv", "b_kv", "w_o2", "b_o2", "ln3_g", "ln3_b", "w_ff1", "b_ff1",
                  "w_ff2", "b_ff2", "lnf_g", "lnf_b", "w_cls", "b_cls", "w_box1", "b_box1",
                  "w_box2", "b_box2", "w_box3", "b_box3")


class CfdetrDecoderWeights(ctypes.Structure):
    _fields_ = ([("n_queries", ctypes.c_int32), ("n_layers", ctypes.c_int32)]
                + [(name, ctypes.c_void_p) for name in DECODER_FIELDS])


NORMS = {"none": 0, "layer": 1, "rms": 2}


class CfdetrRotaryParams(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("base", ctypes.c_double), ("factor", ctypes.c_double), ("trained_len", ctypes.c_double),
                ("keep_turns", ctypes.c_double), ("stretch_turns", ctypes.c_double)]


class CfdetrNormResidualParams(ctypes.Structure):
    _fields_ = [("post", ctypes.c_int), ("pre", ctypes.c_int),
                ("post_g", ctypes.c_void_p), ("post_b", ctypes.c_void_p),
                ("pre_g", ctypes.c_void_p), ("pre_b", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("cu_seqlens", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("res_scale", ctypes.c_float)]


DIFFERENTIAL_FIELDS = ("lambda", "head_g", "post1_g", "post2_g", "gate1", "gate2")


class CfdetrDifferentialWeights(ctypes.Structure):
    _fields_ = ([(name, ctypes.c_void_p) for name in DIFFERENTIAL_FIELDS]
                + [("res_scale", ctypes.c_float), ("rotary", CfdetrRotaryParams)])


class CfdetrMemoryConfig(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("page_size", "n_pages", "max_pages", "max_streams", "n_kv_heads")]


class CfdetrRotaryAxesParams(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("pairs", ctypes.c_int32 * CFDETR_MAX_AXES),
                ("in_turn", ctypes.c_int32), ("shared_ladder", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("base", ctypes.c_double)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libcfdetr.so and declare the prototypes.  Raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2505_23317_amd.build); "
            "there is no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    lib.cfdetr_create.argtypes = [ctypes.POINTER(CfdetrConfig), ctypes.POINTER(CfdetrWeights),
                                  ctypes.POINTER(vp)]
    lib.cfdetr_create.restype = ctypes.c_int
    lib.cfdetr_destroy.argtypes = [vp]
    lib.cfdetr_destroy.restype = None
    lib.cfdetr_last_error.argtypes = [vp]
    lib.cfdetr_last_error.restype = ctypes.c_char_p
    lib.cfdetr_workspace_bytes.argtypes = [vp]
    lib.cfdetr_workspace_bytes.restype = ctypes.c_uint64
    lib.cfdetr_sync_status.argtypes = [vp, vp]
    lib.cfdetr_sync_status.restype = ctypes.c_int
    lib.cfdetr_coarse_encode.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.cfdetr_coarse_encode.restype = ctypes.c_int
    lib.cfdetr_propose_rois.argtypes = [vp, vp, i32, i32, ctypes.POINTER(CfdetrRoiParams), i32,
                                        vp, vp, vp, vp, vp, vp]
    lib.cfdetr_propose_rois.restype = ctypes.c_int
    lib.cfdetr_select_fine.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp]
    lib.cfdetr_select_fine.restype = ctypes.c_int
    lib.cfdetr_select_fine_hard.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
    lib.cfdetr_select_fine_hard.restype = ctypes.c_int
    lib.cfdetr_select_fine_static.argtypes = [ctypes.POINTER(CfdetrConfig), vp, vp, vp, i32, vp, vp,
                                              vp, vp, vp]
    lib.cfdetr_select_fine_static.restype = ctypes.c_int
    lib.cfdetr_fine_encode.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
    lib.cfdetr_fine_encode.restype = ctypes.c_int
    lib.cfdetr_fine_encode_padded.argtypes = [vp, vp, i32, vp, vp, vp, i32, vp, vp]
    lib.cfdetr_fine_encode_padded.restype = ctypes.c_int
    lib.cfdetr_multilevel_batch.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.cfdetr_multilevel_batch.restype = ctypes.c_int
    dp, ip = ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)
    dbl = ctypes.c_double
    lib.cfdetr_sched_response_times.argtypes = [i32, dp, dp, dp, ip]
    lib.cfdetr_sched_response_times.restype = ctypes.c_int
    lib.cfdetr_sched_coarse_batch.argtypes = [i32, dbl, dbl, dp]
    lib.cfdetr_sched_coarse_batch.restype = i32
    lib.cfdetr_sched_fine_batches.argtypes = [i32, ip, dp, dbl, dbl, dp, i32, i32, ip, ip, ip, dp]
    lib.cfdetr_sched_fine_batches.restype = ctypes.c_int
    lib.cfdetr_sched_decide.argtypes = [ctypes.c_int, dbl, i32, ip, i32, ip, ip, dp, dbl, dp, dp,
                                        i32, i32, ip, ip, ip, ip]
    lib.cfdetr_sched_decide.restype = ctypes.c_int
    lib.cfdetr_merge_detections.argtypes = [vp, vp, vp, vp, i32, i32, ctypes.c_float, ctypes.c_float,
                                            vp, vp, vp, vp]
    lib.cfdetr_merge_detections.restype = ctypes.c_int
    lib.cfdetr_decoder_attach.argtypes = [vp, ctypes.POINTER(CfdetrDecoderWeights)]
    lib.cfdetr_decoder_attach.restype = ctypes.c_int
    lib.cfdetr_decode.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.cfdetr_decode.restype = ctypes.c_int
    rot, f32 = ctypes.POINTER(CfdetrRotaryParams), ctypes.c_float
    lib.cfdetr_rotary_frequencies.argtypes = [rot, dp]
    lib.cfdetr_rotary_frequencies.restype = ctypes.c_int
    lib.cfdetr_rotary.argtypes = [vp, rot, vp, vp, i32, vp, i32, vp, i32, f32, vp, i32, vp, i32, vp]
    lib.cfdetr_rotary.restype = ctypes.c_int
    lib.cfdetr_diff_attention.argtypes = [vp, vp, i32, i32, vp, i32, vp, i32, i32, vp, vp, i32, vp, vp, vp,
                                          f32, vp, i32, vp]
    lib.cfdetr_diff_attention.restype = ctypes.c_int
    lib.cfdetr_norm_residual.argtypes = [vp, ctypes.POINTER(CfdetrNormResidualParams), vp, vp, vp, vp, i32, vp]
    lib.cfdetr_norm_residual.restype = ctypes.c_int
    lib.cfdetr_differential_attach.argtypes = [vp, ctypes.POINTER(CfdetrDifferentialWeights)]
    lib.cfdetr_differential_attach.restype = ctypes.c_int
    axes = ctypes.POINTER(CfdetrRotaryAxesParams)
    lib.cfdetr_memory_attach.argtypes = [vp, ctypes.POINTER(CfdetrMemoryConfig)]
    lib.cfdetr_memory_attach.restype = ctypes.c_int
    lib.cfdetr_memory_advance.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.cfdetr_memory_advance.restype = ctypes.c_int
    lib.cfdetr_rotary_axes_table.argtypes = [axes, dp, ctypes.POINTER(ctypes.c_uint8)]
    lib.cfdetr_rotary_axes_table.restype = ctypes.c_int
    lib.cfdetr_rotary_axes.argtypes = [vp, axes, vp, vp, vp, i32, vp, i32, vp, i32, f32, vp, i32, vp, i32, i32, vp]
    lib.cfdetr_rotary_axes.restype = ctypes.c_int
    lib.cfdetr_memory_append.argtypes = [vp, axes, vp, vp, vp, i32, vp, i32, vp, i32, vp, vp, i32, vp, i32, vp]
    lib.cfdetr_memory_append.restype = ctypes.c_int
    lib.cfdetr_memory_attention.argtypes = [vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, f32, vp, i32, vp]
    lib.cfdetr_memory_attention.restype = ctypes.c_int
    lib.cfdetr_profile_begin.argtypes = [vp]
    lib.cfdetr_profile_begin.restype = ctypes.c_int
    lib.cfdetr_profile_end.argtypes = [vp, ctypes.POINTER(ctypes.c_float),
                                       ctypes.POINTER(ctypes.c_int32)]
    lib.cfdetr_profile_end.restype = ctypes.c_int
    _lib = lib
    return lib


class CfdetrError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"cfdetr status {STATUS_NAMES[status] if 0 <= status < 6 else status}"
                         f": {message}")
        self.status = status


def _check(status: int, ctx=None):
    if status != CFDETR_OK:
        raw = load_library().cfdetr_last_error(ctx)
        msg = raw.decode() if raw else ""
        raise CfdetrError(status, msg)


# ---- one-to-one wrappers (raw addresses in, status checked) -----------------
def cfdetr_create(cfg: CfdetrConfig, weights: CfdetrWeights) -> int:
    out = ctypes.c_void_p()
    _check(load_library().cfdetr_create(ctypes.byref(cfg), ctypes.byref(weights),
                                        ctypes.byref(out)))
    return out.value


def cfdetr_destroy(ctx: int) -> None:
    load_library().cfdetr_destroy(ctx)


def cfdetr_last_error(ctx: int) -> str:
    raw = load_library().cfdetr_last_error(ctx)
    return raw.decode() if raw else ""


def cfdetr_workspace_bytes(ctx: int) -> int:
    return int(load_library().cfdetr_workspace_bytes(ctx))


def cfdetr_sync_status(ctx: int, stream: int = 0) -> None:
    _check(load_library().cfdetr_sync_status(ctx, stream), ctx)


def cfdetr_coarse_encode(ctx, images, B, x0_cache, y_coarse, stream=0) -> None:
    _check(load_library().cfdetr_coarse_encode(ctx, images, B, x0_cache, y_coarse, stream), ctx)


def cfdetr_propose_rois(ctx, queries, B, Q, params: CfdetrRoiParams, max_boxes, boxes, tier,
                        box_offsets, hard, mean_conf, stream=0) -> None:
    _check(load_library().cfdetr_propose_rois(ctx, queries, B, Q, ctypes.byref(params), max_boxes,
                                              boxes, tier, box_offsets, hard, mean_conf, stream),
           ctx)


def cfdetr_merge_detections(ctx, coarse, fine, hard, B, Q, tau_hi, tau_fine, det, src, count,
                            stream=0) -> None:
    _check(load_library().cfdetr_merge_detections(ctx, coarse, fine, hard, B, Q, tau_hi, tau_fine,
                                                  det, src, count, stream), ctx)


def cfdetr_decoder_attach(ctx, weights: CfdetrDecoderWeights) -> None:
    _check(load_library().cfdetr_decoder_attach(ctx, ctypes.byref(weights)), ctx)


def cfdetr_decode(ctx, memory, cu_seqlens, B, queries, stream=0) -> None:
    _check(load_library().cfdetr_decode(ctx, memory, cu_seqlens, B, queries, stream), ctx)


def cfdetr_select_fine(ctx, boxes, tier, box_offsets, B, tok_desc, cu_seqlens, level_counts,
                       stream=0) -> None:
    _check(load_library().cfdetr_select_fine(ctx, boxes, tier, box_offsets, B, tok_desc,
                                             cu_seqlens, level_counts, stream), ctx)


def cfdetr_select_fine_hard(ctx, boxes, tier, box_offsets, hard, B, tok_desc, cu_seqlens,
                            level_counts, stream=0) -> None:
    _check(load_library().cfdetr_select_fine_hard(ctx, boxes, tier, box_offsets, hard, B, tok_desc,
                                                  cu_seqlens, level_counts, stream), ctx)


def cfdetr_select_fine_static(cfg: CfdetrConfig, boxes, tier, box_offsets, B, tok_desc, cu_seqlens,
                              level_counts, overflow, stream=0) -> None:
    _check(load_library().cfdetr_select_fine_static(ctypes.byref(cfg), boxes, tier, box_offsets, B,
                                                    tok_desc, cu_seqlens, level_counts, overflow,
                                                    stream), None)


def cfdetr_fine_encode(ctx, images, B, tok_desc, cu_seqlens, x0_cache, y_mixed, stream=0) -> None:
    _check(load_library().cfdetr_fine_encode(ctx, images, B, tok_desc, cu_seqlens, x0_cache,
                                             y_mixed, stream), ctx)


def cfdetr_fine_encode_padded(ctx, images, B, tok_desc, cu_seqlens, x0_cache, t_pad, y_padded,
                              stream=0) -> None:
    _check(load_library().cfdetr_fine_encode_padded(ctx, images, B, tok_desc, cu_seqlens, x0_cache,
                                                    t_pad, y_padded, stream), ctx)


def cfdetr_multilevel_batch(ctx, images, B, boxes, tier, box_offsets, y_coarse, y_mixed,
                            tok_desc, cu_seqlens, level_counts, stream=0) -> None:
    _check(load_library().cfdetr_multilevel_batch(ctx, images, B, boxes, tier, box_offsets,
                                                  y_coarse, y_mixed, tok_desc, cu_seqlens,
                                                  level_counts, stream), ctx)


# ---- scheduling decisions (host data; lists in, lists out) ---------------------
def _darr(v):
    return (ctypes.c_double * max(len(v), 1))(*[float(x) for x in v])


def _iarr(v):
    return (ctypes.c_int32 * max(len(v), 1))(*[int(x) for x in v])


def _fine_table(c_fine):
    """[[level][size]] -> flat row-major table, n_levels, max_size."""
    n_levels, max_size = len(c_fine), len(c_fine[0]) - 1
    flat = [float(x) for row in c_fine for x in row]
    return _darr(flat), n_levels, max_size


def cfdetr_sched_response_times(period, c_coarse):
    n = len(period)
    R = (ctypes.c_double * n)()
    ok = ctypes.c_int32()
    _check(load_library().cfdetr_sched_response_times(n, _darr(period), _darr(c_coarse), R,
                                                      ctypes.byref(ok)))
    return bool(ok.value), list(R)


def cfdetr_sched_coarse_batch(n_active, t, next_release, c_batch_by_size) -> int:
    return int(load_library().cfdetr_sched_coarse_batch(n_active, t, next_release,
                                                        _darr(c_batch_by_size)))


def cfdetr_sched_fine_batches(workload, deadline, t, next_coarse_release, c_fine):
    """Returns (order, cuts, dba) like the paper's tables: cuts are half-open ranges."""
    n = len(workload)
    tab, n_levels, max_size = _fine_table(c_fine)
    order, ends = (ctypes.c_int32 * max(n, 1))(), (ctypes.c_int32 * max(n, 1))()
    nb = ctypes.c_int32()
    dba = (ctypes.c_double * (n + 1))()
    _check(load_library().cfdetr_sched_fine_batches(n, _iarr(workload), _darr(deadline), t,
                                                    next_coarse_release, tab, n_levels, max_size,
                                                    order, ends, ctypes.byref(nb), dba))
    cuts, a = [], 0
    for b in range(nb.value):
        cuts.append((a, ends[b]))
        a = ends[b]
    return list(order)[:n], cuts, list(dba)


def cfdetr_sched_decide(policy: str, t, active_coarse, active_fine, fine_workload, fine_deadline,
                        next_release, c_coarse_by_size, c_fine):
    """Returns (kind, tasks): ("coarse", [tasks]) | ("fine", [[batch], ...]) | ("idle", [])."""
    tab, n_levels, max_size = _fine_table(c_fine)
    m = max(len(active_coarse), len(active_fine), 1)
    kind, nb = ctypes.c_int32(), ctypes.c_int32()
    tasks, ends = (ctypes.c_int32 * m)(), (ctypes.c_int32 * m)()
    _check(load_library().cfdetr_sched_decide(
        POLICIES[policy], t, len(active_coarse), _iarr(active_coarse), len(active_fine),
        _iarr(active_fine), _iarr(fine_workload), _darr(fine_deadline), next_release,
        _darr(c_coarse_by_size), tab, n_levels, max_size, ctypes.byref(kind), tasks, ends,
        ctypes.byref(nb)))
    name = SCHED_ACTIONS[kind.value]
    if name == "coarse":
        return name, list(tasks)[:ends[0]]
    if name == "fine":
        out, a = [], 0
        for b in range(nb.value):
            out.append(list(tasks)[a:ends[b]])
            a = ends[b]
        return name, out
    return name, []


def rotary_params(rot_dim: int, n_axes: int = 2, interleaved: bool = False, base: float = 10000.0,
                  factor: float = 1.0, trained_len: float = 0.0, keep_turns: float = 32.0,
                  stretch_turns: float = 1.0) -> CfdetrRotaryParams:
    return CfdetrRotaryParams(rot_dim, n_axes, int(interleaved), base, factor, trained_len, keep_turns,
                              stretch_turns)


def cfdetr_rotary_frequencies(params: CfdetrRotaryParams):
    """The rot_dim / 2 frequencies as a list (host)."""
    # (a bad rot_dim is refused before anything is written)
    freq = (ctypes.c_double * max(1, params.rot_dim // 2))()
    _check(load_library().cfdetr_rotary_frequencies(ctypes.byref(params), freq))
    return list(freq)


def cfdetr_rotary(ctx, params: CfdetrRotaryParams, freq, pos, M, q, q_ld, q_out, q_out_ld, q_scale, k, k_ld,
                  k_out, k_out_ld, stream=0) -> None:
    _check(load_library().cfdetr_rotary(ctx, ctypes.byref(params), freq, pos, M, q, q_ld, q_out, q_out_ld,
                                        q_scale, k, k_ld, k_out, k_out_ld, stream), ctx)


def cfdetr_diff_attention(ctx, q, q_ld, n_q, k, k_ld, v, v_ld, n_k, cu_q, cu_k, B, key_mask, lambda_, head_g,
                          softmax_scale, out, out_ld, stream=0) -> None:
    _check(load_library().cfdetr_diff_attention(ctx, q, q_ld, n_q, k, k_ld, v, v_ld, n_k, cu_q, cu_k, B,
                                                key_mask, lambda_, head_g, softmax_scale, out, out_ld,
                                                stream), ctx)


def norm_residual_params(post="none", pre="none", post_g=None, post_b=None, pre_g=None, pre_b=None, gate=None,
                         cu_seqlens=None, res_scale=1.0) -> CfdetrNormResidualParams:
    """post, pre: "none", "layer" or "rms"; the vectors are float32 device tensors (cu_seqlens int32), which
    the structure keeps alive."""
    p = CfdetrNormResidualParams(NORMS[post], NORMS[pre])
    p.tensors = dict(post_g=post_g, post_b=post_b, pre_g=pre_g, pre_b=pre_b, gate=gate, cu_seqlens=cu_seqlens)
    for name, t in p.tensors.items():
        if t is not None:
            _expect(t, "int32" if name == "cu_seqlens" else "float32", name)
            setattr(p, name, t.data_ptr())
    p.B = int(cu_seqlens.shape[0]) - 1 if cu_seqlens is not None else 0
    p.res_scale = res_scale
    p.checked = None   # columns and GPU that Encoder.norm_residual has found the tensors to have
    return p


def cfdetr_norm_residual(ctx, params: CfdetrNormResidualParams, x, block, x_out, normed, M, stream=0) -> None:
    _check(load_library().cfdetr_norm_residual(ctx, ctypes.byref(params), x, block, x_out, normed, M, stream),
           ctx)


def cfdetr_differential_attach(ctx, weights: CfdetrDifferentialWeights) -> None:
    _check(load_library().cfdetr_differential_attach(ctx, ctypes.byref(weights)), ctx)


def cfdetr_memory_attach(ctx, cfg: CfdetrMemoryConfig) -> None:
    _check(load_library().cfdetr_memory_attach(ctx, ctypes.byref(cfg)), ctx)


def cfdetr_memory_advance(ctx, B, drop, cu_new, n_new, span, span_out, table, table_out, pool, pool_out, free_pages,
                          slots, stream=0) -> None:
    _check(load_library().cfdetr_memory_advance(ctx, B, drop, cu_new, n_new, span, span_out, table, table_out, pool,
                                                pool_out, free_pages, slots, stream), ctx)


def rotary_axes_params(rot_dim: int, pairs, in_turn: bool = False, shared_ladder: bool = False, interleaved: bool = False,
                       base: float = 10000.0) -> CfdetrRotaryAxesParams:
    """pairs: how many of the rot_dim / 2 pairs each axis has."""
    if not 1 <= len(pairs) <= CFDETR_MAX_AXES:
        raise ValueError(f"pairs: 1 to {CFDETR_MAX_AXES} axes expected")
    return CfdetrRotaryAxesParams(rot_dim, len(pairs), (ctypes.c_int32 * CFDETR_MAX_AXES)(*pairs), int(in_turn),
                                  int(shared_ladder), int(interleaved), base)


def cfdetr_rotary_axes_table(params: CfdetrRotaryAxesParams):
    """Frequency and axis of the rot_dim / 2 pairs, as two lists (host)."""
    # (a bad rot_dim is refused before anything is written)
    n = max(1, params.rot_dim // 2)
    freq, axis = (ctypes.c_double * n)(), (ctypes.c_uint8 * n)()
    _check(load_library().cfdetr_rotary_axes_table(ctypes.byref(params), freq, axis))
    return list(freq), list(axis)


def cfdetr_rotary_axes(ctx, params: CfdetrRotaryAxesParams, freq, axis, pos, M, q, q_ld, q_out, q_out_ld, q_scale, k,
                       k_ld, k_out, k_out_ld, k_heads, stream=0) -> None:
    _check(load_library().cfdetr_rotary_axes(ctx, ctypes.byref(params), freq, axis, pos, M, q, q_ld, q_out, q_out_ld,
                                             q_scale, k, k_ld, k_out, k_out_ld, k_heads, stream), ctx)


def cfdetr_memory_append(ctx, params: Optional[CfdetrRotaryAxesParams], freq, axis, pos, M, k, k_ld, v, v_ld, slots,
                         k_cache, k_cache_ld, v_cache, v_cache_ld, stream=0) -> None:
    _check(load_library().cfdetr_memory_append(ctx, None if params is None else ctypes.byref(params), freq, axis, pos,
                                               M, k, k_ld, v, v_ld, slots, k_cache, k_cache_ld, v_cache, v_cache_ld,
                                               stream), ctx)


def cfdetr_memory_attention(ctx, q, q_ld, B, k_cache, k_cache_ld, v_cache, v_cache_ld, span, table, key_mask,
                            softmax_scale, out, out_ld, stream=0) -> None:
    _check(load_library().cfdetr_memory_attention(ctx, q, q_ld, B, k_cache, k_cache_ld, v_cache, v_cache_ld, span,
                                                  table, key_mask, softmax_scale, out, out_ld, stream), ctx)


def cfdetr_profile_begin(ctx) -> None:
    _check(load_library().cfdetr_profile_begin(ctx), ctx)


def cfdetr_profile_end(ctx) -> Dict[str, Dict[str, float]]:
    ms = (ctypes.c_float * CFDETR_K_COUNT)()
    n = (ctypes.c_int32 * CFDETR_K_COUNT)()
    _check(load_library().cfdetr_profile_end(ctx, ms, n), ctx)
    return {KERNEL_NAMES[k]: {"ms": float(ms[k]), "launches": int(n[k])}
            for k in range(CFDETR_K_COUNT)}


# ---- convenience wrapper ------------------------------------------------------
def _to_device(arr: np.ndarray, as_bf16: bool):
    """numpy float32 -> torch tensor on cuda:0 (bf16 bit patterns or fp32)."""
    import torch
    from . import synth
    if as_bf16:
        bits = synth.bf16_bits(arr).view(np.int16)
        return torch.from_numpy(bits).view(torch.bfloat16).reshape(arr.shape).cuda()
    return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).cuda()


_DTYPES: Dict[str, object] = {}


def _expect(t, dtype: str, what: str, shape=None, gpu=None) -> None:
    """A tensor that the library takes as it lies: contiguous, on the GPU (number `gpu`, if given), of the named type and shape."""
    if not _DTYPES:
        import torch
        _DTYPES.update({n: getattr(torch, n) for n in ("float64", "float32", "bfloat16", "int32", "uint8")})
    on = t.get_device()   # (-1: not on a GPU)
    if (t.dtype is not _DTYPES[dtype] or (shape is not None and t.shape != shape) or not t.is_contiguous() or on < 0
            or (gpu is not None and on != gpu)):
        raise ValueError(f"{what}: contiguous {dtype} on the GPU expected"
                         + (f", shape {tuple(shape)}" if shape is not None else ""))


def _ptr(t):
    return None if t is None else t.data_ptr()


def unpack_tok_desc(desc: np.ndarray) -> np.ndarray:
    """int32 descriptors -> [T,3] (level,row,col)."""
    d = np.asarray(desc).astype(np.int64)
    return np.stack([(d >> 28) & 7, (d >> 14) & 0x3FFF, d & 0x3FFF], axis=1)


class Encoder:
    """Device-resident weights + one library context for one model shape.

    ``cfg`` is a synth.Config (or anything with the same fields); ``weights`` a
    dict of float32 numpy arrays laid out as include/cfdetr.h describes.
    """

    def __init__(self, cfg, weights: Dict[str, np.ndarray], act_dtype: str = "bf16",
                 max_batch: Optional[int] = None, max_tokens_total: Optional[int] = None):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("cfdetr needs a GPU: no CPU fallback exists")
        self.cfg = cfg
        self.act_bf16 = act_dtype == "bf16"
        self.max_batch = max_batch or cfg.B
        top = cfg.n_levels - 1
        self.max_tokens = max_tokens_total or self.max_batch * cfg.n_cells(top)
        self.n0 = cfg.n_cells(0)
        mats = {"w_qkv", "w_o", "w_ff1", "w_ff2"} | {f"w_embed{l}" for l in range(cfg.n_levels)}
        self.dev = {k: _to_device(v, self.act_bf16 and k in mats) for k, v in weights.items()}
        c = CfdetrConfig()
        c.n_levels = cfg.n_levels
        for l in range(CFDETR_MAX_LEVELS):
            c.patch[l] = cfg.patch[l] if l < cfg.n_levels else 0
        c.img_h, c.img_w = cfg.H, cfg.W
        c.d_model, c.n_heads, c.n_layers, c.d_ffn = cfg.d, cfg.heads, cfg.layers, cfg.ffn
        c.max_batch, c.max_tokens_total = self.max_batch, self.max_tokens
        c.image_dtype = CFDETR_BF16 if cfg.image_dtype == "bf16" else CFDETR_FP32
        c.act_dtype = CFDETR_BF16 if self.act_bf16 else CFDETR_FP32
        c.ln_eps = 1e-5
        w = CfdetrWeights()
        for l in range(cfg.n_levels):
            w.w_embed[l] = self.dev[f"w_embed{l}"].data_ptr()
            w.b_embed[l] = self.dev[f"b_embed{l}"].data_ptr()
        for name in ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b",
                     "w_ff1", "b_ff1", "w_ff2", "b_ff2", "lnf_g", "lnf_b"):
            setattr(w, name, self.dev[name].data_ptr())
        self.c_cfg, self.c_w = c, w
        self.act = torch.bfloat16 if self.act_bf16 else torch.float32
        self.gpu = self.dev["lnf_g"].get_device()   # number of the context's GPU
        self.ctx = cfdetr_create(c, w)

    # -- helpers ---------------------------------------------------------------
    def upload_images(self, images: np.ndarray):
        return _to_device(images, self.cfg.image_dtype == "bf16")

    @staticmethod
    def upload_boxes(boxes, tier, box_offsets):
        import torch
        b = torch.from_numpy(np.ascontiguousarray(boxes, dtype=np.int32).reshape(-1, 4)).cuda()
        t = torch.from_numpy(np.ascontiguousarray(tier, dtype=np.uint8)).cuda()
        o = torch.from_numpy(np.ascontiguousarray(box_offsets, dtype=np.int32)).cuda()
        if b.numel() == 0:      # keep a valid address for an empty table
            b = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
            t = torch.zeros(1, dtype=torch.uint8, device="cuda")
        return b, t, o

    @staticmethod
    def _stream() -> int:
        """Address of the current device's current stream.  torch.cuda.current_stream() makes a Python object of it,
        2.7 us a call, a third of what the smallest call (a selection) took; asked for as a number it is 0.25 us.  It also
        refuses to in a child that was forked from a process that uses the GPU, so such a child goes that way still (the
        tensors of a call have initialised the GPU otherwise)."""
        import torch
        c = torch._C
        if c._cuda_isInBadFork():
            return torch.cuda.current_stream().cuda_stream
        return c._cuda_getCurrentRawStream(c._cuda_getDevice())

    def alloc_outputs(self, B: int):
        import torch
        d = self.cfg.d
        return {
            "x0_cache": torch.empty((B * self.n0, d), dtype=torch.float32, device="cuda"),
            "y_coarse": torch.empty((B * self.n0, d), dtype=torch.float32, device="cuda"),
            "y_mixed": torch.zeros((self.max_tokens, d), dtype=torch.float32, device="cuda"),
            "tok_desc": torch.zeros(self.max_tokens, dtype=torch.int32, device="cuda"),
            "cu_seqlens": torch.zeros(B + 1, dtype=torch.int32, device="cuda"),
            "level_counts": torch.zeros((B, self.cfg.n_levels), dtype=torch.int32, device="cuda"),
        }

    # -- the four calls ----------------------------------------------------------
    def coarse_encode(self, images, B, x0_cache, y_coarse):
        cfdetr_coarse_encode(self.ctx, images.data_ptr(), B,
                             x0_cache.data_ptr() if x0_cache is not None else None,
                             y_coarse.data_ptr(), self._stream())

    def propose_rois(self, queries, params: CfdetrRoiParams, boxes, tier, box_offsets, hard,
                     mean_conf):
        """queries: float32 device tensor [B, Q, 5]; the other tensors are outputs."""
        B, Q = int(queries.shape[0]), int(queries.shape[1])
        cfdetr_propose_rois(self.ctx, queries.data_ptr(), B, Q, params, int(boxes.shape[0]),
                            boxes.data_ptr(), tier.data_ptr(), box_offsets.data_ptr(),
                            hard.data_ptr(), mean_conf.data_ptr(), self._stream())

    def merge_detections(self, coarse, fine, hard, tau_hi, tau_fine, det, src, count):
        """coarse, fine: float32 device tensors [B, Q, 5]; det [B, 2Q, 5], src [B, 2Q] uint8 and
        count [B] int32 are outputs."""
        B, Q = int(coarse.shape[0]), int(coarse.shape[1])
        cfdetr_merge_detections(self.ctx, coarse.data_ptr(), fine.data_ptr(), hard.data_ptr(), B, Q,
                                tau_hi, tau_fine, det.data_ptr(), src.data_ptr(), count.data_ptr(),
                                self._stream())

    def attach_decoder(self, weights: Dict[str, np.ndarray]):
        """weights: float32 numpy arrays named as include/cfdetr.h lists them; uploaded here
        (matrices as bf16 bit patterns) and kept alive with the context."""
        self.dec_dev = {k: _to_device(v, k in DECODER_MATRICES) for k, v in weights.items()}
        w = CfdetrDecoderWeights()
        w.n_queries = int(weights["query_embed"].shape[0])
        w.n_layers = int(weights["w_qkv"].shape[0])
        for name in DECODER_FIELDS:
            setattr(w, name, self.dec_dev[name].data_ptr())
        self.n_queries = w.n_queries
        self.c_dec = w
        cfdetr_decoder_attach(self.ctx, w)

    def decode(self, memory, cu_seqlens, B, queries):
        """memory: float32 device tensor [T, d]; queries: float32 device tensor [B, Q, 5] out."""
        cfdetr_decode(self.ctx, memory.data_ptr(), cu_seqlens.data_ptr(), B, queries.data_ptr(),
                      self._stream())

    def select_fine(self, boxes, tier, box_offsets, B, tok_desc, cu_seqlens, level_counts=None):
        cfdetr_select_fine(self.ctx, boxes.data_ptr(), tier.data_ptr(), box_offsets.data_ptr(), B,
                           tok_desc.data_ptr(), cu_seqlens.data_ptr(),
                           level_counts.data_ptr() if level_counts is not None else None,
                           self._stream())

    def select_fine_hard(self, boxes, tier, box_offsets, hard, B, tok_desc, cu_seqlens,
                         level_counts=None):
        cfdetr_select_fine_hard(self.ctx, boxes.data_ptr(), tier.data_ptr(), box_offsets.data_ptr(),
                                hard.data_ptr(), B, tok_desc.data_ptr(), cu_seqlens.data_ptr(),
                                level_counts.data_ptr() if level_counts is not None else None,
                                self._stream())

    def select_fine_static(self, boxes, tier, box_offsets, B, tok_desc, cu_seqlens, level_counts,
                           overflow):
        """The selection through the entry point that allocates nothing and uses no context
        (the configuration structure of this encoder is passed instead)."""
        cfdetr_select_fine_static(self.c_cfg, boxes.data_ptr(), tier.data_ptr(),
                                  box_offsets.data_ptr(), B, tok_desc.data_ptr(),
                                  cu_seqlens.data_ptr(),
                                  level_counts.data_ptr() if level_counts is not None else None,
                                  overflow.data_ptr(), self._stream())

    def fine_encode(self, images, B, tok_desc, cu_seqlens, x0_cache, y_mixed):
        cfdetr_fine_encode(self.ctx, images.data_ptr(), B, tok_desc.data_ptr(),
                           cu_seqlens.data_ptr(),
                           x0_cache.data_ptr() if x0_cache is not None else None,
                           y_mixed.data_ptr(), self._stream())

    def fine_encode_padded(self, images, B, tok_desc, cu_seqlens, x0_cache, t_pad, y_padded):
        cfdetr_fine_encode_padded(self.ctx, images.data_ptr(), B, tok_desc.data_ptr(),
                                  cu_seqlens.data_ptr(),
                                  x0_cache.data_ptr() if x0_cache is not None else None,
                                  t_pad, y_padded.data_ptr(), self._stream())

    def multilevel_batch(self, images, B, boxes, tier, box_offsets, out):
        cfdetr_multilevel_batch(self.ctx, images.data_ptr(), B, boxes.data_ptr(), tier.data_ptr(),
                                box_offsets.data_ptr(), out["y_coarse"].data_ptr(),
                                out["y_mixed"].data_ptr(), out["tok_desc"].data_ptr(),
                                out["cu_seqlens"].data_ptr(), out["level_counts"].data_ptr(),
                                self._stream())

    # -- operators of a differential layer, on the caller's rows -------------------------
    def _rows(self, t, shape, what: str) -> int:
        """Elements from row to row of a tensor [rows, d] in act_dtype whose rows are contiguous.  (Every field of a tensor
        is asked for once: the checks of a rotation take 3 us of its 6.9, the library's call 3.8.)"""
        if t.dtype is not self.act or t.shape != shape or t.get_device() != self.gpu:
            raise ValueError(f"{what}: rows {tuple(shape)} of {self.act} on the context's GPU expected")
        step, one = t.stride()
        if one != 1:
            raise ValueError(f"{what}: the elements of a row must lie next to each other")
        return step if shape[0] > 1 else shape[1]

    def rotary(self, params: CfdetrRotaryParams, freq, pos, q, q_out, k=None, k_out=None, q_scale=1.0):
        """freq: float64 [rot_dim / 2], pos: float32 [M, n_axes]; q, k and the outputs: [M, d] in act_dtype,
        rows may lie apart (columns of a wider tensor)."""
        shape = (q.shape[0], self.cfg.d)
        M = shape[0]
        _expect(freq, "float64", "freq", (params.rot_dim // 2,), self.gpu)
        _expect(pos, "float32", "pos", (M, params.n_axes), self.gpu)
        rows = self._rows
        q_ld, qo_ld, k_ld, ko_ld = rows(q, shape, "q"), rows(q_out, shape, "q_out"), 0, 0
        if k is not None or k_out is not None:
            if k is None or k_out is None:
                raise ValueError("k and k_out go together")
            k_ld, ko_ld = rows(k, shape, "k"), rows(k_out, shape, "k_out")
            k, k_out = k.data_ptr(), k_out.data_ptr()
        cfdetr_rotary(self.ctx, params, freq.data_ptr(), pos.data_ptr(), M, q.data_ptr(), q_ld, q_out.data_ptr(),
                      qo_ld, q_scale, k, k_ld, k_out, ko_ld, self._stream())

    def diff_attention(self, q, k, v, cu_q, cu_k, lambda_, out, head_g=None, key_mask=None, softmax_scale=None):
        """q, out: [n_q, d]; k, v: [n_k, d]; cu_q, cu_k: int32 [B + 1]; lambda_: float32 [n_heads / 2]; head_g:
        float32 [2 d_head] or None; key_mask: uint8 [n_k] or None.  softmax_scale: None for 1 / sqrt(d_head), 0 for
        queries that have been multiplied by log2(e) / sqrt(d_head)."""
        n_q, n_k, B, rows, d = q.shape[0], k.shape[0], cu_q.shape[0] - 1, self._rows, self.cfg.d
        _expect(cu_q, "int32", "cu_q", (B + 1,), self.gpu)
        _expect(cu_k, "int32", "cu_k", (B + 1,), self.gpu)
        _expect(lambda_, "float32", "lambda_", (self.cfg.heads // 2,), self.gpu)
        if head_g is not None:
            _expect(head_g, "float32", "head_g", (2 * self.cfg.d_head,), self.gpu)
        if key_mask is not None:
            _expect(key_mask, "uint8", "key_mask", (n_k,), self.gpu)
        if softmax_scale is None:
            softmax_scale = self.cfg.d_head ** -0.5
        cfdetr_diff_attention(self.ctx, q.data_ptr(), rows(q, (n_q, d), "q"), n_q, k.data_ptr(),
                              rows(k, (n_k, d), "k"), v.data_ptr(), rows(v, (n_k, d), "v"), n_k, cu_q.data_ptr(),
                              cu_k.data_ptr(), B, _ptr(key_mask), lambda_.data_ptr(), _ptr(head_g), softmax_scale,
                              out.data_ptr(), rows(out, (n_q, d), "out"), self._stream())

    def norm_residual(self, params: CfdetrNormResidualParams, x, block, x_out, normed=None):
        """x, x_out: float32 [M, d]; block, normed: [M, d] in act_dtype, contiguous."""
        M, d, act = x.shape[0], self.cfg.d, "bfloat16" if self.act_bf16 else "float32"
        if params.checked != (d, self.gpu):
            for name, t in params.tensors.items():
                if t is not None and name != "cu_seqlens" and t.numel() != (params.B * d if name == "gate" and params.B else d):
                    raise ValueError(f"{name}: {d} columns expected, and a row for every frame of cu_seqlens in the gate")
                if t is not None and t.get_device() != self.gpu:
                    raise ValueError(f"{name}: not on the context's GPU")
            params.checked = (d, self.gpu)
        shape = (M, d)
        _expect(x, "float32", "x", shape, self.gpu)
        _expect(block, act, "block", shape, self.gpu)
        _expect(x_out, "float32", "x_out", shape, self.gpu)
        if normed is not None:
            _expect(normed, act, "normed", shape, self.gpu)
        cfdetr_norm_residual(self.ctx, params, x.data_ptr(), block.data_ptr(), x_out.data_ptr(), _ptr(normed), M,
                             self._stream())

    def attach_differential(self, weights: Dict[str, np.ndarray], rotary: CfdetrRotaryParams, res_scale: float = 1.0):
        """weights: float32 numpy arrays named as include/cfdetr.h lists them ("lambda", and any of "head_g",
        "post1_g", "post2_g", "gate1", "gate2"); uploaded here and kept alive with the context."""
        cfg = self.cfg
        widths = dict.fromkeys(DIFFERENTIAL_FIELDS, cfg.d)
        widths.update({"lambda": cfg.heads // 2, "head_g": 2 * cfg.d_head})
        for name, v in weights.items():
            if name not in widths or v.shape != (cfg.layers, widths[name]):
                raise ValueError(f"{name}: one of {DIFFERENTIAL_FIELDS} expected, a row of its width for every layer")
        dev = {k: _to_device(v, False) for k, v in weights.items()}
        w = CfdetrDifferentialWeights()
        for name, t in dev.items():
            setattr(w, name, t.data_ptr())
        w.res_scale, w.rotary = res_scale, rotary
        cfdetr_differential_attach(self.ctx, w)
        self.diff_dev, self.c_diff = dev, w

    # -- memory of streams -----------------------------------------------------------------
    def attach_memory(self, page_size: int, n_pages: int, max_pages: int, max_streams: int,
                      n_kv_heads: Optional[int] = None):
        """n_kv_heads: key heads, a divisor of the context's heads; None for as many."""
        mem = CfdetrMemoryConfig(page_size, n_pages, max_pages, max_streams, self.cfg.heads if n_kv_heads is None else n_kv_heads)
        cfdetr_memory_attach(self.ctx, mem)
        self.mem, self.kv_dim, self.n_slots = mem, mem.n_kv_heads * self.cfg.d_head, n_pages * page_size

    def alloc_memory(self, B: int):
        """A state of B streams that hold nothing yet, and a cache for the keys and values of one layer."""
        import torch
        m, dev = self._memory(), f"cuda:{self.gpu}"
        return {
            "span": torch.zeros((B, 2), dtype=torch.int32, device=dev),
            "table": torch.zeros((B, m.max_pages), dtype=torch.int32, device=dev),
            "pool": torch.tensor([0, m.n_pages], dtype=torch.int32, device=dev),
            "free_pages": torch.arange(m.n_pages, dtype=torch.int32, device=dev),
            "k_cache": torch.zeros((self.n_slots, self.kv_dim), dtype=self.act, device=dev),
            "v_cache": torch.zeros((self.n_slots, self.kv_dim), dtype=self.act, device=dev),
        }

    def _memory(self) -> CfdetrMemoryConfig:
        mem = getattr(self, "mem", None)
        if mem is None:
            raise ValueError("no memory attached")
        return mem

    def memory_advance(self, cu_new, span, table, pool, free_pages, slots, drop=None, span_out=None, table_out=None,
                       pool_out=None):
        """cu_new: int32 [B + 1]; span: int32 [B, 2]; table: int32 [B, max_pages]; pool: int32 [2]; free_pages: int32
        [n_pages]; slots: int32 [n_new] out; drop: int32 [B] or None.  The outputs are the inputs where they are not given."""
        import torch
        m, gpu, i32 = self._memory(), self.gpu, torch.int32
        B, n_new = span.shape[0], slots.shape[0]
        wide, rows = (B, 2), (B, m.max_pages)
        checks = [(cu_new, (B + 1,), "cu_new"), (slots, (n_new,), "slots"), (free_pages, (m.n_pages,), "free_pages"), (span, wide, "span"),
                  (table, rows, "table"), (pool, (2,), "pool")]
        for t, shape, what in ((drop, (B,), "drop"), (span_out, wide, "span_out"), (table_out, rows, "table_out"), (pool_out, (2,), "pool_out")):
            if t is not None:
                checks.append((t, shape, what))
        for t, shape, what in checks:
            # (what _expect asks for, without a call for each of ten tensors: 8.4 us a step with them)
            if t.dtype is not i32 or t.shape != shape or t.get_device() != gpu or not t.is_contiguous():
                _expect(t, "int32", what, shape, gpu)
        cfdetr_memory_advance(self.ctx, B, _ptr(drop), cu_new.data_ptr(), n_new, span.data_ptr(), (span if span_out is None else span_out).data_ptr(),
                              table.data_ptr(), (table if table_out is None else table_out).data_ptr(), pool.data_ptr(),
                              (pool if pool_out is None else pool_out).data_ptr(), free_pages.data_ptr(), slots.data_ptr(), self._stream())

    def rotary_axes(self, params: CfdetrRotaryAxesParams, freq, axis, pos, q, q_out, k=None, k_out=None, q_scale=1.0):
        """freq: float64, axis: uint8 [rot_dim / 2]; pos: float32 [M, n_axes]; q and q_out: [M, d], k and k_out: [M, key
        heads * d_head] in act_dtype, rows may lie apart (columns of a wider tensor)."""
        shape = (q.shape[0], self.cfg.d)
        M = shape[0]
        self._expect_axes(params, freq, axis, pos, M)
        rows = self._rows
        q_ld, qo_ld, k_ld, ko_ld, k_heads = rows(q, shape, "q"), rows(q_out, shape, "q_out"), 0, 0, 0
        if k is not None or k_out is not None:
            if k is None or k_out is None:
                raise ValueError("k and k_out go together")
            shape = (M, k.shape[1])
            k_heads, rest = divmod(shape[1], self.cfg.d_head)
            if rest:
                raise ValueError("k: whole heads expected")
            k_ld, ko_ld = rows(k, shape, "k"), rows(k_out, shape, "k_out")
            k, k_out = k.data_ptr(), k_out.data_ptr()
        cfdetr_rotary_axes(self.ctx, params, freq.data_ptr(), axis.data_ptr(), pos.data_ptr(), M, q.data_ptr(), q_ld,
                           q_out.data_ptr(), qo_ld, q_scale, k, k_ld, k_out, ko_ld, k_heads, self._stream())

    def _expect_axes(self, params, freq, axis, pos, M):
        n = params.rot_dim // 2
        _expect(freq, "float64", "freq", (n,), self.gpu)
        _expect(axis, "uint8", "axis", (n,), self.gpu)
        _expect(pos, "float32", "pos", (M, params.n_axes), self.gpu)

    def memory_append(self, k, v, slots, k_cache, v_cache, params: Optional[CfdetrRotaryAxesParams] = None, freq=None,
                      axis=None, pos=None):
        """k, v: [M, n_kv_heads * d_head] in act_dtype, caches [n_pages * page_size, n_kv_heads * d_head], rows may lie apart;
        slots: int32 [M].  params: the keys are turned by freq, axis and pos (as for rotary_axes); None: they are not."""
        self._memory()
        M, shape, cache, rows = k.shape[0], (k.shape[0], self.kv_dim), (self.n_slots, self.kv_dim), self._rows
        _expect(slots, "int32", "slots", (M,), self.gpu)
        if params is not None:
            self._expect_axes(params, freq, axis, pos, M)
            freq, axis, pos = freq.data_ptr(), axis.data_ptr(), pos.data_ptr()
        elif freq is not None or axis is not None or pos is not None:
            raise ValueError("freq, axis and pos go with params")
        cfdetr_memory_append(self.ctx, params, freq, axis, pos, M, k.data_ptr(), rows(k, shape, "k"), v.data_ptr(),
                             rows(v, shape, "v"), slots.data_ptr(), k_cache.data_ptr(), rows(k_cache, cache, "k_cache"),
                             v_cache.data_ptr(), rows(v_cache, cache, "v_cache"), self._stream())

    def memory_attention(self, q, k_cache, v_cache, span, table, out, key_mask=None, softmax_scale=None):
        """q, out: [B, d]; caches [n_pages * page_size, n_kv_heads * d_head]; span: int32 [B, 2]; table: int32 [B, max_pages];
        key_mask: uint8 [n_pages * page_size] or None.  softmax_scale: None for 1 / sqrt(d_head), 0 for queries that have
        been multiplied by log2(e) / sqrt(d_head)."""
        m = self._memory()
        B, cache, rows = q.shape[0], (self.n_slots, self.kv_dim), self._rows
        shape = (B, self.cfg.d)
        _expect(span, "int32", "span", (B, 2), self.gpu)
        _expect(table, "int32", "table", (B, m.max_pages), self.gpu)
        if key_mask is not None:
            _expect(key_mask, "uint8", "key_mask", (self.n_slots,), self.gpu)
        if softmax_scale is None:
            softmax_scale = self.cfg.d_head ** -0.5
        cfdetr_memory_attention(self.ctx, q.data_ptr(), rows(q, shape, "q"), B, k_cache.data_ptr(),
                                rows(k_cache, cache, "k_cache"), v_cache.data_ptr(), rows(v_cache, cache, "v_cache"),
                                span.data_ptr(), table.data_ptr(), _ptr(key_mask), softmax_scale, out.data_ptr(),
                                rows(out, shape, "out"), self._stream())

    def sync_status(self):
        cfdetr_sync_status(self.ctx, self._stream())

    def close(self):
        if getattr(self, "ctx", None):
            cfdetr_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
