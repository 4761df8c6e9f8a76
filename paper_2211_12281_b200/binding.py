"""ctypes binding of ``libkge.so``: argument marshalling only.

Every function of ``include/kge.h`` is reachable as ``lib().<name>``; the ``Kge`` class wraps
a handle and converts torch tensors to device pointers.  There is no fallback of any kind:
if the shared library is missing or cannot be loaded, importing the symbols raises
``KgeError`` -- nothing here computes on the CPU.
"""
from __future__ import annotations

import bisect
import ctypes as C
import numbers
import struct
from pathlib import Path

_PKG = Path(__file__).resolve().parent

TRANSE, TRANSH, ROTATE, DISTMULT, COMPLEX, ROTATE_REAL_L1 = range(6)
LOSS_LOGSIGMOID, LOSS_SAMPLED_SOFTMAX = range(2)
OPT_SGD, OPT_ADAM, OPT_ROWWISE_ADAGRAD = range(3)
PREC_FP32, PREC_BF16_TC = range(2)
SCORE_NAMES = {"transe": TRANSE, "transh": TRANSH, "rotate": ROTATE, "distmult": DISTMULT, "complex": COMPLEX,
               "rotate_real_l1": ROTATE_REAL_L1}
LOSS_NAMES = {"logsigmoid": LOSS_LOGSIGMOID, "softmax": LOSS_SAMPLED_SOFTMAX}
OPT_NAMES = {"sgd": OPT_SGD, "adam": OPT_ADAM, "adagrad": OPT_ROWWISE_ADAGRAD}

TAPS = dict(Q=0, FPOS=1, G=2, GRAD_ENT=3, GRAD_REL=4, GRAD_RELW=5, ENT_UNIQ=6, ENT_SEG=7, ENT_PERM=8,
            REL_UNIQ=9, REL_SEG=10, REL_PERM=11, LROW=12, BATCH=13, GRAPH_H=14, GRAPH_R=15, GRAPH_T=16,
            GRAPH_OFF=17, GRAPH_WCUM=18)
_INT_TAPS = {"ENT_UNIQ", "ENT_SEG", "ENT_PERM", "REL_UNIQ", "REL_SEG", "REL_PERM", "BATCH", "GRAPH_H", "GRAPH_R", "GRAPH_T"}
_I64_TAPS = {"GRAPH_OFF": "int64", "GRAPH_WCUM": "uint64"}

KGE_ERR_NO_EXTENSION = -10


class KgeError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: error {code}" + (f" ({detail})" if detail else ""))


class KgeConfig(C.Structure):
    """Mirror of ``kge_config``."""
    _fields_ = [
        ("num_entities", C.c_int64), ("num_relations", C.c_int64),
        ("dim", C.c_int32), ("score", C.c_int32), ("p_norm", C.c_int32), ("loss", C.c_int32),
        ("opt", C.c_int32), ("prec", C.c_int32),
        ("batch", C.c_int32), ("num_neg", C.c_int32), ("num_parts", C.c_int32),
        ("head_part", C.c_int32), ("sample_mode", C.c_int32), ("contract", C.c_int32),
        ("gamma", C.c_float), ("adv_temp", C.c_float), ("ce_correction", C.c_float), ("loss_scale", C.c_float),
        ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
        ("seed", C.c_uint64),
        ("reg_lambda", C.c_float), ("reg_form", C.c_int32), ("feat_dim", C.c_int32), ("feat_shared", C.c_int32),
    ]

    @classmethod
    def make(cls, *, num_entities, num_relations, dim, score, p_norm=1, loss="logsigmoid", opt="sgd",
             prec=PREC_FP32, batch=1, num_neg=1, num_parts=1, head_part=-1, sample_mode=0,
             gamma=0.0, adv_temp=0.0, ce_correction=0.0, loss_scale=1.0, lr=0.1,
             beta1=0.9, beta2=0.999, eps=None, seed=0, reg_lambda=0.0, reg_form=0, feat_dim=0, feat_shared=0, contract=0) -> "KgeConfig":
        score = SCORE_NAMES[score] if isinstance(score, str) else int(score)
        loss = LOSS_NAMES[loss] if isinstance(loss, str) else int(loss)
        opt = OPT_NAMES[opt] if isinstance(opt, str) else int(opt)
        if eps is None:
            eps = 1e-10 if opt == OPT_ROWWISE_ADAGRAD else 1e-8
        return cls(num_entities, num_relations, dim, score, p_norm, loss, opt, prec, batch, num_neg,
                   num_parts, head_part, sample_mode, contract, gamma, adv_temp, ce_correction, loss_scale,
                   lr, beta1, beta2, eps, seed, reg_lambda, reg_form, feat_dim, feat_shared)


# kge_norm_block and kge_norm_grads, packed (a ctypes structure takes five times as long to fill, a microsecond of a call of nine)
KGE_NORM_BLOCK = struct.Struct("8Q3q4i")      # x, y, gate, post_weight, post_bias, scale, pre_weight, pre_bias; ldx, ldy, ld_gate; x_type, block_type, gate_act, layer
KGE_NORM_GRADS = struct.Struct("8Q3q")        # dx, dy, dgate, dpost_weight, dpost_bias, dscale, dpre_weight, dpre_bias; ld_dx, ld_dy, ld_dgate


class KgeAdamwTensor(C.Structure):
    """Mirror of ``kge_adamw_tensor``."""
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("copy", C.c_void_p), ("n", C.c_int64), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32),
                ("weight_decay", C.c_float)]


def library_path() -> Path:
    return _PKG / "libkge.so"


_LIB = None
_i32p, _f32p, _vp = C.POINTER(C.c_int32), C.POINTER(C.c_float), C.c_void_p

# name -> (restype, argtypes); one entry per declaration of include/kge.h
SIGNATURES = {
    "kge_create": (C.c_int, [C.POINTER(KgeConfig), C.POINTER(_vp)]),
    "kge_destroy": (None, [_vp]),
    "kge_workspace_bytes": (C.c_size_t, [_vp, C.c_int64, C.c_int32, C.c_int32]),
    "kge_bind": (C.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_size_t, C.c_int64, C.c_int32, C.c_int32, _vp]),
    "kge_bind_features": (C.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "kge_bind_features_fp8": (C.c_int, [_vp, _vp, C.c_int32, C.c_int64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "kge_graph_load": (C.c_int, [_vp, _vp, _vp, _vp, C.c_int64, _vp]),
    "kge_graph_load_device": (C.c_int, [_vp, _vp, _vp, _vp, C.c_int64, _vp]),
    "kge_init_tables": (C.c_int, [_vp, C.c_float, _vp]),
    "kge_debug_init_words": (C.c_int, [_vp, _vp, C.c_int64, C.c_int32, C.c_uint32, _vp]),
    "kge_sample_batch": (C.c_int, [_vp, C.c_uint64, _vp, _vp, _vp, _vp, _vp]),
    "kge_train_step": (C.c_int, [_vp, C.c_uint64, C.c_float, _vp, _vp, _vp, _vp, _vp, _vp]),
    "kge_gather_rows": (C.c_int, [_vp, _vp, C.c_int32, C.c_int64, _vp, _vp]),
    "kge_train_gradients": (C.c_int, [_vp, C.c_uint64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "kge_gradient_rows": (C.c_int, [_vp, C.POINTER(_vp), C.POINTER(_vp), C.POINTER(_vp)]),
    "kge_apply_scratch_bytes": (C.c_size_t, [_vp, C.c_int32, C.c_int32]),
    "kge_apply_gradients": (C.c_int, [_vp, C.c_int32, _vp, _vp, C.c_int32, C.c_uint64, C.c_float, _vp, C.c_size_t, _vp]),
    "kge_train_step_host": (C.c_int, [_vp, C.c_uint64, C.c_float, _vp, _vp, _vp, _vp, _vp, _vp]),
    "kge_score_all_topk": (C.c_int, [_vp, _vp, _vp, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp, _vp]),
    "kge_score_all_topk_static": (C.c_int, [C.POINTER(KgeConfig), _vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int32, _vp, _vp, _vp,
                                            _vp, _vp]),
    "kge_score_all_topk_host": (C.c_int, [_vp, _vp, _vp, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp, _vp]),
    "kge_refresh_inference_table": (C.c_int, [_vp, _vp]),
    "kge_shard_query_vectors": (C.c_int, [_vp, _vp, _vp, C.c_int32, C.c_int64, _vp, _vp]),
    "kge_shard_true_scores": (C.c_int, [_vp, _vp, _vp, _vp, C.c_int32, C.c_int64, _vp, _vp]),
    "kge_shard_score_topk": (C.c_int, [_vp, _vp, _vp, C.c_int32, C.c_int32, _vp, _vp, C.c_int64, _vp, _vp, _vp, _vp]),
    "kge_merge_topk": (C.c_int, [_vp, _vp, C.c_int32, C.c_int32, C.c_int32, _vp, _vp, _vp]),
    "kge_measure_alu": (C.c_int, [C.c_int32, C.c_int32, C.POINTER(C.c_double), _vp]),
    "kge_eval_mrr": (C.c_int, [_vp, _vp, _vp, _vp, C.c_int32, C.c_int32, C.POINTER(C.c_double), _vp]),
    "kge_mrr_from_ranks": (C.c_int, [_vp, _vp, C.c_int32, C.c_int32, C.POINTER(C.c_double), _vp]),
    "kge_debug_capture_scores": (C.c_int, [_vp, _vp]),
    "kge_debug_set_wait_limit": (C.c_int, [_vp, C.c_int32]),
    "kge_debug_wait_probe": (C.c_int, [_vp, _vp]),
    "kge_debug_set_product_wait_limit": (C.c_int, [C.c_int32]),
    "kge_lr_linear_decay": (C.c_float, [C.c_float, C.c_uint64, C.c_uint64]),
    "kge_ensemble_rank_scores": (C.c_int, [C.c_double, C.c_int32, _vp]),
    "kge_ensemble_topk": (C.c_int, [_vp, C.c_int32, C.c_int32, C.c_int32, _vp, C.c_int32, _vp, _vp, _vp]),
    "kge_embedding_lookup": (C.c_int, [_vp, C.c_int32, C.c_int64, C.c_int32, C.c_int64, _vp, C.c_int32, C.c_float, C.c_int32, _vp, C.c_int32,
                                       C.c_int64, _vp, _vp]),
    "kge_embedding_grad_scratch_bytes": (C.c_size_t, [C.c_int64, C.c_int32, C.c_int32]),
    "kge_embedding_grad": (C.c_int, [_vp, C.c_int32, _vp, C.c_int32, C.c_int64, C.c_float, C.c_int32, C.c_int32, _vp, C.c_int32, C.c_int64,
                                     C.c_int32, C.c_int64, _vp, C.c_size_t, _vp, _vp]),
    "kge_dropout": (C.c_int, [_vp, C.c_int32, _vp, _vp, C.c_int32, C.c_int64, C.c_double, C.c_uint64, C.c_uint64, _vp, C.c_int32, _vp]),
    "kge_fp8_quantize": (C.c_int, [_vp, C.c_int32, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32, _vp, C.c_int64, _vp, _vp,
                                   C.c_int64, _vp, _vp]),
    "kge_fp8_matmul": (C.c_int, [_vp, C.c_int32, C.c_int64, _vp, C.c_int32, _vp, C.c_int32, C.c_int64, _vp, C.c_int32, _vp, C.c_int64, _vp,
                                 C.c_int32, C.c_int64, C.c_int64, C.c_int64, C.c_int64, _vp, _vp]),
    "kge_int8_quantize": (C.c_int, [_vp, C.c_int32, C.c_int64, C.c_int64, C.c_int64, _vp, C.c_int64, _vp, _vp]),
    "kge_int8_matmul": (C.c_int, [_vp, C.c_int64, _vp, _vp, C.c_int64, _vp, _vp, C.c_int64, _vp, C.c_int32, C.c_int64, C.c_int64, C.c_int64, C.c_int64, _vp, _vp]),
    "kge_block_norm": (C.c_int, [_vp, C.c_int64, C.c_int32, _vp, C.c_int64, _vp, C.c_int32, C.c_int64, _vp, C.c_float, _vp, _vp]),
    "kge_block_norm_grad_scratch_bytes": (C.c_size_t, [C.c_int64, C.c_int32]),
    "kge_block_norm_grad": (C.c_int, [_vp, C.c_int64, C.c_int32, _vp, _vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int32,
                                      _vp, C.c_size_t, _vp]),
    "kge_adamw": (C.c_int, [_vp, C.c_int32, C.c_int32, C.c_double, C.c_double, C.c_double, C.c_double, C.c_double, C.c_uint64, _vp, _vp, _vp, C.c_uint64, _vp]),
    "kge_get_status": (C.c_int, [_vp, _vp]),
    "kge_launch_count": (C.c_int64, [_vp]),
    "kge_profile": (C.c_int, [_vp, C.c_int]),
    "kge_profile_read": (C.c_int, [_vp, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.c_int]),
    "kge_error_string": (C.c_char_p, [C.c_int]),
    "kge_last_cuda_error": (C.c_char_p, [_vp]),
    "kge_debug_bytes": (C.c_size_t, [_vp, C.c_int, _vp]),
    "kge_debug_export": (C.c_int, [_vp, C.c_int, _vp, C.c_size_t, _vp]),
}


def lib() -> C.CDLL:
    """The loaded shared library; raises KgeError(KGE_ERR_NO_EXTENSION) if it is not built."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not path.exists():
            raise KgeError(KGE_ERR_NO_EXTENSION, "load", f"{path} is missing: run `python -m paper_2211_12281_b200.build`")
        try:
            handle = C.CDLL(str(path))
        except OSError as exc:
            raise KgeError(KGE_ERR_NO_EXTENSION, "load", str(exc)) from exc
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _LIB = handle
    return _LIB


def _ptr(t):
    """Device (or pinned host) pointer of a torch tensor / numpy array, or NULL."""
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        assert t.is_contiguous()
        return C.c_void_p(t.data_ptr())
    assert t.flags.c_contiguous
    return C.c_void_p(t.ctypes.data)


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def score_all_topk_static(cfg: KgeConfig, ent, rel, relw, q_heads, q_rels, k, true_tails, out_ids, out_scores,
                          out_ranks=None) -> int:
    """kge_score_all_topk_static: full-entity top-k without a handle, a workspace or any
    allocation (at most 64 queries, k <= 32, dim <= 512).  Returns the C status code."""
    return int(lib().kge_score_all_topk_static(C.byref(cfg), _ptr(ent), _ptr(rel), _ptr(relw), _ptr(q_heads),
                                               _ptr(q_rels), q_heads.numel(), k, _ptr(true_tails), _ptr(out_ids),
                                               _ptr(out_scores), _ptr(out_ranks), _stream()))


def measure_alu(mix: int, iters: int = 4096) -> float:
    """kge_measure_alu: lane instructions per second of instruction mix `mix` on the current GPU."""
    out = C.c_double(0.0)
    rc = int(lib().kge_measure_alu(mix, iters, C.byref(out), _stream()))
    if rc != 0:
        raise KgeError(rc, "kge_measure_alu", lib().kge_error_string(rc).decode())
    return out.value


def merge_topk(cand_ids, cand_scores, k, out_ids, out_scores) -> int:
    """kge_merge_topk on device tensors: cand_* [nq, per_query] -> out_* [nq, k]."""
    nq, per_query = cand_ids.shape
    return int(lib().kge_merge_topk(_ptr(cand_ids), _ptr(cand_scores), nq, per_query, k, _ptr(out_ids), _ptr(out_scores), _stream()))


def ensemble_rank_scores(power: float, k_list: int):
    """kge_ensemble_rank_scores: the table of Eq. 2's rank scores as a numpy float64 array [k_list + 1]."""
    import numpy as np
    table = np.empty(k_list + 1, dtype=np.float64)
    rc = int(lib().kge_ensemble_rank_scores(power, k_list, _ptr(table)))
    if rc != 0:
        raise KgeError(rc, "kge_ensemble_rank_scores", lib().kge_error_string(rc).decode())
    return table


def ensemble_topk(lists, table, top_n, out_ids, out_scores=None) -> int:
    """kge_ensemble_topk on device tensors: lists int32 [M, nq, K], table float64 [K + 1]."""
    m, nq, k = lists.shape
    return int(lib().kge_ensemble_topk(_ptr(lists), m, nq, k, _ptr(table), top_n, _ptr(out_ids), _ptr(out_scores), _stream()))


# ---- operators on rows: no handle, every tensor on one device ----
# (The smallest of these calls take a few microseconds on the GPU: what is looked at here is looked at once and without detours.)

KGE_ERR_BAD_ARG = -1
_FLOAT, _FP8 = {}, {}      # torch dtype -> kge_dtype_t, filled on first use: importing this module does not import torch
_torch = _raw_stream = None


def _load_torch():
    global _torch, _raw_stream
    import torch
    _FLOAT.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    _FP8.update({torch.float8_e4m3fn: 3, torch.float8_e5m2: 4})
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _torch = torch


def _bad(where, what):
    return KgeError(KGE_ERR_BAD_ARG, where, what)


def _type_of(t, where, name, table):
    if _torch is None:
        _load_torch()
    code = table.get(t.dtype)
    if code is None:
        raise _bad(where, f"{name} has type {t.dtype}")
    return code


def _matrix(t, where, name):
    """(rows, columns, distance of rows) of a 2-dimensional tensor: its rows may lie apart, the elements of a row may not."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1) or (stride[0] < shape[1] and shape[0] > 1):
        raise _bad(where, f"{name} is not a matrix of contiguous rows")
    return shape[0], shape[1], stride[0] if stride[0] > shape[1] else shape[1]


def _ids_of(ids, where):
    if _torch is None:
        _load_torch()
    if ids.dtype is not _torch.int32 or ids.dim() != 1 or not ids.is_contiguous():
        raise _bad(where, "ids is not a contiguous int32 list")
    return _int32(ids.numel(), where, "number of ids")


def _int32(v, where, name):
    if not -1 << 31 <= v < 1 << 31:
        raise _bad(where, f"{name} {v} is not a 32-bit number")
    return v


def _status_word(status, where):
    if status is None:
        return None
    if status.dtype is not _torch.int32 or status.numel() < 1:
        raise _bad(where, "status is not an int32 tensor")
    return status.data_ptr()


def _device_of(where, *tensors):
    """The ordinal of the GPU that all of the tensors (None: not given) are on."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and (t.get_device() != dev or dev < 0):
            raise _bad(where, "tensors are not on one GPU")
    return dev


def _call(where, fn, dev, *args):
    """Calls the entry point on the current stream of device `dev` and raises on an error code."""
    if _torch.cuda.current_device() == dev:
        rc = fn(*args, _raw_stream(dev))
    else:
        with _torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc != 0:
        raise KgeError(rc, where, lib().kge_error_string(rc).decode())


def _addr(t):
    return None if t is None else t.data_ptr()


def _scratch(scratch, need, dev, where):
    """(address, bytes, tensor) of at least `need` bytes at a multiple of 256: the caller's tensor, or a new one of torch's allocator,
    which hands it on only to what follows on the same stream (and keeps a captured graph's to that graph)."""
    if need == 0:
        return None, 0, None
    if scratch is None:
        scratch = _torch.empty(need + 256, dtype=_torch.uint8, device=dev)
    elif scratch.get_device() != dev or not scratch.is_contiguous():
        raise _bad(where, "scratch is not a contiguous tensor of the operands' device")
    at = scratch.data_ptr()
    off = -at % 256
    return at + off, max(0, scratch.numel() * scratch.element_size() - off), scratch


def embedding_lookup(table, ids, out, scale=1.0, padding_id=-1, status=None):
    """kge_embedding_lookup: out[i] = scale * table[ids[i]]; table [E, d], ids int32 [n], out [n, d] (float32, bfloat16, float16)."""
    w = "kge_embedding_lookup"
    n = _ids_of(ids, w)
    tt, to = _type_of(table, w, "table", _FLOAT), _type_of(out, w, "out", _FLOAT)
    (rows, dim, lt), (out_rows, out_dim, lo) = _matrix(table, w, "table"), _matrix(out, w, "out")
    if out_rows != n or out_dim != dim:
        raise _bad(w, "out is not [number of ids, width of table]")
    dev = _device_of(w, table, ids, out, status)
    _call(w, lib().kge_embedding_lookup, dev, table.data_ptr(), tt, rows, _int32(dim, w, "width"), lt, ids.data_ptr(), n, scale,
          _int32(padding_id, w, "padding_id"), out.data_ptr(), to, lo,
          _status_word(status, w))


def embedding_grad_scratch_bytes(rows, dim, n) -> int:
    """Bytes of scratch an embedding_grad of n ids into a table of `rows` rows needs (a tensor of 256 more is always enough)."""
    w = "kge_embedding_grad_scratch_bytes"
    return int(lib().kge_embedding_grad_scratch_bytes(_int32(rows, w, "rows"), _int32(dim, w, "width"), _int32(n, w, "number of ids")))


def embedding_grad(ids, grads, table_grad, scale=1.0, padding_id=-1, accumulate=False, scratch=None, status=None):
    """kge_embedding_grad: table_grad[e] (+)= scale * sum of grads[i] over ids[i] = e; grads [n, d], table_grad [E, d]."""
    w = "kge_embedding_grad"
    n = _ids_of(ids, w)
    tg, tt = _type_of(grads, w, "grads", _FLOAT), _type_of(table_grad, w, "table_grad", _FLOAT)
    (grad_rows, grad_dim, lg), (rows, dim, lt) = _matrix(grads, w, "grads"), _matrix(table_grad, w, "table_grad")
    if grad_rows != n or grad_dim != dim:
        raise _bad(w, "grads is not [number of ids, width of table_grad]")
    dev = _device_of(w, table_grad, ids, grads, status)
    at, size, keep = _scratch(scratch, lib().kge_embedding_grad_scratch_bytes(rows, _int32(dim, w, "width"), n), dev, w)
    _call(w, lib().kge_embedding_grad, dev, ids.data_ptr(), n, grads.data_ptr(), tg, lg, scale, _int32(padding_id, w, "padding_id"), 1 if accumulate else 0,
          table_grad.data_ptr(), tt, rows, dim, lt, at, size, _status_word(status, w))


def dropout(x, out, p, seed, step=0, site=0, residual=None, step_dev=None):
    """kge_dropout of a contiguous tensor of any shape; the backward pass is the same call on the gradient (without residual)."""
    w = "kge_dropout"
    tx, to, n = _type_of(x, w, "x", _FLOAT), _type_of(out, w, "out", _FLOAT), x.numel()
    if not (x.is_contiguous() and out.is_contiguous() and out.numel() == n):
        raise _bad(w, "x and out are not contiguous tensors of one size")
    if residual is not None and not (residual.is_contiguous() and residual.dtype is out.dtype and residual.numel() == n):
        raise _bad(w, "residual is not a contiguous tensor of out's size and type")
    if step_dev is not None and (step_dev.dtype is not _torch.int64 or step_dev.numel() < 1):
        raise _bad(w, "step_dev is not an int64 tensor")
    if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 64 and 0 <= site < 1 << 31):
        raise _bad(w, "seed and step are 64-bit numbers, site a 31-bit one")
    dev = _device_of(w, x, out, residual, step_dev)
    _call(w, lib().kge_dropout, dev, x.data_ptr(), tx, _addr(residual), out.data_ptr(), to, n, p, seed, step, _addr(step_dev), site)


def _operand(q, scales, where, name):
    """(type, rows, columns, distance of rows, rows to a scale) of an 8-bit operand [R, K] and its scales [ceil(K / 128), R or ceil(R / 128)]."""
    code, (rows, k, ld) = _type_of(q, where, name, _FP8), _matrix(q, where, name)
    if rows <= 1:
        ld = (ld + 15) // 16 * 16
    if scales is None or scales.dtype is not _torch.float32 or not scales.is_contiguous() or scales.dim() != 2:
        raise _bad(where, f"the scales of {name} are not a contiguous float32 matrix")
    kb, per = scales.shape
    if kb != (k + 127) // 128 or per not in (rows, (rows + 127) // 128):
        raise _bad(where, f"the scales of {name} do not fit it")
    return code, rows, k, ld, 1 if per == rows else 128


def fp8_quantize(x, q=None, scales=None, qt=None, scales_t=None, block_rows=1, pow2=False):
    """kge_fp8_quantize: x [R, K] -> q [R, K] (float8_e4m3fn or float8_e5m2, rows a multiple of 16 bytes apart) with scales
    [ceil(K / 128), R] (block_rows = 1) or [ceil(K / 128), ceil(R / 128)] (128), and / or the same of x^T in qt [K, R], scales_t."""
    w = "kge_fp8_quantize"
    tx, (rows, cols, lx) = _type_of(x, w, "x", _FLOAT), _matrix(x, w, "x")
    if block_rows not in (1, 128):
        raise _bad(w, f"block_rows is {block_rows}, not 1 or 128")
    code, at, ld = None, [None, None, None, None], [0, 0]
    for i, (name, t, s, r, k) in enumerate((("q", q, scales, rows, cols), ("qt", qt, scales_t, cols, rows))):
        if t is None:
            continue
        c, tr, tk, ld[i], block = _operand(t, s, w, name)
        if tr != r or tk != k or (block != block_rows and (r + block_rows - 1) // block_rows != s.shape[1]) or code not in (None, c):
            raise _bad(w, f"{name} has another shape than x, scales for another block or another type than q")
        code, at[2 * i], at[2 * i + 1] = c, t.data_ptr(), s.data_ptr()
    if code is None:
        raise _bad(w, "neither q nor qt is given")
    dev = _device_of(w, x, q, scales, qt, scales_t)
    if rows == 0 or cols == 0:
        return
    _call(w, lib().kge_fp8_quantize, dev, x.data_ptr(), tx, rows, cols, lx, code, block_rows, 1 if pow2 else 0, at[0], ld[0], at[1], at[2], ld[1], at[3])


def fp8_matmul(a, a_scales, b, b_scales, out, addend=None, status=None):
    """kge_fp8_matmul: out [M, N] = a [M, K] . b [N, K]^T (+ addend) of operands as fp8_quantize makes them."""
    w = "kge_fp8_matmul"
    ta, m, k, la, ba = _operand(a, a_scales, w, "a")
    tb, n, kb, lb, bb = _operand(b, b_scales, w, "b")
    to, (om, on, lo), ladd = _type_of(out, w, "out", _FLOAT), _matrix(out, w, "out"), 0
    if kb != k or om != m or on != n:
        raise _bad(w, "shapes of a [M, K], b [N, K] and out [M, N] do not fit")
    if addend is not None:
        am, an, ladd = _matrix(addend, w, "addend")
        if am != m or an != n or addend.dtype is not out.dtype:
            raise _bad(w, "addend is not of out's shape and type")
    dev = _device_of(w, a, a_scales, b, b_scales, out, addend, status)
    _call(w, lib().kge_fp8_matmul, dev, a.data_ptr(), ta, la, a_scales.data_ptr(), ba, b.data_ptr(), tb, lb, b_scales.data_ptr(), bb, _addr(addend), ladd,
          out.data_ptr(), to, lo, m, n, k, _status_word(status, w))


def _int8_operand(q, scales, where, name):
    """(rows, columns, distance of rows) of an int8 operand [R, K] with scales [R]."""
    if _torch is None:
        _load_torch()
    if q.dtype is not _torch.int8:
        raise _bad(where, f"{name} has type {q.dtype}")
    rows, k, ld = _matrix(q, where, name)
    if scales is None or scales.dtype is not _torch.float32 or scales.shape != (rows,) or not scales.is_contiguous():
        raise _bad(where, f"the scales of {name} are not a contiguous float32 list of its {rows} rows")
    return rows, k, ld if rows > 1 else (ld + 15) // 16 * 16


def int8_quantize(x, q, scales):
    """kge_int8_quantize: x [R, K] (float32, bfloat16, float16) -> q int8 [R, K] (rows a multiple of 16 bytes apart) with scales float32 [R]."""
    w = "kge_int8_quantize"
    tx, (rows, cols, lx) = _type_of(x, w, "x", _FLOAT), _matrix(x, w, "x")
    qr, qc, lq = _int8_operand(q, scales, w, "q")
    if qr != rows or qc != cols:
        raise _bad(w, "q has another shape than x")
    dev = _device_of(w, x, q, scales)
    _call(w, lib().kge_int8_quantize, dev, x.data_ptr(), tx, rows, cols, lx, q.data_ptr(), lq, scales.data_ptr())


def int8_matmul(a, a_scales, b, b_scales, out, addend=None, status=None):
    """kge_int8_matmul: out [M, N] = a [M, K] . b [N, K]^T (+ addend) of operands as int8_quantize makes them."""
    w = "kge_int8_matmul"
    m, k, la = _int8_operand(a, a_scales, w, "a")
    n, kb, lb = _int8_operand(b, b_scales, w, "b")
    to, (om, on, lo), ladd = _type_of(out, w, "out", _FLOAT), _matrix(out, w, "out"), 0
    if kb != k or om != m or on != n:
        raise _bad(w, "shapes of a [M, K], b [N, K] and out [M, N] do not fit")
    if addend is not None:
        am, an, ladd = _matrix(addend, w, "addend")
        if am != m or an != n or addend.dtype is not out.dtype:
            raise _bad(w, "addend is not of out's shape and type")
    dev = _device_of(w, a, a_scales, b, b_scales, out, addend, status)
    _call(w, lib().kge_int8_matmul, dev, a.data_ptr(), la, a_scales.data_ptr(), b.data_ptr(), lb, b_scales.data_ptr(), _addr(addend), ladd,
          out.data_ptr(), to, lo, m, n, k, _status_word(status, w))


_GATE_ACTS = {"plain": 0, "sigmoid": 1, "silu": 2}
_NORM_KINDS = {"rms": 0, "layer": 1}


def _like(t, shape, dtype, dev, where, name):
    """Distance of rows of a matrix of the shape and type given, on that device."""
    stride = t.stride()
    if t.shape != shape or t.dtype is not dtype or (stride[1] != 1 and shape[1] > 1) or (stride[0] < shape[1] and shape[0] > 1):
        raise _bad(where, f"{name} is not a {list(shape)} matrix of contiguous rows and of type {dtype}")
    if t.get_device() != dev:
        raise _bad(where, "tensors are not on one GPU")
    return stride[0] if stride[0] > shape[1] else shape[1]


def _vector(v, d, dev, where, name):
    """Address of a vector of parameters on the device given, 0 for None."""
    if v is None:
        return 0
    if v.dtype is not _torch.float32 or v.shape != (d,) or not v.is_contiguous():
        raise _bad(where, f"{name} is not a contiguous float32 vector of {d}")
    if v.get_device() != dev:
        raise _bad(where, "tensors are not on one GPU")
    return v.data_ptr()


def _norm_block(w, x, block, y, gate, gate_act, post_weight, post_bias, scale, pre_weight, pre_bias, kind):
    """(kge_norm_block, shape, rows, columns, device) of the operands: block is a tensor that says what type y, gate and z are of."""
    n, d, ldx = _matrix(x, w, "x")
    shape, dev, dtype = x.shape, x.get_device(), block.dtype
    tx, tb = _FLOAT.get(x.dtype), _FLOAT.get(dtype)
    if tx is None or tb is None:
        raise _bad(w, f"x has type {x.dtype}, the block's tensors {dtype}")
    act, layer = _GATE_ACTS.get(gate_act), _NORM_KINDS.get(kind)
    if act is None or layer is None:
        raise _bad(w, f"gate_act is one of {list(_GATE_ACTS)}, kind one of {list(_NORM_KINDS)}")
    if dev < 0:
        raise _bad(w, "tensors are not on one GPU")
    return KGE_NORM_BLOCK.pack(x.data_ptr(), 0 if y is None else y.data_ptr(), 0 if gate is None else gate.data_ptr(), _vector(post_weight, d, dev, w, "post_weight"),
                               _vector(post_bias, d, dev, w, "post_bias"), _vector(scale, d, dev, w, "scale"), _vector(pre_weight, d, dev, w, "pre_weight"),
                               _vector(pre_bias, d, dev, w, "pre_bias"), ldx, 0 if y is None else _like(y, shape, dtype, dev, w, "y"),
                               0 if gate is None else _like(gate, shape, dtype, dev, w, "gate"), tx, tb, act, layer), shape, n, _int32(d, w, "width"), dev


def _stats_of(stats, n, dev, w):
    if stats is None:
        return None
    if stats.dtype is not _torch.float32 or stats.shape != (n, 4) or not stats.is_contiguous() or stats.get_device() != dev:
        raise _bad(w, f"stats is not a contiguous float32 matrix [{n}, 4] on the operands' GPU")
    return stats.data_ptr()


def block_norm(x, z=None, pre_weight=None, pre_bias=None, y=None, h=None, gate=None, gate_act="plain", post_weight=None, post_bias=None, scale=None, kind="rms",
               eps=1e-6, stats=None, z_scales=None):
    """kge_block_norm: h = x + scale act(gate) N(y), z = N(h), row by row.

    x, h [n, d] of one type, y, gate, z of one type; N after the block where post_weight is given, before the next where z (and pre_weight) is; without
    y it is z = N(x).  z may be int8 with scales float32 [n] in z_scales.  gate_act: "plain", "sigmoid", "silu"; kind: "rms", "layer".
    stats float32 [n, 4] receives what block_norm_grad needs.  h may be x, z may be y or gate."""
    w = "kge_block_norm"
    if _torch is None:
        _load_torch()
    z8 = z is not None and z.dtype is _torch.int8
    block = y if y is not None else (x if z8 or z is None else z)
    b, shape, n, d, dev = _norm_block(w, x, block, y, gate, gate_act, post_weight, post_bias, scale, pre_weight, pre_bias, kind)
    ldh = 0 if h is None else _like(h, shape, x.dtype, dev, w, "h")
    ldz = 0
    if z8:
        _, _, ldz = _int8_operand(z, z_scales, w, "z")
        if z.shape != shape or z.get_device() != dev or z_scales.get_device() != dev:
            raise _bad(w, "z is not of x's shape, or it or its scales are not on x's GPU")
    elif z is not None:
        ldz = _like(z, shape, block.dtype, dev, w, "z")
        if z_scales is not None:
            raise _bad(w, "scales are given for a z that is not int8")
    _call(w, lib().kge_block_norm, dev, b, n, d, _addr(h), ldh, _addr(z), 1 if z8 else 0, ldz, _addr(z_scales), eps, _stats_of(stats, n, dev, w))


def block_norm_grad_scratch_bytes(n, d) -> int:
    """Bytes of scratch a block_norm_grad of n rows of d columns needs (a tensor of 256 more is always enough)."""
    w = "kge_block_norm_grad_scratch_bytes"
    return int(lib().kge_block_norm_grad_scratch_bytes(_int32(n, w, "rows"), _int32(d, w, "width")))


def block_norm_grad(x, stats, dx=None, dz=None, dh=None, pre_weight=None, dpre_weight=None, dpre_bias=None, y=None, dy=None, gate=None, dgate=None, gate_act="plain",
                    post_weight=None, post_bias=None, dpost_weight=None, dpost_bias=None, scale=None, dscale=None, kind="rms", accumulate=False, scratch=None):
    """kge_block_norm_grad: the gradients of block_norm's operands from dz (of z's type, or None) and dh (of h's, or None), those that are given; dx, dy, dgate of their operands' types,
    the vectors' float32, written or (accumulate) added to what is there.  x, y, gate and the vectors are the forward call's, stats what it left."""
    w = "kge_block_norm_grad"
    if _torch is None:
        _load_torch()
    block = y if y is not None else (dz if dz is not None else x)
    b, shape, n, d, dev = _norm_block(w, x, block, y, gate, gate_act, post_weight, post_bias, scale, pre_weight, None, kind)
    tx, tb = x.dtype, block.dtype
    at = lambda t, dtype, name: (0, 0) if t is None else (t.data_ptr(), _like(t, shape, dtype, dev, w, name))
    (px, lx), (py, ly), (pg, lg), (pz, lz), (ph, lh) = at(dx, tx, "dx"), at(dy, tb, "dy"), at(dgate, tb, "dgate"), at(dz, tb, "dz"), at(dh, tx, "dh")
    v = [_vector(dpost_weight, d, dev, w, "dpost_weight"), _vector(dpost_bias, d, dev, w, "dpost_bias"), _vector(dscale, d, dev, w, "dscale"),
         _vector(dpre_weight, d, dev, w, "dpre_weight"), _vector(dpre_bias, d, dev, w, "dpre_bias")]
    if stats is None:
        raise _bad(w, "stats is not given")
    place, size, keep = _scratch(scratch, lib().kge_block_norm_grad_scratch_bytes(n, d) if any(v) else 0, dev, w)
    _call(w, lib().kge_block_norm_grad, dev, b, n, d, _stats_of(stats, n, dev, w), pz, lz, ph, lh, KGE_NORM_GRADS.pack(px, py, pg, *v, lx, ly, lg), 1 if accumulate else 0,
          place, size)


class AdamW:
    """kge_adamw over a list of tensors: made once for a model's parameters, then step() after every backward pass.

    params, grads: contiguous tensors (float32, bfloat16, float16) of one size each; a grad may be None (its parameter stays).
    m, v: float32 of the same sizes, or float8_e4m3fn and float8_e5m2 with float32 scales [ceil(n / 128)] in m_scales, v_scales; all zeros begin a run.
    copies: bfloat16 or float16 tensors (or None) that receive the new parameters too.  weight_decay: a number, or one for each tensor.
    The object keeps the tensors and their addresses: gradients are read where they are when step() runs, new ones are named by set_grads()."""

    def __init__(self, params, grads, m, v, m_scales=None, v_scales=None, copies=None, weight_decay=0.0):
        w = "kge_adamw"
        params, count = list(params), len(params)
        lists = {}
        for name, given in (("m", m), ("v", v), ("m_scales", m_scales), ("v_scales", v_scales), ("copies", copies)):
            lists[name] = [None] * count if given is None else list(given)
            if len(lists[name]) != count:
                raise _bad(w, f"{name} is not a list of {count}")
        decay = [float(weight_decay)] * count if isinstance(weight_decay, numbers.Real) else [float(d) for d in weight_decay]
        if len(decay) != count:
            raise _bad(w, f"weight_decay is not a number or a list of {count}")
        if _torch is None:
            _load_torch()
        self._at = (KgeAdamwTensor * max(count, 1))()
        self._count, self._dev, self.bits = count, -1, 32
        self._keep, self._spans, self._ends = (params, lists), [], []
        if count == 0:
            self.set_grads(grads)
            return
        self.bits = 32 if lists["m"][0] is not None and lists["m"][0].dtype is _torch.float32 else 8
        self._dev = params[0].get_device()
        spans = []
        for i, p in enumerate(params):
            t, n = self._at[i], p.numel()
            mi, vi, si, ti, ci = (lists[k][i] for k in ("m", "v", "m_scales", "v_scales", "copies"))
            t.param_type, t.n, t.weight_decay, t.param = _type_of(p, w, f"params[{i}]", _FLOAT), n, decay[i], p.data_ptr()
            states = (_torch.float32, _torch.float32) if self.bits == 32 else (_torch.float8_e4m3fn, _torch.float8_e5m2)
            for name, s, dtype in (("m", mi, states[0]), ("v", vi, states[1])):
                if s is None or s.dtype is not dtype or s.numel() != n or not s.is_contiguous():
                    raise _bad(w, f"{name}[{i}] is not a contiguous tensor of {n} elements and type {dtype}")
            t.m, t.v = mi.data_ptr(), vi.data_ptr()
            if self.bits == 8:
                for name, s in (("m_scales", si), ("v_scales", ti)):
                    if s is None or s.dtype is not _torch.float32 or s.numel() != (n + 127) // 128 or not s.is_contiguous():
                        raise _bad(w, f"{name}[{i}] is not a contiguous float32 tensor of {(n + 127) // 128}")
                t.m_scales, t.v_scales = si.data_ptr(), ti.data_ptr()
            else:
                si = ti = None
            if ci is not None:
                t.copy_type, t.copy = _type_of(ci, w, f"copies[{i}]", _FLOAT), ci.data_ptr()
                if t.copy_type == 0 or ci.numel() != n or not ci.is_contiguous():
                    raise _bad(w, f"copies[{i}] is not a contiguous bfloat16 or float16 tensor of {n} elements")
            if not p.is_contiguous():
                raise _bad(w, f"params[{i}] is not contiguous")
            _device_of(w, p, mi, vi, si, ti, ci)
            if p.get_device() != self._dev:
                raise _bad(w, "tensors are not on one GPU")
            spans += [(a.data_ptr(), a.data_ptr() + a.numel() * a.element_size()) for a in (p, mi, vi, si, ti, ci) if a is not None and a.numel() > 0]
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise _bad(w, "two of the tensors overlap")
        self._spans, self._ends = spans, [s[1] for s in spans]
        self.set_grads(grads)

    def set_grads(self, grads):
        """Other gradients from now on: as many tensors (or Nones) as there are parameters."""
        w, grads = "kge_adamw", list(grads)
        if len(grads) != self._count:
            raise _bad(w, f"grads is not a list of {self._count}")
        at = []
        for i, g in enumerate(grads):
            if g is None:
                at.append((0, None))
                continue
            code = _type_of(g, w, f"grads[{i}]", _FLOAT)
            if g.numel() != self._at[i].n or not g.is_contiguous() or g.get_device() != self._dev:
                raise _bad(w, f"grads[{i}] is not a contiguous tensor of {self._at[i].n} elements on the parameters' GPU")
            begin, end = g.data_ptr(), g.data_ptr() + g.numel() * g.element_size()
            k = bisect.bisect_left(self._ends, begin + 1)          # the first of the step's results that ends behind the gradient's beginning
            if begin < end and k < len(self._spans) and self._spans[k][0] < end:
                raise _bad(w, f"grads[{i}] overlaps a tensor that the step writes")
            at.append((code, begin))
        for t, (code, ptr) in zip(self._at, at):
            t.grad_type, t.grad = code, ptr
        self._grads = grads

    def step(self, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, grad_scale=1.0, step_dev=None, lr_dev=None, grad_scale_dev=None):
        """The step-th step (from 0).  step_dev (int64), lr_dev, grad_scale_dev (float32): numbers on the device, for a captured step."""
        w = "kge_adamw"
        if not (0 <= step < 1 << 62 and 0 <= seed < 1 << 64):
            raise _bad(w, "step is a 62-bit number, seed a 64-bit one")
        for name, t, dtype in (("step_dev", step_dev, "int64"), ("lr_dev", lr_dev, "float32"), ("grad_scale_dev", grad_scale_dev, "float32")):
            if t is not None and (t.dtype is not getattr(_torch, dtype) or t.numel() < 1 or t.get_device() != self._dev):
                raise _bad(w, f"{name} is not a tensor of {dtype} on the parameters' GPU")
        if self._count == 0:
            return
        _call(w, lib().kge_adamw, self._dev, self._at, self._count, self.bits, lr, beta1, beta2, eps, grad_scale, step, _addr(step_dev), _addr(lr_dev),
              _addr(grad_scale_dev), seed)


class Kge:
    """A handle plus the torch tensors bound to it (kept alive here).  Methods carry the
    names of the C entry points without the ``kge_`` prefix and do no arithmetic."""

    def __init__(self, cfg: KgeConfig):
        self.cfg = cfg
        self._h = _vp()
        self._keep = []
        self._check(lib().kge_create(C.byref(cfg), C.byref(self._h)), "kge_create")

    def _check(self, rc, where):
        if rc != 0:
            detail = lib().kge_error_string(rc).decode()
            if rc == -7 and self._h:
                detail += ": " + lib().kge_last_cuda_error(self._h).decode()
            raise KgeError(rc, where, detail)

    def close(self):
        if self._h:
            lib().kge_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self, num_triples=0, max_queries=0, topk=0) -> int:
        return int(lib().kge_workspace_bytes(self._h, num_triples, max_queries, topk))

    def bind(self, ent, rel, relw=None, ent_state=None, rel_state=None, relw_state=None, *,
             num_triples=0, max_queries=0, topk=0, workspace=None):
        import torch
        need = self.workspace_bytes(num_triples, max_queries, topk)
        if workspace is None:
            workspace = torch.empty(need + 256, dtype=torch.uint8, device=ent.device)
        off = (-workspace.data_ptr()) % 256
        ws = workspace[off:]
        self._keep = [ent, rel, relw, ent_state, rel_state, relw_state, workspace]
        self.workspace = workspace
        self._check(lib().kge_bind(self._h, _ptr(ent), _ptr(rel), _ptr(relw), _ptr(ent_state), _ptr(rel_state),
                                   _ptr(relw_state), C.c_void_p(ws.data_ptr()), ws.numel(), num_triples,
                                   max_queries, topk, _stream()), "kge_bind")

    def bind_features(self, feat, MH, MT, MH_state=None, MT_state=None):
        """feat: bfloat16 [E, F] device tensor; MH, MT: float32 [d, F] (the same tensor twice for a shared matrix)."""
        self._keep += [feat, MH, MT, MH_state, MT_state]
        self._check(lib().kge_bind_features(self._h, _ptr(feat), _ptr(MH), _ptr(MT), _ptr(MH_state), _ptr(MT_state), _stream()),
                    "kge_bind_features")

    def bind_features_fp8(self, feat, scales, MH, MT, MH_state=None, MT_state=None):
        """feat: float8 [E, F] and its scales [ceil(F / 128), E] as fp8_quantize makes them; the rest as in bind_features."""
        w = "kge_bind_features_fp8"
        code, rows, cols, ld, block = _operand(feat, scales, w, "feat")
        if rows != self.cfg.num_entities or cols != self.cfg.feat_dim or block != 1:
            raise _bad(w, "feat is not [entities, feat_dim] with a scale per row and block of 128")
        _device_of(w, feat, scales, MH, MT, MH_state, MT_state)
        self._keep += [feat, scales, MH, MT, MH_state, MT_state]
        self._check(lib().kge_bind_features_fp8(self._h, feat.data_ptr(), code, ld, scales.data_ptr(), _ptr(MH), _ptr(MT), _ptr(MH_state),
                                                _ptr(MT_state), _stream()), w)

    def graph_load(self, heads, rels, tails):
        """heads / rels / tails: numpy int32 host arrays."""
        self._check(lib().kge_graph_load(self._h, _ptr(heads), _ptr(rels), _ptr(tails), len(heads), _stream()),
                    "kge_graph_load")

    def graph_load_device(self, heads, rels, tails):
        """heads / rels / tails: int32 device tensors."""
        self._check(lib().kge_graph_load_device(self._h, _ptr(heads), _ptr(rels), _ptr(tails), heads.numel(), _stream()),
                    "kge_graph_load_device")

    def init_tables(self, std):
        self._check(lib().kge_init_tables(self._h, std, _stream()), "kge_init_tables")

    def debug_init_words(self, out, rows, width, stream_id):
        self._check(lib().kge_debug_init_words(self._h, _ptr(out), rows, width, stream_id, _stream()), "kge_debug_init_words")

    def sample_batch(self, step, heads, rels, tails, negs):
        self._check(lib().kge_sample_batch(self._h, step, _ptr(heads), _ptr(rels), _ptr(tails), _ptr(negs), _stream()),
                    "kge_sample_batch")

    def train_step(self, step, lr, heads=None, rels=None, tails=None, negs=None, loss_out=None):
        self._check(lib().kge_train_step(self._h, step, lr, _ptr(heads), _ptr(rels), _ptr(tails), _ptr(negs),
                                         _ptr(loss_out), _stream()), "kge_train_step")

    def gather_rows(self, ids, ent_base, rows_out):
        self._check(lib().kge_gather_rows(self._h, _ptr(ids), ids.numel(), ent_base, _ptr(rows_out), _stream()), "kge_gather_rows")

    def train_gradients(self, step, heads, rels, tails, negs, loss_out=None):
        self._check(lib().kge_train_gradients(self._h, step, _ptr(heads), _ptr(rels), _ptr(tails), _ptr(negs), _ptr(loss_out), _stream()),
                    "kge_train_gradients")

    def gradient_rows(self):
        """Device addresses (ints) of the gradient rows of the last step: (entity slots [2B+N, d], relations [B, k], normals [B, d])."""
        a, b, c = _vp(), _vp(), _vp()
        self._check(lib().kge_gradient_rows(self._h, C.byref(a), C.byref(b), C.byref(c)), "kge_gradient_rows")
        return a.value, b.value, c.value

    def apply_gradients(self, table, ids, grads, step, lr, scratch=None):
        """table: 0 entities, 1 relations, 2 normals; ids int32 [n], grads float32 [n, width] device tensors."""
        import torch
        n = ids.numel()
        need = int(lib().kge_apply_scratch_bytes(self._h, table, n))
        if scratch is None or scratch.numel() < need + 256:
            scratch = torch.empty(need + 256, dtype=torch.uint8, device=ids.device)
        off = (-scratch.data_ptr()) % 256
        self._check(lib().kge_apply_gradients(self._h, table, _ptr(ids), _ptr(grads), n, step, lr, C.c_void_p(scratch.data_ptr() + off),
                                              need, _stream()), "kge_apply_gradients")
        return scratch

    def train_step_host(self, step, lr, heads, rels, tails, negs, loss_out):
        """ids and loss_out are host arrays (pinned torch tensors or numpy)."""
        self._check(lib().kge_train_step_host(self._h, step, lr, _ptr(heads), _ptr(rels), _ptr(tails), _ptr(negs),
                                              _ptr(loss_out), _stream()), "kge_train_step_host")

    def score_all_topk(self, q_heads, q_rels, k, true_tails, out_ids, out_scores, out_ranks=None):
        self._check(lib().kge_score_all_topk(self._h, _ptr(q_heads), _ptr(q_rels), q_heads.numel(), k,
                                             _ptr(true_tails), _ptr(out_ids), _ptr(out_scores), _ptr(out_ranks),
                                             _stream()), "kge_score_all_topk")

    def score_all_topk_host(self, q_heads, q_rels, k, true_tails, out_ids, out_scores, out_ranks=None):
        """Host arrays (pinned torch tensors or numpy) in and out."""
        self._check(lib().kge_score_all_topk_host(self._h, _ptr(q_heads), _ptr(q_rels), len(q_heads), k, _ptr(true_tails),
                                                  _ptr(out_ids), _ptr(out_scores), _ptr(out_ranks), _stream()),
                    "kge_score_all_topk_host")

    def shard_query_vectors(self, q_heads, q_rels, ent_base, qvec_out):
        self._check(lib().kge_shard_query_vectors(self._h, _ptr(q_heads), _ptr(q_rels), q_heads.numel(), ent_base, _ptr(qvec_out),
                                                  _stream()), "kge_shard_query_vectors")

    def shard_true_scores(self, qvec, q_rels, true_tails, ent_base, ftrue_out):
        self._check(lib().kge_shard_true_scores(self._h, _ptr(qvec), _ptr(q_rels), _ptr(true_tails), q_rels.numel(), ent_base,
                                                _ptr(ftrue_out), _stream()), "kge_shard_true_scores")

    def shard_score_topk(self, qvec, q_rels, k, ftrue, true_tails, ent_base, out_ids, out_scores, out_beat=None):
        self._check(lib().kge_shard_score_topk(self._h, _ptr(qvec), _ptr(q_rels), q_rels.numel(), k, _ptr(ftrue), _ptr(true_tails),
                                               ent_base, _ptr(out_ids), _ptr(out_scores), _ptr(out_beat), _stream()),
                    "kge_shard_score_topk")

    def refresh_inference_table(self):
        self._check(lib().kge_refresh_inference_table(self._h, _stream()), "kge_refresh_inference_table")

    def eval_mrr(self, q_heads, q_rels, true_tails, k_cutoff=10) -> float:
        out = C.c_double(0.0)
        self._check(lib().kge_eval_mrr(self._h, _ptr(q_heads), _ptr(q_rels), _ptr(true_tails), q_heads.numel(),
                                       k_cutoff, C.byref(out), _stream()), "kge_eval_mrr")
        return out.value

    def mrr_from_ranks(self, ranks, k_cutoff=10) -> float:
        out = C.c_double(0.0)
        self._check(lib().kge_mrr_from_ranks(self._h, _ptr(ranks), ranks.numel(), k_cutoff, C.byref(out), _stream()),
                    "kge_mrr_from_ranks")
        return out.value

    def debug_capture_scores(self, scores_out):
        """scores_out: float32 device tensor of B * N elements, or None to switch the tap off."""
        self._capture = scores_out
        self._check(lib().kge_debug_capture_scores(self._h, _ptr(scores_out)), "kge_debug_capture_scores")

    def debug_set_wait_limit(self, tries: int):
        self._check(lib().kge_debug_set_wait_limit(self._h, tries), "kge_debug_set_wait_limit")

    def debug_wait_probe(self):
        self._check(lib().kge_debug_wait_probe(self._h, _stream()), "kge_debug_wait_probe")

    def get_status(self) -> int:
        return int(lib().kge_get_status(self._h, _stream()))

    def launch_count(self) -> int:
        return int(lib().kge_launch_count(self._h))

    STAGES = ("sample", "build", "block", "loss", "th_u", "accum_q", "accum_t", "chain", "rank",
              "segment", "update", "th_contract")

    def profile(self, enable: bool):
        self._check(lib().kge_profile(self._h, int(enable)), "kge_profile")

    def profile_read(self, reset=True):
        """{stage: (total ms, launches)} accumulated while profiling was enabled."""
        n = len(self.STAGES)
        ms, cnt = (C.c_double * n)(), (C.c_int64 * n)()
        self._check(lib().kge_profile_read(self._h, ms, cnt, int(reset)), "kge_profile_read")
        return {name: (ms[i], cnt[i]) for i, name in enumerate(self.STAGES)}

    def debug_export(self, tap: str):
        """Parity tap as a numpy array (flat)."""
        import numpy as np
        code = TAPS[tap]
        nbytes = int(lib().kge_debug_bytes(self._h, code, _stream()))
        if tap in _I64_TAPS:
            out = np.empty(nbytes // 8, dtype=_I64_TAPS[tap])
        else:
            out = np.empty(nbytes // 4, dtype=np.int32 if tap in _INT_TAPS else np.float32)
        if nbytes:
            self._check(lib().kge_debug_export(self._h, code, _ptr(out), nbytes, _stream()), "kge_debug_export")
        return out
