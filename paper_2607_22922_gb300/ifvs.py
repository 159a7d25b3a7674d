"""Python binding of the C ABI in include/ifvs.h (argument marshalling only).

Every function here has the name of the C entry point it calls and passes
plain pointers and sizes: numpy arrays for host memory, or CUDA tensors
(anything with ``data_ptr()``) together with ``IFVS_F_DEVICE_IO`` for device
memory.  No computation of the query path happens in Python: if
``libifvs.so`` is missing the import fails.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libifvs.so")

(IFVS_OK, IFVS_ERR_ARG, IFVS_ERR_OOM, IFVS_ERR_CUDA, IFVS_ERR_STATE, IFVS_ERR_UNSUPPORTED,
 IFVS_ERR_TIMEOUT) = 0, -1, -2, -3, -4, -5, -6
IFVS_OP_EQ, IFVS_OP_RANGE, IFVS_OP_GE, IFVS_OP_LT, IFVS_OP_GT, IFVS_OP_LE = 0, 1, 2, 3, 4, 5
IFVS_ATTR_I32, IFVS_ATTR_I16 = 0, 1
IFVS_F_DEVICE_IO, IFVS_F_STAGE_TIMING, IFVS_F_PLAIN_PQ, IFVS_F_PLAIN_LOADS = 0x1, 0x2, 0x4, 0x8
IFVS_MAX_K, IFVS_MAX_M, IFVS_MAX_ATTRS, IFVS_N_STAGES = 256, 128, 4, 9
IFVS_T_F32, IFVS_T_F16, IFVS_T_BF16 = 0, 1, 2
IFVS_ACT_SILU, IFVS_ACT_GELU, IFVS_ACT_RELU, IFVS_ACT_NONE = 0, 1, 2, 3
STAGES = ("predicate", "filter", "condition", "lut", "scan", "merge", "rerank", "layout", "train")

# ifvs_predicate: 104 bytes (n_clauses, reserved, 4 x {col, op, lo, hi})
CLAUSE_DTYPE = np.dtype([("col", "<i4"), ("op", "<i4"), ("lo", "<i8"), ("hi", "<i8")])
PREDICATE_DTYPE = np.dtype([("n_clauses", "<i4"), ("reserved", "<i4"), ("c", CLAUSE_DTYPE, (4,))])


class IfvsError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("ifvs error %d: %s" % (code, msg))
        self.code = code


class SearchParams(C.Structure):
    _fields_ = [("flags", C.c_uint32), ("rerank", C.c_int32), ("sub_batch", C.c_int32),
                ("chunk_blocks", C.c_int32), ("list_max_ppm", C.c_int32), ("pair_min_rows", C.c_int32),
                ("stream", C.c_void_p)]


class JoinParams(C.Structure):
    _fields_ = [("T", C.c_int64), ("D", C.c_int32), ("type", C.c_int32), ("n_seq", C.c_int64),
                ("offsets", C.c_void_p), ("gate", C.c_void_p), ("w_post", C.c_void_p),
                ("w_pre", C.c_void_p), ("res_scale", C.c_float), ("eps", C.c_float),
                ("stream", C.c_void_p)]


class FfnParams(C.Structure):
    _fields_ = [("T", C.c_int64), ("D", C.c_int32), ("F", C.c_int32), ("type", C.c_int32),
                ("act", C.c_int32), ("w_in", C.c_void_p), ("w_out", C.c_void_p),
                ("stream", C.c_void_p)]


class LinearParams(C.Structure):
    _fields_ = [("T", C.c_int64), ("D_in", C.c_int32), ("D_out", C.c_int32), ("type", C.c_int32),
                ("act", C.c_int32), ("w", C.c_void_p), ("bias", C.c_void_p), ("stream", C.c_void_p)]


class AttendParams(C.Structure):
    _fields_ = [("Tq", C.c_int64), ("Tk", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("dh", C.c_int32), ("type", C.c_int32), ("n_seq", C.c_int64), ("q_offsets", C.c_void_p),
                ("kv_offsets", C.c_void_p), ("kv_ids", C.c_void_p), ("scale", C.c_float)] + [
                    ("ld_" + n, C.c_int64) for n in ("q", "k", "v", "out", "d_out", "dq", "dk", "dv")] + [
                        ("stream", C.c_void_p)]


class TrainParams(C.Structure):
    _fields_ = [("tau", C.c_float), ("lam", C.c_float), ("lr", C.c_float), ("lr_wz", C.c_float),
                ("n_pos", C.c_int32), ("n_neg", C.c_int32), ("flags", C.c_uint32),
                ("stream", C.c_void_p)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError("libifvs.so is not built (%s); run `python -c \"import __graft_entry__ "
                          "as g; g.build()\"` or `python -m paper_2607_22922_gb300.build`" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    P, I32, I64, U32, F32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_float
    U64, F64 = C.c_uint64, C.c_double
    sig = {
        "ifvs_load_index": (C.c_int, [P, I32, P, I64, I32, I32, P, P, I32, P, I32, U32]),
        "ifvs_load_codebooks": (C.c_int, [P, P, I32, P, I64, I32, I32, P, P]),
        "ifvs_search_batch": (C.c_int, [P, P, P, I64, I32, P, P, P, P, P]),
        "ifvs_filter": (C.c_int, [P, P, I64, P, P, P]),
        "ifvs_condition": (C.c_int, [P, P, P, I64, P, P, P, P, P, P, P]),
        "ifvs_scan_topk": (C.c_int, [P, P, P, I64, I32, P, P, P]),
        "ifvs_rerank": (C.c_int, [P, P, P, I64, I32, I32, P, P, P]),
        "ifvs_scan_topk_static": (C.c_int, [P, P, P, I64, I32, P, P, P]),
        "ifvs_pq_encode": (C.c_int, [I32, P, I64, I32, I32, I32, P, P, P, U32, P]),
        "ifvs_merge_topk": (C.c_int, [I32, P, P, I64, I32, I32, P, P, U32, P]),
        "ifvs_pq_train": (C.c_int, [I32, P, I64, I32, I32, I32, I32, P, P, P, U32, P]),
        "ifvs_train_grad": (C.c_int, [P, P, P, I64, P, P, P, P, P, P, P]),
        "ifvs_train_step": (C.c_int, [P, P, P, I64, P, P, P, P, P]),
        "ifvs_get_conditioning": (C.c_int, [P, P, P, U32]),
        "ifvs_layers_create": (C.c_int, [P, I32]),
        "ifvs_layers_free": (None, [P]),
        "ifvs_layers_status": (C.c_int, [P]),
        "ifvs_embed": (C.c_int, [P, P, I64, I32, I32, P, I64, F32, P, P]),
        "ifvs_embed_grad": (C.c_int, [P, P, P, I64, I64, I32, I32, F32, P, P]),
        "ifvs_norm_join": (C.c_int, [P, P, P, P, P, P]),
        "ifvs_norm_join_grad": (C.c_int, [P] * 11),
        "ifvs_ffn": (C.c_int, [P, P, P, P]),
        "ifvs_ffn_grad": (C.c_int, [P] * 7),
        "ifvs_linear": (C.c_int, [P] * 5),
        "ifvs_linear_grad": (C.c_int, [P] * 7),
        "ifvs_attend": (C.c_int, [P] * 7),
        "ifvs_attend_grad": (C.c_int, [P] * 11),
        "ifvs_dropout": (C.c_int, [P, P, P, I64, I32, F64, U64, U64, P, P, P]),
        "ifvs_stage_times": (C.c_int, [P, P, P, I32]),
        "ifvs_canonical_predicate": (C.c_int, [P, P, I32, P, P, P]),
        "ifvs_index_info": (C.c_int, [P, P]),
        "ifvs_free": (None, [P]),
        "ifvs_last_error": (C.c_char_p, []),
        "ifvs_version": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    return L


_lib = _load()


def lib():
    return _lib


def ifvs_last_error() -> str:
    return _lib.ifvs_last_error().decode()


def ifvs_version() -> str:
    return _lib.ifvs_version().decode()


def _check(rc):
    if rc != IFVS_OK:
        raise IfvsError(rc, ifvs_last_error())


def _ptr(a):
    """Address of a numpy array or a tensor (None -> NULL)."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if not a.flags.c_contiguous:
            raise ValueError("arrays must be C-contiguous")
        return a.__array_interface__["data"][0]
    if hasattr(a, "data_ptr"):
        if hasattr(a, "is_contiguous") and not a.is_contiguous():
            raise ValueError("tensors must be contiguous")
        return a.data_ptr()
    raise TypeError("expected a numpy array or a tensor, got %r" % type(a))


def _params(flags=0, rerank=0, sub_batch=0, stream=None, chunk_blocks=0, list_max_ppm=0, pair_min_rows=0):
    p = SearchParams()
    p.flags = flags
    p.rerank = rerank
    p.sub_batch = sub_batch
    p.chunk_blocks = chunk_blocks
    p.list_max_ppm = list_max_ppm
    p.pair_min_rows = pair_min_rows
    p.stream = stream
    return p


def _host(a, dtype):
    return None if a is None else np.ascontiguousarray(a, dtype=dtype)


# ------------------------------------------------------------ entry points

def ifvs_load_index(codes, attrs, vectors=None, D=0, device=0, K=256, device_io=False):
    """codes [N][M] uint8; attrs: list of int32 / int16 columns of length N."""
    N, M = int(codes.shape[0]), int(codes.shape[1])
    if not device_io:
        codes = _host(codes, np.uint8)
        attrs = [np.ascontiguousarray(a) for a in attrs]
        vectors = _host(vectors, np.float32)
    types = []
    for a in attrs:
        dt = str(a.dtype).replace("torch.", "")
        if dt == "int32":
            types.append(IFVS_ATTR_I32)
        elif dt == "int16":
            types.append(IFVS_ATTR_I16)
        else:
            raise TypeError("attribute columns must be int32 or int16")
    ptrs = (C.c_void_p * max(1, len(attrs)))(*[_ptr(a) for a in attrs])
    ty = np.array(types if types else [0], dtype=np.int32)
    if vectors is not None and not D:
        D = int(vectors.shape[1])
    h = C.c_void_p()
    _check(_lib.ifvs_load_index(C.byref(h), device, _ptr(codes), N, M, K, ptrs, _ptr(ty),
                                len(attrs), _ptr(vectors), D,
                                IFVS_F_DEVICE_IO if device_io else 0))
    return h


def ifvs_load_codebooks(ix, C_pq, bank=None, h=0, r=0, W=None, hash_seeds=None):
    info = ifvs_index_info(ix)
    C_pq = _host(C_pq, np.float32)
    M, K, ds = C_pq.shape
    if (M, K) != (info["M"], info["K"]):
        raise ValueError("C_pq is %s; the index has M = %d, K = %d" % (C_pq.shape, info["M"], info["K"]))
    bank = _host(bank, np.float32)
    W = _host(W, np.float32)
    seeds = _host(hash_seeds, np.uint64)
    B = 0 if bank is None else bank.shape[0]
    if bank is not None:
        if W is None or seeds is None:
            raise ValueError("W and hash_seeds are required with a bank")
        h = len(seeds)
        r = W.shape[1]
        if W.shape != (M, r, K, ds) or bank.ndim != 2 or bank.shape[1] != M * r:
            raise ValueError("bank %s / W %s do not match M = %d, K = %d, ds = %d"
                             % (bank.shape, W.shape, M, K, ds))
    _check(_lib.ifvs_load_codebooks(ix, _ptr(C_pq), ds, _ptr(bank), B, h, r, _ptr(W), _ptr(seeds)))


def ifvs_search_batch(ix, queries, preds, k, wz=None, ids=None, dists=None, npass=None,
                      flags=0, rerank=0, sub_batch=0, stream=None, chunk_blocks=0, list_max_ppm=0,
                      pair_min_rows=0):
    """Host mode (default): numpy in, numpy out.  With IFVS_F_DEVICE_IO in
    ``flags`` every array (inputs and preallocated outputs) is a device tensor."""
    nq = int(queries.shape[0])
    dio = bool(flags & IFVS_F_DEVICE_IO)
    if not dio:
        queries = _host(queries, np.float32)
        preds = np.ascontiguousarray(preds)
        if preds.dtype.itemsize != 104:
            raise ValueError("predicates must be 104-byte records")
        wz = _host(wz, np.float32)
        if ids is None:
            ids = np.empty((nq, k), np.int64)
        if dists is None:
            dists = np.empty((nq, k), np.float32)
        if npass is None:
            npass = np.empty(nq, np.int64)
    p = _params(flags, rerank, sub_batch, stream, chunk_blocks, list_max_ppm, pair_min_rows)
    _check(_lib.ifvs_search_batch(ix, _ptr(queries), _ptr(preds), nq, k, _ptr(wz), C.byref(p),
                                  _ptr(ids), _ptr(dists), _ptr(npass)))
    return ids, dists, npass


def ifvs_filter(ix, preds, N, flags=0, sub_batch=0):
    preds = np.ascontiguousarray(preds)
    nq = len(preds)
    bm = np.empty((nq, (N + 31) // 32), np.uint32)
    npass = np.empty(nq, np.int64)
    p = _params(flags, 0, sub_batch)
    _check(_lib.ifvs_filter(ix, _ptr(preds), nq, C.byref(p), _ptr(bm), _ptr(npass)))
    return bm, npass


def ifvs_condition(ix, queries, preds, wz=None, M=None, K=256, ds=None, h=0, r=0, flags=0,
                   want_cifvs=False):
    queries = _host(queries, np.float32)
    preds = np.ascontiguousarray(preds)
    wz = _host(wz, np.float32)
    nq, D = queries.shape
    bank_idx = np.empty((nq, max(h, 1)), np.uint32)
    alpha = np.empty((nq, max(M * r, 1)), np.float32)
    wf = np.empty((nq, D), np.float32)
    lut = np.empty((nq, M, K), np.float32)
    cif = np.empty((nq, M, K, ds), np.float32) if want_cifvs else None
    p = _params(flags)
    _check(_lib.ifvs_condition(ix, _ptr(queries), _ptr(preds), nq, _ptr(wz), C.byref(p),
                               _ptr(bank_idx), _ptr(alpha), _ptr(wf), _ptr(cif), _ptr(lut)))
    return dict(bank_idx=bank_idx[:, :h], alpha=alpha[:, :M * r], wf=wf, lut=lut, C_ifvs=cif)


def ifvs_scan_topk(ix, lut, bitmaps, k, flags=0, sub_batch=0):
    lut = _host(lut, np.float32)
    bitmaps = _host(bitmaps, np.uint32)
    nq = lut.shape[0]
    ids = np.empty((nq, k), np.int64)
    dists = np.empty((nq, k), np.float32)
    p = _params(flags, 0, sub_batch)
    _check(_lib.ifvs_scan_topk(ix, _ptr(lut), _ptr(bitmaps), nq, k, C.byref(p), _ptr(ids),
                               _ptr(dists)))
    return ids, dists


def ifvs_scan_topk_static(ix, lut, bitmaps, k, ids, dists, stream=None):
    """Device tensors only (lut [nq][M][K] float32, bitmaps [nq][ceil(N/32)]
    uint32, ids [nq][k] int64, dists [nq][k] float32); enqueues on ``stream``
    and returns without synchronising.  Uses no device allocation."""
    nq = int(lut.shape[0])
    _check(_lib.ifvs_scan_topk_static(ix, _ptr(lut), _ptr(bitmaps), nq, k, stream, _ptr(ids),
                                      _ptr(dists)))
    return ids, dists


def ifvs_merge_topk(dists, ids, k=None, device=0, dists_out=None, ids_out=None, flags=0, stream=None):
    """Select across row shards: dists [G][nq][k] float32 and ids [G][nq][k]
    int64 (global row ids, -1 = padding) -> the k smallest by (dist, id) per
    query, [nq][k] each.  Host mode (default): numpy in, numpy out; with
    IFVS_F_DEVICE_IO every array is a device tensor (outputs preallocated)."""
    dio = bool(flags & IFVS_F_DEVICE_IO)
    G, nq, kk = (int(v) for v in dists.shape)
    k = kk if k is None else k
    if k != kk or tuple(ids.shape) != (G, nq, kk):
        raise ValueError("dists and ids must both be [G][nq][k]")
    if not dio:
        dists = _host(dists, np.float32)
        ids = _host(ids, np.int64)
        dists_out = np.empty((nq, k), np.float32)
        ids_out = np.empty((nq, k), np.int64)
    elif dists_out is None or ids_out is None:
        raise ValueError("device I/O needs preallocated outputs")
    _check(_lib.ifvs_merge_topk(device, _ptr(dists), _ptr(ids), nq, G, k, _ptr(dists_out), _ptr(ids_out),
                                flags, stream))
    return ids_out, dists_out


def ifvs_pq_encode(X, C_pq, device=0, want_dmin=False, codes=None, dmin=None, flags=0,
                   stream=None):
    """Host mode (default): numpy in, codes [n][M] uint8 (and dmin [n][M]
    float32) out.  With IFVS_F_DEVICE_IO in ``flags``, X, C_pq, ``codes``
    (and ``dmin``, if wanted) are preallocated device tensors; with a stream
    the call only enqueues the kernel."""
    dio = bool(flags & IFVS_F_DEVICE_IO)
    if not dio:
        X = _host(X, np.float32)
        C_pq = _host(C_pq, np.float32)
    n, D = int(X.shape[0]), int(X.shape[1])
    M, K, ds = (int(v) for v in C_pq.shape)
    if not dio:
        codes = np.empty((n, M), np.uint8)
        dmin = np.empty((n, M), np.float32) if want_dmin else None
    elif codes is None:
        raise ValueError("device I/O needs a preallocated codes tensor")
    _check(_lib.ifvs_pq_encode(device, _ptr(X), n, D, M, K, _ptr(C_pq), _ptr(codes), _ptr(dmin),
                               flags, stream))
    return (codes, dmin) if (want_dmin or dmin is not None) else codes


def ifvs_pq_train(X, C_init, iters, device=0, C_out=None, objective=None, flags=0, stream=None):
    """Lloyd iterations from C_init [M][K][ds]; returns (C_out, objective
    [iters][M]).  With IFVS_F_DEVICE_IO, X, C_init, ``C_out`` and ``objective``
    (or None) are device tensors."""
    dio = bool(flags & IFVS_F_DEVICE_IO)
    if not dio:
        X = _host(X, np.float32)
        C_init = _host(C_init, np.float32)
    n, D = int(X.shape[0]), int(X.shape[1])
    M, K, ds = (int(v) for v in C_init.shape)
    if not dio:
        C_out = np.empty_like(C_init)
        objective = np.empty((max(iters, 1), M), np.float64)
    elif C_out is None:
        raise ValueError("device I/O needs a preallocated C_out tensor")
    _check(_lib.ifvs_pq_train(device, _ptr(X), n, D, M, K, iters, _ptr(C_init), _ptr(C_out),
                              _ptr(objective), flags, stream))
    return C_out, (objective[:iters] if objective is not None else None)


def _train_params(tau, lam, lr, n_pos, n_neg, flags, stream, lr_wz=None):
    tp = TrainParams()
    tp.tau, tp.lam, tp.lr = float(tau), float(lam), float(lr)
    tp.lr_wz = float(lr if lr_wz is None else lr_wz)
    tp.n_pos, tp.n_neg = int(n_pos), int(n_neg)
    tp.flags = flags
    tp.stream = stream
    return tp


def ifvs_train_grad(ix, queries, preds, wz, cand, n_pos, tau, lam, B, Mr, W_shape, flags=0,
                    stream=None, g_bank=None, g_W=None, g_wz=None):
    """Loss and gradients (dL/dbank [B][Mr], dL/dW, dL/dw_z) of one mini-batch
    for given candidates cand [nq][n_pos + n_neg] (positives first)."""
    dio = bool(flags & IFVS_F_DEVICE_IO)
    nq, V = int(cand.shape[0]), int(cand.shape[1])
    if not dio:
        queries = _host(queries, np.float32)
        preds = np.ascontiguousarray(preds)
        wz = _host(wz, np.float32)
        cand = _host(cand, np.int64)
        g_bank = np.empty((B, Mr), np.float32)
        g_W = np.empty(W_shape, np.float32)
        g_wz = np.empty(wz.shape[-1], np.float32)
    tp = _train_params(tau, lam, 0.0, n_pos, V - n_pos, flags, stream)
    loss = C.c_double(0.0)
    _check(_lib.ifvs_train_grad(ix, _ptr(queries), _ptr(preds), nq, _ptr(wz), _ptr(cand),
                                C.byref(tp), _ptr(g_bank), _ptr(g_W), _ptr(g_wz), C.byref(loss)))
    return loss.value, g_bank, g_W, g_wz


def ifvs_train_step(ix, queries, preds, wz, positives, n_neg, tau, lam, lr, flags=0, stream=None,
                    negatives=None, lr_wz=None):
    """One SGD step (step lr for the bank and W, lr_wz for w_z, default lr);
    updates the index's bank and W and ``wz`` in place.  Returns (loss,
    negatives [nq][n_neg])."""
    dio = bool(flags & IFVS_F_DEVICE_IO)
    nq, P = int(positives.shape[0]), int(positives.shape[1])
    if not dio:
        queries = _host(queries, np.float32)
        preds = np.ascontiguousarray(preds)
        positives = _host(positives, np.int64)
        if not (isinstance(wz, np.ndarray) and wz.dtype == np.float32 and wz.flags.c_contiguous):
            raise ValueError("wz must be a C-contiguous float32 array (updated in place)")
        negatives = np.empty((nq, n_neg), np.int64)
    tp = _train_params(tau, lam, lr, P, n_neg, flags, stream, lr_wz)
    loss = C.c_double(0.0)
    _check(_lib.ifvs_train_step(ix, _ptr(queries), _ptr(preds), nq, _ptr(wz), _ptr(positives),
                                C.byref(tp), _ptr(negatives), C.byref(loss)))
    return loss.value, negatives


def ifvs_get_conditioning(ix, B, Mr, W_shape):
    bank = np.empty((B, Mr), np.float32)
    W = np.empty(W_shape, np.float32)
    _check(_lib.ifvs_get_conditioning(ix, _ptr(bank), _ptr(W), 0))
    return bank, W


# ---- layers of a predicate encoder: CUDA tensors only ----------------------
#
# Streams.  A call with a stream (a torch stream or a raw handle) is enqueued
# there: its inputs have to be ready in that stream's order, and to stay alive
# until its work is done, which for tensors of another stream is the caller's to
# see to (Tensor.record_stream).  Outputs that the call makes are that stream's
# memory.  A call without one runs after everything that torch's current stream
# has been given so far, and has written its outputs when it returns.

_ACTS = {"silu": IFVS_ACT_SILU, "gelu": IFVS_ACT_GELU, "relu": IFVS_ACT_RELU}
_ANY_ACT = dict(_ACTS, none=IFVS_ACT_NONE)      # of the linear layer
_TYPES = {}         # torch's element types -> IFVS_T_*, filled on first use
_INTS = {}          # and its integer types -> their names
_MASK64 = 2**64 - 1
_LEGACY_STREAM = 1  # cudaStreamLegacy: the default stream as a non-NULL handle


def _type(a):
    t = _TYPES.get(a.dtype)
    if t is None:
        name = str(a.dtype).replace("torch.", "")
        if name not in ("float32", "float16", "bfloat16"):
            raise TypeError("tensors must be float32, float16 or bfloat16, got %s" % name)
        t = _TYPES[a.dtype] = {"float32": IFVS_T_F32, "float16": IFVS_T_F16,
                               "bfloat16": IFVS_T_BF16}[name]
    return t


def _is_vector(a, name):
    """Whether ``a`` is a vector of this integer type."""
    t = _INTS.get(a.dtype)
    if t is None:
        t = _INTS[a.dtype] = str(a.dtype).replace("torch.", "")
    return t == name and a.dim() == 1


def _on(L, a, name, stream):
    """The number of a tensor's device, which has to be the handle's.  For a call
    without a stream, waits for torch's current one: the handle's own stream is
    ordered after the default stream alone."""
    at = a.get_device()
    if at != L.device:
        raise ValueError("%s is on %s, the handle on cuda:%d" % (name, a.device, L.device))
    if not stream:
        import torch
        here = torch.cuda.current_stream(at)
        if here.cuda_stream:
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("a call in a capture needs the captured stream")
            here.synchronize()
    return at


def _dev(a, shape, dtype, name, at):
    """Address of a contiguous tensor of this shape and type on CUDA device
    ``at`` (None -> NULL)."""
    if a is None:
        return None
    if a.shape != shape or a.dtype != dtype:
        raise ValueError("%s is %s %s, expected %s %s" % (name, tuple(a.shape), a.dtype, shape, dtype))
    if a.get_device() != at or not a.is_contiguous():
        raise ValueError("%s must be a contiguous tensor on cuda:%d" % (name, at))
    return a.data_ptr() or 256      # a tensor without elements has no address; none is read


def _stream(stream):
    """A raw handle, a torch stream (its default stream is the legacy one) or
    None (the handle's own stream; the call waits)."""
    if stream is None or isinstance(stream, int):
        return stream
    return stream.cuda_stream or _LEGACY_STREAM


def _like(a, stream, *shape, dtype=None):
    """An output: memory of the stream that the call runs on."""
    dtype = a.dtype if dtype is None else dtype
    if stream:
        import torch
        raw = stream if isinstance(stream, int) else stream.cuda_stream
        raw = 0 if raw == _LEGACY_STREAM else raw
        if raw != torch.cuda.current_stream(a.device).cuda_stream:
            if isinstance(stream, int):
                stream = torch.cuda.ExternalStream(raw, a.device) if raw else torch.cuda.default_stream(a.device)
            with torch.cuda.stream(stream):
                return a.new_empty(shape, dtype=dtype)
    return a.new_empty(shape, dtype=dtype)


class _LayersHandle(C.c_void_p):
    device = None       # its number


def ifvs_layers_create(device=0):
    h = _LayersHandle()
    _check(_lib.ifvs_layers_create(C.byref(h), device))
    h.device = device
    return h


def ifvs_layers_free(L):
    _lib.ifvs_layers_free(L)


def ifvs_layers_status(L):
    _check(_lib.ifvs_layers_status(L))


def _ids(ids):
    if not _is_vector(ids, "int32"):
        raise ValueError("ids must be a vector of int32")
    return int(ids.shape[0])


def ifvs_embed(L, table, ids, scale=1.0, out=None, stream=None):
    """out [T][D] = scale table[ids]; id -1 gives a row of zeros."""
    (V, D), T, at = table.shape, _ids(ids), _on(L, table, "table", stream)
    out = _like(table, stream, T, D) if out is None else out
    dt = table.dtype
    _check(_lib.ifvs_embed(L, _dev(table, (V, D), dt, "table", at), V, D, _type(table),
                           _dev(ids, (T,), ids.dtype, "ids", at), T, scale, _dev(out, (T, D), dt, "out", at),
                           _stream(stream)))
    return out


def ifvs_embed_grad(L, d_out, ids, scale=1.0, V=None, d_table=None, stream=None):
    """d_table [V][D]: per id, scale times the sum of its tokens' rows of d_out
    (zeros for ids without tokens).  Give V or d_table."""
    (T, D), dt, at = d_out.shape, d_out.dtype, _on(L, d_out, "d_out", stream)
    d_table = _like(d_out, stream, V, D) if d_table is None else d_table
    V = int(d_table.shape[0])
    _check(_lib.ifvs_embed_grad(L, _dev(d_out, (T, D), dt, "d_out", at),
                                _dev(ids, (_ids(ids),), ids.dtype, "ids", at), _same_length(ids, T), V, D, _type(d_out), scale,
                                _dev(d_table, (V, D), dt, "d_table", at), _stream(stream)))
    return d_table


def _same_length(ids, T):
    if ids.shape[0] != T:
        raise ValueError("%d ids for %d tokens" % (ids.shape[0], T))
    return int(T)


def _join_params(x, gate, w_post, w_pre, offsets, res_scale, eps, stream, at=None):
    (T, D), dt, at = x.shape, x.dtype, x.get_device() if at is None else at
    B, off = 1, None
    if offsets is not None:
        if not _is_vector(offsets, "int64") or offsets.shape[0] < 2:
            raise ValueError("offsets must be a vector of B + 1 int64")
        B = offsets.shape[0] - 1
        off = _dev(offsets, (B + 1,), offsets.dtype, "offsets", at)
    p = JoinParams(T, D, _type(x), B, off, _dev(gate, (B, D), dt, "gate", at),
                   _dev(w_post, (D,), dt, "w_post", at), _dev(w_pre, (D,), dt, "w_pre", at), res_scale, eps, _stream(stream))
    return p, (T, D), (B, D), dt


def ifvs_norm_join(L, x, y=None, gate=None, w_post=None, w_pre=None, offsets=None, res_scale=1.0,
                   eps=1e-5, x_out=None, n_out=None, stream=None):
    """x_out = res_scale x + gate * w_post * y / rms(y) and, with w_pre,
    n_out = w_pre * x_out / rms(x_out); gate [B][D] by the sequences that
    ``offsets`` delimits.  Without y only n_out, of x.  Returns (x_out, n_out)."""
    at = _on(L, x, "x", stream)
    p, td, _, dt = _join_params(x, gate, w_post, w_pre, offsets, res_scale, eps, stream, at)
    if y is not None and x_out is None:
        x_out = _like(x, stream, *td)
    if w_pre is not None and n_out is None:
        n_out = _like(x, stream, *td)
    _check(_lib.ifvs_norm_join(L, C.byref(p), _dev(x, td, dt, "x", at), _dev(y, td, dt, "y", at),
                               _dev(x_out, td, dt, "x_out", at), _dev(n_out, td, dt, "n_out", at)))
    return x_out, n_out


def ifvs_norm_join_grad(L, x_out, y=None, gate=None, w_post=None, w_pre=None, d_x_out=None, d_n=None,
                        offsets=None, res_scale=1.0, eps=1e-5, dx=None, dy=None, d_gate=None,
                        d_w_post=None, d_w_pre=None, stream=None):
    """Gradients through ifvs_norm_join from those of x_out and n_out (either
    may be None).  Returns (dx, dy, d_gate, d_w_post, d_w_pre), None where the
    forward call had no such input."""
    at = _on(L, x_out, "x_out", stream)
    p, td, bd, dt = _join_params(x_out, gate, w_post, w_pre, offsets, res_scale, eps, stream, at)
    dx = _like(x_out, stream, *td) if dx is None else dx
    if y is not None:
        dy = _like(x_out, stream, *td) if dy is None else dy
        d_w_post = _like(x_out, stream, td[1]) if d_w_post is None else d_w_post
        if gate is not None and d_gate is None:
            d_gate = _like(x_out, stream, *bd)
    if d_n is not None and d_w_pre is None:
        d_w_pre = _like(x_out, stream, td[1])
    d = td[1:]
    _check(_lib.ifvs_norm_join_grad(
        L, C.byref(p), _dev(x_out, td, dt, "x_out", at), _dev(y, td, dt, "y", at),
        _dev(d_x_out, td, dt, "d_x_out", at), _dev(d_n, td, dt, "d_n", at), _dev(dx, td, dt, "dx", at),
        _dev(dy, td, dt, "dy", at), _dev(d_gate, bd, dt, "d_gate", at), _dev(d_w_post, d, dt, "d_w_post", at),
        _dev(d_w_pre, d, dt, "d_w_pre", at)))
    return dx, dy, d_gate, d_w_post, d_w_pre


def _ffn_params(x, w_in, w_out, act, stream, at=None):
    (T, D), F, dt, at = x.shape, w_out.shape[1], x.dtype, x.get_device() if at is None else at
    if act not in _ACTS:
        raise ValueError("act must be one of %s" % sorted(_ACTS))
    p = FfnParams(T, D, F, _type(x), _ACTS[act], _dev(w_in, (2 * F, D), dt, "w_in", at),
                  _dev(w_out, (D, F), dt, "w_out", at), _stream(stream))
    return p, (T, D), F, dt


def ifvs_ffn(L, x, w_in, w_out, act="silu", y=None, stream=None):
    """y = (act(x Wg^T) * (x Wu^T)) w_out^T, w_in [2F][D] = [Wg; Wu], w_out [D][F]."""
    at = _on(L, x, "x", stream)
    p, td, _, dt = _ffn_params(x, w_in, w_out, act, stream, at)
    y = _like(x, stream, *td) if y is None else y
    _check(_lib.ifvs_ffn(L, C.byref(p), _dev(x, td, dt, "x", at), _dev(y, td, dt, "y", at)))
    return y


def ifvs_ffn_grad(L, x, w_in, w_out, dy, act="silu", dx=None, d_w_in=None, d_w_out=None, stream=None):
    """Gradients (dx, d_w_in, d_w_out) through ifvs_ffn from dy."""
    at = _on(L, x, "x", stream)
    p, td, F, dt = _ffn_params(x, w_in, w_out, act, stream, at)
    dx = _like(x, stream, *td) if dx is None else dx
    d_w_in = _like(x, stream, 2 * F, td[1]) if d_w_in is None else d_w_in
    d_w_out = _like(x, stream, td[1], F) if d_w_out is None else d_w_out
    _check(_lib.ifvs_ffn_grad(L, C.byref(p), _dev(x, td, dt, "x", at), _dev(dy, td, dt, "dy", at),
                              _dev(dx, td, dt, "dx", at), _dev(d_w_in, (2 * F, td[1]), dt, "d_w_in", at),
                              _dev(d_w_out, (td[1], F), dt, "d_w_out", at)))
    return dx, d_w_in, d_w_out


def _linear_params(x, w, bias, act, stream, at):
    (T, D_in), D_out, dt = x.shape, w.shape[0], x.dtype
    if act not in _ANY_ACT:
        raise ValueError("act must be one of %s" % sorted(_ANY_ACT))
    p = LinearParams(T, D_in, D_out, _type(x), _ANY_ACT[act], _dev(w, (D_out, D_in), dt, "w", at),
                     _dev(bias, (D_out,), dt, "bias", at), _stream(stream))
    return p, (T, D_in), (T, D_out), dt


def ifvs_linear(L, x, w, bias=None, act="none", residual=None, y=None, stream=None):
    """y = act(x w^T + bias) + residual, w [D_out][D_in]."""
    at = _on(L, x, "x", stream)
    p, ti, to, dt = _linear_params(x, w, bias, act, stream, at)
    y = _like(x, stream, *to) if y is None else y
    _check(_lib.ifvs_linear(L, C.byref(p), _dev(x, ti, dt, "x", at), _dev(residual, to, dt, "residual", at),
                            _dev(y, to, dt, "y", at)))
    return y


def ifvs_linear_grad(L, x, w, dy, bias=None, act="none", dx=None, d_w=None, d_bias=None, stream=None):
    """Gradients (dx, d_w, d_bias) through ifvs_linear from dy, which is the
    residual's own; d_bias None without a bias."""
    at = _on(L, x, "x", stream)
    p, ti, to, dt = _linear_params(x, w, bias, act, stream, at)
    dx = _like(x, stream, *ti) if dx is None else dx
    d_w = _like(x, stream, to[1], ti[1]) if d_w is None else d_w
    if bias is not None and d_bias is None:
        d_bias = _like(x, stream, to[1])
    _check(_lib.ifvs_linear_grad(L, C.byref(p), _dev(x, ti, dt, "x", at), _dev(dy, to, dt, "dy", at),
                                 _dev(dx, ti, dt, "dx", at), _dev(d_w, (to[1], ti[1]), dt, "d_w", at),
                                 _dev(d_bias, to[1:], dt, "d_bias", at)))
    return dx, d_w, d_bias


def _heads(a, shape, dtype, name, at):
    """Address and row stride of a tensor [tokens][heads][dh] whose rows may have gaps."""
    if a.shape != shape or a.dtype != dtype:
        raise ValueError("%s is %s %s, expected %s %s" % (name, tuple(a.shape), a.dtype, shape, dtype))
    if a.get_device() != at:
        raise ValueError("%s must be a tensor on cuda:%d" % (name, at))
    (T, H, d), ld = shape, 0
    if not a.is_contiguous():
        s = a.stride()
        if s[2] != 1 or (H > 1 and s[1] != d) or (T > 1 and (s[0] < H * d or s[0] % 8)):
            raise ValueError("%s must hold a token's heads without gaps, its rows a multiple of 8 elements apart" % name)
        ld = s[0] if T > 1 else 0
    return a.data_ptr() or 256, ld


def _offsets(a, name, at):
    if a is None:
        return 1, None
    n = a.shape[0] if _is_vector(a, "int64") else 0
    if n < 2:
        raise ValueError("%s must be a vector of B + 1 int64" % name)
    if a.get_device() != at or not a.is_contiguous():
        raise ValueError("%s must be a contiguous tensor on cuda:%d" % (name, at))
    return n - 1, a.data_ptr()


def _attend_params(q, k, v, q_offsets, kv_offsets, kv_ids, scale, stream, at):
    """The params and the addresses of q, k and v"""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v must be [tokens][heads][dh]")
    (Tq, H, d), (Tk, Hk, _), dt = q.shape, k.shape, q.dtype
    (B, qo), (Bk, ko) = _offsets(q_offsets, "q_offsets", at), _offsets(kv_offsets, "kv_offsets", at)
    if B != Bk:
        raise ValueError("q_offsets delimit %d sequences, kv_offsets %d" % (B, Bk))
    p = AttendParams(Tq, Tk, H, Hk, d, _type(q), B, qo, ko)
    if kv_ids is not None:
        if _ids(kv_ids) != Tk:
            raise ValueError("%d kv_ids for %d keys" % (kv_ids.shape[0], Tk))
        p.kv_ids = _dev(kv_ids, (Tk,), kv_ids.dtype, "kv_ids", at)
    p.scale = d ** -0.5 if scale is None else scale
    p.stream = _stream(stream)
    shapes = (Tq, H, d), (Tk, Hk, d)
    ptr = [0, 0, 0]
    ptr[0], p.ld_q = _heads(q, shapes[0], dt, "q", at)
    ptr[1], p.ld_k = _heads(k, shapes[1], dt, "k", at)
    ptr[2], p.ld_v = _heads(v, shapes[1], dt, "v", at)
    return p, ptr, shapes, dt


def _lse(lse, shape, at):
    if lse is None:
        return None
    import torch
    return _dev(lse, shape, torch.float32, "lse", at)


def ifvs_attend(L, q, k, v, q_offsets=None, kv_offsets=None, kv_ids=None, scale=None, out=None, lse=None, stream=None):
    """out = softmax(scale q k) v for queries [Tq][heads][dh] and the keys and values
    [Tk][kv_heads][dh] of their sequence, which the offsets delimit; keys whose id is
    negative are padding.  scale: dh^-1/2 by default.  Rows may have gaps (k and v
    halves of one tensor).  lse: True or a tensor [Tq][heads] of float32 for the
    logarithm of the softmax's sum, which the gradient takes.  Returns (out, lse)."""
    at = _on(L, q, "q", stream)
    p, ptr, (sq, _), dt = _attend_params(q, k, v, q_offsets, kv_offsets, kv_ids, scale, stream, at)
    out = _like(q, stream, *sq) if out is None else out
    if lse is True:
        import torch
        lse = _like(q, stream, *sq[:2], dtype=torch.float32)
    elif lse is False:
        lse = None
    to, p.ld_out = _heads(out, sq, dt, "out", at)
    _check(_lib.ifvs_attend(L, C.byref(p), *ptr, to, _lse(lse, sq[:2], at)))
    return out, lse


def ifvs_attend_grad(L, q, k, v, out, lse, d_out, q_offsets=None, kv_offsets=None, kv_ids=None, scale=None, dq=None,
                     dk=None, dv=None, stream=None):
    """Gradients (dq, dk, dv) through ifvs_attend from d_out; out and lse as the forward
    call with the same arguments returned them."""
    at = _on(L, q, "q", stream)
    p, ptr, (sq, sk), dt = _attend_params(q, k, v, q_offsets, kv_offsets, kv_ids, scale, stream, at)
    dq = _like(q, stream, *sq) if dq is None else dq
    dk = _like(q, stream, *sk) if dk is None else dk
    dv = _like(q, stream, *sk) if dv is None else dv
    o, p.ld_out = _heads(out, sq, dt, "out", at)
    do, p.ld_d_out = _heads(d_out, sq, dt, "d_out", at)
    to = [0, 0, 0]
    to[0], p.ld_dq = _heads(dq, sq, dt, "dq", at)
    to[1], p.ld_dk = _heads(dk, sk, dt, "dk", at)
    to[2], p.ld_dv = _heads(dv, sk, dt, "dv", at)
    _check(_lib.ifvs_attend_grad(L, C.byref(p), *ptr, o, _lse(lse, sq[:2], at), do, *to))
    return dq, dk, dv


def ifvs_dropout(L, x, p, seed, step=0, residual=None, out=None, stream=None):
    """out = residual + (x / (1 - p) where its random word is at least p 2^32, else
    0), for a tensor of any shape; the words are those of (seed, step).  Of a
    gradient the same call without the residual.  step: a number, or a tensor of one
    int64 on the device that is read when the call runs; seed and number mod 2^64."""
    at = _on(L, x, "x", stream)
    more = None
    if not isinstance(step, int):
        if not _is_vector(step, "int64"):
            raise ValueError("step must be an int or a vector of one int64")
        more, step = _dev(step, (1,), step.dtype, "step", at), 0
    out = _like(x, stream, *x.shape) if out is None else out
    _check(_lib.ifvs_dropout(L, _dev(x, x.shape, x.dtype, "x", at), _dev(residual, x.shape, x.dtype, "residual", at),
                             x.numel(), _type(x), p, seed & _MASK64, step & _MASK64, more,
                             _dev(out, x.shape, x.dtype, "out", at), _stream(stream)))
    return out


def ifvs_rerank(ix, queries, cand, k, flags=0):
    queries = _host(queries, np.float32)
    cand = _host(cand, np.int64)
    nq, R = cand.shape
    ids = np.empty((nq, k), np.int64)
    dists = np.empty((nq, k), np.float32)
    p = _params(flags)
    _check(_lib.ifvs_rerank(ix, _ptr(queries), _ptr(cand), nq, R, k, C.byref(p), _ptr(ids),
                            _ptr(dists)))
    return ids, dists


def ifvs_stage_times(ix, reset=False):
    ms = np.zeros(IFVS_N_STAGES, np.float64)
    n = np.zeros(IFVS_N_STAGES, np.int64)
    _check(_lib.ifvs_stage_times(ix, _ptr(ms), _ptr(n), 1 if reset else 0))
    return {s: (float(ms[i]), int(n[i])) for i, s in enumerate(STAGES)}


def ifvs_canonical_predicate(pred, attr_types):
    pred = np.ascontiguousarray(np.asarray(pred).reshape(1))
    ty = np.ascontiguousarray(attr_types, dtype=np.int32)
    n = len(ty)
    lo = np.zeros(max(n, 1), np.int32)
    wm1 = np.zeros(max(n, 1), np.uint32)
    empty = C.c_int32(0)
    _check(_lib.ifvs_canonical_predicate(_ptr(pred), _ptr(ty), n, _ptr(lo), _ptr(wm1),
                                         C.byref(empty)))
    return lo[:n], wm1[:n], bool(empty.value)


def ifvs_index_info(ix):
    out = np.zeros(8, np.int64)
    _check(_lib.ifvs_index_info(ix, _ptr(out)))
    keys = ("N", "M", "K", "D", "ds", "n_attrs", "has_codebooks", "device_bytes")
    return {k: int(v) for k, v in zip(keys, out)}


def ifvs_free(ix):
    _lib.ifvs_free(ix)


class Index:
    """Owns an ifvs_index handle (freed on close / garbage collection)."""

    def __init__(self, codes, attrs, vectors=None, D=0, device=0, K=256, device_io=False):
        self.h = ifvs_load_index(codes, attrs, vectors, D, device, K, device_io)
        self.N, self.M = int(codes.shape[0]), int(codes.shape[1])
        self.K = K
        self._bank_shape = self._W_shape = None

    def load_codebooks(self, C_pq, bank=None, W=None, hash_seeds=None):
        ifvs_load_codebooks(self.h, C_pq, bank=bank, W=W, hash_seeds=hash_seeds)
        self.ds = int(np.asarray(C_pq).shape[2])
        self.r = 0 if W is None else int(np.asarray(W).shape[1])
        self.hh = 0 if hash_seeds is None else len(hash_seeds)
        if bank is not None:
            self._bank_shape = (int(bank.shape[0]), self.M * self.r)
            self._W_shape = (self.M, self.r, self.K, self.ds)
        else:
            self._bank_shape = self._W_shape = None
        return self

    def search(self, queries, preds, k, wz=None, **kw):
        return ifvs_search_batch(self.h, queries, preds, k, wz=wz, **kw)

    def filter(self, preds, **kw):
        return ifvs_filter(self.h, preds, self.N, **kw)

    def condition(self, queries, preds, wz=None, **kw):
        return ifvs_condition(self.h, queries, preds, wz, M=self.M, K=self.K, ds=self.ds,
                              h=self.hh, r=self.r, **kw)

    def scan_topk(self, lut, bitmaps, k, **kw):
        return ifvs_scan_topk(self.h, lut, bitmaps, k, **kw)

    def rerank(self, queries, cand, k, **kw):
        return ifvs_rerank(self.h, queries, cand, k, **kw)

    def _cond_shapes(self):
        if self._bank_shape is None:
            raise IfvsError(IFVS_ERR_STATE, "no memory bank loaded")
        return self._bank_shape, self._W_shape

    def train_grad(self, queries, preds, wz, cand, n_pos, tau, lam, **kw):
        (B, Mr), Ws = self._cond_shapes()
        return ifvs_train_grad(self.h, queries, preds, wz, cand, n_pos, tau, lam, B, Mr, Ws, **kw)

    def train_step(self, queries, preds, wz, positives, n_neg, tau, lam, lr, **kw):
        return ifvs_train_step(self.h, queries, preds, wz, positives, n_neg, tau, lam, lr, **kw)

    def conditioning(self):
        (B, Mr), Ws = self._cond_shapes()
        return ifvs_get_conditioning(self.h, B, Mr, Ws)

    def stage_times(self, reset=False):
        return ifvs_stage_times(self.h, reset)

    def info(self):
        return ifvs_index_info(self.h)

    def close(self):
        if getattr(self, "h", None):
            ifvs_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Layers:
    """Owns an ifvs_layers handle: the layers of a predicate encoder on one
    device (freed on close / garbage collection).  With ``stream`` a call is
    enqueued there (inputs ready in its order and kept until its work is done);
    without, it follows torch's current stream and waits for its outputs."""

    def __init__(self, device=0):
        self.h = ifvs_layers_create(device)
        # the functions above with this handle as their first argument
        self.embed = functools.partial(ifvs_embed, self.h)
        self.embed_grad = functools.partial(ifvs_embed_grad, self.h)
        self.norm_join = functools.partial(ifvs_norm_join, self.h)
        self.norm_join_grad = functools.partial(ifvs_norm_join_grad, self.h)
        self.ffn = functools.partial(ifvs_ffn, self.h)
        self.ffn_grad = functools.partial(ifvs_ffn_grad, self.h)
        self.linear = functools.partial(ifvs_linear, self.h)
        self.linear_grad = functools.partial(ifvs_linear_grad, self.h)
        self.attend = functools.partial(ifvs_attend, self.h)
        self.attend_grad = functools.partial(ifvs_attend_grad, self.h)
        self.dropout = functools.partial(ifvs_dropout, self.h)

    def status(self):
        """Waits for the enqueued calls; raises what their kernels found."""
        ifvs_layers_status(self.h)

    def close(self):
        if getattr(self, "h", None):
            ifvs_layers_free(self.h)
            self.h.value = None      # the bound functions refuse it from here on
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
