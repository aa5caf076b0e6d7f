"""ctypes binding of librfast.so: argument marshalling only.

Every step of the R-FAST activation path runs inside the CUDA library; this module turns
numpy arrays into the plain pointers of include/rfast.h and back.  The functions carry the
names of the C entry points.  There is no fallback: if the shared library is missing, or no
CUDA device is present, the calls raise.
"""

from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librfast.so")

OK, EINVAL, EGRAPH, ESCHED, ENOMEM, ECUDA, ETIMEOUT, ESTATE = 0, -1, -2, -3, -4, -5, -6, -7
_ERRNAMES = {-1: "EINVAL", -2: "EGRAPH", -3: "ESCHED", -4: "ENOMEM", -5: "ECUDA", -6: "ETIMEOUT", -7: "ESTATE"}

MODEL_IDS = {"quad_diag": 0, "least_squares": 1, "softmax": 2, "mlp": 3, "logistic_sparse": 4}

STATE_X, STATE_Y, STATE_G_LAST, STATE_RHO_LATEST, STATE_RHO_BUF = 0, 1, 2, 3, 4
STATE_T_LOCAL, STATE_USED_TAU_V, STATE_USED_TAU_RHO, STATE_TAU_V_END, STATE_TAU_RHO_END, STATE_ROUND = 5, 6, 7, 8, 9, 10
Q_ROUND, Q_EVENTS_TOTAL, Q_EVENTS_RUN, Q_LAUNCHES, Q_BYTES_RUN, Q_V_SLOTS, Q_RHO_SLOTS = 0, 1, 2, 3, 4, 5, 6
Q_DEVICE_BYTES, Q_N_USED_TAU_V, Q_N_USED_TAU_RHO, Q_BYTES_TOTAL = 7, 8, 9, 10
Q_METHOD_BYTES_RUN, Q_METHOD_BYTES_TOTAL = 11, 12
STATE_V_LATEST, STATE_V_HELD, STATE_TAU_V, STATE_TAU_RHO = 11, 12, 13, 14
STATE_ADAM_M, STATE_ADAM_V = 15, 16
_FLOAT_VIEWS = (STATE_X, STATE_Y, STATE_G_LAST, STATE_RHO_LATEST, STATE_RHO_BUF, STATE_V_LATEST, STATE_ADAM_M, STATE_ADAM_V)
DESCENT_IDS = {"plain": 0, "adamw": 1, "adamw8": 2}
NOT_HELD = 1
GRAPH_R, GRAPH_C = 0, 1


class RFastError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"rfast: {_ERRNAMES.get(code, code)}: {msg}")
        self.code = code


class _Graph(C.Structure):
    _fields_ = [("n_edges", C.c_int32), ("rowptr", C.c_void_p), ("col", C.c_void_p),
                ("w", C.c_void_p), ("diag", C.c_void_p)]


class _Problem(C.Structure):
    _fields_ = [("n", C.c_int32), ("root", C.c_int32), ("p", C.c_int64), ("alpha", C.c_float),
                ("l2", C.c_float), ("G_R", _Graph), ("G_C", _Graph), ("model", C.c_int32),
                ("batch", C.c_int32), ("rows", C.c_int32), ("n_features", C.c_int32),
                ("n_classes", C.c_int32), ("n_hidden", C.c_int32),
                ("quad_d", C.c_void_p), ("quad_b", C.c_void_p), ("feat", C.c_void_p),
                ("target", C.c_void_p), ("label", C.c_void_p), ("sp_rowptr", C.c_void_p),
                ("sp_col", C.c_void_p), ("sp_val", C.c_void_p), ("x0", C.c_void_p),
                ("compensated", C.c_int32), ("tracker", C.c_int32),
                ("norm_groups", C.c_int32), ("norm_act", C.c_int32), ("norm_eps", C.c_double), ("descent", C.c_int32),
                ("beta1", C.c_double), ("beta2", C.c_double), ("adam_eps", C.c_double), ("weight_decay", C.c_double)]


class _Schedule(C.Structure):
    _fields_ = [("K", C.c_int32), ("act_ptr", C.c_void_p), ("act_node", C.c_void_p),
                ("n_send_r", C.c_int64), ("send_r", C.c_void_p), ("n_send_c", C.c_int64),
                ("send_c", C.c_void_p), ("n_batch_idx", C.c_int64), ("batch_idx", C.c_void_p),
                ("alpha_round", C.c_void_p)]


TYPE_IDS = {"f32": 0, "bf16": 1, "f16": 2}
ACT_IDS = {"none": 0, "relu": 1, "silu": 2}
GRAD_NORM_WORKSPACE = 16384
ADAMW_BLOCK = 256


class _AdamW(C.Structure):
    _fields_ = [("n_tensors", C.c_int32), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("state_bits", C.c_int32),
                ("numel", C.c_void_p), ("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("step", C.c_int64), ("d_step", C.c_void_p), ("d_grad_scale", C.c_void_p)]


class _GnShape(C.Structure):
    _fields_ = [("samples", C.c_int64), ("positions", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32),
                ("samples_per_set", C.c_int64), ("type", C.c_int32), ("act", C.c_int32)]


class _EmbShape(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("vocab", C.c_int64), ("width", C.c_int32), ("token_bits", C.c_int32), ("table_type", C.c_int32),
                ("out_type", C.c_int32)]


class _Policy(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("vocab", C.c_int64), ("type", C.c_int32), ("token_bits", C.c_int32),
                ("d_logits", C.c_void_p), ("logits_stride", C.c_int64), ("d_tokens", C.c_void_p), ("d_old_logp", C.c_void_p),
                ("d_ref_logp", C.c_void_p), ("d_advantage", C.c_void_p), ("d_weight", C.c_void_p), ("d_loss_scale", C.c_void_p),
                ("temperature", C.c_double), ("clip_low", C.c_double), ("clip_high", C.c_double), ("kl_coef", C.c_double),
                ("d_loss", C.c_void_p), ("d_token_loss", C.c_void_p), ("d_logp", C.c_void_p), ("d_dlogits", C.c_void_p),
                ("dlogits_stride", C.c_int64)]


class _Muon(C.Structure):
    _fields_ = [("n_tensors", C.c_int32), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("terms", C.c_int32),
                ("rows", C.c_void_p), ("cols", C.c_void_p), ("param", C.c_void_p), ("grad", C.c_void_p), ("momentum", C.c_void_p),
                ("lr", C.c_double), ("momentum_beta", C.c_double), ("weight_decay", C.c_double), ("eps", C.c_double),
                ("nesterov", C.c_int32), ("iterations", C.c_int32), ("size_rule", C.c_int32), ("d_grad_scale", C.c_void_p)]


SIZE_RULES = {"spectral": 0, "rms": 1}

_lib = None


def lib():
    """The loaded shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                               "(python -m paper_2307_11617_b200.build); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        L.rfast_create.argtypes = [C.POINTER(_Problem), C.c_void_p, C.POINTER(C.c_void_p)]
        L.rfast_load_schedule.argtypes = [C.c_void_p, C.POINTER(_Schedule)]
        L.rfast_append_schedule.argtypes = [C.c_void_p, C.POINTER(_Schedule)]
        L.rfast_compile_append_check.argtypes = [C.POINTER(_Problem), C.POINTER(_Schedule), C.POINTER(_Schedule),
                                                 C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_run.argtypes = [C.c_void_p, C.c_int32, C.c_int]
        L.rfast_read_state.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_size_t]
        L.rfast_reset.argtypes = [C.c_void_p]
        L.rfast_sync.argtypes = [C.c_void_p]
        L.rfast_query.argtypes = [C.c_void_p, C.c_int]
        L.rfast_query.restype = C.c_int64
        L.rfast_destroy.argtypes = [C.c_void_p]
        L.rfast_destroy.restype = None
        L.rfast_last_error.argtypes = [C.c_void_p]
        L.rfast_last_error.restype = C.c_char_p
        L.rfast_version.restype = C.c_char_p
        L.rfast_compile_host.argtypes = [C.POINTER(_Problem), C.POINTER(_Schedule)] + [C.c_void_p] * 5 + \
            [C.c_char_p, C.c_size_t]
        L.rfast_compile_digest.argtypes = [C.POINTER(_Problem), C.POINTER(_Schedule), C.POINTER(C.c_uint64), C.c_char_p, C.c_size_t]
        L.rfast_set_option.argtypes = [C.c_void_p, C.c_int, C.c_int64]
        L.rfast_checkpoint_size.argtypes = [C.c_void_p]
        L.rfast_checkpoint_size.restype = C.c_int64
        L.rfast_checkpoint_save.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        L.rfast_checkpoint_load.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        L.rfast_diagnostics.argtypes = [C.c_void_p, C.c_void_p, C.c_int32]
        L.rfast_seek.argtypes = [C.c_void_p, C.c_int32]
        L.rfast_snapshot.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.rfast_snapshot_wait.argtypes = [C.c_void_p]
        L.rfast_write_state.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_size_t]
        L.rfast_read_packet.argtypes = [C.c_void_p, C.c_int, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t]
        L.rfast_write_packet.argtypes = [C.c_void_p, C.c_int, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t]
        L.rfast_ls_gradient_static.argtypes = [C.c_void_p] * 4 + [C.c_int32, C.c_int32, C.c_float,
                                               C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_grad_norm.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_group_norm_workspace.argtypes = [C.POINTER(_GnShape), C.c_int]
        L.rfast_group_norm_workspace.restype = C.c_int64
        L.rfast_group_norm.argtypes = [C.POINTER(_GnShape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_group_norm_backward.argtypes = [C.POINTER(_GnShape)] + [C.c_void_p] * 13 + [C.c_size_t, C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_adamw_step.argtypes = [C.POINTER(_AdamW), C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_embedding.argtypes = [C.POINTER(_EmbShape), C.c_void_p, C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_int64,
                                      C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_embedding_workspace.argtypes = [C.POINTER(_EmbShape)]
        L.rfast_embedding_workspace.restype = C.c_int64
        L.rfast_embedding_backward.argtypes = [C.POINTER(_EmbShape), C.c_void_p, C.c_void_p, C.c_int64, C.c_float, C.c_int, C.c_void_p, C.c_int64,
                                               C.c_void_p, C.c_size_t, C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_muon_workspace.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32]
        L.rfast_muon_workspace.restype = C.c_int64
        L.rfast_muon_step.argtypes = [C.POINTER(_Muon), C.c_void_p, C.c_size_t, C.c_void_p, C.c_char_p, C.c_size_t]
        L.rfast_policy_loss.argtypes = [C.POINTER(_Policy), C.c_void_p, C.c_char_p, C.c_size_t]
        _lib = L
    return _lib


def _arr(a, dtype):
    return np.ascontiguousarray(a, dtype=dtype)


def _ptr(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _graph(g, keep):
    rowptr, col = _arr(g.rowptr, np.int32), _arr(g.col, np.int32)
    w, diag = _arr(g.w, np.float32), _arr(g.diag, np.float32)
    keep += [rowptr, col, w, diag]
    return _Graph(len(col), _ptr(rowptr), _ptr(col), _ptr(w), _ptr(diag))


def _problem(wl, keep):
    """wl: object with n, p, root, alpha, l2, G_R, G_C, model (name), batch, rows, dims, data, x0."""
    P = _Problem()
    P.n, P.root, P.p, P.alpha, P.l2 = int(wl.n), int(wl.root), int(wl.p), float(wl.alpha), float(wl.l2)
    P.G_R, P.G_C = _graph(wl.G_R, keep), _graph(wl.G_C, keep)
    P.model = MODEL_IDS[wl.model] if isinstance(wl.model, str) else int(wl.model)
    P.batch, P.rows = int(wl.batch), int(wl.rows)
    P.compensated = int(getattr(wl, "compensated", 0) or 0)     # False/True/2 -> 0/1/2
    P.tracker = int(getattr(wl, "tracker", 0) or 0)             # 0 running sums, 1 mass buckets
    dims = getattr(wl, "dims", {}) or {}
    P.n_features = int(dims.get("n_features", 0))
    P.n_classes = int(dims.get("n_classes", 0))
    P.n_hidden = int(dims.get("n_hidden", 0))
    P.norm_groups = int(dims.get("norm_groups", 0))             # group norm in the MLP's hidden layer
    P.norm_act = ACT_IDS[dims.get("norm_act", "relu")]
    P.norm_eps = float(dims.get("norm_eps", 1e-5))
    descent = getattr(wl, "descent", None) or {}                # {"kind": "adamw" | "adamw8", "beta1": ..., ...}
    P.descent = DESCENT_IDS[descent.get("kind", "plain")]
    P.beta1, P.beta2 = float(descent.get("beta1", 0.9)), float(descent.get("beta2", 0.999))
    P.adam_eps, P.weight_decay = float(descent.get("eps", 1e-8)), float(descent.get("weight_decay", 0.0))
    data = getattr(wl, "data", {}) or {}
    spec = {"quad_d": ("d", np.float32), "quad_b": ("b", np.float32), "feat": ("feat", np.float32),
            "target": ("target", np.float32), "label": ("label", np.int32),
            "sp_rowptr": ("sp_rowptr", np.int64), "sp_col": ("sp_col", np.int32),
            "sp_val": ("sp_val", np.float32)}
    for field, (key, dt) in spec.items():
        if key in data and data[key] is not None:
            a = _arr(data[key], dt)
            keep.append(a)
            setattr(P, field, _ptr(a))
    if getattr(wl, "x0", None) is not None:
        a = _arr(wl.x0, np.float32)
        keep.append(a)
        P.x0 = _ptr(a)
    return P


def _schedule(s, keep):
    S = _Schedule()
    act_ptr, act_node = _arr(s.act_ptr, np.int32), _arr(s.act_node, np.int32)
    send_r, send_c = _arr(s.send_r, np.int8), _arr(s.send_c, np.int8)
    bidx = _arr(s.batch_idx, np.int32)
    keep += [act_ptr, act_node, send_r, send_c, bidx]
    S.K = int(s.K)
    S.act_ptr, S.act_node = _ptr(act_ptr), _ptr(act_node)
    S.n_send_r, S.send_r = len(send_r), _ptr(send_r)
    S.n_send_c, S.send_c = len(send_c), _ptr(send_c)
    S.n_batch_idx, S.batch_idx = len(bidx), _ptr(bidx)
    if getattr(s, "alpha_round", None) is not None:
        ar = _arr(s.alpha_round, np.float32)
        if len(ar) != int(s.K):
            raise ValueError("alpha_round must hold one step size per round")
        keep.append(ar)
        S.alpha_round = _ptr(ar)
    return S


def _check(rc, handle=None):
    if rc != OK:
        raise RFastError(rc, lib().rfast_last_error(handle).decode())


def rfast_version() -> str:
    return lib().rfast_version().decode()


def rfast_create(wl, cuda_stream: int = 0) -> int:
    """Returns an opaque handle.  cuda_stream: a cudaStream_t as an integer (0: default stream)."""
    keep = []
    P = _problem(wl, keep)
    h = C.c_void_p()
    _check(lib().rfast_create(C.byref(P), C.c_void_p(cuda_stream), C.byref(h)))
    return h.value


def rfast_load_schedule(handle, s) -> None:
    keep = []
    S = _schedule(s, keep)
    _check(lib().rfast_load_schedule(handle, C.byref(S)), handle)


def rfast_append_schedule(handle, more) -> None:
    keep = []
    S = _schedule(more, keep)
    _check(lib().rfast_append_schedule(handle, C.byref(S)), handle)


def rfast_run(handle, rounds: int, sync: bool = True) -> None:
    _check(lib().rfast_run(handle, int(rounds), 1 if sync else 0), handle)


def rfast_reset(handle) -> None:
    _check(lib().rfast_reset(handle), handle)


def rfast_sync(handle) -> None:
    _check(lib().rfast_sync(handle), handle)


def rfast_query(handle, what: int) -> int:
    v = lib().rfast_query(handle, int(what))
    if v < 0:
        _check(int(v), handle)
    return int(v)


def rfast_read_state(handle, which: int, shape, out=None) -> np.ndarray:
    """shape: the view's shape; float views are float32, integer views int32."""
    dt = np.float32 if which in _FLOAT_VIEWS else np.int32
    if out is None:
        out = np.empty(shape, dtype=dt)
    assert out.dtype == dt and out.flags.c_contiguous
    _check(lib().rfast_read_state(handle, int(which), _ptr(out), out.nbytes), handle)
    return out


def rfast_snapshot(handle, x_out: np.ndarray, y_out: np.ndarray) -> None:
    """x_out, y_out: C-contiguous float32 [n][p] host arrays (page-locked for an overlapped transfer)
    that must stay alive until rfast_snapshot_wait."""
    for a in (x_out, y_out):
        if a.dtype != np.float32 or not a.flags["C_CONTIGUOUS"]:
            raise ValueError("snapshot destinations must be C-contiguous float32 arrays")
    _check(lib().rfast_snapshot(handle, _ptr(x_out), _ptr(y_out)), handle)


def rfast_snapshot_wait(handle) -> None:
    _check(lib().rfast_snapshot_wait(handle), handle)


def rfast_seek(handle, rnd: int) -> None:
    _check(lib().rfast_seek(handle, int(rnd)), handle)


def rfast_write_state(handle, which: int, values) -> None:
    """values: the float view as an array (converted to contiguous float32)."""
    a = _arr(values, np.float32)
    _check(lib().rfast_write_state(handle, int(which), _ptr(a), a.nbytes), handle)


def rfast_read_packet(handle, graph: int, ident: int, stamp: int, p: int):
    """Payload (float32 [p]) of one packet version, or None when the engine does not hold it."""
    out = np.empty(int(p), dtype=np.float32)
    rc = lib().rfast_read_packet(handle, int(graph), int(ident), int(stamp), _ptr(out), out.nbytes)
    if rc == NOT_HELD:
        return None
    _check(rc, handle)
    return out


def rfast_write_packet(handle, graph: int, ident: int, stamp: int, values) -> bool:
    """True when the version is held and was written, False when the engine keeps no row for it."""
    a = _arr(values, np.float32)
    rc = lib().rfast_write_packet(handle, int(graph), int(ident), int(stamp), _ptr(a), a.nbytes)
    if rc == NOT_HELD:
        return False
    _check(rc, handle)
    return True


def rfast_destroy(handle) -> None:
    lib().rfast_destroy(handle)


def rfast_compile_host(wl, s):
    """Host-only schedule compilation (no device needed).  Returns a dict of int arrays."""
    keep = []
    P, S = _problem(wl, keep), _schedule(s, keep)
    indeg_r = np.diff(np.asarray(wl.G_R.rowptr)).astype(np.int64)
    indeg_c = np.diff(np.asarray(wl.G_C.rowptr)).astype(np.int64)
    nodes = np.clip(np.asarray(s.act_node, dtype=np.int64), 0, int(wl.n) - 1)   # bad ids are the library's to reject
    ev = len(nodes)
    used_v = np.empty(int(indeg_r[nodes].sum()), np.int32)
    used_r = np.empty(int(indeg_c[nodes].sum()), np.int32)
    v_ver = np.empty((ev, 3), np.int32)
    rho_ver = np.empty((len(s.send_c), 3), np.int32)
    counts = np.zeros(4, np.int64)
    err = C.create_string_buffer(512)
    rc = lib().rfast_compile_host(C.byref(P), C.byref(S), _ptr(used_v), _ptr(used_r), _ptr(v_ver),
                                  _ptr(rho_ver), _ptr(counts), err, 512)
    if rc != OK:
        raise RFastError(rc, err.value.decode())
    return {"used_tau_v": used_v, "used_tau_rho": used_r, "v_ver": v_ver, "rho_ver": rho_ver,
            "v_rows": int(counts[0]), "rho_rows": int(counts[1]), "events": int(counts[2]),
            "streams": int(counts[3])}


def rfast_compile_digest(wl, s) -> int:
    """One number for everything the compiled schedule drives the kernels with (host only)."""
    keep = []
    P, S = _problem(wl, keep), _schedule(s, keep)
    out = C.c_uint64(0)
    err = C.create_string_buffer(512)
    rc = lib().rfast_compile_digest(C.byref(P), C.byref(S), C.byref(out), err, 512)
    if rc != OK:
        raise RFastError(rc, err.value.decode())
    return int(out.value)


def rfast_compile_append_check(wl, first, more):
    """Host only: `first` loaded open-ended and `more` appended keeps every row of `first` in place
    and consumes the stamps of the whole schedule.  Returns the six row counts; raises otherwise."""
    keep = []
    P, S1, S2 = _problem(wl, keep), _schedule(first, keep), _schedule(more, keep)
    counts = np.zeros(6, np.int64)
    err = C.create_string_buffer(512)
    rc = lib().rfast_compile_append_check(C.byref(P), C.byref(S1), C.byref(S2), _ptr(counts), err, 512)
    if rc != OK:
        raise RFastError(rc, err.value.decode())
    return {"first": (int(counts[0]), int(counts[1])), "appended": (int(counts[2]), int(counts[3])),
            "whole": (int(counts[4]), int(counts[5]))}


OPT_PERSISTENT, OPT_GRAPHS, OPT_WAIT_LIMIT_MS, OPT_PHANTOM_ARRIVALS, OPT_ONE_PASS, OPT_CLUSTER_SIZE, OPT_OPEN_END = 0, 1, 2, 3, 4, 5, 6


def rfast_set_option(handle, option: int, value: int) -> None:
    _check(lib().rfast_set_option(handle, int(option), int(value)), handle)


def rfast_checkpoint_save(handle) -> np.ndarray:
    """The handle's complete state as an opaque byte array (see rfast_checkpoint_save in rfast.h)."""
    size = lib().rfast_checkpoint_size(handle)
    if size < 0:
        _check(int(size), handle)
    blob = np.empty(size, dtype=np.uint8)
    _check(lib().rfast_checkpoint_save(handle, _ptr(blob), blob.nbytes), handle)
    return blob


def rfast_checkpoint_load(handle, blob: np.ndarray) -> None:
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    _check(lib().rfast_checkpoint_load(handle, _ptr(blob), blob.nbytes), handle)


def rfast_diagnostics(handle, full: bool = True) -> dict:
    """Consensus error, norm of the mean iterate, conservation residual (Lemma 3) and its scale,
    tracker norm, all computed on the device in one pass over the state; with full=True also the
    full gradient, the merit function and the objective at the mean iterate (a pass over every
    row of every shard)."""
    n_out = 8 if full else 5
    out = np.full(8, np.nan, dtype=np.float64)
    _check(lib().rfast_diagnostics(handle, _ptr(out), n_out), handle)
    return {"consensus_error": out[0], "xbar_norm": out[1], "conservation_residual": out[2],
            "gradient_sum_max": out[3], "tracker_norm": out[4], "full_gradient_norm": out[5],
            "merit": out[6], "objective": out[7]}


STATIC_MAX_ROWS = 65536


def rfast_ls_gradient_static(d_feat: int, d_target: int, d_x: int, d_grad: int, rows: int,
                             n_features: int, l2: float = 0.0, cuda_stream: int = 0) -> None:
    """Full-shard least-squares gradient without any device allocation, for callers that may not
    allocate (a framework that owns all GPU memory, a loop that cannot afford cudaMalloc's
    device-wide synchronisation).  All four arguments are raw DEVICE addresses (integers) of
    caller-owned fp32 arrays: feat [rows][n_features], target [rows], x [n_features] in, grad
    [n_features] out.  Enqueued on cuda_stream; the caller synchronises.  At most
    STATIC_MAX_ROWS rows; calls that overlap on the GPU race on the shared built-in scratch."""
    err = C.create_string_buffer(256)
    rc = lib().rfast_ls_gradient_static(C.c_void_p(d_feat), C.c_void_p(d_target), C.c_void_p(d_x),
                                        C.c_void_p(d_grad), int(rows), int(n_features), float(l2),
                                        C.c_void_p(cuda_stream), err, 256)
    if rc != OK:
        raise RFastError(rc, err.value.decode())


def _type(name):
    if name not in TYPE_IDS:
        raise ValueError(f"unknown type {name!r}: one of {', '.join(TYPE_IDS)}")
    return TYPE_IDS[name]


def _list(values, n=None, what="list"):
    """Sizes or device addresses of a list of tensors as a host array of 64-bit integers."""
    a = np.ascontiguousarray(values, dtype=np.int64)
    if a.ndim != 1 or (n is not None and len(a) != n):
        raise ValueError(f"{what} must hold one entry per tensor")
    return a


def _host(a):
    """Address of a non-empty host array's data (None for an empty one); a.ctypes.data takes three times as long."""
    if not a.size:
        return None
    return C.addressof(C.c_char.from_buffer(a)) if a.flags.writeable else a.ctypes.data


def _op(rc, err):
    if rc != OK:
        raise RFastError(rc, err.value.decode())


def rfast_grad_norm(grad, numel, max_norm: float, d_norm: int, d_scale: int, workspace: int, workspace_bytes: int,
                    grad_type: str = "f32", cuda_stream: int = 0) -> None:
    """2-norm over all gradient tensors into *d_norm and the factor max_norm / max(norm, max_norm) into
    *d_scale (DEVICE addresses of one fp32 value each, 0 for none).  grad: DEVICE addresses of the
    tensors, numel their sizes (sequences or integer arrays); workspace: the DEVICE address of
    GRAD_NORM_WORKSPACE bytes that no other running call uses.  Enqueued on cuda_stream."""
    n = _list(numel, None, "numel")
    g = _list(grad, len(n), "grad")
    err = C.create_string_buffer(256)
    _op(lib().rfast_grad_norm(len(n), _type(grad_type), _host(n), _host(g), max_norm, d_norm or None, d_scale or None,
                              workspace or None, workspace_bytes, cuda_stream or None, err, 256), err)


def rfast_adamw_step(param, grad, m, v, numel, step: int = 0, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                     eps: float = 1e-8, weight_decay: float = 1e-2, m_scale=None, v_scale=None, param_type: str = "f32",
                     grad_type: str = "f32", d_step: int = 0, d_grad_scale: int = 0, cuda_stream: int = 0) -> None:
    """One AdamW step, in place, over many tensors: param, grad, m, v are their DEVICE addresses, numel
    their sizes (sequences or integer arrays).  Moments are fp32; with m_scale and v_scale they are 8-bit
    codes with one fp32 scale per ADAMW_BLOCK values of a tensor.  step counts from 1; d_step: DEVICE
    address of an int64 that holds it instead; d_grad_scale: DEVICE address of an fp32 factor on the
    gradients (rfast_grad_norm writes one).  Enqueued on cuda_stream."""
    n = _list(numel, None, "numel")
    k = len(n)
    lists = [_list(a, k, name) for a, name in ((param, "param"), (grad, "grad"), (m, "m"), (v, "v"))]
    if (m_scale is None) != (v_scale is None):
        raise ValueError("8-bit moments need both m_scale and v_scale")
    bits = 32
    scales = [None, None]
    if m_scale is not None:
        bits = 8
        lists += [_list(m_scale, k, "m_scale"), _list(v_scale, k, "v_scale")]
        scales = [_host(a) for a in lists[4:]]
    args = _AdamW(k, _type(param_type), _type(grad_type), bits, _host(n), *[_host(a) for a in lists[:4]], *scales,
                  lr, beta1, beta2, eps, weight_decay, step, d_step or None, d_grad_scale or None)
    err = C.create_string_buffer(256)
    _op(lib().rfast_adamw_step(C.byref(args), cuda_stream or None, err, 256), err)


def _gn_shape(samples, positions, channels, groups, samples_per_set, type, act):
    if act not in ACT_IDS:
        raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACT_IDS)}")
    return _GnShape(samples, positions, channels, groups, max(samples, 1) if samples_per_set is None else samples_per_set, _type(type), ACT_IDS[act])


def _strides(s):
    return None if s is None else (C.c_int64 * 2)(*s)


def rfast_group_norm_workspace(samples: int, positions: int, channels: int, groups: int, samples_per_set=None, type: str = "f32",
                               act: str = "none", backward: bool = False) -> int:
    """Bytes of DEVICE workspace that a call of this shape needs."""
    need = lib().rfast_group_norm_workspace(C.byref(_gn_shape(samples, positions, channels, groups, samples_per_set, type, act)), 1 if backward else 0)
    if need < 0:
        raise RFastError(int(need), "rfast_group_norm_workspace: the shape is not valid")
    return int(need)


def rfast_group_norm(x: int, gamma: int, beta: int, y: int, mean: int, rstd: int, samples: int, positions: int, channels: int, groups: int,
                     samples_per_set=None, eps: float = 1e-5, act: str = "none", type: str = "f32", x_strides=None, y_strides=None,
                     workspace: int = 0, workspace_bytes: int = 0, cuda_stream: int = 0) -> None:
    """Group norm with an activation, channels last: y = act(gamma (x - mean) rstd + beta) over x
    [samples][positions][channels].  All addresses are DEVICE addresses; x and y have `type`, gamma, beta
    [samples / samples_per_set][channels] and the results mean, rstd [samples][groups] are fp32
    (samples_per_set None: one row for all samples).  Strides: (sample, position) in elements, None for
    contiguous.  workspace: rfast_group_norm_workspace(...) bytes that no other running call uses.
    Enqueued on cuda_stream."""
    shape = _gn_shape(samples, positions, channels, groups, samples_per_set, type, act)
    err = C.create_string_buffer(256)
    _op(lib().rfast_group_norm(C.byref(shape), x or None, _strides(x_strides), gamma or None, beta or None, eps, y or None, _strides(y_strides),
                               mean or None, rstd or None, workspace or None, workspace_bytes, cuda_stream or None, err, 256), err)


def rfast_group_norm_backward(dy: int, x: int, gamma: int, beta: int, mean: int, rstd: int, dx: int, dgamma: int, dbeta: int, samples: int,
                              positions: int, channels: int, groups: int, samples_per_set=None, act: str = "none", type: str = "f32",
                              dy_strides=None, x_strides=None, dx_strides=None, workspace: int = 0, workspace_bytes: int = 0,
                              cuda_stream: int = 0) -> None:
    """Gradients of rfast_group_norm: dx (of `type`), dgamma and dbeta (fp32, one row per set) from dy and
    the forward pass's x, mean and rstd.  workspace: rfast_group_norm_workspace(..., backward=True) bytes
    that no other running call uses.  Enqueued on cuda_stream."""
    shape = _gn_shape(samples, positions, channels, groups, samples_per_set, type, act)
    err = C.create_string_buffer(256)
    _op(lib().rfast_group_norm_backward(C.byref(shape), dy or None, _strides(dy_strides), x or None, _strides(x_strides), gamma or None, beta or None,
                                        mean or None, rstd or None, dx or None, _strides(dx_strides), dgamma or None, dbeta or None,
                                        workspace or None, workspace_bytes, cuda_stream or None, err, 256), err)


def _emb_shape(tokens, vocab, width, token_bits, table_type, out_type):
    return _EmbShape(tokens, vocab, width, token_bits, _type(table_type), _type(out_type))


def rfast_embedding(d_tokens: int, d_table: int, d_out: int, tokens: int, vocab: int, width: int, scale: float = 1.0, token_bits: int = 64,
                    table_type: str = "f32", out_type: str = "f32", table_stride=None, out_stride=None, cuda_stream: int = 0) -> None:
    """out[i] = scale * table[token i]: rows of a table [vocab][width] by token, zero where the token is outside [0, vocab).
    All addresses are DEVICE addresses; tokens are integers of token_bits (32 or 64).  Strides are those of a row in elements,
    None for contiguous rows.  Enqueued on cuda_stream."""
    shape = _emb_shape(tokens, vocab, width, token_bits, table_type, out_type)
    err = C.create_string_buffer(256)
    _op(lib().rfast_embedding(C.byref(shape), d_tokens or None, d_table or None, width if table_stride is None else table_stride, scale,
                              d_out or None, width if out_stride is None else out_stride, cuda_stream or None, err, 256), err)


def rfast_embedding_workspace(tokens: int, vocab: int, width: int) -> int:
    """Bytes of DEVICE workspace that the backward pass of this shape needs."""
    need = lib().rfast_embedding_workspace(C.byref(_emb_shape(tokens, vocab, width, 64, "f32", "f32")))
    if need < 0:
        raise RFastError(int(need), "rfast_embedding_workspace: the shape is not valid")
    return int(need)


def rfast_embedding_backward(d_tokens: int, d_dout: int, d_dtable: int, tokens: int, vocab: int, width: int, scale: float = 1.0,
                             accumulate: bool = False, token_bits: int = 64, out_type: str = "f32", table_type: str = "f32", dout_stride=None,
                             dtable_stride=None, workspace: int = 0, workspace_bytes: int = 0, cuda_stream: int = 0) -> None:
    """Gradient of rfast_embedding in its table: dtable[v] = scale * sum of the rows of dout (of out_type) whose token is v, of
    table_type; with accumulate it is added to what dtable holds.  Sums are formed in fp32 in the order of the positions.
    workspace: rfast_embedding_workspace(...) bytes that no other running call uses.  Enqueued on cuda_stream."""
    shape = _emb_shape(tokens, vocab, width, token_bits, table_type, out_type)
    err = C.create_string_buffer(256)
    _op(lib().rfast_embedding_backward(C.byref(shape), d_tokens or None, d_dout or None, width if dout_stride is None else dout_stride, scale,
                                       1 if accumulate else 0, d_dtable or None, width if dtable_stride is None else dtable_stride,
                                       workspace or None, workspace_bytes, cuda_stream or None, err, 256), err)


def rfast_policy_loss(d_logits: int, d_tokens: int, d_old_logp: int, d_advantage: int, tokens: int, vocab: int, d_loss: int = 0,
                      d_token_loss: int = 0, d_logp: int = 0, d_dlogits: int = 0, d_ref_logp: int = 0, d_weight: int = 0, d_loss_scale: int = 0,
                      temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0, type: str = "f32",
                      token_bits: int = 64, logits_stride=None, dlogits_stride=None, cuda_stream: int = 0) -> None:
    """Clipped policy loss with a KL term out of logits [tokens][vocab], and its gradient: token_loss = weight (-min(r A, clamp(r, 1 -
    clip_low, 1 + clip_high) A) + kl_coef (exp(d) - d - 1)) with r = exp(logp - old_logp), d = ref_logp - logp and logp the token's log
    probability at `temperature`.  All addresses are DEVICE addresses: logits and dlogits have `type`, everything else is fp32 [tokens],
    d_loss and d_loss_scale one value; 0 for what is not given or not wanted (d_old_logp and d_advantage too where d_logp is the only result).
    Rows of weight 0 or with a token outside [0, vocab) do not count.  Enqueued on cuda_stream."""
    args = _Policy(tokens, vocab, _type(type), token_bits, d_logits or None, vocab if logits_stride is None else logits_stride, d_tokens or None,
                   d_old_logp or None, d_ref_logp or None, d_advantage or None, d_weight or None, d_loss_scale or None, temperature, clip_low,
                   clip_high, kl_coef, d_loss or None, d_token_loss or None, d_logp or None, d_dlogits or None,
                   vocab if dlogits_stride is None else dlogits_stride)
    err = C.create_string_buffer(256)
    _op(lib().rfast_policy_loss(C.byref(args), cuda_stream or None, err, 256), err)


def _sides(rows, cols):
    r, c = np.ascontiguousarray(rows, dtype=np.int32), np.ascontiguousarray(cols, dtype=np.int32)
    if r.ndim != 1 or r.shape != c.shape:
        raise ValueError("rows and cols must hold one entry per matrix")
    return r, c


def rfast_muon_workspace(rows, cols, param_type: str = "f32", terms: int = 0) -> int:
    """Bytes of DEVICE workspace that a step over matrices of these rows and columns needs."""
    r, c = _sides(rows, cols)
    _type(param_type)
    need = lib().rfast_muon_workspace(len(r), _host(r), _host(c), terms or (1 if param_type == "bf16" else 2))
    if need < 0:
        raise RFastError(int(need), "rfast_muon_workspace: rows, cols or terms are not valid")
    return int(need)


def rfast_muon_step(param, grad, momentum_buffer, rows, cols, lr: float = 0.02, momentum: float = 0.95, weight_decay: float = 0.0,
                    nesterov: bool = True, eps: float = 1e-7, iterations: int = 5, size_rule: str = "spectral", terms: int = 0,
                    param_type: str = "f32", grad_type: str = "f32", d_grad_scale: int = 0, workspace: int = 0, workspace_bytes: int = 0,
                    cuda_stream: int = 0) -> None:
    """One Muon step, in place, over many matrices: momentum, an update orthogonalised by `iterations` Newton-Schulz steps, decay.
    param, grad and momentum_buffer are the matrices' DEVICE addresses, rows and cols their sizes (sequences or integer arrays);
    momentum is fp32.  size_rule: "spectral" (sqrt(max(1, rows / cols))) or "rms" (0.2 sqrt(max(rows, cols))) times the update;
    terms: fp16 numbers per factor of the products (0: 1 for bf16 parameters, else 2); d_grad_scale: DEVICE address of an fp32
    factor on the gradients.  workspace: rfast_muon_workspace(...) bytes, aligned to 256, that no other running call uses.  Enqueued
    on cuda_stream."""
    r, c = _sides(rows, cols)
    k = len(r)
    lists = [_list(a, k, name) for a, name in ((param, "param"), (grad, "grad"), (momentum_buffer, "momentum_buffer"))]
    if size_rule not in SIZE_RULES:
        raise ValueError(f"unknown size_rule {size_rule!r}: one of {', '.join(SIZE_RULES)}")
    args = _Muon(k, _type(param_type), _type(grad_type), terms, _host(r), _host(c), *[_host(a) for a in lists], lr, momentum, weight_decay, eps,
                 1 if nesterov else 0, iterations, SIZE_RULES[size_rule], d_grad_scale or None)
    err = C.create_string_buffer(256)
    _op(lib().rfast_muon_step(C.byref(args), workspace or None, workspace_bytes, cuda_stream or None, err, 256), err)


class Engine:
    """Convenience wrapper owning one handle."""

    def __init__(self, wl, cuda_stream: int = 0):
        self.n, self.p = int(wl.n), int(wl.p)
        self.n_edges_c = len(wl.G_C.col)
        self.n_edges_r = len(wl.G_R.col)
        self.h = rfast_create(wl, cuda_stream)
        self.K = 0

    def load_schedule(self, s):
        rfast_load_schedule(self.h, s)
        self.K = int(s.K)

    def append_schedule(self, more):
        rfast_append_schedule(self.h, more)
        self.K += int(more.K)

    def run(self, rounds=None, sync=True):
        rfast_run(self.h, self.K - self.query(Q_ROUND) if rounds is None else rounds, sync)

    def reset(self):
        rfast_reset(self.h)

    def sync(self):
        rfast_sync(self.h)

    def query(self, what):
        return rfast_query(self.h, what)

    def read(self, which, out=None):
        n, p = self.n, self.p
        shape = {STATE_X: (n, p), STATE_Y: (n, p), STATE_G_LAST: (n, p),
                 STATE_RHO_LATEST: (self.n_edges_c, p), STATE_RHO_BUF: (self.n_edges_c, p),
                 STATE_T_LOCAL: (n,), STATE_TAU_V_END: (self.n_edges_r,),
                 STATE_TAU_RHO_END: (self.n_edges_c,), STATE_ROUND: (1,),
                 STATE_V_LATEST: (n, p), STATE_V_HELD: (n,), STATE_ADAM_M: (n, p), STATE_ADAM_V: (n, p), STATE_TAU_V: (self.n_edges_r,),
                 STATE_TAU_RHO: (self.n_edges_c,)}.get(which)
        if which == STATE_USED_TAU_V:
            shape = (self.query(Q_N_USED_TAU_V),)
        if which == STATE_USED_TAU_RHO:
            shape = (self.query(Q_N_USED_TAU_RHO),)
        return rfast_read_state(self.h, which, shape, out)

    def seek(self, rnd):
        rfast_seek(self.h, rnd)

    def write(self, which, values):
        rfast_write_state(self.h, which, values)

    def read_packet(self, graph, ident, stamp):
        return rfast_read_packet(self.h, graph, ident, stamp, self.p)

    def write_packet(self, graph, ident, stamp, values):
        return rfast_write_packet(self.h, graph, ident, stamp, values)

    def set_option(self, option, value):
        rfast_set_option(self.h, option, value)

    def checkpoint(self):
        return rfast_checkpoint_save(self.h)

    def restore(self, blob):
        rfast_checkpoint_load(self.h, blob)

    def snapshot(self, x_out, y_out):
        if x_out.shape != (self.n, self.p) or y_out.shape != (self.n, self.p):
            raise ValueError("snapshot destinations must be [n][p]")
        rfast_snapshot(self.h, x_out, y_out)

    def snapshot_wait(self):
        rfast_snapshot_wait(self.h)

    def diagnostics(self, full=True):
        return rfast_diagnostics(self.h, full)

    def close(self):
        if self.h:
            rfast_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()
