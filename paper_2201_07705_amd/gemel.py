"""ctypes binding of libgemel (include/gemel.h): the same entry points,
argument marshalling only. Every layer of every model runs in the HIP
kernels of libgemel.so; there is no Python or CPU fallback: importing this
module without the built library raises.

``Context`` wraps the calls for Python callers: layers are given as dicts
(op, src0, src1, cin, cout, kh, kw, stride, pad, act, res, res_mode, out;
see workloads/zoo.py for the format) with per-layer parameter dicts
(w, b, bn = (gamma, beta, mean, var, eps)); device buffers and streams come
from torch.
"""

from __future__ import annotations

import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgemel.so")

# status codes
OK, EINVAL, ENOMEM, ESHAPE, ENOTMERGEABLE, EBUDGET, EDEVICE, ESTATE = \
    0, -1, -2, -3, -4, -5, -6, -7
STATUS_NAMES = {0: "OK", -1: "EINVAL", -2: "ENOMEM", -3: "ESHAPE",
                -4: "ENOTMERGEABLE", -5: "EBUDGET", -6: "EDEVICE",
                -7: "ESTATE"}
F32, BF16 = 0, 1
OP = {"conv": 0, "fc": 1, "maxpool": 2, "avgpool": 3, "upsample": 4,
      "concat": 5}
ACT = {"none": 0, "relu": 1, "leaky": 2}
RES_MODE = {"add_act": 0, "act_add": 1}
LEAKY_SLOPE = 0.1

Q_UNMERGED_BYTES, Q_MERGED_BYTES, Q_RESIDENT_BYTES, Q_PEAK_BYTES, \
    Q_STREAMED_BYTES, Q_ACTIVATION_BYTES, Q_LAUNCHES, Q_N_MODELS, \
    Q_GRAPH_REPLAYS, Q_STREAMS, Q_ROUND_MODE, Q_ROUND_TUNING, \
    Q_ROUND_LOADED_BYTES, Q_ROUND_EVICTED_BYTES, Q_CACHED_BYTES, \
    Q_CACHE_CAPACITY, Q_PREFETCHES = range(17)
OPT_USE_GRAPH, OPT_SWAP_SLOT_BYTES, OPT_SWAP_SLOTS, OPT_FAIL_COPY_AT, \
    OPT_SPLIT_MERGED, OPT_WEIGHT_BUDGET, OPT_PROFILE, OPT_CONV_TILE, \
    OPT_CONV_SPLITS, OPT_STREAMS, OPT_GRAPH_DAG, OPT_FORK_US, \
    OPT_AUTOTUNE, OPT_SPLITK_FUSED, OPT_TUNE, OPT_FUSE_POOL, \
    OPT_MIXED_SIZES, OPT_PAIRED_ACTS, OPT_FAIL_ALLOC_AT, \
    OPT_GROUP_UNMERGED, OPT_SWAP_CACHE, OPT_PREFETCH = range(22)
KERNEL_FAMILIES = ("conv_mfma", "conv_f32", "splitk_reduce", "fc", "pack",
                   "pool", "route", "export", "conv_merged")

EXPORTED = ("gemel_create", "gemel_register_model", "gemel_merge",
            "gemel_enumerate_groups", "gemel_infer", "gemel_infer_noalloc",
            "gemel_set_next_round", "gemel_load_order",
            "gemel_sla_batches", "gemel_profile_batches",
            "gemel_model_outputs", "gemel_output_shape",
            "gemel_query", "gemel_set_option", "gemel_profile",
            "gemel_last_error", "gemel_destroy",
            "gemel_log_probs", "gemel_distill", "gemel_distill_backward",
            "gemel_mx_quantize", "gemel_mx_dequantize", "gemel_mx_product",
            "gemel_adapter_batch", "gemel_adapter_batch_free",
            "gemel_adapt", "gemel_adapt_backward", "gemel_orthogonalize",
            "gemel_muon_step")
# Operators that serve and retrain merged layers: not part of CPU builds of
# the planner alone.
OPERATORS = EXPORTED[-6:]
# Answers, distillation and 4-bit matrices: builds of the operators above
# alone lack them.
ANSWERS = EXPORTED[-12:-6]

_fp = ctypes.POINTER(ctypes.c_float)


class LayerDesc(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int32), ("src0", ctypes.c_int32),
                ("src1", ctypes.c_int32), ("cin", ctypes.c_int32),
                ("cout", ctypes.c_int32), ("kh", ctypes.c_int32),
                ("kw", ctypes.c_int32), ("stride", ctypes.c_int32),
                ("pad", ctypes.c_int32), ("act", ctypes.c_int32),
                ("act_slope", ctypes.c_float), ("res_src", ctypes.c_int32),
                ("res_mode", ctypes.c_int32), ("is_output", ctypes.c_int32),
                ("weight", _fp), ("bias", _fp), ("bn_gamma", _fp),
                ("bn_beta", _fp), ("bn_mean", _fp), ("bn_var", _fp),
                ("bn_eps", ctypes.c_float)]


class Member(ctypes.Structure):
    _fields_ = [("model_id", ctypes.c_int32), ("layer", ctypes.c_int32)]


class Group(ctypes.Structure):
    _fields_ = [("n_members", ctypes.c_int32),
                ("members", ctypes.POINTER(Member))]


class Projection(ctypes.Structure):
    _fields_ = [("n_in", ctypes.c_int32), ("n_out", ctypes.c_int32),
                ("weight", ctypes.c_void_p),
                ("weight_stride", ctypes.c_int64),
                ("bias", ctypes.c_void_p), ("a", ctypes.c_void_p),
                ("b", ctypes.c_void_p)]


class Answers(ctypes.Structure):
    _fields_ = [("log_prob", ctypes.c_void_p), ("rank", ctypes.c_void_p),
                ("entropy", ctypes.c_void_p), ("log_sum", ctypes.c_void_p),
                ("top_indices", ctypes.c_void_p),
                ("top_log_probs", ctypes.c_void_p)]


class Mx(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class KernelStat(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("launches", ctypes.c_int32),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double),
                ("ms", ctypes.c_double)]


class GemelError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def _hip_runtimes():
    """Paths of every HIP runtime library mapped into this process."""
    paths = set()
    try:
        with open("/proc/self/maps") as f:
            for line in f:
                if "libamdhip64" in line:
                    paths.add(os.path.realpath(line.split()[-1]))
    except OSError:
        pass
    return paths


def load(path):
    """Load another build of the same ABI (e.g. a CPU build of the host
    code used by the tests) with its C signatures declared. Such a build may
    lack the operators of OPERATORS and ANSWERS."""
    return _configure(ctypes.CDLL(path))


def _configure(L):
    """Declare the C signatures of the ABI on a loaded library."""
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    L.gemel_create.argtypes = [ctypes.POINTER(vp), i32, i32,
                               ctypes.c_uint64]
    L.gemel_register_model.argtypes = [vp, ctypes.POINTER(LayerDesc), i32,
                                       i32, i32, i32,
                                       ctypes.POINTER(i32)]
    L.gemel_merge.argtypes = [vp, ctypes.POINTER(Group), i32]
    L.gemel_enumerate_groups.argtypes = [
        vp, ctypes.POINTER(i32), i32, ctypes.POINTER(Group), i32,
        ctypes.POINTER(Member), i32, ctypes.POINTER(i64),
        ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.gemel_infer.argtypes = [vp, ctypes.POINTER(i32), i32,
                              ctypes.POINTER(vp), ctypes.POINTER(i32),
                              ctypes.POINTER(vp), vp]
    L.gemel_infer_noalloc.argtypes = L.gemel_infer.argtypes
    L.gemel_set_next_round.argtypes = [vp, ctypes.POINTER(i32), i32]
    L.gemel_load_order.argtypes = [vp, ctypes.POINTER(i32), i32,
                                   ctypes.POINTER(i32)]
    f64p = ctypes.POINTER(ctypes.c_double)
    L.gemel_sla_batches.argtypes = [i32, i32, f64p, f64p, i32,
                                    ctypes.c_double, ctypes.c_double,
                                    ctypes.POINTER(i32), f64p, f64p]
    L.gemel_profile_batches.argtypes = [vp, ctypes.POINTER(i32), i32, i32,
                                        i32, vp, f64p]
    L.gemel_model_outputs.argtypes = [vp, i32, ctypes.POINTER(i32)]
    L.gemel_output_shape.argtypes = [vp, i32, i32, i32,
                                     ctypes.POINTER(i64)]
    L.gemel_query.argtypes = [vp, i32, ctypes.POINTER(i64)]
    L.gemel_set_option.argtypes = [vp, i32, i64]
    L.gemel_profile.argtypes = [vp, ctypes.POINTER(KernelStat),
                                ctypes.POINTER(i32)]
    L.gemel_last_error.argtypes = [vp]
    L.gemel_last_error.restype = ctypes.c_char_p
    L.gemel_destroy.argtypes = [vp]
    for name in EXPORTED:
        if name != "gemel_last_error" and name not in OPERATORS + ANSWERS:
            getattr(L, name).restype = ctypes.c_int32
    if hasattr(L, OPERATORS[0]):
        _configure_operators(L)
    if hasattr(L, ANSWERS[0]):
        _configure_answers(L)
    return L


def _configure_operators(L):
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    f32, pi32 = ctypes.c_float, ctypes.POINTER(ctypes.c_int32)
    proj = ctypes.POINTER(Projection)
    L.gemel_adapter_batch.argtypes = [vp, pi32, pi32, i32, i32, i32, pi32,
                                      _fp, pi32]
    L.gemel_adapter_batch_free.argtypes = [vp, i32]
    L.gemel_adapt.argtypes = [vp, i32, proj, vp, i64, vp, i64, vp]
    L.gemel_adapt_backward.argtypes = [vp, i32, proj, vp, i64, vp, i64, vp,
                                       i64, vp, vp, vp, vp, vp]
    L.gemel_orthogonalize.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp]
    L.gemel_muon_step.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, f32,
                                  f32, f32, i32, i32, vp]
    for name in OPERATORS:
        getattr(L, name).restype = i32


def _configure_answers(L):
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    f32 = ctypes.c_float
    L.gemel_log_probs.argtypes = [vp, i32, i32, vp, i64, i32, vp, i32, f32,
                                  ctypes.POINTER(Answers), vp]
    L.gemel_distill.argtypes = [vp, i32, i32, vp, i64, i32, vp, vp, i32, f32,
                                vp, vp]
    L.gemel_distill_backward.argtypes = [vp, i32, i32, vp, vp, i64, i32, vp,
                                         vp, i32, f32, vp, i64, vp, vp]
    mx = ctypes.POINTER(Mx)
    L.gemel_mx_quantize.argtypes = [vp, vp, i64, i32, mx, vp]
    L.gemel_mx_dequantize.argtypes = [vp, mx, vp, i64, i32, vp]
    L.gemel_mx_product.argtypes = [vp, i32, vp, i64, mx, mx, vp, vp, i64, vp]
    for name in ANSWERS:
        getattr(L, name).restype = i32


def lib():
    """Load libgemel.so (raises if it has not been built).

    torch brings its own HIP runtime whose soname equals the system one; it
    is loaded first so that libgemel binds to the same runtime instance
    (two HIP runtimes in one process do not share the device)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2201_07705_amd.build` (no fallback exists)")
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        rts = _hip_runtimes()
        if len(rts) > 1:
            raise RuntimeError(f"two HIP runtimes are loaded: {sorted(rts)}")
        _configure(L)
        _lib = L
    return _lib


def _fptr(a):
    return None if a is None else a.ctypes.data_as(_fp)


def layer_descs(layers, params):
    """Marshal layer dicts + parameter dicts into a LayerDesc array. Returns
    (array, keepalive list of the float32 arrays it points into)."""
    arr = (LayerDesc * len(layers))()
    keep = []
    for i, (l, p) in enumerate(zip(layers, params)):
        d = arr[i]
        d.op = OP[l["op"]]
        d.src0, d.src1 = l["src0"], l.get("src1", -1)
        d.cin, d.cout = l["cin"], l["cout"]
        d.kh, d.kw = l.get("kh", 1), l.get("kw", 1)
        d.stride, d.pad = l.get("stride", 1), l.get("pad", 0)
        d.act = ACT[l.get("act", "none")]
        d.act_slope = LEAKY_SLOPE if l.get("act") == "leaky" else 0.0
        d.res_src = l.get("res", -1)
        d.res_mode = RES_MODE[l.get("res_mode", "add_act")]
        d.is_output = 1 if l.get("out") else 0
        if p is not None:
            w = np.ascontiguousarray(p["w"], np.float32)
            keep.append(w)
            d.weight = _fptr(w)
            if p.get("b") is not None:
                b = np.ascontiguousarray(p["b"], np.float32)
                keep.append(b)
                d.bias = _fptr(b)
            if p.get("bn") is not None:
                g, be, mu, var, eps = p["bn"]
                vs = [np.ascontiguousarray(v, np.float32)
                      for v in (g, be, mu, var)]
                keep.extend(vs)
                d.bn_gamma, d.bn_beta, d.bn_mean, d.bn_var = \
                    [_fptr(v) for v in vs]
                d.bn_eps = eps
    return arr, keep


def sla_batches(cost_ms, sla_ms, fps, swap_ms=None, pipelined=True,
                library=None):
    """Per-model batch sizes under a per-frame deadline from a cost table
    [model][batch - 1] (ms): returns (batches, min frames/s, cycle ms)."""
    L = library or lib()
    n, nb = len(cost_ms), len(cost_ms[0])
    flat = (ctypes.c_double * (n * nb))(*[c for row in cost_ms for c in row])
    sw = (ctypes.c_double * n)(*swap_ms) if swap_ms is not None else None
    b = (ctypes.c_int32 * n)()
    v, t = ctypes.c_double(), ctypes.c_double()
    st = L.gemel_sla_batches(n, nb, flat, sw, 1 if pipelined else 0,
                             float(sla_ms), float(fps), b, ctypes.byref(v),
                             ctypes.byref(t))
    if st != OK:
        raise GemelError(st, "gemel_sla_batches: " + STATUS_NAMES.get(st, "?"))
    return list(b), v.value, t.value


_torch_module = None


def _torch():
    """The torch module, imported at the first use."""
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _int32(name, v):
    """v, which ctypes would cut to the C interface's int32 without a word."""
    if not -(1 << 31) <= v < 1 << 31:
        raise ValueError(f"{name} does not fit 32 bits: {v}")
    return v


def _int32s(name, values):
    """An array of int32 (of at least one element)."""
    return (ctypes.c_int32 * max(len(values), 1))(
        *[_int32(name, v) for v in values])


def _current_stream(device):
    """The handle of torch's current stream on the device. The entry that
    gives the handle alone is not a public one; where it is missing a Stream
    object is made for it (1 us of a call's 12)."""
    raw = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return _torch().cuda.current_stream(device).cuda_stream
    return raw(device)


class AdapterBatch:
    """The requests of Context.adapter_batch: rows of the batch, the bank's
    sizes and the library's id. Give it back with close(), or drop it."""

    def __init__(self, ctx, batch_id, rows, n_adapters, rank):
        self._ctx, self.id = ctx, batch_id
        self.rows, self.n_adapters, self.rank = rows, n_adapters, rank

    def close(self):
        if self._ctx is not None and self._ctx._h:
            self._ctx._check(self._ctx._lib.gemel_adapter_batch_free(
                self._ctx._h, self.id))
        self._ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MxMatrix:
    """A matrix [rows, cols] in microscaled 4-bit floating point, as
    Context.mx_quantize makes it: codes [rows, 256 groups] and scales [groups,
    rows, 16], both uint8 (include/gemel.h says which byte is which)."""

    def __init__(self, codes, scales, rows, cols):
        self._codes, self._scales = codes, scales
        self.rows, self.cols = rows, cols
        self._c = None   # the C description, once it was checked

    @property
    def codes(self):
        return self._codes

    @codes.setter
    def codes(self, t):
        self._codes, self._c = t, None   # (another tensor is checked anew)

    @property
    def scales(self):
        return self._scales

    @scales.setter
    def scales(self, t):
        self._scales, self._c = t, None

    def _key(self, device):
        """What a description holds for: tensors can be given other memory or
        another shape in place."""
        a, b = self._codes, self._scales
        return (device, self.rows, self.cols, a.data_ptr(), b.data_ptr(),
                a.shape, b.shape, a.is_contiguous(), b.is_contiguous())

    @staticmethod
    def shapes(rows, cols):
        """Shapes of codes and scales."""
        groups = -(-cols // 512)
        return (rows, 256 * groups), (groups, rows, 16)

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()


class Context:
    """One libgemel context on one device."""

    def __init__(self, device=0, dtype="bf16", budget=0, library=None):
        self._lib = library or lib()
        self._h = ctypes.c_void_p()
        st = self._lib.gemel_create(ctypes.byref(self._h), device,
                                BF16 if dtype == "bf16" else F32, budget)
        if st != OK:
            raise GemelError(st, self._lib.gemel_last_error(None).decode())
        self.dtype = dtype
        self.device = device
        self._in_shape = {}
        self._out_ops = {}

    # -- raw calls (status returned, message on failure) --
    def _check(self, st):
        if st != OK:
            raise GemelError(st, self._lib.gemel_last_error(self._h).decode())
        return st

    def register_model(self, layers, params, in_chw):
        arr, keep = layer_descs(layers, params)
        mid = ctypes.c_int32(-1)
        self._check(self._lib.gemel_register_model(
            self._h, arr, len(layers), in_chw[0], in_chw[1], in_chw[2],
            ctypes.byref(mid)))
        del keep
        self._in_shape[mid.value] = tuple(in_chw)
        self._out_ops[mid.value] = [l["op"] for l in layers if l.get("out")]
        return mid.value

    def merge(self, groups):
        """groups: list of lists of (model_id, layer_index); first = source."""
        n = len(groups)
        garr = (Group * max(n, 1))()
        keep = []
        for i, g in enumerate(groups):
            m = (Member * len(g))(*[Member(a, b) for a, b in g])
            keep.append(m)
            garr[i].n_members = len(g)
            garr[i].members = ctypes.cast(m, ctypes.POINTER(Member))
        self._check(self._lib.gemel_merge(self._h, garr, n))

    def enumerate_groups(self, model_ids):
        """Candidate groups of the models (Section 5.3): a list of
        (total_bytes, [(model_id, layer_index), ...]) in descending order of
        memory, each accepted by merge() as it is."""
        n = len(model_ids)
        ids = (ctypes.c_int32 * max(n, 1))(*model_ids)
        ng, nm = ctypes.c_int32(), ctypes.c_int32()
        self._check(self._lib.gemel_enumerate_groups(
            self._h, ids, n, None, 0, None, 0, None, ctypes.byref(ng),
            ctypes.byref(nm)))
        garr = (Group * max(ng.value, 1))()
        marr = (Member * max(nm.value, 1))()
        nbytes = (ctypes.c_int64 * max(ng.value, 1))()
        self._check(self._lib.gemel_enumerate_groups(
            self._h, ids, n, garr, ng.value, marr, nm.value, nbytes,
            ctypes.byref(ng), ctypes.byref(nm)))
        out, at = [], 0
        for g in range(ng.value):
            k = garr[g].n_members
            out.append((nbytes[g], [(marr[at + j].model_id, marr[at + j].layer)
                                    for j in range(k)]))
            at += k
        return out

    def n_outputs(self, model_id):
        n = ctypes.c_int32()
        self._check(self._lib.gemel_model_outputs(self._h, model_id,
                                              ctypes.byref(n)))
        return n.value

    def output_shape(self, model_id, idx, n_frames):
        dims = (ctypes.c_int64 * 4)()
        self._check(self._lib.gemel_output_shape(self._h, model_id, idx,
                                             n_frames, dims))
        if self._out_ops.get(model_id, [None] * (idx + 1))[idx] == "fc":
            return (n_frames, dims[1])
        return (n_frames, dims[1], dims[2], dims[3])

    def query(self, key):
        v = ctypes.c_int64()
        self._check(self._lib.gemel_query(self._h, key, ctypes.byref(v)))
        return v.value

    def set_option(self, key, value):
        self._check(self._lib.gemel_set_option(self._h, key, value))

    def profile(self):
        """Per-round kernel statistics by family: {name: dict(launches,
        flops, bytes, ms)} and the number of profiled rounds."""
        st = (KernelStat * len(KERNEL_FAMILIES))()
        rounds = ctypes.c_int32()
        self._check(self._lib.gemel_profile(self._h, st, ctypes.byref(rounds)))
        return {name: dict(launches=s.launches, flops=s.flops, bytes=s.bytes,
                           ms=s.ms)
                for name, s in zip(KERNEL_FAMILIES, st)}, rounds.value

    def infer_raw(self, model_ids, frame_ptrs, n_frames, out_ptrs, stream,
                  noalloc=False):
        n = len(model_ids)
        ids = (ctypes.c_int32 * n)(*model_ids)
        fp = (ctypes.c_void_p * n)(*frame_ptrs)
        nf = (ctypes.c_int32 * n)(*n_frames)
        op = (ctypes.c_void_p * max(len(out_ptrs), 1))(*out_ptrs)
        fn = self._lib.gemel_infer_noalloc if noalloc else self._lib.gemel_infer
        return fn(self._h, ids, n, fp, nf, op, ctypes.c_void_p(stream))

    def set_next_round(self, model_ids):
        """Models of the round after the next infer (weight cache pins)."""
        n = len(model_ids)
        ids = (ctypes.c_int32 * max(n, 1))(*model_ids)
        self._check(self._lib.gemel_set_next_round(self._h, ids, n))

    def load_order(self, model_ids):
        """Sharing-aware round-robin load order of the models."""
        n = len(model_ids)
        ids = (ctypes.c_int32 * n)(*model_ids)
        out = (ctypes.c_int32 * n)()
        self._check(self._lib.gemel_load_order(self._h, ids, n, out))
        return list(out)

    def profile_batches(self, model_ids, max_batch, reps=5, stream=None):
        """Measured cost table [model][batch - 1] in ms (nondecreasing
        rows) of each model alone on 1..max_batch frames."""
        import torch
        n = len(model_ids)
        ids = (ctypes.c_int32 * n)(*model_ids)
        out = (ctypes.c_double * (n * max_batch))()
        s = stream if stream is not None else torch.cuda.current_stream()
        self._check(self._lib.gemel_profile_batches(
            self._h, ids, n, max_batch, reps, s.cuda_stream, out))
        return [list(out[i * max_batch:(i + 1) * max_batch])
                for i in range(n)]

    def close(self):
        if self._h:
            st = self._lib.gemel_destroy(self._h)
            self._h = ctypes.c_void_p()
            if st != OK:
                raise GemelError(st, "destroy found a device fault")

    def __del__(self):
        try:
            if self._h:
                self._lib.gemel_destroy(self._h)
        except Exception:
            pass

    # -- torch conveniences --
    def alloc_outputs(self, model_ids, n_frames, device="cuda"):
        import torch
        outs = []
        for mid, n in zip(model_ids, n_frames):
            outs.append([torch.empty(self.output_shape(mid, i, n),
                                     dtype=torch.float32, device=device)
                         for i in range(self.n_outputs(mid))])
        return outs

    def infer(self, model_ids, frames, stream=None, outputs=None,
              noalloc=False):
        """frames: list of float32 NCHW cuda tensors, one per model id.
        Returns (and fills) per-model lists of float32 output tensors.
        noalloc: call gemel_infer_noalloc (outputs must be given)."""
        import torch
        n_frames = [int(f.shape[0]) for f in frames]
        for f in frames:
            assert f.dtype == torch.float32 and f.is_cuda and \
                f.is_contiguous()
        if outputs is None:
            outputs = self.alloc_outputs(model_ids, n_frames,
                                         frames[0].device)
        out_ptrs = [t.data_ptr() for o in outputs for t in o]
        s = stream if stream is not None else torch.cuda.current_stream()
        self._check(self.infer_raw(model_ids, [f.data_ptr() for f in frames],
                                   n_frames, out_ptrs, s.cuda_stream,
                                   noalloc=noalloc))
        return outputs

    # -- serving and retraining merged layers --
    def adapter_batch(self, adapter_ids, n_rows, n_adapters, rank, ranks=None,
                      scales=None):
        """Requests of n_rows[i] rows with adapter adapter_ids[i] (-1: none)
        of a bank of n_adapters adapters of up to `rank`; per adapter its
        rank (None: all `rank`) and scale (None: 1)."""
        n = len(adapter_ids)
        _int32("n_adapters", n_adapters)
        _int32("rank", rank)
        if len(n_rows) != n:
            raise ValueError("adapter_ids and n_rows differ in length")
        for what, v in (("ranks", ranks), ("scales", scales)):
            if v is not None and len(v) != n_adapters:
                raise ValueError(f"{what} must have one entry per adapter")
        out = ctypes.c_int32(-1)
        self._check(self._lib.gemel_adapter_batch(
            self._h, _int32s("adapter_ids", adapter_ids),
            _int32s("n_rows", n_rows), n, n_adapters, rank,
            None if ranks is None else _int32s("ranks", ranks),
            None if scales is None else
            (ctypes.c_float * max(n_adapters, 1))(*scales),
            ctypes.byref(out)))
        return AdapterBatch(self, out.value, sum(n_rows), n_adapters, rank)

    def _torch_dtype(self):
        return _torch().bfloat16 if self.dtype == "bf16" else _torch().float32

    def _tensor(self, name, t, shape, dtype, contiguous=True):
        """Checks one operand: a tensor of the context's device with the
        given shape and type whose rows are contiguous."""
        if t.get_device() != self.device:
            raise ValueError(f"{name} is not on cuda:{self.device}")
        if t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, is {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)}, has "
                             f"{tuple(t.shape)}")
        if t.is_contiguous():
            return
        if contiguous:
            raise ValueError(f"{name} must be contiguous")
        if t.numel() and (t.shape[1] > 1 and t.stride(1) != 1 or
                          t.shape[0] > 1 and t.stride(0) < t.shape[1]):
            raise ValueError(f"{name} must have contiguous rows")

    @staticmethod
    def _stride(t):
        rows, cols = t.shape
        return max(t.stride(0), cols) if rows > 1 else cols

    def _stream(self, stream, *tensors):
        """The handle of the stream to work on. Where that is not the current
        one the tensors are marked as used there, so that memory a caller
        drops is not handed out again before the work is done."""
        current = _current_stream(self.device)
        if stream is None or stream.cuda_stream == current:
            return current
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        return stream.cuda_stream

    @staticmethod
    def _empty(like, shape, dtype, stream):
        """A result's tensor, from the memory of the stream that fills it."""
        if stream is None:
            return like.new_empty(shape, dtype=dtype)
        with _torch().cuda.stream(stream):
            return like.new_empty(shape, dtype=dtype)

    @staticmethod
    def _written(*tensors):
        """Counts a change in place of tensors that a caller passed to be
        written, so that autograd refuses graphs that had saved them."""
        _torch().autograd.graph.increment_version(
            [t for t in tensors if t is not None])

    def _projection(self, batch, weight, a, b, bias):
        if batch._ctx is not self:
            raise ValueError("the batch is closed or of another context")
        if weight.dim() != 2:
            raise ValueError("weight must be [n_out, n_in]")
        dt = self._torch_dtype()
        n, k = weight.shape
        _int32("n_out", n)
        _int32("n_in", k)
        self._tensor("weight", weight, (n, k), dt, contiguous=False)
        if (a is None) != (b is None):
            raise ValueError("a and b come together")
        p = Projection(k, n, weight.data_ptr(), self._stride(weight))
        if a is not None:
            self._tensor("a", a, (batch.n_adapters, batch.rank, k), dt)
            self._tensor("b", b, (batch.n_adapters, n, batch.rank), dt)
            p.a, p.b = a.data_ptr(), b.data_ptr()
        if bias is not None:
            self._tensor("bias", bias, (n,), _torch().float32)
            p.bias = bias.data_ptr()
        return p, n, k, dt

    def adapt(self, batch, x, weight, a=None, b=None, bias=None, out=None,
              stream=None):
        """y = x W^T + bias + scale * (x A^T) B^T, each row with its
        request's adapter: x [rows, n_in], weight [n_out, n_in], a
        [adapters, rank, n_in], b [adapters, n_out, rank] of the context's
        type, bias float32. x, weight and out may have a row stride.

        This and the operators below run on `stream` (None: the current
        one), and make the tensors they return there. A captured call uses
        the workspace of the stream that is captured (on which a call of the
        same sizes has to come first) wherever its graph is replayed, so
        replays and other users of that workspace must be ordered. Autograd
        does not record the operators, whatever their operands require:
        results carry no graph, and gradients are those of adapt_backward.
        Tensors passed to be written count as changed in place."""
        p, n, k, dt = self._projection(batch, weight, a, b, bias)
        rows = batch.rows
        self._tensor("x", x, (rows, k), dt, contiguous=False)
        y = out
        if y is None:
            y = self._empty(x, (rows, n), dt, stream)
        else:
            self._tensor("out", y, (rows, n), dt, contiguous=False)
        self._check(self._lib.gemel_adapt(
            self._h, batch.id, p, x.data_ptr(), self._stride(x),
            y.data_ptr(), self._stride(y),
            self._stream(stream, x, weight, a, b, bias, y)))
        if out is not None:
            self._written(out)
        return y

    def adapt_backward(self, batch, dy, x, weight, a=None, b=None,
                       needs=("x", "weight", "bias", "a", "b"), outputs=None,
                       stream=None):
        """Gradients of adapt for dy [rows, n_out], as a dict of those in
        `needs`: "x" in the context's type; "weight", "bias", "a" and "b"
        in float32. outputs: tensors to write, by name (others are made)."""
        p, n, k, dt = self._projection(batch, weight, a, b, None)
        f32, rows = _torch().float32, batch.rows
        self._tensor("x", x, (rows, k), dt, contiguous=False)
        self._tensor("dy", dy, (rows, n), dt, contiguous=False)
        shapes = {"x": (rows, k), "weight": (n, k), "bias": (n,),
                  "a": (batch.n_adapters, batch.rank, k),
                  "b": (batch.n_adapters, n, batch.rank)}
        res, ptr = {}, {}
        for name in needs:
            if name not in shapes:
                raise ValueError(f"unknown gradient {name!r}")
            if a is None and name in ("a", "b"):
                if needs != ("x", "weight", "bias", "a", "b"):
                    raise ValueError(f"gradient {name!r} without adapters")
                continue
            want = dt if name == "x" else f32
            t = outputs.get(name) if outputs else None
            if t is None:
                t = self._empty(x, shapes[name], want, stream)
            else:
                self._tensor(f"outputs[{name!r}]", t, shapes[name], want,
                             contiguous=name != "x")
            res[name], ptr[name] = t, t.data_ptr()
        self._check(self._lib.gemel_adapt_backward(
            self._h, batch.id, p, x.data_ptr(), self._stride(x),
            dy.data_ptr(), self._stride(dy), ptr.get("x"),
            self._stride(res["x"]) if "x" in res else 0, ptr.get("weight"),
            ptr.get("bias"), ptr.get("a"), ptr.get("b"),
            self._stream(stream, x, dy, weight, a, b, *res.values())))
        if outputs:
            self._written(*(outputs.get(name) for name in res))
        return res

    @staticmethod
    def _matrices(t, steps):
        if t.dim() not in (2, 3):
            raise ValueError("expected [rows, cols] or [count, rows, cols]")
        _int32("steps", steps)
        shape = (1,) * (3 - t.dim()) + tuple(t.shape)
        for name, v in zip(("count", "rows", "cols"), shape):
            _int32(name, v)
        return shape

    def orthogonalize(self, g, steps=5, out=None, stream=None):
        """Newton-Schulz orthogonalisation of [rows, cols] or [count, rows,
        cols] contiguous matrices of the context's type."""
        count, rows, cols = self._matrices(g, steps)
        dt = self._torch_dtype()
        self._tensor("g", g, g.shape, dt)
        o = out
        if o is None:
            o = self._empty(g, g.shape, dt, stream)
        else:
            self._tensor("out", o, g.shape, dt)
        self._check(self._lib.gemel_orthogonalize(
            self._h, count, rows, cols, g.data_ptr(), o.data_ptr(), steps,
            self._stream(stream, g, o)))
        if out is not None:
            self._written(out)
        return o

    def muon_step(self, w, momentum_buffer, g, lr, momentum=0.95,
                  weight_decay=0.0, nesterov=True, steps=5, copy=None,
                  stream=None):
        """One optimiser step, in place, of float32 matrices w [rows, cols]
        or [count, rows, cols] with their momentum buffer and gradient; copy
        (bf16 contexts) receives the new w in bf16."""
        count, rows, cols = self._matrices(w, steps)
        for name, t in (("w", w), ("momentum_buffer", momentum_buffer),
                        ("g", g)):
            self._tensor(name, t, w.shape, _torch().float32)
        if copy is not None:
            self._tensor("copy", copy, w.shape, _torch().bfloat16)
        self._check(self._lib.gemel_muon_step(
            self._h, count, rows, cols, w.data_ptr(),
            momentum_buffer.data_ptr(), g.data_ptr(),
            None if copy is None else copy.data_ptr(), lr, momentum,
            weight_decay, 1 if nesterov else 0, steps,
            self._stream(stream, w, momentum_buffer, g, copy)))
        self._written(w, momentum_buffer, copy)
        return w

    # -- answers of merged models, and their distillation --
    def _logits(self, logits):
        """Rows, classes and type code of logits (bf16 or float32 in every
        context), rows contiguous."""
        torch = _torch()
        if logits.dim() != 2:
            raise ValueError("logits must be [rows, classes]")
        if logits.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("logits must be float32 or bfloat16, are "
                             f"{logits.dtype}")
        rows, classes = logits.shape
        _int32("rows", rows)
        _int32("classes", classes)
        self._tensor("logits", logits, (rows, classes), logits.dtype,
                     contiguous=False)
        return rows, classes, F32 if logits.dtype == torch.float32 else BF16

    def log_probs(self, logits, labels=None, top=0, temperature=1.0,
                  needs=None, outputs=None, stream=None):
        """What logits [rows, classes] (bf16 or float32) answer, as a dict:
        "log_prob" of each row's label and its "rank" (classes before it;
        both with labels, int32 [rows], -1: none), "entropy", "log_sum", and
        with top > 0 "top_indices" (int32, best first, of equal ones the
        lower index) and "top_log_probs" [rows, top] of the softmax of
        logits / temperature. Classes of -inf are not offered: -1 and -inf
        stand where fewer than `top` are. needs: names of those wanted (None:
        all); outputs: tensors to write, by name (others are made; a name
        that is none of these answers is refused)."""
        torch = _torch()
        rows, classes, code = self._logits(logits)
        _int32("top", top)
        f32, i32 = torch.float32, torch.int32
        kinds = {"entropy": ((rows,), f32), "log_sum": ((rows,), f32)}
        if labels is not None:
            self._tensor("labels", labels, (rows,), i32)
            kinds.update(log_prob=((rows,), f32), rank=((rows,), i32))
        if top > 0:
            kinds.update(top_indices=((rows, top), i32),
                         top_log_probs=((rows, top), f32))
        for name in outputs or ():
            if name not in kinds:
                raise ValueError(f"outputs: no answer {name!r} (of these "
                                 "arguments)")
        res, a = {}, Answers()
        if needs is None and not outputs:
            # the numbers of a row are made together, as rows of one tensor
            # (three tensors of their own take 2 us more)
            flat = [name for name in kinds if kinds[name] == ((rows,), f32)]
            made = self._empty(logits, (len(flat), rows), f32, stream)
            res.update(zip(flat, made.unbind(0)))
        for name in kinds if needs is None else needs:
            if name not in kinds:
                raise ValueError(f"no answer {name!r} (of these arguments)")
            shape, dt = kinds[name]
            t = outputs.get(name) if outputs else res.get(name)
            if t is None:
                t = self._empty(logits, shape, dt, stream)
            elif outputs:
                self._tensor(f"outputs[{name!r}]", t, shape, dt)
            res[name] = t
            setattr(a, name, t.data_ptr())
        self._check(self._lib.gemel_log_probs(
            self._h, rows, classes, logits.data_ptr(), self._stride(logits),
            code, None if labels is None else labels.data_ptr(), top,
            temperature, a,
            self._stream(stream, logits, labels, *res.values())))
        if outputs:
            self._written(*(outputs.get(name) for name in res))
        return res

    def _entries(self, logits, indices, values):
        rows, classes, code = self._logits(logits)
        if indices.dim() != 2:
            raise ValueError("indices must be [rows, entries]")
        k = indices.shape[1]
        self._tensor("indices", indices, (rows, k), _torch().int32)
        self._tensor("values", values, (rows, k), _torch().float32)
        return rows, classes, code, k

    def distill(self, logits, indices, values, temperature=1.0, out=None,
                stream=None):
        """Loss [rows] of logits [rows, classes] against a teacher's best
        ones: temperature^2 * sum of q (log q - log p), q the softmax of
        values / temperature over the row's entries (indices int32 and values
        float32 [rows, entries], as the teacher's log_probs gives them; class
        -1 or value -inf: no entry), p that of all logits / temperature."""
        rows, classes, code, k = self._entries(logits, indices, values)
        loss = out
        if loss is None:
            loss = self._empty(logits, (rows,), _torch().float32, stream)
        else:
            self._tensor("out", loss, (rows,), _torch().float32)
        self._check(self._lib.gemel_distill(
            self._h, rows, classes, logits.data_ptr(), self._stride(logits),
            code, indices.data_ptr(), values.data_ptr(), k, temperature,
            loss.data_ptr(),
            self._stream(stream, logits, indices, values, loss)))
        if out is not None:
            self._written(out)
        return loss

    def distill_backward(self, dloss, logits, indices, values,
                         temperature=1.0, loss=None, out=None, stream=None):
        """Gradient of distill for dloss [rows] (None: all 1) with respect to
        the logits, in their type. loss: a tensor [rows] that receives the
        losses too, from the same pass."""
        rows, classes, code, k = self._entries(logits, indices, values)
        f32 = _torch().float32
        for name, t in (("dloss", dloss), ("loss", loss)):
            if t is not None:
                self._tensor(name, t, (rows,), f32)
        d = out
        if d is None:
            d = self._empty(logits, (rows, classes), logits.dtype, stream)
        else:
            self._tensor("out", d, (rows, classes), logits.dtype,
                         contiguous=False)
        self._check(self._lib.gemel_distill_backward(
            self._h, rows, classes,
            None if dloss is None else dloss.data_ptr(), logits.data_ptr(),
            self._stride(logits), code, indices.data_ptr(),
            values.data_ptr(), k, temperature, d.data_ptr(), self._stride(d),
            None if loss is None else loss.data_ptr(),
            self._stream(stream, dloss, logits, indices, values, d, loss)))
        self._written(out, loss)
        return d

    # -- merged layers in 4 bits --
    def _mx(self, name, q):
        """The C description of a quantised matrix, checked (again where
        anything in it is another one than the last time)."""
        if not isinstance(q, MxMatrix):
            raise ValueError(f"{name} must be an MxMatrix")
        c, at = q._c, q._key(self.device)
        if c is not None and c[0] == at:
            return c[1]
        _int32(name + " rows", q.rows)
        _int32(name + " cols", q.cols)
        u8 = _torch().uint8
        codes, scales = MxMatrix.shapes(q.rows, q.cols)
        self._tensor(name + ".codes", q._codes, codes, u8)
        self._tensor(name + ".scales", q._scales, scales, u8)
        q._c = at, Mx(*at[1:5])
        return q._c[1]

    @staticmethod
    def _value_type(name, dtype):
        torch = _torch()
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"{name} must be float32 or bfloat16, is {dtype}")
        return F32 if dtype == torch.float32 else BF16

    def mx_quantize(self, x, out=None, stream=None):
        """x [rows, cols] (bf16 or float32 in every context, rows may have a
        stride) as an MxMatrix: blocks of 32 4-bit floating-point values of a
        row that share a power of two. out: an MxMatrix of that size whose
        memory is written."""
        if x.dim() != 2:
            raise ValueError("x must be [rows, cols]")
        rows, cols = x.shape
        code = self._value_type("x", x.dtype)
        _int32("rows", rows)
        _int32("cols", cols)
        self._tensor("x", x, (rows, cols), x.dtype, contiguous=False)
        q = out
        if q is None:
            u8 = _torch().uint8
            codes, scales = MxMatrix.shapes(rows, cols)
            q = MxMatrix(self._empty(x, codes, u8, stream),
                         self._empty(x, scales, u8, stream), rows, cols)
            at = q._key(self.device)
            q._c = at, Mx(*at[1:5])
            c = q._c[1]
        else:
            if (q.rows, q.cols) != (rows, cols):
                raise ValueError(f"out is [{q.rows}, {q.cols}], "
                                 f"x [{rows}, {cols}]")
            c = self._mx("out", q)
        self._check(self._lib.gemel_mx_quantize(
            self._h, x.data_ptr(), self._stride(x), code, c,
            self._stream(stream, x, q._codes, q._scales)))
        if out is not None:
            self._written(q.codes, q.scales)
        return q

    def mx_dequantize(self, q, dtype=None, out=None, stream=None):
        """The values [rows, cols] of an MxMatrix, in dtype (None: the
        context's; bf16 or float32), exactly."""
        c = self._mx("q", q)
        dt = dtype or (out.dtype if out is not None else self._torch_dtype())
        code = self._value_type("dtype", dt)
        v, ldv = out, q.cols
        if v is None:
            v = self._empty(q.codes, (q.rows, q.cols), dt, stream)
        else:
            self._tensor("out", v, (q.rows, q.cols), dt, contiguous=False)
            ldv = self._stride(v)
        self._check(self._lib.gemel_mx_dequantize(
            self._h, c, v.data_ptr(), ldv, code,
            self._stream(stream, q._codes, q._scales, v)))
        if out is not None:
            self._written(out)
        return v

    def mx_product(self, x, weight, bias=None, out=None, stream=None):
        """y = x W^T + bias with 4-bit weights: weight an MxMatrix [n_out,
        n_in], bias float32, y [rows, n_out] of the context's type. x [rows,
        n_in] is of the context's type and multiplied as it is, or an
        MxMatrix: then both sides are 4 bits."""
        w, dt = self._mx("weight", weight), self._torch_dtype()
        n, k = weight.rows, weight.cols
        if isinstance(x, MxMatrix):
            rows, xq, base = x.rows, self._mx("x", x), x.codes
            if x.cols != k:
                raise ValueError(f"x has {x.cols} columns, weight {k}")
            data, stride, used = None, 0, (x._codes, x._scales)
        else:
            if x.dim() != 2:
                raise ValueError("x must be [rows, n_in]")
            rows, xq, base = x.shape[0], None, x
            _int32("rows", rows)
            self._tensor("x", x, (rows, k), dt, contiguous=False)
            data, stride, used = x.data_ptr(), self._stride(x), (x,)
        if bias is not None:
            self._tensor("bias", bias, (n,), _torch().float32)
        y, ldy = out, n
        if y is None:
            y = self._empty(base, (rows, n), dt, stream)
        else:
            self._tensor("out", y, (rows, n), dt, contiguous=False)
            ldy = self._stride(y)
        self._check(self._lib.gemel_mx_product(
            self._h, rows, data, stride, xq, w,
            None if bias is None else bias.data_ptr(), y.data_ptr(), ldy,
            self._stream(stream, *used, weight._codes, weight._scales, bias, y)))
        if out is not None:
            self._written(out)
        return y
