"""Python binding of libee.so, the MI355X early-exit serving library.

Argument marshalling only: every step of the hot path runs inside the library's HIP kernels.
PyTorch supplies device memory (tensors) and the HIP stream; there is no CPU fallback -- if the
shared library is missing the import of this module fails.
"""
import ctypes as C
import functools
import os
from operator import index

import numpy as np
import torch  # noqa: F401  -- first: libee.so must bind to the HIP runtime PyTorch has already loaded

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libee.so")

EE_OK, EE_ERR_ARG, EE_ERR_SHAPE, EE_ERR_UNSUPPORTED, EE_ERR_DEVICE, EE_ERR_OVERFLOW = 0, -1, -2, -3, -4, -5
EE_I8, EE_BF16 = 0, 1
K_NAMES = ["conv_mfma", "conv_first", "conv_direct", "depthwise", "maxpool", "pad_input", "gap", "fc", "softmax",
           "compact", "admit", "conv_stream", "group_norm"]

RESULT_DT = np.dtype([("exit_idx", "<i4"), ("label", "<i4"), ("conf", "<f4"), ("pad_", "<i4"),
                      ("score", "<i8"), ("latency_ns", "<i8")])
EVENT_DT = np.dtype([("t_ns", "<i8"), ("kind", "<i4"), ("stage", "<i4"), ("b", "<i4"), ("aux", "<i4")])

SYMBOLS = ["ee_strerror", "ee_blob_check", "ee_create", "ee_destroy", "ee_query", "ee_stage_forward", "ee_exit_head",
           "ee_compact_refill", "ee_serve_stream", "ee_schedule_sim", "ee_measure_lut", "ee_profile_enable",
           "ee_profile_read", "ee_kernel_name", "ee_exp2_table", "ee_tune_conv_tile", "ee_ir_count", "ee_ir_layers", "ee_ir_mode", "ee_ir_table", "ee_ir_set", "ee_group_table", "ee_group_set", "ee_last_logits", "ee_profile_reserve", "ee_autotune", "ee_config_table",
           "ee_pair_count", "ee_pair_mode", "ee_pair_table", "ee_config_set", "ee_pair_set", "ee_exit_head_static",
           "ee_static_scratch_bytes", "ee_time_layer", "ee_lanes", "ee_zero_copy_supported", "ee_group_norm_workspace", "ee_group_norm",
           "ee_adapter_bytes", "ee_adapter_pack", "ee_adapter_load", "ee_adapter_workspace", "ee_adapter_project", "ee_verify_workspace", "ee_verify_draft"]
ACTS = {"none": 0, "relu": 1, "relu6": 2, "silu": 3}


class Trace(C.Structure):
    _fields_ = [("n", C.c_int64), ("arrival_ns", C.c_void_p)]


class ServeOpts(C.Structure):
    _fields_ = [("b_max", C.c_int32), ("clock", C.c_int32), ("t_slo_ns", C.c_int64), ("lut_ns", C.c_void_p),
                ("min_incr", C.c_int32), ("refill", C.c_int32), ("t_timeout_ns", C.c_int64), ("lanes", C.c_int32), ("zero_copy", C.c_int32)]


class ServeStats(C.Structure):
    _fields_ = [("rounds", C.c_int64), ("criterion_evals", C.c_int64), ("preemptions", C.c_int64),
                ("end_time_ns", C.c_int64), ("seg_runs", C.c_int64 * 8), ("seg_samples", C.c_int64 * 8),
                ("n_events", C.c_int64)]


class KernelStat(C.Structure):
    _fields_ = [("launches", C.c_int64), ("ms", C.c_double), ("ops", C.c_double), ("bytes", C.c_double)]


class NormDesc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "act", "b", "pixels", "c", "groups", "frac_bits", "res_shift")] + [("eps", C.c_float), ("pad_", C.c_int32)] +
                [(n, C.c_int64) for n in ("x_sample", "x_pixel", "res_sample", "res_pixel", "y_sample", "y_pixel")])


class AdapterDims(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("ci", "co", "adapters", "rank")]


class AdapterCall(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("packed", "pool", "x", "y", "ids", "offsets")] + [("ldx", C.c_int64), ("ldy", C.c_int64)] +
                [(n, C.c_int32) for n in ("rows", "slots", "per", "out_f32")] + [("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)])


class VerifyCall(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("draft", "p", "q", "u", "lengths", "accepted", "tokens")] +
                [(n, C.c_int64) for n in ("draft_row", "u_row", "p_seq", "p_row", "q_seq", "q_row")] +
                [(n, C.c_int32) for n in ("b", "k", "v", "f32")] + [("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)])


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2209_13443_amd.build` "
                      "(there is no fallback implementation)")
_lib = C.CDLL(LIB_PATH)
_lib.ee_strerror.restype = C.c_char_p
_lib.ee_kernel_name.restype = C.c_char_p
_lib.ee_exp2_table.restype = C.POINTER(C.c_uint32)
_V = C.c_void_p
_lib.ee_blob_check.argtypes = [_V, C.c_size_t]
_lib.ee_create.argtypes = [_V, C.c_size_t, C.c_int, C.c_int, _V, C.POINTER(_V)]
_lib.ee_destroy.argtypes = [_V]
_lib.ee_query.argtypes = [_V, C.POINTER(C.c_int), _V, _V]
_lib.ee_stage_forward.argtypes = [_V, C.c_int, C.c_int, _V, _V]
_lib.ee_exit_head.argtypes = [_V, C.c_int, C.c_int, _V, C.c_float, _V, _V, _V, _V]
_lib.ee_exit_head_static.argtypes = [_V, C.c_int, C.c_int, _V, C.c_float, _V, _V, _V, _V]
_lib.ee_static_scratch_bytes.argtypes = []
_lib.ee_lanes.argtypes = [_V, C.c_int]
_lib.ee_time_layer.argtypes = [_V, C.c_int, C.c_int, C.c_int, C.c_int, _V, _V, _V]
_lib.ee_compact_refill.argtypes = [_V, C.c_int, C.c_int, _V, _V, _V, _V, _V, _V, _V, C.c_int, _V, _V]
_lib.ee_serve_stream.argtypes = [_V, C.POINTER(Trace), _V, C.POINTER(ServeOpts), _V, C.POINTER(ServeStats), _V, C.c_int64]
_lib.ee_schedule_sim.argtypes = [C.c_int, C.POINTER(Trace), _V, C.POINTER(ServeOpts), _V, C.POINTER(ServeStats), _V, C.c_int64]
_lib.ee_measure_lut.argtypes = [_V, C.c_int, _V]
_lib.ee_last_logits.argtypes = [_V, C.c_int, _V]
_lib.ee_autotune.argtypes = [_V, C.c_int]
_lib.ee_config_table.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_pair_count.argtypes = [_V]
_lib.ee_zero_copy_supported.argtypes = [_V]
_lib.ee_pair_mode.argtypes = [_V, C.c_int]
_lib.ee_pair_table.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_config_set.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_pair_set.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_ir_count.argtypes = [_V]
_lib.ee_ir_layers.argtypes = [_V, C.c_int]
_lib.ee_ir_mode.argtypes = [_V, C.c_int]
_lib.ee_ir_table.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_ir_set.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_group_table.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_group_set.argtypes = [_V, C.c_int, _V, C.c_int]
_lib.ee_profile_enable.argtypes = [_V, C.c_int]
_lib.ee_profile_read.argtypes = [_V, _V, _V]
_lib.ee_profile_reserve.argtypes = [_V, C.c_int64]
_lib.ee_group_norm_workspace.argtypes = [_V, _V]
_lib.ee_group_norm.argtypes = [_V] * 7 + [C.c_int64, _V]
_lib.ee_adapter_bytes.argtypes = [_V, _V, _V]
_lib.ee_adapter_pack.argtypes = [_V, _V, C.c_int64, _V, _V, _V]
_lib.ee_adapter_load.argtypes = [_V, C.c_int, C.c_int, _V, C.c_int64, _V, C.c_int64, C.c_float, _V, _V]
_lib.ee_adapter_workspace.argtypes = [_V, C.c_int, _V]
_lib.ee_adapter_project.argtypes = [_V, _V, _V]
_lib.ee_verify_workspace.argtypes = [C.c_int, C.c_int, C.c_int, _V]
_lib.ee_verify_draft.argtypes = [_V, _V]


class EEError(RuntimeError):
    def __init__(self, code):
        super().__init__(f"libee: {_lib.ee_strerror(code).decode()} ({code})")
        self.code = code


def _chk(rc):
    if rc != 0:
        raise EEError(rc)


def raw():
    """The ctypes handle (tests call the C ABI directly through it)."""
    return _lib


def strerror(code):
    return _lib.ee_strerror(code).decode()


def blob_check(blob_bytes):
    buf = np.frombuffer(blob_bytes, np.uint8) if not isinstance(blob_bytes, np.ndarray) else blob_bytes
    return _lib.ee_blob_check(buf.ctypes.data, buf.size)


def tune_conv_tile(tile):
    return _lib.ee_tune_conv_tile(int(tile))


def exp2_table():
    return np.ctypeslib.as_array(_lib.ee_exp2_table(), shape=(256,)).copy()


def _np_ptr(a):
    return None if a is None else a.ctypes.data


def _stats_dict(st, n_stages):
    return dict(rounds=st.rounds, criterion_evals=st.criterion_evals, preemptions=st.preemptions,
                end_time_ns=st.end_time_ns, seg_runs=list(st.seg_runs)[:n_stages],
                seg_samples=list(st.seg_samples)[:n_stages], n_events=st.n_events)


def schedule_sim(n_stages, arrival_ns, forced_exit, b_max, lut_ns, t_slo_ns=-1, min_incr=1, refill=1, max_events=0, t_timeout_ns=0, lanes=1):
    """ee_schedule_sim: Algorithm 1 on the virtual clock with forced exits (host only)."""
    arrival_ns = np.ascontiguousarray(arrival_ns, np.int64)
    forced_exit = np.ascontiguousarray(forced_exit, np.int32)
    lut_ns = np.ascontiguousarray(lut_ns, np.int64)
    n = arrival_ns.size
    tr = Trace(n, arrival_ns.ctypes.data)
    opts = ServeOpts(b_max, 1, t_slo_ns, lut_ns.ctypes.data, min_incr, refill, t_timeout_ns, lanes, 0)
    res = np.zeros(n, RESULT_DT)
    ev = np.zeros(max(max_events, 1), EVENT_DT)
    st = ServeStats()
    _chk(_lib.ee_schedule_sim(n_stages, C.byref(tr), forced_exit.ctypes.data, C.byref(opts), res.ctypes.data,
                              C.byref(st), ev.ctypes.data if max_events else None, max_events))
    return res, _stats_dict(st, n_stages), ev[:min(st.n_events, max_events)]


class Engine:
    """One network resident on the GPU.  Tensors are torch CUDA tensors (int8, or int16 holding bf16 bits)."""

    def __init__(self, blob, b_max, stream=None):
        import torch
        self.torch = torch
        buf = blob.buffer() if hasattr(blob, "buffer") else np.frombuffer(blob, np.uint8)
        self.dtype = int(np.frombuffer(buf[12:16].tobytes(), "<i4")[0])
        self.b_max = b_max
        self.stream = torch.cuda.current_stream() if stream is None else stream
        h = _V()
        _chk(_lib.ee_create(buf.ctypes.data, buf.size, b_max, self.dtype, _V(self.stream.cuda_stream), C.byref(h)))
        self._h = h
        n = C.c_int()
        ib, ob = (C.c_int64 * 8)(), (C.c_int64 * 8)()
        _chk(_lib.ee_query(self._h, C.byref(n), ib, ob))
        self.n_stages = n.value
        self.stage_in_bytes, self.stage_out_bytes = list(ib)[:n.value], list(ob)[:n.value]
        self.tdtype = torch.int8 if self.dtype == EE_I8 else torch.int16
        self.esize = 1 if self.dtype == EE_I8 else 2
        self._counts = torch.zeros(2, dtype=torch.int32, pin_memory=True)

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:      # module globals are gone at interpreter exit
            _lib.ee_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()

    # -- single steps ----------------------------------------------------------------------
    def stage_forward(self, stage, act_in, out_shape):
        t = self.torch
        b = act_in.shape[0]
        out = t.empty((b,) + tuple(out_shape), dtype=self.tdtype, device=act_in.device)
        _chk(_lib.ee_stage_forward(self._h, stage, b, act_in.data_ptr(), out.data_ptr()))
        return out

    def exit_head(self, stage, act, thr):
        t = self.torch
        b, dev = act.shape[0], act.device
        label = t.empty(b, dtype=t.int32, device=dev)
        conf = t.empty(b, dtype=t.float32, device=dev)
        score = t.empty(b, dtype=t.int64, device=dev)
        flag = t.empty(b, dtype=t.uint8, device=dev)
        _chk(_lib.ee_exit_head(self._h, stage, b, act.data_ptr(), thr, label.data_ptr(), conf.data_ptr(),
                               score.data_ptr(), flag.data_ptr()))
        return label, conf, score, flag

    def exit_head_static(self, stage, act, thr, label, conf, score, flag):
        """ee_exit_head_static: the caller brings the four per-slot output tensors; nothing is allocated."""
        _chk(_lib.ee_exit_head_static(self._h, stage, act.shape[0], act.data_ptr(), thr, label.data_ptr(), conf.data_ptr(),
                                      score.data_ptr(), flag.data_ptr()))

    def last_logits(self, b, n_cls):
        out = np.empty((b, n_cls), np.int32 if self.dtype == EE_I8 else np.float32)
        _chk(_lib.ee_last_logits(self._h, b, out.ctypes.data))
        return out

    def compact_refill(self, stage, flags, act_src, ids_src, refill_act=None, refill_ids=None):
        t = self.torch
        b, dev = act_src.shape[0], act_src.device
        b_incr = 0 if refill_act is None else refill_act.shape[0]
        # the call writes every row that is handed back; rows whose id nobody gives stay -1
        dst = t.empty((b + b_incr,) + tuple(act_src.shape[1:]), dtype=act_src.dtype, device=dev)
        ids_dst = (t.full((b + b_incr,), -1, dtype=t.int32, device=dev) if b_incr and refill_ids is None
                   else t.empty(b + b_incr, dtype=t.int32, device=dev))
        counts = self._counts                           # pinned: written by the kernel, read without a copy
        _chk(_lib.ee_compact_refill(self._h, stage, b, flags.data_ptr(), act_src.data_ptr(), dst.data_ptr(),
                                    ids_src.data_ptr(), ids_dst.data_ptr(),
                                    None if refill_act is None else refill_act.data_ptr(),
                                    None if refill_ids is None else refill_ids.data_ptr(), b_incr,
                                    counts.data_ptr(), counts.data_ptr() + 4))
        self.stream.synchronize()
        b_rem, b_merged = counts.tolist()
        return dst[:b_merged], ids_dst[:b_merged], b_rem, b_merged

    # -- stream serving ----------------------------------------------------------------------
    def serve_stream(self, arrival_ns, pool, lut_ns, b_max=None, clock=0, t_slo_ns=-1, min_incr=1, refill=1, max_events=0, t_timeout_ns=0, lanes=1,
                     zero_copy=0):
        arrival_ns = np.ascontiguousarray(arrival_ns, np.int64)
        lut_ns = np.ascontiguousarray(lut_ns, np.int64)
        b_max = b_max or self.b_max
        assert lut_ns.shape == (self.n_stages, b_max)
        n = arrival_ns.size
        tr = Trace(n, arrival_ns.ctypes.data)
        opts = ServeOpts(b_max, clock, t_slo_ns, lut_ns.ctypes.data, min_incr, refill, t_timeout_ns, lanes, int(zero_copy))
        res = np.zeros(n, RESULT_DT)
        ev = np.zeros(max(max_events, 1), EVENT_DT)
        st = ServeStats()
        _chk(_lib.ee_serve_stream(self._h, C.byref(tr), pool.data_ptr(), C.byref(opts), res.ctypes.data, C.byref(st),
                                  ev.ctypes.data if max_events else None, max_events))
        return res, _stats_dict(st, self.n_stages), ev[:min(st.n_events, max_events)]

    def zero_copy_supported(self):
        return _lib.ee_zero_copy_supported(self._h) == 1

    def set_lanes(self, n):
        """ee_lanes: workspace and streams for n concurrent steps of the stage-pool policy; returns the lane count"""
        rc = _lib.ee_lanes(self._h, int(n))
        if rc < 0:
            _chk(rc)
        return rc

    def measure_lut(self, reps=3):
        lut = np.zeros((self.n_stages, self.b_max), np.int64)
        _chk(_lib.ee_measure_lut(self._h, reps, lut.ctypes.data))
        return lut

    def time_layer(self, layer, b, cfg=0, reps=20):
        """(microseconds per launch, 2 * MACs, algorithmic bytes) of one layer alone; None when the configuration does not exist"""
        us, ops, byt = C.c_double(), C.c_double(), C.c_double()
        rc = _lib.ee_time_layer(self._h, int(layer), int(b), int(cfg), int(reps), C.byref(us), C.byref(ops), C.byref(byt))
        if rc == EE_ERR_DEVICE and cfg:
            return None
        _chk(rc)
        return us.value, ops.value, byt.value

    def autotune(self, reps=5):
        _chk(_lib.ee_autotune(self._h, int(reps)))

    def config_table(self, layer):
        buf = (C.c_int * 16)()
        n = _lib.ee_config_table(self._h, int(layer), buf, 16)
        if n < 0:
            _chk(n)
        return list(buf)[:n]

    def tables(self):
        """The tuned tables as plain data: {"config": {layer: [...]}, "pair": {layer: [...]}} (layers that have one)."""
        out = {"config": {}, "pair": {}, "ir": {}, "group": {}}
        buf = (C.c_int * 16)()
        layer = 0
        while True:
            n = _lib.ee_config_table(self._h, layer, buf, 16)
            if n < 0:                                   # past the last layer
                return out
            if n:
                out["config"][str(layer)] = list(buf)[:n]
            n = _lib.ee_pair_table(self._h, layer, buf, 16)
            if n > 0:
                out["pair"][str(layer)] = list(buf)[:n]
            n = _lib.ee_ir_table(self._h, layer, buf, 16)
            if n > 0:
                out["ir"][str(layer)] = list(buf)[:n]
            n = _lib.ee_group_table(self._h, layer, buf, 16)
            if n > 0:
                out["group"][str(layer)] = list(buf)[:n]
            layer += 1

    def load_tables(self, tables):
        for key, fn in (("config", _lib.ee_config_set), ("pair", _lib.ee_pair_set), ("ir", _lib.ee_ir_set), ("group", _lib.ee_group_set)):
            for layer, cfg in tables.get(key, {}).items():
                buf = (C.c_int * len(cfg))(*cfg)
                _chk(fn(self._h, int(layer), buf, len(cfg)))

    def pair_count(self):
        n = _lib.ee_pair_count(self._h)
        if n < 0:
            _chk(n)
        return n

    def pair_mode(self, mode):
        _chk(_lib.ee_pair_mode(self._h, int(mode)))

    def ir_count(self):
        n = _lib.ee_ir_count(self._h)
        if n < 0:
            _chk(n)
        return n

    def ir_layers(self, layer):
        """layers of the fused block headed by `layer`, 0 when it heads none"""
        n = _lib.ee_ir_layers(self._h, int(layer))
        if n < 0:
            _chk(n)
        return n

    def ir_mode(self, mode):
        _chk(_lib.ee_ir_mode(self._h, int(mode)))

    def ir_table(self, layer):
        buf = (C.c_int * 16)()
        n = _lib.ee_ir_table(self._h, int(layer), buf, 16)
        return list(buf)[:max(n, 0)]

    def pair_table(self, layer):
        buf = (C.c_int * 16)()
        n = _lib.ee_pair_table(self._h, int(layer), buf, 16)
        if n < 0:
            _chk(n)
        return list(buf)[:n]

    def profile(self, enable):
        _chk(_lib.ee_profile_enable(self._h, int(enable)))

    def profile_reserve(self, n_pairs):
        _chk(_lib.ee_profile_reserve(self._h, int(n_pairs)))

    def profile_read(self, n_layers=0):
        arr = (KernelStat * len(K_NAMES))()
        lay = (KernelStat * n_layers)() if n_layers else None
        _chk(_lib.ee_profile_read(self._h, arr, lay))
        cls = {K_NAMES[i]: dict(launches=arr[i].launches, ms=arr[i].ms, ops=arr[i].ops, bytes=arr[i].bytes)
               for i in range(len(K_NAMES))}
        if not n_layers:
            return cls
        return cls, [dict(launches=x.launches, ms=x.ms, ops=x.ops, bytes=x.bytes) for x in lay]


# -- operators on a batch of in-flight requests, outside a network: on the current stream of their tensors' device --------------
def _need(ok, what, code=EE_ERR_ARG):
    if not ok:
        e = EEError(code)
        e.args = (f"{e.args[0]}: {what}",)
        raise e


def _int32(n, what):
    """n for an int32 of the library's: ctypes would cut its upper bits off without a word."""
    n = index(n)
    _need(-1 << 31 <= n < 1 << 31, f"{what} do not fit 32 bits", EE_ERR_OVERFLOW)
    return n


# torch.cuda.current_stream() builds an object for this number: 2.6 us of a call of 8
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _on(device, f, *args):
    """f(*args, handle of the device's current stream) with `device` (its index) current."""
    if device == torch.cuda.current_device():
        _chk(f(*args, _stream_of(device)))
    else:
        with torch.cuda.device(device):
            _chk(f(*args, _stream_of(device)))


def _key(t):
    """All that a call's plan needs to know of a tensor, or of None; device -1: not on a GPU."""
    if t is None:
        return None
    try:
        return t.shape, t.stride(), t.dtype, t.get_device()
    except (AttributeError, TypeError, RuntimeError):
        return (), (), None, -1              # not a tensor, or none with strides: _check says so


def _check(key, name, dtypes, device=None):
    """Of _key(t); returns the device's index (device: the one it has to be)."""
    if key is None or key[2] not in dtypes:
        _need(False, f"{name} has to be a tensor of {' or '.join(str(d) for d in dtypes)}", EE_ERR_UNSUPPORTED)
    _need(key[3] >= 0 and (device is None or key[3] == device), "tensors have to be on the GPU, all on the same one")
    return key[3]


def _pixels(shape, stride, name):
    """(samples, pixels, channels, sample stride, pixel stride) of [b, ..., c]; the dimensions between have to lie behind one another."""
    _need(len(shape) >= 2 and (shape[-1] == 1 or stride[-1] == 1), f"{name} has to be [samples, ..., channels] with neighbouring channels")
    pixels, step = 1, None
    for n, s in zip(shape[-2:0:-1], stride[-2:0:-1]):
        if n > 1:
            _need(step is None or s == step * pixels, f"the pixels of {name} have to lie one stride apart")
            step = s if step is None else step
        pixels *= n
    return shape[0], pixels, shape[-1], stride[0], shape[-1] if step is None else step


def _rows(shape, stride, name):
    """(samples, rows of a sample, channels, stride of the rows) where all rows lie one stride apart."""
    b, inner, c, sample, pixel = _pixels(shape, stride, name)
    _need(inner == 1 or b <= 1 or sample == inner * pixel, f"the rows of {name} have to lie one stride apart")
    return b, inner, c, c if b * inner <= 1 else sample if inner == 1 else pixel


def _workspace(bytes_, device):
    return torch.empty(bytes_, dtype=torch.uint8, device=device) if bytes_ else None


def _ptr(t):
    return None if t is None else t.data_ptr()


# What follows from types, shapes and strides alone is worked out, and checked, once for each of them: 4 to 7 us of a call.

@functools.lru_cache(maxsize=1024)
def _norm_plan(x, out, residual, weight, bias, groups, eps, act, frac_bits, res_shift):
    dev = _check(x, "x", (torch.bfloat16, torch.int8, torch.int16))
    for t, name, dtype in ((out, "out", x[2]), (residual, "residual", x[2]), (weight, "weight", torch.float32), (bias, "bias", torch.float32)):
        if t is not None:
            _check(t, name, (dtype,), dev)
    b, pixels, c, sample, pixel = _pixels(x[0], x[1], "x")
    y = (b, pixels, c, pixels * c, c)
    if out is not None:
        y = _pixels(out[0], out[1], "out")
        _need(out[0] == x[0], "out has to have the shape of x")
        step, step_pixel = abs(y[3]), y[4] if pixels > 1 else c
        _need(b <= 1 or pixels == 0 or step >= (pixels - 1) * step_pixel + c or c <= step and step_pixel >= (b - 1) * step + c, "the samples of out must not share elements")
    r = (0, 0, 0, 0, 0)
    if residual is not None:
        _need(residual[0] == x[0], "residual has to have the shape of x")
        r = _pixels(residual[0], residual[1], "residual")
    for t, name in ((weight, "weight"), (bias, "bias")):
        _need(t is None or t[0] == (c,) and (c == 1 or t[1] == (1,)), f"{name} has to be dense [channels]")
    _need(act in ACTS, f"act has to be one of {', '.join(ACTS)}")
    ints = [_int32(n, "sizes") for n in (b, pixels, c, groups, frac_bits, res_shift)]
    d = NormDesc(EE_I8 if x[2] == torch.int8 else EE_BF16, ACTS[act], *ints, eps, 0, sample, pixel, r[3], r[4], y[3], y[4])
    need = C.c_int64()
    _chk(_lib.ee_group_norm_workspace(C.byref(d), C.byref(need)))
    return dev, C.byref(d), need.value


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, act="none", residual=None, frac_bits=0, res_shift=0, out=None):
    """ee_group_norm: act(group norm of x + residual) on x[b, ..., c] (int8, bfloat16 or int16 holding bf16 bits; any sample stride, one pixel stride, channel slices included).
    weight, bias: float32 [c].  act: "none", "relu", "relu6", "silu" (not int8).  int8: the result is in units of 2^-frac_bits, the residual enters times 2^res_shift.
    out may be x or residual, or share nothing with them."""
    dev, desc, need = _norm_plan(_key(x), _key(out), _key(residual), _key(weight), _key(bias), index(groups), float(eps), act, index(frac_bits), index(res_shift))
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    ws = _workspace(need, x.device)
    _on(dev, _lib.ee_group_norm, desc, x.data_ptr(), _ptr(weight), _ptr(bias), _ptr(residual), out.data_ptr(), _ptr(ws), need)
    return out


@functools.lru_cache(maxsize=1024)
def _adapter_plan(dev, ci, co, adapters, rank, dtype, x, ids, offsets, out):
    _check(x, "x", (torch.bfloat16,), dev)
    _need(dtype in (torch.bfloat16, torch.float32), "results are bfloat16 or float32", EE_ERR_UNSUPPORTED)
    for t, name, kind in ((offsets, "offsets", torch.int32), (ids, "ids", torch.int32), (out, "out", dtype)):
        if t is not None:
            _check(t, name, (kind,), dev)
    if offsets is not None:
        _need(len(x[0]) == 2 and len(offsets[0]) == 1 and offsets[0][0] >= 1 and (offsets[0][0] == 1 or offsets[1] == (1,)), "offsets go with x [rows, ci]")
    b, inner, channels, ldx = _rows(x[0], x[1], "x")
    _need(channels == ci, "x has to have ci channels")
    slots, per = (b, inner) if offsets is None else (offsets[0][0] - 1, 0)
    _need(ids is None or ids[0] == (slots,) and (slots <= 1 or ids[1] == (1,)), "ids has to be dense [slots]")
    ldy = co
    if out is not None:
        _need(out[0] == x[0][:-1] + (co,), "out has to have the shape of x with co channels")
        ldy = _rows(out[0], out[1], "out")[3]
        _need(b * inner <= 1 or ldy >= co, "the rows of out must not share elements")
    rows = _int32(b * inner, "rows")
    dims, need = AdapterDims(ci, co, adapters, rank), C.c_int64()
    _chk(_lib.ee_adapter_workspace(C.byref(dims), rows, C.byref(need)))
    return rows, _int32(slots, "slots"), _int32(per, "rows"), ldx, ldy, need.value


class AdapterProjection:
    """ee_adapter_*: a shared projection x w^T + bias and, beside it, the low-rank adapter of each request.  weight: bfloat16 [co, ci]; bias: float32 [co].
    Room for `adapters` adapters of rank <= `rank`; load() puts one in (also between calls), unload() takes it out."""

    def __init__(self, weight, bias=None, adapters=0, rank=16):
        at = _check(_key(weight), "weight", (torch.bfloat16,))
        dev = weight.device
        _need(weight.dim() == 2 and (weight.stride(1) == 1 or weight.shape[1] == 1), "weight has to be [co, ci] with dense rows")
        co, ci = weight.shape
        if bias is not None:
            _check(_key(bias), "bias", (torch.float32,), at)
            _need(bias.shape == (co,) and bias.is_contiguous(), "bias has to be dense [co]")
        adapters, rank = _int32(adapters, "adapters"), _int32(rank, "ranks")
        self.device, self.ci, self.co, self.adapters, self.rank = dev, _int32(ci, "columns"), _int32(co, "outputs"), adapters, rank
        self._dims = AdapterDims(ci, co, adapters, rank)
        packed, pool = C.c_int64(), C.c_int64()
        _chk(_lib.ee_adapter_bytes(C.byref(self._dims), C.byref(packed), C.byref(pool)))
        self._packed = torch.empty(packed.value, dtype=torch.uint8, device=dev)
        self._pool = torch.zeros(pool.value, dtype=torch.uint8, device=dev)
        _on(at, _lib.ee_adapter_pack, C.byref(self._dims), weight.data_ptr(), weight.stride(0) if co > 1 else ci, _ptr(bias), self._packed.data_ptr())

    def load(self, i, a, b, scale=1.0):
        """Adapter i becomes scale * b a (a: bfloat16 [r, ci], b: bfloat16 [co, r], r <= rank), for the calls behind this one on its stream."""
        at, ka, kb = self.device.index, _key(a), _key(b)
        _check(ka, "a", (torch.bfloat16,), at)
        _check(kb, "b", (torch.bfloat16,), at)
        _need(len(ka[0]) == 2 and len(kb[0]) == 2, "a has to be [r, ci] and b [co, r]")
        r = _int32(ka[0][0], "ranks")
        _need(ka[0] == (r, self.ci) and kb[0] == (self.co, r), "a has to be [r, ci] and b [co, r]")
        _need((ka[1][1] == 1 or self.ci == 1) and (kb[1][1] == 1 or r == 1), "a and b have to have dense rows")
        _on(at, _lib.ee_adapter_load, C.byref(self._dims), _int32(i, "adapters"), r, a.data_ptr(), ka[1][0] if r > 1 else self.ci, b.data_ptr(), kb[1][0] if self.co > 1 else r, scale, self._pool.data_ptr())

    def unload(self, i):
        _on(self.device.index, _lib.ee_adapter_load, C.byref(self._dims), _int32(i, "adapters"), 0, None, 0, None, 0, 0.0, self._pool.data_ptr())

    def __call__(self, x, ids=None, offsets=None, out=None, dtype=torch.bfloat16):
        """x: bfloat16 [slots, ..., ci] or, with offsets (int32 [slots + 1]), [rows, ci] with the rows of slot s at offsets[s]..offsets[s + 1]; ids: int32 [slots], the adapter of
        every slot, outside [0, adapters): none.  Returns bfloat16 or float32 (dtype) with co in place of ci; out must not overlap x.  Rows that belong to no slot are left as they were
        in out; where out is not given they hold whatever the new memory held."""
        dev = self.device.index
        rows, slots, per, ldx, ldy, need = _adapter_plan(dev, self.ci, self.co, self.adapters, self.rank, dtype, _key(x), _key(ids), _key(offsets), _key(out))
        if out is None:
            out = torch.empty(x.shape[:-1] + (self.co,), dtype=dtype, device=self.device)
        ws = _workspace(need, self.device)
        c = AdapterCall(self._packed.data_ptr(), self._pool.data_ptr(), x.data_ptr(), out.data_ptr(), _ptr(ids), _ptr(offsets), ldx, ldy, rows, slots, per,
                        dtype == torch.float32, _ptr(ws), need)
        _on(dev, _lib.ee_adapter_project, C.byref(self._dims), C.byref(c))
        return out


@functools.lru_cache(maxsize=1024)
def _verify_plan(p, draft, u, q, lengths):
    dev = _check(p, "target_probs", (torch.float32, torch.bfloat16))
    _check(draft, "draft", (torch.int32,), dev)
    _check(u, "u", (torch.float32,), dev)
    if q is not None:
        _check(q, "draft_probs", (p[2],), dev)
    if lengths is not None:
        _check(lengths, "lengths", (torch.int32,), dev)
    dense = lambda t: t[0][-1] <= 1 or t[1][-1] == 1
    _need(len(draft[0]) == 2 and len(p[0]) == 3, "draft has to be [b, k], target_probs [b, k + 1, v]")
    (b, k), v = draft[0], p[0][2]
    _need(p[0][:2] == (b, k + 1) and u[0] == (b, k + 1), "target_probs and u have to have k + 1 rows a sequence")
    _need(dense(p) and dense(draft) and dense(u), "the last dimension has to be dense")
    _need(q is None or q[0] == (b, k, v) and dense(q), "draft_probs has to be [b, k, v] with dense rows")
    _need(lengths is None or lengths[0] == (b,) and (b <= 1 or lengths[1] == (1,)), "lengths has to be dense [b]")
    b, k, v = _int32(b, "sequences"), _int32(k, "drafts"), _int32(v, "tokens")
    need = C.c_int64()
    _chk(_lib.ee_verify_workspace(b, k, v, C.byref(need)))
    return dev, b, k, v, (draft[1][0], u[1][0], p[1][0], p[1][1]) + ((0, 0) if q is None else q[1][:2]), need.value


def verify_draft(draft, target_probs, u, draft_probs=None, lengths=None):
    """ee_verify_draft: (accepted int32 [b], tokens int32 [b, k + 1]) for draft int32 [b, k] against target_probs [b, k + 1, v] (float32 or bfloat16), drawn from draft_probs
    [b, k, v] (same type; None: certain), with the random numbers u float32 [b, k + 1] in [0, 1).  lengths int32 [b]: drafts per sequence, < 0: an empty slot."""
    at, b, k, v, strides, need = _verify_plan(_key(target_probs), _key(draft), _key(u), _key(draft_probs), _key(lengths))
    dev = target_probs.device
    accepted = torch.empty(b, dtype=torch.int32, device=dev)
    tokens = torch.empty((b, k + 1), dtype=torch.int32, device=dev)
    ws = _workspace(need, dev)
    c = VerifyCall(draft.data_ptr(), target_probs.data_ptr(), _ptr(draft_probs), u.data_ptr(), _ptr(lengths), accepted.data_ptr(), tokens.data_ptr(), *strides, b, k, v,
                   target_probs.dtype == torch.float32, _ptr(ws), need)
    _on(at, _lib.ee_verify_draft, C.byref(c))
    return accepted, tokens
