"""ctypes binding of include/flashoptim.h: argument marshalling only.

Every function here has the name of the C entry point it calls (without the
`flashoptim_` prefix) and does nothing but turn torch tensors into device pointers.
torch is used for device memory and streams only.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libflashoptim.so")
_lib = None

KIND = {"adamw": 0, "sgd": 1, "lion": 2}

EXPORTED_SYMBOLS = [
    "flashoptim_adamw_step", "flashoptim_adamw_step_exact", "flashoptim_sgd_step", "flashoptim_lion_step",
    "flashoptim_split_weights", "flashoptim_reconstruct_weights",
    "flashoptim_quantize_momentum", "flashoptim_dequantize_momentum",
    "flashoptim_quantize_variance", "flashoptim_dequantize_variance",
    "flashoptim_checkpoint_size", "flashoptim_checkpoint_pack", "flashoptim_checkpoint_unpack",
    "flashoptim_strerror", "flashoptim_last_hip_error", "flashoptim_release_cache", "flashoptim_version",
    "flashoptim_faithful_rounding_stats", "flashoptim_short_sqrt_state", "flashoptim_clock_monitor",
    "flashoptim_step_launch_count",
    "flashoptim_selftest", "flashoptim_split_weights_i16", "flashoptim_reconstruct_weights_i16",
    "flashoptim_reconstruction_sweep", "flashoptim_reconstruction_sweep_ex",
    "flashoptim_adamw_step_ex", "flashoptim_sgd_step_ex", "flashoptim_lion_step_ex",
    "flashoptim_quantize_state", "flashoptim_dequantize_state", "flashoptim_quantization_nmse",
    "flashoptim_compress_state", "flashoptim_decompress_state", "flashoptim_stream_probe",
    "flashoptim_adamw_step_noalloc", "flashoptim_shard_range",
    "flashoptim_mx4_quantize", "flashoptim_mx4_dequantize", "flashoptim_mx4_matmul_workspace", "flashoptim_mx4_linear_workspace",
    "flashoptim_mx4_linear_backward_workspace", "flashoptim_mx4_matmul", "flashoptim_mx4_linear", "flashoptim_mx4_linear_backward",
    "flashoptim_block_norm", "flashoptim_block_norm_backward_workspace", "flashoptim_block_norm_backward",
    "flashoptim_token_logprob_workspace", "flashoptim_token_logprob", "flashoptim_token_logprob_backward",
    "flashoptim_policy_loss_workspace", "flashoptim_policy_loss", "flashoptim_preference_loss",
    "flashoptim_grad_norm_workspace", "flashoptim_grad_norm", "flashoptim_clip_factor_from_sum", "flashoptim_clip_gradients",
    "flashoptim_adamw_step_clipped", "flashoptim_adamw_step_exact_clipped", "flashoptim_sgd_step_clipped", "flashoptim_lion_step_clipped",
]


class FlashOptimError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = strerror(status)
        if status == -4:
            msg += f" (hipError_t {load_library().flashoptim_last_hip_error()})"
        super().__init__(f"{where}: {msg} [{status}]")


class _Tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("rho", C.c_void_p), ("grad", C.c_void_p),
                ("m_q", C.c_void_p), ("m_scale", C.c_void_p), ("v_q", C.c_void_p), ("v_scale", C.c_void_p),
                ("numel", C.c_int64), ("lr", C.c_float), ("weight_decay", C.c_float)]


class _TensorEx(C.Structure):
    _fields_ = [("t", _Tensor), ("theta", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p)]


SPLIT_WEIGHTS, QUANTIZE_STATES = 1, 2


class _AdamWHp(C.Structure):
    _fields_ = [("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("step", C.c_int64)]


class _SgdHp(C.Structure):
    _fields_ = [("momentum", C.c_float)]


class _LionHp(C.Structure):
    _fields_ = [("beta1", C.c_float), ("beta2", C.c_float)]


class _Matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("stride", C.c_int64), ("dtype", C.c_int32)]


class _Mx4(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64)]


class _BlockNormSpec(C.Structure):
    _fields_ = [("cols", C.c_int64), ("kind", C.c_int32), ("post_norm", C.c_int32), ("gate_act", C.c_int32),
                ("param_dtype", C.c_int32), ("eps", C.c_float), ("residual_scale", C.c_float), ("branch_scale", C.c_float),
                ("post_weight", C.c_void_p), ("post_bias", C.c_void_p), ("pre_weight", C.c_void_p), ("pre_bias", C.c_void_p)]


class _BlockNormGrads(C.Structure):
    _fields_ = [(n, C.POINTER(_Matrix)) for n in ("dy", "dh", "dx", "df", "dgate")] + \
               [(n, C.c_void_p) for n in ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")]


class _PolicySpec(C.Structure):
    _fields_ = [(n, C.c_float) for n in ("temperature", "clip_low", "clip_high", "kl_weight", "grad_scale")]


class _PolicyInputs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("advantages", "old_logprob", "ref_logprob", "weights")]


class _PreferenceSpec(C.Structure):
    _fields_ = [("kind", C.c_int32), ("order", C.c_int32), ("beta", C.c_float), ("label_smoothing", C.c_float), ("grad_scale", C.c_float)]


class _Gradient(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("numel", C.c_int64)]


def library_path():
    return _LIB_PATH


def load_library():
    """Loads the in-tree HIP library.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python paper_2602_23349_amd/build.py`")
    L = C.CDLL(_LIB_PATH)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    L.flashoptim_adamw_step.argtypes = [C.POINTER(_Tensor), i64, C.POINTER(_AdamWHp), vp]
    L.flashoptim_adamw_step_exact.argtypes = [C.POINTER(_Tensor), i64, C.POINTER(_AdamWHp), vp]
    L.flashoptim_adamw_step_noalloc.argtypes = [C.POINTER(_Tensor), i64, C.POINTER(_AdamWHp), vp]
    L.flashoptim_shard_range.argtypes = [i64, i64, i64, C.POINTER(i64), C.POINTER(i64)]
    L.flashoptim_sgd_step.argtypes = [C.POINTER(_Tensor), i64, C.POINTER(_SgdHp), vp]
    L.flashoptim_lion_step.argtypes = [C.POINTER(_Tensor), i64, C.POINTER(_LionHp), vp]
    L.flashoptim_adamw_step_ex.argtypes = [C.POINTER(_TensorEx), i64, C.POINTER(_AdamWHp), C.c_uint, vp]
    L.flashoptim_sgd_step_ex.argtypes = [C.POINTER(_TensorEx), i64, C.POINTER(_SgdHp), C.c_uint, vp]
    L.flashoptim_lion_step_ex.argtypes = [C.POINTER(_TensorEx), i64, C.POINTER(_LionHp), C.c_uint, vp]
    L.flashoptim_reconstruction_sweep.argtypes = [i32, C.c_uint64, C.c_uint64, C.POINTER(C.c_double), vp]
    L.flashoptim_reconstruction_sweep_ex.argtypes = [i32, i32, C.c_uint64, C.c_uint64, C.POINTER(C.c_double), vp]
    for name in ("flashoptim_split_weights", "flashoptim_reconstruct_weights", "flashoptim_split_weights_i16",
                 "flashoptim_reconstruct_weights_i16", "flashoptim_quantize_momentum",
                 "flashoptim_dequantize_momentum", "flashoptim_quantize_variance", "flashoptim_dequantize_variance"):
        getattr(L, name).argtypes = [vp, vp, vp, i64, vp]
    L.flashoptim_compress_state.argtypes = [i32, C.POINTER(_TensorEx), i64, vp]
    L.flashoptim_decompress_state.argtypes = [i32, C.POINTER(_TensorEx), i64, vp]
    L.flashoptim_stream_probe.argtypes = [i32, C.POINTER(_Tensor), i64, vp]
    L.flashoptim_quantize_state.argtypes = [i32, i32, vp, vp, vp, i64, vp]
    L.flashoptim_dequantize_state.argtypes = [i32, i32, vp, vp, vp, i64, vp]
    L.flashoptim_quantization_nmse.argtypes = [i32, i32, vp, i64, C.POINTER(C.c_double), vp]
    L.flashoptim_checkpoint_size.argtypes = [i32, C.POINTER(i64), i64]
    L.flashoptim_checkpoint_size.restype = i64
    L.flashoptim_step_launch_count.argtypes = [i32, C.POINTER(i64), i64]
    L.flashoptim_step_launch_count.restype = i64
    L.flashoptim_checkpoint_pack.argtypes = [i32, C.POINTER(_Tensor), i64, i64, vp, i64, vp]
    L.flashoptim_checkpoint_unpack.argtypes = [i32, vp, i64, C.POINTER(_Tensor), i64, C.POINTER(i64), vp]
    L.flashoptim_selftest.argtypes = [C.POINTER(i64), C.POINTER(i64), vp]
    L.flashoptim_faithful_rounding_stats.argtypes = [C.POINTER(i64), vp]
    L.flashoptim_clock_monitor.argtypes = [C.POINTER(C.c_uint64), i64, C.c_double, C.POINTER(C.c_double), vp]
    mat, mx4, spec = C.POINTER(_Matrix), C.POINTER(_Mx4), C.POINTER(_BlockNormSpec)
    L.flashoptim_mx4_quantize.argtypes = [mat, vp, vp, mx4, mx4, vp]
    L.flashoptim_mx4_dequantize.argtypes = [mx4, mat, vp]
    L.flashoptim_mx4_matmul.argtypes = [mx4, mx4, mat, vp, i64, vp]
    L.flashoptim_mx4_linear.argtypes = [mat, mx4, mx4, mat, vp, i64, vp]
    L.flashoptim_mx4_linear_backward.argtypes = [mat, vp, mx4, mx4, mat, mat, vp, i64, vp]
    L.flashoptim_block_norm.argtypes = [spec, mat, mat, mat, mat, mat, vp, vp]
    L.flashoptim_block_norm_backward.argtypes = [spec, mat, mat, mat, vp, C.POINTER(_BlockNormGrads), vp, i64, vp]
    L.flashoptim_block_norm_backward_workspace.argtypes = [spec, i64, i64]
    for name in ("flashoptim_mx4_matmul_workspace", "flashoptim_mx4_linear_workspace", "flashoptim_mx4_linear_backward_workspace"):
        getattr(L, name).argtypes = [i64, i64, i64]
    for name in ("flashoptim_token_logprob_workspace", "flashoptim_policy_loss_workspace"):
        getattr(L, name).argtypes = [i64, i64, i32]
    L.flashoptim_token_logprob.argtypes = [mat, vp, C.c_float, vp, vp, vp, vp, i64, vp]
    L.flashoptim_token_logprob_backward.argtypes = [mat, vp, C.c_float, vp, vp, mat, vp]
    L.flashoptim_policy_loss.argtypes = [C.POINTER(_PolicySpec), mat, vp, C.POINTER(_PolicyInputs), vp, vp, mat, vp, i64, vp]
    L.flashoptim_preference_loss.argtypes = [C.POINTER(_PreferenceSpec), vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp]
    grads = C.POINTER(_Gradient)
    L.flashoptim_grad_norm_workspace.argtypes = [grads, i64, i32]
    L.flashoptim_grad_norm.argtypes = [grads, i64, i32, C.c_float, vp, vp, i64, vp]
    L.flashoptim_clip_factor_from_sum.argtypes = [vp, C.c_float, vp]
    L.flashoptim_clip_gradients.argtypes = [grads, i64, i32, i32, vp, vp]
    for name, hp in (("adamw_step", _AdamWHp), ("adamw_step_exact", _AdamWHp), ("sgd_step", _SgdHp), ("lion_step", _LionHp)):
        getattr(L, f"flashoptim_{name}_clipped").argtypes = [C.POINTER(_Tensor), i64, C.POINTER(hp), vp, vp]
    L.flashoptim_strerror.argtypes = [i32]
    L.flashoptim_strerror.restype = C.c_char_p
    for name in EXPORTED_SYMBOLS:
        if name.endswith("_workspace"):
            getattr(L, name).restype = i64
        elif name not in ("flashoptim_checkpoint_size", "flashoptim_strerror"):
            getattr(L, name).restype = i32
    _lib = L
    return L


_fast = None


def _marshal():
    """The module that turns tensors into the C ABI's matrices (csrc/marshal.cpp), with this library's entry points bound to it."""
    global _fast
    if _fast is None:
        try:
            from . import _marshal as fast
        except ImportError as e:
            raise RuntimeError("_marshal.so is missing: build it with `python paper_2602_23349_amd/build.py`") from e
        lib = load_library()
        names = [n for n in EXPORTED_SYMBOLS if n.startswith(("flashoptim_mx4_", "flashoptim_block_norm", "flashoptim_token_logprob",
                                                             "flashoptim_policy_loss", "flashoptim_preference_loss", "flashoptim_grad_norm",
                                                             "flashoptim_clip_gradients"))]
        fast.bind({n: C.cast(getattr(lib, n), C.c_void_p).value for n in names}, torch._C._cuda_getCurrentRawStream,
                  torch._C._cuda_getDevice)
        torch.cuda.init()
        _fast = fast
    return _fast


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle straight from torch's runtime: building a torch.cuda.Stream object for it costs 2.7 us,
# as much as the launch itself; asking for the current device through torch.cuda, which initialises CUDA first, another
# 0.15, and wrapping the handle 0.1 (a plain integer is what the argument types take anyway).
_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_current_device = getattr(torch._C, "_cuda_getDevice", None)
_cuda_initialized = torch.cuda.is_initialized


def _stream_handle(stream):
    if stream is None:
        if _raw_current_stream is not None and _raw_current_device is not None and _cuda_initialized():
            return _raw_current_stream(_raw_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _current_device():
    return (_raw_current_device or torch.cuda.current_device)()


def _stream(stream):
    return C.c_void_p(_stream_handle(stream))


def _check(status, where):
    if status != 0:
        raise FlashOptimError(status, where)


class ParamBuffers:
    """Device buffers of one parameter (allocation only).  split_weights / quantize_states choose the
    compressed layout (default) or the FP32 arrays of the ablation variants for each half."""

    def __init__(self, numel, kind, device="cuda", with_grad=True, split_weights=True, quantize_states=True):
        ng = (numel + 31) // 32
        has_v = kind == "adamw"
        self.numel, self.kind = int(numel), kind
        self.split_weights, self.quantize_states = split_weights, quantize_states
        z = lambda n, dt: torch.zeros(n, dtype=dt, device=device)
        self.param = z(numel, torch.bfloat16) if split_weights else None
        self.rho = z(numel, torch.int8) if split_weights else None
        self.theta = None if split_weights else z(numel, torch.float32)
        self.grad = z(numel, torch.bfloat16) if with_grad else None
        self.m_q = z(numel, torch.int8) if quantize_states else None
        self.m_scale = z(ng, torch.float16) if quantize_states else None
        self.v_q = z(numel, torch.uint8) if (quantize_states and has_v) else None
        self.v_scale = z(ng, torch.float16) if (quantize_states and has_v) else None
        self.m = None if quantize_states else z(numel, torch.float32)
        self.v = z(numel, torch.float32) if (not quantize_states and has_v) else None
        self.lr, self.weight_decay = 0.0, 0.0

    @property
    def flags(self):
        return (SPLIT_WEIGHTS if self.split_weights else 0) | (QUANTIZE_STATES if self.quantize_states else 0)

    def shard(self, begin, length):
        """The same buffers restricted to elements [begin, begin + length): views (pointer offsets), no copy.
        begin must be a multiple of 256 (see flashoptim_shard_range)."""
        assert begin % 256 == 0 and 0 <= begin and begin + length <= self.numel
        out = ParamBuffers.__new__(ParamBuffers)
        out.numel, out.kind = int(length), self.kind
        out.split_weights, out.quantize_states = self.split_weights, self.quantize_states
        el = lambda t: None if t is None else t[begin:begin + length]
        gr = lambda t: None if t is None else t[begin // 32:begin // 32 + (length + 31) // 32]
        out.param, out.rho, out.theta, out.grad = el(self.param), el(self.rho), el(self.theta), el(self.grad)
        out.m_q, out.v_q, out.m, out.v = el(self.m_q), el(self.v_q), el(self.m), el(self.v)
        out.m_scale, out.v_scale = gr(self.m_scale), gr(self.v_scale)
        out.lr, out.weight_decay = self.lr, self.weight_decay
        return out


def _device(t):
    return None if t is None else t.get_device()


class TensorList:
    """A host array of flashoptim_tensor descriptors, built once and reused across steps."""

    def __init__(self, buffers):
        self.buffers = list(buffers)
        self.n = len(self.buffers)
        self._lies_on, self._devices = [_device(b.grad) for b in self.buffers], None
        self.array = (_Tensor * max(self.n, 1))()
        for i, b in enumerate(self.buffers):
            d = self.array[i]
            d.param, d.rho, d.grad = _ptr(b.param), _ptr(b.rho), _ptr(b.grad)
            d.m_q, d.m_scale, d.v_q, d.v_scale = _ptr(b.m_q), _ptr(b.m_scale), _ptr(b.v_q), _ptr(b.v_scale)
            d.numel, d.lr, d.weight_decay = b.numel, b.lr, b.weight_decay

    def set_hyper(self, i, lr=None, weight_decay=None):
        if lr is not None:
            self.array[i].lr = lr
        if weight_decay is not None:
            self.array[i].weight_decay = weight_decay

    def set_grad(self, i, grad):
        self.array[i].grad = _ptr(grad)
        device = _device(grad)
        if device != self._lies_on[i]:
            self._lies_on[i], self._devices = device, None

    def grad_device(self):
        """The device of all gradients, None where there are none.  The steps do not ask for it."""
        if self._devices is None:
            self._devices = set(self._lies_on) - {None}
        if len(self._devices) > 1 or -1 in self._devices:
            raise ValueError("gradients: tensors on one GPU")
        return next(iter(self._devices), None)

    def slice(self, i):
        """A one-element list viewing tensor i (for per-tensor, gradient-release style calls)."""
        out = TensorList.__new__(TensorList)
        out.buffers, out.n = [self.buffers[i]], 1
        out._lies_on, out._devices = [self._lies_on[i]], None
        out.array = (_Tensor * 1)()
        C.memmove(out.array, C.byref(self.array[i]), C.sizeof(_Tensor))
        return out


class TensorListEx:
    """Host array of flashoptim_tensor_ex descriptors (ablation and conversion entry points)."""

    def __init__(self, buffers, check_flags=True):
        self.buffers = list(buffers)
        self.n = len(self.buffers)
        self.flags = self.buffers[0].flags if self.buffers else 3
        assert not check_flags or all(b.flags == self.flags for b in self.buffers)
        self.array = (_TensorEx * max(self.n, 1))()
        for i, b in enumerate(self.buffers):
            d = self.array[i]
            d.t.param, d.t.rho, d.t.grad = _ptr(b.param), _ptr(b.rho), _ptr(b.grad)
            d.t.m_q, d.t.m_scale, d.t.v_q, d.t.v_scale = _ptr(b.m_q), _ptr(b.m_scale), _ptr(b.v_q), _ptr(b.v_scale)
            d.t.numel, d.t.lr, d.t.weight_decay = b.numel, b.lr, b.weight_decay
            d.theta, d.m, d.v = _ptr(b.theta), _ptr(b.m), _ptr(b.v)


def _as_list_ex(tensors):
    return tensors if isinstance(tensors, TensorListEx) else TensorListEx(tensors)


def adamw_step_ex(tensors, beta1, beta2, eps, step, flags=None, stream=None):
    tl = _as_list_ex(tensors)
    hp = _AdamWHp(beta1, beta2, eps, int(step))
    _check(load_library().flashoptim_adamw_step_ex(tl.array, tl.n, C.byref(hp), tl.flags if flags is None else flags,
                                                   _stream(stream)), "flashoptim_adamw_step_ex")


def sgd_step_ex(tensors, momentum, flags=None, stream=None):
    tl = _as_list_ex(tensors)
    hp = _SgdHp(momentum)
    _check(load_library().flashoptim_sgd_step_ex(tl.array, tl.n, C.byref(hp), tl.flags if flags is None else flags,
                                                 _stream(stream)), "flashoptim_sgd_step_ex")


def lion_step_ex(tensors, beta1, beta2, flags=None, stream=None):
    tl = _as_list_ex(tensors)
    hp = _LionHp(beta1, beta2)
    _check(load_library().flashoptim_lion_step_ex(tl.array, tl.n, C.byref(hp), tl.flags if flags is None else flags,
                                                  _stream(stream)), "flashoptim_lion_step_ex")


def compress_state(kind, tensors, stream=None):
    tl = tensors if isinstance(tensors, TensorListEx) else TensorListEx(tensors, check_flags=False)
    _check(load_library().flashoptim_compress_state(KIND[kind], tl.array, tl.n, _stream(stream)),
           "flashoptim_compress_state")


def decompress_state(kind, tensors, stream=None):
    tl = tensors if isinstance(tensors, TensorListEx) else TensorListEx(tensors, check_flags=False)
    _check(load_library().flashoptim_decompress_state(KIND[kind], tl.array, tl.n, _stream(stream)),
           "flashoptim_decompress_state")


def _as_list(tensors):
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def _on_current(factor, stream):
    """(launches go to the current device)"""
    if factor.device != _current_device():
        raise ValueError("the factor lies on another device than the current one")
    _check_stream(stream)


def _clipped(name, tl, hp, clip, stream):
    call = f"flashoptim_{name}_clipped"
    _on_current(clip, stream)
    if tl.grad_device() not in (None, clip.device):
        raise ValueError("the gradients and the factor lie on different devices")
    _check(getattr(load_library(), call)(tl.array, tl.n, hp, clip.address, _stream_handle(stream)), call)


def adamw_step(tensors, beta1, beta2, eps, step, stream=None, clip=None):
    """`clip` (ClipFactor, here and in the steps below): the gradients count times its scale; NaN there leaves everything as it is."""
    tl = _as_list(tensors)
    hp = _AdamWHp(beta1, beta2, eps, int(step))
    if clip is not None:
        return _clipped("adamw_step", tl, hp, clip, stream)
    _check(load_library().flashoptim_adamw_step(tl.array, tl.n, hp, _stream_handle(stream)), "flashoptim_adamw_step")


def adamw_step_exact(tensors, beta1, beta2, eps, step, stream=None, clip=None):
    tl = _as_list(tensors)
    hp = _AdamWHp(beta1, beta2, eps, int(step))
    if clip is not None:
        return _clipped("adamw_step_exact", tl, hp, clip, stream)
    _check(load_library().flashoptim_adamw_step_exact(tl.array, tl.n, hp, _stream_handle(stream)),
           "flashoptim_adamw_step_exact")


def adamw_step_noalloc(tensors, beta1, beta2, eps, step, stream=None):
    tl = _as_list(tensors)
    hp = _AdamWHp(beta1, beta2, eps, int(step))
    _check(load_library().flashoptim_adamw_step_noalloc(tl.array, tl.n, hp, _stream_handle(stream)),
           "flashoptim_adamw_step_noalloc")


def shard_range(numel, world, rank):
    """(begin, len) of `rank`'s shard of a flat tensor cut on multiples of 256 elements."""
    begin, length = C.c_int64(0), C.c_int64(0)
    _check(load_library().flashoptim_shard_range(int(numel), int(world), int(rank), C.byref(begin), C.byref(length)),
           "flashoptim_shard_range")
    return int(begin.value), int(length.value)


def sgd_step(tensors, momentum, stream=None, clip=None):
    tl = _as_list(tensors)
    hp = _SgdHp(momentum)
    if clip is not None:
        return _clipped("sgd_step", tl, hp, clip, stream)
    _check(load_library().flashoptim_sgd_step(tl.array, tl.n, hp, _stream_handle(stream)), "flashoptim_sgd_step")


def lion_step(tensors, beta1, beta2, stream=None, clip=None):
    tl = _as_list(tensors)
    hp = _LionHp(beta1, beta2)
    if clip is not None:
        return _clipped("lion_step", tl, hp, clip, stream)
    _check(load_library().flashoptim_lion_step(tl.array, tl.n, hp, _stream_handle(stream)), "flashoptim_lion_step")


def stream_probe(kind, tensors, stream=None):
    """Moves the bytes of one step of `kind` over the list with no arithmetic (state unchanged)."""
    tl = _as_list(tensors)
    _check(load_library().flashoptim_stream_probe(KIND[kind], tl.array, tl.n, _stream(stream)), "flashoptim_stream_probe")


def split_weights(theta, param_bf16, rho, stream=None):
    n = theta.numel()
    _check(load_library().flashoptim_split_weights(_ptr(theta), _ptr(param_bf16), _ptr(rho), n, _stream(stream)),
           "flashoptim_split_weights")


def reconstruct_weights(param_bf16, rho, theta, stream=None):
    n = param_bf16.numel()
    _check(load_library().flashoptim_reconstruct_weights(_ptr(param_bf16), _ptr(rho), _ptr(theta), n, _stream(stream)),
           "flashoptim_reconstruct_weights")


def split_weights_i16(theta, param_bf16, rho, stream=None):
    _check(load_library().flashoptim_split_weights_i16(_ptr(theta), _ptr(param_bf16), _ptr(rho), theta.numel(),
                                                       _stream(stream)), "flashoptim_split_weights_i16")


def reconstruct_weights_i16(param_bf16, rho, theta, stream=None):
    _check(load_library().flashoptim_reconstruct_weights_i16(_ptr(param_bf16), _ptr(rho), _ptr(theta),
                                                             param_bf16.numel(), _stream(stream)),
           "flashoptim_reconstruct_weights_i16")


def reconstruction_sweep(correction_bits, first=0, stride=1, stream=None):
    """Returns the 520 statistics of flashoptim_reconstruction_sweep as a list of floats."""
    stats = (C.c_double * 520)()
    _check(load_library().flashoptim_reconstruction_sweep(int(correction_bits), int(first), int(stride), stats,
                                                          _stream(stream)), "flashoptim_reconstruction_sweep")
    return list(stats)


def reconstruction_sweep_ex(correction_bits, ulp_reading, first=0, stride=1, stream=None):
    """Returns the 776 statistics of flashoptim_reconstruction_sweep_ex (ulp_reading 0 literal, 1 directional)."""
    stats = (C.c_double * 776)()
    _check(load_library().flashoptim_reconstruction_sweep_ex(int(correction_bits), int(ulp_reading), int(first),
                                                             int(stride), stats, _stream(stream)),
           "flashoptim_reconstruction_sweep_ex")
    return list(stats)


def quantize_momentum(m, q, scale, stream=None):
    _check(load_library().flashoptim_quantize_momentum(_ptr(m), _ptr(q), _ptr(scale), m.numel(), _stream(stream)),
           "flashoptim_quantize_momentum")


def dequantize_momentum(q, scale, m, stream=None):
    _check(load_library().flashoptim_dequantize_momentum(_ptr(q), _ptr(scale), _ptr(m), q.numel(), _stream(stream)),
           "flashoptim_dequantize_momentum")


def quantize_variance(v, q, scale, stream=None):
    _check(load_library().flashoptim_quantize_variance(_ptr(v), _ptr(q), _ptr(scale), v.numel(), _stream(stream)),
           "flashoptim_quantize_variance")


def dequantize_variance(q, scale, v, stream=None):
    _check(load_library().flashoptim_dequantize_variance(_ptr(q), _ptr(scale), _ptr(v), q.numel(), _stream(stream)),
           "flashoptim_dequantize_variance")


_STATE = {"momentum": 0, "variance": 1}


def quantize_state(state, linear, x, q, scale, stream=None):
    _check(load_library().flashoptim_quantize_state(_STATE[state], int(bool(linear)), _ptr(x), _ptr(q), _ptr(scale),
                                                    x.numel(), _stream(stream)), "flashoptim_quantize_state")


def dequantize_state(state, linear, q, scale, x, stream=None):
    _check(load_library().flashoptim_dequantize_state(_STATE[state], int(bool(linear)), _ptr(q), _ptr(scale), _ptr(x),
                                                      q.numel(), _stream(stream)), "flashoptim_dequantize_state")


def quantization_nmse(state, linear, x, stream=None):
    """Returns (sum of squared errors, sum of squares) of quantize -> dequantize over x."""
    sums = (C.c_double * 2)()
    _check(load_library().flashoptim_quantization_nmse(_STATE[state], int(bool(linear)), _ptr(x), x.numel(), sums,
                                                       _stream(stream)), "flashoptim_quantization_nmse")
    return float(sums[0]), float(sums[1])


def checkpoint_size(kind, numels):
    arr = (C.c_int64 * max(len(numels), 1))(*[int(x) for x in numels])
    r = load_library().flashoptim_checkpoint_size(KIND[kind], arr, len(numels))
    if r < 0:
        raise FlashOptimError(int(r), "flashoptim_checkpoint_size")
    return int(r)


def checkpoint_pack(kind, tensors, step, blob, stream=None):
    tl = _as_list(tensors)
    _check(load_library().flashoptim_checkpoint_pack(KIND[kind], tl.array, tl.n, int(step), _ptr(blob),
                                                     blob.numel() * blob.element_size(), _stream(stream)),
           "flashoptim_checkpoint_pack")


def checkpoint_unpack(kind, blob, tensors, stream=None):
    tl = _as_list(tensors)
    step = C.c_int64(0)
    _check(load_library().flashoptim_checkpoint_unpack(KIND[kind], _ptr(blob), blob.numel() * blob.element_size(),
                                                       tl.array, tl.n, C.byref(step), _stream(stream)),
           "flashoptim_checkpoint_unpack")
    return int(step.value)


_DTYPE = {torch.bfloat16: 0, torch.float32: 1}


def _handle(stream):
    """What csrc/marshal.cpp takes for a stream: None is the current one."""
    return None if stream is None else _stream_handle(stream)


def _check_stream(stream):
    """(losses, and calls on gradients: their tensors and their stream are the current device's)"""
    device = getattr(stream, "device_index", None)
    if device is not None and device != _current_device():
        raise ValueError("the stream is another device's than the current one")


def _handle_here(stream):
    if stream is None:
        return None
    _check_stream(stream)
    return _stream_handle(stream)


class Mx4Tensor:
    """A matrix of rows by cols values in microscaled 4 bits: `codes` [rows, 128 ceil(cols/256)] and `scales`
    [rows, 16 ceil(cols/512)], both uint8, laid out as flashoptim.h describes.  A new one is a matrix of
    zeros; `buffers`: a (codes, scales) pair to use instead of new memory, of which a call that writes the matrix writes every byte."""

    def __init__(self, rows, cols, device="cuda", buffers=None):
        self.rows, self.cols = int(rows), int(cols)
        shapes = ((self.rows, 128 * -(-self.cols // 256)), (self.rows, 16 * -(-self.cols // 512)))
        if buffers is None:
            buffers = [torch.zeros(s, dtype=torch.uint8, device=device) for s in shapes]
        for t, s in zip(buffers, shapes):
            if t.dtype != torch.uint8 or tuple(t.shape) != s or not t.is_contiguous():
                raise ValueError(f"a {self.rows} by {self.cols} matrix in 4 bits takes contiguous uint8 of shapes {shapes}")
        self.codes, self.scales = buffers
        self.desc = _Mx4(self.codes.data_ptr(), self.scales.data_ptr(), self.rows, self.cols)
        self.address = C.addressof(self.desc) if self.codes.is_cuda and self.scales.is_cuda else -1


def mx4_quantize(x, out=None, out_t=None, rho=None, rand=None, stream=None):
    """out <- x, out_t <- the transpose of x, each in 4 bits along its own rows (Mx4Tensor; either may be None).  rho: x holds
    BF16 weights with these INT8 corrections.  rand: random bytes for stochastic rounding."""
    status = (_fast or _marshal()).quantize(x, None if out is None else out.address, None if out_t is None else out_t.address, rho, rand,
                                            _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_mx4_quantize")


def mx4_dequantize(q, out, stream=None):
    status = (_fast or _marshal()).dequantize(q.address, out, _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_mx4_dequantize")


def _size(r, where):
    if r < 0:
        raise FlashOptimError(int(r), where)
    return int(r)


def mx4_matmul_workspace(m, n, k):
    """Bytes of workspace of mx4_matmul for an m by n result of sums over k terms."""
    return _size(load_library().flashoptim_mx4_matmul_workspace(m, n, k), "flashoptim_mx4_matmul_workspace")


def mx4_linear_workspace(m, n, k):
    return _size(load_library().flashoptim_mx4_linear_workspace(m, n, k), "flashoptim_mx4_linear_workspace")


def mx4_linear_backward_workspace(m, n, k):
    return _size(load_library().flashoptim_mx4_linear_backward_workspace(m, n, k), "flashoptim_mx4_linear_backward_workspace")


def mx4_matmul(a, b, out, workspace=None, stream=None):
    """out [m, n] <- a [m, k] b [n, k]^T, both Mx4Tensor."""
    status = (_fast or _marshal()).matmul(a.address, b.address, out, workspace, _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_mx4_matmul")


def mx4_linear(x, w, out, xt=None, workspace=None, stream=None):
    """out [m, n] <- Q(x) w^T with x [m, k] quantised on the way, w an Mx4Tensor [n, k]; xt: Mx4Tensor [k, m] for Q(x^T).  Without xt
    a few rows, up to 16 where they are not long, are one launch that takes no workspace."""
    status = (_fast or _marshal()).linear(x, w.address, None if xt is None else xt.address, out, workspace, _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_mx4_linear")


def mx4_linear_backward(dy, wt, xt, dx, dw, rand=None, workspace=None, stream=None):
    """dx [m, k] <- Q(dy) wt^T and dw [n, k] <- Q(dy^T) xt^T, with wt [k, n] and xt [k, m] Mx4Tensor; a pair (wt, dx) or (xt, dw)
    may be None."""
    status = (_fast or _marshal()).linear_backward(dy, rand, None if wt is None else wt.address, None if xt is None else xt.address, dx, dw,
                                                   workspace, _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_mx4_linear_backward")


class BlockNorm:
    """The norms between two blocks of `cols` channels: which there are, their weights and scales (flashoptim_block_norm_spec).  The
    weights and biases are BF16 or FP32, all of one type."""

    def __init__(self, cols, kind="rms", eps=1e-5, post_norm=False, gate_act="linear", residual_scale=1.0, branch_scale=1.0,
                 post_weight=None, post_bias=None, pre_weight=None, pre_bias=None):
        self.params = dict(post_weight=post_weight, post_bias=post_bias, pre_weight=pre_weight, pre_bias=pre_bias)
        given = [t for t in self.params.values() if t is not None]
        dtype = given[0].dtype if given else torch.bfloat16
        for name, t in self.params.items():
            if t is not None and (t.dtype not in _DTYPE or t.dtype != dtype or t.numel() != cols or not t.is_contiguous() or not t.is_cuda):
                raise ValueError(f"{name}: {cols} contiguous values on the GPU, bfloat16 or float32, one type for all weights and biases")
        self.cols = int(cols)
        self.desc = _BlockNormSpec(self.cols, {"rms": 0, "layer": 1}.get(kind, -1), int(post_norm),
                                   {"linear": 0, "sigmoid": 1}.get(gate_act, -1), _DTYPE[dtype], eps, residual_scale, branch_scale,
                                   *(_ptr(t) for t in self.params.values()))
        self.address = C.addressof(self.desc)


def block_norm(spec, x, f=None, gate=None, h=None, y=None, stats=None, stream=None):
    """h <- residual_scale x + branch_scale act(gate) u, u = f or its norm; y <- the norm of h (of x without f); stats [4, rows] for
    the backward pass."""
    status = (_fast or _marshal()).norm(spec.address, x, f, gate, h, y, stats, _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_block_norm")


def block_norm_backward_workspace(spec, rows, gates=1):
    return _size(load_library().flashoptim_block_norm_backward_workspace(spec.desc, rows, gates),
                 "flashoptim_block_norm_backward_workspace")


def block_norm_backward(spec, h, stats, f=None, gate=None, dy=None, dh=None, dx=None, df=None, dgate=None, dpost_weight=None,
                        dpost_bias=None, dpre_weight=None, dpre_bias=None, workspace=None, stream=None):
    """The gradients of block_norm that are not None, from dy and dh (either may be None); h is x where there is no branch."""
    status = (_fast or _marshal()).norm_backward(spec.address, h, stats, f, gate, dy, dh, dx, df, dgate, dpost_weight, dpost_bias,
                                                 dpre_weight, dpre_bias, workspace, _handle(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_block_norm_backward")


def token_logprob_workspace(logits):
    """Bytes of workspace of token_logprob for logits of this shape and type."""
    return _size(load_library().flashoptim_token_logprob_workspace(*logits.shape, _DTYPE[logits.dtype]), "flashoptim_token_logprob_workspace")


def token_logprob(logits, tokens, logprob=None, lse=None, temperature=1.0, logprob64=None, workspace=None, stream=None):
    """logprob [rows] <- the log-probability of each row's token (int64, negative: the row does not count), logprob64 the same in float64,
    lse <- the log of the row's sum of exponentials, for the backward pass; what is None is left out."""
    status = (_fast or _marshal()).logprob(logits, tokens, temperature, logprob, logprob64, lse, workspace, _handle_here(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_token_logprob")


def token_logprob_backward(logits, tokens, lse, dlogprob, dlogits, temperature=1.0, stream=None):
    """dlogits <- the gradient of the logits (which it may replace in their memory) from that of the log-probabilities."""
    status = (_fast or _marshal()).logprob_backward(logits, tokens, temperature, lse, dlogprob, dlogits, _handle_here(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_token_logprob_backward")


class PolicyLoss:
    """What a clipped policy loss is made of (flashoptim_policy_spec)."""

    def __init__(self, clip_low=0.2, clip_high=0.2, kl_weight=0.0, temperature=1.0, grad_scale=1.0):
        self.desc = _PolicySpec(temperature, clip_low, clip_high, kl_weight, grad_scale)
        self.address = C.addressof(self.desc)


def policy_loss_workspace(logits):
    return _size(load_library().flashoptim_policy_loss_workspace(*logits.shape, _DTYPE[logits.dtype]), "flashoptim_policy_loss_workspace")


def policy_loss(spec, logits, tokens, advantages, stats, old_logprob=None, ref_logprob=None, weights=None, logprob=None, dlogits=None,
                workspace=None, stream=None):
    """stats [4] <- the loss, its surrogate, KL and clipped parts; logprob [rows] and the gradient dlogits (which may replace the logits
    in their memory) where they are not None."""
    status = (_fast or _marshal()).policy(spec.address, logits, tokens, advantages, old_logprob, ref_logprob, weights, stats, logprob, dlogits,
                                          workspace, _handle_here(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_policy_loss")


class PreferenceLoss:
    """What a preference loss is made of (flashoptim_preference_spec).  order: "by_turns" or "halves"."""

    def __init__(self, beta=0.1, kind="sigmoid", label_smoothing=0.0, order="by_turns", grad_scale=1.0):
        self.desc = _PreferenceSpec({"sigmoid": 0, "hinge": 1, "squared": 2}.get(kind, -1), {"by_turns": 0, "halves": 1}.get(order, -1),
                                    beta, label_smoothing, grad_scale)
        self.address = C.addressof(self.desc)


def preference_loss(spec, logprob, offsets, loss, ref_logprob=None, weights=None, margins=None, dlogprob=None, stream=None):
    """loss [1] <- the mean over pairs of sequences, sequence i being the rows offsets[i] .. offsets[i + 1] - 1 of logprob (float32, or
    float64 as token_logprob leaves it in logprob64); margins [pairs] and the gradient dlogprob [rows] where they are not None.  Rows that do not
    count, those of negative tokens among them, have the weight 0."""
    status = (_fast or _marshal()).preference(spec.address, logprob, offsets, loss, ref_logprob, weights, margins, dlogprob, _handle_here(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_preference_loss")


class GradList:
    """A host array of flashoptim_gradient descriptors, built once and reused: `src` contiguous GPU tensors of one type, bfloat16 or
    float32, `dst` where clip_gradients leaves them (None: in place), of that type or bfloat16."""

    params = None

    def __init__(self, src, dst=None):
        self.src, self.dst = list(src), None if dst is None else list(dst)
        if self.dst is not None and len(self.dst) != len(self.src):
            raise ValueError("as many destinations as gradients")
        self.n = len(self.src)
        self.array = (_Gradient * max(self.n, 1))()
        self.device = self.src[0].get_device() if self.src else None
        self.src_dtype = self._type(self.src, "gradients")
        self.dst_dtype = self.src_dtype if self.dst is None else self._type(self.dst, "destinations")
        for i, t in enumerate(self.src):
            to = t if self.dst is None else self.dst[i]
            if to.numel() != t.numel():
                raise ValueError("a destination has the elements of its gradient")
            d = self.array[i]
            d.src, d.dst, d.numel = t.data_ptr(), to.data_ptr(), t.numel()
        self._pack()

    def _pack(self):
        self.args = C.addressof(self.array), self.n, self.src_dtype, self.dst_dtype

    def _type(self, tensors, what):
        if any(t.dtype not in _DTYPE or t.dtype != tensors[0].dtype or not t.is_contiguous() or not t.is_cuda or t.get_device() != self.device
               for t in tensors):
            raise ValueError(f"{what}: contiguous tensors on one GPU, bfloat16 or float32, one type for all")
        return _DTYPE[tensors[0].dtype] if tensors else 0

    @classmethod
    def of(cls, params):
        """The gradients of a TensorList, clipped in place: at each call those that its steps take then, also behind a set_grad (a captured
        call keeps those that it was captured with).  As for the steps, their memory is the caller's to keep."""
        out = cls([])
        out.device = params.grad_device()
        out.n = params.n
        out.array = (_Gradient * max(out.n, 1))()
        for d, t in zip(out.array, params.array[:params.n]):
            d.src, d.dst, d.numel = t.grad, t.grad, t.numel
        out.src = out.params = params
        out._pack()
        return out

    def follow(self):
        self.device = self.params.grad_device()
        (_fast or _marshal()).follow(self.args[0], C.addressof(self.params.array), self.n)


class ClipFactor:
    """The device record of a norm (flashoptim_clip_factor): `sum_squares` (float64), `norm` and `scale` (float32) are views of one
    element each."""

    def __init__(self, device="cuda"):
        self.data = torch.zeros(2, dtype=torch.float64, device=device)
        if not self.data.is_cuda:
            raise ValueError("a factor lies on the GPU")
        self.sum_squares = self.data[:1]
        self.norm, self.scale = self.data.view(torch.float32)[2:3], self.data.view(torch.float32)[3:4]
        self.address, self.device = self.data.data_ptr(), self.data.get_device()


def grad_norm_workspace(grads):
    """Bytes of workspace of grad_norm for this list."""
    return _size(load_library().flashoptim_grad_norm_workspace(grads.array, grads.n, grads.src_dtype), "flashoptim_grad_norm_workspace")


def _ready(grads, factor):
    if grads.params is not None:
        grads.follow()
    if grads.device not in (None, factor.device):
        raise ValueError("the gradients and the factor lie on different devices")


def grad_norm(grads, max_norm, factor, workspace=None, stream=None):
    """factor (ClipFactor) <- the norm of all gradients of a GradList, and max_norm / norm where that is less than 1."""
    _ready(grads, factor)
    status = (_fast or _marshal()).grad_norm(*grads.args, factor.device, max_norm, factor.address, workspace, _handle_here(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_grad_norm")


def clip_factor_from_sum(factor, max_norm, stream=None):
    """norm and scale of `factor` from its sum_squares as it is now."""
    _on_current(factor, stream)
    _check(load_library().flashoptim_clip_factor_from_sum(factor.address, max_norm, _stream_handle(stream)), "flashoptim_clip_factor_from_sum")


def clip_gradients(grads, factor, stream=None):
    """The destinations of a GradList <- its gradients times the factor's scale."""
    _ready(grads, factor)
    status = (_fast or _marshal()).clip(*grads.args, factor.device, factor.address, _handle_here(stream))
    if status:
        raise FlashOptimError(status, "flashoptim_clip_gradients")


def faithful_rounding_stats(stream=None):
    """(division operand pairs checked, quotients of the default AdamW step's division that are not the exactly
    rounded one)."""
    counts = (C.c_int64 * 2)()
    _check(load_library().flashoptim_faithful_rounding_stats(counts, _stream(stream)), "flashoptim_faithful_rounding_stats")
    return tuple(counts)


class ClockMonitor:
    """Samples the shader clock on a stream of its own while other work runs: start(), run the work, then
    ghz() waits for the monitor and returns one value per sample (numpy array)."""

    def __init__(self, n_samples=200, seconds_per_sample=1e-3, device="cuda"):
        self.n, self.dt = int(n_samples), float(seconds_per_sample)
        self.samples = torch.zeros(2 * self.n, dtype=torch.int64, device=device)
        self.stream = torch.cuda.Stream(device=device)
        self.tick_hz = C.c_double(0.0)

    def start(self):
        self.samples.zero_()
        torch.cuda.current_stream().synchronize()
        self.stream.wait_stream(torch.cuda.current_stream())
        _check(load_library().flashoptim_clock_monitor(C.cast(self.samples.data_ptr(), C.POINTER(C.c_uint64)), self.n,
                                                       self.dt, C.byref(self.tick_hz), _stream(self.stream)),
               "flashoptim_clock_monitor")

    def ghz(self):
        self.stream.synchronize()
        o = self.samples.cpu().numpy().reshape(self.n, 2).astype("float64")
        return o[:, 1] / o[:, 0] * self.tick_hz.value / 1e9


def short_sqrt_state():
    """0 not checked yet, 1 verified on this device, 2 not in use (check failed or switched off by the environment)."""
    return int(load_library().flashoptim_short_sqrt_state())


def selftest(stream=None):
    """Runs the device self-test; returns (status, checked[7], failed[7])."""
    checked = (C.c_int64 * 7)()
    failed = (C.c_int64 * 7)()
    status = load_library().flashoptim_selftest(checked, failed, _stream(stream))
    if status not in (0, -6):
        raise FlashOptimError(status, "flashoptim_selftest")
    return status, list(checked), list(failed)


def strerror(status):
    return load_library().flashoptim_strerror(int(status)).decode()


def step_launch_count(kind, numels):
    """Kernel launches that one step call of `kind` issues for a list with these element counts."""
    arr = (C.c_int64 * max(len(numels), 1))(*[int(n) for n in numels])
    n = int(load_library().flashoptim_step_launch_count(KIND[kind], arr, len(numels)))
    if n < 0:
        raise FlashOptimError(n, "flashoptim_step_launch_count")
    return n


def release_cache():
    _check(load_library().flashoptim_release_cache(), "flashoptim_release_cache")


def version():
    return int(load_library().flashoptim_version())
