"""Thin Python binding of libsolo (see include/solo.h): argument marshalling only.

Every function has the name and meaning of the C entry point it calls; all of the
optimizer step runs in the HIP kernels of the library.  Tensors are torch tensors
on an AMD GPU (torch is used for device memory and streams only); a tensor is
passed as its device pointer, the stream as the current torch stream's handle.
The calls of a step are marshalled by a small native module (csrc/solo_py.cpp) where
one has been built for this interpreter, the others through ctypes; arguments that only
ctypes knows how to pass (its own integer objects) take its way in a step, too.  The module
fails loudly when the library has not been built: there is no fallback path for it.
"""
import ctypes as C
import functools
import importlib.util
import os
import sysconfig
import threading

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libsolo.so")
NATIVE_PATH = os.path.join(_HERE, "lib", "_solo_native" + sysconfig.get_config_var("EXT_SUFFIX"))

SOLO_OK, SOLO_E_INVALID, SOLO_E_UNSUPPORTED, SOLO_E_HIP = 0, -1, -2, -3
SOLO_GRAD_FP32, SOLO_GRAD_BF16 = 0, 1
SOLO_FLAG_STOCHASTIC = 1
SOLO_FLAG_M_DYNAMIC_EXPONENT = 2
SOLO_FLAG_ADABELIEF = 4
SOLO_FLAG_COUPLED_DECAY = 8
SOLO_TABLE_BF16_COPY, SOLO_TABLE_SHORT_BLOCK = 1, 2
SOLO_FP32, SOLO_BF16 = 0, 1
SOLO_EMBEDDING_ACCUMULATE = 1
SOLO_TOP_MAX = 32


class solo_config(C.Structure):
    _fields_ = [("bits_m", C.c_uint32), ("bits_v", C.c_uint32), ("block_size", C.c_uint32),
                ("grad_dtype", C.c_uint32),
                ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("quantile_p", C.c_float),
                ("flags", C.c_uint32), ("reserved", C.c_uint32),
                ("seed", C.c_uint64), ("index_offset", C.c_uint64)]


def make_config(bits_m=4, bits_v=4, block_size=128, grad_dtype=SOLO_GRAD_FP32, lr=1e-3,
                beta1=None, beta2=0.999, eps=1e-8, weight_decay=0.01, quantile_p=0.1,
                flags=SOLO_FLAG_STOCHASTIC, seed=42, index_offset=0):
    if beta1 is None:
        beta1 = solo_beta1_default(bits_m, 0)
    return solo_config(bits_m, bits_v, block_size, grad_dtype, lr, beta1, beta2, eps,
                       weight_decay, quantile_p, flags, 0, seed, index_offset)


class solo_tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("param_bf16", C.c_void_p), ("grad", C.c_void_p),
                ("m_codes", C.c_void_p), ("m_scale", C.c_void_p), ("v_codes", C.c_void_p),
                ("v_scale", C.c_void_p), ("v_base", C.c_void_p), ("n", C.c_uint64)]


class solo_grad(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("clipped", C.c_void_p), ("n", C.c_uint64), ("dtype", C.c_uint32), ("reserved", C.c_uint32)]


class solo_embedding_shape(C.Structure):
    _fields_ = [("vocab", C.c_uint64), ("dim", C.c_uint64), ("tokens", C.c_uint64), ("table_stride", C.c_uint64),
                ("rows_stride", C.c_uint64), ("table_dtype", C.c_uint32), ("rows_dtype", C.c_uint32),
                ("token_bits", C.c_uint32), ("flags", C.c_uint32), ("scale", C.c_float), ("reserved", C.c_uint32)]


class solo_logits(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("cols", C.c_uint64), ("stride", C.c_uint64), ("grad_stride", C.c_uint64),
                ("dtype", C.c_uint32), ("target_bits", C.c_uint32), ("top", C.c_uint32), ("reserved", C.c_uint32),
                ("scale", C.c_float), ("reserved2", C.c_uint32)]


class SoloError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"libsolo error {code}: {solo_strerror(code)}")


_lib = None
_step = _multi = None            # the calls of a step: native, or through ctypes
_calls = None                    # those of the operators around the step, by name
_torch = None
_device_now = _stream_now = None    # torch's current device, and the handle of the current stream of a device
_loading = threading.RLock()


def lib():
    """Load libsolo.so (built by ``python -m paper_2505_00347_amd.build``)."""
    global _lib, _step, _multi, _calls, _torch, _device_now, _stream_now
    if _lib is not None:
        return _lib
    with _loading:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise ImportError(f"{LIB_PATH} is missing: build it with "
                                  "`python -m paper_2505_00347_amd.build` (needs hipcc)")
            # torch first: the wheel brings a HIP runtime of its own and exports it to the process.
            # Loaded after it, libsolo binds to that runtime, the one the tensors and streams of the
            # callers belong to; loaded before it, libsolo would bind to the system's copy, and every
            # launch on a torch stream would fail.
            import torch
            L = _declared(C.CDLL(LIB_PATH))
            step, multi = functools.partial(_step_by_ctypes, L), functools.partial(_multi_by_ctypes, L)
            calls = {name: functools.partial(_by_ctypes, getattr(L, name)) for name in _OPERATIONS}
            if os.path.exists(NATIVE_PATH):
                native = _native_calls(L, step, multi)
                step, multi = native.step, native.multi
                native.bind_operations({name: (C.cast(getattr(L, name), C.c_void_p).value, call) for name, call in calls.items()})
                calls = {name: getattr(native, name) for name in _OPERATIONS}
            _step, _multi, _calls, _torch = step, multi, calls, torch
            _device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
            _stream_now = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
            _lib = L                 # last: a thread that finds it set finds the others set
    return _lib


def _declared(L):
    vp, u32, u64, cfgp = C.c_void_p, C.c_uint32, C.c_uint64, C.POINTER(solo_config)
    L.solo_code_words.restype = C.c_size_t; L.solo_code_words.argtypes = [u64, u32]
    L.solo_num_blocks.restype = C.c_size_t; L.solo_num_blocks.argtypes = [u64, u32]
    L.solo_state_bytes.restype = C.c_size_t; L.solo_state_bytes.argtypes = [u64, cfgp]
    L.solo_beta1_default.restype = C.c_float; L.solo_beta1_default.argtypes = [u32, C.c_int]
    L.solo_beta1_bound.restype = C.c_float
    L.solo_beta1_bound.argtypes = [C.c_float, C.c_float, C.c_float]
    L.solo_strerror.restype = C.c_char_p; L.solo_strerror.argtypes = [C.c_int]
    L.solo_state_init.restype = C.c_int
    L.solo_state_init.argtypes = [vp, vp, vp, vp, vp, u64, cfgp, vp]
    L.solo_adamw_step.restype = C.c_int
    L.solo_adamw_step.argtypes = [vp, vp, vp, vp, vp, vp, vp, u64, u64, cfgp, vp]
    L.solo_adamw_step_mp.restype = C.c_int
    L.solo_adamw_step_mp.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, u64, u64, cfgp, vp]
    tp = C.POINTER(solo_tensor)
    L.solo_multi_units.restype = C.c_uint64; L.solo_multi_units.argtypes = [tp, u32, cfgp]
    L.solo_multi_table_bytes.restype = C.c_size_t; L.solo_multi_table_bytes.argtypes = [u32, u64]
    L.solo_multi_table_build.restype = C.c_int
    L.solo_multi_table_build.argtypes = [tp, u32, cfgp, vp, C.c_size_t, C.POINTER(C.c_uint32)]
    L.solo_adamw_step_multi.restype = C.c_int
    L.solo_adamw_step_multi.argtypes = [vp, u32, u64, u32, vp, u64, cfgp, vp]
    gp, size = C.POINTER(solo_grad), C.c_size_t
    L.solo_norm_units.restype = u64; L.solo_norm_units.argtypes = [gp, u32]
    L.solo_norm_table_bytes.restype = size; L.solo_norm_table_bytes.argtypes = [u32, u64]
    L.solo_norm_workspace_bytes.restype = size; L.solo_norm_workspace_bytes.argtypes = [u64]
    L.solo_norm_table_build.restype = C.c_int; L.solo_norm_table_build.argtypes = [gp, u32, vp, size]
    L.solo_embedding_workspace_bytes.restype = size
    L.solo_embedding_workspace_bytes.argtypes = [C.POINTER(solo_embedding_shape)]
    norm = [vp, u32, u64, vp, C.c_float, vp, vp, vp, vp, vp]
    for name, types in {"solo_grad_norm": norm, "solo_grad_clip": norm, "solo_embedding": [vp] * 5,
                        "solo_embedding_grad": [vp, vp, vp, vp, size, vp, vp], "solo_logprob": [vp] * 10,
                        "solo_logprob_grad": [vp] * 9, "solo_logprob_with_grad": [vp] * 9}.items():
        getattr(L, name).restype, getattr(L, name).argtypes = C.c_int, types
    return L


_OPERATIONS = ("solo_grad_norm", "solo_grad_clip", "solo_embedding", "solo_embedding_grad", "solo_logprob",
               "solo_logprob_grad", "solo_logprob_with_grad")


def _by_ctypes(function, *args):
    return function(*[a.data_ptr() if hasattr(a, "data_ptr") else a for a in args[:-1]], _stream(args[-1]))


def _operation(name, check, *args):
    """Calls an operator around the step; the last argument is the stream."""
    if _calls is None:
        lib()
    rc = _calls[name](*args)
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc


def _address(struct, kind):
    if not isinstance(struct, kind):
        raise C.ArgumentError(f"a {kind.__name__} expected, got {type(struct).__name__}")
    return C.addressof(struct)


def _native_calls(L, step, multi):
    """The native module (csrc/solo_py.cpp), which hands what it does not take to `step` and `multi`."""
    import torch
    spec = importlib.util.spec_from_file_location("_solo_native", NATIVE_PATH)
    native = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(native)
    address = lambda f: C.cast(f, C.c_void_p).value
    native.bind(address(L.solo_adamw_step_mp), address(L.solo_adamw_step_multi), solo_config, C.sizeof(solo_config),
                C.ArgumentError, C._SimpleCData, step, multi, _stream_of_now,
                getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None))
    os.register_at_fork(after_in_child=native.forked)
    return native


def _step_by_ctypes(L, param, param_bf16, grad, grad_scale, m_codes, m_scale, v_codes, v_scale, v_base, n, step, cfg, stream):
    return L.solo_adamw_step_mp(_ptr(param), _ptr(param_bf16), _ptr(grad), _ptr(grad_scale), _ptr(m_codes), _ptr(m_scale),
                                _ptr(v_codes), _ptr(v_scale), _ptr(v_base), n, step, C.byref(cfg),
                                _stream(stream) if n else None)


def _multi_by_ctypes(L, table_device, count, units, table_flags, grad_scale, step, cfg, stream):
    return L.solo_adamw_step_multi(_ptr(table_device), count, units, table_flags, _ptr(grad_scale), step, C.byref(cfg),
                                   _stream(stream) if units else None)


def _stream_of_now():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _ptr(t):
    """Device pointer of a torch tensor (or a raw integer address)."""
    if t is None:
        return None
    return t if isinstance(t, int) else t.data_ptr()


def _stream(stream):
    if stream is None:
        return _stream_of_now()
    return stream if isinstance(stream, int) else stream.cuda_stream


def solo_code_words(n, bits): return lib().solo_code_words(n, bits)
def solo_num_blocks(n, block_size): return lib().solo_num_blocks(n, block_size)
def solo_state_bytes(n, cfg): return lib().solo_state_bytes(n, C.byref(cfg))
def solo_beta1_default(bits_m, from_scratch=0): return lib().solo_beta1_default(bits_m, from_scratch)
def solo_beta1_bound(beta, r_median_b, r_median_bprime): return lib().solo_beta1_bound(beta, r_median_b, r_median_bprime)
def solo_strerror(code): return lib().solo_strerror(code).decode()


def solo_state_init(m_codes, m_scale, v_codes, v_scale, v_base, n, cfg, stream=None, check=True):
    rc = lib().solo_state_init(_ptr(m_codes), _ptr(m_scale), _ptr(v_codes), _ptr(v_scale),
                               _ptr(v_base), n, C.byref(cfg), _stream(stream) if n else None)
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc


def solo_adamw_step(param, grad, m_codes, m_scale, v_codes, v_scale, v_base, n, step, cfg,
                    stream=None, check=True):
    # (solo_adamw_step of the library is this call with both extras NULL)
    if _step is None:
        lib()
    rc = _step(param, None, grad, None, m_codes, m_scale, v_codes, v_scale, v_base, n, step, cfg, stream)
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc


def solo_adamw_step_mp(param, param_bf16, grad, grad_scale, m_codes, m_scale, v_codes, v_scale,
                       v_base, n, step, cfg, stream=None, check=True):
    """param_bf16 (bf16 tensor) and grad_scale (one-element float32 device tensor) may be None."""
    if _step is None:
        lib()
    rc = _step(param, param_bf16, grad, grad_scale, m_codes, m_scale, v_codes, v_scale, v_base, n, step, cfg, stream)
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc


def solo_multi_units(tensors, count, cfg): return lib().solo_multi_units(tensors, count, C.byref(cfg))
def solo_multi_table_bytes(count, units): return lib().solo_multi_table_bytes(count, units)


def solo_multi_table_build(tensors, count, cfg, table_host, table_bytes, check=True):
    """Returns (return code, table flags)."""
    flags = C.c_uint32(0)
    rc = lib().solo_multi_table_build(tensors, count, C.byref(cfg), table_host, table_bytes, C.byref(flags))
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc, flags.value


def solo_adamw_step_multi(table_device, count, units, table_flags, grad_scale, step, cfg, stream=None,
                          check=True):
    if _multi is None:
        lib()
    rc = _multi(table_device, count, units, table_flags, grad_scale, step, cfg, stream)
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc


class SoloMultiTable:
    """The device table of a multi-tensor step, built from per-tensor (param, grad, SoloState[,
    param_bf16]) tuples of torch tensors: marshals the descriptors, lets the library build the
    table in host memory and copies it to the device."""

    def __init__(self, items, cfg, device="cuda"):
        import torch
        self.cfg, self.count = cfg, len(items)
        arr = (solo_tensor * self.count)()
        self._keep = []                            # the memory the table points to (behind an address it is the caller's to keep)
        for k, it in enumerate(items):
            p, g, st = it[0], it[1], it[2]
            h = it[3] if len(it) > 3 else None
            buffers = p, h, g, st.m_codes, st.m_scale, st.v_codes, st.v_scale, st.v_base
            arr[k] = solo_tensor(*map(_ptr, buffers), st.n)
            self._keep += [t.detach() for t in buffers if hasattr(t, "detach")]
        self.units = solo_multi_units(arr, self.count, cfg)
        nbytes = solo_multi_table_bytes(self.count, self.units)
        host = torch.empty((nbytes + 15) // 16 * 16, dtype=torch.uint8)
        _, self.flags = solo_multi_table_build(arr, self.count, cfg, host.data_ptr(), nbytes)
        self.table = host.to(device)

    def step(self, step, grad_scale=None, stream=None):
        return solo_adamw_step_multi(self.table, self.count, self.units, self.flags, grad_scale, step,
                                     self.cfg, stream)


# ---- around the step: norm and clipping, embedding, log probabilities (include/solo.h) ----------

def solo_norm_units(grads, count): return lib().solo_norm_units(grads, count)
def solo_norm_table_bytes(count, units): return lib().solo_norm_table_bytes(count, units)
def solo_norm_workspace_bytes(units): return lib().solo_norm_workspace_bytes(units)


def solo_norm_table_build(grads, count, table_host, table_bytes, check=True):
    rc = lib().solo_norm_table_build(grads, count, table_host, table_bytes)
    if check and rc != SOLO_OK:
        raise SoloError(rc)
    return rc


def solo_grad_norm(table_device, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace, stream=None, check=True):
    return _operation("solo_grad_norm", check, table_device, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace, stream)


def solo_grad_clip(table_device, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace, stream=None, check=True):
    return _operation("solo_grad_clip", check, table_device, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace, stream)


def solo_embedding(table, tokens, rows, shape, stream=None, check=True):
    return _operation("solo_embedding", check, table, tokens, rows, _address(shape, solo_embedding_shape), stream)


def solo_embedding_workspace_bytes(shape): return lib().solo_embedding_workspace_bytes(C.byref(shape))


def solo_embedding_grad(grad_rows, tokens, grad_table, workspace, workspace_bytes, shape, stream=None, check=True):
    return _operation("solo_embedding_grad", check, grad_rows, tokens, grad_table, workspace, workspace_bytes,
                      _address(shape, solo_embedding_shape), stream)


def solo_logprob(logits, targets, logprob, entropy, rank, top_logprob, top_token, stats, shape, stream=None, check=True):
    return _operation("solo_logprob", check, logits, targets, logprob, entropy, rank, top_logprob, top_token, stats,
                      _address(shape, solo_logits), stream)


def solo_logprob_grad(logits, targets, entropy, stats, grad_logprob, grad_entropy, grad_logits, shape, stream=None, check=True):
    return _operation("solo_logprob_grad", check, logits, targets, entropy, stats, grad_logprob, grad_entropy, grad_logits,
                      _address(shape, solo_logits), stream)


def solo_logprob_with_grad(logits, targets, grad_logprob, grad_entropy, logprob, entropy, grad_logits, shape, stream=None, check=True):
    return _operation("solo_logprob_with_grad", check, logits, targets, grad_logprob, grad_entropy, logprob, entropy, grad_logits,
                      _address(shape, solo_logits), stream)


def _dtype(tensor):
    if tensor.dtype is _torch.float32:
        return SOLO_FP32
    if tensor.dtype is _torch.bfloat16:
        return SOLO_BF16
    raise TypeError(f"float32 or bfloat16 expected, got {tensor.dtype}")


def _token_bits(tensor, n):
    if tensor.dim() != 1 or tensor.numel() != n:
        raise ValueError(f"{n} tokens in one dimension expected, got {tuple(tensor.shape)}")
    if n > 1 and tensor.stride(0) != 1:
        raise ValueError("tokens must be contiguous")
    if tensor.dtype is _torch.int64:
        return 64
    if tensor.dtype is _torch.int32:
        return 32
    raise TypeError(f"int64 or int32 tokens expected, got {tensor.dtype}")


def _row_stride(tensor, rows, cols, name):
    """Elements from row to row of a matrix whose rows are contiguous."""
    if tuple(tensor.shape) != (rows, cols):
        raise ValueError(f"{name}: shape {(rows, cols)} expected, got {tuple(tensor.shape)}")
    if cols > 1 and tensor.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    stride = tensor.stride(0) if rows > 1 else cols
    if stride < cols:
        raise ValueError(f"{name}: rows must not overlap")
    return stride


def _row_weights(tensor, rows, name, device):
    if tensor is None:
        return
    if tensor.dtype is not _torch.float32 or tensor.dim() != 1 or tensor.numel() != rows or not tensor.is_contiguous():
        raise ValueError(f"{name}: {rows} contiguous float32 values expected")
    if tensor.device != device:
        raise ValueError(f"{name}: on {device} expected, got {tensor.device}")


def _layout(tensor):
    """What a handle's checks look at."""
    return None if tensor is None else (tensor.shape, tensor.stride(), tensor.dtype, tensor.device)


def _on(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} expected, got {t.device}")


class _Handle:
    """Device and streams of a handle.  A call takes tensors of the handle's device, which has to be torch's current one.

    Its buffers are made on torch's current stream, and a call may run on another one (`stream`, or what is
    current then).  The first call on such a stream waits for what was enqueued on the current stream when the buffers were made (a
    new buffer may be memory that earlier work still uses), and the allocator learns that this stream uses them.  The calls of
    a handle follow each other, each with the buffers that the one before has left: on several streams the caller orders them, and of
    calls on a stream that is not torch's (a bare number, another library's object) it keeps the handle until they are done."""

    _buffers, _home = (), None

    def __init__(self, device):
        lib()
        self.device = _torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = _torch.device("cuda", _torch.cuda.current_device())
        self._index = self.device.index if self.device.type == "cuda" else None

    def _hold(self, *buffers):
        self._others, self._home, self._ready = {}, None, None
        if self._index is not None:
            stream = _torch.cuda.current_stream(self.device)
            self._home = stream.cuda_stream
            if not _torch.cuda.is_current_stream_capturing():
                self._ready = stream.record_event()
        self._buffers = [b for b in buffers if b is not None]          # (last: a lookup of another thread finds all of it or none)

    def _on_stream(self, stream):
        """The number of the stream that a call runs on, ready for the buffers."""
        if self._index is None or _device_now() != self._index:
            raise ValueError(f"a call runs on the GPU that is torch's current device, this handle is on {self.device}")
        number = _stream_now(self._index) if stream is None else stream if isinstance(stream, int) else self._number_of(stream)
        if number != self._home and self._buffers and number not in self._others:
            self._visit(stream, number)
        return number

    def _number_of(self, stream):
        if getattr(stream, "device_index", self._index) != self._index:
            raise ValueError(f"a stream on {self.device} expected, got {stream}")
        number = stream.cuda_stream
        return getattr(number, "value", number) or 0       # (one of ctypes; None: the default stream)

    def _visit(self, stream, number):
        foreign = not (stream is None or isinstance(stream, _torch.cuda.Stream))
        if foreign:
            stream = _torch.cuda.ExternalStream(number)
        elif stream is None:
            stream = _torch.cuda.current_stream()
        with _torch.cuda.stream(stream):
            if _torch.cuda.is_current_stream_capturing():  # (a graph's nodes wait for nothing outside; capturing begins on an idle GPU)
                return
        if self._ready is not None:
            stream.wait_event(self._ready)
        if foreign:                                        # (there may be another stream of this number later, or none)
            return
        for b in self._buffers:
            b.record_stream(stream)
        self._others[number] = stream


class SoloGradNorm(_Handle):
    """Global norm of a set of gradient tensors, and clipping: the device table of the tensors (of any shape, contiguous,
    float32 or bfloat16) with its workspace and results.  `clipped`: tensors of the same shapes and types that clip()
    writes; they may be the gradients themselves (clipping in place).

    norm() and clip() return (norm [1], grad_scale [1], tensor_norm [count]): buffers of this object that the next
    call overwrites.  grad_scale is what SoloState.step and SoloMultiTable.step take.

    The table names the memory of the tensors as it is when the object is made, and the object keeps it.  Gradients that a training loop
    sets to None or replaces are other tensors: keep them (zero_grad(set_to_none=False)) or make another object."""

    def __init__(self, grads, clipped=None, device="cuda"):
        super().__init__(device)
        self.count = len(grads)
        if clipped is not None and len(clipped) != self.count:
            raise ValueError(f"{self.count} clipped tensors expected, got {len(clipped)}")
        arr = (solo_grad * self.count)()
        for k, g in enumerate(grads):
            c = clipped[k] if clipped is not None else None
            if not g.is_contiguous() or (c is not None and (not c.is_contiguous() or c.dtype is not g.dtype or c.shape != g.shape)):
                raise ValueError(f"tensor {k}: contiguous gradients, and clipped ones of the same shapes and types, expected")
            _on(self.device, g, c)
            arr[k] = solo_grad(_ptr(g), _ptr(c), g.numel(), _dtype(g), 0)
        self.units = solo_norm_units(arr, self.count)
        nbytes = solo_norm_table_bytes(self.count, self.units)
        host = _torch.empty((nbytes + 15) // 16 * 16, dtype=_torch.uint8)
        if self.count:
            solo_norm_table_build(arr, self.count, host.data_ptr(), nbytes)
        device = self.device
        self.table = host.to(device)
        self.workspace = _torch.empty(solo_norm_workspace_bytes(self.units), dtype=_torch.uint8, device=device)
        self.results = _torch.zeros(1, device=device), _torch.ones(1, device=device), _torch.zeros(self.count, device=device)
        self.writes = clipped is not None
        self._hold(self.table, self.workspace, *self.results)
        # the buffers the table points to: the caller's lists may change, and so may the storage that a tensor of theirs names
        self._keep = [t.detach() for t in (*grads, *(clipped or ())) if t is not None]

    def _run(self, name, max_norm, unscale, stream):
        if unscale is not None:
            if unscale.dtype is not _torch.float32 or unscale.numel() != 1:
                raise TypeError(f"unscale: one float32 value expected, got {unscale.numel()} of {unscale.dtype}")
            if unscale.device != self.device:
                raise ValueError(f"unscale: on {self.device} expected, got {unscale.device}")
        _operation(name, True, self.table, self.count, self.units, unscale, max_norm, *self.results, self.workspace, self._on_stream(stream))
        return self.results

    def norm(self, max_norm=float("inf"), unscale=None, stream=None):
        return self._run("solo_grad_norm", max_norm, unscale, stream)

    def clip(self, max_norm, unscale=None, stream=None):
        if not self.writes:
            raise ValueError("no tensors to write the clipped gradients to")
        return self._run("solo_grad_clip", max_norm, unscale, stream)


class SoloEmbedding(_Handle):
    """Lookup in an embedding table [vocab, dim] and the table's gradient, for up to `tokens` tokens a call: the workspace
    that the gradient needs.  Tables and rows may be float32 or bfloat16, each on its own; their rows contiguous, at any
    distance; tokens int64 or int32, those outside the table are padding.  Lookups may run beside each other; gradients share the
    workspace and follow each other."""

    def __init__(self, vocab, dim, tokens, scale=1.0, device="cuda"):
        super().__init__(device)
        self.vocab, self.dim, self.tokens, self.scale = vocab, dim, tokens, scale
        self._last = None, None
        # (of the rows' type that needs more: a call says which it has)
        self.workspace_bytes = max(solo_embedding_workspace_bytes(solo_embedding_shape(vocab, dim, tokens, dim, dim, SOLO_FP32, rows, 64, 0, scale, 0))
                                   for rows in (SOLO_FP32, SOLO_BF16))
        if not self.workspace_bytes:
            raise SoloError(SOLO_E_INVALID)
        self.workspace = None                      # of the first gradient

    def _shape(self, table, rows, ids, flags):
        """The C struct of these tensors.  The checks and the struct are made when the tensors' layout is another than in the
        call before: 3.6 us of the 5.9 that a lookup of a few tokens took.  (Layout and struct are read and stored as one: another thread's
        call may come in between, and a struct of other tensors would send the kernel out of these.)"""
        layout = _layout(table), _layout(rows), _layout(ids), flags, self.scale
        seen, made = self._last
        if layout != seen:
            n = ids.numel()
            if n > self.tokens:
                raise ValueError(f"at most {self.tokens} tokens expected, got {n}")
            made = solo_embedding_shape(self.vocab, self.dim, n, _row_stride(table, self.vocab, self.dim, "table"),
                                        _row_stride(rows, n, self.dim, "rows"), _dtype(table), _dtype(rows), _token_bits(ids, n),
                                        flags, self.scale, 0)
            _on(self.device, table, rows, ids)
            self._last = layout, made
        return made

    def lookup(self, table, ids, out, stream=None):
        """out[i] = scale * table[ids[i]]"""
        shape = self._shape(table, out, ids, 0)
        _operation("solo_embedding", True, table, ids, out, C.addressof(shape), self._on_stream(stream))
        return out

    def grad(self, grad_rows, ids, out, accumulate=False, stream=None):
        """out[v] = scale * the sum of the rows whose token is v; added to `out` if `accumulate`."""
        shape = self._shape(out, grad_rows, ids, SOLO_EMBEDDING_ACCUMULATE if accumulate else 0)
        if self.workspace is None:
            self.workspace = _torch.empty(self.workspace_bytes, dtype=_torch.uint8, device=self.device)
            self._hold(self.workspace)
        _operation("solo_embedding_grad", True, grad_rows, ids, out, self.workspace, self.workspace_bytes, C.addressof(shape), self._on_stream(stream))
        return out


class SoloLogprob(_Handle):
    """Log probabilities, entropies, ranks and `top` alternatives of up to `rows` rows of `cols` logits (float32 or
    bfloat16, rows contiguous, at any distance), and the gradient: the buffers of the results, which the next call overwrites.
    Targets are int64 or int32; one outside the columns is a padding position."""

    def __init__(self, rows, cols, top=0, rank=False, scale=1.0, device="cuda"):
        super().__init__(device)
        if not 0 <= top <= SOLO_TOP_MAX:
            raise ValueError(f"0 to {SOLO_TOP_MAX} alternatives expected, got {top}")
        self.rows, self.cols, self.top, self.scale = rows, cols, top, scale
        self._last = None, None
        f32, i32 = dict(dtype=_torch.float32, device=self.device), dict(dtype=_torch.int32, device=self.device)
        self.logprob, self.entropy = _torch.empty(rows, **f32), _torch.empty(rows, **f32)
        self.stats = _torch.empty((rows, 2), **f32)
        self._entropy_with_grad = _torch.empty(rows, **f32)            # (entropy and stats are a pair: forward_grad() leaves both as they are)
        self._summed = 0, None                     # rows and scale of what they are of
        self.rank = _torch.empty(rows, **i32) if rank else None
        self.top_logprob = _torch.empty((rows, top), **f32) if top else None
        self.top_token = _torch.empty((rows, top), **i32) if top else None
        self._hold(self.logprob, self.entropy, self.stats, self._entropy_with_grad, self.rank, self.top_logprob, self.top_token)

    def _shape(self, logits, targets, out=None):
        """The C struct of these tensors, made when their layout is another than in the call before (as in SoloEmbedding)."""
        layout = _layout(logits), _layout(targets), _layout(out), self.scale
        seen, made = self._last
        if layout != seen:
            r = logits.shape[0]
            if r > self.rows:
                raise ValueError(f"at most {self.rows} rows expected, got {r}")
            stride = _row_stride(logits, r, self.cols, "logits")
            grad_stride = stride
            if out is not None:
                grad_stride = _row_stride(out, r, self.cols, "gradient")
                if out.dtype is not logits.dtype:
                    raise TypeError(f"gradient: {logits.dtype} expected, got {out.dtype}")
            made = solo_logits(r, self.cols, stride, grad_stride, _dtype(logits), 64 if targets is None else _token_bits(targets, r),
                               self.top, 0, self.scale, 0)
            _on(self.device, logits, targets, out)
            self._last = layout, made
        return made

    def forward(self, logits, targets, stream=None):
        """(logprob, entropy[, rank][, top_logprob, top_token]); without targets, logprob and rank are None."""
        shape = self._shape(logits, targets)
        none = targets is None
        logprob, rank = (None, None) if none else (self.logprob, self.rank)
        _operation("solo_logprob", True, logits, targets, logprob, self.entropy, rank, self.top_logprob, self.top_token, self.stats,
                   C.addressof(shape), self._on_stream(stream))
        self._summed = shape.rows, shape.scale
        results = [logprob, self.entropy]
        if self.rank is not None:
            results.append(rank)
        if self.top:
            results += [self.top_logprob, self.top_token]
        return tuple(results) if shape.rows == self.rows else tuple(t if t is None else t[:shape.rows] for t in results)

    def grad(self, logits, targets, grad_logprob, grad_entropy, out, stream=None):
        """Gradient of the logits behind forward() on the same ones, for the gradients of logprob and entropy (or None).  forward_grad() in
        between, on whatever logits, changes nothing."""
        shape = self._shape(logits, targets, out)
        _row_weights(grad_logprob, shape.rows, "grad_logprob", self.device)
        _row_weights(grad_entropy, shape.rows, "grad_entropy", self.device)
        rows, scale = self._summed
        if rows < shape.rows or scale != shape.scale:
            raise ValueError(f"grad() takes what forward() left on the same rows: {shape.rows} with scale {shape.scale} expected, got {rows} with {scale}")
        _operation("solo_logprob_grad", True, logits, targets, self.entropy, self.stats, grad_logprob, grad_entropy, out,
                   C.addressof(shape), self._on_stream(stream))
        return out

    def forward_grad(self, logits, targets, grad_logprob, grad_entropy, out, stream=None):
        """(logprob, entropy, gradient) in one pass, for row weights that are known beforehand."""
        shape = self._shape(logits, targets, out)
        _row_weights(grad_logprob, shape.rows, "grad_logprob", self.device)
        _row_weights(grad_entropy, shape.rows, "grad_entropy", self.device)
        logprob = None if targets is None else self.logprob
        _operation("solo_logprob_with_grad", True, logits, targets, grad_logprob, grad_entropy, logprob, self._entropy_with_grad, out,
                   C.addressof(shape), self._on_stream(stream))
        if shape.rows != self.rows:
            return None if logprob is None else logprob[:shape.rows], self._entropy_with_grad[:shape.rows], out
        return logprob, self._entropy_with_grad, out


HBM_REGION_BYTES = 96 << 30      # an MI355X behaves as three such regions of physical memory


class state_region:
    """Context manager for the placement rule of include/solo.h (performance note): tensors that
    are allocated inside it come to lie behind the first 96 GiB that this process has allocated on
    the device, i.e. (in a process that started on an idle GPU, which receives physical memory in
    allocation order) in another third of HBM than the parameters allocated before it.

        p, g = ...                                   # resident_bytes of them, allocated first
        with solo.state_region(resident_bytes):
            state = solo.SoloState(n, cfg)

    It allocates a spacer up to the region boundary on entry and returns it to the driver on exit.
    Nothing happens if the resident bytes already fill a region, or if the device has no room."""

    def __init__(self, resident_bytes, keep_free=8 << 30):
        self.resident, self.keep_free, self.spacer = int(resident_bytes), keep_free, None

    def __enter__(self):
        import torch
        gap = HBM_REGION_BYTES - self.resident
        if 0 < gap < torch.cuda.mem_get_info()[0] - self.keep_free:
            self.spacer = torch.empty(gap, dtype=torch.uint8, device="cuda")
        return self

    def __exit__(self, *exc):
        import torch
        if self.spacer is not None:
            self.spacer = None
            torch.cuda.empty_cache()     # the spacer goes back to the driver, not into torch's cache
        return False


class SoloState:
    """Device buffers of the packed optimizer state of n elements (caller-owned memory:
    plain torch tensors; int32 tensors carry the uint32 code words)."""

    def __init__(self, n, cfg, device="cuda", init=True):
        import torch
        self.n, self.cfg = n, cfg
        nb = solo_num_blocks(n, cfg.block_size)
        self.m_codes = torch.empty(solo_code_words(n, cfg.bits_m), dtype=torch.int32, device=device)
        self.v_codes = torch.empty(solo_code_words(n, cfg.bits_v), dtype=torch.int32, device=device)
        self.m_scale = torch.empty(nb, dtype=torch.float32, device=device)
        self.v_scale = torch.empty(nb, dtype=torch.float32, device=device)
        self.v_base = torch.empty(nb, dtype=torch.float32, device=device)
        if init:
            solo_state_init(self.m_codes, self.m_scale, self.v_codes, self.v_scale, self.v_base,
                            n, cfg)

    def buffers(self):
        return (self.m_codes, self.m_scale, self.v_codes, self.v_scale, self.v_base)

    def step(self, param, grad, step, stream=None, param_bf16=None, grad_scale=None):
        # (solo_adamw_step_mp without its frame: 0.2 of the 3.9 us that a call of 4096 elements takes)
        if _step is None:
            lib()
        rc = _step(param, param_bf16, grad, grad_scale, *self.buffers(), self.n, step, self.cfg, stream)
        if rc != SOLO_OK:
            raise SoloError(rc)
        return rc
