"""ctypes binding of libkvlinc.so.  Same names and argument order as include/kvlinc.h, include/kvlinc_context.h and include/kvlinc_bounded.h."""
import contextlib
import ctypes
import math
import os

HERE = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(HERE, "libkvlinc.so")

KVLINC_OK, KVLINC_EINVAL, KVLINC_EWORKSPACE, KVLINC_EHIP, KVLINC_ESCRATCH = 0, -1, -2, -3, -4
KVLINC_STATIC_SCRATCH_BYTES = 16 << 20
KVLINC_FLAG_ALG1_LITERAL = 1
KVLINC_FLAG_SLIDING_VALUES = 2
KVLINC_F16, KVLINC_BF16, KVLINC_F32 = 0, 1, 2
KVLINC_ST_CAPACITY, KVLINC_ST_NONFINITE, KVLINC_ST_STATIC, KVLINC_ST_STATE_RANGE = 1, 2, 4, 8
KVLINC_ST_BOUND = 16


class KVLincError(RuntimeError):
    pass


class CacheStruct(ctypes.Structure):
    """Mirror of struct kvlinc_cache."""
    _fields_ = [
        ("B", ctypes.c_int32), ("H_q", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32),
        ("G", ctypes.c_int32), ("R", ctypes.c_int32), ("D", ctypes.c_int32), ("bits", ctypes.c_int32),
        ("max_groups", ctypes.c_int64),
        ("groups", ctypes.c_void_p),
        ("k_res", ctypes.c_void_p), ("v_res", ctypes.c_void_p),
        ("n_quant", ctypes.c_void_p), ("n_res", ctypes.c_void_p),
        ("S", ctypes.c_void_p), ("S16", ctypes.c_void_p), ("P", ctypes.c_void_p),
        ("Wq", ctypes.c_void_p), ("Wk", ctypes.c_void_p),
        ("status", ctypes.c_void_p), ("split_done", ctypes.c_void_p),
        ("flags", ctypes.c_int32),
    ]


class RotationStruct(ctypes.Structure):
    """Mirror of struct kvlinc_rotation."""
    _fields_ = [("channels", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("magnitude", ctypes.c_float), ("freq", ctypes.c_void_p)]


class RowsStruct(ctypes.Structure):
    """Mirror of struct kvlinc_rows."""
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("sequence_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


def _load():
    if not os.path.exists(lib_path):
        raise ImportError(
            "libkvlinc.so is not built (%s missing): run `python -c 'import __graft_entry__ as g; g.build()'` or "
            "`python paper_2510_05373_amd/build.py`; there is no fallback path" % lib_path)
    # PyTorch carries its own copy of the HIP runtime under the same soname as the system one, and the first copy
    # loaded serves the whole process.  The tensors and streams passed to this library come from torch, so torch's
    # runtime has to be that copy: import torch before the library is opened.
    import torch  # noqa: F401
    L = ctypes.CDLL(lib_path)
    P = ctypes.POINTER(CacheStruct)
    L.kvlinc_version.restype = ctypes.c_int
    L.kvlinc_version.argtypes = []
    L.kvlinc_strerror.restype = ctypes.c_char_p
    L.kvlinc_strerror.argtypes = [ctypes.c_int]
    L.kvlinc_cache_validate.restype = ctypes.c_int
    L.kvlinc_cache_validate.argtypes = [P]
    L.kvlinc_append_quantize.restype = ctypes.c_int
    L.kvlinc_append_quantize.argtypes = [P, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                         ctypes.c_int32, ctypes.c_void_p]
    L.kvlinc_decode_workspace_bytes.restype = ctypes.c_size_t
    L.kvlinc_decode_workspace_bytes.argtypes = [P, ctypes.c_int32]
    L.kvlinc_decode_attention.restype = ctypes.c_int
    L.kvlinc_decode_attention.argtypes = [P, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                          ctypes.c_int32, ctypes.c_void_p]
    L.kvlinc_decode_attention_timed.restype = ctypes.c_int
    L.kvlinc_decode_attention_timed.argtypes = [P, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    L.kvlinc_decode_attention_noalloc.restype = ctypes.c_int
    L.kvlinc_decode_attention_noalloc.argtypes = [P, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p]
    i32, ptr = ctypes.c_int32, ctypes.c_void_p
    L.kvlinc_prompt_workspace_bytes.restype = ctypes.c_size_t
    L.kvlinc_prompt_workspace_bytes.argtypes = [P, i32, i32, i32, i32]
    L.kvlinc_prompt_attention.restype = ctypes.c_int
    L.kvlinc_prompt_attention.argtypes = [P, ptr, ptr, ptr, ptr, i32, i32, i32, ptr, ptr, ctypes.c_size_t, i32, ptr]
    L.kvlinc_decode_windowed_workspace_bytes.restype = ctypes.c_size_t
    L.kvlinc_decode_windowed_workspace_bytes.argtypes = [P, i32, i32, i32]
    L.kvlinc_decode_attention_windowed.restype = ctypes.c_int
    L.kvlinc_decode_attention_windowed.argtypes = [P, ptr, i32, i32, ptr, ptr, ctypes.c_size_t, i32, ptr]
    L.kvlinc_cache_read.restype = ctypes.c_int
    L.kvlinc_cache_read.argtypes = [P, ptr, i32, ptr, ptr, i32, i32, ptr]
    f32, size, rows = ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(RowsStruct)
    L.kvlinc_rotary.restype = ctypes.c_int
    L.kvlinc_rotary.argtypes = [P, ctypes.POINTER(RotationStruct), rows, rows, rows, i32, ptr, ptr, ptr, i32, i32, i32, ptr]
    L.kvlinc_decode_mass_workspace_bytes.restype = size
    L.kvlinc_decode_mass_workspace_bytes.argtypes = [P, i32]
    L.kvlinc_decode_attention_mass.restype = ctypes.c_int
    L.kvlinc_decode_attention_mass.argtypes = [P, ptr, ptr, ptr, f32, ptr, ptr, size, i32, ptr]
    L.kvlinc_attention_mass_workspace_bytes.restype = size
    L.kvlinc_attention_mass_workspace_bytes.argtypes = [P, i32, i32]
    L.kvlinc_attention_mass.restype = ctypes.c_int
    L.kvlinc_attention_mass.argtypes = [P, ptr, ptr, i32, ptr, f32, ptr, ptr, size, i32, ptr]
    L.kvlinc_cache_evict_workspace_bytes.restype = size
    L.kvlinc_cache_evict_workspace_bytes.argtypes = [P]
    L.kvlinc_cache_evict.restype = ctypes.c_int
    L.kvlinc_cache_evict.argtypes = [P, P, ptr, ptr, i32, i32, i32, i32, ptr, ptr, ptr, ptr, size, ptr]
    return L


lib = _load()


# A generation step of a small batch takes about as long on the GPU as these calls take on the host: addresses go through the
# declared argument types as plain integers, and the current stream is asked for as a raw handle (through torch's own shortcut,
# which is not part of its public interface: without it the public call serves).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _current_device():
    import torch
    try:
        return torch._C._cuda_getDevice()
    except AttributeError:
        return torch.cuda.current_device()


def _stream(stream):
    if stream is None:
        import torch
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            return torch.cuda.current_stream().cuda_stream
    if hasattr(stream, "cuda_stream"):
        return stream.cuda_stream
    return int(stream)


def _struct(cache):
    return cache.struct if isinstance(cache, KVLincCache) else cache


def kvlinc_version():
    return lib.kvlinc_version()


def kvlinc_strerror(code):
    return lib.kvlinc_strerror(code).decode()


def kvlinc_cache_validate(cache):
    return lib.kvlinc_cache_validate(ctypes.byref(_struct(cache)))


def kvlinc_append_quantize(cache, k_new, v_new, n_new=None, T=None, keep_residual=0, stream=None):
    """k_new, v_new: [B, H_kv, T, 128] fp16 device tensors (contiguous); n_new: [B] int32 device tensor or None."""
    if T is None:
        T = k_new.shape[2]
    return lib.kvlinc_append_quantize(ctypes.byref(_struct(cache)), _ptr(k_new), _ptr(v_new), _ptr(n_new), int(T),
                                      int(keep_residual), _stream(stream))


def kvlinc_decode_workspace_bytes(cache, max_context=0):
    return lib.kvlinc_decode_workspace_bytes(ctypes.byref(_struct(cache)), int(max_context))


def kvlinc_decode_attention(cache, q, out, workspace, workspace_bytes=None, max_context=0, stream=None):
    """q, out: [B, H_q, 128] fp16 device tensors; workspace: device tensor of at least the advertised bytes."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    return lib.kvlinc_decode_attention(ctypes.byref(_struct(cache)), _ptr(q), _ptr(out), _ptr(workspace),
                                       int(workspace_bytes), int(max_context), _stream(stream))


def kvlinc_decode_attention_timed(cache, q, out, workspace, start_event, stop_event, workspace_bytes=None,
                                  max_context=0, stream=None):
    """As kvlinc_decode_attention; start_event / stop_event are raw hipEvent_t handles (integers)."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    return lib.kvlinc_decode_attention_timed(ctypes.byref(_struct(cache)), _ptr(q), _ptr(out), _ptr(workspace),
                                             int(workspace_bytes), int(max_context), _stream(stream),
                                             ctypes.c_void_p(int(start_event)), ctypes.c_void_p(int(stop_event)))


def kvlinc_decode_attention_noalloc(cache, q, out, max_context=0, stream=None):
    """As kvlinc_decode_attention, with the library's static scratch buffer in place of a workspace."""
    return lib.kvlinc_decode_attention_noalloc(ctypes.byref(_struct(cache)), _ptr(q), _ptr(out), int(max_context),
                                               _stream(stream))


def _bytes_of(workspace, workspace_bytes):
    if workspace_bytes is not None:
        return int(workspace_bytes)
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def kvlinc_prompt_workspace_bytes(cache, T, window=0, sinks=0, max_context=0):
    return lib.kvlinc_prompt_workspace_bytes(ctypes.byref(_struct(cache)), int(T), int(window), int(sinks), int(max_context))


def kvlinc_prompt_attention(cache, q, k_new, v_new, n_new, T, window, sinks, out, workspace, workspace_bytes=None, max_context=0,
                            stream=None):
    """q, out: [B, H_q, T, 128]; k_new, v_new: [B, H_kv, T, 128]; fp16 device tensors (contiguous); n_new: [B] int32 or None."""
    return lib.kvlinc_prompt_attention(ctypes.byref(_struct(cache)), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(n_new), int(T), int(window),
                                       int(sinks), _ptr(out), _ptr(workspace), _bytes_of(workspace, workspace_bytes), int(max_context),
                                       _stream(stream))


def kvlinc_decode_windowed_workspace_bytes(cache, window, sinks=0, max_context=0):
    return lib.kvlinc_decode_windowed_workspace_bytes(ctypes.byref(_struct(cache)), int(window), int(sinks), int(max_context))


def kvlinc_decode_attention_windowed(cache, q, window, sinks, out, workspace, workspace_bytes=None, max_context=0, stream=None):
    """q, out: [B, H_q, 128] fp16 device tensors (contiguous)."""
    return lib.kvlinc_decode_attention_windowed(ctypes.byref(_struct(cache)), _ptr(q), int(window), int(sinks), _ptr(out), _ptr(workspace),
                                                _bytes_of(workspace, workspace_bytes), int(max_context), _stream(stream))


def kvlinc_cache_read(cache, first, T, k_out, v_out, dtype=KVLINC_F16, rotated=0, stream=None):
    """k_out, v_out: [B, H_kv, T, 128] device tensors of the type dtype (KVLINC_F16, ...), either may be None; first: [B] int32 or None."""
    return lib.kvlinc_cache_read(ctypes.byref(_struct(cache)), _ptr(first), int(T), _ptr(k_out), _ptr(v_out), int(dtype), int(rotated),
                                 _stream(stream))


def kvlinc_rotary(cache, rotation, q, k, v, T, n_new=None, first=None, depth=None, counted=1, dtype_in=KVLINC_F16, dtype_out=KVLINC_F16, stream=None):
    """rotation: RotationStruct; q, k, v: RowsStruct or None; n_new, first: [B], depth: [B, T] int32 device tensors or None."""
    return lib.kvlinc_rotary(_struct(cache), rotation, q, k, v, int(T), _ptr(n_new), _ptr(first), _ptr(depth), int(counted), int(dtype_in), int(dtype_out),
                             _stream(stream))


def kvlinc_decode_mass_workspace_bytes(cache, max_context=0):
    return lib.kvlinc_decode_mass_workspace_bytes(ctypes.byref(_struct(cache)), int(max_context))


def kvlinc_decode_attention_mass(cache, q, out, mass, decay, mass_out, workspace, workspace_bytes=None, max_context=0, stream=None):
    """q, out: [B, H_q, 128] fp16; mass, mass_out: [B, H_kv, max_groups + 1] fp32; device tensors (contiguous), mass may be None."""
    return lib.kvlinc_decode_attention_mass(ctypes.byref(_struct(cache)), _ptr(q), _ptr(out), _ptr(mass), float(decay), _ptr(mass_out), _ptr(workspace),
                                            _bytes_of(workspace, workspace_bytes), int(max_context), _stream(stream))


def kvlinc_attention_mass_workspace_bytes(cache, T, max_context=0):
    return lib.kvlinc_attention_mass_workspace_bytes(ctypes.byref(_struct(cache)), int(T), int(max_context))


def kvlinc_attention_mass(cache, q, n_rows, T, mass, decay, mass_out, workspace, workspace_bytes=None, max_context=0, stream=None):
    """q: [B, H_q, T, 128] fp16; n_rows: [B] int32 or None; mass, mass_out: [B, H_kv, max_groups + 1] fp32; device tensors (contiguous), mass may be None."""
    return lib.kvlinc_attention_mass(ctypes.byref(_struct(cache)), _ptr(q), _ptr(n_rows), int(T), _ptr(mass), float(decay), _ptr(mass_out), _ptr(workspace),
                                     _bytes_of(workspace, workspace_bytes), int(max_context), _stream(stream))


def kvlinc_cache_evict_workspace_bytes(cache):
    return lib.kvlinc_cache_evict_workspace_bytes(ctypes.byref(_struct(cache)))


def kvlinc_cache_evict(cache, to, mass, mass_out, keep, limit, first, last, offset, offset_out, kept, workspace, workspace_bytes=None, stream=None):
    """mass: [B, H_kv, max_groups + 1] fp32, mass_out the same of `to`; offset, offset_out: [B] int32 or None; kept: [B, H_kv, max_groups of `to`] int32 or None."""
    return lib.kvlinc_cache_evict(ctypes.byref(_struct(cache)), ctypes.byref(_struct(to)), _ptr(mass), _ptr(mass_out), int(keep), int(limit), int(first),
                                  int(last), _ptr(offset), _ptr(offset_out), _ptr(kept), _ptr(workspace), _bytes_of(workspace, workspace_bytes),
                                  _stream(stream))


def rotary_frequencies(channels=128, base=10000.0, scaling=None, factor=1.0, original=0, low=1.0, high=32.0):
    """Angles per position of the channels / 2 pairs, base^(-2 i / channels), for KVLincRotary; for contexts `factor` times as long as those of `original`
    tokens that a model has learnt, scaled
      "linear"  all divided by the factor: positions in between;
      "base"    the base times factor^(channels / (channels - 2)): the last pair divided by it, the first left as it is;
      "parts"   pairs that turn more than `high` times in `original` tokens left as they are, those below `low` divided by the factor, a ramp between
                (used with a magnitude of 0.1 ln(factor) + 1, or of 1)."""
    if channels < 2 or channels > 128 or channels % 2:
        raise KVLincError("channels has to be even, 2 .. 128, not %s" % channels)
    if not base > 0.0 or not factor > 0.0:
        raise KVLincError("base and factor have to be above 0, not %s and %s" % (base, factor))
    if scaling not in (None, "linear", "base", "parts"):
        raise KVLincError("scaling has to be None, 'linear', 'base' or 'parts', not %r" % (scaling,))
    if scaling == "base" and channels > 2:
        base = base * factor ** (channels / (channels - 2.0))
    freq = [base ** (-2.0 * i / channels) for i in range(channels // 2)]
    if scaling == "linear":
        freq = [f / factor for f in freq]
    elif scaling == "parts":
        if not original > 0 or not high > low:
            raise KVLincError("scaling by parts needs original > 0 and high > low, not %s, %s and %s" % (original, high, low))
        kept = [min(1.0, max(0.0, (original * f / (2.0 * math.pi) - low) / (high - low))) for f in freq]
        freq = [k * f + (1.0 - k) * f / factor for k, f in zip(kept, freq)]
    return freq


class KVLincRotary:
    """Rotary positions as KVLincCache.rotary takes them: the angle per position of every pair, on the device.

    freq: channels / 2 numbers (rotary_frequencies, or a model's own); interleaved: pairs are channels 2 i and 2 i + 1, else i and i + channels / 2;
    magnitude: what the rotated channels are multiplied with."""

    def __init__(self, freq, interleaved=False, magnitude=1.0, device="cuda"):
        import torch
        self.freq = torch.as_tensor(freq, dtype=torch.float64).to(device).contiguous()
        self.channels = 2 * self.freq.numel()
        if self.freq.dim() != 1 or not 2 <= self.channels <= 128:
            raise KVLincError("freq has to be 1 to 64 numbers, not a tensor of shape %s" % (tuple(self.freq.shape),))
        if not math.isfinite(magnitude):
            raise KVLincError("magnitude has to be finite, not %s" % magnitude)
        self.interleaved, self.magnitude = bool(interleaved), float(magnitude)
        self.struct = RotationStruct(channels=self.channels, interleaved=int(self.interleaved), magnitude=self.magnitude, freq=self.freq.data_ptr())

    def inverse(self):
        """The rotation back."""
        if self.magnitude == 0.0:
            raise KVLincError("a magnitude of 0 has no inverse")
        return KVLincRotary(-self.freq, self.interleaved, 1.0 / self.magnitude, self.freq.device)


_NOTHING = contextlib.nullcontext()
_ROW_TYPES = {}


def _row_types():
    """KVLINC_F16, _BF16 or _F32 of torch's types."""
    if not _ROW_TYPES:
        import torch
        _ROW_TYPES.update({torch.float16: KVLINC_F16, torch.bfloat16: KVLINC_BF16, torch.float32: KVLINC_F32})
    return _ROW_TYPES


class KVLincCache:
    """Device buffers of one layer's cache plus the descriptor that points at them (allocation only)."""

    def __init__(self, B, H_q, H_kv, max_context, R=128, Wq=None, Wk=None, device="cuda", state_storage="fp32",
                 flags=0, bits=2):
        """state_storage: "fp32" keeps the fp32 master copy of S next to its binary16 tiles, "fp16" stores the state in
        the binary16 tiles only; flags: KVLINC_FLAG_* bits; bits: width of the codes, 2 or 4 (group records of 2304 or
        4352 words)."""
        import torch
        assert bits in (2, 4)
        self.B, self.H_q, self.H_kv, self.R, self.bits = B, H_q, H_kv, R, bits
        self.max_groups = max(1, -(-int(max_context) // 128))
        dev = torch.device(device)
        mg = self.max_groups
        z = lambda *s, dt: torch.zeros(*s, dtype=dt, device=dev)
        self.groups = z(B, H_kv, mg, 2304 if bits == 2 else 4352, dt=torch.int32)
        self.k_res = z(B, H_kv, R, 128, dt=torch.float16)
        self.v_res = z(B, H_kv, R // 4, 128, 4, dt=torch.float16)
        self.n_quant = z(B, dt=torch.int32)
        self.n_res = z(B, dt=torch.int32)
        self.status = z(1, dt=torch.int32)
        self.split_done = z(B, H_kv, dt=torch.int32)
        self.Wq, self.Wk = Wq, Wk
        if Wq is not None:
            assert Wk is not None and tuple(Wq.shape) == (H_q, 2, 128, 128) and tuple(Wk.shape) == (H_kv, 2, 128, 128)
            assert Wq.dtype == torch.float16 and Wk.dtype == torch.float16 and Wq.is_contiguous() and Wk.is_contiguous()
            assert state_storage in ("fp32", "fp16")
            self.S = z(B, H_kv, 256, 128, dt=torch.float32) if state_storage == "fp32" else None
            self.S16 = z(B, H_kv, 128, 64, 4, dt=torch.float16)
            self.P = z(B, H_kv, 256, dt=torch.float32)
        else:
            self.S = self.S16 = self.P = None
        self.struct = CacheStruct(
            B=B, H_q=H_q, H_kv=H_kv, d=128, G=128, R=R, D=256, bits=bits, max_groups=mg,
            groups=self.groups.data_ptr(),
            k_res=self.k_res.data_ptr(), v_res=self.v_res.data_ptr(),
            n_quant=self.n_quant.data_ptr(), n_res=self.n_res.data_ptr(),
            S=None if self.S is None else self.S.data_ptr(), S16=None if self.S16 is None else self.S16.data_ptr(),
            P=None if self.P is None else self.P.data_ptr(),
            Wq=None if Wq is None else Wq.data_ptr(), Wk=None if Wk is None else Wk.data_ptr(),
            status=self.status.data_ptr(), split_done=self.split_done.data_ptr(), flags=int(flags))
        self._ws = None
        self._device = self.groups.device
        self._context_ws = None  # scratch of prompt_attention and decode_windowed, and the streams that have used it
        self._context_streams = set()
        self._captured_ws = []
        self._seen_streams = set()  # those that a caller has named

    def bytes(self):
        ts = [self.groups, self.k_res, self.v_res]
        if self.S16 is not None:
            ts += [self.S16, self.P] + ([self.S] if self.S is not None else [])
        return sum(t.numel() * t.element_size() for t in ts)

    def append(self, k_new, v_new, n_new=None, keep_residual=0, stream=None):
        rc = kvlinc_append_quantize(self, k_new, v_new, n_new, k_new.shape[2], keep_residual, stream)
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_append_quantize: " + kvlinc_strerror(rc))

    def workspace(self, max_context=0):
        import torch
        need = kvlinc_decode_workspace_bytes(self, max_context)
        if self._ws is None or self._ws.numel() * 4 < need:
            self._ws = torch.empty((need + 3) // 4, dtype=torch.float32, device=self.groups.device)
        return self._ws

    def decode(self, q, out=None, max_context=0, stream=None):
        import torch
        if out is None:
            out = torch.empty_like(q)
        # the library checks the size before it launches anything: asked for only where the workspace at hand does not do
        ws = self._ws
        rc = KVLINC_EWORKSPACE if ws is None else kvlinc_decode_attention(self, q, out, ws, ws.numel() * 4, max_context, stream)
        if rc == KVLINC_EWORKSPACE:
            ws = self.workspace(max_context)
            rc = kvlinc_decode_attention(self, q, out, ws, ws.numel() * 4, max_context, stream)
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_decode_attention: " + kvlinc_strerror(rc))
        return out

    # The calls below check their tensors: what the C entry points take is an address.
    def _tensor(self, t, name, shape, dtype):
        try:
            if t.dtype is dtype and t.shape == shape and t.device == self._device and t.is_contiguous():
                return
        except AttributeError:
            pass
        import torch
        if not torch.is_tensor(t) or t.dtype != dtype or t.shape != shape:
            raise KVLincError("%s has to be a %s tensor of shape %s" % (name, dtype, tuple(shape)))
        if t.device != self._device:
            raise KVLincError("%s is on %s, the cache on %s" % (name, t.device, self._device))
        if not t.is_contiguous():
            raise KVLincError("%s has to be contiguous" % name)

    def _on(self, stream, *tensors):
        """The cache's device current, and `stream`, if one is given: what is allocated inside belongs to the stream that uses it, and the
        caller's tensors and the cache's are not handed out again before it is done with them."""
        import torch
        dev = self._device
        if dev.type != "cuda":
            raise KVLincError("the cache is on %s: the kernels need a GPU" % dev)
        here = _current_device() == dev.index
        if stream is None:
            return _NOTHING if here else torch.cuda.device(dev)
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=dev)
        if stream.device != dev:
            raise KVLincError("the stream is on %s, the cache on %s" % (stream.device, dev))
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        if stream.cuda_stream not in self._seen_streams:
            for t in (self.groups, self.k_res, self.v_res, self.n_quant, self.n_res, self.status, self.split_done, self.Wq, self.Wk, self.S, self.S16, self.P):
                if t is not None:
                    t.record_stream(stream)
            self._seen_streams.add(stream.cuda_stream)
        return torch.cuda.stream(stream)  # (makes its device current, too)

    @staticmethod
    def _limits(window, sinks, max_context):
        """(They go to the library as 32 bits.)"""
        if not (0 <= window < 1 << 31 and 0 <= sinks < 1 << 31):
            raise KVLincError("window and sinks have to be 0 or more, below 2^31, not %s and %s" % (window, sinks))
        if not -1 << 31 <= max_context < 1 << 31:
            raise KVLincError("max_context is below 2^31 either way, not %s" % max_context)

    def _with_scratch(self, call, need):
        """call(scratch, stream) on the current stream, with the scratch at hand if it does (the library looks before it launches anything), else with
        one of need() bytes.  One that a captured graph uses is kept as long as the cache."""
        import torch
        ws, stream = self._context_ws, _stream(None)
        rc = call(ws, stream)
        if rc == KVLINC_EWORKSPACE:
            ws = self._context_ws = torch.empty((need() + 3) // 4, dtype=torch.float32, device=self.groups.device)
            self._context_streams = {stream}
            rc = call(ws, stream)
        elif ws is not None and stream not in self._context_streams:  # (not handed out again before this stream is done with it)
            ws.record_stream(torch.cuda.current_stream())
            self._context_streams.add(stream)
        if ws is not None and torch.cuda.is_current_stream_capturing() and not any(ws is t for t in self._captured_ws):
            self._captured_ws.append(ws)
        return rc

    def prompt_attention(self, q, k_new, v_new, n_new=None, window=0, sinks=0, out=None, max_context=0, stream=None):
        """Attention of T new tokens of every sequence over the cache and, causally, their own rows; append them afterwards.

        q: [B, H_q, T, 128], k_new, v_new: [B, H_kv, T, 128] fp16; n_new: [B] int32 on the device or None (all T).  Returns out, [B, H_q, T,
        128] fp16; rows beyond n_new are left as they are (zero in an `out` made here).  window, sinks: kvlinc_context.h.

        max_context: the most tokens that any sequence holds before the call (0: whatever the cache has room for; 1 for an empty cache).  A call
        of more than 512 rows of a KV head keeps 580 bytes of scratch for each of them and KV head; a sequence that holds more gets zeros, and
        KVLINC_ST_BOUND is set in `status`."""
        import torch
        if not torch.is_tensor(q) or q.dim() != 4:
            raise KVLincError("q has to be a tensor of shape [B, H_q, T, 128]")
        T, half = q.shape[2], torch.float16
        self._limits(window, sinks, max_context)
        if T < 1:
            raise KVLincError("q has no rows")
        self._tensor(q, "q", (self.B, self.H_q, T, 128), half)
        self._tensor(k_new, "k_new", (self.B, self.H_kv, T, 128), half)
        self._tensor(v_new, "v_new", (self.B, self.H_kv, T, 128), half)
        if n_new is not None:
            self._tensor(n_new, "n_new", (self.B,), torch.int32)
        if out is not None:
            self._tensor(out, "out", q.shape, half)
        with self._on(stream, q, k_new, v_new, n_new, out):
            if out is None:
                out = torch.empty_like(q) if n_new is None else torch.zeros_like(q)
            rc = self._with_scratch(lambda ws, s: kvlinc_prompt_attention(self, q, k_new, v_new, n_new, T, window, sinks, out, ws, None, max_context, s),
                                    lambda: kvlinc_prompt_workspace_bytes(self, T, window, sinks, max_context))
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_prompt_attention: " + kvlinc_strerror(rc))
        return out

    def decode_windowed(self, q, window, sinks=0, out=None, max_context=0, stream=None):
        """decode() over the newest `window` tokens and the first `sinks` ones (window = 0: all).  q: [B, H_q, 128] fp16."""
        import torch
        half = torch.float16
        self._limits(window, sinks, max_context)
        self._tensor(q, "q", (self.B, self.H_q, 128), half)
        if out is not None:
            self._tensor(out, "out", q.shape, half)
        with self._on(stream, q, out):
            if out is None:
                out = torch.empty_like(q)
            rc = self._with_scratch(lambda ws, s: kvlinc_decode_attention_windowed(self, q, window, sinks, out, ws, None, max_context, s),
                                    lambda: kvlinc_decode_windowed_workspace_bytes(self, window, sinks, max_context))
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_decode_attention_windowed: " + kvlinc_strerror(rc))
        return out

    def read(self, first=None, T=None, dtype=None, rotated=False, k_out=None, v_out=None, stream=None):
        """Keys and values of tokens first[b] .. first[b] + T - 1 (first: [B] int32 on the device, None: 0), dequantized: (k_out, v_out), [B,
        H_kv, T, 128].  With one of the two given, only that one is read; with none, both are made here, in `dtype` (fp16), and zero where a
        sequence has no such token.  rotated: values in the basis they are stored in."""
        import torch
        types = {torch.float16: KVLINC_F16, torch.bfloat16: KVLINC_BF16, torch.float32: KVLINC_F32}
        given = [t for t in (k_out, v_out) if t is not None]
        if T is None:
            if not given or not torch.is_tensor(given[0]) or given[0].dim() != 4:
                raise KVLincError("T is needed where neither k_out nor v_out, [B, H_kv, T, 128], gives it")
            T = given[0].shape[2]
        if T < 1:
            raise KVLincError("T has to be 1 or more, not %s" % T)
        if dtype is None:
            dtype = given[0].dtype if given and torch.is_tensor(given[0]) else torch.float16
        if dtype not in types:
            raise KVLincError("dtype has to be one of %s" % ", ".join(str(t) for t in types))
        shape = (self.B, self.H_kv, int(T), 128)
        for t, name in ((k_out, "k_out"), (v_out, "v_out")):
            if t is not None:
                self._tensor(t, name, shape, dtype)
        if first is not None:
            self._tensor(first, "first", (self.B,), torch.int32)
        with self._on(stream, first, k_out, v_out):
            if not given:
                k_out, v_out = (torch.zeros(shape, dtype=dtype, device=self.groups.device) for _ in range(2))
            rc = kvlinc_cache_read(self, first, T, k_out, v_out, types[dtype], int(bool(rotated)), stream)
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_cache_read: " + kvlinc_strerror(rc))
        return k_out, v_out

    # ---- long generation in a cache of bounded size (kvlinc_bounded.h) ----

    def rotary(self, plan, q=None, k=None, v=None, n_new=None, first=None, depth=None, counted=True, q_out=None, k_out=None, v_out=None, dtype=None,
               stream=None):
        """Queries and keys of T new tokens of every sequence rotated to their positions, values taken along: (q_out, k_out, v_out), [B, heads, T, 128],
        contiguous, in `dtype` (fp16), as append, prompt_attention and, at T = 1, the decode calls take them.

        plan: KVLincRotary; q: [B, H_q, T, 128], k, v: [B, H_kv, T, 128], any of the three, fp16, bf16 or fp32, of any strides that are multiples of 16
        bytes with contiguous rows (a projection's output [B, T, heads, 128] transposed, say).  n_new: [B] int32 or None (all T); rows beyond it
        are left as they are (zero in outputs made here).  Row i is at position first[b] + depth[b, i] (None: 0; i) and, if counted, the tokens in
        the cache."""
        types = _row_types()
        if not isinstance(plan, KVLincRotary):
            raise KVLincError("plan has to be a KVLincRotary")
        dev, B = self._device, self.B
        if plan.freq.device != dev:
            raise KVLincError("the plan is on %s, the cache on %s" % (plan.freq.device, dev))
        some = q if q is not None else k if k is not None else v
        taken = getattr(some, "dtype", None)
        if taken not in types or some.dim() != 4:
            raise KVLincError("q, k or v is needed, a tensor of shape [B, heads, T, 128] and type %s" % ", ".join(str(t) for t in types))
        T = some.shape[2]
        if T < 1:
            raise KVLincError("there are no rows")
        if dtype is None:
            given = q_out if q_out is not None else k_out if k_out is not None else v_out
            dtype = next(iter(types)) if given is None else getattr(given, "dtype", None)
        if dtype not in types:
            raise KVLincError("dtype has to be one of %s" % ", ".join(str(t) for t in types))
        rows, missing = [None, None, None], False
        for i, t, out, h in ((0, q, q_out, self.H_q), (1, k, k_out, self.H_kv), (2, v, v_out, self.H_kv)):
            if t is None:
                if out is not None:
                    raise KVLincError("%s_out without %s" % ("qkv"[i], "qkv"[i]))
                continue
            shape = (B, h, T, 128)
            if getattr(t, "dtype", None) is not taken or t.shape != shape:
                raise KVLincError("%s has to be a %s tensor of shape %s" % ("qkv"[i], taken, shape))
            if t.device != dev:
                raise KVLincError("%s is on %s, the cache on %s" % ("qkv"[i], t.device, dev))
            of_sequence, of_head, of_token, of_channel = t.stride()
            if of_channel != 1:
                raise KVLincError("the rows of %s have to be contiguous" % "qkv"[i])
            to = 0
            if out is None:
                missing = True
            else:
                if getattr(out, "dtype", None) is not dtype or out.shape != shape or out.device != dev or not out.is_contiguous():
                    self._tensor(out, "qkv"[i] + "_out", shape, dtype)  # (says what is wrong)
                to = out.data_ptr()
            rows[i] = RowsStruct(t.data_ptr(), to, of_sequence if B > 1 else 0, of_head if h > 1 else 0, of_token if T > 1 else 0)
        if n_new is not None:
            self._tensor(n_new, "n_new", (B,), self.n_quant.dtype)
        if first is not None:
            self._tensor(first, "first", (B,), self.n_quant.dtype)
        if depth is not None:
            self._tensor(depth, "depth", (B, T), self.n_quant.dtype)
        outs = [q_out, k_out, v_out]
        with self._on(stream, plan.freq, n_new, first, depth, q, k, v, q_out, k_out, v_out):
            if missing:
                import torch
                make = torch.empty if n_new is None else torch.zeros
                for i, h in enumerate((self.H_q, self.H_kv, self.H_kv)):
                    if rows[i] is not None and outs[i] is None:
                        outs[i] = make((B, h, T, 128), dtype=dtype, device=dev)
                        rows[i].out = outs[i].data_ptr()
            rc = lib.kvlinc_rotary(self.struct, plan.struct, rows[0], rows[1], rows[2], T, _ptr(n_new), _ptr(first), _ptr(depth), 1 if counted else 0,
                                   types[taken], types[dtype], _stream(stream))
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_rotary: " + kvlinc_strerror(rc))
        return tuple(outs)

    def new_mass(self):
        """Accumulated attention weight of the groups, and of the window behind the last: zeros, [B, H_kv, max_groups + 1] fp32."""
        import torch
        return torch.zeros(self.B, self.H_kv, self.max_groups + 1, dtype=torch.float32, device=self._device)

    def _mass_tensors(self, mass, mass_out, decay):
        import torch
        shape = (self.B, self.H_kv, self.max_groups + 1)
        for t, name in ((mass, "mass"), (mass_out, "mass_out")):
            if t is not None:
                self._tensor(t, name, shape, torch.float32)
        if not 0.0 <= decay <= 1.0:
            raise KVLincError("decay has to be 0 to 1, not %s" % decay)

    def decode_mass(self, q, mass, decay=1.0, mass_out=None, out=None, max_context=0, stream=None):
        """One decode step over the whole cache that also accumulates the attention weight of every group: mass_out = decay mass + the weights of this
        query (mass_out None: in mass itself; mass None: zeros).  q: [B, H_q, 128] fp16.  Returns out."""
        import torch
        half = torch.float16
        self._limits(0, 0, max_context)
        self._tensor(q, "q", (self.B, self.H_q, 128), half)
        if mass_out is None:
            mass_out = mass
        if mass_out is None:
            raise KVLincError("mass or mass_out is needed")
        self._mass_tensors(mass, mass_out, decay)
        if out is not None:
            self._tensor(out, "out", q.shape, half)
        with self._on(stream, q, out, mass, mass_out):
            if out is None:
                out = torch.empty_like(q)
            rc = self._with_scratch(lambda ws, s: kvlinc_decode_attention_mass(self, q, out, mass, decay, mass_out, ws, None, max_context, s),
                                    lambda: kvlinc_decode_mass_workspace_bytes(self, max_context))
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_decode_attention_mass: " + kvlinc_strerror(rc))
        return out

    def attention_mass(self, q, mass=None, n_rows=None, decay=1.0, mass_out=None, max_context=0, stream=None):
        """The attention weight that the groups receive from T query rows of every sequence, its newest tokens, which the cache already holds: mass_out =
        decay mass + their weights (mass_out None: in mass itself, or a new one; mass None: zeros).  q: [B, H_q, T, 128] fp16; n_rows: [B] int32 or None
        (all T).  max_context: the most tokens that any sequence holds (0: whatever the cache has room for); one that holds more adds
        nothing, and KVLINC_ST_BOUND is set in `status`.  The scratch, kept with the cache, is 4 bytes for every row of a query head and group of max_context
        (all rows of 32768 tokens, 32 heads: 1.1 GB): a long prompt chunk by chunk, a call behind each append, needs that of a chunk.  Returns mass_out."""
        import torch
        if not torch.is_tensor(q) or q.dim() != 4:
            raise KVLincError("q has to be a tensor of shape [B, H_q, T, 128]")
        T = q.shape[2]
        self._limits(0, 0, max_context)
        if T < 1:
            raise KVLincError("q has no rows")
        self._tensor(q, "q", (self.B, self.H_q, T, 128), torch.float16)
        if n_rows is not None:
            self._tensor(n_rows, "n_rows", (self.B,), torch.int32)
        if mass_out is None:
            mass_out = mass
        self._mass_tensors(mass, mass_out, decay)
        with self._on(stream, q, n_rows, mass, mass_out):
            if mass_out is None:
                mass_out = self.new_mass()
            rc = self._with_scratch(lambda ws, s: kvlinc_attention_mass(self, q, n_rows, T, mass, decay, mass_out, ws, None, max_context, s),
                                    lambda: kvlinc_attention_mass_workspace_bytes(self, T, max_context))
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_attention_mass: " + kvlinc_strerror(rc))
        return mass_out

    def evict(self, mass, keep, limit=None, first=1, last=1, to=None, mass_out=None, offset=None, offset_out=None, kept=None, stream=None):
        """Sequences of more than `limit` groups (None: keep) cut to `keep` of them, of each KV head the first, the newest `last` and those with the largest
        mass: in place, or into the cache `to`.  mass: [B, H_kv, max_groups + 1] fp32, as decode_mass and attention_mass leave it; mass_out: where that
        of what is kept goes, in the shape of `to` (None: in mass itself, in place only).  offset, offset_out: [B] int32 or None, tokens dropped so
        far (offset_out None: in offset itself), what rotary takes as `first`.  kept: [B, H_kv, max_groups of `to`] int32 or None, the slots that the
        groups had.  Returns the cache."""
        import torch
        if to is None:
            to = self
        if not isinstance(to, KVLincCache):
            raise KVLincError("to has to be a KVLincCache")
        if to._device != self._device:
            raise KVLincError("to is on %s, the cache on %s" % (to._device, self._device))
        if limit is None:
            limit = keep
        if not (0 <= keep < 1 << 31 and 0 <= limit < 1 << 31 and 0 <= first < 1 << 31 and 0 <= last < 1 << 31):
            raise KVLincError("keep, limit, first and last have to be 0 or more, below 2^31, not %s, %s, %s and %s" % (keep, limit, first, last))
        if mass_out is None and to is self:
            mass_out = mass
        if offset_out is None:
            offset_out = offset
        self._tensor(mass, "mass", (self.B, self.H_kv, self.max_groups + 1), torch.float32)
        if mass_out is not mass or to is not self:
            to._tensor(mass_out, "mass_out", (to.B, to.H_kv, to.max_groups + 1), torch.float32)
        if offset is not None:
            self._tensor(offset, "offset", (self.B,), torch.int32)
        if offset_out is not offset:
            self._tensor(offset_out, "offset_out", (self.B,), torch.int32)
        if kept is not None:
            self._tensor(kept, "kept", (to.B, to.H_kv, to.max_groups), torch.int32)
        theirs = () if to is self else (to.groups, to.k_res, to.v_res, to.n_quant, to.n_res, to.split_done)
        with self._on(stream, mass, mass_out, offset, offset_out, kept, *theirs):
            rc = self._with_scratch(lambda ws, s: kvlinc_cache_evict(self, to, mass, mass_out, keep, limit, first, last, offset, offset_out, kept, ws, None, s),
                                    lambda: kvlinc_cache_evict_workspace_bytes(self))
        if rc != KVLINC_OK:
            raise KVLincError("kvlinc_cache_evict: " + kvlinc_strerror(rc))
        return to
