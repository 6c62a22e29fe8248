"""ctypes binding of include/spconv.h: same names, argument marshalling only.

torch is used for device memory and the current HIP stream; every step of the
computation runs inside libspconv.so.

Stream ordering: every call enqueues its work on `stream` (default: torch's
current stream) and returns without waiting.  A tensor that a call returns or
fills is therefore ordered on that stream only: read it on the same stream, or
synchronise that stream first (`tensor.cpu()` runs on torch's current stream).
The memory of what a call returns comes from torch's pool of that stream.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

OP_FWD, OP_DGRAD, OP_WGRAD = 0, 1, 2
FLAG_SLABS = 1
_CUDA = torch.device("cuda")
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class SpconvError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = load_library()
        msg = lib.spconv_strerror(status).decode()
        hip = lib.spconv_last_hip_error().decode()
        super().__init__(f"{where}: {msg} ({status})" + (f" [{hip}]" if status == -6 and hip else ""))
        self.status = status


class Config(C.Structure):
    """Mirror of spconv_config (zero = library defaults)."""
    _fields_ = [("n_split", C.c_int32), ("tile_m", C.c_int32), ("tile_n", C.c_int32),
                ("wgrad_pairs", C.c_int32), ("kernel", C.c_int32), ("flags", C.c_int32), ("reserved", C.c_int32 * 2)]

    def __repr__(self):
        return (f"Config(n_split={self.n_split}, tile_m={self.tile_m}, tile_n={self.tile_n}, "
                f"wgrad_pairs={self.wgrad_pairs}, kernel={self.kernel}" + (f", flags={self.flags}" if self.flags else "") + ")")


class LayerShape(C.Structure):
    """Mirror of spconv_layer_shape."""
    _fields_ = [("c_in", C.c_int32), ("c_out", C.c_int32)]


class Q8(C.Structure):
    """Mirror of spconv_q8."""
    _fields_ = [("data", C.c_void_p), ("exps", C.c_void_p)]


class LaunchInfo(C.Structure):
    """Mirror of spconv_launch_info."""
    _fields_ = [("kernel", C.c_int32), ("parts", C.c_int32), ("sorted", C.c_int32), ("tile_m", C.c_int32),
                ("tile_n", C.c_int32), ("k_steps", C.c_int32), ("waves", C.c_int32), ("threads", C.c_int32),
                ("grid", C.c_int32 * 3), ("xcd_ranges", C.c_int32), ("lo", C.c_int32 * 4), ("width", C.c_int32 * 4),
                ("lds_bytes", C.c_int64), ("slab_bytes", C.c_int64), ("slab_map_bytes", C.c_int64),
                ("rows_pad", C.c_int64), ("n_tiles", C.c_int64), ("map_elems", C.c_int64 * 4)]


_LIB = None


def lib_path() -> str:
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspconv.so")


def load_library():
    """Loads libspconv.so and declares every prototype of include/spconv.h."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2311_12862_amd.build` "
                          "(there is no fallback implementation)")
    lib = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
    cfgp = C.POINTER(Config)
    protos = {
        "spconv_build_kmap": (i32, [vp, i64, i32, i32, i32, vp, C.POINTER(vp)]),
        "spconv_build_kmap_async": (i32, [vp, i64, i32, i32, i32, vp, C.POINTER(vp)]),
        "spconv_build_kmap_dilated": (i32, [vp, i64, i32, vp, C.POINTER(vp)]),
        "spconv_kmap_status": (i32, [vp, vp]),
        "spconv_kmap_transpose": (i32, [vp, vp, C.POINTER(vp)]),
        "spconv_kmap_pointwise": (i32, [vp, i32, vp, C.POINTER(vp)]),
        "spconv_kmap_sizes": (i32, [vp, C.POINTER(i64), C.POINTER(i64), C.POINTER(i64)]),
        "spconv_kmap_out_coords": (i32, [vp, vp, vp]),
        "spconv_kmap_in_coords": (i32, [vp, vp, vp]),
        "spconv_kmap_export": (i32, [vp, vp, vp]),
        "spconv_kmap_export_mask": (i32, [vp, vp, vp]),
        "spconv_kmap_prepare": (i32, [vp, i32, cfgp, vp]),
        "spconv_kmap_drop_plans": (i32, [vp]),
        "spconv_kmap_export_perm": (i32, [vp, i32, cfgp, i32, vp, vp]),
        "spconv_kmap_mac_units": (i32, [vp, i32, cfgp, C.POINTER(i64), C.POINTER(i64), vp]),
        "spconv_kmap_destroy": (None, [vp]),
        "spconv_fwd": (i32, [vp, vp, vp, i32, i32, i32, cfgp, vp, vp]),
        "spconv_fwd_noalloc": (i32, [vp, vp, vp, i32, i32, i32, cfgp, vp, vp]),
        "spconv_dgrad": (i32, [vp, vp, vp, i32, i32, i32, cfgp, vp, vp]),
        "spconv_wgrad": (i32, [vp, vp, vp, i32, i32, i32, cfgp, vp, vp]),
        "spconv_tune": (i32, [vp, i32, i32, i32, i32, i32, cfgp, C.POINTER(C.c_float), vp]),
        "spconv_tune_group": (i32, [vp, C.POINTER(LayerShape), i32, i32, i32, i32, cfgp, cfgp, cfgp,
                                    C.POINTER(C.c_float), vp]),
        "spconv_ew": (i32, [i32, vp, vp, vp, i64, i32, vp]),
        "spconv_copy_cols": (i32, [vp, i32, i32, vp, i32, i32, i32, i64, i32, vp]),
        "spconv_q8_pack": (i32, [vp, i64, i32, i32, C.POINTER(Q8), vp]),
        "spconv_q8_unpack": (i32, [C.POINTER(Q8), i64, i32, i32, vp, vp]),
        "spconv_relu_bwd_q8": (i32, [vp, C.POINTER(Q8), vp, i64, i32, vp]),
        "spconv_wgrad_q8": (i32, [C.POINTER(Q8), vp, vp, i32, i32, i32, cfgp, vp, vp]),
        "spconv_layer_norm_fwd": (i32, [vp, vp, vp, vp, C.c_float, i32, i64, i32, i32, vp, vp, C.POINTER(Q8),
                                        C.POINTER(Q8), vp]),
        "spconv_layer_norm_bwd_workspace": (i64, [i64, i32]),
        "spconv_layer_norm_bwd": (i32, [vp, vp, C.POINTER(Q8), vp, C.POINTER(Q8), vp, vp, i64, i32, i32, vp, vp, vp, vp,
                                        vp, i64, vp]),
        "spconv_set_allocator": (i32, [vp, vp, vp]),
        "spconv_describe_launch": (i32, [i32, i64, i64, i32, i32, i32, cfgp, i32, C.POINTER(LaunchInfo)]),
        "spconv_measure_peaks": (i32, [C.POINTER(C.c_double), C.POINTER(C.c_double), vp]),
        "spconv_strerror": (C.c_char_p, [i32]),
        "spconv_last_hip_error": (C.c_char_p, []),
        "spconv_version": (i32, []),
    }
    for name, (res, args) in protos.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


_ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p)
_FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p, C.c_void_p)
_allocator_refs = None   # keeps the ctypes thunks of the installed callbacks alive


def set_allocator(alloc=None, free=None):
    """spconv_set_allocator: alloc(bytes, stream) -> device address (int, 0 = out of memory) and
    free(address, stream) serve every device allocation the library makes from now on; stream is the
    raw hipStream_t (int, 0 = null stream) of the library call in progress.  (None, None) restores the
    library's own pool.  Switch only while no kmap is alive."""
    global _allocator_refs
    if (alloc is None) != (free is None):
        raise ValueError("give both callbacks or neither")
    lib = load_library()
    if alloc is None:
        _check(lib.spconv_set_allocator(None, None, None), "spconv_set_allocator")
        _allocator_refs = None
        return
    a = _ALLOC_FN(lambda n, stream, _user: int(alloc(int(n), int(stream or 0))) or None)
    f = _FREE_FN(lambda ptr, stream, _user: free(int(ptr or 0), int(stream or 0)))
    _check(lib.spconv_set_allocator(C.cast(a, C.c_void_p), C.cast(f, C.c_void_p), None), "spconv_set_allocator")
    _allocator_refs = (a, f)


def _check(status: int, where: str):
    if status != 0:
        raise SpconvError(status, where)


def _current_stream():
    """Handle of torch's current stream.  torch.cuda.current_stream() builds a Stream object on the way (2.7 us of
    the 9 us that a call of this module took); the handle itself is a look-up (0.1 us)."""
    global _current_stream
    handle = torch.cuda.current_stream().cuda_stream   # (initialises the device if nothing has yet)
    raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and dev is not None and raw(dev()) == handle:
        _current_stream = lambda: raw(dev())
    return handle


def _stream(stream):
    """None: torch's current stream; a torch stream; or a raw hipStream_t handle as int (0 = null stream)."""
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _device_now():
    """Number of the current device (a look-up, as in _current_stream)."""
    global _device_now
    torch.cuda.current_device()   # (initialises the device if nothing has yet)
    _device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _device_now()


def _stream_here(dev):
    """_stream(None) where the current device's number is known."""
    return _raw_stream(dev) if _raw_stream is not None else _stream(None)


def _elsewhere(dev, stream, call, *args):
    """call(*args) with device dev current, and on it `stream` unless that is None.  What the call allocates then comes from the pool
    of the stream that uses it: a block of another stream's pool may still be read or written by that one's kernels.  The tensors that it
    returns may be read on the stream that was current before as well, once the caller has ordered the two; torch is told, so that it
    keeps a block that is given back until that stream is done with it."""
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError(f"a stream of device {stream.device_index} for tensors on device {dev}")
    if dev != _device_now():
        with torch.cuda.device(dev):
            return _elsewhere(dev, stream, call, *args)
    handle = None if stream is None else _stream(stream)
    if handle is None or handle == _stream_here(dev):
        return call(*args)
    before = torch.cuda.current_stream(dev)
    with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=dev) if handle else torch.cuda.default_stream(dev)):
        made = call(*args)
    for t in made if isinstance(made, tuple) else (made,):
        if t is not None:
            t.record_stream(before)
    return made


def _made_on(stream, like, shape, dtype):
    """The tensor that a call on `stream` is to fill (_elsewhere)."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    return _elsewhere(like.get_device(), stream, lambda: like.new_empty(shape, dtype=dtype))


def _ints_on(stream, shape):
    make = lambda: torch.empty(shape, dtype=torch.int32, device=_CUDA)
    return make() if stream is None else _elsewhere(_device_now(), stream, make)


def _cfg(cfg):
    return None if cfg is None else C.byref(cfg)


def _ptr(t):
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _dev_tensor(t, dtype=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return t


class KMap:
    """Owner of an spconv_kmap handle."""

    def __init__(self, handle, K):
        self._h = handle
        self.K = K
        self.V = K ** 3
        n_in, n_out = C.c_int64(), C.c_int64()
        _check(load_library().spconv_kmap_sizes(self._h, C.byref(n_in), C.byref(n_out), None), "spconv_kmap_sizes")
        self.n_in, self.n_out = n_in.value, n_out.value

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("kmap was destroyed")
        return self._h

    def status(self, stream=None):
        """spconv_kmap_status: raises on a range / duplicate error of an asynchronous build."""
        _check(load_library().spconv_kmap_status(self.handle, _stream(stream)), "spconv_kmap_status")

    def transpose(self, stream=None) -> "KMap":
        """spconv_kmap_transpose: the kmap of the paired transposed convolution, derived from this one."""
        h = C.c_void_p()
        _check(load_library().spconv_kmap_transpose(self.handle, _stream(stream), C.byref(h)), "spconv_kmap_transpose")
        return KMap(h, self.K)

    def pointwise(self, on_outputs: bool = False, stream=None) -> "KMap":
        """spconv_kmap_pointwise: the K = 1 kmap over this kmap's input (or output) rows."""
        h = C.c_void_p()
        _check(load_library().spconv_kmap_pointwise(self.handle, int(bool(on_outputs)), _stream(stream), C.byref(h)),
               "spconv_kmap_pointwise")
        return KMap(h, 1)

    def n_pairs(self) -> int:
        v = C.c_int64()
        _check(load_library().spconv_kmap_sizes(self.handle, None, None, C.byref(v)), "spconv_kmap_sizes")
        return v.value

    def out_coords(self, stream=None):
        dst = _ints_on(stream, (self.n_out, 4))
        _check(load_library().spconv_kmap_out_coords(self.handle, _ptr(dst), _stream(stream)), "spconv_kmap_out_coords")
        return dst

    def in_coords(self, stream=None):
        dst = _ints_on(stream, (self.n_in, 4))
        _check(load_library().spconv_kmap_in_coords(self.handle, _ptr(dst), _stream(stream)), "spconv_kmap_in_coords")
        return dst

    def export(self, stream=None):
        dst = _ints_on(stream, (self.n_out, self.V))
        _check(load_library().spconv_kmap_export(self.handle, _ptr(dst), _stream(stream)), "spconv_kmap_export")
        return dst

    def export_mask(self, stream=None):
        # bit patterns of uint32; K = 5: four words per row (bit k of the mask is bit k % 32 of word k // 32)
        shape = (self.n_out, 4) if self.K == 5 else (self.n_out,)
        dst = _ints_on(stream, shape)
        _check(load_library().spconv_kmap_export_mask(self.handle, _ptr(dst), _stream(stream)), "spconv_kmap_export_mask")
        return dst

    def prepare(self, op, cfg=None, stream=None):
        _check(load_library().spconv_kmap_prepare(self.handle, op, _cfg(cfg), _stream(stream)), "spconv_kmap_prepare")

    def drop_plans(self):
        _check(load_library().spconv_kmap_drop_plans(self.handle), "spconv_kmap_drop_plans")

    def export_perm(self, op, cfg, split, stream=None):
        rows = self.n_out if op == OP_FWD else self.n_in
        dst = _ints_on(stream, (rows,))
        _check(load_library().spconv_kmap_export_perm(self.handle, op, _cfg(cfg), split, _ptr(dst), _stream(stream)),
               "spconv_kmap_export_perm")
        return dst

    def mac_units(self, op, cfg=None, stream=None):
        ex, ef = C.c_int64(), C.c_int64()
        _check(load_library().spconv_kmap_mac_units(self.handle, op, _cfg(cfg), C.byref(ex), C.byref(ef),
                                                    _stream(stream)), "spconv_kmap_mac_units")
        return ex.value, ef.value

    def destroy(self):
        if self._h is not None:
            load_library().spconv_kmap_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def build_kmap(coords, K: int = 3, stride: int = 1, transposed: bool = False, stream=None,
               asynchronous: bool = False, dilate: bool = False) -> KMap:
    """spconv_build_kmap (or spconv_build_kmap_async, or spconv_build_kmap_dilated with dilate=True):
    coords is an int32 device tensor [N, 4] = (b, x, y, z)."""
    _dev_tensor(coords, torch.int32)
    if coords.ndim != 2 or coords.shape[1] != 4:
        raise ValueError("coords must be [N, 4]")
    h = C.c_void_p()
    lib = _LIB or load_library()
    if dilate:
        if stride != 1 or transposed or asynchronous:
            raise ValueError("dilated kmaps are stride 1, not transposed, built synchronously")
        _check(lib.spconv_build_kmap_dilated(_ptr(coords), coords.shape[0], K, _stream(stream), C.byref(h)),
               "spconv_build_kmap_dilated")
        return KMap(h, K)
    fn, name = (lib.spconv_build_kmap_async, "spconv_build_kmap_async") if asynchronous else \
               (lib.spconv_build_kmap, "spconv_build_kmap")
    _check(fn(_ptr(coords), coords.shape[0], K, stride, int(transposed), _stream(stream), C.byref(h)), name)
    return KMap(h, K)


def _out_tensor(out, shape, dtype, like):
    """A caller-supplied output: exactly the shape, type and device the call writes (the C ABI has
    no row count to catch a wrong one), contiguous."""
    _dev_tensor(out, dtype)
    if tuple(out.shape) != tuple(shape) or out.device != like.device:
        raise SpconvError(-5, f"out is {tuple(out.shape)} on {out.device}, the call writes {tuple(shape)} on {like.device}")
    return out


def _conv_args(a, w_or_b, kmap, rows_a):
    """The data type's number; what does not fit raises."""
    dt = _DTYPES.get(a.dtype)
    if (dt is not None and a.is_cuda and a.is_contiguous() and w_or_b.is_cuda and w_or_b.is_contiguous()
            and w_or_b.dtype is a.dtype and a.ndim == 2 and a.shape[0] == rows_a):
        return dt
    _dev_tensor(a)
    if a.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {a.dtype}")
    if a.ndim != 2 or a.shape[0] != rows_a:
        raise SpconvError(-5, f"feature rows {tuple(a.shape)} do not fit the kmap ({rows_a} rows)")
    _dev_tensor(w_or_b, a.dtype)
    return _DTYPES[a.dtype]


def fwd(feats, weights, kmap: KMap, cfg: Config | None = None, out=None, stream=None):
    """spconv_fwd: feats [n_in, C_in], weights [K^3, C_in, C_out] -> out [n_out, C_out]."""
    dt = _conv_args(feats, weights, kmap, kmap.n_in)
    V, c_in, c_out = weights.shape
    if V != kmap.V or c_in != feats.shape[1]:
        raise SpconvError(-5, "weights shape does not fit")
    if out is None:
        out = _made_on(stream, feats, (kmap.n_out, c_out), feats.dtype)
    else:
        _out_tensor(out, (kmap.n_out, c_out), feats.dtype, feats)
    status = _LIB.spconv_fwd(_ptr(feats), _ptr(weights), kmap.handle, c_in, c_out, dt, _cfg(cfg), _ptr(out),
                             _stream(stream))
    if status:
        _check(status, "spconv_fwd")
    return out


def fwd_noalloc(feats, weights, kmap: KMap, out, cfg: Config | None = None, stream=None):
    """spconv_fwd_noalloc: spconv_fwd into the caller's `out` on a prepared plan, without any allocation."""
    dt = _conv_args(feats, weights, kmap, kmap.n_in)
    V, c_in, c_out = weights.shape
    if V != kmap.V or c_in != feats.shape[1]:
        raise SpconvError(-5, "weights shape does not fit")
    _out_tensor(out, (kmap.n_out, c_out), feats.dtype, feats)
    _check(load_library().spconv_fwd_noalloc(_ptr(feats), _ptr(weights), kmap.handle, c_in, c_out, dt, _cfg(cfg),
                                             _ptr(out), _stream(stream)), "spconv_fwd_noalloc")
    return out


def dgrad(dout, weights, kmap: KMap, cfg: Config | None = None, out=None, stream=None):
    """spconv_dgrad: dout [n_out, C_out], weights [K^3, C_in, C_out] -> din [n_in, C_in]."""
    dt = _conv_args(dout, weights, kmap, kmap.n_out)
    V, c_in, c_out = weights.shape
    if V != kmap.V or c_out != dout.shape[1]:
        raise SpconvError(-5, "weights shape does not fit")
    if out is None:
        out = _made_on(stream, dout, (kmap.n_in, c_in), dout.dtype)
    else:
        _out_tensor(out, (kmap.n_in, c_in), dout.dtype, dout)
    status = _LIB.spconv_dgrad(_ptr(dout), _ptr(weights), kmap.handle, c_in, c_out, dt, _cfg(cfg), _ptr(out),
                               _stream(stream))
    if status:
        _check(status, "spconv_dgrad")
    return out


def wgrad(feats, dout, kmap: KMap, cfg: Config | None = None, out=None, stream=None):
    """spconv_wgrad: feats [n_in, C_in], dout [n_out, C_out] -> dweights fp32 [K^3, C_in, C_out].
    feats may be a Checkpoint of the layer's input (spconv_wgrad_q8)."""
    if isinstance(feats, Checkpoint):
        return _wgrad_q8(feats, dout, kmap, cfg, out, stream)
    dt = _conv_args(feats, dout, kmap, kmap.n_in)
    if dout.ndim != 2 or dout.shape[0] != kmap.n_out:
        raise SpconvError(-5, "dout rows do not fit the kmap")
    c_in, c_out = feats.shape[1], dout.shape[1]
    if out is None:
        out = _made_on(stream, feats, (kmap.V, c_in, c_out), torch.float32)
    else:
        _out_tensor(out, (kmap.V, c_in, c_out), torch.float32, feats)
    status = _LIB.spconv_wgrad(_ptr(feats), _ptr(dout), kmap.handle, c_in, c_out, dt, _cfg(cfg), _ptr(out),
                               _stream(stream))
    if status:
        _check(status, "spconv_wgrad")
    return out


def _wgrad_q8(kept, dout, kmap, cfg, out, stream=None):
    dt, shape, dev = _row_args(dout)
    if shape[0] != kmap.n_out or kept.rows != kmap.n_in:
        raise SpconvError(-5, f"rows of the checkpoint ({kept.rows}) or of dout {tuple(shape)} do not fit the kmap "
                              f"({kmap.n_in} in, {kmap.n_out} out)")
    if kept.get_device() != dev:
        raise ValueError(f"tensors on {dout.device} and {kept.device}")
    if stream is not None or dev != _device_now():
        return _elsewhere(dev, stream, _wgrad_q8, kept, dout, kmap, cfg, out)
    c_in, c_out = kept.channels, shape[1]
    if out is None:
        out = dout.new_empty((kmap.V, c_in, c_out), dtype=torch.float32)
    else:
        _out_tensor(out, (kmap.V, c_in, c_out), torch.float32, dout)
    status = _LIB.spconv_wgrad_q8(kept.byref, dout.data_ptr() or None, kmap.handle, c_in, c_out, dt, _cfg(cfg), out.data_ptr(),
                                  _stream_here(dev))
    if status:
        _check(status, "spconv_wgrad_q8")
    return out


def tune(kmap: KMap, c_in: int, c_out: int, dtype, op: int, layers_sharing_kmap: int = 1, stream=None):
    """spconv_tune: returns (Config, microseconds)."""
    best, us = Config(), C.c_float()
    _check(load_library().spconv_tune(kmap.handle, c_in, c_out, _DTYPES[dtype], op, layers_sharing_kmap,
                                      C.byref(best), C.byref(us), _stream(stream)), "spconv_tune")
    return best, us.value


def tune_group(kmap: KMap, layers, dtype, training: bool = False, bind_fwd_dgrad: bool = True, stream=None):
    """spconv_tune_group: layers is a sequence of (c_in, c_out) of the layers that run on kmap.
    Returns (fwd, dgrad, wgrad, microseconds): lists of Config, one per layer (dgrad and wgrad are
    None for training=False)."""
    n = len(layers)
    shapes = (LayerShape * n)(*[LayerShape(int(ci), int(co)) for ci, co in layers])
    fwd = (Config * n)()
    dg = (Config * n)() if training else None
    wg = (Config * n)() if training else None
    us = C.c_float()
    _check(load_library().spconv_tune_group(kmap.handle, shapes, n, _DTYPES[dtype], int(training), int(bind_fwd_dgrad),
                                            fwd, dg, wg, C.byref(us), _stream(stream)), "spconv_tune_group")
    copy = lambda arr: None if arr is None else [Config.from_buffer_copy(c) for c in arr]
    return copy(fwd), copy(dg), copy(wg), us.value


def describe_launch(K: int, rows: int, rows_src: int, c_red: int, c_cols: int, dtype, cfg: Config | None = None,
                    dgrad: bool = False) -> LaunchInfo:
    """spconv_describe_launch: the launch geometry of a forward / dgrad call (host arithmetic; needs no GPU)."""
    info = LaunchInfo()
    _check(load_library().spconv_describe_launch(K, rows, rows_src, c_red, c_cols, _DTYPES[dtype], _cfg(cfg), int(dgrad),
                                                 C.byref(info)), "spconv_describe_launch")
    return info


def measure_peaks(stream=None):
    """spconv_measure_peaks: (streaming-copy GB/s, fp16 MFMA TFLOP/s) measured on the current device."""
    hbm, mfma = C.c_double(), C.c_double()
    _check(load_library().spconv_measure_peaks(C.byref(hbm), C.byref(mfma), _stream(stream)), "spconv_measure_peaks")
    return hbm.value, mfma.value


EW_RELU, EW_ADD, EW_ADD_RELU, EW_RELU_BWD = 0, 1, 2, 3


def ew(op: int, a, b=None, out=None, stream=None):
    """spconv_ew: element-wise glue (see include/spconv.h); out defaults to a new tensor like a.
    For EW_RELU_BWD, b may be a Checkpoint of the ReLU's output (spconv_relu_bwd_q8)."""
    if isinstance(b, Checkpoint):
        return _relu_bwd_q8(op, a, b, out, stream)
    _dev_tensor(a)
    if b is not None:
        _dev_tensor(b, a.dtype)
        if b.shape != a.shape:
            raise ValueError("shape mismatch")
    if out is None:
        out = _made_on(stream, a, a.shape, a.dtype)
    status = load_library().spconv_ew(op, _ptr(a), _ptr(b), _ptr(out), a.numel(), _DTYPES[a.dtype], _stream(stream))
    if status:
        _check(status, "spconv_ew")
    return out


def _relu_bwd_q8(op, a, kept, out, stream=None):
    if op != EW_RELU_BWD:
        raise ValueError("a Checkpoint stands for the output of EW_RELU_BWD only")
    dt, shape, dev = _row_args(a)
    if shape != (kept.rows, kept.channels):
        raise ValueError("shape mismatch")
    ref = _kept_like(kept, a, shape, dev)
    if stream is not None or dev != _device_now():
        return _elsewhere(dev, stream, _relu_bwd_q8, op, a, kept, out)
    if out is None:
        out = torch.empty_like(a)
        to = out.data_ptr() or None
    else:
        to = _like(out, a, shape, dev)
    status = (_LIB or load_library()).spconv_relu_bwd_q8(a.data_ptr() or None, ref, to, kept.rows * kept.channels, dt,
                                                         _stream_here(dev))
    if status:
        _check(status, "spconv_relu_bwd_q8")
    return out


def copy_cols(src, src_off: int, dst, dst_off: int, cols: int, stream=None):
    """spconv_copy_cols on two [rows, ld] tensors."""
    _dev_tensor(src)
    _dev_tensor(dst, src.dtype)
    if src.shape[0] != dst.shape[0]:
        raise ValueError("row mismatch")
    _check(load_library().spconv_copy_cols(_ptr(src), src.shape[1], src_off, _ptr(dst), dst.shape[1], dst_off, cols,
                                           src.shape[0], _DTYPES[src.dtype], _stream(stream)), "spconv_copy_cols")
    return dst


# ---- layer norm and 8-bit checkpoints ------------------------------------------------------------
# A call of these takes 6 to 14 us on the host (two of each three go to torch's allocations and the launches), more than many of
# their kernels: checks read a tensor's attributes once, and the device is switched only where it is another one.

def _row_args(x):
    """Data type's number, shape and device of a tensor [rows, channels]; what is none raises."""
    dt, shape, dev = _DTYPES.get(x.dtype), x.shape, x.get_device()
    if dt is None or len(shape) != 2 or dev < 0 or not x.is_contiguous():
        _dev_tensor(x)
        raise ValueError(f"expected a tensor [rows, channels] of {', '.join(map(str, _DTYPES))}, got {tuple(shape)} of {x.dtype}")
    return dt, shape, dev


def _like(t, x, shape, dev):
    """Address of a tensor that a call takes or fills beside x, of the same shape, type and device."""
    if t.dtype is not x.dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _out_tensor(t, shape, x.dtype, x)
    return t.data_ptr() or None


def _kept_like(kept, x, shape, dev):
    """The checkpoint of a tensor like x, for the C call."""
    if not isinstance(kept, Checkpoint):
        raise ValueError(f"expected a Checkpoint, got {type(kept).__name__}")
    if (kept.rows, kept.channels) != shape:
        raise SpconvError(-5, f"the checkpoint is {(kept.rows, kept.channels)}, the tensor {tuple(shape)}")
    if kept.get_device() != dev:
        raise ValueError(f"tensors on {x.device} and {kept.device}")
    return kept.byref


def _floats(t, shape, x, dev):
    """Address of fp32 values that a call reads beside x."""
    if t.dtype is not torch.float32 or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _dev_tensor(t, torch.float32)
        if t.shape != shape:
            raise SpconvError(-5, f"expected fp32 values {shape}, got {tuple(t.shape)}")
        raise ValueError(f"tensors on {x.device} and {t.device}")
    return t.data_ptr() or None


class Checkpoint:
    """An activation [rows, channels] kept in 8 bits (spconv_q8): data int8 [rows, channels], exps uint8
    [rows, ceil(channels / 32)].  What a backward pass reads an activation for takes a Checkpoint in its place: `wgrad`,
    `layer_norm_bwd` and the gradient through a ReLU, `ew(EW_RELU_BWD, ...)`."""
    __slots__ = ("rows", "channels", "byref", "_room", "_tensors")   # byref: the spconv_q8 of it, for the C calls

    def __init__(self, data, exps):
        _dev_tensor(data, torch.int8)
        _dev_tensor(exps, torch.uint8)
        if data.ndim != 2 or exps.ndim != 2 or exps.shape != (data.shape[0], -(-data.shape[1] // 32)):
            raise ValueError(f"data is {tuple(data.shape)}, exps {tuple(exps.shape)}: expected [rows, C] and [rows, ceil(C / 32)]")
        if data.device != exps.device:
            raise ValueError(f"tensors on {data.device} and {exps.device}")
        self.rows, self.channels = data.shape
        self._room, self._tensors = data, (data, exps)
        self.byref = C.byref(Q8(_ptr(data), _ptr(exps)))

    @classmethod
    def empty(cls, rows: int, channels: int, device=_CUDA) -> "Checkpoint":
        """Room for the checkpoint of a tensor [rows, channels] (one allocation: data, then exps)."""
        if rows < 0 or channels < 1:
            raise ValueError(f"no tensor is [{rows}, {channels}]")
        self = cls.__new__(cls)
        self.rows, self.channels = rows, channels
        at = (rows * channels + 15) // 16 * 16
        self._room = torch.empty((at + rows * (-(-channels // 32)),), dtype=torch.int8, device=device)
        self._tensors = None
        if not self._room.is_cuda:
            raise ValueError(f"expected a device, got {device}")
        base = self._room.data_ptr()
        self.byref = C.byref(Q8(base or None, base + at or None))
        return self

    def _views(self):
        """(data, exps); made when they are asked for, and there for other threads once both are."""
        views = self._tensors
        if views is None:
            rows, channels, room = self.rows, self.channels, self._room
            size = rows * channels
            exps = room[(size + 15) // 16 * 16:].view(torch.uint8).view(rows, -(-channels // 32))
            self._tensors = views = room[:size].view(rows, channels), exps
        return views

    @property
    def data(self):
        return self._views()[0]

    @property
    def exps(self):
        return self._views()[1]

    @property
    def device(self):
        return self._room.device

    def get_device(self) -> int:
        return self._room.get_device()

    def record_stream(self, stream):
        for t in self._tensors or (self._room,):
            t.record_stream(stream)


def q8_pack(x, out: Checkpoint | None = None, stream=None) -> Checkpoint:
    """spconv_q8_pack: the 8-bit checkpoint of x [rows, channels]."""
    dt, shape, dev = _row_args(x)
    if stream is not None or dev != _device_now():
        return _elsewhere(dev, stream, q8_pack, x, out)
    rows, channels = shape
    if out is None:
        out = Checkpoint.empty(rows, channels)
    status = (_LIB or load_library()).spconv_q8_pack(x.data_ptr() or None, rows, channels, dt, _kept_like(out, x, shape, dev),
                                                     _stream_here(dev))
    if status:
        _check(status, "spconv_q8_pack")
    return out


def q8_unpack(kept: Checkpoint, dtype, out=None, stream=None):
    """spconv_q8_unpack: the values that a checkpoint stands for, as a tensor of dtype."""
    dt = _DTYPES.get(dtype)
    if dt is None:
        raise ValueError(f"unsupported dtype {dtype}")
    dev = kept.get_device()
    if stream is not None or dev != _device_now():
        return _elsewhere(dev, stream, q8_unpack, kept, dtype, out)
    rows, channels = kept.rows, kept.channels
    if out is None:
        out = kept._room.new_empty((rows, channels), dtype=dtype)
    else:
        _out_tensor(out, (rows, channels), dtype, kept)
    status = (_LIB or load_library()).spconv_q8_unpack(kept.byref, rows, channels, dt, out.data_ptr() or None,
                                                       _stream_here(dev))
    if status:
        _check(status, "spconv_q8_unpack")
    return out


def layer_norm_fwd(x, weight=None, bias=None, eps: float = 1e-5, relu: bool = False, residual=None, out=None,
                   keep_x: Checkpoint | None = None, keep_y: Checkpoint | None = None, stream=None):
    """spconv_layer_norm_fwd: (y, stats) with y = act(norm(x) * weight + bias + residual), x and y [rows, channels],
    weight and bias fp32 [channels], stats fp32 [rows, 2] = (mean, 1 / std) for layer_norm_bwd.  keep_x and keep_y are
    filled with checkpoints of x and y in the same pass."""
    dt, shape, dev = _row_args(x)
    if stream is not None or dev != _device_now():
        return _elsewhere(dev, stream, layer_norm_fwd, x, weight, bias, eps, relu, residual, out, keep_x, keep_y)
    rows, channels = shape
    w = None if weight is None else _floats(weight, (channels,), x, dev)
    b = None if bias is None else _floats(bias, (channels,), x, dev)
    res = None if residual is None else _like(residual, x, shape, dev)
    kept_x = None if keep_x is None else _kept_like(keep_x, x, shape, dev)
    kept_y = None if keep_y is None else _kept_like(keep_y, x, shape, dev)
    if out is None:
        out = torch.empty_like(x)
        y = out.data_ptr() or None
    else:
        y = _like(out, x, shape, dev)
    stats = x.new_empty((rows, 2), dtype=torch.float32)
    status = (_LIB or load_library()).spconv_layer_norm_fwd(
        x.data_ptr() or None, res, w, b, eps, 1 if relu else 0, rows, channels, dt, y, stats.data_ptr() or None, kept_x, kept_y,
        _stream_here(dev))
    if status:
        _check(status, "spconv_layer_norm_fwd")
    return out, stats


def layer_norm_bwd(dout, x, stats, weight=None, gate=None, residual: bool = False, affine: bool = True, stream=None):
    """spconv_layer_norm_bwd: (dx, dweight, dbias, dresidual) for a layer_norm_fwd that left stats.  x: its input or the
    Checkpoint of it; gate: its output or the Checkpoint of it where it had a ReLU.  dweight and dbias are fp32 [channels]
    (None for affine=False), dresidual is None unless residual is set."""
    dt, shape, dev = _row_args(dout)
    if stream is not None or dev != _device_now():
        return _elsewhere(dev, stream, layer_norm_bwd, dout, x, stats, weight, gate, residual, affine)
    rows, channels = shape
    stats_ptr = _floats(stats, (rows, 2), dout, dev)
    w = None if weight is None else _floats(weight, (channels,), dout, dev)
    x_ptr = kept_x = y_ptr = kept_y = None
    if x is None:
        raise ValueError("x is the norm's input or its Checkpoint")
    if isinstance(x, Checkpoint):
        kept_x = _kept_like(x, dout, shape, dev)
    else:
        x_ptr = _like(x, dout, shape, dev)
    if isinstance(gate, Checkpoint):
        kept_y = _kept_like(gate, dout, shape, dev)
    elif gate is not None:
        y_ptr = _like(gate, dout, shape, dev)
    lib = _LIB or load_library()
    dx = torch.empty_like(dout)
    dres = torch.empty_like(dout) if residual else None
    dweight = dbias = dw_ptr = db_ptr = ws_ptr = None
    need = 0
    if affine:
        need = lib.spconv_layer_norm_bwd_workspace(rows, channels)
        if need < 0:
            _check(need, "spconv_layer_norm_bwd_workspace")
        dweight = stats.new_empty((channels,))
        dbias = stats.new_empty((channels,))
        dw_ptr, db_ptr = dweight.data_ptr(), dbias.data_ptr()
        if need:
            workspace = stats.new_empty((need // 4,))
            ws_ptr = workspace.data_ptr()
    status = lib.spconv_layer_norm_bwd(dout.data_ptr() or None, x_ptr, kept_x, y_ptr, kept_y, w, stats_ptr, rows, channels, dt,
                                       dx.data_ptr() or None, None if dres is None else dres.data_ptr() or None, dw_ptr, db_ptr,
                                       ws_ptr, need, _stream_here(dev))
    if status:
        _check(status, "spconv_layer_norm_bwd")
    return dx, dweight, dbias, dres
