"""ctypes binding of libfbsr.so (see include/fbsr.h for the contract of each call).

Argument marshalling only.  Tensors must live on a CUDA device (except for
``fbsr_round_host``), be contiguous and have the dtype the C signature implies;
output tensors are allocated with torch when not supplied.  Calls are enqueued on
torch's current stream of the tensors' device.
"""
import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libfbsr.so")

FMT = {"bf16": 0, "fp16": 1, "e4m3": 2, "e5m2": 3, "b8p4": 4}
FP32 = 0x20               # FBSR_FP32: names binary32 where a source may have several types
OVF_IEEE = 0x100          # or into a format id, or append "+ieee" to a format name: IEEE overflow instead of saturation
VARIANT = {"srff": 0, "srf": 1, "src": 2, "rtne": 3, "rta": 4, "rto": 5}
CODE_DTYPE = {"bf16": torch.uint16, "fp16": torch.uint16, "e4m3": torch.uint8, "e5m2": torch.uint8, "b8p4": torch.uint8}
VIEW_DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn,    # b8p4: torch has no such dtype
              "e5m2": torch.float8_e5m2}


class FbsrError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (what, fbsr_status_string(status), status))


class FbsrStats(ctypes.Structure):
    _fields_ = [("n_finite", ctypes.c_uint64), ("n_up", ctypes.c_uint64), ("n_nan", ctypes.c_uint64),
                ("n_inf", ctypes.c_uint64), ("n_sat", ctypes.c_uint64), ("sum_e", ctypes.c_double),
                ("sum_e2", ctypes.c_double), ("sum_signed_e", ctypes.c_double), ("sum_abs_e", ctypes.c_double)]


class FbsrFormatDesc(ctypes.Structure):
    """fbsr_format_desc of include/fbsr.h: a format (K, P, B; M) given at run time."""
    _fields_ = [("K", ctypes.c_int32), ("P", ctypes.c_int32), ("B", ctypes.c_int32), ("max_code", ctypes.c_uint32),
                ("has_inf", ctypes.c_int32), ("inf_code", ctypes.c_uint32), ("nan_code", ctypes.c_uint32),
                ("single_zero", ctypes.c_int32)]


class FbsrAdamwTensor(ctypes.Structure):
    """fbsr_adamw_tensor of include/fbsr.h."""
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("w_lp", ctypes.c_void_p),
                ("n", ctypes.c_uint64), ("offset", ctypes.c_uint64)]


def format_desc(K, P, B, max_code, inf_code=None, nan_code=0, single_zero=False):
    """Fill in an FbsrFormatDesc; inf_code=None means that the format has no infinity."""
    return FbsrFormatDesc(K, P, B, max_code, 0 if inf_code is None else 1, 0 if inf_code is None else inf_code,
                          nan_code, 1 if single_zero else 0)


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError("libfbsr.so is not built: run `python -m paper_2504_20634_b200.build` "
                          "(there is no fallback implementation)")
    L = ctypes.CDLL(_LIB_PATH)
    vp, sz, i, u64, f = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint64, ctypes.c_float
    d = ctypes.c_double
    L.fbsr_round.argtypes = [vp, vp, sz, i, i, i, u64, u64, f, vp]
    L.fbsr_round_bits.argtypes = [vp, vp, sz, i, i, i, vp, f, vp]
    L.fbsr_round_mx.argtypes = [vp, vp, vp, sz, i, i, i, u64, u64, vp]
    L.fbsr_round_mx.restype = i
    L.fbsr_round_lp.argtypes = [vp, i, vp, sz, i, i, i, u64, u64, f, vp]
    L.fbsr_round_lp.restype = i
    L.fbsr_round_desc.argtypes = [vp, vp, sz, ctypes.POINTER(FbsrFormatDesc), i, i, i, u64, u64, f, vp]
    L.fbsr_round_desc.restype = i
    L.fbsr_format_desc_valid.argtypes = [ctypes.POINTER(FbsrFormatDesc)]
    L.fbsr_format_desc_valid.restype = i
    L.fbsr_stats_workspace_bytes.argtypes = []
    L.fbsr_stats_workspace_bytes.restype = sz
    L.fbsr_round_stats.argtypes = [vp, vp, sz, i, i, i, u64, u64, f, sz, vp, vp, vp, vp, sz, vp]
    L.fbsr_round_stats_noalloc.argtypes = [vp, vp, sz, i, i, i, u64, u64, f, sz, vp, vp, vp, vp]
    L.fbsr_round_stats_noalloc.restype = i
    L.fbsr_sgd_update.argtypes = [vp, vp, vp, vp, sz, i, i, i, u64, u64, f, f, vp]
    L.fbsr_adam_update.argtypes = [vp, vp, vp, vp, vp, sz, i, i, i, u64, u64, f, f, f, f, i, vp]
    L.fbsr_accumulate.argtypes = [vp, vp, sz, i, i, i, u64, u64, vp]
    L.fbsr_qat_update.argtypes = [vp, vp, sz, i, i, i, i, u64, u64, vp]
    L.fbsr_qat_update.restype = i
    L.fbsr_qat_adamw_step.argtypes = [vp, vp, vp, vp, sz, i, i, i, i, u64, u64, f, f, f, f, f, i, vp]
    L.fbsr_qat_adamw_step.restype = i
    L.fbsr_adamw_multi.argtypes = [ctypes.POINTER(FbsrAdamwTensor), sz, i, i, i, i, i, u64, d, d, d, d, d, i, vp, vp]
    L.fbsr_adamw_multi.restype = i
    i64 = ctypes.c_int64
    L.fbsr_w4_padded.argtypes = [sz]
    L.fbsr_w4_padded.restype = sz
    L.fbsr_round_w4.argtypes = [vp, i, i64, sz, sz, vp, vp, i, i, vp, i64, i, i, u64, u64, vp]
    L.fbsr_round_w4.restype = i
    L.fbsr_gemv_w4.argtypes = [vp, i, i64, sz, vp, vp, i, i, sz, sz, vp, i, i64, vp]
    L.fbsr_gemv_w4.restype = i
    L.fbsr_round_host_min_workspace.argtypes = []
    L.fbsr_round_host_min_workspace.restype = sz
    L.fbsr_round_host.argtypes = [vp, vp, sz, i, i, i, u64, u64, f, vp, sz, vp]
    L.fbsr_adam_scalars.argtypes = [f, f, f, i, ctypes.POINTER(ctypes.c_float)]
    L.fbsr_adam_scalars.restype = None
    L.fbsr_tile_elements.argtypes = [i]
    L.fbsr_tile_elements.restype = sz
    L.fbsr_launch_count.argtypes = []
    L.fbsr_launch_count.restype = u64
    L.fbsr_status_string.argtypes = [i]
    L.fbsr_status_string.restype = ctypes.c_char_p
    L.fbsr_version.argtypes = []
    L.fbsr_version.restype = i
    for name in ("fbsr_round", "fbsr_round_bits", "fbsr_round_stats", "fbsr_sgd_update", "fbsr_adam_update",
                 "fbsr_accumulate", "fbsr_round_host"):
        getattr(L, name).restype = i
    return L


_L = _load()


def library_path():
    return _LIB_PATH


def fbsr_status_string(status):
    return _L.fbsr_status_string(int(status)).decode()


def fbsr_version():
    return int(_L.fbsr_version())


def fbsr_tile_elements(k_bits):
    return int(_L.fbsr_tile_elements(int(k_bits)))


def fbsr_adam_scalars(lr, beta1, beta2, step):
    """(c1, c2, a1, a2) of fbsr_adam_update / fbsr_qat_adamw_step as binary32 values (host only)."""
    out = (ctypes.c_float * 4)()
    _L.fbsr_adam_scalars(lr, beta1, beta2, step, out)
    return tuple(float(x) for x in out)


def fbsr_launch_count():
    return int(_L.fbsr_launch_count())


def fbsr_stats_workspace_bytes():
    return int(_L.fbsr_stats_workspace_bytes())


def fbsr_round_host_min_workspace():
    return int(_L.fbsr_round_host_min_workspace())


def _fmt(fmt):
    if isinstance(fmt, int):
        return fmt
    return FMT[fmt[:-5]] | OVF_IEEE if fmt.endswith("+ieee") else FMT[fmt]


def _fmt_name(fmt):
    # unknown integers fall through to the library, which rejects them with a status code
    if isinstance(fmt, str):
        return fmt[:-5] if fmt.endswith("+ieee") else fmt
    return {v: k for k, v in FMT.items()}.get(fmt & ~OVF_IEEE, "bf16")


def _var(variant):
    return variant if isinstance(variant, int) else VARIANT[variant]


def _dev(t, dtype, what):
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise TypeError("%s must be a contiguous CUDA tensor of dtype %s" % (what, dtype))
    return ctypes.c_void_p(t.data_ptr())


def _stream(t):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def _check(status, what):
    if status != 0:
        raise FbsrError(status, what)


def _out(src, fmt, out):
    dt = CODE_DTYPE[_fmt_name(fmt)]
    if out is None:
        out = torch.empty(src.numel(), dtype=dt, device=src.device)
    return out, _dev(out, dt, "out")


def fbsr_round(src, fmt, variant, k_bits, seed, offset=0, scale=1.0, out=None):
    """dst = FBSR(fl32(src * scale)); returns the tensor of codes (uint16 / uint8)."""
    out, po = _out(src, fmt, out)
    with torch.cuda.device(src.device):
        _check(_L.fbsr_round(_dev(src, torch.float32, "src"), po, src.numel(), _fmt(fmt), _var(variant), k_bits,
                             seed, offset, scale, _stream(src)), "fbsr_round")
    return out


def fbsr_round_mx(src, fmt, variant, k_bits, seed, offset=0, out=None, scales=None):
    """Block-scaled rounding (blocks of 32 elements, shared power-of-two scale); returns (codes, scale bytes)."""
    out, po = _out(src, fmt, out)
    if scales is None:
        scales = torch.empty((src.numel() + 31) // 32, dtype=torch.uint8, device=src.device)
    with torch.cuda.device(src.device):
        _check(_L.fbsr_round_mx(_dev(src, torch.float32, "src"), po, _dev(scales, torch.uint8, "scales"), src.numel(),
                                _fmt(fmt), _var(variant), k_bits, seed, offset, _stream(src)), "fbsr_round_mx")
    return out, scales


def fbsr_round_desc(src, desc, variant, k_bits, seed, offset=0, scale=1.0, ovf_ieee=False, out=None):
    """fbsr_round for a format described at run time (an FbsrFormatDesc); returns uint8 or uint16 codes."""
    dt = torch.uint16 if desc.K == 16 else torch.uint8
    if out is None:
        out = torch.empty(src.numel(), dtype=dt, device=src.device)
    with torch.cuda.device(src.device):
        _check(_L.fbsr_round_desc(_dev(src, torch.float32, "src"), _dev(out, dt, "out"), src.numel(), ctypes.byref(desc),
                                  1 if ovf_ieee else 0, _var(variant), k_bits, seed, offset, scale, _stream(src)),
               "fbsr_round_desc")
    return out


def fbsr_format_desc_valid(desc):
    return bool(_L.fbsr_format_desc_valid(ctypes.byref(desc)))


def fbsr_round_lp(src_codes, src_fmt, fmt, variant, k_bits, seed, offset=0, scale=1.0, out=None):
    """Round a tensor of bf16/fp16 codes (uint16) to an 8-bit format; returns the uint8 codes."""
    out, po = _out(src_codes, fmt, out)
    with torch.cuda.device(src_codes.device):
        _check(_L.fbsr_round_lp(_dev(src_codes, torch.uint16, "src_codes"), _fmt(src_fmt), po, src_codes.numel(),
                                _fmt(fmt), _var(variant), k_bits, seed, offset, scale, _stream(src_codes)),
               "fbsr_round_lp")
    return out


def fbsr_round_bits(src, fmt, variant, k_bits, rand_words, scale=1.0, out=None):
    out, po = _out(src, fmt, out)
    with torch.cuda.device(src.device):
        _check(_L.fbsr_round_bits(_dev(src, torch.float32, "src"), po, src.numel(), _fmt(fmt), _var(variant),
                                  k_bits, _dev(rand_words, torch.uint32, "rand_words"), scale, _stream(src)),
               "fbsr_round_bits")
    return out


def fbsr_round_stats(src, fmt, variant, k_bits, seed, offset=0, scale=1.0, group_size=0, out=None,
                     workspace=None, total=None, read_back=True):
    """Returns (codes, stats dict, group_sum_e, group_sum_e2); the stats dict is read back with one
    device-to-host copy after the call.  With read_back=False nothing is copied or synchronised and the
    second item is the 72-byte device tensor holding the fbsr_stats record (decode it with
    stats_from_bytes once the stream has been synchronised); `total` and `workspace` may be supplied so
    that repeated calls allocate nothing."""
    out, po = _out(src, fmt, out)
    n = src.numel()
    groups = (n + group_size - 1) // group_size if group_size else 0
    ge = torch.empty(max(groups, 1), dtype=torch.float64, device=src.device) if groups or read_back else None
    ge2 = torch.empty(max(groups, 1), dtype=torch.float64, device=src.device) if groups or read_back else None
    if total is None:
        total = torch.empty(ctypes.sizeof(FbsrStats), dtype=torch.uint8, device=src.device)
    if workspace is None:
        workspace = torch.empty(fbsr_stats_workspace_bytes(), dtype=torch.uint8, device=src.device)
    with torch.cuda.device(src.device):
        _check(_L.fbsr_round_stats(_dev(src, torch.float32, "src"), po, n, _fmt(fmt), _var(variant), k_bits, seed,
                                   offset, scale, group_size, ctypes.c_void_p(ge.data_ptr()) if ge is not None else None,
                                   ctypes.c_void_p(ge2.data_ptr()) if ge2 is not None else None,
                                   ctypes.c_void_p(total.data_ptr()),
                                   ctypes.c_void_p(workspace.data_ptr()), workspace.numel(), _stream(src)),
               "fbsr_round_stats")
    if not read_back:
        return out, total, (ge[:groups] if ge is not None else None), (ge2[:groups] if ge2 is not None else None)
    st = FbsrStats.from_buffer_copy(total.cpu().numpy().tobytes())
    return out, {name: getattr(st, name) for name, _ in FbsrStats._fields_}, ge[:groups], ge2[:groups]


def fbsr_round_stats_noalloc(src, out, total, fmt, variant, k_bits, seed, offset=0, scale=1.0, group_size=0,
                             group_sum_e=None, group_sum_e2=None):
    """fbsr_round_stats for callers that cannot allocate: every buffer (codes `out`, the 72-byte
    `total`, the optional group arrays) is supplied by the caller and the library's own built-in
    scratch is used, so neither this wrapper nor the C call allocates anything.  Returns None;
    read `total` (uint8[72], layout of FbsrStats) after synchronising the stream."""
    pe = ctypes.c_void_p(group_sum_e.data_ptr()) if group_sum_e is not None else None
    pe2 = ctypes.c_void_p(group_sum_e2.data_ptr()) if group_sum_e2 is not None else None
    with torch.cuda.device(src.device):
        _check(_L.fbsr_round_stats_noalloc(_dev(src, torch.float32, "src"),
                                           _dev(out, CODE_DTYPE[_fmt_name(fmt)], "out"), src.numel(), _fmt(fmt),
                                           _var(variant), k_bits, seed, offset, scale, group_size, pe, pe2,
                                           _dev(total, torch.uint8, "total"), _stream(src)),
               "fbsr_round_stats_noalloc")


def stats_from_bytes(total):
    """Decode a 72-byte device or host uint8 tensor holding an fbsr_stats record."""
    st = FbsrStats.from_buffer_copy(total.cpu().numpy().tobytes())
    return {name: getattr(st, name) for name, _ in FbsrStats._fields_}


def fbsr_sgd_update(master_w, grad, momentum, fmt, variant, k_bits, seed, offset, lr, mu, out=None):
    out, po = _out(master_w, fmt, out)
    f32 = torch.float32
    with torch.cuda.device(master_w.device):
        _check(_L.fbsr_sgd_update(_dev(master_w, f32, "master_w"), _dev(grad, f32, "grad"),
                                  _dev(momentum, f32, "momentum"), po, master_w.numel(), _fmt(fmt), _var(variant),
                                  k_bits, seed, offset, lr, mu, _stream(master_w)), "fbsr_sgd_update")
    return out


def fbsr_adam_update(master_w, grad, m, v, fmt, variant, k_bits, seed, offset, lr, beta1, beta2, eps, step,
                     out=None):
    out, po = _out(master_w, fmt, out)
    f32 = torch.float32
    with torch.cuda.device(master_w.device):
        _check(_L.fbsr_adam_update(_dev(master_w, f32, "master_w"), _dev(grad, f32, "grad"), _dev(m, f32, "m"),
                                   _dev(v, f32, "v"), po, master_w.numel(), _fmt(fmt), _var(variant), k_bits, seed,
                                   offset, lr, beta1, beta2, eps, step, _stream(master_w)), "fbsr_adam_update")
    return out


def fbsr_accumulate(w_lp, update, fmt, variant, k_bits, seed, offset=0):
    """In place on w_lp (tensor of codes)."""
    with torch.cuda.device(w_lp.device):
        _check(_L.fbsr_accumulate(_dev(w_lp, CODE_DTYPE[_fmt_name(fmt)], "w_lp"), _dev(update, torch.float32, "update"),
                                  w_lp.numel(), _fmt(fmt), _var(variant), k_bits, seed, offset, _stream(w_lp)),
               "fbsr_accumulate")
    return w_lp


def fbsr_qat_update(w8, update16, w_fmt, u_fmt, variant, k_bits, seed, offset=0):
    """In place on w8 (uint8 codes): w8 <- FBSR(RTNE_16(value(w8) + value(update16)))."""
    with torch.cuda.device(w8.device):
        _check(_L.fbsr_qat_update(_dev(w8, torch.uint8, "w8"), _dev(update16, torch.uint16, "update16"), w8.numel(),
                                  _fmt(w_fmt), _fmt(u_fmt), _var(variant), k_bits, seed, offset, _stream(w8)),
               "fbsr_qat_update")
    return w8


def fbsr_qat_adamw_step(w8, grad16, m, v, w_fmt, g_fmt, variant, k_bits, seed, offset, lr, beta1, beta2, eps,
                        weight_decay, step):
    """One iteration of Algorithm 1, in place on w8 (uint8 codes), m and v (float32); grad16 holds g_fmt codes."""
    with torch.cuda.device(w8.device):
        _check(_L.fbsr_qat_adamw_step(_dev(w8, torch.uint8, "w8"), _dev(grad16, torch.uint16, "grad16"),
                                      _dev(m, torch.float32, "m"), _dev(v, torch.float32, "v"), w8.numel(), _fmt(w_fmt),
                                      _fmt(g_fmt), _var(variant), k_bits, seed, offset, lr, beta1, beta2, eps, weight_decay,
                                      step, _stream(w8)), "fbsr_qat_adamw_step")
    return w8


ADAMW_BLOCK = 256         # elements that share a scale of the 8-bit state
SOURCE_TYPE = {torch.float32: FP32, torch.bfloat16: FMT["bf16"], torch.float16: FMT["fp16"]}


class FbsrAdamwTensors:
    """The tensors of one fbsr_adamw_multi call: lists of equal length, one entry per tensor.

    w: float32 masters; g: gradients, all float32, all bfloat16 or all float16; m, v: float32 moments, or 8-bit codes
    (uint8 or float8_e4m3fn) with m_scale, v_scale (float32, one per 256 elements); lp: the low-precision copies (codes
    of `fmt`, or a tensor of the torch dtype of that format), with None for tensors that have none, or None for all.
    offsets: the tensors' places in the stream of random draws, multiples of 256; by default each tensor starts at the
    next multiple of 256 after the previous one.  What a step writes must lie apart.  Holds references to the tensors;
    set_grads() exchanges the gradients."""

    def __init__(self, w, g, m, v, lp=None, fmt="bf16", m_scale=None, v_scale=None, offsets=None):
        count = len(w)
        if offsets is None:
            offsets, at = [], 0
            for t in w:
                offsets.append(at)
                at += -(-t.numel() // ADAMW_BLOCK) * ADAMW_BLOCK
        if lp is None:
            lp = [None] * count
        if (m_scale is None) != (v_scale is None):
            raise ValueError("m_scale and v_scale belong together")
        self.state_bits = 32 if m_scale is None else 8
        if m_scale is None:
            m_scale = v_scale = [None] * count
        for what, x in (("g", g), ("m", m), ("v", v), ("lp", lp), ("m_scale", m_scale), ("v_scale", v_scale), ("offsets", offsets)):
            if len(x) != count:
                raise ValueError("%s has %d entries for %d tensors" % (what, len(x), count))
        self.fmt, self.device = fmt, w[0].device if count else None
        self._ordinal = w[0].get_device() if count else -1
        self.array = (FbsrAdamwTensor * max(count, 1))()
        self.count = count
        self._w, self._state, self._lp = list(w), (list(m), list(v), list(m_scale), list(v_scale)), list(lp)
        state = (torch.float32,) if self.state_bits == 32 else (torch.uint8, torch.float8_e4m3fn)
        code = (CODE_DTYPE[_fmt_name(fmt)],) + ((VIEW_DTYPE[_fmt_name(fmt)],) if _fmt_name(fmt) in VIEW_DTYPE else ())
        state_bytes, code_bytes = self.state_bits // 8, code[0].itemsize
        spans = []                                   # (first byte, last byte + 1) of what a step writes
        for i in range(count):
            n, d = w[i].numel(), self.array[i]
            blocks = -(-n // ADAMW_BLOCK)
            d.w = at = self._pointer(w[i], n, (torch.float32,), "w", i)
            spans.append((at, at + 4 * n))
            d.m = at = self._pointer(m[i], n, state, "m", i)
            spans.append((at, at + state_bytes * n))
            d.v = at = self._pointer(v[i], n, state, "v", i)
            spans.append((at, at + state_bytes * n))
            if self.state_bits == 8:
                d.m_scale = at = self._pointer(m_scale[i], blocks, (torch.float32,), "m_scale", i)
                spans.append((at, at + 4 * blocks))
                d.v_scale = at = self._pointer(v_scale[i], blocks, (torch.float32,), "v_scale", i)
                spans.append((at, at + 4 * blocks))
            if lp[i] is not None:
                d.w_lp = at = self._pointer(lp[i], n, code, "lp", i)
                spans.append((at, at + code_bytes * n))
            offset = int(offsets[i])
            if not 0 <= offset < 1 << 64:
                raise ValueError("offsets[%d] must be from 0 to 2^64 - 1" % i)
            d.n, d.offset = n, offset
        # a parameter listed twice would be stepped by two warps at once
        spans.sort()
        reach = 0
        for start, end in spans:
            if start < reach and start < end:
                raise ValueError("tensors that a step writes overlap, or one is listed twice")
            if end > reach:
                reach = end
        self.set_grads(g)

    def _pointer(self, t, n, dtypes, what, i):
        if not (t.dtype in dtypes and t.is_cuda and t.get_device() == self._ordinal and t.is_contiguous()):
            raise TypeError("%s[%d] must be a contiguous tensor of %s on %s" % (what, i, " or ".join(map(str, dtypes)), self.device))
        if t.numel() != n:
            raise ValueError("%s[%d] has %d elements, expected %d" % (what, i, t.numel(), n))
        return t.data_ptr()

    def set_grads(self, g):
        if len(g) != self.count:
            raise ValueError("g has %d entries for %d tensors" % (len(g), self.count))
        dtype = g[0].dtype if self.count else torch.float32
        if dtype not in SOURCE_TYPE:
            raise TypeError("gradients must be float32, bfloat16 or float16")
        pointers = [self._pointer(t, self._w[i].numel(), (dtype,), "g", i) for i, t in enumerate(g)]
        for d, p in zip(self.array, pointers):
            d.g = p
        self.g_fmt, self._g = SOURCE_TYPE[dtype], list(g)


def fbsr_adamw_multi(tensors, variant, k_bits, seed, lr, beta1, beta2, eps, weight_decay, step, grad_scale=None):
    """One AdamW step over all tensors of an FbsrAdamwTensors, in place.  grad_scale: a one-element float32 CUDA tensor."""
    if tensors.count == 0:
        return tensors
    gs = None
    if grad_scale is not None:
        if grad_scale.numel() != 1 or grad_scale.device != tensors.device:
            raise ValueError("grad_scale must be one element on %s" % tensors.device)
        gs = _dev(grad_scale, torch.float32, "grad_scale")
    device = tensors.device.index
    with _on(device):
        status = _L.fbsr_adamw_multi(tensors.array, tensors.count, tensors.state_bits, tensors.g_fmt, _fmt(tensors.fmt),
                                     _var(variant), k_bits, seed, lr, beta1, beta2, eps, weight_decay, step, gs, _raw_stream(device))
    if status:
        _check(status, "fbsr_adamw_multi")
    return tensors


W4_SCALE = {"e8m0": 0, "bf16": 1}                                 # FBSR_SCALE_*
W4_SCALE_DTYPE = {"e8m0": torch.uint8, "bf16": torch.bfloat16}


_SOURCES = (torch.float32, torch.bfloat16, torch.float16)
_HALF = (torch.bfloat16, torch.float16)
_OUT = (None,) + _SOURCES
_HERE_ALREADY = contextlib.nullcontext()
_raw_stream = torch._C._cuda_getCurrentRawStream


def _on(device):
    """A context with CUDA device `device` (an ordinal) current: nothing to do, and nothing spent, where it is already."""
    return _HERE_ALREADY if torch._C._cuda_getDevice() == device else torch.cuda.device(device)


def _matrix(t, dtypes, what):
    """(address, leading dimension) of a 2-D CUDA tensor whose rows are contiguous and apart: a row repeated or overlapped by
    the next (expand, unfold) has a stride below its length, and is not taken."""
    if t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda:
        raise TypeError("%s must be a 2-D CUDA tensor of %s" % (what, " or ".join(map(str, dtypes))))
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise TypeError("%s must have contiguous rows" % what)
    if rows <= 1:
        return t.data_ptr(), cols
    if ld < cols:
        raise TypeError("%s must have rows that do not overlap: they are %d elements apart and %d long" % (what, ld, cols))
    return t.data_ptr(), ld


def fbsr_w4_padded(cols):
    """Columns of a 4-bit row with its padding: cols rounded up to a multiple of 128."""
    return int(_L.fbsr_w4_padded(int(cols)))


def fbsr_round_w4(src, variant, k_bits, seed, offset=0, group=32, scale_fmt="e8m0", values=None, out=None, scales=None):
    """Round a matrix (float32, bfloat16 or float16; rows may be strided) to 4 bits with a scale per `group` elements of a
    row; returns (codes uint8 [rows, padded / 2], scales [rows, padded / group]).  `values`, if given, receives the
    values that the codes stand for (same shape and dtype as src, not overlapping it)."""
    ps, ld = _matrix(src, _SOURCES, "src")
    rows, cols = src.shape
    device, group, half_row = src.get_device(), int(group), (cols + 127) // 128 * 64
    if scale_fmt not in W4_SCALE:
        raise ValueError("scale_fmt must be one of %s" % sorted(W4_SCALE))
    scale_dtype, groups = W4_SCALE_DTYPE[scale_fmt], 2 * half_row // max(group, 1)
    if out is None:
        out = src.new_empty((rows, half_row), dtype=torch.uint8)
    elif out.dtype is not torch.uint8 or out.shape != (rows, half_row) or out.get_device() != device or not out.is_contiguous():
        raise ValueError("out must be a contiguous uint8 tensor of shape (%d, %d) on %s" % (rows, half_row, src.device))
    if scales is None:
        scales = src.new_empty((rows, groups), dtype=scale_dtype)
    elif scales.dtype is not scale_dtype or scales.shape != (rows, groups) or scales.get_device() != device or not scales.is_contiguous():
        raise ValueError("scales must be a contiguous %s tensor of shape (%d, %d) on %s" % (scale_dtype, rows, groups, src.device))
    pv, vld = None, 0
    if values is not None:
        if values.shape != src.shape or values.get_device() != device:
            raise ValueError("values must have the shape and device of src")
        pv, vld = _matrix(values, (src.dtype,), "values")
    with _on(device):
        status = _L.fbsr_round_w4(ps, SOURCE_TYPE[src.dtype], ld, rows, cols, out.data_ptr(), scales.data_ptr(), W4_SCALE[scale_fmt],
                                  group, pv, vld, _var(variant), k_bits, seed, offset, _raw_stream(device))
    if status:
        _check(status, "fbsr_round_w4")
    return out, scales


def fbsr_gemv_w4(x, codes, scales, group=32, out=None, out_dtype=None):
    """x W^T for rows x [m, k] (bfloat16 or float16; rows may be strided) and a 4-bit matrix W [n, k] as fbsr_round_w4 returns
    it.  The result [m, n] has out_dtype (float32, bfloat16 or float16; by default that of x).  A 1-D x gives a 1-D result."""
    if x.dim() == 1:
        if out is not None and out.dim() != 1:
            raise ValueError("out must have one dimension as x has")
        y = fbsr_gemv_w4(x[None], codes, scales, group, None if out is None else out[None], out_dtype)
        return y[0] if out is None else out
    px, ldx = _matrix(x, _HALF, "x")
    m, k = x.shape
    device, group, half_row = x.get_device(), int(group), (k + 127) // 128 * 64
    n = codes.shape[0]
    if codes.dtype is not torch.uint8 or codes.shape != (n, half_row) or codes.get_device() != device or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous uint8 tensor of shape (n, %d) on %s" % (half_row, x.device))
    scale_fmt = 0 if scales.dtype is torch.uint8 else 1
    if scale_fmt and scales.dtype is not torch.bfloat16:
        raise TypeError("scales must be uint8 or bfloat16")
    if scales.shape != (n, 2 * half_row // max(group, 1)) or scales.get_device() != device or not scales.is_contiguous():
        raise ValueError("scales must be a contiguous tensor of shape (%d, %d) on %s" % (n, 2 * half_row // max(group, 1), x.device))
    if out is None:
        if out_dtype not in _OUT:
            raise TypeError("out_dtype must be one of %s" % ", ".join(map(str, _SOURCES)))
        out = x.new_empty((m, n), dtype=out_dtype)
        py, ldy = out.data_ptr(), n
    else:
        if out.shape != (m, n) or out.get_device() != device or out_dtype not in (None, out.dtype):
            raise ValueError("out must have shape (%d, %d) on %s and the dtype asked for" % (m, n, x.device))
        py, ldy = _matrix(out, _SOURCES, "out")
    with _on(device):
        status = _L.fbsr_gemv_w4(px, SOURCE_TYPE[x.dtype], ldx, m, codes.data_ptr(), scales.data_ptr(), scale_fmt, group, n, k, py,
                                 SOURCE_TYPE[out.dtype], ldy, _raw_stream(device))
    if status:
        _check(status, "fbsr_gemv_w4")
    return out


def fbsr_round_host(src_host, dst_host, fmt, variant, k_bits, seed, offset, scale, workspace):
    """Host tensors in and out (pinned for overlap); `workspace` is a CUDA uint8 tensor used as staging.
    Enqueues on the current stream of the workspace's device; synchronise it before reading dst_host."""
    if src_host.is_cuda or dst_host.is_cuda or src_host.dtype != torch.float32 or not src_host.is_contiguous():
        raise TypeError("src_host/dst_host must be contiguous host tensors (float32 in)")
    if dst_host.dtype != CODE_DTYPE[_fmt_name(fmt)] or not dst_host.is_contiguous():
        raise TypeError("dst_host has the wrong dtype")
    with torch.cuda.device(workspace.device):
        _check(_L.fbsr_round_host(ctypes.c_void_p(src_host.data_ptr()), ctypes.c_void_p(dst_host.data_ptr()),
                                  src_host.numel(), _fmt(fmt), _var(variant), k_bits, seed, offset, scale,
                                  _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(workspace)),
               "fbsr_round_host")
    return dst_host
