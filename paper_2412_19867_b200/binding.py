"""Thin ctypes binding of the C ABI in ``include/wfq.h`` (argument marshalling only).

Every step of the computation runs in the CUDA kernels of ``libwfq.so``.  PyTorch is
used by callers for device memory and streams; this module only passes raw pointers.
If the library has not been built the import-time loader raises: there is no
fallback path.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwfq.so")

WFQ_OK, WFQ_ERR_INVALID_ARG, WFQ_ERR_UNSUPPORTED, WFQ_ERR_ALLOC = 0, 1, 2, 3
WFQ_ERR_NOT_PREPARED, WFQ_ERR_CUDA, WFQ_ERR_TIMEOUT, WFQ_ERR_SCRATCH_TOO_SMALL = 4, 5, 6, 7
WFQ_STATIC_SCRATCH_FLOATS = 4 * 1024 * 1024
WFQ_F32, WFQ_F16, WFQ_BF16 = 0, 1, 2
WFQ_ACT_NONE, WFQ_ACT_RELU, WFQ_ACT_SILU, WFQ_ACT_GELU = 0, 1, 2, 3
WFQ_Y_FP32, WFQ_Y_TILE, WFQ_Y_ROW = 0, 1, 2
WFQ_NCHW, WFQ_NHWC = 0, 1
WFQ_BUF_XQ, WFQ_BUF_SX, WFQ_BUF_WQ, WFQ_BUF_SW, WFQ_BUF_Y, WFQ_BUF_STATUS = range(6)
WFQ_DEBUG_WAIT_CYCLES, WFQ_DEBUG_SKIP_INPUT_ITEM, WFQ_DEBUG_INPUT_TRANSFORM_KERNEL = range(3)
WFQ_DEBUG_SKIP_GEMM_STAGE = 3
WFQ_DEBUG_GEMM_SHAPE, WFQ_DEBUG_GEMM_CTAS = 4, 5

# every symbol include/wfq.h declares
EXPORTS = [
    "wfq_plan_create", "wfq_plan_set_input_dtype", "wfq_plan_workspace_bytes",
    "wfq_plan_set_workspace", "wfq_prepare_filters", "wfq_conv_forward",
    "wfq_conv_forward_host", "wfq_input_transform_quantize", "wfq_gemm_dequantize",
    "wfq_output_transform", "wfq_debug_gemm_acc32", "wfq_debug_get",
    "wfq_check_device_status", "wfq_plan_destroy", "wfq_status_string", "wfq_version",
    "wfq_quantize_filters_static", "wfq_plan_set_debug_option", "wfq_debug_int8_mma_rate",
    "wfq_plan_set_epilogue", "wfq_plan_set_full_quant", "wfq_plan_set_output_dtype", "wfq_plan_set_weight_bits",
    "wfq_conv_forward_host_async", "wfq_filters_bytes", "wfq_filters_export", "wfq_filters_import",
    "wfq_plan_set_input_layout",
    "wfq_rms_norm_quantize", "wfq_quantize_rows", "wfq_dequantize_rows",
    "wfq_linear_create", "wfq_linear_set_input_dtype", "wfq_linear_set_output_dtype", "wfq_linear_set_epilogue",
    "wfq_linear_workspace_bytes", "wfq_linear_set_workspace", "wfq_linear_prepare_weights", "wfq_linear_forward",
    "wfq_linear_forward_codes", "wfq_linear_set_debug_option", "wfq_linear_check_status", "wfq_linear_debug_get",
    "wfq_linear_destroy",
]

_lib = None


class WfqError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


def load():
    """Load libwfq.so and declare the prototypes.  Raises if the library is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2412_19867_b200.build` (no CPU fallback exists)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.wfq_plan_create.argtypes = [ctypes.POINTER(vp)] + [ci] * 9
    lib.wfq_plan_set_input_dtype.argtypes = [vp, ci]
    lib.wfq_plan_workspace_bytes.argtypes = [vp]
    lib.wfq_plan_workspace_bytes.restype = sz
    lib.wfq_plan_set_workspace.argtypes = [vp, vp, sz]
    lib.wfq_prepare_filters.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.wfq_conv_forward.argtypes = [vp, vp, vp, vp]
    lib.wfq_conv_forward_host.argtypes = [vp, vp, vp, vp]
    lib.wfq_conv_forward_host_async.argtypes = [vp, vp, vp, vp]
    lib.wfq_filters_bytes.argtypes = [vp]
    lib.wfq_filters_bytes.restype = ctypes.c_size_t
    lib.wfq_filters_export.argtypes = [vp, vp, ctypes.c_size_t, vp]
    lib.wfq_filters_import.argtypes = [vp, vp, ctypes.c_size_t, vp]
    lib.wfq_input_transform_quantize.argtypes = [vp, vp, vp]
    lib.wfq_gemm_dequantize.argtypes = [vp, vp]
    lib.wfq_output_transform.argtypes = [vp, vp, vp]
    lib.wfq_debug_gemm_acc32.argtypes = [vp, vp, vp]
    lib.wfq_debug_get.argtypes = [vp, ci, ctypes.POINTER(vp), ctypes.POINTER(sz)]
    lib.wfq_check_device_status.argtypes = [vp, vp, ctypes.POINTER(ci)]
    lib.wfq_plan_destroy.argtypes = [vp]
    lib.wfq_quantize_filters_static.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp]
    lib.wfq_plan_set_epilogue.argtypes = [vp, vp, ci]
    lib.wfq_plan_set_full_quant.argtypes = [vp, ci, ci]
    lib.wfq_plan_set_output_dtype.argtypes = [vp, ci]
    lib.wfq_plan_set_weight_bits.argtypes = [vp, ci]
    lib.wfq_plan_set_input_layout.argtypes = [vp, ci]
    lib.wfq_plan_set_debug_option.argtypes = [vp, ci, ctypes.c_longlong]
    lib.wfq_debug_int8_mma_rate.argtypes = [vp, ci, ci, ctypes.POINTER(ctypes.c_longlong), vp]
    ll = ctypes.c_longlong
    lib.wfq_rms_norm_quantize.argtypes = [vp, ll, vp, ll, vp, ctypes.c_float, ci, ci, ci, ci, vp, ll, vp, vp, vp]
    lib.wfq_quantize_rows.argtypes = [vp, ll, ci, ci, ci, ci, vp, vp, vp]
    lib.wfq_dequantize_rows.argtypes = [vp, vp, ci, ci, ci, ci, vp, ll, vp]
    lib.wfq_linear_create.argtypes = [ctypes.POINTER(vp), ci, ci, ci, ci]
    lib.wfq_linear_set_input_dtype.argtypes = [vp, ci]
    lib.wfq_linear_set_output_dtype.argtypes = [vp, ci]
    lib.wfq_linear_set_epilogue.argtypes = [vp, vp, ci]
    lib.wfq_linear_workspace_bytes.argtypes = [vp, ci]
    lib.wfq_linear_workspace_bytes.restype = sz
    lib.wfq_linear_set_workspace.argtypes = [vp, vp, sz, ci]
    lib.wfq_linear_prepare_weights.argtypes = [vp, vp, ll, ci, vp]
    lib.wfq_linear_forward.argtypes = [vp, vp, ll, ci, vp, ll, vp, ll, vp]
    lib.wfq_linear_forward_codes.argtypes = [vp, vp, vp, ci, vp, ll, vp, ll, vp]
    lib.wfq_linear_set_debug_option.argtypes = [vp, ci, ll]
    lib.wfq_linear_check_status.argtypes = [vp, vp, ctypes.POINTER(ci)]
    lib.wfq_linear_debug_get.argtypes = [vp, ci, ctypes.POINTER(vp), ctypes.POINTER(sz)]
    lib.wfq_linear_destroy.argtypes = [vp]
    lib.wfq_status_string.argtypes = [ci]
    lib.wfq_status_string.restype = ctypes.c_char_p
    lib.wfq_version.restype = ci
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is ctypes.c_int and name not in ("wfq_version",):
            fn.restype = ci
    _lib = lib
    return lib


def status_string(status):
    return load().wfq_status_string(int(status)).decode()


def _check(status, what):
    if status != WFQ_OK:
        raise WfqError(status, what)


def _host_floats(values):
    if values is None:
        return None, None
    arr = (ctypes.c_float * len(values))(*[float(v) for v in values])
    return arr, ctypes.cast(arr, ctypes.c_void_p)


# ---- the C calls, same names, raw pointers (ints) in and out ------------------------

def wfq_plan_create(N, C, K, H, W, m, r=3, group_size=64, bits=8):
    plan = ctypes.c_void_p()
    _check(load().wfq_plan_create(ctypes.byref(plan), N, C, K, H, W, m, r, group_size, bits),
           "wfq_plan_create")
    return plan


def wfq_plan_set_input_dtype(plan, dtype):
    _check(load().wfq_plan_set_input_dtype(plan, dtype), "wfq_plan_set_input_dtype")


def wfq_plan_set_epilogue(plan, bias_dev, act=WFQ_ACT_NONE):
    _check(load().wfq_plan_set_epilogue(plan, bias_dev, act), "wfq_plan_set_epilogue")


def wfq_plan_set_input_layout(plan, layout):
    _check(load().wfq_plan_set_input_layout(plan, layout), "wfq_plan_set_input_layout")


def wfq_plan_set_weight_bits(plan, bits):
    _check(load().wfq_plan_set_weight_bits(plan, bits), "wfq_plan_set_weight_bits")


def wfq_plan_set_output_dtype(plan, dtype):
    _check(load().wfq_plan_set_output_dtype(plan, dtype), "wfq_plan_set_output_dtype")


def wfq_plan_set_full_quant(plan, quant_input, y_mode):
    _check(load().wfq_plan_set_full_quant(plan, int(quant_input), y_mode), "wfq_plan_set_full_quant")


def wfq_plan_workspace_bytes(plan):
    return int(load().wfq_plan_workspace_bytes(plan))


def wfq_plan_set_workspace(plan, dev_ptr, nbytes):
    _check(load().wfq_plan_set_workspace(plan, dev_ptr, nbytes), "wfq_plan_set_workspace")


def wfq_prepare_filters(plan, w_dev, sB=None, sG=None, sA=None, stream=0):
    kb, pb = _host_floats(sB)
    kg, pg = _host_floats(sG)
    ka, pa = _host_floats(sA)
    _check(load().wfq_prepare_filters(plan, w_dev, pb, pg, pa, stream), "wfq_prepare_filters")


def wfq_conv_forward(plan, x_dev, y_dev, stream=0):
    status = (_lib or load()).wfq_conv_forward(plan, x_dev, y_dev, stream)
    if status != WFQ_OK:
        _check(status, "wfq_conv_forward")


def wfq_conv_forward_host(plan, x_host, y_host, stream=0):
    _check(load().wfq_conv_forward_host(plan, x_host, y_host, stream), "wfq_conv_forward_host")


def wfq_filters_bytes(plan):
    return int(load().wfq_filters_bytes(plan))


def wfq_filters_export(plan, stream=0):
    """The prepared filters of the plan as a bytes-like host buffer (ctypes array)."""
    n = wfq_filters_bytes(plan)
    buf = (ctypes.c_char * n)()
    _check(load().wfq_filters_export(plan, ctypes.cast(buf, ctypes.c_void_p), n, stream), "wfq_filters_export")
    return buf


def wfq_filters_import(plan, blob, stream=0):
    raw = bytes(blob)
    _check(load().wfq_filters_import(plan, ctypes.cast(ctypes.c_char_p(raw), ctypes.c_void_p), len(raw), stream),
           "wfq_filters_import")


def wfq_conv_forward_host_async(plan, x_host, y_host, stream=0):
    _check(load().wfq_conv_forward_host_async(plan, x_host, y_host, stream), "wfq_conv_forward_host_async")


def wfq_input_transform_quantize(plan, x_dev, stream=0):
    _check(load().wfq_input_transform_quantize(plan, x_dev, stream), "wfq_input_transform_quantize")


def wfq_gemm_dequantize(plan, stream=0):
    _check(load().wfq_gemm_dequantize(plan, stream), "wfq_gemm_dequantize")


def wfq_output_transform(plan, y_dev, stream=0):
    _check(load().wfq_output_transform(plan, y_dev, stream), "wfq_output_transform")


def wfq_debug_gemm_acc32(plan, acc_dev, stream=0):
    _check(load().wfq_debug_gemm_acc32(plan, acc_dev, stream), "wfq_debug_gemm_acc32")


def wfq_debug_get(plan, which):
    ptr, nbytes = ctypes.c_void_p(), ctypes.c_size_t()
    _check(load().wfq_debug_get(plan, which, ctypes.byref(ptr), ctypes.byref(nbytes)), "wfq_debug_get")
    return ptr.value, nbytes.value


def wfq_check_device_status(plan, stream=0):
    where = ctypes.c_int(0)
    st = load().wfq_check_device_status(plan, stream, ctypes.byref(where))
    return st, where.value


def wfq_quantize_filters_static(w_dev, K, C, m, group_size, sG, wq_dev, sw_dev, stream=0):
    """Allocation-free filter quantization into caller-owned device buffers."""
    keep, pg = _host_floats(sG)
    _check(load().wfq_quantize_filters_static(w_dev, K, C, m, group_size, pg, wq_dev, sw_dev, stream),
           "wfq_quantize_filters_static")


def wfq_plan_set_debug_option(plan, option, value):
    _check(load().wfq_plan_set_debug_option(plan, option, value), "wfq_plan_set_debug_option")


def wfq_debug_int8_mma_rate(plan, n_cols, mmas_per_sm, stream=0):
    """Enqueues the tensor-pipe rate kernel; returns the integer operations it performs."""
    ops = ctypes.c_longlong(0)
    _check(load().wfq_debug_int8_mma_rate(plan, n_cols, mmas_per_sm, ctypes.byref(ops), stream),
           "wfq_debug_int8_mma_rate")
    return ops.value


def wfq_plan_destroy(plan):
    _check(load().wfq_plan_destroy(plan), "wfq_plan_destroy")


def _sizes(*sizes):
    """Refuses sizes that ctypes would cut to their low 32 bits."""
    for n in sizes:
        if not -2 ** 31 <= n < 2 ** 31:
            raise WfqError(WFQ_ERR_UNSUPPORTED, f"size {n}")


def wfq_rms_norm_quantize(x_dev, ldx, residual_dev, ldr, gain_dev, eps, dtype, rows, C, group_size, h_dev, ldh,
                          codes_dev, scales_dev, stream=0):
    _sizes(rows, C, group_size)
    status = (_lib or load()).wfq_rms_norm_quantize(x_dev, ldx, residual_dev, ldr, gain_dev, eps, dtype, rows, C,
                                                    group_size, h_dev, ldh, codes_dev, scales_dev, stream)
    if status != WFQ_OK:
        _check(status, "wfq_rms_norm_quantize")


def wfq_quantize_rows(x_dev, ldx, dtype, rows, C, group_size, codes_dev, scales_dev, stream=0):
    _sizes(rows, C, group_size)
    status = (_lib or load()).wfq_quantize_rows(x_dev, ldx, dtype, rows, C, group_size, codes_dev, scales_dev, stream)
    if status != WFQ_OK:
        _check(status, "wfq_quantize_rows")


def wfq_dequantize_rows(codes_dev, scales_dev, rows, C, group_size, dtype, v_dev, ldv, stream=0):
    _sizes(rows, C, group_size)
    status = (_lib or load()).wfq_dequantize_rows(codes_dev, scales_dev, rows, C, group_size, dtype, v_dev, ldv, stream)
    if status != WFQ_OK:
        _check(status, "wfq_dequantize_rows")


def wfq_linear_create(C, K, group_size, gated=0):
    _sizes(C, K, group_size)
    lin = ctypes.c_void_p()
    _check(load().wfq_linear_create(ctypes.byref(lin), C, K, group_size, int(gated)), "wfq_linear_create")
    return lin


def wfq_linear_set_input_dtype(lin, dtype):
    _check(load().wfq_linear_set_input_dtype(lin, dtype), "wfq_linear_set_input_dtype")


def wfq_linear_set_output_dtype(lin, dtype):
    _check(load().wfq_linear_set_output_dtype(lin, dtype), "wfq_linear_set_output_dtype")


def wfq_linear_set_epilogue(lin, bias_dev, act=WFQ_ACT_NONE):
    _check(load().wfq_linear_set_epilogue(lin, bias_dev, act), "wfq_linear_set_epilogue")


def wfq_linear_workspace_bytes(lin, rows):
    _sizes(rows)
    return int(load().wfq_linear_workspace_bytes(lin, rows))


def wfq_linear_set_workspace(lin, dev_ptr, nbytes, rows):
    _sizes(rows)
    _check(load().wfq_linear_set_workspace(lin, dev_ptr, nbytes, rows), "wfq_linear_set_workspace")


def wfq_linear_prepare_weights(lin, w_dev, ldw, dtype, stream=0):
    _check(load().wfq_linear_prepare_weights(lin, w_dev, ldw, dtype, stream), "wfq_linear_prepare_weights")


def wfq_linear_forward(lin, x_dev, ldx, rows, residual_dev, ldr, y_dev, ldy, stream=0):
    _sizes(rows)
    status = (_lib or load()).wfq_linear_forward(lin, x_dev, ldx, rows, residual_dev, ldr, y_dev, ldy, stream)
    if status != WFQ_OK:
        _check(status, "wfq_linear_forward")


def wfq_linear_forward_codes(lin, codes_dev, scales_dev, rows, residual_dev, ldr, y_dev, ldy, stream=0):
    _sizes(rows)
    status = (_lib or load()).wfq_linear_forward_codes(lin, codes_dev, scales_dev, rows, residual_dev, ldr, y_dev, ldy,
                                                       stream)
    if status != WFQ_OK:
        _check(status, "wfq_linear_forward_codes")


def wfq_linear_set_debug_option(lin, option, value):
    _check(load().wfq_linear_set_debug_option(lin, option, value), "wfq_linear_set_debug_option")


def wfq_linear_check_status(lin, stream=0):
    where = ctypes.c_int(0)
    st = load().wfq_linear_check_status(lin, stream, ctypes.byref(where))
    return st, where.value


def wfq_linear_debug_get(lin, which):
    ptr, nbytes = ctypes.c_void_p(), ctypes.c_size_t()
    _check(load().wfq_linear_debug_get(lin, which, ctypes.byref(ptr), ctypes.byref(nbytes)), "wfq_linear_debug_get")
    return ptr.value, nbytes.value


def wfq_linear_destroy(lin):
    _check(load().wfq_linear_destroy(lin), "wfq_linear_destroy")


# ---- convenience wrapper holding torch tensors for the device buffers ----------------

class _DevicePointer:
    """Exposes a raw device pointer through __cuda_array_interface__ (no copy)."""

    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr,
                                         "data": (int(ptr), False), "version": 2}


class Conv:
    """One layer: plan + workspace + prepared filters, driven with torch CUDA tensors."""

    def __init__(self, N, C, K, H, W, m, group_size, in_dtype="f16", device="cuda:0"):
        import torch
        self.torch = torch
        self.shape = (N, C, K, H, W)
        self._y_shape, self._y_stride = (N, K, H, W), (K * H * W, H * W, W, 1)
        self.m, self.gs = m, group_size
        self.device = torch.device(device)
        self.in_dtype = in_dtype
        self.in_layout, self.out_dtype = "nchw", "f32"
        self.plan = wfq_plan_create(N, C, K, H, W, m, 3, group_size, 8)
        wfq_plan_set_input_dtype(self.plan, WFQ_F16 if in_dtype == "f16" else WFQ_F32)
        nbytes = wfq_plan_workspace_bytes(self.plan)
        # torch's caching allocator returns 512-byte aligned blocks; over-allocate and
        # round the base up to the 1024-byte alignment the TMA tiles want
        self._ws = torch.empty(nbytes + 1024, dtype=torch.uint8, device=self.device)
        base = (self._ws.data_ptr() + 1023) // 1024 * 1024
        with torch.cuda.device(self.device):
            wfq_plan_set_workspace(self.plan, base, nbytes)
        n = m + 2
        self.P, self.G = n * n, C // group_size
        self.T = N * (-(-H // m)) * (-(-W // m))
        self.Tp = (self.T + 31) // 32 * 32
        self.Ts = (self.T + 127) // 128 * 128
        self.Kp = (K + 127) // 128 * 128

    def _stream(self):
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def prepare(self, w, sB=None, sG=None, sA=None):
        torch = self.torch
        assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous()
        with torch.cuda.device(self.device):
            wfq_prepare_filters(self.plan, w.data_ptr(), sB, sG, sA, self._stream())

    def set_input_layout(self, layout):
        """"nchw" (default) or "nhwc": forward() then takes x of shape (N, H, W, C)."""
        self.in_layout = layout
        wfq_plan_set_input_layout(self.plan, WFQ_NHWC if layout == "nhwc" else WFQ_NCHW)

    def set_weight_bits(self, bits):
        """8 (default) or 4; call before prepare()."""
        wfq_plan_set_weight_bits(self.plan, bits)

    def set_output_dtype(self, dtype):
        """"f32" (default), "f16" or "bf16": element type of the tensors forward() returns or fills."""
        self.out_dtype = dtype
        wfq_plan_set_output_dtype(self.plan, {"f32": WFQ_F32, "f16": WFQ_F16, "bf16": WFQ_BF16}[dtype])

    def set_epilogue(self, bias=None, act=WFQ_ACT_NONE):
        """bias: fp32 CUDA tensor [K] or None; kept alive by this object."""
        if bias is not None:
            assert bias.is_cuda and bias.dtype == self.torch.float32 and bias.is_contiguous()
            assert bias.numel() == self.shape[2]
        self._bias = bias
        wfq_plan_set_epilogue(self.plan, None if bias is None else bias.data_ptr(), act)

    def forward(self, x, y=None):
        # a small layer's kernels take less than this call: nothing here that is not needed per call
        torch = self.torch
        N, C, K, H, W = self.shape
        assert x.shape == ((N, H, W, C) if self.in_layout == "nhwc" else (N, C, H, W))
        assert x.is_cuda and x.is_contiguous()
        assert x.dtype is (torch.float16 if self.in_dtype == "f16" else torch.float32)
        out = self.out_dtype
        ydt = torch.float32 if out == "f32" else torch.float16 if out == "f16" else torch.bfloat16
        if y is None:
            # with its strides given, and the device looked up directly below: queued calls of a small layer take
            # 10.2 us, 11.2 us with torch.empty, 10.4 us with torch.cuda.current_device
            y = torch.empty_strided(self._y_shape, self._y_stride, dtype=ydt, device=self.device)
        else:
            assert y.dtype is ydt and y.is_contiguous() and y.shape == self._y_shape
        here, index = torch._C._cuda_getDevice(), self.device.index
        if index is None or index == here:
            wfq_conv_forward(self.plan, x.data_ptr(), y.data_ptr(), torch._C._cuda_getCurrentRawStream(here))
        else:
            with torch.cuda.device(self.device):
                wfq_conv_forward(self.plan, x.data_ptr(), y.data_ptr(), self._stream())
        return y

    def forward_host(self, x_host, y_host):
        """x_host / y_host: CPU tensors (pinned for speed); synchronous."""
        with self.torch.cuda.device(self.device):
            wfq_conv_forward_host(self.plan, x_host.data_ptr(), y_host.data_ptr(), self._stream())
        return y_host

    def forward_host_async(self, x_host, y_host, stream=None):
        """The same without the final wait; `stream`: a torch.cuda.Stream (default: the current
        one).  y_host is valid after that stream has been synchronised."""
        sptr = self._stream() if stream is None else stream.cuda_stream
        with self.torch.cuda.device(self.device):
            wfq_conv_forward_host_async(self.plan, x_host.data_ptr(), y_host.data_ptr(), sptr)
        return y_host

    def buffer(self, which):
        """A torch tensor aliasing an internal buffer, shaped per include/wfq.h."""
        torch = self.torch
        ptr, nbytes = wfq_debug_get(self.plan, which)
        N, C, K, H, W = self.shape
        shapes = {WFQ_BUF_XQ: ((self.P, self.T, C), "|i1", 1),
                  WFQ_BUF_SX: ((self.P, self.G, self.Ts), "<f4", 4),
                  WFQ_BUF_WQ: ((self.P, K, C), "|i1", 1),
                  WFQ_BUF_SW: ((self.P, self.G, self.Kp), "<f4", 4),
                  WFQ_BUF_Y: ((self.P, K, self.Tp), "<f4", 4),
                  WFQ_BUF_STATUS: ((4,), "<i4", 4)}
        shape, typestr, esz = shapes[which]
        count = 1
        for d in shape:
            count *= d
        assert count * esz == nbytes, (which, shape, nbytes)
        holder = _DevicePointer(ptr, shape, typestr)
        with torch.cuda.device(self.device):
            return torch.as_tensor(holder, device=self.device)

    def write_buffer(self, which, tensor):
        """Overwrite an internal buffer (feeding a later stage with chosen operands)."""
        dst = self.buffer(which)
        dst.copy_(tensor.to(self.device).reshape(dst.shape))
        self.torch.cuda.synchronize(self.device)

    def check_status(self):
        st, where = wfq_check_device_status(self.plan, self._stream())
        if st != WFQ_OK:
            raise WfqError(st, f"device status (wait id {where})")

    def close(self):
        if self.plan is not None:
            wfq_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- the operators around the convolutions --------------------------------------------
# A decoding step's kernels take less than these calls: nothing in them that is not needed per call (queued, one row of
# 4096: norm and dequantization 28 us with an import, a dict and two allocations more per call).

_DTYPES = {"f32": WFQ_F32, "f16": WFQ_F16, "bf16": WFQ_BF16}
_torch = None          # the module, and its types by the library's codes, once something here has been called
_CODES = {}
_NAMED = {}


def _load_torch():
    global _torch
    import torch
    _CODES.update({torch.float32: WFQ_F32, torch.float16: WFQ_F16, torch.bfloat16: WFQ_BF16})
    _NAMED.update({"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16})
    _torch = torch
    return torch


def _rows_of(x, C, what):
    """Rows and leading dimension of a tensor [..., C] whose rows lie one after another at one distance."""
    shape = x.shape
    assert x.is_cuda and shape and shape[-1] == C, what
    rows = x.numel() // C
    if rows >> 31:
        _sizes(rows)
    if x.is_contiguous() or rows == 0:
        return rows, C
    assert C == 1 or x.stride(-1) == 1, f"{what}: channels must be contiguous"
    ld, span = None, 1                   # distance between rows, rows that the dimensions behind this one hold
    for size, stride in zip(reversed(shape[:-1]), reversed(x.stride()[:-1])):
        if size != 1:
            if ld is None:
                ld = stride
            assert stride == ld * span, f"{what}: rows must lie at one distance from each other"
        span *= size
    ld = C if ld is None else ld
    assert rows == 1 or ld >= C, f"{what}: rows overlap"
    return rows, max(ld, C)


def _empty(shape, dtype, device):
    # with its strides given: a microsecond less than torch.empty
    if len(shape) == 2:
        return _torch.empty_strided(shape, (shape[1] or 1, 1), dtype=dtype, device=device)
    strides, n = [], 1
    for size in reversed(shape):
        strides.append(n)
        n *= size if size else 1
    return _torch.empty_strided(shape, strides[::-1], dtype=dtype, device=device)


def _call(index, fn, *args):
    """The library's fn(*args, stream) with device `index` current, on its current stream."""
    c = _torch._C
    if c._cuda_getDevice() == index:
        status = fn(*args, c._cuda_getCurrentRawStream(index))
    else:
        with _torch.cuda.device(index):
            status = fn(*args, c._cuda_getCurrentRawStream(index))
    if status != WFQ_OK:
        _check(status, fn.__name__)


class QuantizedRows:
    """int8 codes [rows][Cp] and fp32 scales [G][Rs] of rows of C channels (layouts: include/wfq.h) in one buffer."""
    __slots__ = ("rows", "C", "group_size", "shape", "groups", "index", "_buf", "_codes", "_scales", "_at")

    def __init__(self, rows, C, group_size, device, shape=None):
        if _torch is None:
            _load_torch()
        if (rows | C | group_size) >> 31:               # one of them is negative or does not fit
            _sizes(rows, C, group_size)
        self.rows, self.C, self.group_size = rows, C, group_size
        self.shape = (rows, C) if shape is None else shape
        self.groups = 1 if group_size == 0 or group_size >= C else -(-C // group_size)
        self._at = (rows * ((C + 31) // 32 * 32) + 255) // 256 * 256             # where the scales begin
        self._buf = _torch.empty_strided((self._at + 4 * self.groups * ((rows + 127) // 128 * 128),), (1,),
                                         dtype=_torch.int8, device=device)
        self._codes = self._buf.data_ptr()
        self._scales = self._codes + self._at
        self.index = self._buf.get_device()

    @property
    def codes(self):
        Cp = (self.C + 31) // 32 * 32
        return self._buf[:self.rows * Cp].view(self.rows, Cp)

    @property
    def scales(self):
        return self._buf[self._at:].view(_torch.float32).view(self.groups, (self.rows + 127) // 128 * 128)


def rms_norm_quantize(x, gain, eps=1e-6, group_size=128, residual=None, out=None):
    """Root-mean-square norm of the rows of x (+ residual) as (QuantizedRows, h).

    x, residual: CUDA tensors [..., C] of one type (fp32, fp16, bf16); gain: fp32 [C].  h is the sum in x's type, written
    to `out` where given (x or residual itself, or memory that overlaps neither); without a residual it is x."""
    torch = _torch or _load_torch()
    C, dtype = gain.numel(), x.dtype
    code, index = _CODES.get(dtype), x.get_device()
    assert code is not None, "x: fp32, fp16 or bf16"
    assert gain.dtype is torch.float32 and gain.get_device() == index and gain.is_contiguous(), "gain"
    rows, ldx = _rows_of(x, C, "x")
    shape, device = x.shape, x.device
    q = QuantizedRows(rows, C, group_size, device, shape)
    if residual is None:
        assert out is None, "out: only with a residual"
        _call(index, (_lib or load()).wfq_rms_norm_quantize, x.data_ptr(), ldx, None, 0, gain.data_ptr(), eps, code, rows, C, group_size,
              None, 0, q._codes, q._scales)
        return q, x
    assert residual.shape == shape and residual.dtype is dtype and residual.get_device() == index, "residual"
    _, ldr = _rows_of(residual, C, "residual")
    if out is None:
        h, ldh = torch.empty_like(x) if ldx == C and x.is_contiguous() else _empty(shape, dtype, device), C
    else:
        h = out
        assert h.shape == shape and h.dtype is dtype and h.get_device() == index, "out"
        _, ldh = _rows_of(h, C, "out")
    _call(index, (_lib or load()).wfq_rms_norm_quantize, x.data_ptr(), ldx, residual.data_ptr(), ldr, gain.data_ptr(), eps, code, rows, C,
          group_size, h.data_ptr(), ldh, q._codes, q._scales)
    return q, h


def quantize_rows(x, group_size=128):
    """The rows of a CUDA tensor [..., C] as QuantizedRows."""
    if _torch is None:
        _load_torch()
    code, C = _CODES.get(x.dtype), x.shape[-1]
    assert code is not None, "x: fp32, fp16 or bf16"
    rows, ldx = _rows_of(x, C, "x")
    q = QuantizedRows(rows, C, group_size, x.device, x.shape)
    _call(q.index, (_lib or load()).wfq_quantize_rows, x.data_ptr(), ldx, code, rows, C, group_size, q._codes, q._scales)
    return q


def dequantize_rows(q, dtype="f16"):
    """The values of QuantizedRows in "f32", "f16" or "bf16", shaped like the tensor they came from."""
    v = _empty(q.shape, _NAMED[dtype], q._buf.device)
    _call(q.index, (_lib or load()).wfq_dequantize_rows, q._codes, q._scales, q.rows, q.C, q.group_size, _DTYPES[dtype], v.data_ptr(), q.C)
    return v


class Linear:
    """A linear layer on group-wise int8 operands (include/wfq.h): C channels to K outputs, up to max_rows rows a call."""

    def __init__(self, C, K, group_size=128, max_rows=1, dtype="f16", out_dtype=None, gated=False, device="cuda:0"):
        torch = _torch or _load_torch()
        self.lin = None
        self.C, self.K, self.gs, self.gated = C, K, group_size, bool(gated)
        self.max_rows = max_rows
        self._in, self._out = _NAMED[dtype], _NAMED[out_dtype or dtype]
        self._bias = None
        self.lin = wfq_linear_create(C, K, group_size, gated)
        wfq_linear_set_input_dtype(self.lin, _DTYPES[dtype])
        wfq_linear_set_output_dtype(self.lin, _DTYPES[out_dtype or dtype])
        nbytes = wfq_linear_workspace_bytes(self.lin, max_rows)
        self._ws = torch.empty(nbytes + 1024, dtype=torch.uint8, device=device)
        self.device, self.index = self._ws.device, self._ws.get_device()
        with torch.cuda.device(self.index):
            wfq_linear_set_workspace(self.lin, (self._ws.data_ptr() + 1023) // 1024 * 1024, nbytes, max_rows)

    def prepare(self, w):
        """w: CUDA tensor [K][C] ([2K][C] if gated: gates, then values), fp32, fp16 or bf16."""
        assert w.get_device() == self.index and w.dtype in _CODES
        assert w.shape == ((2 if self.gated else 1) * self.K, self.C)
        _, ldw = _rows_of(w, self.C, "w")
        _call(self.index, _lib.wfq_linear_prepare_weights, self.lin, w.data_ptr(), ldw, _CODES[w.dtype])

    def set_epilogue(self, bias=None, act=WFQ_ACT_NONE):
        """bias: fp32 CUDA tensor [K] ([2K] if gated) or None; kept alive by this object."""
        if bias is not None:
            assert bias.get_device() == self.index and bias.dtype is _torch.float32 and bias.is_contiguous()
            assert bias.numel() == (2 if self.gated else 1) * self.K
        wfq_linear_set_epilogue(self.lin, None if bias is None else bias.data_ptr(), act)
        self._bias = bias

    def _outputs(self, lead, residual, y):
        K, shape = self.K, (*lead, self.K)
        if y is None:
            y, ldy = _empty(shape, self._out, self.device), K
        else:
            assert y.shape == shape and y.dtype is self._out and y.get_device() == self.index, "y"
            _, ldy = _rows_of(y, K, "y")
        if residual is None:
            return y, ldy, None, 0
        assert residual.shape == shape and residual.dtype is self._out and residual.get_device() == self.index, "residual"
        _, ldr = _rows_of(residual, K, "residual")
        return y, ldy, residual.data_ptr(), ldr

    def forward(self, x, residual=None, y=None):
        """x [..., C] -> y [..., K] (+ residual, which may be y).  y overlaps neither x nor, else, the residual."""
        assert x.dtype is self._in and x.get_device() == self.index, "x"
        rows, ldx = _rows_of(x, self.C, "x")
        y, ldy, res, ldr = self._outputs(x.shape[:-1], residual, y)
        _call(self.index, _lib.wfq_linear_forward, self.lin, x.data_ptr(), ldx, rows, res, ldr, y.data_ptr(), ldy)
        return y

    def forward_codes(self, q, residual=None, y=None):
        """The same on QuantizedRows of C channels in this layer's groups."""
        assert q.C == self.C and q.index == self.index, "q"
        assert q.group_size == self.gs or (q.groups == 1 and (self.gs == 0 or self.gs >= self.C)), "q: groups"
        y, ldy, res, ldr = self._outputs(q.shape[:-1], residual, y)
        _call(self.index, _lib.wfq_linear_forward_codes, self.lin, q._codes, q._scales, q.rows, res, ldr, y.data_ptr(), ldy)
        return y

    def check_status(self):
        with _torch.cuda.device(self.index):
            st, where = wfq_linear_check_status(self.lin, _torch._C._cuda_getCurrentRawStream(self.index))
        if st != WFQ_OK:
            raise WfqError(st, f"device status (wait id {where})")

    def close(self):
        if self.lin is not None:
            wfq_linear_destroy(self.lin)
            self.lin = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
