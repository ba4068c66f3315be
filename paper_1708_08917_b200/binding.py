"""ctypes binding of ``libcirc.so``: the same names as ``include/circ.h``, argument marshalling only.

Every step of the forward pass runs inside the CUDA library; nothing here computes.  torch (or any
other owner of device memory) is used by callers for allocation and streams only: tensors are
passed as raw device pointers, streams as ``cudaStream_t`` integers.  If the library has not been
built, or cannot be loaded, importing a function from here raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import numpy as np

_HERE = Path(__file__).resolve().parent
LIB_PATH = _HERE / "libcirc.so"

CIRC_OK = 0
CIRC_ERR_ARG, CIRC_ERR_SHAPE, CIRC_ERR_ALLOC, CIRC_ERR_CUDA, CIRC_ERR_DEVICE_TIMEOUT, CIRC_ERR_UNSUPPORTED = -1, -2, -3, -4, -5, -6
CIRC_F32, CIRC_BF16, CIRC_E4M3 = 0, 1, 2
CIRC_I32, CIRC_I64 = 0, 1
CIRC_POOL_MAX, CIRC_POOL_AVG, CIRC_POOL_L2 = 0, 1, 2
CIRC_ACT_NONE, CIRC_ACT_RELU, CIRC_ACT_SILU = 0, 1, 2
CIRC_VARIANT_AUTO, CIRC_VARIANT_FUSED, CIRC_VARIANT_STAGED, CIRC_VARIANT_TENSOR = 0, 1, 2, 3
# include/circ_debug.h
CIRC_STAGE_INPUT_FFT, CIRC_STAGE_CONTRACTION, CIRC_STAGE_OUTPUT_IFFT, CIRC_STAGE_FUSED = 0, 1, 2, 3
CIRC_KERNEL_NONE, CIRC_KERNEL_S1_LOADS, CIRC_KERNEL_S1_BULK = 0, 1, 2
CIRC_KERNEL_S2_TENSOR_TWIN, CIRC_KERNEL_S2_ROWS, CIRC_KERNEL_S2_ROWS_TWIN = 12, 13, 14
CIRC_KERNEL_S2_FMA, CIRC_KERNEL_S2_TENSOR, CIRC_KERNEL_S3_LOADS, CIRC_KERNEL_S3_BULK, CIRC_KERNEL_S4_FUSED = 10, 11, 20, 21, 30
CIRC_KERNEL_S3_TMA = 22
CIRC_INJECT_NONE, CIRC_INJECT_TENSOR_NO_COPY, CIRC_INJECT_BULK_NO_COPY = 0, 1, 2

# name -> (restype, argtypes); mirrors include/circ.h one to one
_vp, _ci, _cl, _cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_float
SIGNATURES = {
    "circ_fc_create": (_vp, [_ci, _ci, _ci, _vp]),
    "circ_fc_forward": (_ci, [_vp, _vp, _vp, _ci, _vp]),
    "circ_conv_create": (_vp, [_ci, _ci, _ci, _ci, _ci, _vp]),
    "circ_conv_forward": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _vp]),
    "circ_fc_forward_host": (_ci, [_vp, _vp, _vp, _ci, _vp]),
    "circ_conv_forward_host": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _vp]),
    "circ_fc_forward_noalloc": (_ci, [_vp, _vp, _vp, _ci, _vp]),
    "circ_noalloc_max_bytes": (_cl, []),
    "circ_fc_backward": (_ci, [_vp, _vp, _vp, _vp, _vp, _ci, _vp]),
    "circ_conv_backward_input": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _vp]),
    "circ_conv_backward_weight": (_ci, [_vp, _vp, _vp, _vp, _ci, _ci, _ci, _vp]),
    "circ_stack_create": (_vp, [_vp, _ci]),
    "circ_stack_forward": (_ci, [_vp, _vp, _vp, _ci, _vp]),
    "circ_stack_reserve": (_ci, [_vp, _cl]),
    "circ_stack_relayed": (_ci, [_vp]),
    "circ_stack_destroy": (None, [_vp]),
    "circ_device_status": (_ci, [_vp]),
    "circ_destroy": (None, [_vp]),
    "circ_set_bias": (_ci, [_vp, _vp]),
    "circ_set_activation": (_ci, [_vp, _ci]),
    "circ_set_io_dtype": (_ci, [_vp, _ci, _ci]),
    "circ_set_convention": (_ci, [_vp, _ci]),
    "circ_set_spectrum_dtype": (_ci, [_vp, _ci]),
    "circ_set_variant": (_ci, [_vp, _ci]),
    "circ_reserve": (_ci, [_vp, _cl]),
    "circ_workspace_bytes": (_cl, [_vp]),
    "circ_last_variant": (_ci, [_vp]),
    "circ_weight_bytes": (_cl, [_vp]),
    # include/circ_debug.h
    "circ_debug_forward_repeat": (_ci, [_vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _vp]),
    "circ_debug_last_kernels": (_ci, [_vp, _vp]),
    "circ_debug_launch_count": (_cl, []),
    "circ_debug_fma_burn": (_ci, [_vp, _ci, _ci, _vp, _vp]),
    "circ_debug_empty_kernel": (_ci, [_vp]),
    "circ_debug_inject": (_ci, [_vp, _ci]),
    "circ_debug_fail_alloc_after": (_ci, [_cl]),
    "circ_debug_set_fused_split": (_ci, [_vp, _ci]),
    "circ_debug_set_contraction": (_ci, [_vp, _ci, _ci]),
    "circ_debug_set_transforms": (_ci, [_vp, _ci, _ci]),
    "circ_conv_set_stride": (_ci, [_vp, _ci]),
    "circ_pool_forward": (_ci, [_vp, _vp, _ci, _ci, _ci, _ci, _ci, _ci, _ci, _ci, _vp]),
    "circ_embed_create": (_vp, [_ci, _ci]),
    "circ_embed_set_dtypes": (_ci, [_vp, _ci, _ci, _ci]),
    "circ_embed_set_scale": (_ci, [_vp, _cf]),
    "circ_embed_set_padding": (_ci, [_vp, _cl]),
    "circ_embed_reserve": (_ci, [_vp, _cl]),
    "circ_embed_forward": (_ci, [_vp, _vp, _vp, _vp, _cl, _vp]),
    "circ_embed_backward": (_ci, [_vp, _vp, _vp, _vp, _cl, _vp]),
    "circ_embed_destroy": (None, [_vp]),
    "circ_norm_create": (_vp, [_ci, _cf]),
    "circ_norm_set_dtypes": (_ci, [_vp, _ci, _ci]),
    "circ_norm_set_group": (_ci, [_vp, _ci]),
    "circ_norm_reserve": (_ci, [_vp]),
    "circ_norm_forward": (_ci, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _cl, _vp]),
    "circ_norm_backward": (_ci, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _cl, _vp]),
    "circ_norm_unpack": (_ci, [_vp, _vp, _vp, _vp, _ci, _cl, _vp]),
    "circ_norm_destroy": (None, [_vp]),
    "circ_loss_create": (_vp, [_ci]),
    "circ_loss_set_dtypes": (_ci, [_vp, _ci, _ci]),
    "circ_loss_set_ignore": (_ci, [_vp, _cl]),
    "circ_loss_reserve": (_ci, [_vp, _cl]),
    "circ_loss_forward": (_ci, [_vp, _vp, _cl, _vp, _vp, _vp, _vp, _cl, _vp]),
    "circ_loss_backward": (_ci, [_vp, _vp, _cl, _vp, _vp, _vp, _vp, _vp, _cl, _cf, _cl, _vp]),
    "circ_loss_destroy": (None, [_vp]),
    "circ_clip_create": (_vp, [_ci, _vp, _vp, _vp]),
    "circ_clip_set_tensors": (_ci, [_vp, _vp, _vp, _vp]),
    "circ_clip_forward": (_ci, [_vp, _cf, _vp, _vp]),
    "circ_clip_destroy": (None, [_vp]),
    "circ_top_create": (_vp, [_ci, _ci]),
    "circ_top_set_dtypes": (_ci, [_vp, _ci, _ci]),
    "circ_top_set_temperature": (_ci, [_vp, _cf]),
    "circ_top_reserve": (_ci, [_vp, _cl]),
    "circ_top_forward": (_ci, [_vp, _vp, _cl, _vp, _vp, _vp, _cl, _vp]),
    "circ_top_destroy": (None, [_vp]),
    "circ_distill_create": (_vp, [_ci, _ci]),
    "circ_distill_set_dtypes": (_ci, [_vp, _ci, _ci, _ci]),
    "circ_distill_set_temperature": (_ci, [_vp, _cf]),
    "circ_distill_set_rest": (_ci, [_vp, _ci]),
    "circ_distill_set_add": (_ci, [_vp, _ci]),
    "circ_distill_reserve": (_ci, [_vp, _cl]),
    "circ_distill_forward": (_ci, [_vp, _vp, _cl, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _cl, _vp]),
    "circ_distill_backward": (_ci, [_vp, _vp, _cl, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _cl, _cf, _cl, _vp]),
    "circ_distill_destroy": (None, [_vp]),
    "circ_gnorm_create": (_vp, [_ci, _ci, _cf]),
    "circ_gnorm_set_dtypes": (_ci, [_vp, _ci, _ci]),
    "circ_gnorm_set_activation": (_ci, [_vp, _ci]),
    "circ_gnorm_reserve": (_ci, [_vp, _ci, _ci, _ci]),
    "circ_gnorm_forward": (_ci, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _vp]),
    "circ_gnorm_backward": (_ci, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _vp]),
    "circ_gnorm_destroy": (None, [_vp]),
    "circ_last_error": (ctypes.c_char_p, []),
    "circ_last_code": (_ci, []),
}

_lib = None


class CircError(RuntimeError):
    """A libcirc call failed; ``code`` is the CIRC_ERR_* value."""

    def __init__(self, code: int, message: str):
        super().__init__(f"libcirc error {code}: {message}")
        self.code = code


def load() -> ctypes.CDLL:
    """Load ``libcirc.so`` (built by ``paper_1708_08917_b200.build``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1708_08917_b200.build` "
                              "(there is no CPU or PyTorch fallback)")
        lib = ctypes.CDLL(str(LIB_PATH))
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _ptr(a) -> int | None:
    """Raw address of a torch tensor, a numpy array, an int, or None."""
    if a is None:
        return None
    if isinstance(a, int):
        return a
    if isinstance(a, np.ndarray):
        assert a.flags["C_CONTIGUOUS"]
        return a.ctypes.data
    assert a.is_contiguous()
    return a.data_ptr()


def _rows_ptr(a) -> int | None:
    """Address of a matrix whose rows may lie further apart than they are long (the call is told the stride)."""
    if a is None or isinstance(a, (int, np.ndarray)):
        return _ptr(a)
    assert a.numel() == 0 or a.stride(-1) == 1
    return a.data_ptr()


def _made(h):
    """The handle of a create call; raises if it is NULL."""
    if not h:
        raise CircError(circ_last_code(), circ_last_error())
    return h


def _stream(stream) -> int | None:
    if stream is None or isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(rc: int) -> None:
    if rc != CIRC_OK:
        raise CircError(rc, circ_last_error())


def _weights(w):
    if isinstance(w, np.ndarray):
        w = np.ascontiguousarray(w, dtype=np.float32)
    return w


def circ_last_error() -> str:
    return load().circ_last_error().decode()


def circ_last_code() -> int:
    return load().circ_last_code()


def circ_fc_create(m: int, n: int, k: int, w) -> int:
    """``w``: float32 ``[p][q][k]`` defining vectors (numpy array on the host or a device tensor)."""
    w = _weights(w)
    h = load().circ_fc_create(m, n, k, _ptr(w))
    if not h:
        raise CircError(circ_last_code(), circ_last_error())
    return h


def circ_conv_create(c_out: int, c_in: int, r: int, pad: int, k: int, w) -> int:
    """``w``: float32 ``[r][r][p][q][k]``."""
    w = _weights(w)
    h = load().circ_conv_create(c_out, c_in, r, pad, k, _ptr(w))
    if not h:
        raise CircError(circ_last_code(), circ_last_error())
    return h


def circ_fc_forward(h: int, x, y, batch: int, stream=None) -> None:
    """Enqueue ``y[batch][m] = psi(W x + theta)``; ``x``, ``y`` are device tensors or raw device addresses."""
    _check(load().circ_fc_forward(h, _ptr(x), _ptr(y), batch, _stream(stream)))


def circ_conv_forward(h: int, x, y, N: int, H: int, W: int, stream=None) -> None:
    """Enqueue the channel-last convolution ``x[N][H][W][C] -> y[N][Ho][Wo][P]``."""
    _check(load().circ_conv_forward(h, _ptr(x), _ptr(y), N, H, W, _stream(stream)))


def circ_conv_set_stride(h: int, stride: int) -> None:
    _check(load().circ_conv_set_stride(h, int(stride)))


def circ_pool_forward(x, y, N: int, H: int, W: int, C: int, window: int, stride: int, mode: int, dtype: int, stream=None) -> None:
    """Enqueue the pooling layer ``x[N][H][W][C] -> y[N][Ho][Wo][C]`` (whole windows, no padding)."""
    _check(load().circ_pool_forward(_ptr(x), _ptr(y), N, H, W, C, window, stride, mode, dtype, _stream(stream)))


def circ_fc_forward_host(h: int, x_host, y_host, batch: int, stream=None) -> None:
    """Host-memory variant: ``x_host`` / ``y_host`` are (pinned) CPU tensors, numpy arrays or addresses."""
    _check(load().circ_fc_forward_host(h, _ptr(x_host), _ptr(y_host), batch, _stream(stream)))


def circ_conv_forward_host(h: int, x_host, y_host, N: int, H: int, W: int, stream=None) -> None:
    _check(load().circ_conv_forward_host(h, _ptr(x_host), _ptr(y_host), N, H, W, _stream(stream)))


def circ_fc_forward_noalloc(h: int, x, y, batch: int, stream=None) -> None:
    """``circ_fc_forward`` for callers that may not allocate: scratch lives in a fixed array inside the library.

    Use it from code that cannot afford (or is not permitted) a ``cudaMalloc`` at forward time.  The batch is
    limited by ``circ_noalloc_max_bytes()``; all calls share one scratch array, so do not overlap them on the GPU;
    make the first call on a device outside stream capture.
    """
    _check(load().circ_fc_forward_noalloc(h, _ptr(x), _ptr(y), batch, _stream(stream)))


def circ_noalloc_max_bytes() -> int:
    return load().circ_noalloc_max_bytes()


def circ_fc_backward(h: int, x, grad_a, grad_x, grad_w, batch: int, stream=None) -> None:
    """Enqueue ``grad_x = W^T grad_a`` and ``grad_w[p][q][k]`` (either may be None) from ``grad_a = dL/da``."""
    _check(load().circ_fc_backward(h, _ptr(x), _ptr(grad_a), _ptr(grad_x), _ptr(grad_w), batch, _stream(stream)))


def circ_conv_backward_input(h: int, grad_y, grad_x, N: int, H: int, W: int, stream=None) -> None:
    """Enqueue ``grad_x[N][H][W][C]`` from ``grad_y[N][Ho][Wo][P]``; ``N, H, W`` are the forward input's extent."""
    _check(load().circ_conv_backward_input(h, _ptr(grad_y), _ptr(grad_x), N, H, W, _stream(stream)))


def circ_conv_backward_weight(h: int, x, grad_y, grad_w, N: int, H: int, W: int, stream=None) -> None:
    """Enqueue ``grad_w[r][r][p][q][k]`` (float32) from the forward input ``x`` and ``grad_y``."""
    _check(load().circ_conv_backward_weight(h, _ptr(x), _ptr(grad_y), _ptr(grad_w), N, H, W, _stream(stream)))


def circ_stack_create(layers) -> int:
    """A stack over fully-connected layer handles (borrowed: destroy the stack first, then the layers)."""
    arr = (ctypes.c_void_p * len(layers))(*layers)
    s = load().circ_stack_create(ctypes.addressof(arr), len(layers))
    if not s:
        raise CircError(circ_last_code(), circ_last_error())
    return s


def circ_stack_forward(s: int, x, y, batch: int, stream=None) -> None:
    """Enqueue all layers; boundaries between staged layers of equal block size run as one relay kernel."""
    _check(load().circ_stack_forward(s, _ptr(x), _ptr(y), batch, _stream(stream)))


def circ_stack_reserve(s: int, max_batch: int) -> None:
    _check(load().circ_stack_reserve(s, max_batch))


def circ_stack_relayed(s: int) -> int:
    return load().circ_stack_relayed(s)


def circ_stack_destroy(s: int | None) -> None:
    load().circ_stack_destroy(s)


def circ_device_status(h: int) -> None:
    """Blocks until the device is idle; raises CircError(CIRC_ERR_DEVICE_TIMEOUT) if a bounded wait expired."""
    _check(load().circ_device_status(h))


def circ_destroy(h: int | None) -> None:
    load().circ_destroy(h)


def circ_set_bias(h: int, bias) -> None:
    if isinstance(bias, np.ndarray):
        bias = np.ascontiguousarray(bias, dtype=np.float32)
    _check(load().circ_set_bias(h, _ptr(bias)))


def circ_set_activation(h: int, relu: int) -> None:
    _check(load().circ_set_activation(h, int(relu)))


def circ_set_io_dtype(h: int, x_dtype: int, y_dtype: int) -> None:
    _check(load().circ_set_io_dtype(h, x_dtype, y_dtype))


def circ_set_convention(h: int, convention: int) -> None:
    _check(load().circ_set_convention(h, convention))


def circ_set_spectrum_dtype(h: int, dtype: int) -> None:
    """CIRC_BF16: the small-batch streaming kernel reads bfloat16 weight spectra (half the bytes)."""
    _check(load().circ_set_spectrum_dtype(h, dtype))


def circ_set_variant(h: int, variant: int) -> None:
    _check(load().circ_set_variant(h, variant))


def circ_reserve(h: int, max_batch: int) -> None:
    _check(load().circ_reserve(h, max_batch))


def circ_workspace_bytes(h: int) -> int:
    return load().circ_workspace_bytes(h)


def circ_last_variant(h: int) -> int:
    return load().circ_last_variant(h)


def circ_weight_bytes(h: int) -> int:
    """Bytes of device memory the handle holds for the layer's weights in all stored forms."""
    return load().circ_weight_bytes(h)


# ---- operators around the circulant layers of a token model ------------------------------------------

def circ_embed_create(vocab: int, dim: int) -> int:
    return _made(load().circ_embed_create(vocab, dim))


def circ_embed_set_dtypes(h: int, table_dtype: int, y_dtype: int, ids_type: int) -> None:
    _check(load().circ_embed_set_dtypes(h, table_dtype, y_dtype, ids_type))


def circ_embed_set_scale(h: int, scale: float) -> None:
    _check(load().circ_embed_set_scale(h, scale))


def circ_embed_set_padding(h: int, padding: int) -> None:
    """``padding``: the id that stands for no token (-1: none)."""
    _check(load().circ_embed_set_padding(h, padding))


def circ_embed_reserve(h: int, max_tokens: int) -> None:
    _check(load().circ_embed_reserve(h, max_tokens))


def circ_embed_forward(h: int, table, ids, y, tokens: int, stream=None) -> None:
    """Enqueue ``y[t] = scale * table[ids[t]]`` (a zero row for the padding id and for ids outside the table)."""
    _check(load().circ_embed_forward(h, _ptr(table), _ptr(ids), _ptr(y), tokens, _stream(stream)))


def circ_embed_backward(h: int, ids, grad_y, grad_table, tokens: int, stream=None) -> None:
    """Enqueue ``grad_table[v] = scale * sum of grad_y[t] over tokens with ids[t] == v`` (every row is written)."""
    _check(load().circ_embed_backward(h, _ptr(ids), _ptr(grad_y), _ptr(grad_table), tokens, _stream(stream)))


def circ_embed_destroy(h: int | None) -> None:
    load().circ_embed_destroy(h)


def circ_norm_create(dim: int, eps: float) -> int:
    return _made(load().circ_norm_create(dim, eps))


def circ_norm_set_dtypes(h: int, x_dtype: int, y_dtype: int) -> None:
    _check(load().circ_norm_set_dtypes(h, x_dtype, y_dtype))


def circ_norm_set_group(h: int, group: int) -> None:
    """Elements that share a scale of an 8-bit output: 32, 64, 128, or 0 for a whole row."""
    _check(load().circ_norm_set_group(h, group))


def circ_norm_reserve(h: int) -> None:
    _check(load().circ_norm_reserve(h))


def circ_norm_forward(h: int, x, residual, gain, sum, y, y_scale, rstd, rows: int, stream=None) -> None:
    """Enqueue ``sum = x + residual; y = sum * rstd * gain``; ``residual``, ``gain``, ``sum``, ``rstd`` may be None."""
    _check(load().circ_norm_forward(h, _ptr(x), _ptr(residual), _ptr(gain), _ptr(sum), _ptr(y), _ptr(y_scale), _ptr(rstd), rows, _stream(stream)))


def circ_norm_backward(h: int, sum, gain, rstd, grad_y, grad_sum, grad_x, grad_gain, rows: int, stream=None) -> None:
    """Enqueue the gradients of the norm; ``grad_sum`` (what flows past the norm), ``grad_x`` or ``grad_gain`` may be None."""
    _check(load().circ_norm_backward(h, _ptr(sum), _ptr(gain), _ptr(rstd), _ptr(grad_y), _ptr(grad_sum), _ptr(grad_x), _ptr(grad_gain), rows,
                                     _stream(stream)))


def circ_norm_unpack(h: int, y, y_scale, out, out_dtype: int, rows: int, stream=None) -> None:
    """Enqueue ``out = y_scale * y`` for an 8-bit output of ``circ_norm_forward``."""
    _check(load().circ_norm_unpack(h, _ptr(y), _ptr(y_scale), _ptr(out), out_dtype, rows, _stream(stream)))


def circ_norm_destroy(h: int | None) -> None:
    load().circ_norm_destroy(h)


def circ_loss_create(classes: int) -> int:
    return _made(load().circ_loss_create(classes))


def circ_loss_set_dtypes(h: int, logits_dtype: int, ids_type: int) -> None:
    _check(load().circ_loss_set_dtypes(h, logits_dtype, ids_type))


def circ_loss_set_ignore(h: int, ignore: int) -> None:
    _check(load().circ_loss_set_ignore(h, ignore))


def circ_loss_reserve(h: int, max_rows: int) -> None:
    _check(load().circ_loss_reserve(h, max_rows))


def circ_loss_forward(h: int, logits, stride: int, targets, row_loss, lse, mean, rows: int, stream=None) -> None:
    """Enqueue the softmax cross entropy; ``stride``: elements between rows of ``logits``; results that are None are skipped."""
    _check(load().circ_loss_forward(h, _rows_ptr(logits), stride, _ptr(targets), _ptr(row_loss), _ptr(lse), _ptr(mean), rows, _stream(stream)))


def circ_loss_backward(h: int, logits, stride: int, targets, row_loss, lse, mean, grad_logits, grad_stride: int, grad_mean: float, rows: int,
                       stream=None) -> None:
    """``circ_loss_forward`` and the gradient of ``grad_mean * mean`` with respect to the logits (may replace them)."""
    _check(load().circ_loss_backward(h, _rows_ptr(logits), stride, _ptr(targets), _ptr(row_loss), _ptr(lse), _ptr(mean), _rows_ptr(grad_logits),
                                     grad_stride, grad_mean, rows, _stream(stream)))


def circ_loss_destroy(h: int | None) -> None:
    load().circ_loss_destroy(h)


def circ_clip_create(sizes, grad_dtypes, out_dtypes) -> int:
    """``sizes``: elements of each tensor; the types: one code for all tensors, or one for each."""
    n = len(sizes)
    grads, outs = ([t] * n if isinstance(t, int) else list(t) for t in (grad_dtypes, out_dtypes))
    assert len(grads) == n and len(outs) == n
    return _made(load().circ_clip_create(n, (ctypes.c_long * n)(*sizes), (ctypes.c_int * n)(*grads), (ctypes.c_int * n)(*outs)))


def circ_clip_set_tensors(h: int, grads, outs=None, stream=None) -> None:
    """The tensors of the following ``circ_clip_forward`` calls, in the order of their sizes; ``outs`` None: in place."""
    n = len(grads)
    assert outs is None or len(outs) == n
    g = (ctypes.c_void_p * n)(*map(_ptr, grads))
    o = None if outs is None else (ctypes.c_void_p * n)(*map(_ptr, outs))
    _check(load().circ_clip_set_tensors(h, g, o, _stream(stream)))


def circ_clip_forward(h: int, max_norm: float, norm, stream=None) -> None:
    """Enqueue the norm over all tensors (``norm``: a device float, or None) and their scaling."""
    _check(load().circ_clip_forward(h, max_norm, _ptr(norm), _stream(stream)))


def circ_clip_destroy(h: int | None) -> None:
    load().circ_clip_destroy(h)


# ---- operators that train a compressed network in the place of an uncompressed one ---------------------

def circ_top_create(classes: int, count: int) -> int:
    return _made(load().circ_top_create(classes, count))


def circ_top_set_dtypes(h: int, logits_dtype: int, ids_type: int) -> None:
    _check(load().circ_top_set_dtypes(h, logits_dtype, ids_type))


def circ_top_set_temperature(h: int, temperature: float) -> None:
    _check(load().circ_top_set_temperature(h, temperature))


def circ_top_reserve(h: int, max_rows: int) -> None:
    _check(load().circ_top_reserve(h, max_rows))


def circ_top_forward(h: int, logits, stride: int, values, ids, lse, rows: int, stream=None) -> None:
    """Enqueue the selection of each row's largest logits, descending, and log sum exp(logits / temperature); results that are None are skipped."""
    _check(load().circ_top_forward(h, _rows_ptr(logits), stride, _ptr(values), _ptr(ids), _ptr(lse), rows, _stream(stream)))


def circ_top_destroy(h: int | None) -> None:
    load().circ_top_destroy(h)


def circ_distill_create(classes: int, count: int) -> int:
    return _made(load().circ_distill_create(classes, count))


def circ_distill_set_dtypes(h: int, logits_dtype: int, values_dtype: int, ids_type: int) -> None:
    _check(load().circ_distill_set_dtypes(h, logits_dtype, values_dtype, ids_type))


def circ_distill_set_temperature(h: int, temperature: float) -> None:
    _check(load().circ_distill_set_temperature(h, temperature))


def circ_distill_set_rest(h: int, rest: int) -> None:
    """1: the classes outside a list count as one class more (the calls need the teacher's lse then)."""
    _check(load().circ_distill_set_rest(h, int(rest)))


def circ_distill_set_add(h: int, add: int) -> None:
    """1: gradients are added to what ``grad_logits`` holds."""
    _check(load().circ_distill_set_add(h, int(add)))


def circ_distill_reserve(h: int, max_rows: int) -> None:
    _check(load().circ_distill_reserve(h, max_rows))


def circ_distill_forward(h: int, logits, stride: int, values, ids, lse, weights, row_loss, student_lse, mean, rows: int, stream=None) -> None:
    """Enqueue the divergence from the teacher's lists ``values``, ``ids`` [rows][count]; ``lse``, ``weights`` and any result may be None."""
    _check(load().circ_distill_forward(h, _rows_ptr(logits), stride, _ptr(values), _ptr(ids), _ptr(lse), _ptr(weights), _ptr(row_loss),
                                       _ptr(student_lse), _ptr(mean), rows, _stream(stream)))


def circ_distill_backward(h: int, logits, stride: int, values, ids, lse, weights, row_loss, student_lse, mean, grad_logits, grad_stride: int,
                          grad_mean: float, rows: int, stream=None) -> None:
    """``circ_distill_forward`` and the gradient of ``grad_mean * mean`` with respect to the logits (may replace them)."""
    _check(load().circ_distill_backward(h, _rows_ptr(logits), stride, _ptr(values), _ptr(ids), _ptr(lse), _ptr(weights), _ptr(row_loss),
                                        _ptr(student_lse), _ptr(mean), _rows_ptr(grad_logits), grad_stride, grad_mean, rows, _stream(stream)))


def circ_distill_destroy(h: int | None) -> None:
    load().circ_distill_destroy(h)


def circ_gnorm_create(channels: int, groups: int, eps: float) -> int:
    return _made(load().circ_gnorm_create(channels, groups, eps))


def circ_gnorm_set_dtypes(h: int, x_dtype: int, y_dtype: int) -> None:
    _check(load().circ_gnorm_set_dtypes(h, x_dtype, y_dtype))


def circ_gnorm_set_activation(h: int, activation: int) -> None:
    """``activation``: CIRC_ACT_NONE, CIRC_ACT_RELU or CIRC_ACT_SILU."""
    _check(load().circ_gnorm_set_activation(h, activation))


def circ_gnorm_reserve(h: int, N: int, H: int, W: int) -> None:
    _check(load().circ_gnorm_reserve(h, N, H, W))


def circ_gnorm_forward(h: int, x, gain, bias, y, mean, rstd, N: int, H: int, W: int, stream=None) -> None:
    """Enqueue ``y = act(gain (x - mean) rstd + bias)`` on ``x[N][H][W][channels]``; ``gain``, ``bias``, ``mean``, ``rstd`` may be None."""
    _check(load().circ_gnorm_forward(h, _ptr(x), _ptr(gain), _ptr(bias), _ptr(y), _ptr(mean), _ptr(rstd), N, H, W, _stream(stream)))


def circ_gnorm_backward(h: int, x, gain, bias, mean, rstd, grad_y, grad_x, grad_gain, grad_bias, N: int, H: int, W: int, stream=None) -> None:
    """Enqueue the gradients of the group norm; any of ``grad_x``, ``grad_gain``, ``grad_bias`` may be None."""
    _check(load().circ_gnorm_backward(h, _ptr(x), _ptr(gain), _ptr(bias), _ptr(mean), _ptr(rstd), _ptr(grad_y), _ptr(grad_x), _ptr(grad_gain),
                                      _ptr(grad_bias), N, H, W, _stream(stream)))


def circ_gnorm_destroy(h: int | None) -> None:
    load().circ_gnorm_destroy(h)


# ---- include/circ_debug.h: test and measurement aids ------------------------------------------------

def circ_debug_forward_repeat(h: int, x, y, N: int, H: int, W: int, stage: int, times: int, stream=None) -> None:
    """The forward pass with the kernel of ``stage`` launched ``times`` times (results unchanged): per-kernel timing."""
    _check(load().circ_debug_forward_repeat(h, _ptr(x), _ptr(y), N, H, W, stage, times, _stream(stream)))


def circ_debug_last_kernels(h: int) -> list[int]:
    """CIRC_KERNEL_* ids of the S1 / S2 / S3 kernels of the handle's most recent staged forward."""
    ids = (ctypes.c_int * 3)()
    _check(load().circ_debug_last_kernels(h, ctypes.addressof(ids)))
    return list(ids)


def circ_debug_launch_count() -> int:
    return load().circ_debug_launch_count()


def circ_debug_fma_burn(sink, blocks: int, iters: int, stream=None) -> float:
    """Enqueue the float32 FMA micro-benchmark kernel; returns the flops of the launch."""
    flops = ctypes.c_double(0.0)
    _check(load().circ_debug_fma_burn(_ptr(sink), blocks, iters, ctypes.addressof(flops), _stream(stream)))
    return flops.value


def circ_debug_empty_kernel(stream=None) -> None:
    _check(load().circ_debug_empty_kernel(_stream(stream)))


def circ_debug_inject(h: int, kind: int) -> None:
    _check(load().circ_debug_inject(h, kind))


def circ_debug_set_fused_split(h: int, slices: int) -> None:
    _check(load().circ_debug_set_fused_split(h, slices))


def circ_debug_set_contraction(h: int, allow_twin: int, allow_rows: int) -> None:
    _check(load().circ_debug_set_contraction(h, int(allow_twin), int(allow_rows)))


def circ_debug_set_transforms(h: int, allow_tma_input: int, allow_tma_output: int = 1) -> None:
    _check(load().circ_debug_set_transforms(h, int(allow_tma_input), int(allow_tma_output)))


def circ_debug_fail_alloc_after(n: int) -> None:
    _check(load().circ_debug_fail_alloc_after(n))
