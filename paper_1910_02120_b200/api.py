"""ctypes binding of libist.so: the same calls as include/ist.h, with torch tensors as the
owners of device memory.  Argument marshalling only; every step of a round runs inside the
library's CUDA kernels.  There is no CPU fallback: if the shared library is missing, import
fails with instructions to build it.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os
import weakref
from array import array
from typing import List, Optional, Sequence, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("IST_LIB_PATH") or os.path.join(_HERE, "libist.so")

IST_OK = 0
IST_ERR_ARG, IST_ERR_STATE, IST_ERR_WORKSPACE, IST_ERR_CUDA = -1, -2, -3, -4
IST_ERR_DEVICE_CHECK, IST_ERR_DEVICE_TIMEOUT, IST_ERR_UNSUPPORTED = -5, -6, -7
IST_FP32, IST_BF16 = 0, 1
IST_X_DENSE_F32, IST_X_DENSE_BF16, IST_X_CSR = 0, 1, 2

EXPORTS = [
    "ist_workspace_bytes", "ist_create", "ist_bind_weights", "ist_partition", "ist_get_partition",
    "ist_get_subnet_params", "ist_local_steps", "ist_reassemble", "ist_eval", "ist_sync_status",
    "ist_kernel_launches", "ist_last_error", "ist_destroy", "ist_profile", "ist_profile_read",
    "ist_partition_layer_static", "ist_norm_workspace_bytes", "ist_enable_normalization", "ist_calibrate",
    "ist_set_subnet_range", "ist_packed_layer", "ist_workspace_bytes2", "ist_create2",
    "ist_selftest_wait_expiry", "ist_subnet_slice_shape", "ist_static_partition_status", "ist_local_steps_dx",
    "ist_layer_norm_forward", "ist_layer_norm_workspace_bytes", "ist_layer_norm_backward", "ist_adamw_workspace_bytes",
    "ist_adamw_step", "ist_adamw_state_values", "ist_layer_norm_status", "ist_selftest_layer_norm_wait",
]
IST_PART_BALANCED, IST_PART_IID = 0, 1
IST_STATIC_MAX_NEURONS, IST_STATIC_MAX_SUBNETS = 65536, 64
IST_T_F32, IST_T_BF16 = 0, 1
IST_ADAMW_BLOCK = 128

KERNEL_CLASSES = ["partition", "gather", "stage", "fwd", "loss", "dx", "dw_sgd", "bias_sgd", "spmm",
                  "scatter", "eval", "norm"]


class IstInput(ctypes.Structure):
    _fields_ = [
        ("kind", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("dense", ctypes.c_void_p),
        ("row_ptr", ctypes.c_void_p),
        ("col", ctypes.c_void_p),
        ("val", ctypes.c_void_p),
        ("stride_subnet", ctypes.c_int64),
        ("stride_step", ctypes.c_int64),
    ]


# One row of ist_adamw_step's table.
ADAMW_TENSOR = np.dtype([(name, np.uint64) for name in ("param", "grad", "exp_avg", "exp_avg_sq", "exp_avg_base",
                                                         "exp_avg_sq_base", "param_bf16")]
                        + [("n", np.int64), ("weight_decay", np.float64)])


class AdamWArgs(ctypes.Structure):
    _fields_ = [
        ("lr", ctypes.c_double),
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("max_norm", ctypes.c_double),
        ("step", ctypes.c_int64),
        ("seed", ctypes.c_uint64),
        ("state_bits", ctypes.c_int32),
        ("grad_type", ctypes.c_int32),
        ("step_dev", ctypes.c_void_p),
        ("lr_dev", ctypes.c_void_p),
        ("norm_out_dev", ctypes.c_void_p),
    ]


class IstError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"ist_status {status}: {message}")
        self.status = status


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_1910_02120_b200.build` "
            "(needs nvcc); there is no fallback implementation")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    p64 = ctypes.POINTER(ctypes.c_int64)
    lib.ist_workspace_bytes.restype = sz
    lib.ist_workspace_bytes.argtypes = [p64, i32, i32, i32, i32, i32]
    lib.ist_workspace_bytes2.restype = sz
    lib.ist_workspace_bytes2.argtypes = [p64, i32, i32, i32, i32, i32, i32]
    lib.ist_create2.restype = ctypes.c_int32
    lib.ist_create2.argtypes = [ctypes.POINTER(vp), p64, i32, i32, i32, i32, i32, i32, vp, sz, vp]
    lib.ist_create.restype = ctypes.c_int32
    lib.ist_create.argtypes = [ctypes.POINTER(vp), p64, i32, i32, i32, i32, i32, vp, sz, vp]
    lib.ist_bind_weights.restype = ctypes.c_int32
    lib.ist_bind_weights.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp)]
    lib.ist_partition.restype = ctypes.c_int32
    lib.ist_partition.argtypes = [vp, u64]
    lib.ist_get_partition.restype = ctypes.c_int32
    lib.ist_get_partition.argtypes = [vp, i32, vp, vp]
    lib.ist_get_subnet_params.restype = ctypes.c_int32
    lib.ist_get_subnet_params.argtypes = [vp, i32, i32, vp, vp]
    lib.ist_subnet_slice_shape.restype = ctypes.c_int32
    lib.ist_subnet_slice_shape.argtypes = [vp, i32, i32, p64, p64]
    lib.ist_static_partition_status.restype = ctypes.c_int32
    lib.ist_static_partition_status.argtypes = [vp]
    lib.ist_local_steps.restype = ctypes.c_int32
    lib.ist_local_steps.argtypes = [vp, ctypes.POINTER(IstInput), vp, ctypes.c_float, i32, vp]
    lib.ist_local_steps_dx.restype = ctypes.c_int32
    lib.ist_local_steps_dx.argtypes = [vp, ctypes.POINTER(IstInput), vp, ctypes.c_float, i32, vp, vp]
    lib.ist_reassemble.restype = ctypes.c_int32
    lib.ist_reassemble.argtypes = [vp]
    lib.ist_eval.restype = ctypes.c_int32
    lib.ist_eval.argtypes = [vp, ctypes.POINTER(IstInput), vp, i64, vp, vp]
    lib.ist_sync_status.restype = ctypes.c_int32
    lib.ist_sync_status.argtypes = [vp]
    lib.ist_selftest_wait_expiry.restype = ctypes.c_int32
    lib.ist_selftest_wait_expiry.argtypes = [vp, i64]
    lib.ist_kernel_launches.restype = i64
    lib.ist_kernel_launches.argtypes = [vp]
    lib.ist_last_error.restype = ctypes.c_char_p
    lib.ist_last_error.argtypes = [vp]
    lib.ist_profile.restype = ctypes.c_int32
    lib.ist_profile.argtypes = [vp, i32]
    lib.ist_profile_read.restype = ctypes.c_int32
    lib.ist_profile_read.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double)]
    lib.ist_partition_layer_static.restype = ctypes.c_int32
    lib.ist_partition_layer_static.argtypes = [u64, i32, i64, i32, vp, vp, vp]
    lib.ist_destroy.restype = None
    lib.ist_norm_workspace_bytes.argtypes = [vp]
    lib.ist_norm_workspace_bytes.restype = sz
    lib.ist_enable_normalization.argtypes = [vp, ctypes.c_float, vp, sz]
    lib.ist_enable_normalization.restype = i32
    lib.ist_calibrate.argtypes = [vp, ctypes.POINTER(IstInput), i64]
    lib.ist_calibrate.restype = i32
    lib.ist_set_subnet_range.argtypes = [vp, i32, i32]
    lib.ist_set_subnet_range.restype = i32
    lib.ist_packed_layer.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(sz), ctypes.POINTER(vp),
                                     ctypes.POINTER(sz)]
    lib.ist_packed_layer.restype = i32
    lib.ist_destroy.argtypes = [vp]
    f32 = ctypes.c_float
    lib.ist_layer_norm_forward.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp, f32, vp, i32, i64, vp, vp, vp]
    lib.ist_layer_norm_forward.restype = ctypes.c_int32
    lib.ist_layer_norm_workspace_bytes.argtypes = [i64, i64, i32]
    lib.ist_layer_norm_workspace_bytes.restype = sz
    lib.ist_layer_norm_backward.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, i32, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.ist_layer_norm_backward.restype = ctypes.c_int32
    lib.ist_layer_norm_status.argtypes = [vp]
    lib.ist_layer_norm_status.restype = ctypes.c_int32
    lib.ist_selftest_layer_norm_wait.argtypes = [vp, vp, vp, i64, i64, vp, i64, vp]
    lib.ist_selftest_layer_norm_wait.restype = ctypes.c_int32
    lib.ist_adamw_workspace_bytes.argtypes = [i64]
    lib.ist_adamw_workspace_bytes.restype = sz
    lib.ist_adamw_step.argtypes = [vp, i64, ctypes.POINTER(AdamWArgs), vp, sz, vp]
    lib.ist_adamw_step.restype = ctypes.c_int32
    lib.ist_adamw_state_values.argtypes = [vp, vp, vp, vp, i64, i32, vp, vp, vp]
    lib.ist_adamw_state_values.restype = ctypes.c_int32
    return lib


lib = _load()


def _dims(layer_dims: Sequence[int]):
    arr = (ctypes.c_int64 * len(layer_dims))(*[int(d) for d in layer_dims])
    return arr, len(layer_dims)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _check(handle, status: int):
    if status != IST_OK:
        raise IstError(status, lib.ist_last_error(handle).decode())


def ist_workspace_bytes2(layer_dims, S, precision, max_batch, input_is_csr=False, partition_rule=0) -> int:
    arr, n = _dims(layer_dims)
    return int(lib.ist_workspace_bytes2(arr, n, S, precision, max_batch, int(bool(input_is_csr)), partition_rule))


def ist_workspace_bytes(layer_dims, S, precision, max_batch, input_is_csr=False) -> int:
    arr, n = _dims(layer_dims)
    return int(lib.ist_workspace_bytes(arr, n, S, precision, max_batch, int(bool(input_is_csr))))


def make_input(X, batch: int, stride_subnet: int, stride_step: int) -> Tuple[IstInput, tuple]:
    """X: a CUDA tensor of rows (fp32 or bf16, last dim N_0) or a (row_ptr, col, val) triple of
    CUDA tensors (int32, int32, fp32).  Returns the struct and the tensors it points into."""
    inp = IstInput()
    inp.batch = int(batch)
    inp.stride_subnet = int(stride_subnet)
    inp.stride_step = int(stride_step)
    if isinstance(X, (tuple, list)):
        rp, col, val = X
        assert rp.dtype == torch.int32 and col.dtype == torch.int32 and val.dtype == torch.float32
        assert rp.is_cuda and col.is_cuda and val.is_cuda
        inp.kind = IST_X_CSR
        inp.row_ptr, inp.col, inp.val = rp.data_ptr(), col.data_ptr(), val.data_ptr()
        return inp, (rp, col, val)
    assert X.is_cuda and X.is_contiguous()
    if X.dtype == torch.float32:
        inp.kind = IST_X_DENSE_F32
    elif X.dtype == torch.bfloat16:
        inp.kind = IST_X_DENSE_BF16
    else:
        raise TypeError(f"unsupported input dtype {X.dtype}")
    inp.dense = X.data_ptr()
    return inp, (X,)


def ist_partition_layer_static(seed: int, hidden_layer: int, n_neurons: int, S: int,
                               idx_out: torch.Tensor, off_out: torch.Tensor,
                               stream: Optional[torch.cuda.Stream] = None) -> int:
    """Partition of one hidden layer into caller-owned int32 tensors, using the library's built-in
    device scratch instead of a workspace (for callers that must not allocate).  Returns the
    ist_status; work is asynchronous on `stream` (default: the current stream of idx_out's device)."""
    assert idx_out.is_cuda and idx_out.dtype == torch.int32 and idx_out.numel() >= n_neurons
    assert off_out.is_cuda and off_out.dtype == torch.int32 and off_out.numel() >= S + 1
    with torch.cuda.device(idx_out.device):
        s = stream if stream is not None else torch.cuda.current_stream(idx_out.device)
        return int(lib.ist_partition_layer_static(ctypes.c_uint64(seed & (2 ** 64 - 1)), hidden_layer, n_neurons, S,
                                                  idx_out.data_ptr(), off_out.data_ptr(),
                                                  ctypes.c_void_p(s.cuda_stream)))


def ist_static_partition_status(stream: Optional[torch.cuda.Stream] = None, device=None) -> int:
    """Waits for `stream` and returns the device status word of ist_partition_layer_static's kernels
    on the current device (IST_OK unless one of their bounds checks tripped)."""
    dev = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
    with torch.cuda.device(dev):
        s = stream if stream is not None else torch.cuda.current_stream(dev)
        return int(lib.ist_static_partition_status(ctypes.c_void_p(s.cuda_stream)))


class Ist:
    """One IST context: owns the workspace tensor, borrows the full network's tensors.

    Method names mirror the C calls (ist_partition -> partition, ...)."""

    def __init__(self, layer_dims: Sequence[int], S: int, precision: int, max_batch: int,
                 input_is_csr: bool = False, device: str = "cuda:0", stream: Optional[torch.cuda.Stream] = None,
                 partition_rule: int = IST_PART_BALANCED):
        self.partition_rule = int(partition_rule)
        self.layer_dims = [int(d) for d in layer_dims]
        self.t = len(self.layer_dims) - 1
        self.S, self.precision, self.max_batch = int(S), int(precision), int(max_batch)
        self.input_is_csr = bool(input_is_csr)
        self.device = torch.device(device)
        self.stream = stream
        self.handle = ctypes.c_void_p()
        nbytes = ist_workspace_bytes2(self.layer_dims, S, precision, max_batch, input_is_csr, self.partition_rule)
        if nbytes == 0:
            raise IstError(IST_ERR_ARG, lib.ist_last_error(None).decode())
        self.workspace_bytes = nbytes
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            arr, n = _dims(self.layer_dims)
            st = lib.ist_create2(ctypes.byref(self.handle), arr, n, self.S, self.precision, self.max_batch,
                                 int(self.input_is_csr), self.partition_rule, self.workspace.data_ptr(), nbytes,
                                 self._stream_ptr())
        if st != IST_OK:
            self.handle = ctypes.c_void_p()
            raise IstError(st, lib.ist_last_error(None).decode())
        self.W: List[torch.Tensor] = []
        self.b: List[torch.Tensor] = []

    def _stream_ptr(self):
        s = self.stream if self.stream is not None else torch.cuda.current_stream(self.device)
        return ctypes.c_void_p(s.cuda_stream)

    def close(self):
        if getattr(self, "handle", None) and self.handle.value:
            lib.ist_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # --- calls -----------------------------------------------------------------------------
    def bind_weights(self, W: Sequence[torch.Tensor], b: Sequence[torch.Tensor]):
        assert len(W) == self.t and len(b) == self.t
        for l in range(self.t):
            assert W[l].is_cuda and W[l].dtype == torch.float32 and W[l].is_contiguous()
            assert tuple(W[l].shape) == (self.layer_dims[l], self.layer_dims[l + 1])
            assert b[l].is_cuda and b[l].dtype == torch.float32 and tuple(b[l].shape) == (self.layer_dims[l + 1],)
        self.W, self.b = list(W), list(b)
        Wp = (ctypes.c_void_p * self.t)(*[w.data_ptr() for w in W])
        bp = (ctypes.c_void_p * self.t)(*[v.data_ptr() for v in b])
        _check(self.handle, lib.ist_bind_weights(self.handle, Wp, bp))

    def partition(self, seed: int):
        _check(self.handle, lib.ist_partition(self.handle, ctypes.c_uint64(seed & (2 ** 64 - 1))))

    def get_partition(self, hidden_layer: int):
        idx = torch.empty(self.layer_dims[hidden_layer], dtype=torch.int32, device=self.device)
        off = torch.empty(self.S + 1, dtype=torch.int32, device=self.device)
        _check(self.handle, lib.ist_get_partition(self.handle, hidden_layer, idx.data_ptr(), off.data_ptr()))
        return idx, off

    def subnet_slice_shape(self, layer: int, s: int) -> Tuple[int, int]:
        """(rows, cols) of subnet s's slice of layer `layer` under the partition in place."""
        rows, cols = ctypes.c_int64(), ctypes.c_int64()
        _check(self.handle, lib.ist_subnet_slice_shape(self.handle, layer, s, ctypes.byref(rows), ctypes.byref(cols)))
        return int(rows.value), int(cols.value)

    def get_subnet_params(self, layer: int, s: int):
        rows, cols = self.subnet_slice_shape(layer, s)
        Wt = torch.empty((rows, cols), dtype=torch.float32, device=self.device)
        bt = torch.empty(cols, dtype=torch.float32, device=self.device)
        _check(self.handle, lib.ist_get_subnet_params(self.handle, layer, s, Wt.data_ptr(), bt.data_ptr()))
        return Wt, bt

    def local_steps(self, X, y: torch.Tensor, lr: float, K: int, batch: int,
                    stride_subnet: Optional[int] = None, stride_step: Optional[int] = None,
                    loss_out: Optional[torch.Tensor] = None, want_loss: bool = True,
                    dx_out: Optional[torch.Tensor] = None):
        """X rows ordered [S][K][batch] by default (stride_subnet = K*batch, stride_step = batch).
        dx_out: fp32 [rows of X][N_0], receives the loss gradient with respect to every input row
        (ist_local_steps_dx)."""
        if stride_subnet is None:
            stride_subnet = K * batch
        if stride_step is None:
            stride_step = batch
        inp, keep = make_input(X, batch, stride_subnet, stride_step)
        assert y.is_cuda and y.dtype == torch.int32 and y.is_contiguous()
        n_sub = getattr(self, "sub_count", self.S)
        if loss_out is None and want_loss:
            loss_out = torch.empty(n_sub * K, dtype=torch.float32, device=self.device)
        if dx_out is not None:
            assert dx_out.is_cuda and dx_out.dtype == torch.float32 and dx_out.is_contiguous()
            _check(self.handle, lib.ist_local_steps_dx(self.handle, ctypes.byref(inp), y.data_ptr(),
                                                       ctypes.c_float(lr), K, _ptr(loss_out), dx_out.data_ptr()))
        else:
            _check(self.handle, lib.ist_local_steps(self.handle, ctypes.byref(inp), y.data_ptr(),
                                                    ctypes.c_float(lr), K, _ptr(loss_out)))
        return loss_out.view(n_sub, K) if loss_out is not None else None

    def reassemble(self):
        _check(self.handle, lib.ist_reassemble(self.handle))

    def eval(self, X, y: torch.Tensor, n: int):
        inp, keep = make_input(X, 0, 0, 0)
        loss = torch.empty(1, dtype=torch.float32, device=self.device)
        correct = torch.empty(1, dtype=torch.int64, device=self.device)
        _check(self.handle, lib.ist_eval(self.handle, ctypes.byref(inp), y.data_ptr(), n,
                                         loss.data_ptr(), correct.data_ptr()))
        return loss, correct

    def set_subnet_range(self, first: int, count: int):
        """Train only subnets first .. first+count-1 in local_steps (the others are trained elsewhere)."""
        _check(self.handle, lib.ist_set_subnet_range(self.handle, first, count))
        self.sub_first, self.sub_count = first, count

    def packed_layer(self, layer: int):
        """(master [S][elems] fp32, bias [S][ld] fp32): views of the workspace, for the slice exchange."""
        mp, mb, bp, bb = ctypes.c_void_p(), ctypes.c_size_t(), ctypes.c_void_p(), ctypes.c_size_t()
        _check(self.handle, lib.ist_packed_layer(self.handle, layer, ctypes.byref(mp), ctypes.byref(mb),
                                                 ctypes.byref(bp), ctypes.byref(bb)))
        base = self.workspace.data_ptr()

        def view(ptr, nbytes):
            off = ptr.value - base
            return self.workspace[off:off + self.S * nbytes].view(torch.float32).view(self.S, nbytes // 4)

        return view(mp, mb.value), view(bp, bb.value)

    def enable_normalization(self, eps: float):
        """Sec. 2.2 batch standardisation of the hidden layers for all later calls."""
        nbytes = int(lib.ist_norm_workspace_bytes(self.handle))
        with torch.cuda.device(self.device):
            self.norm_workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(self.handle, lib.ist_enable_normalization(self.handle, ctypes.c_float(eps),
                                                         self.norm_workspace.data_ptr(), nbytes))

    def calibrate(self, X, n: int):
        inp, keep = make_input(X, 0, 0, 0)
        _check(self.handle, lib.ist_calibrate(self.handle, ctypes.byref(inp), n))

    def sync_status(self):
        _check(self.handle, lib.ist_sync_status(self.handle))

    def selftest_wait_expiry(self, limit_cycles: int):
        """Enqueues a kernel whose bounded wait must expire; sync_status() then raises with
        IST_ERR_DEVICE_TIMEOUT."""
        _check(self.handle, lib.ist_selftest_wait_expiry(self.handle, int(limit_cycles)))

    def profile(self, enable: bool):
        _check(self.handle, lib.ist_profile(self.handle, int(bool(enable))))

    def profile_read(self):
        """{class name: (kernels launched, device milliseconds)} since profiling was enabled."""
        out = {}
        for k, name in enumerate(KERNEL_CLASSES):
            n, ms = ctypes.c_int64(), ctypes.c_double()
            _check(self.handle, lib.ist_profile_read(self.handle, k, ctypes.byref(n), ctypes.byref(ms)))
            out[name] = (int(n.value), float(ms.value))
        return out

    def kernel_launches(self) -> int:
        return int(lib.ist_kernel_launches(self.handle))

    # --- one whole round ---------------------------------------------------------------------
    def round(self, seed: int, X, y, lr: float, K: int, batch: int, loss_out=None, want_loss=True):
        self.partition(seed)
        loss = self.local_steps(X, y, lr, K, batch, loss_out=loss_out, want_loss=want_loss)
        self.reassemble()
        return loss


# --- operators for a trunk in front of the partitioned layers: no context -------------------------------

_TYPES = {torch.float32: IST_T_F32, torch.bfloat16: IST_T_BF16}


def _refuse(message: str):
    raise IstError(IST_ERR_ARG, message)


_Tensor, _dtype_of = torch._C.TensorBase, operator.attrgetter("dtype")
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(index: int, function, *args):
    """function(*args, stream) with device `index` current, on that device's current stream."""
    if index != _current_device():
        with torch.cuda.device(index):
            return _call(index, function, *args)
    status = function(*args, _raw_stream(index))
    if status != IST_OK:
        raise IstError(status, lib.ist_last_error(None).decode())


def _written(tensors: Sequence[torch.Tensor]) -> None:
    """Tells autograd of a call's writes: a graph that still needs the old values raises an error when it gets there."""
    torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


def _on(stream: torch.cuda.Stream, tensor: torch.Tensor):
    """Makes `stream` current: what a call allocates then belongs to the stream that it runs on."""
    if stream.device != tensor.device:
        _refuse(f"the stream belongs to another device than {tensor.device}")
    return torch.cuda.stream(stream)


def _rows(t: torch.Tensor, name: str, cols: int, index: int, rows: int = -1) -> Tuple[int, int, int]:
    """(element type, rows, stride) of a tensor whose last dimension is `cols` elements that lie together."""
    if t.get_device() != index or index < 0:
        _refuse(f"{name} is on {t.device}: one CUDA device for all tensors is needed")
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"unsupported dtype {t.dtype} of {name}")
    if t.dim() == 0 or t.shape[-1] != cols or (cols > 1 and t.stride(-1) != 1 and t.numel()):
        _refuse(f"{name}'s last dimension must be {cols} adjacent elements")
    n = t.numel() // cols
    if rows >= 0 and n != rows:
        _refuse(f"{name} has {n} rows, not {rows}")
    if n <= 1 or t.is_contiguous():
        return kind, n, cols
    if t.dim() != 2:
        try:
            t = t.view(-1, cols)
        except RuntimeError:
            _refuse(f"{name}'s leading dimensions have no common stride")
    return kind, n, t.stride(0)


def _vector(t: Optional[torch.Tensor], name: str, count: int, index: int) -> Optional[int]:
    if t is None:
        return None
    if t.get_device() != index or t.dtype != torch.float32 or t.numel() != count or not t.is_contiguous():
        _refuse(f"{name} must be {count} contiguous fp32 values on the rows' device")
    return t.data_ptr()


def _norm_shape(x: torch.Tensor, groups: int) -> Tuple[int, int]:
    if x.dim() == 0 or x.shape[-1] == 0:
        _refuse("x needs a last dimension of at least one element")
    if not 1 <= groups < 2 ** 31:
        _refuse("groups must be in 1..2^31 - 1")
    return x.shape[-1], x.get_device()


def _like(x: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """An uninitialised contiguous tensor of x's shape."""
    if x.is_contiguous():
        return torch.empty_like(x) if dtype is None or dtype == x.dtype else torch.empty_like(x, dtype=dtype)
    return torch.empty(x.shape, dtype=dtype if dtype is not None else x.dtype, device=x.device)


def ist_layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                           eps: float = 1e-5, groups: int = 1, y: Optional[torch.Tensor] = None,
                           y_dtype: Optional[torch.dtype] = None, want_stats: bool = True,
                           stream: Optional[torch.cuda.Stream] = None):
    """Layer norm over x's last dimension (fp32 or bf16; rows may have a stride).  weight, bias: fp32 [groups][cols], the
    rows belong in order to `groups` sites.  Returns (y, mean, rstd), y of y_dtype (default x's) or written into the tensor
    `y`; mean and rstd are fp32 [rows], or None without want_stats.  Runs on `stream` or the device's current stream."""
    if stream is not None:
        with _on(stream, x):
            return ist_layer_norm_forward(x, weight, bias, eps, groups, y, y_dtype, want_stats)
    cols, index = _norm_shape(x, groups)
    x_type, rows, x_stride = _rows(x, "x", cols, index)
    given = y is not None
    if not given:
        y = _like(x, y_dtype)
        y_type, y_stride = _TYPES.get(y.dtype, -1), cols
        if y_type < 0:
            raise TypeError(f"unsupported dtype {y.dtype} of y")
    else:
        if y_dtype is not None and y.dtype != y_dtype:
            _refuse(f"y is {y.dtype}, not {y_dtype}")
        y_type, _, y_stride = _rows(y, "y", cols, index, rows)
    mean = rstd = mean_at = rstd_at = None
    if want_stats:
        mean = torch.empty(rows, dtype=torch.float32, device=index)
        rstd = torch.empty_like(mean)                 # half the price of an empty() with arguments
        mean_at, rstd_at = mean.data_ptr(), rstd.data_ptr()
    _call(index, lib.ist_layer_norm_forward, x.data_ptr(), x_type, x_stride, rows, cols, groups,
          _vector(weight, "weight", groups * cols, index), _vector(bias, "bias", groups * cols, index), eps, y.data_ptr(), y_type,
          y_stride, mean_at, rstd_at)
    if given:
        _written([y])
    return y, mean, rstd


@functools.lru_cache(maxsize=1024)
def _norm_workspace(rows: int, cols: int, groups: int) -> int:
    return int(lib.ist_layer_norm_workspace_bytes(rows, cols, groups))


def ist_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                            rstd: torch.Tensor, groups: int = 1, want_dx: bool = True, want_dweight: bool = True,
                            want_dbias: bool = True, dx: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None):
    """(dx, dweight, dbias) from the gradient of ist_layer_norm_forward's output and what that call read and returned; dx
    has x's type (or is written into the tensor `dx`), the others are fp32 [groups][cols], None where not wanted."""
    if stream is not None:
        with _on(stream, x):
            return ist_layer_norm_backward(dy, x, weight, mean, rstd, groups, want_dx, want_dweight, want_dbias, dx)
    cols, index = _norm_shape(x, groups)
    x_type, rows, x_stride = _rows(x, "x", cols, index)
    dy_type, _, dy_stride = _rows(dy, "dy", cols, index, rows)
    dx_stride, given = cols, dx is not None
    if given:
        if dx.dtype != x.dtype:
            _refuse("dx must have x's dtype")
        _, _, dx_stride = _rows(dx, "dx", cols, index, rows)
    elif want_dx:
        dx = _like(x)
    dx_at = dweight_at = dbias_at = workspace_at = dweight = dbias = None
    nbytes = 0
    if dx is not None:
        dx_at = dx.data_ptr()
    if want_dweight:
        dweight = torch.empty((groups, cols), dtype=torch.float32, device=index)
        dweight_at = dweight.data_ptr()
    if want_dbias:
        dbias = torch.empty_like(dweight) if want_dweight else torch.empty((groups, cols), dtype=torch.float32, device=index)
        dbias_at = dbias.data_ptr()
    if want_dweight or want_dbias:
        nbytes = _norm_workspace(rows, cols, groups)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=index)
            workspace_at = workspace.data_ptr()
    _call(index, lib.ist_layer_norm_backward, dy.data_ptr(), dy_type, dy_stride, x.data_ptr(), x_type, x_stride, rows, cols, groups,
          _vector(weight, "weight", groups * cols, index), _vector(mean, "mean", rows, index),
          _vector(rstd, "rstd", rows, index), dx_at, dx_stride, dweight_at, dbias_at, workspace_at, nbytes)
    if given:
        _written([dx])
    return dx, dweight, dbias


def ist_layer_norm_status(stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for `stream` (default: the current one) and raises an IstError (IST_ERR_DEVICE_TIMEOUT) if a wait of layer norm's
    kernels on its device gave up since this was last called; the rows concerned hold NaN."""
    with torch.cuda.stream(stream):
        _call(_current_device(), lib.ist_layer_norm_status)


def _cuda_device(t: torch.Tensor, name: str) -> torch.device:
    if t.device.type != "cuda":
        _refuse(f"{name} are on {t.device}: a CUDA device is needed")
    return t.device


class AdamW:
    """AdamW over a list of fp32 tensors, one ist_adamw_step per step(): borrows the parameters (and their bf16 operand
    `copies`, where given) and owns the states, unless they are handed in.

    state: {"exp_avg", "exp_avg_sq"} and with state_bits = 8 {"exp_avg_base", "exp_avg_sq_base"}: flat tensors in which
    tensor i starts at offsets[i], a multiple of IST_ADAMW_BLOCK values; zeros before the first step.
    A step looks where its tensors lie: parameters, copies and entries of `state` may be given other storage of the same size
    and type (Module.to and back, `p.data = ...`, a loaded state) between steps; a captured step keeps the storage of its capture.
    weight_decay: a number, or one per tensor.  max_norm: bound of the global gradient norm (None: no clipping).
    step: steps taken so far.  step_dev (int64 [1]), lr_dev (fp32 [1]): device scalars that replace the host's step and lr,
    for steps that are captured into a graph; step() then adds one to step_dev on the stream before the update.
    A step runs on `stream` or on the device's current stream.  With `stream` the object's own states and workspace belong to that
    stream from the start; without it, to the stream that is current at construction, and steps on another one have to be ordered
    behind it.  What the caller hands in (parameters, copies, states, gradients) the caller orders before a step's stream.  The
    object has to outlive the graphs that captured its steps."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, weight_decay=0.01, state_bits: int = 32, max_norm: Optional[float] = None,
                 copies: Optional[Sequence[torch.Tensor]] = None, state: Optional[dict] = None, seed: int = 0, step: int = 0,
                 step_dev: Optional[torch.Tensor] = None, lr_dev: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None):
        self.params, self.copies = list(params), None if copies is None else list(copies)
        if not self.params:
            _refuse("no parameters")
        dev = self.device = _cuda_device(self.params[0], "parameters")
        self.index = self.params[0].get_device()
        if state_bits not in (8, 32):
            _refuse("state_bits is 32 or 8")
        self.lr, self.steps, self.stream = float(lr), int(step), stream
        if stream is not None and stream.device != dev:
            _refuse(f"the stream belongs to another device than {dev}")
        self.sizes = [p.numel() for p in self.params]
        room = [-(-n // IST_ADAMW_BLOCK) * IST_ADAMW_BLOCK for n in self.sizes]
        self.offsets = [0]
        for r in room:
            self.offsets.append(self.offsets[-1] + r)
        total = self.offsets.pop()
        names = ["exp_avg", "exp_avg_sq"] + (["exp_avg_base", "exp_avg_sq_base"] if state_bits == 8 else [])
        self.shapes = {n: (torch.int16, total // IST_ADAMW_BLOCK) if n.endswith("base") else
                       (torch.uint8 if state_bits == 8 else torch.float32, total) for n in names}
        if state is None:
            with torch.cuda.stream(stream):             # the steps' stream: its first reads come after these writes
                state = {n: torch.zeros(size, dtype=dtype, device=dev) for n, (dtype, size) in self.shapes.items()}
        self.state = dict(state)
        decay = [float(weight_decay)] * len(self.params) if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
        if len(decay) != len(self.params):
            _refuse("one weight decay per parameter is needed")
        self.table = np.zeros(len(self.params), ADAMW_TENSOR)
        self.table["n"], self.table["weight_decay"] = self.sizes, decay
        self.table_at, self.words = self.table.ctypes.data, memoryview(self.table.view(np.uint64)).cast("B").cast("Q")
        self.step_dev, self.lr_dev = step_dev, lr_dev
        self.args = AdamWArgs(lr=self.lr, beta1=betas[0], beta2=betas[1], eps=eps, max_norm=max_norm or 0.0,
                              seed=seed & (2 ** 64 - 1), state_bits=state_bits)
        self._bind()
        self.workspace = None
        self.workspace_bytes = int(lib.ist_adamw_workspace_bytes(len(self.params))) if max_norm else 0
        if max_norm:
            with torch.cuda.stream(stream):
                self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=dev)
                self.norm_like = torch.empty(1, dtype=torch.float32, device=dev)

    def _tensors(self) -> List[torch.Tensor]:
        """Everything whose address a step hands to the library, but for the gradients."""
        tensors = [*self.params, *self.state.values()]
        if self.copies is not None:
            tensors += self.copies
        if self.step_dev is not None:
            tensors.append(self.step_dev)
        if self.lr_dev is not None:
            tensors.append(self.lr_dev)
        return tensors

    def _bind(self) -> None:
        """Checks the tensors and notes where they lie."""
        dev, params, copies, state = self.device, self.params, self.copies, self.state
        if set(state) != set(self.shapes):
            _refuse(f"state needs {list(self.shapes)}")
        for n, (dtype, size) in self.shapes.items():
            t = state[n]
            if t.device != dev or t.dtype != dtype or tuple(t.shape) != (size,) or not t.is_contiguous():
                _refuse(f"state {n} must be {size} contiguous values of {dtype} on {dev}")
        if len(params) != len(self.sizes):
            _refuse(f"{len(params)} parameters, not {len(self.sizes)}")
        if copies is not None and len(copies) != len(params):
            _refuse("one copy per parameter is needed")
        for name, tensors, dtype in (("parameter", params, torch.float32), ("copy", copies or [], torch.bfloat16)):
            for i, t in enumerate(tensors):
                if t.device != dev or t.dtype != dtype or t.numel() != self.sizes[i] or not t.is_contiguous():
                    _refuse(f"{name} {i} must be {self.sizes[i]} contiguous values of {dtype} on {dev}")
        for name, t, dtype in (("step_dev", self.step_dev, torch.int64), ("lr_dev", self.lr_dev, torch.float32)):
            if t is not None and (t.device != dev or t.dtype != dtype or t.numel() != 1):
                _refuse(f"{name} must be one value of {dtype} on {dev}")
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())
                       for t in [*params, *(copies or ()), *state.values()] if t.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            _refuse("parameters, copies and states must not overlap")
        self.table["param"] = [p.data_ptr() for p in params]
        for n in self.shapes:
            base, size, per = state[n].data_ptr(), state[n].element_size(), IST_ADAMW_BLOCK if n.endswith("base") else 1
            self.table[n] = [base + o // per * size for o in self.offsets]
        self.table["param_bf16"] = 0 if copies is None else [c.data_ptr() for c in copies]
        self.args.step_dev, self.args.lr_dev = _ptr(self.step_dev), _ptr(self.lr_dev)
        tensors = self._tensors()
        self.written = [t for t in [*params, *(copies or ()), *state.values()] if not t.is_inference()]
        self.held, self.state_sizes = list(map(_Tensor.data_ptr, tensors)), [t.numel() for t in state.values()]
        # a storage that goes away leaves its reference here: as long as none has, an address that is the same is the same memory
        self.freed: list = []
        self.watched = [weakref.ref(t.untyped_storage(), self.freed.append) for t in tensors]

    def _follow(self) -> None:
        """Takes over tensors that have moved since the last look."""
        if (self.freed or list(map(_Tensor.data_ptr, self._tensors())) != self.held
                or list(map(_Tensor.numel, self.state.values())) != self.state_sizes):
            self._bind()

    def step(self, grads: Optional[Sequence[Optional[torch.Tensor]]] = None, lr: Optional[float] = None) -> Optional[torch.Tensor]:
        """One step with `grads` (default: the parameters' .grad), all fp32 or all bf16; a None passes its tensor over.
        They may overlap one another but no parameter, copy or state, except that one may be its own parameter.
        Returns the gradients' norm (fp32 [1]) if they are clipped.  The gradients may be freed or written once the
        work on the stream that follows allows it, as with any asynchronous call."""
        if self.stream is not None and _raw_stream(self.index) != self.stream.cuda_stream:
            with torch.cuda.stream(self.stream):
                return self.step(grads, lr)
        if grads is None:
            grads = [p.grad for p in self.params]
        if len(grads) != len(self.sizes):
            _refuse("one gradient (or None) per parameter is needed")
        self._follow()
        index, dtype = self.index, None
        try:                                            # the table's second word of nine is the gradient's address
            self.words[1::9] = array("Q", map(_Tensor.data_ptr, grads))
            given, sizes = grads, self.sizes
        except TypeError:                               # there is a None among them
            given = [g for g in grads if g is not None]
            sizes = [n for g, n in zip(grads, self.sizes) if g is not None]
            self.words[1::9] = array("Q", [0 if g is None else g.data_ptr() for g in grads])
        if given:
            dtype = given[0].dtype
            if (list(map(_Tensor.numel, given)) != sizes or not all(map(_Tensor.is_contiguous, given))
                    or set(map(_Tensor.get_device, given)) != {index} or len(set(map(_dtype_of, given))) != 1):
                _refuse(f"gradients must be contiguous, of their parameters' sizes, of one dtype and on {self.device}")
        kind = IST_T_F32 if dtype is None else _TYPES.get(dtype)
        if kind is None:
            raise TypeError(f"unsupported gradient dtype {dtype}")
        args = self.args
        args.grad_type = kind
        rate = self.lr if lr is None else float(lr)
        args.lr, args.step = rate, self.steps + 1
        norm = workspace_at = None
        if self.workspace is not None:
            workspace_at = self.workspace.data_ptr()
            norm = torch.empty_like(self.norm_like)     # half the price of an empty() with arguments
            args.norm_out_dev = norm.data_ptr()
        if self.step_dev is not None:
            self.step_dev.add_(1)
        try:
            _call(index, lib.ist_adamw_step, self.table_at, len(self.sizes), args, workspace_at, self.workspace_bytes)
        except IstError:
            if self.step_dev is not None:               # a refused step is no step
                self.step_dev.sub_(1)
            raise
        self.steps += 1
        self.lr = rate
        torch.autograd.graph.increment_version(self.written)    # a graph that still needs the old values is told
        return norm

    def state_values(self, dtype: torch.dtype = torch.float32) -> Tuple[torch.Tensor, torch.Tensor]:
        """First and second moments as flat tensors of `dtype` (fp32 or bf16), tensor i from offsets[i] on."""
        if dtype not in _TYPES:
            raise TypeError(f"unsupported dtype {dtype}")
        if self.stream is not None and _raw_stream(self.index) != self.stream.cuda_stream:
            with torch.cuda.stream(self.stream):
                return self.state_values(dtype)
        self._follow()
        m, v = self.state["exp_avg"], self.state["exp_avg_sq"]
        if "exp_avg_base" not in self.state:
            return m.to(dtype, copy=True), v.to(dtype, copy=True)
        a, b = torch.empty_like(m, dtype=dtype), torch.empty_like(v, dtype=dtype)
        _call(self.index, lib.ist_adamw_state_values, m.data_ptr(), self.state["exp_avg_base"].data_ptr(), v.data_ptr(),
              self.state["exp_avg_sq_base"].data_ptr(), m.numel(), _TYPES[dtype], a.data_ptr(), b.data_ptr())
        return a, b
