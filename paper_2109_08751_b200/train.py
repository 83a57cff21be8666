"""ctypes binding of include/sparbit_train.h: argument marshalling only.

Operators of a training step whose state is divided over the ranks of a communicator.  Tensors are torch
tensors in device (or pinned host) memory, whose type has to be the operator's (TypeError); numpy arrays,
addresses and other objects with `data_ptr()` are taken as they are.  Row strides (`*_ld`, in elements)
default to the row's width, which a tensor with gaps between its rows does not have (ValueError: give its
stride); a view that no row stride describes (heads apart from one another, a padded batch) is a ValueError, too.  Everything runs in the library's CUDA kernels; there is no fallback.
"""
from __future__ import annotations

import ctypes

from .binding import ERR_TIMEOUT, OK, SparbitError, _i, _sz, _vp, lib
from .binding import _ptr as _address

F32, BF16, F16 = range(3)
PRODUCTS_AUTO, PRODUCTS_ONE, PRODUCTS_THREE = 0, 1, 3
ROUTER_MAX_EXPERTS, ROUTER_MAX_K = 1024, 32
LINEAR_ATTENTION_MAX_SIZE, NORM_MAX_WIDTH = 128, 32768

_f = ctypes.c_float
_ps = ctypes.POINTER(_sz)
_pp = ctypes.POINTER(_vp)


class MuonArgs(ctypes.Structure):
    """sparbit_muon"""

    _fields_ = [("grad", _vp), ("grad_ld", _sz), ("grad_stride", _sz), ("momentum_in", _vp), ("momentum_out", _vp),
                ("momentum_ld", _sz), ("momentum_stride", _sz), ("weight_in", _vp), ("weight_out", _vp),
                ("weight_ld", _sz), ("weight_stride", _sz), ("weight_dtype", _i), ("nesterov", _i), ("lr", _f),
                ("momentum", _f), ("weight_decay", _f), ("scale", _f)]


#: every symbol include/sparbit_train.h declares, with (restype, argtypes)
SYMBOLS = {
    "sparbit_scan_plan_create": (_i, [_i, _ps, _sz, _i, _pp]),
    "sparbit_scan_plan_destroy": (_i, [_vp]),
    "sparbit_scan_plan_workspace_bytes": (_sz, [_vp]),
    "sparbit_scan_plan_carry_bytes": (_sz, [_vp]),
    "sparbit_scan_plan_set_workspace": (_i, [_vp, _vp, _sz]),
    "sparbit_scan_plan_status": (_i, [_vp]),
    "sparbit_scan_plan_set_wait_test": (_i, [_vp, _i, ctypes.c_uint64]),
    "sparbit_scan_forward": (_i, [_vp, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _vp]),
    "sparbit_scan_backward": (_i, [_vp, _vp, _sz, _vp, _sz, _vp, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp]),
    "sparbit_scan_step": (_i, [_sz, _sz, _i, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _sz, _vp, _sz, _vp]),
    "sparbit_scan_join": (_i, [_i, _i, _i, _sz, _vp, _vp, _vp, _sz, _i, _vp]),
    "sparbit_ortho_plan_create": (_i, [_i, _sz, _sz, _i, _i, ctypes.POINTER(_f), _f, _pp]),
    "sparbit_ortho_plan_destroy": (_i, [_vp]),
    "sparbit_ortho_plan_set_products": (_i, [_vp, _i]),
    "sparbit_ortho_plan_workspace_bytes": (_sz, [_vp]),
    "sparbit_ortho_plan_set_workspace": (_i, [_vp, _vp, _sz]),
    "sparbit_ortho_plan_status": (_i, [_vp]),
    "sparbit_ortho_plan_set_wait_test": (_i, [_vp, _i, ctypes.c_uint64]),
    "sparbit_orthogonalize": (_i, [_vp, _vp, _sz, _sz, _vp, _sz, _sz, _vp]),
    "sparbit_muon_step": (_i, [_vp, ctypes.POINTER(MuonArgs), _vp]),
    "sparbit_router_plan_create": (_i, [_i, _ps, _i, _i, _i, _i, _pp]),
    "sparbit_router_plan_destroy": (_i, [_vp]),
    "sparbit_router_plan_workspace_bytes": (_sz, [_vp]),
    "sparbit_router_plan_set_workspace": (_i, [_vp, _vp, _sz]),
    "sparbit_router_forward": (_i, [_vp, _vp, _sz, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sparbit_router_balance": (_i, [_vp, _vp, _i, _vp, _f, _f, _vp, _vp]),
    "sparbit_router_backward": (_i, [_vp, _vp, _sz, _vp, _vp, _vp, _vp, _vp, _i, _vp, _f, _f, _vp, _vp, _sz, _vp]),
    "sparbit_linear_attention_plan_create": (_i, [_i, _ps, _i, _i, _i, _i, _f, _pp]),
    "sparbit_linear_attention_plan_destroy": (_i, [_vp]),
    "sparbit_linear_attention_plan_workspace_bytes": (_sz, [_vp]),
    "sparbit_linear_attention_plan_set_workspace": (_i, [_vp, _vp, _sz]),
    "sparbit_linear_attention_plan_status": (_i, [_vp]),
    "sparbit_linear_attention_plan_set_wait_test": (_i, [_vp, _i, ctypes.c_uint64]),
    "sparbit_linear_attention_forward": (_i, [_vp, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _vp, _sz, _vp, _vp]),
    "sparbit_linear_attention_backward": (_i, [_vp, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _vp, _sz, _vp, _vp, _sz, _vp,
                                               _sz, _vp, _sz, _vp, _vp]),
    "sparbit_linear_attention_step": (_i, [_sz, _i, _i, _i, _i, _f, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _sz, _vp, _vp,
                                           _vp, _sz, _vp]),
    "sparbit_linear_attention_join": (_i, [_i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _i, _vp]),
    "sparbit_norm_plan_create": (_i, [_sz, _i, _i, _f, _i, _pp]),
    "sparbit_norm_plan_destroy": (_i, [_vp]),
    "sparbit_norm_plan_workspace_bytes": (_sz, [_vp]),
    "sparbit_norm_plan_set_workspace": (_i, [_vp, _vp, _sz]),
    "sparbit_norm_forward": (_i, [_vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _vp]),
    "sparbit_norm_backward": (_i, [_vp, _sz, _vp, _sz, _vp, _sz, _vp, _vp, _vp, _sz, _vp, _sz, _vp, _vp]),
    "sparbit_clip_plan_create": (_i, [_i, _sz, _ps, ctypes.POINTER(_i), ctypes.POINTER(_i), _pp]),
    "sparbit_clip_plan_destroy": (_i, [_vp]),
    "sparbit_clip_plan_workspace_bytes": (_sz, [_vp]),
    "sparbit_clip_plan_set_workspace": (_i, [_vp, _vp, _sz]),
    "sparbit_clip_plan_set_tensors": (_i, [_vp, _pp, _pp]),
    "sparbit_clip_sums": (_i, [_vp, _vp, _vp]),
    "sparbit_clip_scale": (_i, [_vp, _vp, _i, _f, _f, _vp, _vp]),
}
for _name, (_res, _args) in SYMBOLS.items():
    _fn = getattr(lib, _name)  # AttributeError here means the library does not match the header
    _fn.restype = _res
    _fn.argtypes = _args


def _words(name):
    """The function for arguments that are all integers and addresses, a machine word each: ctypes converts an int to
    void* faster than to size_t (a token's step 0.5 us), but nothing that only behaves like an int (numpy's), which
    raises ArgumentError and goes the declared way."""
    return ctypes.CFUNCTYPE(_i, *[_vp] * len(getattr(lib, name).argtypes))((name, lib))


_scan_step, _router_forward = _words("sparbit_scan_step"), _words("sparbit_router_forward")


# What a tensor has to be: device memory of the type that the kernels read, and without gaps where no row stride is
# given.  The calls below can be shorter than their own marshalling (a token's step takes the GPU 3 us), so the common
# cases come first, and the two shortest calls look at all their tensors in one go.
_I32, _BYTE, _F64, _E4M3 = 3, 4, 5, 6
_NAMES = {F32: "float32", BF16: "bfloat16", F16: "float16", _I32: "int32", _BYTE: "uint8 or bool", _F64: "float64",
          _E4M3: "float8_e4m3fn or uint8"}
_KNOWN = {"torch.float32": F32, "torch.bfloat16": BF16, "torch.float16": F16, "torch.int32": _I32, "torch.uint8": _BYTE,
          "torch.int8": _BYTE, "torch.bool": _BYTE, "torch.float64": _F64, "torch.float8_e4m3fn": _E4M3}
_codes = {}  # of the torch types met so far
_types = {}  # and the other way round


def _address_of(x, code):
    """Address of a tensor of the type `code` (None: any), or of anything binding._ptr knows."""
    if x is None:
        return None
    try:
        if (_codes[x.dtype] == code or code is None) and x.is_cuda:
            return x.data_ptr()
    except (AttributeError, KeyError):
        pass
    return _address_checked(x, code)


def _address_checked(x, code):
    if not (hasattr(x, "data_ptr") and hasattr(x, "dtype") and hasattr(x, "is_cuda")):
        return _address(x)  # a number, a numpy array, anything else with an address: the caller's word
    dtype = str(x.dtype)
    met = _codes[x.dtype] = _KNOWN.get(dtype, -1)
    _types[met] = x.dtype
    if code is not None and met != code and not (code == _E4M3 and dtype == "torch.uint8"):
        raise TypeError(f"a tensor of {_NAMES.get(code, code)} is wanted, not of {dtype}")
    if not (x.is_cuda or x.is_pinned()):
        raise TypeError("a tensor on the GPU is wanted")
    return x.data_ptr()


def _stride_of(x, ld, width, evenly=True):
    """The row stride: the one that is given, or the width for a tensor whose rows follow one another."""
    if ld is not None:
        return ld if x is None or _in_rows(x, width, evenly) else None
    return width if x is None or _dense(x) else None


def _in_rows(x, width, evenly=True):
    """True, or ValueError for a view that no row stride describes: `width` elements that do not follow one another (heads
    that lie apart, say), or (`evenly`) rows that do not lie equally far apart (a padded batch)."""
    try:
        if x.is_contiguous():
            return True
        sizes, strides = x.shape, x.stride()
    except AttributeError:
        return True
    if strides[-1:] == (1,):  # the usual parts of wider rows, plain or in heads
        if len(strides) == 2 and sizes[1] >= width:
            return True
        if len(strides) == 3 and sizes[2] == strides[1] and sizes[1] * sizes[2] == width:
            return True
    follow, at = 1, None  # elements of a row so far; behind those how far the next size's elements lie apart
    for size, stride in zip(reversed(sizes), reversed(strides)):
        if size == 1:
            continue
        if follow < width:
            if stride != follow:
                raise ValueError("the elements of a row have to follow one another, those of its heads too")
            follow *= size
        else:
            if evenly and at is not None and stride != at:
                raise ValueError("the rows have to lie equally far apart")
            at = stride * size
    return True


def _dense(x):
    """True, or ValueError for a tensor with gaps."""
    try:
        if x.is_contiguous():
            return True
    except AttributeError:
        return True
    raise ValueError("a tensor with gaps between its rows needs its row stride (*_ld)")


def _flat(x, code):
    """Address of an array that has no row stride."""
    if x is None:
        return None
    try:
        if (_codes[x.dtype] == code or code is None) and x.is_cuda and x.is_contiguous():
            return x.data_ptr()
    except (AttributeError, KeyError):
        pass
    return _address_checked(x, code) if _dense(x) else None


def _rows_of(x, code, ld, width):
    """Address of a tensor with the row stride `ld`, or of one without."""
    if ld is None:
        return _flat(x, code)
    address = _address_of(x, code)
    return address if x is None or _in_rows(x, width) else None


def _stream_handle(stream):
    if stream is None or isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(code: int, where: str) -> None:
    if code != OK:
        raise SparbitError(code, where)


class _TrainPlan:
    """What the plans of this header have in common."""

    _kind = ""

    def _create(self, *args) -> None:
        h = _vp()
        name = f"sparbit_{self._kind}_plan_create"
        _check(getattr(lib, name)(*args, ctypes.byref(h)), name)
        self._h = h
        self._workspace = None

    @property
    def workspace_bytes(self) -> int:
        return getattr(lib, f"sparbit_{self._kind}_plan_workspace_bytes")(self._h)

    def set_workspace(self, dev, nbytes: int) -> None:
        name = f"sparbit_{self._kind}_plan_set_workspace"
        _check(getattr(lib, name)(self._h, _flat(dev, None), nbytes), name)
        self._workspace = dev  # keep the owner alive

    def status(self) -> int:
        """Synchronises; OK or ERR_TIMEOUT (raises on other errors).  Plans with waits in their kernels."""
        name = f"sparbit_{self._kind}_plan_status"
        code = getattr(lib, name)(self._h)
        if code != ERR_TIMEOUT:
            _check(code, name)
        return code

    def set_wait_test(self, withhold: bool, timeout_ns: int = 0) -> None:
        """Test hook of the bounded waits inside the kernels.  Plans with waits in their kernels."""
        name = f"sparbit_{self._kind}_plan_set_wait_test"
        _check(getattr(lib, name)(self._h, int(bool(withhold)), timeout_ns), name)

    def destroy(self) -> None:
        if getattr(self, "_h", None):
            h, self._h = self._h, None
            name = f"sparbit_{self._kind}_plan_destroy"
            _check(getattr(lib, name)(h), name)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _counts(values):
    values = [int(v) for v in values]
    if any(v < 0 for v in values):
        raise ValueError("a length is negative")
    return len(values), (_sz * len(values))(*values)


class ScanPlan(_TrainPlan):
    """Gated linear recurrence over sequences of the given lengths (sparbit_scan_plan_create)."""

    _kind = "scan"

    def __init__(self, lengths, channels: int, dtype: int = BF16):
        n, arr = _counts(lengths)
        self._create(n, arr, channels, dtype)
        self.channels, self.dtype = channels, dtype

    @property
    def carry_bytes(self) -> int:
        return lib.sparbit_scan_plan_carry_bytes(self._h)

    def forward(self, gate, x, y, h0=None, summary=None, carry=None, stream=None, gate_ld=None, x_ld=None, y_ld=None,
                h0_ld=None) -> None:
        d, t = self.channels, self.dtype
        _check(lib.sparbit_scan_forward(self._h, _address_of(gate, t), _stride_of(gate, gate_ld, d), _address_of(x, t),
                             _stride_of(x, x_ld, d), _address_of(h0, F32), _stride_of(h0, h0_ld, d), _address_of(y, t),
                             _stride_of(y, y_ld, d), _flat(summary, F32), _flat(carry, None), _stream_handle(stream)),
               "sparbit_scan_forward")

    def backward(self, gate, x, carry, dy, dgate, dx, dlast=None, dsummary=None, stream=None, gate_ld=None, x_ld=None,
                 dy_ld=None, dgate_ld=None, dx_ld=None, dlast_ld=None) -> None:
        d, t = self.channels, self.dtype
        _check(lib.sparbit_scan_backward(self._h, _address_of(gate, t), _stride_of(gate, gate_ld, d), _address_of(x, t),
                              _stride_of(x, x_ld, d), _flat(carry, None), _address_of(dy, t), _stride_of(dy, dy_ld, d),
                              _address_of(dlast, F32), _stride_of(dlast, dlast_ld, d), _address_of(dgate, t),
                              _stride_of(dgate, dgate_ld, d), _address_of(dx, t), _stride_of(dx, dx_ld, d),
                              _flat(dsummary, F32), _stream_handle(stream)),
               "sparbit_scan_backward")


def scan_step(rows: int, channels: int, dtype: int, gate, x, state_in, state_out, y, slots=None, n_slots=None,
              stream=None, gate_ld=None, x_ld=None, y_ld=None, state_ld=None) -> None:
    """One token for each of `rows` running sequences; n_slots defaults to `rows`."""
    try:
        t, f = _types[dtype], _types[F32]
        usual = (gate.dtype is x.dtype is y.dtype is t and state_in.dtype is state_out.dtype is f
                 and gate.is_cuda and x.is_cuda and y.is_cuda and state_in.is_cuda and state_out.is_cuda
                 and (gate.is_contiguous() if gate_ld is None else _in_rows(gate, channels))
                 and (x.is_contiguous() if x_ld is None else _in_rows(x, channels))
                 and (y.is_contiguous() if y_ld is None else _in_rows(y, channels))
                 and (state_in.is_contiguous() and state_out.is_contiguous() if state_ld is None
                      else _in_rows(state_in, channels) and _in_rows(state_out, channels)))
    except (AttributeError, KeyError):
        usual = False
    if usual:
        gate, x, y, state_in, state_out = (gate.data_ptr(), x.data_ptr(), y.data_ptr(), state_in.data_ptr(),
                                           state_out.data_ptr())
    else:
        gate, x, y = _rows_of(gate, dtype, gate_ld, channels), _rows_of(x, dtype, x_ld, channels), _rows_of(y, dtype, y_ld, channels)
        state_in, state_out = _rows_of(state_in, F32, state_ld, channels), _rows_of(state_out, F32, state_ld, channels)
    d = channels
    args = (rows, d, dtype, gate, d if gate_ld is None else gate_ld, x, d if x_ld is None else x_ld, _flat(slots, _I32),
            rows if n_slots is None else n_slots, state_in, state_out, d if state_ld is None else state_ld, y,
            d if y_ld is None else y_ld, _stream_handle(stream))
    try:
        code = _scan_step(*args)
    except ctypes.ArgumentError:
        code = lib.sparbit_scan_step(*args)
    if code != OK:
        raise SparbitError(code, "sparbit_scan_step")


def scan_join(P: int, channels: int, gathered, out, h0=None, reverse: bool = False, first_rank: int = 0,
              n_ranks=None, out_ld=None, stream=None) -> None:
    """First states of the slices first_rank .. first_rank + n_ranks - 1 (default: all P)."""
    _check(lib.sparbit_scan_join(P, first_rank, P if n_ranks is None else n_ranks, channels,
                                 _flat(gathered, F32), _flat(h0, F32), _address_of(out, F32),
                                 _stride_of(out, out_ld, channels), int(bool(reverse)), _stream_handle(stream)),
           "sparbit_scan_join")


class RouterPlan(_TrainPlan):
    """k of `experts` for every token of the ranks' tokens (sparbit_router_plan_create)."""

    _kind = "router"

    def __init__(self, tokens, experts: int, k: int, dtype: int = BF16, renormalize: bool = False):
        n, arr = _counts(tokens)
        self._create(n, arr, experts, k, dtype, int(bool(renormalize)))
        self.experts, self.k, self.dtype = experts, k, dtype

    def forward(self, logits, indices, weights, lse, counts, sums, mask=None, stream=None, ld=None) -> None:
        try:
            t, f, i = _types[self.dtype], _types[F32], _types[_I32]
            usual = (logits.dtype is t and indices.dtype is counts.dtype is i
                     and weights.dtype is lse.dtype is sums.dtype is f and logits.is_cuda and indices.is_cuda
                     and weights.is_cuda and lse.is_cuda and counts.is_cuda and sums.is_cuda
                     and (logits.is_contiguous() if ld is None else _in_rows(logits, self.experts)) and indices.is_contiguous()
                     and weights.is_contiguous() and lse.is_contiguous() and counts.is_contiguous()
                     and sums.is_contiguous())
        except (AttributeError, KeyError):
            usual = False
        if usual:
            logits, indices, weights, lse, counts, sums = (logits.data_ptr(), indices.data_ptr(), weights.data_ptr(),
                                                           lse.data_ptr(), counts.data_ptr(), sums.data_ptr())
        else:
            logits = _rows_of(logits, self.dtype, ld, self.experts)
            indices, weights, lse = _flat(indices, _I32), _flat(weights, F32), _flat(lse, F32)
            counts, sums = _flat(counts, _I32), _flat(sums, F32)
        args = (self._h, logits, self.experts if ld is None else ld, _flat(mask, _BYTE), indices, weights, lse, counts,
                sums, _stream_handle(stream))
        try:
            code = _router_forward(*args)
        except ctypes.ArgumentError:
            code = lib.sparbit_router_forward(*args)
        if code != OK:
            raise SparbitError(code, "sparbit_router_forward")

    def balance(self, gathered, G: int, sums, loss, alpha: float, beta: float = 0.0, stream=None) -> None:
        _check(lib.sparbit_router_balance(self._h, _flat(gathered, _I32), G, _flat(sums, F32), alpha, beta,
                                          _flat(loss, F32), _stream_handle(stream)), "sparbit_router_balance")

    def backward(self, logits, indices, weights, lse, gathered, G: int, dlogits, dweights=None, alpha: float = 0.0,
                 beta: float = 0.0, dloss=None, mask=None, stream=None, ld=None, dlogits_ld=None) -> None:
        t, e = self.dtype, self.experts
        _check(lib.sparbit_router_backward(self._h, _address_of(logits, t), _stride_of(logits, ld, e),
                                           _flat(mask, _BYTE), _flat(indices, _I32), _flat(weights, F32),
                                           _flat(lse, F32), _flat(gathered, _I32), G, _flat(dweights, F32), alpha, beta,
                                           _flat(dloss, F32), _address_of(dlogits, t),
                                           _stride_of(dlogits, dlogits_ld, e), _stream_handle(stream)),
               "sparbit_router_backward")


class OrthoPlan(_TrainPlan):
    """`count` matrices of rows x cols, orthogonalised by Newton-Schulz products (sparbit_ortho_plan_create).
    coefficients: `steps` triples (a, b, c), or None for the usual quintic.  Strides between matrices
    default to rows * ld."""

    _kind = "ortho"

    def __init__(self, count: int, rows: int, cols: int, dtype: int = BF16, steps: int = 5, coefficients=None,
                 eps: float = 1e-7, products: int = PRODUCTS_AUTO):
        arr = None
        if coefficients is not None:
            flat = [float(v) for triple in coefficients for v in triple]
            if len(flat) != 3 * steps:
                raise ValueError(f"{steps} steps need {steps} triples of coefficients")
            arr = (_f * len(flat))(*flat)
        self._create(count, rows, cols, dtype, steps, arr, eps)
        self.rows, self.cols, self.dtype = rows, cols, dtype
        if products != PRODUCTS_AUTO:
            self.set_products(products)

    def set_products(self, products: int) -> None:
        _check(lib.sparbit_ortho_plan_set_products(self._h, products), "sparbit_ortho_plan_set_products")

    def orthogonalize(self, update, out, stream=None, ld=None, stride=None, out_ld=None, out_stride=None) -> None:
        # matrices have a stride of their own
        t, ld, out_ld = self.dtype, _stride_of(update, ld, self.cols, False), _stride_of(out, out_ld, self.cols, False)
        stride = self.rows * ld if stride is None else stride
        out_stride = self.rows * out_ld if out_stride is None else out_stride
        _check(lib.sparbit_orthogonalize(self._h, _address_of(update, t), ld, stride, _address_of(out, t), out_ld,
                                         out_stride, _stream_handle(stream)), "sparbit_orthogonalize")

    def muon_step(self, grad, momentum_in, momentum_out, weight_in, weight_out, weight_dtype: int, lr: float,
                  momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale: float = 1.0,
                  stream=None, grad_ld=None, grad_stride=None, momentum_ld=None, momentum_stride=None, weight_ld=None,
                  weight_stride=None) -> None:
        r, c = self.rows, self.cols
        _stride_of(momentum_in, momentum_ld, c, False), _stride_of(weight_in, weight_ld, c, False)
        gl, ml = _stride_of(grad, grad_ld, c, False), _stride_of(momentum_out, momentum_ld, c, False)
        wl = _stride_of(weight_out, weight_ld, c, False)
        args = MuonArgs(_address_of(grad, self.dtype), gl, r * gl if grad_stride is None else grad_stride,
                        _address_of(momentum_in, F32), _address_of(momentum_out, F32), ml,
                        r * ml if momentum_stride is None else momentum_stride, _address_of(weight_in, weight_dtype),
                        _address_of(weight_out, weight_dtype), wl, r * wl if weight_stride is None else weight_stride,
                        weight_dtype, int(bool(nesterov)), lr, momentum, weight_decay, scale)
        _check(lib.sparbit_muon_step(self._h, ctypes.byref(args), _stream_handle(stream)), "sparbit_muon_step")


def _attention_scale(key_size, scale):
    """The usual scale where none is given (any for a size that the library refuses)."""
    return float(scale) if scale is not None else key_size ** -0.5 if key_size > 0 else 1.0


class LinearAttentionPlan(_TrainPlan):
    """Linear attention with a decay for each head over sequences of the given lengths
    (sparbit_linear_attention_plan_create).  scale: key_size ** -0.5 where it is None.  Row strides default to heads *
    size; a tensor of [rows][heads][size] that is part of a wider one needs its own."""

    _kind = "linear_attention"

    def __init__(self, lengths, heads: int, key_size: int, value_size: int, dtype: int = BF16, scale=None):
        n, arr = _counts(lengths)
        self.scale = _attention_scale(key_size, scale)
        self._create(n, arr, heads, key_size, value_size, dtype, self.scale)
        self.heads, self.key_size, self.value_size, self.dtype = heads, key_size, value_size, dtype

    def forward(self, q, k, v, log_decay, o, first=None, summary=None, stream=None, q_ld=None, k_ld=None, v_ld=None,
                o_ld=None) -> None:
        t, wk, wv = self.dtype, self.heads * self.key_size, self.heads * self.value_size
        _check(lib.sparbit_linear_attention_forward(
            self._h, _address_of(q, t), _stride_of(q, q_ld, wk), _address_of(k, t), _stride_of(k, k_ld, wk),
            _address_of(v, t), _stride_of(v, v_ld, wv), _flat(log_decay, F32), _flat(first, F32), _address_of(o, t),
            _stride_of(o, o_ld, wv), _flat(summary, F32), _stream_handle(stream)), "sparbit_linear_attention_forward")

    def backward(self, q, k, v, log_decay, do, dq, dk, dv, first=None, dlast=None, dsummary=None, stream=None, q_ld=None,
                 k_ld=None, v_ld=None, do_ld=None, dq_ld=None, dk_ld=None, dv_ld=None) -> None:
        t, wk, wv = self.dtype, self.heads * self.key_size, self.heads * self.value_size
        _check(lib.sparbit_linear_attention_backward(
            self._h, _address_of(q, t), _stride_of(q, q_ld, wk), _address_of(k, t), _stride_of(k, k_ld, wk),
            _address_of(v, t), _stride_of(v, v_ld, wv), _flat(log_decay, F32), _flat(first, F32), _address_of(do, t),
            _stride_of(do, do_ld, wv), _flat(dlast, F32), _address_of(dq, t), _stride_of(dq, dq_ld, wk),
            _address_of(dk, t), _stride_of(dk, dk_ld, wk), _address_of(dv, t), _stride_of(dv, dv_ld, wv),
            _flat(dsummary, F32), _stream_handle(stream)), "sparbit_linear_attention_backward")


def linear_attention_step(rows: int, heads: int, key_size: int, value_size: int, dtype: int, q, k, v, log_decay, state_in,
                          state_out, o, scale=None, slots=None, n_slots=None, stream=None, q_ld=None, k_ld=None,
                          v_ld=None, o_ld=None) -> None:
    """One token for each of `rows` running sequences; n_slots defaults to `rows`, scale to key_size ** -0.5."""
    wk, wv = heads * key_size, heads * value_size
    code = lib.sparbit_linear_attention_step(
        rows, heads, key_size, value_size, dtype, _attention_scale(key_size, scale),
        _address_of(q, dtype), _stride_of(q, q_ld, wk),
        _address_of(k, dtype), _stride_of(k, k_ld, wk),
        _address_of(v, dtype), _stride_of(v, v_ld, wv), _flat(log_decay, F32), _flat(slots, _I32),
        rows if n_slots is None else n_slots, _flat(state_in, F32), _flat(state_out, F32), _address_of(o, dtype),
        _stride_of(o, o_ld, wv), _stream_handle(stream))
    if code != OK:
        raise SparbitError(code, "sparbit_linear_attention_step")


def linear_attention_join(P: int, heads: int, key_size: int, value_size: int, gathered, out, first=None,
                          reverse: bool = False, first_rank: int = 0, n_ranks=None, stream=None) -> None:
    """First states of the slices first_rank .. first_rank + n_ranks - 1 (default: all P)."""
    _check(lib.sparbit_linear_attention_join(P, first_rank, P if n_ranks is None else n_ranks, heads, key_size,
                                             value_size, _flat(gathered, F32), _flat(first, F32), _flat(out, F32),
                                             int(bool(reverse)), _stream_handle(stream)),
           "sparbit_linear_attention_join")


class NormPlan(_TrainPlan):
    """Root-mean-square norm of rows of `width` elements (sparbit_norm_plan_create).  block: columns of a scale of the
    8-bit rows, 0 = one scale a row; weight_dtype defaults to dtype.  Only `backward` needs the workspace."""

    _kind = "norm"

    def __init__(self, width: int, dtype: int = BF16, weight_dtype=None, eps: float = 1e-6, block: int = 0):
        weight_dtype = dtype if weight_dtype is None else weight_dtype
        self._create(width, dtype, weight_dtype, eps, block)
        self.width, self.dtype, self.weight_dtype = width, dtype, weight_dtype

    def forward(self, rows: int, x, weight=None, residual=None, sum=None, y=None, y8=None, scales=None, rstd=None,
                stream=None, x_ld=None, residual_ld=None, sum_ld=None, y_ld=None, y8_ld=None) -> None:
        w, t = self.width, self.dtype
        code = lib.sparbit_norm_forward(
            self._h, rows, _address_of(x, t), _stride_of(x, x_ld, w), _address_of(residual, t),
            _stride_of(residual, residual_ld, w), _flat(weight, self.weight_dtype), _address_of(sum, t),
            _stride_of(sum, sum_ld, w), _address_of(y, t), _stride_of(y, y_ld, w), _address_of(y8, _E4M3),
            _stride_of(y8, y8_ld, w), _flat(scales, F32), _flat(rstd, F32), _stream_handle(stream))
        if code != OK:
            raise SparbitError(code, "sparbit_norm_forward")

    def backward(self, rows: int, dy, sum, weight, rstd, dx, dweight=None, dsum=None, stream=None, dy_ld=None,
                 sum_ld=None, dx_ld=None, dsum_ld=None) -> None:
        w, t = self.width, self.dtype
        _check(lib.sparbit_norm_backward(
            self._h, rows, _address_of(dy, t), _stride_of(dy, dy_ld, w), _address_of(sum, t), _stride_of(sum, sum_ld, w),
            _flat(weight, self.weight_dtype), _flat(rstd, F32), _address_of(dsum, t), _stride_of(dsum, dsum_ld, w),
            _address_of(dx, t), _stride_of(dx, dx_ld, w), _flat(dweight, F32), _stream_handle(stream)),
            "sparbit_norm_backward")


class ClipPlan(_TrainPlan):
    """Norm of all gradients and their clipping (sparbit_clip_plan_create): tensors of the given lengths (in elements) and
    types, each owned by one of n_ranks virtual ranks (all by rank 0 where `ranks` is None)."""

    _kind = "clip"

    def __init__(self, lengths, dtypes, ranks=None, n_ranks: int = 1):
        n, arr = _counts(lengths)
        self.dtypes = [int(d) for d in dtypes]
        if len(self.dtypes) != n or (ranks is not None and len(ranks) != n):
            raise ValueError("lengths, dtypes and ranks belong together")
        owners = None if ranks is None else (_i * n)(*[int(r) for r in ranks])
        self._create(n_ranks, n, arr, (_i * n)(*self.dtypes), owners)

    def set_tensors(self, tensors, out=None) -> None:
        """The tensors that are summed, and those that get the clipped elements (the same ones: in place; None: only
        sums and norms are wanted).  Synchronises."""
        kept, addresses = [], []
        for given in (tensors, out):
            given = None if given is None else list(given)
            if given is not None and len(given) != len(self.dtypes):
                raise ValueError(f"{len(self.dtypes)} tensors are wanted, not {len(given)}")
            kept.append(given)
            addresses.append(None if given is None else (_vp * len(given))(
                *[_flat(x, t) for x, t in zip(given, self.dtypes)]))
        _check(lib.sparbit_clip_plan_set_tensors(self._h, addresses[0], addresses[1]), "sparbit_clip_plan_set_tensors")
        self._tensors = kept  # keep the owners alive

    def sums(self, sums, stream=None) -> None:
        _check(lib.sparbit_clip_sums(self._h, _flat(sums, _F64), _stream_handle(stream)), "sparbit_clip_sums")

    def scale(self, gathered, G: int, most: float, norms, eps: float = 1e-6, stream=None) -> None:
        _check(lib.sparbit_clip_scale(self._h, _flat(gathered, _F64), G, most, eps, _flat(norms, F32),
                                      _stream_handle(stream)), "sparbit_clip_scale")
