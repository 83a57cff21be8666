"""ctypes binding of include/sparbit_train.h: argument marshalling only.

Operators of a training step whose state is divided over the ranks of a communicator.  Tensors are
any objects with `data_ptr()` (or numpy arrays, or addresses); row strides (`*_ld`, in elements)
default to the row's width.  Everything runs in the library's CUDA kernels; there is no fallback.
"""
from __future__ import annotations

import ctypes

from .binding import ERR_TIMEOUT, OK, SparbitError, _i, _sz, _vp, lib
from .binding import _ptr as _address

F32, BF16, F16 = range(3)
PRODUCTS_AUTO, PRODUCTS_ONE, PRODUCTS_THREE = 0, 1, 3
ROUTER_MAX_EXPERTS, ROUTER_MAX_K = 1024, 32

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
}
for _name, (_res, _args) in SYMBOLS.items():
    _fn = getattr(lib, _name)  # AttributeError here means the library does not match the header
    _fn.restype = _res
    _fn.argtypes = _args
_scan_forward, _scan_backward, _scan_step = lib.sparbit_scan_forward, lib.sparbit_scan_backward, lib.sparbit_scan_step


# The calls below can be shorter than their own marshalling (a token's step takes the GPU 3 us), so
# the common cases come first.
def _ptr(x):
    """Address of a tensor (or of anything binding._ptr knows)."""
    if x is None:
        return None
    try:
        return x.data_ptr()
    except AttributeError:
        return _address(x)


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
        _check(getattr(lib, name)(self._h, _ptr(dev), nbytes), name)
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
        self.channels = channels

    @property
    def carry_bytes(self) -> int:
        return lib.sparbit_scan_plan_carry_bytes(self._h)

    def forward(self, gate, x, y, h0=None, summary=None, carry=None, stream=None, gate_ld=None, x_ld=None, y_ld=None,
                h0_ld=None) -> None:
        d = self.channels
        _check(_scan_forward(self._h, _ptr(gate), gate_ld or d, _ptr(x), x_ld or d, _ptr(h0), h0_ld or d,
                                        _ptr(y), y_ld or d, _ptr(summary), _ptr(carry), _stream_handle(stream)),
               "sparbit_scan_forward")

    def backward(self, gate, x, carry, dy, dgate, dx, dlast=None, dsummary=None, stream=None, gate_ld=None, x_ld=None,
                 dy_ld=None, dgate_ld=None, dx_ld=None, dlast_ld=None) -> None:
        d = self.channels
        _check(_scan_backward(self._h, _ptr(gate), gate_ld or d, _ptr(x), x_ld or d, _ptr(carry), _ptr(dy),
                                         dy_ld or d, _ptr(dlast), dlast_ld or d, _ptr(dgate), dgate_ld or d,
                                         _ptr(dx), dx_ld or d, _ptr(dsummary), _stream_handle(stream)),
               "sparbit_scan_backward")


def scan_step(rows: int, channels: int, dtype: int, gate, x, state_in, state_out, y, slots=None, n_slots=None,
              stream=None, gate_ld=None, x_ld=None, y_ld=None, state_ld=None) -> None:
    """One token for each of `rows` running sequences; n_slots defaults to `rows`."""
    d = channels
    _check(_scan_step(rows, d, dtype, _ptr(gate), gate_ld or d, _ptr(x), x_ld or d, _ptr(slots),
                                 rows if n_slots is None else n_slots, _ptr(state_in), _ptr(state_out), state_ld or d,
                                 _ptr(y), y_ld or d, _stream_handle(stream)), "sparbit_scan_step")


def scan_join(P: int, channels: int, gathered, out, h0=None, reverse: bool = False, first_rank: int = 0,
              n_ranks=None, out_ld=None, stream=None) -> None:
    """First states of the slices first_rank .. first_rank + n_ranks - 1 (default: all P)."""
    _check(lib.sparbit_scan_join(P, first_rank, P if n_ranks is None else n_ranks, channels, _ptr(gathered), _ptr(h0),
                                 _ptr(out), out_ld or channels, int(bool(reverse)), _stream_handle(stream)),
           "sparbit_scan_join")


class RouterPlan(_TrainPlan):
    """k of `experts` for every token of the ranks' tokens (sparbit_router_plan_create)."""

    _kind = "router"

    def __init__(self, tokens, experts: int, k: int, dtype: int = BF16, renormalize: bool = False):
        n, arr = _counts(tokens)
        self._create(n, arr, experts, k, dtype, int(bool(renormalize)))
        self.experts, self.k = experts, k

    def forward(self, logits, indices, weights, lse, counts, sums, mask=None, stream=None, ld=None) -> None:
        _check(lib.sparbit_router_forward(self._h, _ptr(logits), ld or self.experts, _ptr(mask), _ptr(indices),
                                          _ptr(weights), _ptr(lse), _ptr(counts), _ptr(sums), _stream_handle(stream)),
               "sparbit_router_forward")

    def balance(self, gathered, G: int, sums, loss, alpha: float, beta: float = 0.0, stream=None) -> None:
        _check(lib.sparbit_router_balance(self._h, _ptr(gathered), G, _ptr(sums), alpha, beta, _ptr(loss),
                                          _stream_handle(stream)), "sparbit_router_balance")

    def backward(self, logits, indices, weights, lse, gathered, G: int, dlogits, dweights=None, alpha: float = 0.0,
                 beta: float = 0.0, dloss=None, mask=None, stream=None, ld=None, dlogits_ld=None) -> None:
        _check(lib.sparbit_router_backward(self._h, _ptr(logits), ld or self.experts, _ptr(mask), _ptr(indices),
                                           _ptr(weights), _ptr(lse), _ptr(gathered), G, _ptr(dweights), alpha, beta,
                                           _ptr(dloss), _ptr(dlogits), dlogits_ld or self.experts,
                                           _stream_handle(stream)), "sparbit_router_backward")


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
        self.rows, self.cols = rows, cols
        if products != PRODUCTS_AUTO:
            self.set_products(products)

    def set_products(self, products: int) -> None:
        _check(lib.sparbit_ortho_plan_set_products(self._h, products), "sparbit_ortho_plan_set_products")

    def orthogonalize(self, update, out, stream=None, ld=None, stride=None, out_ld=None, out_stride=None) -> None:
        ld, out_ld = ld or self.cols, out_ld or self.cols
        _check(lib.sparbit_orthogonalize(self._h, _ptr(update), ld, self.rows * ld if stride is None else stride,
                                         _ptr(out), out_ld, self.rows * out_ld if out_stride is None else out_stride,
                                         _stream_handle(stream)), "sparbit_orthogonalize")

    def muon_step(self, grad, momentum_in, momentum_out, weight_in, weight_out, weight_dtype: int, lr: float,
                  momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale: float = 1.0,
                  stream=None, grad_ld=None, grad_stride=None, momentum_ld=None, momentum_stride=None, weight_ld=None,
                  weight_stride=None) -> None:
        gl, ml, wl = grad_ld or self.cols, momentum_ld or self.cols, weight_ld or self.cols
        r = self.rows
        args = MuonArgs(_ptr(grad), gl, r * gl if grad_stride is None else grad_stride, _ptr(momentum_in),
                        _ptr(momentum_out), ml, r * ml if momentum_stride is None else momentum_stride,
                        _ptr(weight_in), _ptr(weight_out), wl, r * wl if weight_stride is None else weight_stride,
                        weight_dtype, int(bool(nesterov)), lr, momentum, weight_decay, scale)
        _check(lib.sparbit_muon_step(self._h, ctypes.byref(args), _stream_handle(stream)), "sparbit_muon_step")
