"""ctypes binding of the 8-bit integer operators declared in include/int8.h (argument marshalling only)."""
import ctypes as C

from .binding import lib, DitError, DIT_OK, STATUS_NAMES

_vp, _i, _sz, _f = C.c_void_p, C.c_int, C.c_size_t, C.c_float

X_BF16, X_F32 = 0, 1
MAX_ROW, MAX_K = 16384, 131072 - 128

_SIGS = {
    "dit_op_quantize_i8": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _i, _vp]),
    "dit_op_rmsnorm_i8": (_i, [_vp, _vp, _i, _vp, _i, _i, _vp, _f, _i, _i, _vp, _i, _vp, _i, _vp]),
    "dit_op_gemm_i8": (_i, [_vp, _vp, _i, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _sz]),
    "dit_op_gemm_i8_geglu": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _i, _vp, _sz]),
    "dit_op_gemm_i8_transposed": (_i, [_vp, _vp, _i, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _vp, _i, _vp, _vp, _sz]),
    "dit_op_gemm_i8_work_bytes": (_sz, [_i, _i, _i, _i]),
}
EXPORTS = sorted(_SIGS)
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(lib, _name)
    _fn.restype, _fn.argtypes = _res, _args
    globals()[_name] = _fn


def check(status):
    """Raises DitError unless an operator returned DIT_OK."""
    if status != DIT_OK:
        raise DitError(status, "8-bit operator refused its arguments" if status in STATUS_NAMES else "unknown status")
