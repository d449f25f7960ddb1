"""ctypes binding of the 8-bit integer operators and of the Encode stage on them, declared in include/int8.h (argument
marshalling only)."""
import ctypes as C

from .binding import lib, DitError, DIT_OK, STATUS_NAMES
from .encoder import Encoder, _lens

_vp, _i, _sz, _f, _ip = C.c_void_p, C.c_int, C.c_size_t, C.c_float, C.POINTER(C.c_int)

X_BF16, X_F32 = 0, 1
MAX_ROW, MAX_ROWS, MAX_K = 16384, 1 << 23, 131072 - 128

_SIGS = {
    "dit_op_quantize_i8": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _i, _vp]),
    "dit_op_rmsnorm_i8": (_i, [_vp, _vp, _i, _vp, _i, _i, _vp, _f, _i, _i, _vp, _i, _vp, _i, _vp]),
    "dit_op_gemm_i8": (_i, [_vp, _vp, _i, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _sz]),
    "dit_op_gemm_i8_geglu": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _i, _vp, _sz]),
    "dit_op_gemm_i8_transposed": (_i, [_vp, _vp, _i, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _vp, _i, _vp, _vp, _sz]),
    "dit_op_gemm_i8_work_bytes": (_sz, [_i, _i, _i, _i]),
    "dit_op_gemm_i8_tile": (_i, [_i, _i, _i, _i, _sz, _ip]),
    "enc_i8_weight_bytes": (_sz, [_vp]),
    "enc_i8_workspace_bytes": (_sz, [_vp, _i, _ip]),
    "enc_i8_quantize": (_i, [_vp, _vp, _sz]),
    "enc_i8_forward": (_i, [_vp, _i, _ip, _vp, _vp, _vp]),
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


class EncoderI8(Encoder):
    """An encoder whose products run on 8-bit codes.  quantize() after the weights are set, and again after they change."""

    codes = None

    def workspace_bytes(self, lens):
        a, p = _lens(lens)
        return enc_i8_workspace_bytes(self.ctx, len(a), p)

    def code_bytes(self):
        return enc_i8_weight_bytes(self.ctx)

    def quantize(self):
        if self.codes is None:
            self.codes = self.torch.empty(self.code_bytes(), dtype=self.torch.uint8, device=f"cuda:{self.device}")
        self.check(enc_i8_quantize(self.ctx, self.codes.data_ptr(), self.codes.numel()))

    def forward(self, lens, tokens, out_bf16=None, out_f32=None):
        a, p = _lens(lens)
        self.check(enc_i8_forward(self.ctx, len(a), p, tokens.data_ptr(), out_bf16.data_ptr() if out_bf16 is not None else None,
                                  out_f32.data_ptr() if out_f32 is not None else None))
