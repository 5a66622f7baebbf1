"""Bit-pattern decoders used by the oracle.

bf16 is the upper half of an IEEE-754 binary32, so decoding is a 16-bit left
shift. OCP FP8 E4M3FN (the OCP 8-bit floating point specification, "E4M3"
variant with finite-only encoding): 1 sign bit, 4 exponent bits with bias 7, 3
mantissa bits; exponent field 0 encodes subnormals m * 2^-9; S.1111.111 is NaN;
there is no infinity, so S.1111.110 = +-448 is the largest finite value.

MXFP4 (the OCP microscaling formats specification): E2M1 codes (1 sign bit, 2
exponent bits with bias 1, 1 mantissa bit; exponent field 0 encodes m * 0.5) in
groups of 32 that share a scale 2^(byte - 127); byte 255 is NaN.
"""

import numpy as np


def bf16_bits_to_f64(u16: np.ndarray) -> np.ndarray:
    u32 = np.asarray(u16, dtype=np.uint16).astype(np.uint32) << np.uint32(16)
    return u32.view(np.float32).astype(np.float64)


def e4m3fn_value(code: int) -> float:
    """Value of one E4M3FN code, read field by field."""
    code = int(code) & 0xFF
    sign = -1.0 if code & 0x80 else 1.0
    exp_field = (code >> 3) & 0xF
    mant = code & 0x7
    if exp_field == 0xF and mant == 0x7:
        return float("nan")
    if exp_field == 0:
        return sign * mant * 2.0 ** -9
    return sign * (1.0 + mant / 8.0) * 2.0 ** (exp_field - 7)


E4M3FN_TABLE = np.array([e4m3fn_value(c) for c in range(256)], dtype=np.float64)


def e4m3fn_bits_to_f64(u8: np.ndarray) -> np.ndarray:
    return E4M3FN_TABLE[np.asarray(u8, dtype=np.uint8)]


def e2m1_value(code: int) -> float:
    """Value of one E2M1 code (4 bits), read field by field."""
    sign = -1.0 if code & 8 else 1.0
    exp_field, mant = (code >> 1) & 3, code & 1
    return sign * (0.5 * mant if exp_field == 0 else (1.0 + 0.5 * mant) * 2.0 ** (exp_field - 1))


E2M1_TABLE = np.array([e2m1_value(c) for c in range(16)], dtype=np.float64)


def mxfp4_encode(x: np.ndarray):
    """Rows x [..., 128] (float) -> codes [..., 128] and scale bytes [..., 4].
    With a the largest magnitude of a group of 32 in [1.75 * 2^(E-1), 1.75 *
    2^E), the scale is 2^X, X = E - 2 held in [-125, 125] (-125 for a = 0); each
    code is the level nearest to x / 2^X, ties to the even code, saturating."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    a = np.abs(g).max(axis=-1)
    power = np.full(a.shape, -125, np.int64)
    nz = a > 0
    # a / 1.75 = f * 2^e with f in [0.5, 1): a in [1.75 * 2^(e-1), 1.75 * 2^e)
    power[nz] = np.clip(np.frexp(a[nz] / 1.75)[1] - 2, -125, 125)
    y = np.abs(g) * 2.0 ** (-power[..., None].astype(np.float64))
    gap = np.abs(y[..., None] - E2M1_TABLE[:8])
    near = gap == gap.min(axis=-1, keepdims=True)
    odd_first = near.argmax(axis=-1)                       # the lower of two equally near codes
    tie = near.sum(axis=-1) == 2
    code = np.where(tie & (odd_first % 2 == 1), odd_first + 1, odd_first)
    code = code | np.where(np.signbit(g), 8, 0)
    return code.astype(np.uint8).reshape(x.shape), (power + 127).astype(np.uint8)


CELL = 1088        # bytes of one (block, KV head) of an MXFP4 pool: 1024 of codes, 64 of scales


def mxfp4_places(h_kv: int, head: int, token: int, is_v: bool):
    """Where a pool block keeps one token of one KV head: the (byte, nibble) of
    each of its 128 dims, and the byte of each of its 4 scales."""
    dim = np.arange(128)
    grp = np.arange(4)
    if is_v:
        nib = (token // 4) * 512 + (dim // 8) * 32 + (token % 4) * 8 + dim % 8
        at = grp * 16 + token
    else:
        nib = token * 128 + dim
        at = token * 4 + grp
    return head * 1024 + nib // 2, nib % 2, h_kv * 1024 + head * 64 + at


def mxfp4_blocks_to_f64(raw: np.ndarray, is_v: bool) -> np.ndarray:
    """Pool blocks [n, h_kv * 1088] -> [n, h_kv, 16, 128]."""
    h_kv = raw.shape[1] // CELL
    out = np.empty((raw.shape[0], h_kv, 16, 128))
    for h in range(h_kv):
        for t in range(16):
            byte, nib, at = mxfp4_places(h_kv, h, t, is_v)
            codes = (raw[:, byte] >> (4 * nib).astype(np.uint8)) & 15
            scale = raw[:, at].astype(np.float64)
            power = np.where(scale == 255, np.nan, 2.0 ** (scale - 127.0))
            out[:, h, t] = E2M1_TABLE[codes] * np.repeat(power, 32, axis=1)
    return out


def storage_to_f64(x: np.ndarray, dtype: str) -> np.ndarray:
    if dtype == "f32":
        return np.asarray(x, dtype=np.float32).astype(np.float64)
    if dtype == "bf16":
        return bf16_bits_to_f64(x)
    if dtype == "fp8":
        return e4m3fn_bits_to_f64(x)
    raise ValueError(dtype)


# Finite non-negative E4M3FN values in code order (codes 0x00 .. 0x7E); the
# value grows with the code, so nearest-value search is a sorted search.
_POS_VALUES = E4M3FN_TABLE[:0x7F]


def e4m3fn_encode(y: np.ndarray) -> np.ndarray:
    """float32 -> E4M3FN codes: the nearest finite value, ties to the code with
    an even mantissa (round to nearest even), magnitudes beyond 448 saturate
    to +-448, the sign of zero is kept. Found by searching the value table,
    not by manipulating bits."""
    y = np.asarray(y, dtype=np.float32).astype(np.float64)
    a = np.minimum(np.abs(y), 448.0)
    hi = np.searchsorted(_POS_VALUES, a, side="left")          # first value >= a
    hi = np.minimum(hi, 0x7E)
    lo = np.maximum(hi - 1, 0)
    d_lo = a - _POS_VALUES[lo]
    d_hi = _POS_VALUES[hi] - a
    pick_hi = (d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0))
    code = np.where(pick_hi, hi, lo)
    code = np.where(a == _POS_VALUES[hi], hi, code)             # exact hits
    sign = np.signbit(y)
    return (code | (sign.astype(np.int64) << 7)).astype(np.uint8)
