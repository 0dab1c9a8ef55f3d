"""Plain CPU oracle of the MX4 operators and the quantizing norm, in numpy and
64 bits, written from the definitions in include/apt_mx.h; it shares no code
with the GPU path."""
from __future__ import annotations

import numpy as np

#: Values of the sixteen E2M1 codes.
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=np.float64)
BLOCK, STEP, GROUP = 32, 256, 16


def to_bf16(x) -> np.ndarray:
    """float32 values rounded to nearest even to bfloat16, as float32."""
    x = np.asarray(x, dtype=np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


def rounded(x, kind: str) -> np.ndarray:
    """float64 values rounded once to fp16 / bf16 / fp32, as float64.  (Through
    float32 for bf16: exact where x is a float32 already.)"""
    with np.errstate(over="ignore"):
        if kind == "fp16":
            return np.asarray(x, dtype=np.float64).astype(np.float16).astype(np.float64)
        y = np.asarray(x, dtype=np.float64).astype(np.float32)
        return (to_bf16(y) if kind == "bf16" else y).astype(np.float64)


def blocks(K: int) -> int:
    return -(-K // BLOCK)


def quantize(x: np.ndarray):
    """(codes uint8 [R][K], scale bytes uint8 [R][blocks]) of rows x."""
    x = np.asarray(x, dtype=np.float64)
    R, K = x.shape
    codes = np.zeros((R, K), dtype=np.uint8)
    scales = np.zeros((R, blocks(K)), dtype=np.uint8)
    half = (E2M1[1:8] + E2M1[:7]) / 2  # borders between neighbours
    for b in range(blocks(K)):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        good = np.isfinite(v).all(axis=1)
        m = np.abs(np.where(good[:, None], v, 0.0)).max(axis=1)
        e = np.where(m > 0, np.frexp(np.where(m > 0, m, 1.0))[1] - 1 - 2, -127)
        e = np.maximum(e, -127)
        a = np.ldexp(np.abs(np.where(good[:, None], v, 0.0)), -e[:, None])
        low = (a[:, :, None] > half).sum(axis=2)   # a tie counts as below the border
        high = (a[:, :, None] >= half).sum(axis=2)  # ... as above
        c = np.where(low % 2 == 0, low, high).astype(np.uint8)
        c |= (np.signbit(v).astype(np.uint8) << 3)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.where(good[:, None], c, 0)
        scales[:, b] = np.where(good, e + 127, 255)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """float64 values of codes [R][K] with their scale bytes."""
    K = codes.shape[1]
    s = np.repeat(np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127)), BLOCK, axis=1)[:, :K]
    return E2M1[codes] * s


def nibbles(codes: np.ndarray) -> np.ndarray:
    """codes [R][K] two to a byte, the even element low: uint8 [R][ceil(K / 2)]."""
    R, K = codes.shape
    c = np.zeros((R, K + K % 2), dtype=np.uint8)
    c[:, :K] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def operand_bytes(rows: int, K: int) -> int:
    return -(-rows // GROUP) * -(-K // STEP) * (2048 + 128)


def operand(codes: np.ndarray, scales: np.ndarray):
    """(bytes, written): the operand's buffer, and which of its bytes the definition gives a value."""
    R, K = codes.shape
    G, S = -(-R // GROUP), -(-K // STEP)
    buf = np.zeros(operand_bytes(R, K), dtype=np.uint8)
    written = np.zeros(buf.shape, dtype=bool)
    c = np.zeros((R, S * STEP), dtype=np.uint8)
    c[:, :K] = codes
    s = np.zeros((R, S * STEP // BLOCK), dtype=np.uint8)
    s[:, :scales.shape[1]] = scales
    for r in range(R):
        g, row = divmod(r, GROUP)
        for t in range(S):
            for b in range(STEP // BLOCK):
                v = c[r, t * STEP + b * BLOCK:t * STEP + (b + 1) * BLOCK]
                at = ((g * S + t) * 8 + b) * 256 + row * 16
                buf[at:at + 16] = v[0::2] | (v[1::2] << 4)
                written[at:at + 16] = True
                at = G * S * 2048 + (g * S + t) * 128 + (b % 2) * 64 + row * 4 + b // 2
                buf[at] = s[r, t * 8 + b]
                written[at] = True
    return buf, written


def product(a: np.ndarray, w: np.ndarray):
    """(C, T): float64 A W^T and the sums of the terms' magnitudes."""
    with np.errstate(invalid="ignore", over="ignore"):
        return a @ w.T, np.abs(a) @ np.abs(w).T


def product_bounds(C: np.ndarray, T: np.ndarray, K: int, kind: str):
    """(low, high): between which an output of type `kind` lies.  The products are exact in fp32 (at
    most 6 bits of significand); each MFMA adds 64 or 128 of them to the sum, off by at most one unit
    of fp32, 2^-23, of the terms' magnitudes T that it has seen; at most ceil(K / 64) MFMAs follow
    each other and at most 64 partial sums are then added, each addition off by half a unit.  The
    sum is then rounded once, and rounding keeps order, overflow to infinity included."""
    acc = (-(-K // 64) * 2.0 ** -23 + 64 * 2.0 ** -24) * T + K * 2.0 ** -149
    return rounded(C - acc, kind), rounded(C + acc, kind)


def norm(x, residual, gain, eps: float, kind: str):
    """(h, y) of the norm for inputs of type `kind` (float64 arrays), rounded where the definition rounds."""
    h = np.asarray(x, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if residual is not None:
            h = rounded((h + residual).astype(np.float32), kind)
        f = np.float32(1.0 / np.sqrt((h * h).sum(axis=1) / h.shape[1] + eps))[:, None]
        y = np.float32(h) * f  # IEEE fp32 products
        if gain is not None:
            y = y * np.float32(gain)
        return h, rounded(y, kind)


def codes(y: np.ndarray, q: int):
    """(codes int8 [M][K], scales float64 [M]) of rows y; a NaN scale and codes 0 for a row that has none."""
    y = np.asarray(y, dtype=np.float64)
    top = (1 << q) - 1
    with np.errstate(over="ignore", invalid="ignore"):
        good = np.isfinite(y).all(axis=1)
        m = np.abs(np.where(good[:, None], y, 0.0)).max(axis=1)
        s = (np.float32(m) / np.float32(top)).astype(np.float16).astype(np.float64)
        good &= np.isfinite(s)
    use = good & (s > 0)
    t = np.floor(np.where(use[:, None], y, 0.0) / (2.0 * np.where(use, s, 1.0))[:, None])
    c = np.clip(t, -(1 << (q - 1)), (1 << (q - 1)) - 1).astype(np.int8)
    return c, np.where(good, s, np.nan)
