"""4-bit weights with group scales from their definitions in float64 numpy. Test infrastructure; shares no code with the GPU
path."""
import numpy as np


def bf16(v):
    """v rounded to the nearest bfloat16, ties to the even fraction (normal range)."""
    v = np.asarray(v, np.float64)
    _, p = np.frexp(v)
    step = np.exp2(p - 8.0)
    return np.round(v / step) * step


def quantized(w, group):
    """(codes, scales [..., groups]) of w, groups along its last axis."""
    w = np.asarray(w, np.float64)
    k = w.shape[-1]
    v = np.concatenate([w, np.zeros(w.shape[:-1] + (-k % group,))], -1).reshape(w.shape[:-1] + (-1, group))
    fine = np.isfinite(v).all(-1)
    top = np.where(fine, np.abs(np.where(np.isfinite(v), v, 0.0)).max(-1), 0.0)
    scale = bf16((top.astype(np.float32) / np.float32(7)).astype(np.float64))
    scale = np.where(scale < 2.0 ** -126, 0.0, scale)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.round((v.astype(np.float32) / scale[..., None].astype(np.float32)).astype(np.float64))
    codes = np.where((scale > 0)[..., None] & fine[..., None], np.clip(np.where(np.isfinite(q), q, 0), -8, 7), 0)
    return codes.reshape(w.shape[:-1] + (-1,))[..., :k], np.where(fine, scale, np.nan)


def values(codes, scales, group):
    return codes * np.repeat(scales, group, -1)[..., :codes.shape[-1]]


def product(x, codes, scales, group, b=None):
    """z = x w^T + b, and the sum of the magnitudes of its terms."""
    w = values(codes, scales, group)
    z, mag = x @ np.swapaxes(w, -1, -2), np.abs(x) @ np.swapaxes(np.abs(w), -1, -2)
    if b is not None:
        z, mag = z + b[..., None, :], mag + np.abs(b)[..., None, :]
    return z, mag
