"""Dense substrate layers in 8-bit floating point, from their definitions in float64 numpy: the block-scaled
e4m3 format, the layer, its slope and gradients. Test infrastructure; shares no code with the GPU path."""
import numpy as np

BLOCK = 128
ACTS = ("identity", "sigmoid", "tanh", "gauss", "sin", "abs")


def e4m3(v):
    """v rounded to the nearest e4m3 value, ties to the even fraction (|v| <= 448; NaN stays)."""
    v = np.asarray(v, np.float64)
    _, p = np.frexp(v)
    step = np.exp2(np.maximum(p - 1, -6) - 3.0)
    return np.round(v / step) * step


def block_scales(x):
    """Power-of-two scales [..., blocks] of x, blocks of 128 along its last axis."""
    x = np.asarray(x, np.float64)
    n = x.shape[-1]
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    a = np.concatenate([a, np.zeros(a.shape[:-1] + (-n % BLOCK,))], -1)
    top = a.reshape(a.shape[:-1] + (-1, BLOCK)).max(-1)
    m, p = np.frexp(top / 448.0)                      # top / 448 = m 2^p, m in [1/2, 1)
    # top is a float32 and 448 = 7 * 2^6: the quotient is a power of two only when it is exact
    e = np.where(m == 0.5, p - 1, p)
    return np.exp2(np.where(top > 0, np.clip(e, -126, 127), 0).astype(np.float64))


def held(x):
    """The values that x is held as, blocks along its last axis; infinities become NaN."""
    x = np.asarray(x, np.float64)
    s = np.repeat(block_scales(x), BLOCK, -1)[..., :x.shape[-1]]
    with np.errstate(invalid="ignore"):
        return e4m3(np.where(np.isfinite(x), x, np.nan) / s) * s


def act(z, name):
    z = np.asarray(z, np.float64)
    with np.errstate(over="ignore"):
        return {"identity": lambda: z, "sigmoid": lambda: 1 / (1 + np.exp(-z)), "tanh": lambda: np.tanh(z),
                "gauss": lambda: np.exp(-z * z), "sin": lambda: np.sin(z), "abs": lambda: np.abs(z)}[name]()


def slope(z, name):
    z = np.asarray(z, np.float64)
    t = np.exp(-np.abs(z))
    return {"identity": lambda: np.ones_like(z), "sigmoid": lambda: t / (1 + t) ** 2,
            "tanh": lambda: 4 * t * t / (1 + t * t) ** 2, "gauss": lambda: -2 * z * np.exp(-z * z),
            "sin": lambda: np.cos(z), "abs": lambda: np.sign(z)}[name]()


def product(x, w, b=None):
    """z = x w^T + b of held values, and the sum of the magnitudes of its terms."""
    z = x @ np.swapaxes(w, -1, -2)
    mag = np.abs(x) @ np.swapaxes(np.abs(w), -1, -2)
    if b is not None:
        z, mag = z + b[..., None, :], mag + np.abs(b)[..., None, :]
    return z, mag
