"""Quantised rows in 64 bits from their definition (numpy, no code of the library):
d codes of e4m3 and a scale 2^e, e the smallest integer of [-120, 119] with
max |x| <= 448 2^e over the row's finite values."""
import numpy as np
import torch


def exponent(top):
    """e of rows whose largest finite size is top."""
    top = np.asarray(top, dtype=np.float64)
    e = np.full(top.shape, -120)
    for c in range(-120, 119):
        e[top > 448.0 * 2.0 ** c] = c + 1
    return e


def rounded(x, e):
    """x to the grid of codes times 2^e: ties to even, +-448 beyond, NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    y = np.where(np.isfinite(x), x, 0.0) / 2.0 ** np.asarray(e, dtype=np.float64)
    with np.errstate(divide="ignore"):
        step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(y))), -6) - 3)
    v = np.clip(np.rint(y / step) * step, -448, 448) * 2.0 ** np.asarray(e, dtype=np.float64)
    return np.where(np.isfinite(x), v, np.nan)


def quantised(x):
    """(values, e [..., 1]) of the rows of x [..., d]."""
    x = np.asarray(x, dtype=np.float64)
    e = exponent(np.where(np.isfinite(x), np.abs(x), 0.0).max(-1))[..., None]
    return rounded(x, e), e


def values(codes, scale):
    """What pool rows stand for: codes [..., d] e4m3, scale [...] uint8."""
    return codes.cpu().view(torch.uint8).view(torch.float8_e4m3fn).float().double().numpy() * \
        2.0 ** (scale.cpu().double().numpy()[..., None] - 127)


def pool(x):
    """(codes, scale) tensors of the rows of x, for caches that a test fills itself."""
    x = torch.as_tensor(x).double()
    v, e = quantised(x.numpy())
    codes = torch.from_numpy(v / 2.0 ** e).float().to(torch.float8_e4m3fn)
    return codes, torch.from_numpy((e[..., 0] + 127).astype(np.uint8))


def between(got, x, slack, e):
    """Whether every value is the rounding, under its row's e, of something within slack of x (rounding is monotone)."""
    e = np.asarray(e)[..., None]
    return (got >= rounded(x - slack, e)) & (got <= rounded(x + slack, e))
