"""The 4-bit format of the paged cache, in fp64 from its definition: groups of 32 components, a scale
byte each, (u - 8) s with four bits u."""
import numpy as np

GROUP = 32
SCALES = 252  # bytes from here on mark a group that holds no numbers


def scale_value(b):
    """(4 + b % 4) 2^(b // 4 - 40); NaN from 252 on."""
    b = np.asarray(b, np.int64)
    s = (4.0 + b % 4) * np.exp2((b // 4 - 40).astype(np.float64))
    return np.where(b < SCALES, s, np.nan)


def encode(a):
    """Codes (uint8 0 .. 15 per component) and scale bytes of the groups of a's last dimension."""
    g = np.asarray(a, np.float64).reshape(a.shape[:-1] + (a.shape[-1] // GROUP, GROUP))
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    reach = 7.0 * scale_value(np.arange(SCALES))
    b = np.minimum(np.searchsorted(reach, np.abs(g).max(-1)), SCALES - 1)
    u = np.clip(np.rint(g / scale_value(b)[..., None]), -7, 7) + 8  # (rint: ties to even)
    return u.astype(np.uint8).reshape(a.shape), np.where(fine, b, 255).astype(np.uint8)


def decode(codes, scales):
    g = codes.astype(np.float64).reshape(codes.shape[:-1] + (codes.shape[-1] // GROUP, GROUP)) - 8.0
    return (g * scale_value(scales)[..., None]).reshape(codes.shape)


def pack(codes):
    """Two codes a byte, the even component in the lower half."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(b):
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (2 * b.shape[-1],))
