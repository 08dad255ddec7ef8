"""Rows held in 4 bits, in plain 64-bit steps, for the tests: the format by its definition, pages as bytes."""
import numpy as np
import torch

SIZES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def block_scale(block):
    """The scale of 32 values: of the smallest power of two that leaves the largest value below 7, within 2 .. 252; 255: not finite."""
    if not np.isfinite(block).all():
        return 255
    top = np.abs(block).max()
    for scale in range(2, 252):
        if top / 2.0 ** (scale - 127) < 7:
            return scale
    return 252


def encode(rows):
    """Codes [n, D] and scales [n, D / 32] of float64 rows [n, D]."""
    n, D = rows.shape
    blocks = rows.reshape(n, D // 32, 32)
    scales = np.array([[block_scale(b) for b in r] for r in blocks], dtype=np.uint8)
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.abs(blocks) / 2.0 ** (scales.astype(np.float64) - 127)[..., None]
        d = np.abs(a[..., None] - SIZES)
    best = d.min(-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    codes = np.where(even.any(-1), even.argmax(-1), near.argmax(-1)) + 8 * np.signbit(blocks)
    codes[scales == 255] = 0
    return codes.reshape(n, D).astype(np.uint8), scales


def decode(codes, scales):
    """float64 rows [..., D] of codes [..., D] and scales [..., D / 32]."""
    x = SIZES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return x * np.repeat(power, 32, axis=-1)


def hold(rows):
    return decode(*encode(rows))


def pack(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(b):
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


def parts(pages, ps, D):
    """Views [..., ps, D / 2] of the codes' bytes and [..., ps, D / 32] of the scales of pages [..., bytes] (numpy)."""
    at = ps * (D // 2)
    return pages[..., :at].reshape(*pages.shape[:-1], ps, D // 2), pages[..., at:at + ps * (D // 32)].reshape(*pages.shape[:-1], ps, D // 32)


def values(pages, ps, D):
    """float64 [..., ps, D] of pages [..., bytes] (a tensor)."""
    codes, scales = parts(pages.cpu().contiguous().numpy(), ps, D)
    return torch.from_numpy(decode(unpack(codes), scales))
