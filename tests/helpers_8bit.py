"""The 8-bit operators in plain numpy: e4m3 with a scale for each block of 128, products and the expert in 64 bits."""
import numpy as np
import torch

BLOCK = 128
TINY = np.float32(2.0 ** -126)


def decode(bits):
    """e4m3 bytes -> float64."""
    return torch.from_numpy(np.ascontiguousarray(bits)).view(torch.float8_e4m3fn).to(torch.float64).numpy()


def encode(x):
    """float32 -> e4m3 bytes, to nearest even."""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def spread(scale, rows, cols, block_rows):
    s = np.repeat(scale, BLOCK, axis=-1)[..., :cols]
    return np.repeat(s, block_rows, axis=-2)[..., :rows, :] if block_rows > 1 else s


def quantize(x, block_rows=1):
    """x [..][rows][cols] (float32) -> bytes, float32 scales, as the header defines them."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape[-2:]
    pad = [(0, 0)] * (x.ndim - 2) + [(0, -rows % block_rows), (0, -cols % BLOCK)]
    m = np.abs(np.pad(x, pad))
    m = m.reshape(*x.shape[:-2], m.shape[-2] // block_rows, block_rows, m.shape[-1] // BLOCK, BLOCK).max(axis=(-3, -1))
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.where(np.isfinite(m), np.maximum(m / np.float32(448), TINY), np.float32(np.nan)).astype(np.float32)
        q = encode(x / spread(s, rows, cols, block_rows))
    return q, s


def values(q, s, block_rows=1):
    """What the bytes and scales stand for, float64."""
    return decode(q) * spread(s.astype(np.float64), *q.shape[-2:], block_rows)


def silu(g):
    return g / (1.0 + np.exp(-g))


def product_error(abs_sum, Kd):
    """Bound of a 32-bit product's error, given sum |a w|: every one of a block's 128 additions, the two roundings of the
    scale and the block's addition are off by half a step of 2^-24 relative to at most that sum."""
    return (128 + 3 * -(-Kd // BLOCK) + 4) * 2.0 ** -24 * abs_sum


def tensor(a):
    """numpy -> GPU tensor; bytes stay bytes."""
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16)
