"""Plain reference of a cache in 4 bits: its rounding, its layout and its values."""
import numpy as np
import torch

from tests.cache_util import TORCH_DTYPES

BLOCK = 32
LEAST = {torch.float16: -23, torch.bfloat16: -125}
GREATEST = {torch.float16: 14, torch.bfloat16: 126}  # 4 times such a scale is not a number of the type
NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(D):
    return D // 2 + -(-D // BLOCK)


def quantise(x):
    """[..., D] values of a 16-bit type: codes [..., D] and scale bytes [..., blocks], on the host, in 64 bits."""
    least, values = LEAST[x.dtype], x.double().cpu().numpy()
    D = values.shape[-1]
    codes = np.zeros(values.shape, np.uint8)
    scales = np.zeros((*values.shape[:-1], -(-D // BLOCK)), np.uint8)
    for i in range(scales.shape[-1]):
        block = values[..., i * BLOCK:(i + 1) * BLOCK]
        finite = np.isfinite(block).all(-1)
        block = np.where(finite[..., None], block, 0.0)
        most = np.abs(block).max(-1)
        # the power of two that brings `most` into 3.5 .. 7
        e = np.floor(np.log2(np.where(most > 0, most, 1.0) / 3.5)).astype(int)
        e += (most >= 7.0 * 2.0 ** e).astype(int) - (most < 3.5 * 2.0 ** e).astype(int)
        e = np.where(most > 0, np.maximum(e, least), least)
        y = np.abs(block) / 2.0 ** e[..., None]
        # the nearest number; of two as near the one with the even code
        off = np.abs(y[..., None] - NUMBERS)
        off = off + np.where(np.arange(8) % 2 == 1, 1e-12, 0.0) * 1.0
        off = np.where((e[..., None, None] == GREATEST[x.dtype]) & (NUMBERS >= 4.0), np.inf, off)
        code = off.argmin(-1) + 8 * np.signbit(block)
        codes[..., i * BLOCK:(i + 1) * BLOCK] = np.where(finite[..., None], code, 0)
        scales[..., i] = np.where(finite, e + 127, 255)
    return codes, scales


def values(codes, scales):
    """What they stand for, in 64 bits."""
    v = NUMBERS[codes & 7] * np.where(codes >= 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(int) - 127.0))
    return v * np.repeat(s, BLOCK, -1)[..., :v.shape[-1]]


def pack(cache):
    """A cache [pages, heads, page, D] in 4 bits, [pages, heads, page * row] uint8 on its device."""
    N, K, P, D = cache.shape
    codes, scales = quantise(cache)
    both = codes[..., 0::2] | (codes[..., 1::2] << 4)
    packed = np.concatenate([both.reshape(N, K, -1), scales.reshape(N, K, -1)], -1)
    return torch.from_numpy(np.ascontiguousarray(packed)).to(cache.device)


def unpack(packed, P, D, dtype):
    """Its values, [pages, heads, page, D] of `dtype` on its device."""
    data = packed.cpu().numpy()
    N, K, _ = data.shape
    both = data[..., :P * D // 2].reshape(N, K, P, D // 2)
    codes = np.stack([both & 15, both >> 4], -1).reshape(N, K, P, D)
    x = values(codes, data[..., P * D // 2:].reshape(N, K, P, -1))
    return torch.from_numpy(x).to(packed.device).to(TORCH_DTYPES.get(dtype, dtype))
