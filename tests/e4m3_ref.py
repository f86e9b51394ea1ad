"""Plain forms of pages of 8 bits, on the CPU: what their codes stand for, and what append does to a block."""
import math

import numpy as np
import torch

MOST, STEP, SMALL = 448.0, 2.0 ** -4, 2.0 ** -10         # the largest number; half a step of a normal one (relative) and of a subnormal one


def numbers(codes):
    """float64 of e4m3 codes."""
    return codes.detach().cpu().view(torch.float8_e4m3fn).float().double()


def code(x):
    """Codes (uint8) of float64 numbers within 448, rounded to nearest even from the definition: steps of 2^(e - 3), e >= -6."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.where((a > 0) & np.isfinite(a), a, 1.0))), -6)
    e = np.where(a >= 2.0 ** (e + 1), e + 1, e)
    n = np.rint(a / 2.0 ** (e - 3))                       # 8 .. 16 (below for subnormals)
    up = n == 16
    e, n = e + up, np.where(up, 8, n)
    normal = n >= 8
    bits = np.where(normal, (e + 7) * 8 + n - 8, n)
    bits = np.where(np.isfinite(a), np.where(np.isfinite(bits), bits, 0), 127).astype(np.int64)
    assert (bits <= 127).all() and (bits[np.isfinite(a)] <= 126).all(), "beyond 448"
    return (bits | (np.signbit(x) << 7)).astype(np.uint8)


def scale_for(x):
    """The smallest power of two s, from 2^-100 on, with |x| <= 448 s for the finite ones."""
    a = np.abs(np.asarray(x, np.float64))
    top = a[np.isfinite(a)].max(initial=0.0)
    if top == 0:
        return 2.0 ** -100
    k = math.floor(math.log2(top / MOST)) - 1
    while top > MOST * 2.0 ** k:
        k += 1
    return 2.0 ** max(k, -100)


def rows(pool, layer, row, n):
    """Keys and values float64 [n, Hkv, d] of the first n tokens of a row of the table, and their scales [n, Hkv, 2]."""
    page = pool.page
    numbers_of = pool.table[row, :-(-n // page)].long().cpu()
    k, v, s = numbers(pool.k_pages)[layer][numbers_of], numbers(pool.v_pages)[layer][numbers_of], pool.scales.cpu().double()[layer][numbers_of]
    m, Hkv, d = len(numbers_of), pool.Hkv, pool.d
    s = s.repeat_interleave(16, 2).permute(0, 2, 1, 3).reshape(m * page, Hkv, 2)
    k = k.permute(0, 3, 1, 2, 4).reshape(m * page, Hkv, d) * s[..., :1]
    v = v.permute(0, 2, 4, 1, 3).reshape(m * page, Hkv, d) * s[..., 1:]
    return k[:n].numpy(), v[:n].numpy(), s[:n].numpy()
