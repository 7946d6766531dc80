"""Rows of a table and rows in 8 bits, from their definitions: host, plain, slow."""
import math

import numpy as np
import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}


def e4m3_values():
    """The non-negative numbers with four bits of exponent (bias 7) and three of fraction, code 0 .. 126."""
    out = []
    for code in range(127):
        e, f = code >> 3, code & 7
        out.append(math.ldexp(8 + f, e - 10) if e else math.ldexp(f, -9))
    return np.array(out)


E4M3 = e4m3_values()


def nearest_e4m3(v):
    """Codes of the nearest numbers (ties: the even code), v float64 within +-448."""
    m = np.abs(v)
    high = np.clip(np.searchsorted(E4M3, m), 1, 126)
    low = high - 1
    below, above = m - E4M3[low], E4M3[high] - m
    take = np.where(below < above, low, np.where(above < below, high, np.where(low % 2 == 0, low, high)))
    return (take | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quantize(v, group, kind):
    """(codes as bytes, scales) of fp32 values [rows, d]: every operation one rounded fp32 one."""
    v = v.float().numpy()
    rows, d = v.shape
    group = group or d
    q = np.float32(LARGEST[kind])
    codes = np.zeros((rows, d), np.uint8)
    scales = np.zeros((rows, -(-d // group)), np.float32)
    with np.errstate(all="ignore"):
        for g in range(scales.shape[1]):
            part = v[:, g * group:(g + 1) * group]
            m = np.abs(part).max(1)  # (NaN where there is one)
            m = np.where(np.isnan(m), m, np.maximum(m, np.float32(2.0 ** -90))).astype(np.float32)
            scale = m / q
            x = part * (np.float32(1.0) / scale)[:, None]
            assert scale.dtype == x.dtype == np.float32
            scales[:, g] = scale
            x = x.astype(np.float64)
            if kind == torch.int8:
                c = np.where(np.isnan(x), 0, np.clip(np.rint(x), -127, 127)).astype(np.int8).view(np.uint8)
            else:
                c = np.where(np.isnan(x), 127, nearest_e4m3(np.clip(np.where(np.isnan(x), 0, x), -448, 448)))
            codes[:, g * group:(g + 1) * group] = c
    return torch.from_numpy(codes), torch.from_numpy(scales)


def values(codes, scales, group, kind):
    """What codes (bytes, [.., d]) and scales stand for, float64."""
    d = codes.shape[-1]
    group = group or d
    if kind == torch.int8:
        v = codes.view(torch.int8).double()
    else:
        table = torch.tensor(np.concatenate([E4M3, [math.nan], -E4M3, [math.nan]]))
        v = table[codes.long()]
    return v * scales.double().repeat_interleave(group, -1)[..., :d]


def places(pages, page_rows, num_pages, n, offsets=None, starts=None):
    """Row of the cache of each of the call's n rows: -1 without a place, -2 of no sequence."""
    batch = pages.shape[0]
    if offsets is None:
        per = n // batch if batch else 0
        offsets = [k * per for k in range(batch + 1)]
    out = [-2] * n
    for s in range(batch):
        for r in range(offsets[s], min(offsets[s + 1], n)):
            pos = (starts[s] if starts is not None else 0) + r - offsets[s]
            out[r] = -1
            if 0 <= pos < pages.shape[1] * page_rows:
                page = int(pages[s, pos // page_rows])
                if 0 <= page < num_pages:
                    out[r] = page * page_rows + pos % page_rows
    return out


def table_sums(grad, ids, vocab, skip=-1):
    """Sums of the gradient rows of each id, and of their magnitudes; float64."""
    keep = (ids >= 0) & (ids < vocab) & (ids != skip)
    s = torch.zeros(vocab, grad.shape[1], dtype=torch.float64)
    l1 = torch.zeros_like(s)
    s.index_add_(0, ids[keep].long(), grad[keep].double())
    l1.index_add_(0, ids[keep].long(), grad[keep].double().abs())
    return s, l1


def attention(q, k, v, bias=None):
    """q [heads, dim], k, v [keys, dim], bias [keys, heads], float64: (result, probabilities [heads, keys])"""
    x = q @ k.t()
    if bias is not None:
        x = x + bias.t()
    p = torch.softmax(x, 1)
    return p @ v, p
