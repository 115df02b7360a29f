"""The cache format and its attention in 64 bits, written from the format's description: quantised values, the bytes of a
page by index formula, attention over what the codes stand for."""
import numpy as np
import torch

GRID = {4: [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0],
        8: [(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127]}


def quantise(x, bits):
    """float64 [..., 128] -> (codes uint8 [..., 128], exponents uint8 [..., 4])."""
    x = np.asarray(x, np.float64)
    g = np.array(GRID[bits])
    blk = x.reshape(x.shape[:-1] + (4, 32))
    top = np.abs(blk).max(-1)
    mant, ex = np.frexp(top / g[-1])              # top / M = mant 2^ex, mant in [0.5, 1)
    e = np.where(top == 0, -126, np.where(mant == 0.5, ex - 1, ex))
    e = np.maximum(e, -126)
    y = blk / np.exp2(e.astype(np.float64))[..., None]
    a = np.abs(y)
    hi = np.minimum(np.searchsorted(g, a), len(g) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = g[hi] - a, a - g[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code | np.where(np.signbit(y), 8 if bits == 4 else 128, 0)
    return code.reshape(x.shape).astype(np.uint8), (e + 127).astype(np.uint8)


def values(code, exponent, bits):
    g = np.array(GRID[bits])
    sign = 8 if bits == 4 else 128
    v = np.where(code & sign, -1.0, 1.0) * g[code & (sign - 1)]
    s = np.exp2(exponent.astype(np.float64) - 127)
    return (v.reshape(v.shape[:-1] + (4, 32)) * s[..., None]).reshape(v.shape)


def places(bits, is_value):
    """Byte of each row's columns [64, 128] and of its scales [64, 4] within a page."""
    r, c = np.arange(64)[:, None], np.arange(128)[None]
    C, e, j = 16 * bits, bits, np.arange(4)[None]
    i, within = c // 8, (c % 8) * bits // 8
    if not is_value:
        return r * C + i * e + within, 64 * C + 16 * j * 4 + (r % 16) * 4 + r // 16
    return (r // 4) * 4 * C + 4 * i * e + (r % 4) * e + within, 64 * C + (r // 4 % 4) * 64 + 16 * j + (r // 16) * 4 + r % 4


def page_bytes(bits):
    return 64 * 16 * bits + 256


def unpack(blob, bits, is_value):
    """uint8 [..., pages, bytes] -> codes [..., rows, 128], exponents [..., rows, 4]."""
    at, se = places(bits, is_value)
    raw = blob[..., at]
    if bits == 4:
        raw = np.where(np.arange(128) % 2 == 0, raw & 15, raw >> 4)
    lead = blob.shape[:-2]
    return raw.reshape(lead + (-1, 128)), blob[..., se].reshape(lead + (-1, 4))


def pack(code, exponent, bits, is_value, fill=0xFF):
    """Rows [..., n, 128] to pages; bytes of rows that are not there are `fill`."""
    at, se = places(bits, is_value)
    lead, n = code.shape[:-2], code.shape[-2]
    pages = (n + 63) // 64
    pad = [(0, 0)] * len(lead) + [(0, pages * 64 - n), (0, 0)]
    wide = 15 if bits == 4 else 255
    c = np.pad(code, pad, constant_values=fill & wide).reshape(lead + (pages, 64, 128))
    s = np.pad(exponent, pad, constant_values=fill).reshape(lead + (pages, 64, 4))
    blob = np.zeros(lead + (pages, page_bytes(bits)), np.uint8)
    if bits == 4:
        blob[..., at[:, 0::2]] = c[..., 0::2] | c[..., 1::2] << 4
    else:
        blob[..., at] = c
    blob[..., se] = s
    return blob


def attend(q, k, v, lens, counts, scale):
    """float64 CUDA tensors q [B, Hq, n, 128], k, v [B, Hkv, rows, 128] -> (o, A = sum of w |v|, S = largest scale sum |q k|
    of a query and its keys), zero rows where nothing is seen."""
    B, Hq, n, _ = q.shape
    g = Hq // k.shape[1]
    o, mag = torch.zeros_like(q), torch.zeros_like(q)
    big = torch.zeros(q.shape[:3], dtype=torch.float64, device=q.device)
    for b in range(B):
        first = max(0, counts[b] - lens[b])              # queries before that see nothing
        t = torch.arange(first, counts[b], device=q.device)
        if len(t) == 0 or lens[b] == 0:
            continue
        unseen = torch.arange(lens[b], device=q.device) > (lens[b] - counts[b] + t)[:, None]
        for h in range(Hq):
            kk, vv, qq = k[b, h // g, :lens[b]], v[b, h // g, :lens[b]], q[b, h, first:counts[b]]
            w = torch.softmax((qq @ kk.T.contiguous() * scale).masked_fill(unseen, -torch.inf), 1)
            o[b, h, first:counts[b]], mag[b, h, first:counts[b]] = w @ vv, w @ vv.abs()
            big[b, h, first:counts[b]] = (qq.abs() @ kk.abs().T.contiguous() * scale).masked_fill(unseen, 0.0).amax(1)
    return o, mag, big[..., None]
