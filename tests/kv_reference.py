"""Plain 64-bit implementations of the operators around the quantized cache, for the tests: no code of the package, the layout from the
header's words."""
import math

import numpy as np
import torch

QMAX = {4: 15, 8: 255}


def quantize(x, bits):
    """codes (int64), scale and least value (float64, both fp16 numbers) of fp16 heads [..., hd], by the header's definition."""
    x = np.asarray(x, np.float16).astype(np.float64)
    nan = np.isnan(x)
    x = np.clip(x, -65504.0, 65504.0)
    lo = np.where(nan, np.inf, x).min(-1, keepdims=True)
    hi = np.where(nan, -np.inf, x).max(-1, keepdims=True)
    none = nan.all(-1, keepdims=True)
    lo, hi = np.where(none, 0.0, lo) + 0.0, np.where(none, 0.0, hi)
    span = (hi - lo).astype(np.float32)
    scale = (span / np.float32(QMAX[bits])).astype(np.float16)
    scale = np.where(scale == 0, np.float16(2.0 ** -24), scale).astype(np.float64)
    diff = (np.where(nan, lo, x) - lo).astype(np.float32)
    codes = np.clip(np.rint(diff / scale.astype(np.float32)), 0, QMAX[bits])
    return codes.astype(np.int64), scale[..., 0], lo[..., 0]


def held(codes, scale, lo):
    """The fp16 numbers that a read returns: lo + scale * code rounded to fp32, no more than 65504, then rounded to fp16."""
    return np.minimum((lo[..., None] + scale[..., None] * codes).astype(np.float32), np.float32(65504)).astype(np.float16)


def code_place(token, channel, hd, bits, value):
    """(byte in a block's codes, shift in the byte) of a code; arrays."""
    h, p = token // 8, channel % 16 // 8
    if value:
        r, c, b = channel % 8, token % 8 // 2, token % 2
    else:
        r, c, b = token % 8, channel % 8 // 2, channel % 2
    if bits == 4:
        w, byte, shift = channel // 16, 2 * b + h, 4 * p
    else:
        w = 2 * (channel // 16) + (p if value else h)
        byte, shift = (2 * h + b if value else 2 * p + b), 0 * p
    return 512 * (w // 4) + 16 * (4 * r + c) + 4 * (w % 4) + byte, shift


class Cache:
    """Pages on the CPU (numpy) that stand for known codes; built from fp16 keys and values per sequence."""

    def __init__(self, heads, hd, bits, page, n_pages, rng):
        self.heads, self.hd, self.bits, self.page = heads, hd, bits, page
        self.cb = 2 * hd * bits
        self.block = 2 * self.cb + 128
        self.pages = rng.integers(0, 256, (n_pages, heads, page // 16, self.block), dtype=np.uint8)   # whatever was there

    def put(self, pages, first, k, v):
        """Quantizes fp16 k, v [tokens][heads][hd] as tokens first, first + 1, ... of the sequence with that page list."""
        ch = np.arange(self.hd)
        for value, x in ((False, k), (True, v)):
            codes, scale, lo = quantize(x, self.bits)
            for i in range(x.shape[0]):
                t = first + i
                page, blk, slot = pages[t // self.page], t % self.page // 16, t % 16
                at, shift = code_place(np.full_like(ch, slot), ch, self.hd, self.bits, value)
                for h in range(self.heads):
                    raw = self.pages[page, h, blk]
                    part = raw[self.cb:2 * self.cb] if value else raw[:self.cb]
                    if self.bits == 4:
                        for s in (0, 4):
                            m = shift == s
                            part[at[m]] = (part[at[m]] & (0xf0 >> s)) | (codes[i, h][m] << s).astype(np.uint8)
                    else:
                        part[at] = codes[i, h].astype(np.uint8)
                    pair = np.array([scale[i, h], lo[i, h]], np.float16).view(np.uint8)
                    raw[2 * self.cb + 64 * value + 4 * slot:][:4] = pair


def values(pages_tensor, heads, hd, bits, page, table, n):
    """(codes * scale, least value, scale) of keys and of values, float64 torch [tokens][heads][hd] ([..., 1] the others), of the first n tokens of a page list.
    On the device of `pages_tensor` (uint8 [n_pages][bytes])."""
    dev = pages_tensor.device
    blocks = (n + 15) // 16
    t, ch = torch.meshgrid(torch.arange(16, device=dev), torch.arange(hd, device=dev), indexing="ij")
    cb = 2 * hd * bits
    raw = pages_tensor.view(pages_tensor.shape[0], heads, page // 16, 2 * cb + 128)
    b = torch.arange(blocks, device=dev)
    raw = raw[table[(b * 16 // page)].long(), :, b % (page // 16)]                  # block, head, bytes
    out = []
    for value in (False, True):
        at, shift = code_place(t, ch, hd, bits, value)
        code = raw[..., cb * value:cb * value + cb][..., at].long()
        if bits == 4:
            code = (code >> shift) & 15
        pair = raw[..., 2 * cb + 64 * value:2 * cb + 64 * value + 64].contiguous().view(torch.float16).view(blocks, heads, 16, 2).double()
        s, lo = pair[..., :1], pair[..., 1:]
        out.append([x.transpose(1, 2).reshape(blocks * 16, heads, -1)[:n] for x in (code * s, lo, s)])
    return out


def attention(q, kv, seen, scale):
    """(out, bound) of query rows q [n][hq][hd] (float64) over kv = values(...) of all tokens, row i seeing the tokens where seen[i] is true.

    bound, element by element: half a step of the fp16 result, and in units of A + B with A = sum p s d / sum p, B = sum p |lo| / sum p
      2^-11                    the weights' 11 bits, each off by no more than that from a factor that all of a row share
      (tokens / 16 + 64) 2^-23 one accumulator update per 16 tokens (the tensor core truncates), and the joining of partial sums
      2^-20 m                  scores: fp32 sums of terms up to m = scale (|q| s c + |sum q| |lo|), a few roundings, and the exponential
    and 2^-25 of the greatest weight per token, for weights that fp16 holds as subnormal numbers."""
    (kc, kl, _), (vc, vl, vs) = kv
    n, hq, hd = q.shape
    g = hq // kc.shape[1]
    rep = lambda x: x.repeat_interleave(g, 1)  # noqa: E731
    k = rep(kc + kl)
    scores = torch.einsum("nhd,thd->nht", q, k) * scale
    m = (torch.einsum("nhd,thd->nht", q.abs(), rep(kc)) + q.sum(-1, keepdim=True).abs() * rep(kl)[..., 0].T.abs()[None]) * abs(scale)
    scores = torch.where(seen[:, None, :], scores, torch.full_like(scores, -math.inf))
    m = torch.where(seen[:, None, :], m, torch.zeros_like(m)).amax(-1, keepdim=True) if k.shape[0] else torch.zeros((n, hq, 1), device=q.device)
    any_seen = seen.any(-1)[:, None, None]
    if k.shape[0] == 0:
        z = torch.zeros_like(q)
        return z, z
    top = scores.amax(-1, keepdim=True)
    p = torch.where(any_seen, torch.exp(scores - torch.where(any_seen, top, torch.zeros_like(top))), torch.zeros_like(scores))
    p = torch.where(seen[:, None, :], p, torch.zeros_like(p))
    den = p.sum(-1, keepdim=True).clamp(min=1e-300)
    out = torch.einsum("nht,thd->nhd", p, rep(vc + vl)) / den
    a = torch.einsum("nht,thd->nhd", p, rep(vc)) / den
    b = torch.einsum("nht,th->nh", p, rep(vl)[..., 0].abs())[..., None] / den
    tokens = k.shape[0]
    small = tokens * 2.0 ** -25 * (p * rep(vs)[..., 0].T[None]).amax(-1, keepdim=True) * vc.div(vs.clamp(min=1e-30)).amax() / den
    bound = 2.0 ** -11 * out.abs() + 2.0 ** -25 + (2.0 ** -11 + (tokens / 16 + 64) * 2.0 ** -23 + 2.0 ** -20 * (1 + m)) * (a + b) + small
    return torch.where(any_seen, out, torch.zeros_like(out)), bound


def attention_norm(q, kv, seen, scale, updates=128):
    """(out, bound) as attention(), with a bound [n][hq] of the norm of a row and head's error.

    In terms of w = p / sum p and S = sqrt(sum w^2 |v - out|^2), the norm that errors of the weights add up to when they are independent:
      2^-11 |out|                    the result's rounding
      2 * 2^-11 S                    the weights' 11 bits, the same in products and sums.  Each is off by at most 2^-11 and by 0.42 * 2^-11 in the mean square (an
                                     error uniform in half a step either way, a mantissa of logarithmic density): nearly five deviations, and for up to four tokens the worst case
      updates 2^-23 * 4 (|out| + S)  accumulators: each update cuts off less than 2^-23 of what they hold, a walk of no more than some S
      2 * 2^-20 (1 + m) S            scores: an error of up to 2^-20 (1 + m), as in attention(), is one of the weight, and has as little to do with the value as the weight's rounding
    and half a step of a subnormal result per channel."""
    (kc, kl, _), (vc, vl, _) = kv
    n, hq, hd = q.shape
    rep = lambda x: x.repeat_interleave(hq // kc.shape[1], 1)  # noqa: E731
    hide = ~seen[:, None, :]
    scores = (torch.einsum("nhd,thd->nht", q, rep(kc + kl)) * scale).masked_fill(hide, -math.inf)
    m = (torch.einsum("nhd,thd->nht", q.abs(), rep(kc)) + q.sum(-1, keepdim=True).abs() * rep(kl)[..., 0].T.abs()[None]) * abs(scale)
    m = m.masked_fill(hide, 0).amax(-1)
    w, v = torch.softmax(scores, -1).nan_to_num(0.0), rep(vc + vl)
    out = torch.einsum("nht,thd->nhd", w, v)
    size = out.norm(dim=-1)
    away = (v.pow(2).sum(-1).T[None] - 2 * torch.einsum("nhd,thd->nht", out, v) + size[..., None] ** 2).clamp(min=0)
    s = (w ** 2 * away).sum(-1).sqrt()
    bound = 2.0 ** -11 * (size + 2 * s) + updates * 2.0 ** -21 * (size + s) + 2.0 ** -19 * (1 + m) * s + 2.0 ** -25 * hd ** 0.5
    return out, bound


def rope(x, positions, freq, rot, interleaved, magnitude):
    """(y, bound) of fp16 heads x [rows][heads][hd], 64 bits; freq [rot / 2]."""
    x = np.asarray(x, np.float16).astype(np.float64)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(freq, np.float64)[None, :]
    c, s = (magnitude * f(angle)[:, None, :] for f in (np.cos, np.sin))
    y, mag = x.copy(), np.zeros_like(x)
    ia = np.arange(rot // 2) * 2 if interleaved else np.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia] = mag[..., ib] = np.abs(a) + np.abs(b)
    # the result's rounding, and sine and cosine: an angle within 2^-24 of itself and 2^-33 turns, two roundings of theirs, two products and a sum
    return y, 2.0 ** -11 * np.abs(y) + 2.0 ** -25 + 2.0 ** -20 * abs(magnitude) * mag
