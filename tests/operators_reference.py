"""Plain 64-bit forms of the operators around the cache, for their tests (numpy; written from the formulas)."""
from __future__ import annotations

import numpy as np

from oracle import kivi_oracle as ko


def table(positions, rotary_dim, base=10000.0):
    """Cosines and sines [positions, rotary_dim] in fp32."""
    angle = np.arange(positions)[:, None] * base ** (-np.arange(0, rotary_dim, 2) / rotary_dim)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


def _pairs(rotary_dim, interleaved):
    i = np.arange(rotary_dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary_dim // 2)


def rotate(x, rows, interleaved=False):
    """x [..., rows, heads, 128], rows [..., rows, rotary_dim] of the table; in x's precision, every operation rounded on its own."""
    x = x.copy()
    half = rows.shape[-1] // 2
    a, b = _pairs(2 * half, interleaved)
    c, s = (r[..., None, :].astype(x.dtype) for r in (rows[..., :half], rows[..., half:]))
    xa, xb = x[..., a], x[..., b]
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def visible(n_q, n_k, window, sinks):
    """[n_q, n_k]: whether query i (at key n_k - n_q + i) sees key j."""
    p, j = np.arange(n_q)[:, None] + n_k - n_q, np.arange(n_k)
    see = j <= p
    if window:
        see &= (p - j < window) | (j < sinks)
    return see


def attention(q, k, v, scale, see):
    """q [n_q, H_q, 128], k, v [n_k, H_kv, 128], see [n_q, n_k].  Returns the output, the mean of |v| under the same weights, and
    scale * sum |q| |k| of the largest logit terms (what the error of a logit is relative to), all [n_q, H_q, 128] or [n_q, H_q, 1]."""
    rep = q.shape[1] // k.shape[1]
    out, mean_abs, terms = (np.zeros(q.shape) for _ in range(3))
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    for h in range(q.shape[1]):
        kh, vh = k[:, h // rep], v[:, h // rep]
        x = np.where(see, scale * (q[:, h] @ kh.T), -np.inf)
        m = x.max(1, keepdims=True, initial=-1e300)
        p = np.where(see, np.exp(x - m), 0.0)
        total = p.sum(1, keepdims=True)
        p /= np.where(total == 0, 1.0, total)
        out[:, h], mean_abs[:, h] = p @ vh, p @ np.abs(vh)
        if k.shape[0]:
            terms[:, h] = (abs(scale) * np.where(see, np.abs(q[:, h]) @ np.abs(kh).T, 0.0)).max(1, keepdims=True, initial=0.0)
    return out, mean_abs, terms[..., :1]


class Sequence:
    """One sequence of a paged cache, by the oracle: keys and values [tokens, H_kv, 128] fp16 (keys rotated already)."""

    def __init__(self, kv_heads, bits, residual):
        self.cache = ko.StreamingCache(1, kv_heads, 128, bits, 32, residual, "window")
        self.bits, self.residual = bits, residual

    def append(self, k, v):
        if self.cache.length == 0:
            self.cache.prefill(k.transpose(1, 0, 2)[None], v.transpose(1, 0, 2)[None])
            return
        for i in range(k.shape[0]):
            self.cache.append(k[i][None], v[i][None])

    @property
    def length(self):
        return self.cache.length

    def records(self):
        """[records, H_kv, words] as the cache stores them."""
        c, n = self.cache, self.cache.n_kq // 32
        if n == 0:
            return np.zeros((0, c.k_codes.shape[1], 256 + 256 * self.bits // 1), np.uint32)
        kc, vc = ko.pack_key_codes(c.k_codes, self.bits)[0], ko.pack_value_codes(c.v_codes, self.bits)[0]
        h = kc.shape[0]
        scales = [np.ascontiguousarray(x[0]).reshape(h, n, 128).view(np.uint32) for x in (c.k_scale, c.k_zero, c.v_scale, c.v_zero)]
        return np.concatenate([kc.reshape(h, n, -1)] + scales + [vc.reshape(h, n, -1)], 2).transpose(1, 0, 2)

    def rows(self):
        """keys, values [rows, H_kv, 128] of the window."""
        return self.cache.k_resid[0].transpose(1, 0, 2), self.cache.v_resid[0].transpose(1, 0, 2)

    def values(self):
        """keys, values [tokens, H_kv, 128] in 64 bits as the cache stands for them, and the magnitudes that the logits' and outputs'
        terms have (code times scale plus zero-point)."""
        c = self.cache
        k = ko.dequantize_key(c.k_codes, c.k_scale, c.k_zero, 32)[0]
        v = ko.dequantize_value(c.v_codes, c.v_scale, c.v_zero, 32)[0]
        kz, vz = (np.abs(x[0].astype(np.float64)) for x in (c.k_zero, c.v_zero))
        km = np.abs(k) + 2 * np.repeat(kz, 32, 1)[:, :k.shape[1]]
        vm = np.abs(v) + 2 * np.repeat(vz, 32, 2)
        join = lambda a, b: np.concatenate([a, b[0].astype(np.float64)], 1).transpose(1, 0, 2)   # noqa: E731
        return join(k, c.k_resid), join(v, c.v_resid), join(km, np.abs(c.k_resid)), join(vm, np.abs(c.v_resid))
