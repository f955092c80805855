"""Plain implementations of the operators around the training step, for their tests: layer norm and its
gradients in 64 bits, and the AdamW step, its states in the fp32 arithmetic that the header defines (each
fused multiply-add as a 64-bit sum rounded once: the product of two fp32 values is exact there)."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24     # half a step of fp32, relative
U16 = 2.0 ** -8      # of bf16
M64 = (1 << 64) - 1


def layer_norm(h, w, b, eps):
    h = h.astype(np.float64)
    mean = h.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    xh = (h - mean) * rstd
    return xh * (1.0 if w is None else w) + (0.0 if b is None else b), mean, rstd


def layer_norm_grads(h, w, mean, rstd, dx):
    """dH, dweight, dbias, in 64 bits from the given mean and rstd."""
    h, dx = h.astype(np.float64), dx.astype(np.float64)
    xh = (h - mean) * rstd
    q = dx * (1.0 if w is None else w.astype(np.float64))
    s, t = q.mean(1, keepdims=True), (q * xh).mean(1, keepdims=True)
    return rstd * (q - s - xh * t), (dx * xh).sum(0), dx.sum(0)


def splitmix64(seed, i):
    """Output i (an array of uint64) of the stream of a seed."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed & M64) + (np.asarray(i, np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def e4m3(code):
    """E4M3 bytes as fp64: bias 7, no infinities, 0x7f NaN."""
    c = np.asarray(code, np.int64)
    e, f = (c >> 3) & 15, c & 7
    x = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c & 128, -x, x)


def scale_of(s):
    return np.where(np.asarray(s) == 0, 0.0, 2.0 ** (np.asarray(s, np.float64) - 127))


def _blocks(x):
    pad = np.zeros(-len(x) % 32, x.dtype)
    return np.concatenate([x, pad]).reshape(-1, 32)


def _store(x, d, root):
    """(codes, scales) of the fp32 values x under the 16-bit draws d."""
    n = len(x)
    a = np.abs(_blocks(x.astype(np.float64)))
    fin = np.where(np.isfinite(a), a, 0.0)
    top = fin.max(1)
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1 + 127, 0)
    s = np.maximum(e, 23) - 7
    y = fin * 2.0 ** (127.0 - s)[:, None]
    small = y < 2.0 ** -6
    step = np.where(small, 2.0 ** -9, 2.0 ** (np.floor(np.log2(np.where(small, 1.0, y))) - 3))
    q = np.floor(y / step + _blocks(d.astype(np.float64)) / 65536.0) * step
    if root:
        q = np.where((fin > 0) & (q == 0), 2.0 ** -9, q)
    f, ex = np.frexp(np.where(q >= 2.0 ** -6, q, 1.0))
    code = np.where(q >= 2.0 ** -6, (ex + 6) * 8 + np.rint(f * 16) - 8, np.rint(q * 512)).astype(np.int64)
    code = np.where(np.isfinite(a), code, 127).reshape(-1)[:n]
    if not root:
        code = code | np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8), s.astype(np.uint8)


def adamw(w, g, m, v, scale, o, k=0, lr_scale=1.0, decay=0.0, gs=1.0, first=0):
    """One step on fp32 arrays w (the weights before their rounding), g, m, v; scale is None or the 8-bit
    moments' scales [blocks, 2] with m, v their bytes.  o: the options as a dict; first: the place of w[0] in
    tensor k of the list, a multiple of 32.  Returns (w in 64 bits, the size of its update, m, v, scale)."""
    f32 = np.float32
    n = len(w)
    with np.errstate(all="ignore"):
        g = g.astype(f32) * f32(gs)
        if scale is not None:
            sm, sv = (np.repeat(scale_of(scale[:, j]), 32)[:n] for j in (0, 1))
            m = (e4m3(m) * sm).astype(f32)
            v = (e4m3(v) * sv).astype(f32)
            v = v * v
        b1, c1, b2, c2 = f32(o["beta1"]), f32(1 - o["beta1"]), f32(o["beta2"]), f32(1 - o["beta2"])
        m = (np.float64(b1) * m.astype(np.float64) + (c1 * g).astype(np.float64)).astype(f32)
        v = (np.float64(b2) * v.astype(np.float64) + (c2 * g * g).astype(np.float64)).astype(f32)
        r = np.sqrt(v.astype(np.float64)).astype(f32)
        t = o["step"]
        lr = o["lr"] * lr_scale
        u = m.astype(np.float64) / (1 - o["beta1"] ** t) / (np.sqrt(v.astype(np.float64)) / np.sqrt(1 - o["beta2"] ** t)
                                                           + o["eps"])
        w = w.astype(np.float64)
        step = lr * (decay * w + u)
        if scale is None:
            return w - step, np.abs(lr * u) + np.abs(lr * decay * w), m, v, None
        i = np.arange(first, first + n, dtype=np.uint64)
        z = splitmix64(int(splitmix64(o["seed"] + t, 0)), (np.uint64(k) << np.uint64(40)) + (i >> np.uint64(2)))
        d = ((z >> (np.uint64(16) * (i & np.uint64(3)))) & np.uint64(0xffff)).astype(np.int64)
        qm, em = _store(m, d, False)
        qv, ev = _store(r, 65535 - d, True)
        return w - step, np.abs(lr * u) + np.abs(lr * decay * w), qm, qv, np.stack([em, ev], 1)
