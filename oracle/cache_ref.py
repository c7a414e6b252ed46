"""Oracle of the quantised cache: quantiser, rows read back and attention, written from their definitions with numpy.

Codes are decisions on 32-bit numbers (differences, products with the reciprocal) and 16-bit scales and zeros; everything that
follows from them is 64 bits, apart from the rounding steps that the definition of a row read back names."""
import numpy as np

DIM = 128
TOP = 65504.0


def to_type(x, bf16):
    """Rounds 32-bit numbers to fp16 or bf16 (nearest even), as 64-bit values."""
    x = np.asarray(x, dtype=np.float32)
    if not bf16:
        return x.astype(np.float16).astype(np.float64)
    b = x.view(np.uint32).astype(np.uint64)
    b = ((b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32)
    return b.view(np.float32).astype(np.float64)


def transform32(x, factor):
    """H x * factor in 32 bits, scaled first: sums and differences at strides 1, 2, ..., 64."""
    y = (np.asarray(x, dtype=np.float32) * np.float32(factor)).astype(np.float32)
    h = 1
    while h < DIM:
        y = y.reshape(-1, DIM // (2 * h), 2, h)
        y = np.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], axis=2)
        h *= 2
    return y.reshape(np.shape(x))


def hadamard():
    h = np.ones((1, 1))
    while h.shape[0] < DIM:
        h = np.block([[h, h], [h, -h]])
    return h


class Tensor:
    """The rows [..., 128] of K or V as the cache holds them: codes, and scale and zero per channel (64-bit values of fp16 numbers)."""

    def __init__(self, x, bits, group, bf16, rotate=False):
        x = np.asarray(x, dtype=np.float32)
        if rotate:
            top = np.float32(3.3895313892515355e38 if bf16 else TOP)
            x = to_type(np.clip(transform32(x, 0.125), -top, top), bf16).astype(np.float32)
        x = np.clip(np.where(np.isnan(x), np.float32(0), x), np.float32(-TOP), np.float32(TOP))
        g = x.reshape(*x.shape[:-1], DIM // group, group)
        lo, hi = g.min(-1, keepdims=True) + np.float32(0), g.max(-1, keepdims=True) + np.float32(0)
        zero = lo.astype(np.float16)
        scale = ((hi - lo) / np.float32(2 ** bits - 1)).astype(np.float16)
        s32 = scale.astype(np.float32)
        inv = np.where(s32 > 0, np.float32(1) / np.where(s32 > 0, s32, np.float32(1)), np.float32(0)).astype(np.float32)
        code = np.clip(np.rint((g - zero.astype(np.float32)) * inv), 0, 2 ** bits - 1)
        self.code = code.reshape(x.shape).astype(np.float64)
        self.scale = np.broadcast_to(scale.astype(np.float64), g.shape).reshape(x.shape)
        self.zero = np.broadcast_to(zero.astype(np.float64), g.shape).reshape(x.shape)
        self.rotate = rotate

    def values(self):
        """What the rows stand for (rotated rows: still rotated)."""
        return self.code * self.scale + self.zero

    def parts(self):
        """|code * scale| + |zero|: the sizes that rounding errors go by."""
        return self.code * self.scale + np.abs(self.zero)

    def read_back(self, bf16):
        """Rows read back: one fused multiply-add in 32 bits, the rotation in 32 bits, limited to +-65504, rounded to the type."""
        x = self.values().astype(np.float32)
        if self.rotate:
            x = transform32(x, 0.0625)
        return to_type(np.clip(x, np.float32(-TOP), np.float32(TOP)), bf16)


def attention(q, k, v, seen, scale, per_kv):
    """One sequence.  q [new, q_heads, 128] (64-bit), k, v: Tensor [tokens, kv_heads, 128], seen [new, tokens].
    Returns out, lse and, for tolerances, per output the sum of weight * |value| and per row the largest sum of |products|."""
    if k.rotate:
        q = q @ hadamard() / 16
    new, heads, _ = q.shape
    kv, vv, kp, vp = k.values(), v.values(), k.parts(), v.parts()
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((new, heads), -np.inf), np.zeros((new, heads))
    for h in range(heads):
        s = q[:, h] @ kv[:, h // per_kv].T * scale
        b = np.abs(q[:, h]) @ kp[:, h // per_kv].T * abs(scale)
        for r in range(new):
            at = np.flatnonzero(seen[r])
            if not at.size:
                continue
            top = s[r, at].max()
            w = np.exp(s[r, at] - top)
            lse[r, h] = top + np.log(w.sum())
            w /= w.sum()
            out[r, h] = w @ vv[at, h // per_kv]
            size[r, h] = w @ vp[at, h // per_kv]
            reach[r, h] = b[r, at].max()
    return out, lse, size, reach
