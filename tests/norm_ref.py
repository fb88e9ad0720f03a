"""The normed rotation and its gradient in 64 bits, in numpy, from their definition, and
how far fp32 arithmetic may take a result from them.

Tolerances: a sum of d squares takes at most 2 N + 4 <= 20 roundings of 2^-24 (16 values a
lane, then the lanes), its inverse root half of them and 1.5 steps of its own, so r is
within 2^-20 of itself, and so is n = x r.  The rotation is off by (|x1| + |x2|) scale 2^-20
(tests/test_gpu_rope.py).  So out is off by (|y1| + |y2|) scale 2^-19; with A = |w| (|g1| +
|g2|) scale, a bound of |w g|, dx is off by r (A + |n| mean(A |n|)) 2^-18; and dw by the sum
of its terms' bounds, 2^-18 of each and 2^-24 for each rounding of the sum.  Where rows are
bf16, half a step more (2^-8 of the value)."""
import numpy as np

from tests import q8_ref as ref


class Norm:
    """x, dout [L, B, n, H, d], w [L, d], pos [3, B, n]; all in 64 bits."""

    def __init__(self, x, w, pos, rot, freq, ax, adjacent, inverse=False, scale=1.0, eps=1e-6, count=None):
        self.x, self.w = np.asarray(x, np.float64), np.asarray(w, np.float64)[:, None, None, None]
        self.pos, self.args, self.scale = pos, (rot, freq, ax, adjacent), scale
        self.inverse = inverse
        self.r = 1.0 / np.sqrt((self.x ** 2).mean(axis=-1, keepdims=True) + np.float64(np.float32(eps)))
        self.n = self.x * self.r
        B, n = x.shape[1:3]
        live = np.arange(n)[None] < np.asarray([n] * B if count is None else count)[:, None]
        self.live = np.broadcast_to(live[None, :, :, None, None], self.x.shape)

    def _turn(self, y, inverse):
        out = np.empty_like(y)
        for l in range(y.shape[0]):
            for b in range(y.shape[1]):
                for h in range(y.shape[3]):
                    out[l, b, :, h] = ref.rope(y[l, b, :, h], self.pos[:, b], *self.args, inverse, self.scale)
        return out

    def _pairs(self, y):
        """|y1| + |y2| of each channel's pair, times the scale."""
        rot, _, _, adjacent = self.args
        out, a = np.abs(y), np.abs(y)
        for i in range(rot // 2):
            p, q = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
            out[..., p] = out[..., q] = (a[..., p] + a[..., q]) * abs(self.scale)
        return out

    def forward(self):
        return self._turn(self.n * self.w, self.inverse)

    def forward_tol(self, fp32):
        return self._pairs(self.n * self.w) * 2.0 ** -19 + (0 if fp32 else np.abs(self.forward()) * 2.0 ** -8)

    def grad(self, dout):
        """(dx, dw) and their tolerances for fp32 rows; `roundings` of the sum for dw are added by the caller."""
        dout = np.asarray(dout, np.float64)
        g = self._turn(dout, not self.inverse)
        A = self._pairs(dout)
        dn = self.w * g
        dx = self.r * (dn - self.n * (dn * self.n).mean(axis=-1, keepdims=True))
        bound = np.abs(self.w) * A
        dx_tol = self.r * (bound + np.abs(self.n) * (bound * np.abs(self.n)).mean(axis=-1, keepdims=True)) * 2.0 ** -18
        terms, size = np.where(self.live, g * self.n, 0), np.where(self.live, A * np.abs(self.n), 0)
        return dx, terms.sum(axis=(1, 2, 3)), dx_tol, size.sum(axis=(1, 2, 3))
