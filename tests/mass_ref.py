"""Attention that adds up its rows' weights, in 64 bits, in numpy, from its definition, and
how far fp32 arithmetic may take a result from it.

Tolerances: bf16 products are exact in fp32, and a logit is a sum of d of them with the
scale's two roundings, so it is within E = (d + 4) 2^-24 scale sum |q K| of its value, the
largest over the query's rows.  A weight p takes the errors of its own logit and of the
others' through the sum (2 E), the exponential (2^-22), and the roundings of the sum of r
rows, which lanes form 32 rows apart and then join: delta = 2 E + (r / 32 + 64) 2^-24 of
itself.  An output is the sum of p V: sum p |V| times delta and its own roundings, (r / 16
+ 64) 2^-24.  A weight that is rounded to bf16 first (prompts with bf16 outputs) adds half
a step, 2^-8 of itself; so does a bf16 output.  A mass is the sum of a row's weights over
c columns: the weights' deltas and (c / 32 + 64) 2^-24 of their sum, and 2^-23 of what was
there before and of the result."""
import numpy as np


class Unit:
    """One unit: K, V [rows, d] and mass [rows] of the rows it holds, room for cap."""

    def __init__(self, K, V, mass, cap):
        self.K, self.V, self.mass, self.cap = K, V, np.asarray(mass, np.float64), cap
        self.mass_tol = np.zeros_like(self.mass)

    def attend(self, q, scale, knew=None, vnew=None, decay=1.0, max_rows=None):
        """q [c, G, d] -> (out [c, G, d], its tolerance with fp32 outputs and unrounded weights,
        sum p |V|); the unit's rows and masses become those after the call."""
        c, G, d = q.shape
        out, tol, size = np.zeros((c, G, d)), np.zeros((c, G, d)), np.zeros((c, G, d))
        if c == 0:
            return out, tol, size
        if knew is not None:
            base, room = len(self.K), min(c, self.cap - len(self.K))
            self.K, self.V = np.concatenate((self.K, knew[:room])), np.concatenate((self.V, vnew[:room]))
            self.mass = np.concatenate((self.mass, np.zeros(room)))
            self.mass_tol = np.concatenate((self.mass_tol, np.zeros(room)))
        else:
            base = len(self.K) - c
        top = len(self.K) if max_rows is None else min(len(self.K), max_rows)
        K, V = self.K[:top].astype(np.float64), self.V[:top].astype(np.float64)
        got, got_tol = np.zeros(top), np.zeros(top)
        for i in range(c):
            r = max(min(base + i + 1, top), 0)
            if r == 0:
                continue
            x = q[i].astype(np.float64)
            S = scale * (x @ K[:r].T)
            E = (d + 4) * 2.0 ** -24 * scale * (np.abs(x) @ np.abs(K[:r]).T).max(axis=1, keepdims=True)
            p = np.exp(S - S.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            delta = 2 * E + (r / 32 + 64) * 2.0 ** -24
            out[i], size[i] = p @ V[:r], p @ np.abs(V[:r])
            tol[i] = size[i] * (delta + (r / 16 + 64) * 2.0 ** -24)
            got[:r] += p.sum(axis=0)
            got_tol[:r] += (p * (delta + (c * G / 32 + 64) * 2.0 ** -24)).sum(axis=0)
        new = decay * self.mass[:top] + got
        self.mass_tol[:top] = decay * self.mass_tol[:top] + got_tol + (decay * self.mass[:top] + new) * 2.0 ** -23
        self.mass[:top] = new
        return out, tol, size


def out_tol(want, tol, size, fp32, rounded_weights):
    return tol + (0 if fp32 else np.abs(want) * 2.0 ** -8 * 1.01) + (size * 2.0 ** -8 if rounded_weights and not fp32 else 0)
