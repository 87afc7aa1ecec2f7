"""Operators of a training step around the draft layer's kernels, from their definitions, in 64 bits (numpy)."""
import math

import numpy as np

from .layer8 import rotary


def embed(table, tok, scale=1.0):
    table, tok = np.asarray(table, np.float64), np.asarray(tok)
    real = (tok >= 0) & (tok < table.shape[0])
    out = np.zeros((len(tok), table.shape[1]))
    out[real] = table[tok[real]] * scale
    return out


def embed_grad(dy, tok, vocab, scale=1.0):
    dy, tok = np.asarray(dy, np.float64), np.asarray(tok)
    real = (tok >= 0) & (tok < vocab)
    out = np.zeros((vocab, dy.shape[1]))
    np.add.at(out, tok[real], dy[real])
    return out * scale


def headnorm(x, w, eps, offset=0.0):
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (offset + np.asarray(w, np.float64))


def headnorm_rotary(x, w, eps, offset, pos, freq, mscale, rot, layout):
    return rotary(headnorm(x, w, eps, offset), pos, freq, mscale, rot, layout)


def headnorm_rotary_grad(dy, x, w, eps, offset, pos, freq, mscale, rot, layout):
    """(gradient of x, gradient of w)"""
    x, w = np.asarray(x, np.float64), offset + np.asarray(w, np.float64)
    dz = rotary(dy, pos, freq, mscale, rot, layout, adjoint=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return r * (w * dz - x * r * r * (w * dz * x).mean(-1, keepdims=True)), (dz * x * r).sum((0, 1))


def activation(act, g):
    """act(g) and its slope."""
    g = np.asarray(g, np.float64)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if act == "gelu":
        p = 0.5 * np.vectorize(math.erfc)(-g * math.sqrt(0.5))
        return g * p, p + g * np.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = np.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def ffn_gated(x, w_gate, w_up, act):
    x, w_gate, w_up = (np.asarray(t, np.float64) for t in (x, w_gate, w_up))
    return activation(act, x @ w_gate.T)[0] * (x @ w_up.T)


def ffn_gated_grad(x, w_gate, w_up, dh, act):
    """(dx, dw_gate, dw_up)"""
    x, w_gate, w_up, dh = (np.asarray(t, np.float64) for t in (x, w_gate, w_up, dh))
    a, slope = activation(act, x @ w_gate.T)
    dg, du = dh * (x @ w_up.T) * slope, dh * a
    return dg @ w_gate + du @ w_up, dg.T @ x, du.T @ x


def grad_clip(grads, max_norm):
    """(norm, the gradients scaled)"""
    grads = [np.asarray(g, np.float64) for g in grads]
    norm = math.sqrt(math.fsum(float((g * g).sum()) for g in grads))
    return norm, [g * min(1.0, max_norm / (norm + 1e-6)) for g in grads]
