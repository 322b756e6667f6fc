"""fp64 definition of bc_block_norm and its gradient, from the formulas."""
import numpy as np


def unit(v, w, eps):
    return v / np.sqrt((v ** 2).mean(-1, keepdims=True) + eps) * w


def stream(x, h, gate, post, post_weight, scale, eps):
    """The new residual stream before it is rounded."""
    u = unit(x, post_weight, eps) if post else x
    return h + scale * gate * u


def unit_grad(v, w, eps, g):
    """Gradients of unit(v, w) for v and, row by row, for w."""
    r = 1.0 / np.sqrt((v ** 2).mean(-1, keepdims=True) + eps)
    return r * w * g - v * r ** 3 * (v * w * g).mean(-1, keepdims=True), g * v * r


def grad(x, h_out, gate, post, post_weight, pre_weight, scale, eps, a, b):
    """dx, dh and, row by row, the gradients of gate, post_weight and pre_weight; h_out is the stream as it was stored."""
    dz, dpre = unit_grad(h_out, pre_weight, eps, b)
    dh = a + dz
    u = unit(x, post_weight, eps) if post else x
    du = scale * gate * dh
    dx, dpost = unit_grad(x, post_weight, eps, du) if post else (du, np.zeros_like(x))
    return dx, dh, scale * dh * u, dpost, dpre
