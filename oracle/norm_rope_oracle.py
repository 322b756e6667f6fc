"""Norm of query and key heads followed by the rotation, and its gradient, fp64 (TEST INFRASTRUCTURE ONLY).

    y = x / sqrt(mean(x^2) + eps) * w,   out = R(pos) y      (R: the half-split rotation of rope_oracle.py)

Gradient with g = d loss / d out, r = 1 / sqrt(mean(x^2) + eps):  dy = R(pos)^T g,
dx = r (w dy - x r^2 mean(x w dy)),  dw = sum x r dy.
Pinned by tests/test_norm_rope_oracle_pins.py (definition by hand, differences of the forward).
"""
import numpy as np

from oracle.rope_oracle import rope


def norm(x, w, eps):
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(w, dtype=np.float64)


def heads(qkv, q_heads, kv_heads, head_dim):
    x = np.asarray(qkv, dtype=np.float64).reshape(len(qkv), q_heads + 2 * kv_heads, head_dim)
    return x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]


def norm_rope_split(qkv, pos, q_heads, kv_heads, head_dim, theta, q_weight, k_weight, eps):
    q, k, v = heads(qkv, q_heads, kv_heads, head_dim)
    p = np.asarray(pos, dtype=np.float64)[:, None]
    return rope(norm(q, q_weight, eps), p, theta), rope(norm(k, k_weight, eps), p, theta), v


def grad(x, w, eps, pos, theta, g):
    """Of one kind of heads: x, g [n, heads, D] -> (dx, dw, size of the terms of dx, size of the terms of dw)."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    dy = rope(g, -np.asarray(pos, dtype=np.float64)[:, None], theta)
    r = 1 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    a = w * dy
    dx = r * (a - x * r * r * np.mean(x * a, axis=-1, keepdims=True))
    mag = r * (np.abs(a) + np.abs(x) * r * r * np.mean(np.abs(x * a), axis=-1, keepdims=True))
    return dx, (x * r * dy).sum(axis=(0, 1)), mag, np.abs(x * r * dy).sum(axis=(0, 1))
