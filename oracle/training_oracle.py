"""The operators around a network's layers in plain numpy, 64 bits throughout: layer
norm, lookup of learned rows, distillation from a teacher's top logits, each with
its gradient, row by row as their formulas have it."""
from __future__ import annotations

import numpy as np


def norm_stats(x, eps):
    """(rows, 2): each row's mean, and 1 / sqrt(variance + eps)."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    return np.stack([mean, 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)], 1)


def norm(x, weight=None, bias=None, eps=1e-5, relu=False):
    x = np.asarray(x, np.float64)
    mean, r = norm_stats(x, eps).T[:, :, None]
    z = (x - mean) * r
    if weight is not None:
        z = z * np.asarray(weight, np.float64)
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    return np.where(z <= 0, 0.0, z) if relu else z


def norm_backward(dz, x, stats, weight=None, zero=None):
    """(dx, dw, db) of z = (x - mean) r weight + bias, the mean and r of stats being
    x's own; zero: where x, a ReLU's output, is zero, and dx is then 0."""
    dz, x, stats = (np.asarray(v, np.float64) for v in (dz, x, stats))
    mean, r = stats[:, :1], stats[:, 1:]
    xh = (x - mean) * r
    g = dz if weight is None else dz * np.asarray(weight, np.float64)
    dx = r * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx if zero is None else np.where(zero, 0.0, dx), (dz * xh).sum(0), dz.sum(0)


def lookup(table, ids, scale=1.0):
    table = np.asarray(table, np.float64)
    y = np.zeros((len(ids), table.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < len(table):
            y[i] = scale * table[v]
    return y


def lookup_grad(dy, ids, n, scale=1.0):
    dy = np.asarray(dy, np.float64)
    dt = np.zeros((n, dy.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < n:
            dt[v] += dy[i]
    return scale * dt


def distill(x, classes, teacher, temperature=1.0, row_weight=None):
    """(loss (rows), dx) of each row's own weight."""
    x, teacher = np.asarray(x, np.float64), np.asarray(teacher, np.float64)
    loss, dx = np.zeros(len(x)), np.zeros(x.shape)
    for i in range(len(x)):
        w = 1.0 if row_weight is None else float(row_weight[i])
        given = (classes[i] >= 0) & (classes[i] < x.shape[1])
        c, t = classes[i][given], teacher[i][given]
        if w == 0 or not (t > -np.inf).any() | np.isnan(t).any() or not (x[i] > -np.inf).any() | np.isnan(x[i]).any():
            continue
        with np.errstate(divide="ignore", invalid="ignore"):
            p = np.exp((t - t.max()) / temperature)
            log_p = (t - t.max()) / temperature - np.log(p.sum())
            p = p / p.sum()
            q = np.exp((x[i] - x[i].max()) / temperature)
            log_q = (x[i] - x[i].max()) / temperature - np.log(q.sum())
            q = q / q.sum()
            terms = np.where(p == 0, 0.0, p * (log_p - log_q[c]))
        loss[i] = w * temperature ** 2 * terms.sum()
        grad = q.copy()
        np.add.at(grad, c, -p)
        dx[i] = w * temperature * grad
    return loss, dx
