"""Row operators in fp64: layer norm forward and backward, dropout of rows, RMS
norm forward and backward, the top logits of a row, and the distillation loss
with its gradient.

Test infrastructure only (see the package docstring). Each function is the
textbook definition written out: layer normalisation over the channels of a
row; Hinton's distillation loss with temperature T (soft targets weighted by
T^2) restricted to the teacher's listed classes, mixed with the labels'
cross-entropy.
"""
import numpy as np

from oracle import philox


def layernorm_forward(x, gamma, beta, eps):
    """(y, mean, rstd) of rows x [R][D]; gamma, beta [D] or None."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean, rstd


def layernorm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) from the forward pass's input and statistics."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    xh = (x - mean) * rstd
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = rstd * (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True))
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


def dropout_factor(seed, step, rows, width, p):
    """The factor keep / (1 - p) of every element of rows x width: element j of
    row r draws word j mod 4 of the counter (r ceil(width / 4) + j div 4)."""
    padded = (width + 3) // 4 * 4
    keep = philox.dropout_keep(seed, step, rows, padded, p)[:, :width]
    return keep * philox.dropout_params(p)[1]


def rmsnorm_forward(h, gamma, eps):
    """(y, rstd) of rows h [R][D]; gamma [D] or None."""
    h = np.asarray(h, np.float64)
    rstd = 1.0 / np.sqrt((h ** 2).mean(axis=1) + eps)
    y = h * rstd[:, None]
    return (y if gamma is None else y * np.asarray(gamma, np.float64)), rstd


def rmsnorm_backward(dy, dr, h, gamma, rstd):
    """(dh, dgamma) from the forward pass's rows and statistic; dr: what else
    the rows' gradient receives, or None."""
    dy, h, rstd = (np.asarray(a, np.float64) for a in (dy, h, rstd))
    xh = h * rstd[:, None]
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dh = rstd[:, None] * (g - xh * (g * xh).mean(axis=1, keepdims=True))
    return (dh if dr is None else dh + np.asarray(dr, np.float64)), (dy * xh).sum(axis=0)


def topk(z, k):
    """(values, classes) of the k largest entries of every row, in descending
    order, equal values in the order of their classes, NaN above everything."""
    z = np.asarray(z, np.float64)
    vals, idx = np.empty((len(z), k)), np.empty((len(z), k), np.int64)
    for r, row in enumerate(z):
        order = sorted(range(len(row)), key=lambda c: (0, 0.0, c) if np.isnan(row[c]) else (1, -row[c], c))[:k]
        idx[r], vals[r] = order, row[order]
    return vals, idx


def _log_softmax(v):
    m = v.max()
    return v - m - np.log(np.exp(v - m).sum())


def distill(z, t_vals, t_idx, labels, weight, temperature, alpha, scale):
    """(row_loss, loss, dz): one row at a time, the teacher's list as it is
    written (duplicates add up; entries with a class outside [0, C) or the
    value -inf are left out). labels, weight may be None."""
    z = np.asarray(z, np.float64)
    R, C = z.shape
    row_loss, dz = np.zeros(R), np.zeros((R, C))
    for r in range(R):
        w = 1.0 if weight is None else float(weight[r])
        if w == 0.0 or np.all(z[r] == -np.inf):
            continue
        entries = [(int(i), float(t)) for t, i in zip(t_vals[r], t_idx[r]) if 0 <= i < C and t != -np.inf]
        loss, g = 0.0, np.zeros(C)
        if entries and alpha != 0.0:
            lq = _log_softmax(np.array([t for _, t in entries]) / temperature)
            lp = _log_softmax(z[r] / temperature)
            g += alpha * temperature * np.exp(lp)
            for (i, _), l in zip(entries, lq):
                q = np.exp(l)
                if q != 0.0:
                    loss += alpha * temperature ** 2 * q * (l - lp[i])
                g[i] -= alpha * temperature * q
        if labels is not None and alpha != 1.0 and 0 <= labels[r] < C:
            lp = _log_softmax(z[r])
            loss -= (1.0 - alpha) * lp[labels[r]]
            g += (1.0 - alpha) * np.exp(lp)
            g[labels[r]] -= 1.0 - alpha
        row_loss[r], dz[r] = w * loss, scale * w * g
    return row_loss, scale * row_loss.sum(), dz
