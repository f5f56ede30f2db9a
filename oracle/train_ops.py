"""The operators around the chunks of a training iteration as their definitions, in numpy float64: embedding with a scale,
the residual join (post-norm, gate, residual scales, pre-norm), the gradient norm and its clipping factor.  The paper prints
none of them; they are the standard ones."""

import numpy as np


def embedding_forward(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < len(table):
            out[t] = scale * table[v]
    return out


def embedding_backward(tokens, dout, scale, vocab):
    """(d_table, for each entry the sum of the absolute values of what was added, how many rows each token has)."""
    d, size, n = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros(vocab, dtype=int)
    for t, v in enumerate(tokens):
        if 0 <= v < vocab:
            d[v] += dout[t]
            size[v] += np.abs(dout[t])
            n[v] += 1
    return scale * d, abs(scale) * size, n


def moments(v, kind, eps):
    if kind == "none":
        return np.zeros((len(v), 1)), np.ones((len(v), 1))
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((len(v), 1))
    return mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)


def affine(vhat, w, kind):
    H = vhat.shape[1]
    return vhat if kind == "none" else vhat * w[:H] + w[H:] if kind == "layer" else vhat * w


def residual_forward(x, branch, gate, post, pre, kinds, x_scale, branch_scale, eps):
    """(x_out, h or None, stats [rows][4])."""
    m1, r1 = moments(branch, kinds[0], eps)
    u = affine((branch - m1) * r1, post, kinds[0])
    x_out = x_scale * x + branch_scale * (u if gate is None else gate * u)
    m2, r2 = moments(x_out, kinds[1], eps)
    h = affine((x_out - m2) * r2, pre, kinds[1]) if kinds[1] != "none" else None
    return x_out, h, np.concatenate([m1, r1, m2, r2], 1)


def _norm_backward(dout, vhat, rstd, w, kind):
    if kind == "none":
        return dout, None
    a = dout * w[:vhat.shape[1]]
    d = a - vhat * (a * vhat).mean(1, keepdims=True)
    sums = [(dout * vhat).sum(0)]
    if kind == "layer":
        d = d - a.mean(1, keepdims=True)
        sums.append(dout.sum(0))
    return rstd * d, np.concatenate(sums)


def residual_backward(x_out, branch, gate, post, pre, stats, dh, dx_out, kinds, x_scale, branch_scale):
    """(dx, dbranch, dgate, d_post, d_pre); None for what there is not."""
    m1, r1, m2, r2 = (stats[:, i:i + 1] for i in range(4))
    d = np.zeros_like(branch) if dx_out is None else dx_out
    d_pre = None
    if kinds[1] != "none":
        dx, d_pre = _norm_backward(dh, (x_out - m2) * r2, r2, pre, kinds[1])
        d = d + dx
    fhat = (branch - m1) * r1
    q = branch_scale * d
    dgate = None
    if gate is not None:
        dgate = q * affine(fhat, post, kinds[0])
        if gate.ndim == 1:
            dgate = dgate.sum(0)
        q = q * gate
    dbranch, d_post = _norm_backward(q, fhat, r1, post, kinds[0])
    return x_scale * d, dbranch, dgate, d_post, d_pre


def grad_norm(grads):
    return float(np.sqrt(sum(float(np.dot(g.ravel(), g.ravel())) for g in grads)))


def clip_scale(norm, max_norm):
    """1 for a norm that is not finite: the gradients are left as they are."""
    return max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
