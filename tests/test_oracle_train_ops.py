"""The oracle of the operators around the chunks against differences, autograd and hand-worked cases (no GPU)."""

import itertools

import numpy as np
import pytest
import torch

from oracle import train_ops as OT

KINDS = ("none", "layer", "rms")


def join_case(rng, rows, H, kinds, gate):
    w = lambda k: None if k == "none" else 1 + 0.3 * rng.normal(size=2 * H if k == "layer" else H)
    g = {"none": None, "channel": rng.normal(size=H), "element": rng.normal(size=(rows, H))}[gate]
    return dict(x=rng.normal(size=(rows, H)), branch=rng.normal(size=(rows, H)) + 0.5, gate=g, post=w(kinds[0]), pre=w(kinds[1]))


@pytest.mark.parametrize("post,pre,gate", list(itertools.product(KINDS, KINDS, ("none", "channel", "element"))))
def test_residual_gradients_against_differences(post, pre, gate):
    rng = np.random.default_rng(5)
    rows, H, kinds, xs, bs, eps = 3, 8, (post, pre), 0.75, 0.5, 1e-3
    c = join_case(rng, rows, H, kinds, gate)
    dxo, dh = rng.normal(size=(rows, H)), rng.normal(size=(rows, H))

    def loss(**kw):
        a = dict(c, **kw)
        x_out, h, _ = OT.residual_forward(a["x"], a["branch"], a["gate"], a["post"], a["pre"], kinds, xs, bs, eps)
        return (x_out * dxo).sum() + (0 if h is None else (h * dh).sum())

    x_out, h, stats = OT.residual_forward(c["x"], c["branch"], c["gate"], c["post"], c["pre"], kinds, xs, bs, eps)
    got = OT.residual_backward(x_out, c["branch"], c["gate"], c["post"], c["pre"], stats, dh if h is not None else None, dxo,
                               kinds, xs, bs)
    for name, g in zip(("x", "branch", "gate", "post", "pre"), got):
        assert (g is None) == (c[name] is None)
        if g is None:
            continue
        base = c[name]
        for i in np.ndindex(base.shape):
            e = np.zeros_like(base)
            e[i] = 1e-5
            want = (loss(**{name: base + e}) - loss(**{name: base - e})) / 2e-5
            assert abs(g[i] - want) <= 1e-6 * max(1.0, abs(want)), (name, i)


def test_norms_are_torch_norms():
    rng = np.random.default_rng(1)
    v, w = rng.normal(size=(5, 16)), rng.normal(size=32)
    m, r = OT.moments(v, "layer", 1e-5)
    want = torch.nn.functional.layer_norm(torch.from_numpy(v), (16,), torch.from_numpy(w[:16]), torch.from_numpy(w[16:]), 1e-5)
    assert np.allclose(OT.affine((v - m) * r, w, "layer"), want.numpy(), atol=1e-12)
    m, r = OT.moments(v, "rms", 1e-5)
    want = torch.nn.functional.rms_norm(torch.from_numpy(v), (16,), torch.from_numpy(w[:16]), 1e-5)
    assert np.allclose(OT.affine((v - m) * r, w[:16], "rms"), want.numpy(), atol=1e-12)


def test_embedding_is_torch_embedding():
    rng = np.random.default_rng(2)
    table, tok = rng.normal(size=(7, 8)), np.array([3, 0, 3, 6, -1, 7, 3])
    t = torch.from_numpy(table).requires_grad_()
    known = (tok >= 0) & (tok < 7)
    out = 2.5 * torch.nn.functional.embedding(torch.from_numpy(tok[known]), t)
    got = OT.embedding_forward(table, tok, 2.5)
    assert np.allclose(got[known], out.detach().numpy()) and not got[~known].any()
    dout = rng.normal(size=(7, 8))
    out.backward(torch.from_numpy(dout[known]))
    d, size, n = OT.embedding_backward(tok, dout, 2.5, 7)
    assert np.allclose(d, t.grad.numpy()) and list(n) == [1, 0, 0, 3, 0, 0, 1] and (size >= np.abs(d) - 1e-12).all()


def test_clipping_is_torch_clipping():
    rng = np.random.default_rng(3)
    gs = [rng.normal(size=n) for n in (1, 17, 300)]
    ps = [torch.nn.Parameter(torch.zeros(g.size, dtype=torch.float64)) for g in gs]
    for p, g in zip(ps, gs):
        p.grad = torch.from_numpy(g.copy())
    want = torch.nn.utils.clip_grad_norm_(ps, 2.0)
    norm = OT.grad_norm(gs)
    assert abs(norm - float(want)) <= 1e-12 * norm
    k = OT.clip_scale(norm, 2.0)
    for p, g in zip(ps, gs):
        assert np.allclose(p.grad.numpy(), k * g, rtol=1e-6)   # torch adds 1e-6 to the norm
    assert OT.clip_scale(1.0, 2.0) == 1.0 and OT.clip_scale(np.inf, 2.0) == 1.0 and OT.clip_scale(np.nan, 2.0) == 1.0
