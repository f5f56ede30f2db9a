"""The operators around the chunks (embedding with a scale, residual join, gradient norm and clipping) against their
definitions in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32, `half(t)` half a step of the storage type (bf16 2^-8), both relative to the value.  A stored
result is off by at most half(t) |value| plus what the fp32 arithmetic before it is off: a sum of n terms in any order by at
most (n - 1) u times the sum of their absolute values, a product by u.  The row sums here run over chains of at most
H / 64 + 6 + H / 512 additions; K = 256 steps cover the longest of them (H = 4096: 78) together with the few products, the division, the
square root (2 u) and the deviations from the mean that lead to a result.  K u multiplies the size of the terms that
are added, not of their sum, so that cancelling terms are allowed for; (1 + |mean| / deviation) is the condition of a centred value."""

import itertools

import numpy as np
import pytest
import torch

from oracle import train_ops as OT
from oracle import ends as OE
from paper_2308_15762_amd import hanayo as hn
from helpers import dev, host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
K = 256
DT = {"fp32": hn.FP32, "bf16": hn.BF16}
TD = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": U, "bf16": 2.0 ** -8}
EPS = float(np.float32(1e-5))


def values(rng, shape, dtype, std=1.0, mean=0.0):
    """Values that the type holds exactly, on the GPU and in 64 bits."""
    t = torch.from_numpy((mean + std * rng.normal(size=shape)).astype(np.float32)).to(TD[dtype])
    return t.cuda(), t.double().numpy()


def near(got, want, bound, what):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    bad = np.abs(got - want) > bound
    assert np.isfinite(got).all() and not bad.any(), "%s: %d of %d off, worst by %.3g of the bound, first at %s" % (
        what, bad.sum(), bad.size, float((np.abs(got - want) / np.maximum(bound, 1e-300)).max()), np.argwhere(bad)[:1])


def room(n):
    return torch.full((max(1, int(n)),), 0xA5, dtype=torch.uint8, device="cuda")   # nothing has to be cleared


# ------------------------------------------------------------------ embedding

def tokens_of(kind, rng, rows, vocab):
    if kind == "one":
        return np.full(rows, min(5, vocab - 1))
    if kind == "distinct":
        return rng.permutation(max(rows, vocab))[:rows] % vocab
    if kind == "none":
        return np.where(np.arange(rows) % 2, -1, vocab)
    p = 1.0 / np.arange(1, vocab + 1)
    tok = rng.choice(vocab, size=rows, p=p / p.sum())
    if kind == "padded":                        # the last third of the positions holds no token, of all kinds
        tok[2 * rows // 3:] = rng.choice([-1, vocab, np.iinfo(np.int32).min, np.iinfo(np.int32).max], size=rows - 2 * rows // 3)
    return tok


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,H,vocab", [(1, 8, 1), (5, 520, 37), (64, 64, 512), (257, 1024, 300), (4097, 72, 50304)])
def test_embedding_forward(dtype, rows, H, vocab):
    rng = np.random.default_rng(rows + H)
    table, t64 = values(rng, (vocab, H), dtype)
    tok = tokens_of("padded", rng, rows, vocab)
    out = torch.full((rows + 1, H), 7.0, dtype=TD[dtype], device="cuda")
    hn.hanayo_op_embedding_forward(DT[dtype], table, torch.from_numpy(tok.astype(np.int32)).cuda(), 31.75, out, rows, H, vocab)
    want = OT.embedding_forward(t64, tok, 31.75)
    near(out[:rows], want, np.abs(want) * (HALF[dtype] + U), "out")
    assert (out[rows] == 7.0).all()             # the row behind the last one


def embedding_backward(dtype, tok, dout, scale, base, rows, H, vocab, accumulate, work=None):
    d = torch.from_numpy(base.astype(np.float32)).cuda()
    work = room(hn.hanayo_op_embedding_workspace_bytes(rows, H, vocab)) if work is None else work
    hn.hanayo_op_embedding_backward(DT[dtype], torch.from_numpy(tok.astype(np.int32)).cuda(), dout, scale, d, rows, H, vocab,
                                    accumulate, work)
    return d


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["one", "distinct", "none", "zipf", "padded"])
@pytest.mark.parametrize("rows,H,vocab", [(1, 8, 1), (2, 16, 3), (63, 520, 37), (64, 8, 512), (65, 1032, 4), (1000, 136, 90),
                                          (4097, 64, 3001), (9000, 24, 30000), (20011, 16, 700), (70001, 8, 1000)])
def test_embedding_backward(dtype, kind, rows, H, vocab):
    rng = np.random.default_rng(rows * 7 + H)
    tok = tokens_of(kind, rng, rows, vocab)
    dout, d64 = values(rng, (rows, H), dtype)
    known = (tok >= 0) & (tok < vocab)
    dout[torch.from_numpy(~known).cuda()] = float("nan")      # what stands behind no token reaches nothing
    want, size, n = OT.embedding_backward(tok, np.where(known[:, None], d64, 0), 1.5, vocab)
    base = rng.normal(size=(vocab, H)).astype(np.float32)
    # n rows of a token: n - 1 additions, the scale, the addition to what is there
    bound = lambda b: (n[:, None] + 2) * U * (size + np.abs(b))
    add = embedding_backward(dtype, tok, dout, 1.5, base, rows, H, vocab, True)
    near(add, base + want, bound(base), "added")
    assert torch.equal(add[torch.from_numpy(n == 0).cuda()], torch.from_numpy(base[n == 0]).cuda())
    first = embedding_backward(dtype, tok, dout, 1.5, np.full_like(base, np.nan), rows, H, vocab, False)
    near(first, want, bound(0), "written")
    assert torch.equal(first, embedding_backward(dtype, tok, dout, 1.5, base, rows, H, vocab, False))     # bit for bit


# (rows, columns, vocabulary) on both sides of every choice: one launch up to 1024 rows and 8192 tokens times slabs of 512
# columns; comparison of all pairs up to 12288 rows; one, two and three digits of the radix sort; pieces of 8 to 64 rows
BORDERS = [(1024, 512, 8192), (1024, 520, 4097), (1025, 8, 10), (12288, 8, 99), (12289, 8, 99), (12289, 8, 511), (12300, 8, 512),
           (13000, 8, 262143), (13001, 8, 300000), (40000, 1040, 50), (70000, 2056, 40), (150001, 1024, 600)]


@pytest.mark.parametrize("kind", ["half", "zipf"])
@pytest.mark.parametrize("rows,H,vocab", BORDERS)
def test_embedding_backward_at_the_borders_of_its_variants(kind, rows, H, vocab):
    """Also a batch of which half is one token (padding by a token of the vocabulary), and what lies behind the workspace."""
    rng = np.random.default_rng(rows + vocab)
    tok = tokens_of("zipf", rng, rows, vocab)
    if kind == "half":
        tok[rng.permutation(rows)[:rows // 2]] = vocab // 2
    dout = torch.randint(-8, 9, (rows, H), device="cuda").to(torch.bfloat16)      # whole numbers: every sum is exact
    t = torch.from_numpy(tok).cuda()
    want = torch.zeros((vocab, H), dtype=torch.float64, device="cuda").index_add_(0, t, dout.double())
    need = hn.hanayo_op_embedding_workspace_bytes(rows, H, vocab)
    work = room(need + 512)
    for accumulate in (True, False):
        d = torch.full((vocab, H), 3.0, device="cuda")
        hn.hanayo_op_embedding_backward(hn.BF16, t.int(), dout, 0.5, d, rows, H, vocab, accumulate, work)
        assert torch.equal(d.double(), 0.5 * want + (3.0 if accumulate else 0.0))
        assert (work[need:] == 0xA5).all()


def test_embedding_without_rows():
    e = torch.empty(0, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    table = torch.ones((4, 8), device="cuda")
    hn.hanayo_op_embedding_forward(hn.FP32, table, t, 1.0, e, 0, 8, 4)
    work = room(hn.hanayo_op_embedding_workspace_bytes(0, 8, 4))
    hn.hanayo_op_embedding_backward(hn.FP32, t, e, 1.0, table, 0, 8, 4, True, work)
    assert (table == 1).all()
    hn.hanayo_op_embedding_backward(hn.FP32, t, e, 1.0, table, 0, 8, 4, False, work)
    assert not table.any()


def test_embedding_table_past_32_bit_offsets():
    """A table of 2^31 elements and more: the last token's row lies beyond what 32-bit offsets reach."""
    vocab, H, rows = 524296, 4096, 70
    table = torch.empty((vocab, H), dtype=torch.bfloat16, device="cuda")
    tok = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    tok[::2] = vocab - 2
    table[vocab - 2:] = 0.5
    table[vocab - 1] = 2.0
    out = torch.empty((rows, H), dtype=torch.bfloat16, device="cuda")
    hn.hanayo_op_embedding_forward(hn.BF16, table, tok, 2.0, out, rows, H, vocab)
    assert (out[::2] == 1.0).all() and (out[1::2] == 4.0).all()
    del table
    d = torch.empty((vocab, H), device="cuda")
    d[vocab - 3:] = 1.0
    hn.hanayo_op_embedding_backward(hn.BF16, tok, out, 1.0, d, rows, H, vocab, True,
                                    room(hn.hanayo_op_embedding_workspace_bytes(rows, H, vocab)))
    assert (d[vocab - 3] == 1.0).all() and (d[vocab - 2] == 36.0).all() and (d[vocab - 1] == 141.0).all()


# ------------------------------------------------------------------ residual join

KINDS = ("none", "layer", "rms")
NORMS = {"none": hn.NORM_NONE, "layer": hn.NORM_LAYER, "rms": hn.NORM_RMS}
GATES = {"none": hn.GATE_NONE, "channel": hn.GATE_CHANNEL, "element": hn.GATE_ELEMENT}


class Join:
    def __init__(self, dtype, rows, H, post, pre, gate, x_scale=0.75, branch_scale=0.5, seed=0, mean=0.25):
        rng = np.random.default_rng(seed + rows * 31 + H)
        self.dtype, self.rows, self.H, self.kinds, self.xs, self.bs = dtype, rows, H, (post, pre), x_scale, branch_scale
        self.desc = hn.ResidualDesc(rows, H, DT[dtype], NORMS[post], NORMS[pre], GATES[gate], x_scale, branch_scale, EPS)
        self.gate_kind = gate
        v = lambda shape, std=1.0, m=0.0: values(rng, shape, dtype, std, m)
        w = lambda k: (None, None) if k == "none" else v(2 * H if k == "layer" else H, 0.2, 1.0)
        self.x, self.x64 = v((rows, H), 2.0, mean)
        self.branch, self.b64 = v((rows, H), 1.0, mean)
        self.gate, self.g64 = {"none": lambda: (None, None), "channel": lambda: v(H), "element": lambda: v((rows, H))}[gate]()
        (self.post, self.post64), (self.pre, self.pre64) = w(post), w(pre)
        self.dh, self.dh64 = v((rows, H)) if pre != "none" else (None, None)
        self.dxo, self.dxo64 = v((rows, H))

    def empty(self):
        return torch.full((self.rows, self.H), float("nan"), dtype=TD[self.dtype], device="cuda")

    def forward(self, x_out=None, stats=True):
        x_out = self.empty() if x_out is None else x_out
        h = self.empty() if self.kinds[1] != "none" else None
        st = torch.full((self.rows, 4), float("nan"), device="cuda") if stats else None
        hn.hanayo_op_residual_forward(self.desc, self.x, self.branch, self.gate, self.post, self.pre, x_out, h, st)
        return x_out, h, st

    def backward(self, x_out, stats, dx_out, accumulate=False, fill=0.0, dx=None, scratch=None):
        z = lambda p: None if p is None else torch.full((p.numel(),), fill, device="cuda")
        d_post, d_pre = z(self.post), z(self.pre)
        dgate = None if self.gate is None else self.empty() if self.gate_kind == "element" else z(self.gate)
        dx, dbranch = self.empty() if dx is None else dx, self.empty()
        scratch = room(hn.hanayo_op_residual_scratch_bytes(self.desc)) if scratch is None else scratch
        hn.hanayo_op_residual_backward(self.desc, x_out, self.branch, self.gate, self.post, self.pre, stats, self.dh, dx_out, dx,
                                       dbranch, dgate, d_post, d_pre, accumulate, scratch)
        return dx, dbranch, dgate, d_post, d_pre


def size_of_norm(v, size, mean, rstd, w, kind):
    """Size of the terms of a normed value: K u times it bounds what fp32 is off; `size` bounds the terms of v."""
    if kind == "none":
        return size
    vhat, H = np.abs(v - mean) * rstd, v.shape[1]
    cond = 1 + np.abs(mean) * rstd + (size.max(1, keepdims=True) * rstd)
    return (vhat + cond) * np.abs(w[:H]) + (np.abs(w[H:]) if kind == "layer" else 0)


def check_forward(j, x_out, h, stats):
    want_x, want_h, want_s = OT.residual_forward(j.x64, j.b64, j.g64, j.post64, j.pre64, j.kinds, j.xs, j.bs, EPS)
    m1, r1, m2, r2 = (want_s[:, i:i + 1] for i in range(4))
    u = size_of_norm(j.b64, np.abs(j.b64), m1, r1, j.post64, j.kinds[0])
    size = np.abs(j.xs * j.x64) + abs(j.bs) * u * (1 if j.g64 is None else np.abs(j.g64))
    near(x_out, want_x, K * U * size + HALF[j.dtype] * np.abs(want_x), "x_out")
    if h is not None:
        near(h, want_h, 2 * K * U * size_of_norm(want_x, size, m2, r2, j.pre64, j.kinds[1]) + HALF[j.dtype] * np.abs(want_h), "h")
    if stats is not None:
        top = lambda a: np.abs(a).max(1)
        for i, (a, s) in enumerate(((j.b64, np.abs(j.b64)), (None, None), (want_x, size), (None, None))):
            if a is not None:
                near(stats[:, i], want_s[:, i], K * U * top(s) + 1e-30, "mean %d" % i)
                r = want_s[:, i + 1]
                near(stats[:, i + 1], r, 2 * K * U * r * (1 + top(s) * r), "rstd %d" % i)


def check_backward(j, x_out, stats, dx_out, got, base=0.0):
    """x_out and stats: what the call was given."""
    xo, st = x_out.double().cpu().numpy(), stats.double().cpu().numpy()
    dxo = None if dx_out is None else j.dxo64
    want = OT.residual_backward(xo, j.b64, j.g64, j.post64, j.pre64, st, j.dh64, dxo, j.kinds, j.xs, j.bs)
    m1, r1, m2, r2 = (st[:, i:i + 1] for i in range(4))
    H, n = j.H, j.rows
    row = lambda a: a.mean(1, keepdims=True)
    a_ = lambda t: 1.0 if t is None else np.abs(t)
    size = np.zeros((n, H)) if dxo is None else np.abs(dxo)
    if j.kinds[1] != "none":
        xh = np.abs(xo - m2) * r2 + np.abs(m2) * r2
        a = np.abs(j.dh64 * j.pre64[:H])
        size = size + r2 * (a + row(a) + xh * row(a * xh))
    fh = np.abs(j.b64 - m1) * r1 + np.abs(m1) * r1
    q = abs(j.bs) * size * a_(j.g64)
    p = 1.0 if j.post64 is None else np.abs(j.post64[:H])
    beta = np.abs(j.post64[H:]) if j.kinds[0] == "layer" else 0.0
    b = q * p
    size_b = b if j.kinds[0] == "none" else r1 * (b + row(b) + fh * row(b * fh))
    half = HALF[j.dtype]
    near(got[0], want[0], 2 * K * U * abs(j.xs) * size + half * np.abs(want[0]), "dx")
    near(got[1], want[1], 4 * K * U * size_b + half * np.abs(want[1]), "dbranch")
    # column sums: n rows of terms that are K steps off each, added with n more
    steps = (4 * K + n) * U
    cols = lambda t: steps * (t.sum(0) + abs(base)) + 2 * U * abs(base)
    if j.g64 is not None:
        size_g = abs(j.bs) * size * (fh * p + beta)
        if j.g64.ndim == 2:
            near(got[2], want[2], 4 * K * U * size_g + half * np.abs(want[2]), "dgate")
        else:
            near(got[2], want[2] + base, cols(size_g), "dgate")
    for g, w, t, kind, what in ((got[3], want[3], (q * fh, q), j.kinds[0], "d_post"),
                                (got[4], want[4], None if j.dh64 is None else (np.abs(j.dh64) * xh, np.abs(j.dh64)), j.kinds[1], "d_pre")):
        assert (g is None) == (w is None)
        if g is not None:
            near(g, w + base, np.concatenate([cols(s) for s in t[:2 if kind == "layer" else 1]]), what)


def run_join(j, with_dx_out=True, accumulate=False):
    x_out, h, st = j.forward()
    check_forward(j, x_out, h, st)
    dx_out = j.dxo if with_dx_out or j.kinds[1] == "none" else None
    base = 3.0 if accumulate else 0.0
    got = j.backward(x_out, st, dx_out, accumulate, base if accumulate else float("nan"))
    check_backward(j, x_out, st, dx_out, got, base)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("post,pre,gate", list(itertools.product(KINDS, KINDS, ("none", "channel", "element"))))
def test_residual_kinds(dtype, post, pre, gate):
    run_join(Join(dtype, 37, 264, post, pre, gate))
    run_join(Join(dtype, 70, 1024, post, pre, gate), with_dx_out=False, accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,H", [(1, 8), (1, 4096), (3, 512), (7, 520), (2, 1016), (130, 1032), (33, 2056), (9, 2560), (11, 3584),
                                    (517, 4096), (300, 1528), (4500, 64), (2100, 1024), (700, 4088), (1100, 2048), (1030, 2560), (600, 2568),
                                    (5, 1280), (5, 1288)])
def test_residual_sizes(dtype, rows, H):
    run_join(Join(dtype, rows, H, "layer", "rms", "channel"))
    run_join(Join(dtype, rows, H, "rms", "layer", "element", seed=1), accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_residual_in_place_and_for_inference(dtype):
    j = Join(dtype, 37, 1032, "layer", "rms", "channel")
    x_out, h, st = j.forward()
    want = j.backward(x_out, st, j.dxo)
    x = j.x.clone()
    j.x = x
    again, h2, none = j.forward(x_out=x, stats=False)          # x_out is x, nothing kept for a backward pass
    assert none is None and torch.equal(again, x_out) and torch.equal(h2, h)
    d = j.dxo.clone()
    got = j.backward(x_out, st, d, dx=d)                        # dx is dx_out
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_residual_rows_without_variance(dtype, kind):
    """Rows of zeros and of one number, whose deviation is that of eps alone, and a large mean on a small deviation."""
    j = Join(dtype, 6, 520, kind, kind, "none", x_scale=1.0, branch_scale=1.0)
    for row, value in ((0, 0.0), (1, 3.0)):
        for t, t64 in ((j.branch, j.b64), (j.x, j.x64)):
            t[row] = value
            t64[row] = value
    run_join(j)


def test_residual_a_bad_row_stays_in_its_row():
    j = Join("bf16", 40, 1032, "layer", "layer", "element")
    x_out, h, st = j.forward()
    good = j.backward(x_out, st, j.dxo)
    j.branch[7] = float("nan")
    j.x[9, 3] = float("inf")
    x2, h2, st2 = j.forward()
    bad = j.backward(x2, st2, j.dxo)
    keep = [r for r in range(40) if r not in (7, 9)]
    for a, b in ((x_out, x2), (h, h2), (st, st2), (good[0], bad[0]), (good[1], bad[1]), (good[2], bad[2])):
        assert torch.equal(a[keep], b[keep])
    assert not torch.isfinite(x2[7].float()).any() and not torch.isfinite(h2[9].float()).any()


def test_residual_without_rows():
    for accumulate, left in ((True, 2.0), (False, 0.0)):
        j = Join("fp32", 0, 64, "layer", "rms", "channel")
        x_out, h, st = j.forward()
        got = j.backward(x_out, st, j.dxo, accumulate, 2.0)
        assert all((t == left).all() for t in got[2:])


def test_residual_past_32_bit_offsets():
    """2^31 elements and more: the last rows come out as they do alone."""
    H, n = 4096, 5
    rows = (1 << 31) // H + n
    j = Join("bf16", n, H, "rms", "layer", "element")
    x_out, h, st = j.forward()
    alone = j.backward(x_out, st, j.dxo)

    def wide(t):
        out = torch.zeros((rows, t.shape[1]), dtype=t.dtype, device="cuda")
        out[-n:] = t
        return out

    big = Join("bf16", 1, H, "rms", "layer", "element")
    big.rows, big.desc.rows = rows, rows
    big.post, big.pre = j.post, j.pre
    big.x, big.branch, big.gate, big.dh = wide(j.x), wide(j.branch), wide(j.gate), wide(j.dh)
    bx, bh, bst = big.forward()
    assert torch.equal(bx[-n:], x_out) and torch.equal(bh[-n:], h) and torch.equal(bst[-n:], st)
    got = big.backward(bx, bst, wide(j.dxo))
    assert all(torch.equal(g[-n:], a) for g, a in zip(got[:3], alone[:3]))


@pytest.mark.parametrize("rows,H", [(1, 8), (37, 264), (3000, 512), (300, 4096)])
@pytest.mark.parametrize("pre", ["none", "rms"])
def test_residual_scratch_is_as_large_as_it_says(rows, H, pre):
    j = Join("fp32", rows, H, "layer", pre, "channel")
    x_out, h, st = j.forward()
    need = hn.hanayo_op_residual_scratch_bytes(j.desc)
    scratch = room(need + 512)
    j.backward(x_out, st, j.dxo, scratch=scratch)
    assert (scratch[need:] == 0xA5).all()


def test_residual_repeats_bit_for_bit():
    j = Join("bf16", 2100, 1024, "layer", "layer", "channel")
    x_out, h, st = j.forward()
    a, b = j.backward(x_out, st, j.dxo), j.backward(x_out, st, j.dxo)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


# ------------------------------------------------------------------ gradient norm and clipping

def tensors(rng, counts, dtype, std=1.0, shift=0):
    """Tensors one behind another, `shift` elements off the start of their buffer."""
    out, want = [], []
    kinds = [dtype if dtype != "mixed" else ("fp32", "bf16")[i % 2] for i in range(len(counts))]
    flat = {k: values(rng, sum(c for c, d in zip(counts, kinds) if d == k) + shift, k, std) for k in TD}
    at = {k: shift for k in TD}
    for c, k in zip(counts, kinds):
        out.append(flat[k][0][at[k]:at[k] + c])
        want.append(flat[k][1][at[k]:at[k] + c])
        at[k] += c
    return out, want


def sumsq_of(grads, outs=None):
    lst = hn.grad_list(grads, outs)
    s = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda")
    hn.hanayo_op_grad_sumsq(lst, s, room(hn.hanayo_op_grad_workspace_bytes(len(grads))))
    return lst, s


def check_clip(grads, want, max_norm, norm64, outs=None):
    lst, s = sumsq_of(grads, outs)
    got = torch.full((1,), float("nan"), device="cuda")
    hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, max_norm, got))
    # n squares in 64 bits: n 2^-53, below fp32's last step for the sizes here; then one rounding
    assert abs(float(got) - norm64) <= 1.01 * U * norm64
    k = OT.clip_scale(norm64, max_norm)
    for g, w in zip(grads if outs is None else outs, want):
        half = HALF["bf16" if g.dtype == torch.bfloat16 else "fp32"]
        if g.numel():
            near(g, k * w, np.abs(k * w) * (half + 3 * U), "clipped")   # the factor, the product, the rounding


SHAPES = [[1], [0, 3, 0, 5], [8191, 8192, 8193], [1 + 7 * i for i in range(230)], [100003], [4, 8, 12, 65536 * 3 + 1, 2], [0, 0]]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 5])
@pytest.mark.parametrize("counts", SHAPES, ids=["%d_of_%d" % (len(c), sum(c)) for c in SHAPES])
def test_norm_and_clipping(dtype, shift, counts):
    rng = np.random.default_rng(len(counts) + shift)
    grads, want = tensors(rng, counts, dtype, 0.5, shift)
    norm = OT.grad_norm(want)
    before = [g.clone() for g in grads]
    outs = [torch.empty_like(g) for g in grads]
    check_clip(grads, want, 0.37 * norm, norm, outs)              # into other tensors
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    check_clip(grads, want, 1.5 * norm, norm, outs)               # nothing to scale: a copy
    assert all(torch.equal(a, b) for a, b in zip(outs, before))
    check_clip(grads, want, float("inf"), norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    check_clip(grads, want, 0.37 * norm, norm)                    # in place
    _, s = sumsq_of(grads)
    if norm:
        assert abs(float(s) ** 0.5 - 0.37 * norm) <= 0.37 * norm * (HALF["bf16"] if dtype != "fp32" else 4 * U)


def test_clipping_leaves_the_neighbours_alone():
    flat = torch.ones(5000, device="cuda")
    views = [flat[1:4], flat[7:8], flat[1001:3003], flat[4990:4999]]
    lst, s = sumsq_of(views)
    assert float(s) == sum(v.numel() for v in views)
    hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, 0.0))          # a limit of zero clears them
    for v in views:
        assert not v.any()
    assert float(flat.sum()) == 5000 - sum(v.numel() for v in views)


def test_tensors_that_share_memory_are_not_clipped():
    flat = torch.ones(100, device="cuda")
    other = torch.zeros(100, device="cuda")
    for grads, outs, fine in (([flat[:60], flat[59:]], None, False), ([flat, flat], None, False), ([flat[:50], flat[50:]], None, True),
                              ([flat, flat], [other, other], False), ([flat[:60], flat[40:]], [other[:60], other[60:]], True),
                              ([flat[:0], flat[:50], flat[10:10]], None, True)):
        if outs is not None:
            grads = [g[:o.numel()] for g, o in zip(grads, outs)]
        lst, s = sumsq_of(grads, outs)
        assert float(s) == sum(g.numel() for g in grads)          # the norm counts what the list holds
        if fine:
            hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, 1e9))
        else:
            with pytest.raises(hn.HanayoError) as ei:
                hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, 1e9))
            assert ei.value.code == hn.EINVAL
    assert (flat == 1).all()


@pytest.mark.parametrize("size", [1e30, 3e38, 1e-30, 1e-44])
def test_norm_of_very_large_and_very_small_gradients(size):
    g = torch.full((3000,), size, device="cuda")
    w = g.double().cpu().numpy()
    norm = OT.grad_norm([w])
    _, s = sumsq_of([g])
    assert abs(float(s) - norm ** 2) <= 1e-12 * norm ** 2
    out = torch.empty_like(g)
    lst, s = sumsq_of([g], [out])
    with np.errstate(over="ignore"):
        limit = float(np.float32(norm / 4))      # as the call takes it: infinite for the largest gradients, whose norm is 1.6e40
    hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, limit))
    want = OT.clip_scale(norm, limit) * w
    near(out, want, np.abs(want) * 4 * U + 2.0 ** -149, "clipped")     # 2^-149: the smallest step of fp32


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_shows_and_changes_nothing(bad):
    g = [torch.ones(9001, device="cuda"), torch.ones(77, dtype=torch.bfloat16, device="cuda")]
    g[0][8999] = bad
    before = [t.clone() for t in g]
    lst, s = sumsq_of(g)
    n = torch.zeros(1, device="cuda")
    hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, 0.5, n))
    assert not np.isfinite(float(n))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, before))
    p, m, v = (torch.full((16,), x, device="cuda") for x in (1.0, 2.0, 3.0))
    gr = torch.ones(16, device="cuda")
    for zero in (0, 1):
        n.zero_()
        hn.hanayo_adam_step_clipped(hn.Adam(0.1, 0.9, 0.999, 1e-8, 0.1, 1, zero), hn.make_clip(s, 1, 0.5, n), hn.FP32, p, None, gr, m, v, 16)
        assert (p == 1).all() and (m == 2).all() and (v == 3).all() and (gr == 1 - zero).all() and not np.isfinite(float(n))


def test_norm_past_32_bit_offsets():
    g = torch.zeros((1 << 31) + 77, device="cuda")
    g[-3:] = torch.tensor([1.0, -2.0, 4.0])
    g[5] = 8.0
    lst, s = sumsq_of([g[3:], g[:3]])
    assert float(s) == 85.0
    hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, float(np.float32(85.0 ** 0.5 / 2))))
    near(g[-3:], np.array([0.5, -1.0, 2.0]), 4 * U * np.array([1.0, 2.0, 4.0]), "clipped")
    assert int(torch.count_nonzero(g)) == 4


@pytest.mark.parametrize("n", [0, 1, 100, 101, 350])
def test_norm_workspace_is_as_large_as_it_says(n):
    grads = [torch.ones(40000 + i, device="cuda") for i in range(n)]
    need = hn.hanayo_op_grad_workspace_bytes(n)
    work = room(need + 512)
    s = torch.zeros(1, dtype=torch.float64, device="cuda")
    hn.hanayo_op_grad_sumsq(hn.grad_list(grads), s, work)
    assert float(s) == sum(g.numel() for g in grads) and (work[need:] == 0xA5).all()


def test_norm_of_several_ranks():
    rng = np.random.default_rng(4)
    grads, want = tensors(rng, [1000, 77, 5], "fp32")
    parts = torch.cat([sumsq_of([g])[1] for g in grads])
    norm, n = OT.grad_norm(want), torch.zeros(1, device="cuda")
    outs = [torch.empty_like(g) for g in grads]
    hn.hanayo_op_grad_clip(hn.grad_list(grads, outs), hn.make_clip(parts, 3, 1.0, n))
    assert abs(float(n) - norm) <= 1.01 * U * norm
    for o, w in zip(outs, want):
        near(o, w / norm, np.abs(w / norm) * 4 * U, "clipped")


def test_norm_repeats_bit_for_bit():
    grads, _ = tensors(np.random.default_rng(6), [3000001, 17, 50000], "mixed")
    assert len({float(sumsq_of(grads)[1]) for _ in range(3)}) == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [4, 1028, 2500000])
@pytest.mark.parametrize("share", [0.25, 2.0])
def test_clipped_adam(dtype, n, share):
    """Against the oracle's Adam on the scaled gradients.  Hyper-parameters that fp32 holds exactly; the update is a quotient of
    sums of two positive terms: 16 steps of fp32 cover it."""
    rng = np.random.default_rng(n)
    g, g64 = values(rng, n, "fp32", 0.3)
    m, m64 = values(rng, n, "fp32", 0.1)
    v, v64 = values(rng, n, "fp32", 0.1)
    v, v64 = v.abs(), np.abs(v64)
    p, p64 = values(rng, n, "fp32", 0.02)
    store = p.to(TD[dtype])
    norm = OT.grad_norm([g64])
    clip_at = float(np.float32(share * norm))
    lst, s = sumsq_of([g])
    adam = hn.Adam(2.0 ** -10, 0.875, 0.9375, 1e-8, 0.125, 3, 1)
    norm_out = torch.zeros(1, device="cuda")
    params = store if dtype == "bf16" else p
    hn.hanayo_adam_step_clipped(adam, hn.make_clip(s, 1, clip_at, norm_out), DT[dtype], params, p if dtype == "bf16" else None, g, m, v, n)
    k = OT.clip_scale(norm, clip_at)
    gs = k * g64
    wp, wm, wv = OE.adam_step(p64, gs, m64, v64, 3, 2.0 ** -10, 0.875, 0.9375, 1e-8, 0.125)
    near(m, wm, 4 * U * (np.abs(m64) + np.abs(gs)), "m")
    near(v, wv, 8 * U * (v64 + gs * gs), "v")
    mhat, vhat = (np.abs(m64) + np.abs(gs)) / (1 - 0.875 ** 3), wv / (1 - 0.9375 ** 3)
    near(p, wp, 2 * U * np.abs(p64) + 16 * U * 2.0 ** -10 * (mhat / (np.sqrt(vhat) + 1e-8) + 0.125 * np.abs(p64)), "p")
    if dtype == "bf16":
        assert torch.equal(params, p.bfloat16())
    assert not g.any() and abs(float(norm_out) - norm) <= 1.01 * U * norm


def test_clipped_chunk_update_decays_matrices_only():
    """The chunk's form: the same update as the array's, with the decay on the four matrices alone."""
    d = hn.make_desc(2, 64, 2, 128, 16, 1, hn.PRE_LN, hn.MASK_CAUSAL, hn.FP32)
    n = hn.hanayo_grad_bytes(d) // 4
    rng = np.random.default_rng(8)
    start = [values(rng, n, "fp32", s)[0] for s in (0.02, 0.3, 0.1, 0.1)]
    start[3].abs_()
    _, s = sumsq_of([start[1]])
    clip = hn.make_clip(s, 1, 0.5)

    def run(call, wd):
        w, g, m, v = (t.clone() for t in start)
        call(hn.Adam(2.0 ** -7, 0.875, 0.9375, 1e-8, wd, 2, 0), w, g, m, v)
        return w

    got = run(lambda a, w, g, m, v: hn.hanayo_chunk_adam_step_clipped(a, clip, d, w, None, g, m, v), 0.5)
    flat = lambda a, w, g, m, v: hn.hanayo_adam_step_clipped(a, clip, hn.FP32, w, None, g, m, v, n)
    decayed, plain = run(flat, 0.5), run(flat, 0.0)
    for block in range(2):
        for i, name in enumerate(hn.PARAM_NAMES):
            o, c = hn.hanayo_param_span(d, block, i)
            want = decayed if name in ("wqkv", "wo", "w1", "w2") else plain
            assert torch.equal(got[o:o + c], want[o:o + c]), name


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_rank_updates_with_clipping(dtype):
    """GpuRank's flush: all its gradients (chunks, tables, final LayerNorm) under one norm; every parameter moves as the oracle's Adam
    moves it with the scaled gradient.  A first step moves a parameter by lr g / (|g| + eps'), whose fp32 error is within 16
    steps of lr, and the parameter is rounded once (its master copy to fp32)."""
    from paper_2308_15762_amd import synth
    from paper_2308_15762_amd.runner import GpuRank
    wl = synth.WORKLOADS["tiny_gpt_fp32"].scaled(dtype=dtype, hidden=64, ffn=128, seq=32)
    lr, b1, b2, eps, wd = 2.0 ** -8, 0.875, 0.9375, 1e-8, 0.125

    def ready():
        gpu = GpuRank(wl, 0, ends=True)
        gpu.zero_grads()
        gpu.run()
        gpu.init_optimizer()
        return gpu

    gpu = ready()
    grads = [o["g"].double().cpu().numpy().ravel() for o in gpu.opt]
    before = [(o["w"] if o["master"] is None else o["master"]).double().cpu().numpy().ravel() for o in gpu.opt]
    norm = OT.grad_norm(grads)
    limit = float(np.float32(norm / 3))
    gpu.adam_step(lr, b1, b2, eps, wd, max_norm=limit)
    assert abs(float(gpu.grad_norm) - norm) <= 1.01 * U * norm
    k = OT.clip_scale(norm, limit)
    matrices = np.zeros(grads[0].size, dtype=bool)
    for blk in range(wl.n_blocks):
        for i, name in enumerate(hn.PARAM_NAMES):
            if name in ("wqkv", "wo", "w1", "w2"):
                off, cnt = hn.hanayo_param_span(gpu.desc, blk, i)
                matrices[off:off + cnt] = True
    for o, g, p in zip(gpu.opt, grads, before):
        decay = matrices if o["kind"] == "chunk" else np.full(g.size, o["kind"] != "lnf")
        z = np.zeros_like(g)
        with_wd, plain = (OE.adam_step(p, k * g, z, z, 1, lr, b1, b2, eps, w)[0] for w in (wd, 0.0))
        want = np.where(decay, with_wd, plain)
        got = (o["w"] if o["master"] is None else o["master"]).view(-1)
        near(got, want, 2 * U * np.abs(p) + 16 * U * lr * (1 + wd * np.abs(p)), o["kind"])
        assert not o["g"].any()
    # the same limit on the norm of two ranks together: this one's and another that is three times as large
    two = ready()
    parts = torch.cat([two.grad_sumsq(), 9 * two.grad_sumsq()])
    two.adam_step(lr, b1, b2, eps, wd, max_norm=limit, sumsq=parts)
    assert abs(float(two.grad_norm) - 10 ** 0.5 * norm) <= 4 * U * 10 ** 0.5 * norm


# ------------------------------------------------------------------ as they are used together

class Iteration:
    """Tokens -> scaled embedding -> two joins (the branch between them: the normed rows themselves) -> gradients -> norm ->
    clipped update of the table and the norms' parameters, on buffers of its own."""

    def __init__(self, dtype="bf16", rows=200, H=264, vocab=97, seed=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.rows, self.H, self.vocab = dtype, rows, H, vocab
        v = lambda shape, std=1.0, mean=0.0: values(rng, shape, dtype, std, mean)[0]
        self.tok = torch.from_numpy(tokens_of("padded", rng, rows, vocab).astype(np.int32)).cuda()
        self.table = v((vocab, H), 0.1)
        self.w = [v(2 * H, 0.1, 1.0), v(H, 0.1, 1.0)]
        self.gate, self.up = v(H), v((rows, H), 0.1)
        self.desc = hn.ResidualDesc(rows, H, DT[dtype], hn.NORM_LAYER, hn.NORM_RMS, hn.GATE_CHANNEL, 1.0, 0.5, EPS)
        e = lambda: torch.empty((rows, H), dtype=TD[dtype], device="cuda")
        self.x0, self.x1, self.h, self.dx, self.db, self.dsum = e(), e(), e(), e(), e(), e()
        self.stats = torch.empty((rows, 4), device="cuda")
        self.grads = torch.empty(vocab * H + 4 * H, device="cuda")
        at = 0
        self.parts = []
        for n in (vocab * H, H, 2 * H, H):
            self.parts.append(self.grads[at:at + n])
            at += n
        self.params = [self.table, self.gate, self.w[0], self.w[1]]
        self.master = [p.float().view(-1) for p in self.params]
        self.m, self.v = ([torch.zeros_like(g) for g in self.parts] for _ in range(2))
        self.work = [room(hn.hanayo_op_embedding_workspace_bytes(rows, H, vocab)), room(hn.hanayo_op_residual_scratch_bytes(self.desc)),
                     room(hn.hanayo_op_grad_workspace_bytes(4))]
        self.list = hn.grad_list(self.parts)
        self.sumsq, self.norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
        self.clip = hn.make_clip(self.sumsq, 1, 0.75, self.norm)

    def run(self, step=1, stream=None):
        dt, rows, H, V = DT[self.dtype], self.rows, self.H, self.vocab
        hn.hanayo_op_embedding_forward(dt, self.table, self.tok, 16.0, self.x0, rows, H, V, stream)
        hn.hanayo_op_residual_forward(self.desc, self.x0, self.x0, self.gate, self.w[0], self.w[1], self.x1, self.h, self.stats, stream)
        hn.hanayo_op_residual_backward(self.desc, self.x1, self.x0, self.gate, self.w[0], self.w[1], self.stats, self.up, None, self.dx,
                                       self.db, self.parts[1], self.parts[2], self.parts[3], False, self.work[1], stream)
        hn.hanayo_op_embedding_backward(dt, self.tok, self.dx, 16.0, self.parts[0], rows, H, V, False, self.work[0], stream)
        hn.hanayo_op_embedding_backward(dt, self.tok, self.db, 16.0, self.parts[0], rows, H, V, True, self.work[0], stream)
        hn.hanayo_op_grad_sumsq(self.list, self.sumsq, self.work[2], stream)
        for p, q, g, m, v in zip(self.params, self.master, self.parts, self.m, self.v):
            hn.hanayo_adam_step_clipped(hn.Adam(2.0 ** -8, 0.875, 0.9375, 1e-8, 0.0, step, 0), self.clip, dt, p,
                                        q if self.dtype == "bf16" else None, g, m, v, g.numel(), stream)

    def state(self):
        return [self.grads, self.norm, self.h, *self.params, *self.master, *self.m, *self.v]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_an_iteration_of_them(dtype):
    """The gradients that reach the norm are those of the composed function: autograd of its formula in 64 bits."""
    it = Iteration(dtype)
    wide = lambda t: t.double().cpu().requires_grad_()
    table, gate, w0, w1 = (wide(p) for p in it.params)
    tok, H = it.tok.cpu().long(), it.H
    known = ((tok >= 0) & (tok < it.vocab))[:, None]
    it.run()
    x0 = torch.where(known, 16.0 * table[tok.clamp(0, it.vocab - 1)], torch.zeros(()).double())
    if dtype == "bf16":                                    # the stored tensors are rounded: the formula is taken at their values
        x0 = x0 + (it.x0.double().cpu() - x0).detach()
    norm = lambda t, centre: (lambda c: c * torch.rsqrt((c * c).mean(1, keepdim=True) + EPS))(t - t.mean(1, keepdim=True) if centre else t)
    x1 = x0 + 0.5 * gate * (norm(x0, True) * w0[:H] + w0[H:])
    if dtype == "bf16":
        x1 = x1 + (it.x1.double().cpu() - x1).detach()
    h = norm(x1, False) * w1
    want = torch.autograd.grad((h * it.up.double().cpu()).sum(), [table, gate, w0, w1])
    # dx and dbranch are rounded to the type once before they are added up; everything else stays in fp32
    tol = 2e-5 if dtype == "fp32" else 2 * HALF["bf16"]
    total = 0.0
    for got, g in zip(it.parts, want):
        g = g.reshape(-1)
        off = float((got.double().cpu() - g).norm() / g.norm())
        assert off <= tol, off
        total += float((g * g).sum())
    assert abs(float(it.norm) - total ** 0.5) <= tol * total ** 0.5


def test_captured_iterations_replay_like_eager_ones():
    """Two iterations captured into graphs of their own, replayed in turn with eager work between, against the same eager ones."""
    eager, graphed = ([Iteration(seed=s) for s in (1, 2)] for _ in range(2))
    side = torch.cuda.Stream()
    warm = Iteration(seed=3)
    warm.run(stream=side.cuda_stream)
    torch.cuda.synchronize()
    graphs = []
    for g in graphed:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            g.run(step=2, stream=torch.cuda.current_stream().cuda_stream)
        graphs.append(graph)
    for _ in range(4):
        for e, g, graph in zip(eager, graphed, graphs):
            e.run(step=2)
            graph.replay()
            warm.run()
            torch.cuda.synchronize()
            for a, b in zip(e.state(), g.state()):
                assert torch.equal(a, b)


def test_two_streams_at_once():
    alone, both = ([Iteration(seed=s, rows=3000, H=520) for s in (1, 2)] for _ in range(2))
    for it in alone:
        it.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for it, st in zip(both, streams):
        it.run(stream=st.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert all(torch.equal(p, q) for p, q in zip(a.state(), b.state()))


def test_strided_operands_are_refused():
    t = torch.zeros((8, 32), device="cuda")
    tok = torch.zeros(8, dtype=torch.int32, device="cuda")
    for args in ((hn.FP32, t[:, :16], tok, 1.0, t, 8, 16, 8), (hn.FP32, t, tok[::2], 1.0, t, 4, 32, 8),
                 (hn.BF16, t, tok, 1.0, t, 8, 32, 8), (hn.FP32, t, tok, 1.0, t[:4], 8, 32, 8)):
        with pytest.raises(hn.HanayoError) as ei:
            hn.hanayo_op_embedding_forward(*args)
        assert ei.value.code == hn.EINVAL


def test_tensors_that_others_read_are_not_written():
    """Outputs that lie on another tensor of the list, or on a part of their own: refused before anything is launched."""
    flat, other = torch.ones(100, device="cuda"), torch.zeros(100, device="cuda")
    a, b = flat[:50], flat[50:]
    for grads, outs, fine in (([a, b], [b, other[:50]], False), ([a, b], [other[:50], a], False), ([a, b], [b, a], False),
                              ([a, b], [None, a], False), ([flat[:60]], [flat[40:]], False), ([flat[40:]], [flat[:60]], False),
                              ([a, a], [None, other[:50]], False), ([a, a], [other[:50], other[50:]], True), ([a, b], [a, None], True),
                              ([a, flat[50:50]], [other[:50], flat[20:20]], True), ([a, b], [other[50:], other[:50]], True)):
        lst, s = sumsq_of(grads, outs)
        if fine:
            hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, 1e9))
        else:
            with pytest.raises(hn.HanayoError) as ei:
                hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, 1e9))
            assert ei.value.code == hn.EINVAL
    assert (flat == 1).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("limit", [100.0, 1.0, 1e-20, 1e-38])
def test_factors_below_the_range_of_fp32(dtype, limit):
    """The largest gradients under ordinary and small limits: max_norm / norm has few bits in fp32 or none, the product is what it
    is for any other norm (and a gradient whose product is no fp32 number vanishes)."""
    limit = float(np.float32(limit))
    g = torch.full((3000,), 3e38, dtype=TD[dtype], device="cuda")
    g[1::7], g[2::7] = -2.5e37, 1e-3
    w = g.double().cpu().numpy()
    norm = OT.grad_norm([w])
    k = OT.clip_scale(norm, limit)
    assert k < 2.0 ** -126
    out = torch.empty_like(g)
    lst, s = sumsq_of([g], [out])
    hn.hanayo_op_grad_clip(lst, hn.make_clip(s, 1, limit))
    # two roundings of fp32 (the factor, the product) and one to the type, or half a step of its smallest numbers
    least = 2.0 ** -149 if dtype == "fp32" else 2.0 ** -133
    near(out, k * w, np.abs(k * w) * (HALF[dtype] + 3 * U) + least, "clipped")
    hn.hanayo_op_grad_clip(hn.grad_list([g]), hn.make_clip(s, 1, limit))
    assert torch.equal(g, out)                                         # in place
    if dtype == "fp32":
        g = torch.from_numpy(w.astype(np.float32)).cuda()
        p, m, v = (torch.full((3000,), x, device="cuda") for x in (0.5, 0.0, 0.0))
        hn.hanayo_adam_step_clipped(hn.Adam(2.0 ** -10, 0.875, 0.9375, 1e-8, 0.125, 1, 0), hn.make_clip(s, 1, limit), hn.FP32, p, None, g,
                                    m, v, 3000)
        _, wm, wv = OE.adam_step(np.full(3000, 0.5), k * w, np.zeros(3000), np.zeros(3000), 1, 2.0 ** -10, 0.875, 0.9375, 1e-8, 0.125)
        near(m, wm, 4 * U * np.abs(k * w) + 2 * least, "m")
        near(v, wv, 8 * U * (k * w) ** 2 + 2 * least, "v")


def test_operands_of_another_type_are_refused():
    """Tensors as large as the right ones, of types that other values stand for."""
    rows, H, V = 8, 16, 8
    z = lambda dtype, n=256: torch.zeros(n, dtype=dtype, device="cuda")
    b16, f32, i32, f64 = z(torch.bfloat16), z(torch.float32), z(torch.int32), z(torch.float64)
    swap = {torch.bfloat16: (z(torch.float16), z(torch.int16)), torch.float32: (i32, z(torch.uint32)), torch.int32: (f32, z(torch.uint32)),
            torch.float64: (z(torch.int64),)}
    room_ = z(torch.uint8, 1 << 20)
    desc = hn.ResidualDesc(rows, H, hn.BF16, hn.NORM_LAYER, hn.NORM_RMS, hn.GATE_CHANNEL, 1.0, 1.0, EPS)
    r = lambda: z(torch.bfloat16)
    # every call is right as it stands
    calls = [(hn.hanayo_op_embedding_forward, [hn.BF16, b16, i32, 1.0, r(), rows, H, V]),
             (hn.hanayo_op_embedding_forward, [hn.FP32, f32, i32, 1.0, z(torch.float32), rows, H, V]),
             (hn.hanayo_op_embedding_backward, [hn.BF16, i32, b16, 1.0, f32, rows, H, V, False, room_]),
             (hn.hanayo_op_residual_forward, [desc, b16, r(), r(), r(), r(), r(), r(), f32]),
             (hn.hanayo_op_residual_backward, [desc, b16, r(), r(), r(), r(), f32, r(), r(), r(), r(), z(torch.float32), z(torch.float32),
                                               z(torch.float32), False, room_]),
             (hn.hanayo_op_grad_sumsq, [hn.grad_list([f32]), f64, room_]),
             (hn.make_clip, [f64, 1, 1.0, f32]),
             (hn.hanayo_adam_step_clipped, [hn.Adam(0.1, 0.9, 0.999, 1e-8, 0.1, 1, 0), hn.make_clip(f64, 1, 1.0), hn.BF16, b16, f32,
                                            z(torch.float32), z(torch.float32), z(torch.float32), 256])]
    for call, args in calls:
        call(*args)
        seen = 0
        for at, arg in enumerate(args):
            if isinstance(arg, torch.Tensor) and arg is not room_:
                for other in swap[arg.dtype]:
                    with pytest.raises(hn.HanayoError) as ei:
                        call(*(args[:at] + [other] + args[at + 1:]))
                    assert ei.value.code == hn.EINVAL
                    seen += 1
        assert seen
    for bad in (z(torch.float16), i32, f64):
        with pytest.raises(hn.HanayoError):
            hn.grad_list([bad])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bad_at", [(0,), (1,), (0, 1, 3)])
def test_an_update_that_did_not_happen_is_not_counted(dtype, bad_at):
    """Four updates, some with an infinite gradient among them, against the good ones alone, which count what they are: the same bits."""
    n, rng = 1028, np.random.default_rng(9)
    start = [values(rng, n, "fp32", std)[0] for std in (0.02, 0.1, 0.1)]
    start[2].abs_()
    grads = [values(rng, n, "fp32", 0.3)[0] for _ in range(4)]
    s, skipped = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def run(steps, counter):
        p, m, v = (t.clone() for t in start)
        q = p.bfloat16()
        for step, g in steps:
            g = g.clone()
            hn.hanayo_op_grad_sumsq(hn.grad_list([g]), s, room(hn.hanayo_op_grad_workspace_bytes(1)))
            hn.hanayo_adam_step_clipped(hn.Adam(2.0 ** -8, 0.875, 0.999, 1e-8, 0.125, step, 0), hn.make_clip(s, 1, 1.0, None, counter), DT[dtype],
                                        q if dtype == "bf16" else p, p if dtype == "bf16" else None, g, m, v, n)
        return p, q, m, v

    good = [g for i, g in enumerate(grads) if i not in bad_at]
    for i in bad_at:
        grads[i] = grads[i].clone()
        grads[i][77] = float("inf")
    want = run(list(enumerate(good, 1)), None)
    got = run(list(enumerate(grads, 1)), skipped[:1])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert skipped.tolist() == [len(bad_at), 0]


@pytest.mark.parametrize("mixed", [False, True])
def test_a_rank_does_not_count_a_flush_that_did_not_happen(mixed):
    """GpuRank: a flush with an infinite gradient, then a good one (mixed: a clipped and an unclipped one), against the good ones alone."""
    from paper_2308_15762_amd import synth
    from paper_2308_15762_amd.runner import GpuRank
    wl = synth.WORKLOADS["tiny_gpt_fp32"].scaled(hidden=64, ffn=128, seq=32)
    ends = []
    for bad in (True, False):
        gpu = GpuRank(wl, 0, ends=True)
        gpu.zero_grads()
        gpu.init_optimizer()
        if bad:
            gpu.opt[1]["g"][0] = float("inf")
            gpu.adam_step(2.0 ** -8, max_norm=0.5)
            assert not np.isfinite(float(gpu.grad_norm)) and not any(o["m"].any() or o["g"].any() for o in gpu.opt)
        for limit in (0.5, None) if mixed else (0.5,):
            gpu.run()
            gpu.adam_step(2.0 ** -8, max_norm=limit)
        ends.append(gpu)
    for a, b in zip(*(g.opt for g in ends)):
        assert all(torch.equal(a[k], b[k]) for k in ("w", "m", "v"))
    # a call that is refused counts nothing either
    before = gpu.opt_step
    with pytest.raises(hn.HanayoError):
        gpu.adam_step(2.0 ** -8, max_norm=-1.0)
    assert gpu.opt_step == before
