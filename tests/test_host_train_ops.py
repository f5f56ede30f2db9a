"""What the operators around the chunks refuse, without touching a GPU: addresses here are numbers that nothing reads, since
every call ends in its argument checks."""

import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2308_15762_amd import hanayo as hn

A, B_, C, D, E, G, I = (0x10000 * k for k in range(1, 8))


def refuses(code, fn, *args):
    with pytest.raises(hn.HanayoError) as ei:
        fn(*args)
    assert ei.value.code == code, ei.value
    return str(ei.value)


def test_embedding_forward():
    f = hn.hanayo_op_embedding_forward
    good = [hn.BF16, A, B_, 1.0, C, 4, 16, 8]
    for at, bad in ((0, 2), (1, None), (2, None), (3, float("nan")), (3, float("inf")), (4, None), (5, -1), (6, 12), (6, 0), (7, 0),
                    (1, A + 8), (2, B_ + 2), (4, C + 8)):
        refuses(hn.EINVAL, f, *(good[:at] + [bad] + good[at + 1:]))
    for at, bad in ((5, (1 << 24) + 1), (6, 65544), (7, (1 << 28) + 1)):
        refuses(hn.EUNSUPPORTED, f, *(good[:at] + [bad] + good[at + 1:]))


def test_embedding_backward():
    f = hn.hanayo_op_embedding_backward
    good = [hn.FP32, A, B_, 1.0, C, 4, 16, 8, True, D]
    for at, bad in ((0, -1), (1, None), (2, None), (3, float("nan")), (4, None), (5, -1), (6, 4), (7, 0), (9, None), (1, A + 1),
                    (2, B_ + 4), (4, C + 4), (9, D + 8)):
        refuses(hn.EINVAL, f, *(good[:at] + [bad] + good[at + 1:]))
    refuses(hn.EUNSUPPORTED, f, *(good[:5] + [(1 << 24) + 1] + good[6:]))
    refuses(hn.EINVAL, hn.hanayo_op_embedding_workspace_bytes, 1, 12, 8)
    assert hn.hanayo_op_embedding_workspace_bytes(0, 8, 1) > 0
    assert hn.hanayo_op_embedding_workspace_bytes(1 << 24, 65536, 8) >= (1 << 24) * 8


def desc(**kw):
    d = dict(rows=4, hidden=16, dtype=hn.BF16, post_norm=hn.NORM_LAYER, pre_norm=hn.NORM_RMS, gate=hn.GATE_CHANNEL, x_scale=1.0,
             branch_scale=1.0, eps=1e-5)
    d.update(kw)
    return hn.ResidualDesc(*[d[k] for k, _ in hn.ResidualDesc._fields_])


BAD_DESCS = [dict(rows=-1), dict(hidden=12), dict(hidden=0), dict(dtype=2), dict(post_norm=3), dict(pre_norm=-1), dict(gate=3),
             dict(x_scale=float("nan")), dict(branch_scale=float("inf")), dict(eps=0.0), dict(eps=float("nan"))]


def test_residual_forward():
    f = hn.hanayo_op_residual_forward
    good = [desc(), A, B_, C, D, E, G, I, 0x100000]
    for kw in BAD_DESCS:
        refuses(hn.EINVAL, f, desc(**kw), *good[1:])
    refuses(hn.EUNSUPPORTED, f, desc(hidden=4104), *good[1:])
    refuses(hn.EUNSUPPORTED, f, desc(rows=(1 << 30) + 1), *good[1:])
    for at in range(1, 8):                       # every operand is needed, on a 16-byte boundary
        refuses(hn.EINVAL, f, *(good[:at] + [None] + good[at + 1:]))
        refuses(hn.EINVAL, f, *(good[:at] + [good[at] + 8] + good[at + 1:]))
    refuses(hn.EINVAL, f, *(good[:8] + [0x100004]))
    for at, same in ((6, B_), (7, G), (7, A), (7, B_)):
        assert "alias" in refuses(hn.EINVAL, f, *(good[:at] + [same] + good[at + 1:]))


def test_residual_backward():
    f = hn.hanayo_op_residual_backward
    names = "d x_out branch gate post pre stats dh dx_out dx dbranch dgate d_post d_pre accumulate scratch".split()
    good = [desc()] + [0x10000 * k for k in range(1, 14)] + [False, 0x200000]
    for kw in BAD_DESCS:
        refuses(hn.EINVAL, f, desc(**kw), *good[1:])
    for n in names[1:]:
        if n in ("accumulate", "dx_out"):
            continue
        at = names.index(n)
        refuses(hn.EINVAL, f, *(good[:at] + [None] + good[at + 1:]))
        refuses(hn.EINVAL, f, *(good[:at] + [good[at] + 2] + good[at + 1:]))
    refuses(hn.EINVAL, f, desc(pre_norm=hn.NORM_NONE), *(good[1:8] + [None] + good[9:]))   # no gradient at all
    for out in ("dx", "dbranch"):
        for src in ("x_out", "branch", "dh"):
            args = list(good)
            args[names.index(out)] = args[names.index(src)]
            assert "alias" in refuses(hn.EINVAL, f, *args)
    args = list(good)
    args[names.index("dbranch")] = args[names.index("dx")]
    refuses(hn.EINVAL, f, *args)
    refuses(hn.EINVAL, hn.hanayo_op_residual_scratch_bytes, desc(hidden=20))
    assert hn.hanayo_op_residual_scratch_bytes(desc(rows=0)) > 0


def raw_list(*entries):
    arr = (hn.Grad * max(1, len(entries)))(*[hn.Grad(*e) for e in entries])

    class L:
        array, count, overlap = arr, len(entries), False
    return L


def test_gradient_norm_and_clipping():
    s, c = hn.hanayo_op_grad_sumsq, hn.hanayo_op_grad_clip
    one = raw_list((A, None, 5, hn.FP32))
    for bad in (raw_list((A, None, 5, 2)), raw_list((None, None, 5, hn.FP32)), raw_list((A + 2, None, 5, hn.FP32)),
                raw_list((A + 1, None, 5, hn.BF16)), raw_list((A, None, 0, hn.FP32), (None, None, 1, hn.BF16))):
        refuses(hn.EINVAL, s, bad, B_, C)
        refuses(hn.EINVAL, c, bad, hn.make_clip(B_, 1, 1.0, C))
    for args in ((None, C), (B_, None), (B_ + 4, C), (B_, C + 4)):
        refuses(hn.EINVAL, s, one, *args)
    refuses(hn.EUNSUPPORTED, s, raw_list((A, None, 1 << 39, hn.FP32), (A, None, (1 << 39) + 1, hn.BF16)), B_, C)
    refuses(hn.EINVAL, c, raw_list((A, A + 2, 5, hn.FP32)), hn.make_clip(B_, 1, 1.0))
    for sumsq, parts, most, norm in ((None, 1, 1.0, C), (B_, 0, 1.0, C), (B_, 65537, 1.0, C), (B_, 1, -1.0, C), (B_, 1, float("nan"), C),
                                     (B_ + 4, 1, 1.0, C), (B_, 1, 1.0, C + 2)):
        refuses(hn.EINVAL, c, one, hn.make_clip(sumsq, parts, most, norm))
    assert hn._lib.hanayo_op_grad_clip(ctypes.addressof(one.array), 1, None, None) == hn.EINVAL
    assert hn._lib.hanayo_op_grad_sumsq(None, 1, B_, C, None) == hn.EINVAL
    assert hn.hanayo_op_grad_workspace_bytes(0) > 0
    assert hn.hanayo_op_grad_workspace_bytes(1000) >= hn.hanayo_op_grad_workspace_bytes(1)


def test_clipped_updates():
    f = hn.hanayo_adam_step_clipped
    adam, clip = hn.Adam(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0), hn.make_clip(A, 1, 1.0)
    good = [adam, clip, hn.BF16, B_, C, D, E, G, 16]
    for at, bad in ((0, hn.Adam(1e-3, 0.9, 0.999, 1e-8, 0.0, 0, 0)), (0, hn.Adam(1e-3, 1.0, 0.999, 1e-8, 0.0, 1, 0)),
                    (1, hn.make_clip(None, 1, 1.0)), (1, hn.make_clip(A, 0, 1.0)), (2, 5), (3, None), (4, None), (5, None), (6, None),
                    (7, None), (8, 0), (8, 18), (3, B_ + 4), (4, C + 4), (5, D + 8), (6, E + 4), (7, G + 8)):
        refuses(hn.EINVAL, f, *(good[:at] + [bad] + good[at + 1:]))
    d = hn.make_desc(1, 256, 4, 1024, 128, 2, hn.PRE_LN, hn.MASK_CAUSAL, hn.BF16)
    refuses(hn.EINVAL, hn.hanayo_chunk_adam_step_clipped, adam, hn.make_clip(A, 1, -2.0), d, B_, C, D, E, G)
    refuses(hn.EINVAL, hn.hanayo_chunk_adam_step_clipped, adam, clip, d, B_, C, D + 8, E, G)
    bad = hn.make_desc(1, 256, 3, 1024, 128, 2, hn.PRE_LN, hn.MASK_CAUSAL, hn.BF16)
    refuses(hn.EINVAL, hn.hanayo_chunk_adam_step_clipped, adam, clip, bad, B_, C, D, E, G)


def test_operands_have_to_be_on_the_gpu():
    host = torch.zeros(64, dtype=torch.float32)
    refuses(hn.EINVAL, hn.hanayo_op_embedding_forward, hn.FP32, host, B_, 1.0, C, 4, 16, 4)
    refuses(hn.EINVAL, hn.hanayo_op_embedding_forward, hn.FP32, np.zeros(64, dtype=np.float32), B_, 1.0, C, 4, 16, 4)
    refuses(hn.EINVAL, hn.hanayo_op_residual_forward, desc(), host, B_, C, D, E, G, I, None)
    refuses(hn.EINVAL, hn.grad_list, [host])
    refuses(hn.EINVAL, hn.grad_list, [torch.zeros(4, dtype=torch.float64)])
    refuses(hn.EINVAL, hn.grad_list, [host], [])
    refuses(hn.EINVAL, hn.make_clip, torch.zeros(1, dtype=torch.float64), 1, 1.0)


def test_clipping_past_the_tensor_itself():
    """An output that begins inside its own tensor, or in front of it: other workgroups would read what one has written."""
    c = hn.hanayo_op_grad_clip
    for first, to, count, dtype in ((A, A + 4, 2, hn.FP32), (A + 4, A, 2, hn.FP32), (A, A + 1998, 1000, hn.BF16), (A, A + 4, 1 << 39, hn.FP32)):
        assert "overlaps" in refuses(hn.EINVAL, c, raw_list((B_, None, 3, hn.FP32), (first, to, count, dtype)), hn.make_clip(B_, 1, 1.0))


def test_ranges_that_conflict():
    """Against every pair of ranges looked at by itself."""
    assert not hn.ranges_conflict([])
    rng = np.random.default_rng(0)
    seen = [0, 0]
    for _ in range(4000):
        spans = []
        for _ in range(int(rng.integers(1, 6))):
            first = int(rng.integers(0, 40))
            spans.append((first, first + int(rng.integers(0, 12)), bool(rng.integers(0, 2))))
        want = any(max(a[0], b[0]) < min(a[1], b[1]) and (a[2] or b[2]) for i, a in enumerate(spans) for b in spans[:i])
        assert hn.ranges_conflict(spans) == want, spans
        seen[want] += 1
    assert min(seen) > 500


def test_the_counter_of_skipped_updates():
    adam = hn.Adam(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0)
    refuses(hn.EINVAL, hn.hanayo_adam_step_clipped, adam, hn.make_clip(A, 1, 1.0, None, I + 2), hn.BF16, B_, C, D, E, G, 16)
    refuses(hn.EINVAL, hn.make_clip, A, 1, 1.0, None, torch.zeros(1, dtype=torch.int32))
    assert hn.Clip(A, 1, 1.0, None).skipped is None


def test_norms_without_a_limit_are_refused():
    from paper_2308_15762_amd.runner import GpuRank
    refuses(hn.EINVAL, lambda: GpuRank.adam_step(None, 1e-3, sumsq=torch.zeros(2, dtype=torch.float64)))


def test_a_limit_without_an_update_is_refused_by_the_benchmark():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "bench.py"), "--max-norm", "1.0"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 2 and "--adam" in r.stderr and not r.stdout
