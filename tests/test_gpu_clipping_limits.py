"""Clipping where the norm, the limit or the factor leaves the range of fp32.

Bounds.  The factor is made in 64 bits from the norm: the 64-bit one in the call
that does both, else the given fp32 number (off by 2^-24).  Its rounding to fp32
and the product's are 2^-24 each, so 3 * 2^-24 bounds a value's relative error;
its type adds half a step, and half of the smallest subnormal where it underflows.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import clip_grad_norm, clip_grads, grad_norm  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
U32 = 2.0 ** -24
INF = float("inf")


def gradients(value, dtype, tensors):
    """One long tensor and short ones: up to 160 go in one launch, which makes the norm and clips."""
    return [torch.full((5_000 if k == 0 else 3,), value, device="cuda", dtype=dtype) for k in range(tensors)]


def clipped(grads, max_norm, how):
    """(norm, clipped tensors)."""
    if how == "out":
        outs = [torch.full_like(g, 7) for g in grads]
        return clip_grad_norm(grads, max_norm, out=outs), outs
    if how == "in place":
        return clip_grad_norm(grads, max_norm), grads
    norm = grad_norm(grads)
    clip_grads(grads, norm, max_norm)
    return norm, grads


@pytest.mark.parametrize("tensors", [2, 161])
@pytest.mark.parametrize("how", ["out", "in place", "two calls"])
@pytest.mark.parametrize("limit", [0.0, 1.0, 3e38, INF])
def test_infinite_norm_clips_to_zero(limit, how, tensors):
    """Whatever the limit, and only what was infinite is no number."""
    grads = gradients(2.0, F32, tensors)
    grads[0][17] = -INF
    norm, got = clipped(grads, limit, how)
    assert float(norm) == INF
    assert bool(got[0][17].isnan())
    got[0][17] = 0
    assert all(bool((t == 0).all()) for t in got)


@pytest.mark.parametrize("tensors", [2, 161])
@pytest.mark.parametrize("how", ["out", "in place"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("limit", [1.0, 1e38, INF])
def test_norm_above_fp32(limit, dtype, how, tensors):
    """Finite gradients whose norm is no finite fp32 number: the factor comes from the 64-bit norm."""
    grads = gradients(2.0 ** 127, dtype, tensors)
    want = 2.0 ** 127 * math.sqrt(sum(g.numel() for g in grads))
    norm, got = clipped(grads, limit, how)
    assert float(norm) == INF  # what fp32 holds of it
    ref = 2.0 ** 127 * min(1.0, float(np.float32(limit)) / want)
    for t in got:
        assert bool(((t.double() - ref).abs() <= (torch.finfo(dtype).eps / 2 * (dtype != F32) + 3 * U32) * ref).all())


@pytest.mark.parametrize("tensors", [2, 161])
@pytest.mark.parametrize("how", ["out", "in place", "two calls"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value,limit", [(2.0 ** 115, 1e-3), (2.0 ** 120, 1e-6), (2.0 ** 121, 1e-15), (2.0 ** 110, 1e-30),
                                         (2.0 ** 121, 1e-42)])
def test_factor_below_fp32s_normal_numbers(value, limit, dtype, how, tensors):
    grads = gradients(value, dtype, tensors)
    want = value * math.sqrt(sum(g.numel() for g in grads))
    factor = float(np.float32(limit)) / (want + float(np.float32(1e-6)))
    assert factor < 2.0 ** -121 and want < 3e38
    norm, got = clipped(grads, limit, how)
    assert abs(float(norm) - want) <= 1.01 * U32 * want
    ref = value * factor
    tol = (torch.finfo(dtype).eps / 2 * (dtype != F32) + 3 * U32) * ref
    tol += torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for t in got:
        assert bool(((t.double() - ref).abs() <= tol).all())
