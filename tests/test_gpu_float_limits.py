"""The operators on floating-point activations at the ends of their types' ranges."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import test_gpu_float_ops as ops  # noqa: E402
from test_gpu_float_ops import BF16, FP16, FP32, gen, hq, normal, out_matrix  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def quantized(x, group):
    """The definition in 64 bits on the scale in 32: integers of at most 127, scales, and the scales by column."""
    rows, cols = x.shape
    padded = torch.nn.functional.pad(x.double(), (0, ops.groups(cols, group) * group - cols))
    s = (padded.view(rows, -1, group).abs().amax(dim=2) / 127).float()
    wide = s.double().repeat_interleave(group, dim=1)[:, :cols]
    q = torch.where(wide > 0, torch.round(x.double() / wide), 0.0).clamp(-127, 127)
    return q.to(torch.int8), s, wide


# ------------------------------------------------------------------------------------------------ saved integers
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_act_rounding_borders(hq, dtype):  # noqa: F811
    """Values on and beside the borders between two integers, for many scales down to the smallest."""
    g = gen(11)
    top = torch.cat([torch.arange(1, 2049, device="cuda", dtype=torch.float64) / 1024,
                     torch.exp2(-torch.arange(0, 149, device="cuda", dtype=torch.float64)) * (1 if dtype != FP16 else 1024)]).to(dtype).double()
    rows, group = top.numel(), 32
    s = (top / 127).float().double()
    m = torch.randint(-127, 127, (rows, group), generator=g, device="cuda").double()
    x = ((m + 0.5) * s[:, None]).to(dtype).double()
    x[:, 1::4] = top[:, None] / 2
    x[:, 2::8] = -top[:, None] / 2
    x = torch.minimum(torch.maximum(x, -top[:, None]), top[:, None]).to(dtype)
    if dtype == FP32:
        x[:, 3::8] = torch.nextafter(x[:, 3::8], torch.zeros_like(x[:, 3::8]))
    x[:, 0] = top.to(dtype)
    xq, xs = ops.saved_pair(rows, group, group)
    assert hq.act_save8(x, None, "none", group, None, xq, xs) == 0
    hq.sync()
    want_q, want_s, _ = quantized(x, group)
    assert torch.equal(xs, want_s)
    assert torch.equal(xq, want_q)


@pytest.mark.parametrize("cols", [64, 61])
def test_act_smallest_magnitudes_keep_their_sign(hq, cols):  # noqa: F811
    """32-bit groups whose largest magnitude is 1 .. 17000 units of 2^-149: the scale has few bits, or none."""
    units = torch.cat([torch.arange(0, 1200, device="cuda"), torch.arange(1200, 17000, 13, device="cuda")]).double()
    rows, group = units.numel(), 32
    x = torch.round(torch.rand((rows, cols), generator=gen(12), device="cuda", dtype=torch.float64) * 2 * units[:, None] - units[:, None])
    x[:, 0], x[:, 1], x[:, 40], x[:, 41] = units, -units, -units, units
    x = (x * 2.0 ** -149).float()
    (xq, xs), (gq, gs) = ops.saved_pair(rows, cols, group), ops.saved_pair(rows, cols, group)
    assert hq.act_save8(x, -x, "none", group, None, xq, xs, gq, gs) == 0
    hq.sync()
    want_q, want_s, wide = quantized(x, group)
    assert torch.equal(xs, want_s) and torch.equal(xq, want_q) and torch.equal(gs, want_s) and torch.equal(gq, -want_q)
    assert bool((xq.double() * x.double() >= 0).all())
    # half a step is lost, and what a quotient beyond 127 loses: 63 steps at 190 units
    assert bool(((xq.double() * wide - x.double()).abs() <= torch.maximum(wide * 63, x.double().abs() * (wide == 0))).all())
