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


# ------------------------------------------------------------------------------------------------ scales of weights that are not finite
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("k,group", [(256, 32), (256, 64), (512, 128), (100, 32), (16384, 128)])
@pytest.mark.parametrize("m", [1, 3, 8, 16, 17, 70])
def test_linear_w4_infinite_scales(hq, m, k, group, dtype):  # noqa: F811
    """q * infinity by IEEE's rules, term by term: infinite where all terms of the group are, with one sign, NaN otherwise."""
    g = gen(31)
    n, groups = 48, ops.groups(k, group)
    v = torch.randint(-7, 8, (n, k), generator=g, device="cuda")
    v[v == 0] = 5
    x = normal(g, m, k)
    x[x == 0] = 1
    s = torch.full((n, groups), 0.5, device="cuda", dtype=dtype)
    sign = torch.sign(x[0])
    hit = slice(group * (groups - 1), k)                          # the last group, which may be shorter
    for i, mode in enumerate(("plain", "one sign", "other sign", "both signs", "a zero", "first group", "nan")):
        if mode == "plain":
            continue
        at = slice(0, group) if mode == "first group" else hit
        s[i, 0 if mode == "first group" else groups - 1] = float("nan") if mode == "nan" else float("-inf" if mode == "other sign" else "inf")
        v[i, at] = (v[i, at].abs() * sign[at]).long()             # every term of row 0 positive
        if mode == "both signs":
            v[i, at.stop - 1] = -v[i, at.stop - 1]
        if mode == "a zero":
            v[i, at.stop - 1] = 0
    bits = (v & 15).to(torch.int32)
    q = (bits[:, 0::2] | (bits[:, 1::2] << 4)).to(torch.uint8)
    x = x.to(dtype)
    out = out_matrix(m, n, dtype)
    assert hq.linear_w4(x, q, s, group, None, out) == 0
    hq.sync()
    # (a product of matrices may skip or reorder nothing here: term by term, in 64 bits)
    w = v.double() * s.double().repeat_interleave(group, dim=1)[:, :k]
    ref = torch.stack([(x.double()[r] * w).sum(dim=1) for r in range(m)])
    assert bool(torch.isinf(ref[0, 1])) and bool(torch.isinf(ref[0, 2])) and bool(torch.isinf(ref[0, 5])) and bool(torch.isnan(ref[0, 3:5]).all())
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    infinite = torch.isinf(ref)
    assert torch.equal(out[infinite].double(), ref[infinite]) and bool(torch.isfinite(out[torch.isfinite(ref)]).all())


def test_linear_w4_sums_beyond_32_bits_are_infinite(hq):  # noqa: F811
    """Finite scales and activations whose products pass the 32-bit range: infinite with the sign of the sum, few rows and many."""
    for m in (1, 4, 40):
        q = torch.full((32, 64), 0x77, dtype=torch.uint8, device="cuda")
        q[16:] = 0x99                                             # -7
        s = torch.full((32, 1), 2.0 ** 60, dtype=BF16, device="cuda")
        x = torch.full((m, 128), 2.0 ** 72, dtype=BF16, device="cuda")
        out = out_matrix(m, 32, BF16)
        assert hq.linear_w4(x, q, s, 128, None, out) == 0
        hq.sync()
        assert bool((out[:, :16] == float("inf")).all()) and bool((out[:, 16:] == float("-inf")).all())


# ------------------------------------------------------------------------------------------------ far tails
# Exponents of up to 130 (in base two) are products in 32 bits: off by 2.5 * 130 * ln(2) * 2^-24 of the result, and a few roundings.
TAIL = 2.0 ** -15


def check_tail(got, ref, dtype):
    """Relative wherever the result is a normal number; half a unit of the subnormal ones of the type (an intermediate rounds there too)."""
    err, unit = (got.double() - ref).abs(), torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    bound = (TAIL + 1.01 * ops.u(dtype)) * ref.abs() + 1.01 * unit
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cols", [4096, 4093])
def test_silu_far_to_the_left(hq, dtype, gated, cols):  # noqa: F811
    """x e^x is a normal 32-bit number down to x = -91.9, where e^x itself is not."""
    x = torch.linspace(-91.5, -80.0, cols, device="cuda", dtype=torch.float64)[None].to(dtype).repeat(3, 1)
    x[1] = x[1].flip(0)
    x[2, ::2] = 3.0
    gate = normal(gen(41), 3, cols).abs().add(1).to(dtype) if gated else None
    y, (xq, xs), (gq, gs) = out_matrix(3, cols, dtype), ops.saved_pair(3, cols, 128), ops.saved_pair(3, cols, 128)
    assert hq.act_save8(x, gate, "silu", 128, y, xq, xs, *((gq, gs) if gated else ())) == 0
    hq.sync()
    f = ops.f_df("silu", x.double())[0]
    check_tail(y, f * gate.double() if gated else f, dtype)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("act,left,right", [("silu", -91.0, -60.0), ("gelu", -13.2, -10.0)])
def test_slopes_far_to_the_left(hq, act, left, right, dtype, gated):  # noqa: F811
    """From saved values of every magnitude in that range: one group of 32 per scale."""
    rows, cols = 96, 32
    xs = (torch.linspace(-left, -right, rows, device="cuda", dtype=torch.float64) / 127).float()[:, None].contiguous()
    xq = torch.arange(127, 127 - cols, -1, device="cuda").neg().to(torch.int8).repeat(rows, 1).contiguous()
    xq[:, 5], xq[:, 9] = 127, 0
    gq, gs = torch.full_like(xq, 127), torch.full_like(xs, 2.0 / 127)
    dy, dx, dgate = torch.full((rows, cols), 1.5, device="cuda", dtype=dtype), out_matrix(rows, cols, dtype), out_matrix(rows, cols, dtype)
    if gated:
        assert hq.act_backward8(dy, xq, xs, gq, gs, act, 32, dx, dgate) == 0
    else:
        assert hq.act_backward8(dy, xq, xs, None, None, act, 32, dx) == 0
    hq.sync()
    kept = xq.double() * xs.double()
    f, df = ops.f_df(act, kept)
    df_scale = 127 * gs.double() if gated else 1.0
    keep = df.abs() > 1e-3 * ops.f_df(act, kept + 0.01)[1].abs()            # (none lies next to a zero of the derivative)
    assert bool(keep.all())
    check_tail(dx, 1.5 * df * df_scale, dtype)
    if gated:
        check_tail(dgate, 1.5 * f, dtype)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 2.0 ** 80, -(2.0 ** 75)])
@pytest.mark.parametrize("at", [3, 8000, 16381])
@pytest.mark.parametrize("m,n", [(1, 64), (2, 40), (11, 4097)])
def test_linear_w4_large_values_anywhere_in_a_row(hq, m, n, at, bad):  # noqa: F811
    """One value that the 16-bit form of few rows does not hold, in the inputs of any CTA that shares the row; strided output, bias."""
    g, k, group = gen(33), 16384, 128
    q, s, w = ops.random_w4(g, n, k, group, BF16)
    x = normal(g, m, k).to(BF16)
    x[m - 1, at] = bad
    bias = normal(g, n).to(BF16)
    out = out_matrix(m, n, BF16, n + 7)
    assert hq.linear_w4(x, q, s, group, bias, out) == 0
    hq.sync()
    wx = w * x.double()[:, None, :] if m * n < 1000 else None
    ref = (wx.sum(dim=2) if wx is not None else torch.stack([(w * r).sum(dim=1) for r in x.double()])) + bias.double()
    magnitude = torch.stack([(w * r).abs().sum(dim=1) for r in x.double()]) + bias.double().abs()
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    fine = torch.isfinite(ref)
    assert torch.equal(out[~fine & ~torch.isnan(ref)].double(), ref[~fine & ~torch.isnan(ref)])
    # (few rows: a value above 2^73 makes all rows of the call go value by value)
    bound = 1.01 * ops.u(BF16) * ref.abs() + (k + 16) * 2.0 ** -24 * magnitude
    assert bool(((out.double() - ref).abs() <= bound)[fine].all())
    assert ops.unwritten_between(out)
