"""The operators on floating-point activations against plain implementations in 64 bits.

Tolerances.  u(T) = eps(T) / 2 is the largest relative error of one rounding to T.  A product sum of R terms held in 32 bits
is off by at most (R + 16) 2^-24 S, S the sum of the terms' magnitudes (each of its additions rounds a partial sum that is at most
S; the 16 stand for the few further roundings: scales, bias, joined partial sums), its weights rounded to T by at most u(T) S, and
the rounding of the result by u(T) of it.  The 2-norm of the rounding errors of one rounding is at most u(T) times the 2-norm of
what is rounded; for independent terms of zero mean that also holds for the sum's error from rounded weights.
"""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def u(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.fixture(scope="module")
def hq():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2011_10680_b200 import binding, build
    build.build()
    h = binding.Handle(0)
    yield h
    h.close()


def out_matrix(rows, cols, dtype, stride=None):
    """An output between guard bands; with a stride, the values between its rows are guarded too (see unwritten_between)."""
    from paper_2011_10680_b200 import binding
    stride = stride or cols
    size = torch.finfo(dtype).bits // 8
    flat = binding.alloc_out(1, 1, 1, max(rows, 1) * stride * size, 8, 0).view(-1)
    flat.fill_(0xA5)
    return flat.view(dtype).view(-1, stride)[:rows, :cols]


def unwritten_between(t):
    """The values behind the last column of every row still hold what out_matrix put there."""
    rows, cols = t.shape
    stride = t.stride(0)
    if rows == 0 or stride == cols:
        return True
    whole = t.as_strided((rows, stride), (stride, 1))
    return bool((whole[:, cols:].contiguous().view(torch.uint8) == 0xA5).all())


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float64)


def strided(t, stride):
    """The same values with `stride` between the rows, NaN in the values between them."""
    if stride is None:
        return t.contiguous()
    whole = torch.full((t.shape[0], stride), float("nan"), dtype=t.dtype, device=t.device)
    whole[:, :t.shape[1]] = t
    return whole[:, :t.shape[1]]


def groups(cols, group):
    return -(-cols // group)


def random_w4(g, n, k, group, dtype):
    """Every 4-bit value, -8 among them, and scales spread over a factor of 16.  Returns (packed, scales, weights in 64 bits)."""
    v = torch.randint(-8, 8, (n, k), generator=g, device="cuda")
    s = (torch.exp2(torch.rand((n, groups(k, group)), generator=g, device="cuda", dtype=torch.float64) * 4 - 4) / math.sqrt(k)).to(dtype)
    bits = (v & 15).to(torch.int32)
    q = (bits[:, 0::2] | (bits[:, 1::2] << 4)).to(torch.uint8)
    return q, s, v.double() * s.double().repeat_interleave(group, dim=1)[:, :k]


def check_product(got, ref, magnitude, terms, dtype, rounded):
    """`magnitude`: sum of the terms' magnitudes; `rounded`: the quantized operand is rounded to the type first."""
    assert bool(torch.isfinite(got).all())
    err = (got.double() - ref).abs()
    bound = u(dtype) * ref.abs() * 1.01 + magnitude * ((u(dtype) if rounded else 0) + (terms + 16) * 2.0 ** -24) + torch.finfo(dtype).tiny
    worst = float((err / bound).max()) if err.numel() else 0.0
    assert worst <= 1, f"{worst} times the bound at {int((err / bound).argmax())} of {tuple(got.shape)}"
    norm = float(ref.norm())
    if got.numel() >= 256 and norm > 0:
        assert float(err.norm()) <= (2 if rounded else 1) * u(dtype) * norm + (terms + 16) ** 0.5 * 2.0 ** -23 * float(magnitude.norm())


# ------------------------------------------------------------------------------------------------ hq_linear_w4
def rounds_weights(m, k, group):
    """Whether weights are rounded to the activations' type first: not for few rows (see hq_linear_w4)."""
    parts = 1 if group >= k or group % 128 == 0 else 2 if group % 64 == 0 else 4
    return m * parts > 16


LINEAR = [
    # m, n, k, group: one token and a few, around the sizes where another kernel takes over; ragged outputs, last groups, last steps
    (1, 1, 32, 32), (1, 16, 128, 128), (1, 17, 128, 64), (1, 100, 96, 32), (2, 33, 160, 64), (3, 64, 256, 96), (7, 129, 512, 128),
    (8, 48, 2048, 256), (9, 31, 640, 32), (15, 257, 384, 64), (16, 128, 1024, 4096), (1, 1000, 2048, 128), (5, 40, 4096, 128),
    (1, 2300, 416, 32), (4, 4113, 128, 128), (16, 16, 8192, 64),
    # few outputs and many inputs, or rows too long for one CTA: the CTAs of a cluster share the inputs
    (1, 64, 16384, 128), (2, 40, 32768, 64), (16, 48, 16384, 128), (4, 33, 12288, 32), (3, 2500, 16416, 128), (9, 700, 8224, 8224),
    (17, 128, 64, 32), (18, 1, 32, 32), (31, 130, 96, 64), (32, 64, 128, 128), (33, 129, 160, 32), (48, 300, 512, 256), (64, 128, 1024, 64),
    (65, 127, 192, 96), (100, 200, 288, 128), (129, 257, 320, 64), (256, 128, 256, 128), (257, 384, 448, 32), (300, 513, 1056, 128),
    (1000, 640, 128, 32), (513, 1030, 2080, 96), (2, 3000, 32, 64), (700, 96, 4096, 128),
    # shapes that only the plain kernel takes: rows of packed weights off their 16 bytes
    (1, 10, 2, 32), (3, 70, 50, 32), (20, 65, 1000, 64), (70, 130, 100, 128),
]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("m,n,k,group", LINEAR)
def test_linear_w4(hq, m, n, k, group, dtype):
    g = gen(1000 + m * 7 + n)
    q, s, w = random_w4(g, n, k, group, dtype)
    x = normal(g, m, k).to(dtype)
    bias = normal(g, n).to(dtype) if (m + n) % 2 else None
    out = out_matrix(m, n, dtype)
    assert hq.linear_w4(x, q, s, group, bias, out) == 0
    hq.sync()
    ref, magnitude = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    if bias is not None:
        ref, magnitude = ref + bias.double(), magnitude + bias.double().abs()
    check_product(out, ref, magnitude, k, dtype, rounds_weights(m, k, group))


@pytest.mark.parametrize("m,n,k,group,x_stride,out_stride", [
    (1, 65, 256, 64, 300, 80), (5, 64, 256, 64, 264, 72), (16, 130, 128, 128, 129, 131), (40, 130, 256, 64, 264, 136), (40, 130, 256, 64, 257, 131),
    (300, 257, 128, 32, 136, 264), (300, 257, 128, 32, 130, 259), (65, 64, 1000, 64, 1008, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_linear_w4_strided_rows(hq, m, n, k, group, x_stride, out_stride, dtype):
    g = gen(77)
    q, s, w = random_w4(g, n, k, group, dtype)
    x = strided(normal(g, m, k).to(dtype), x_stride)
    out = out_matrix(m, n, dtype, out_stride)
    assert hq.linear_w4(x, q, s, group, None, out) == 0
    hq.sync()
    check_product(out, x.double() @ w.t(), x.double().abs() @ w.abs().t(), k, dtype, rounds_weights(m, k, group))
    assert unwritten_between(out)


@pytest.mark.parametrize("m", [1, 6, 16, 17, 70, 300])
@pytest.mark.parametrize("k,group", [(256, 32), (256, 128), (100, 32)])
def test_linear_w4_infinities_stay_in_their_row(hq, m, k, group):
    g = gen(5)
    n = 200
    q, s, w = random_w4(g, n, k, group, BF16)
    x = normal(g, m, k).to(BF16)
    x[m // 2, 3] = float("nan")
    if m > 2:
        x[m - 1, k - 1] = float("inf")
    out = out_matrix(m, n, BF16)
    assert hq.linear_w4(x, q, s, group, None, out) == 0
    hq.sync()
    ref = x.double() @ w.t()
    assert torch.equal(torch.isnan(out), torch.isnan(ref)) and torch.equal(torch.isinf(out), torch.isinf(ref))
    fine = torch.isfinite(ref)
    assert torch.equal(out[~fine & ~torch.isnan(ref)].double(), ref[~fine & ~torch.isnan(ref)])
    assert bool(((out.double() - ref).abs()[fine] <= 1e-2 * float(torch.where(fine, ref, 0.0).abs().max())).all())


def test_linear_w4_results_beyond_fp16_are_infinite(hq):
    k = 128
    for m in (1, 40):
        q = torch.full((16, k // 2), 0x77, dtype=torch.uint8, device="cuda")
        s = torch.full((16, 1), 8.0, dtype=FP16, device="cuda")
        x = torch.full((m, k), 100.0, dtype=FP16, device="cuda")
        out = out_matrix(m, 16, FP16)
        assert hq.linear_w4(x, q, s, 128, None, out) == 0
        hq.sync()
        assert bool(torch.isinf(out).all())                    # 128 * 100 * 56 = 716800


def test_linear_w4_rows_that_do_not_fit_on_chip(hq):
    """Few rows, but longer than the shared memory of a cluster: the path of many rows takes them, with its rounding."""
    m, n, k, group = 16, 72, 131072, 128
    g = gen(6)
    q, s, w = random_w4(g, n, k, group, BF16)
    x = normal(g, m, k).to(BF16)
    out = out_matrix(m, n, BF16)
    assert hq.linear_w4(x, q, s, group, None, out) == 0
    hq.sync()
    check_product(out, x.double() @ w.t(), x.double().abs() @ w.abs().t(), k, BF16, True)


@pytest.mark.parametrize("exponent", [-126, -100, -30, 50, 80, 100])
@pytest.mark.parametrize("m", [1, 8, 40])
def test_linear_w4_magnitudes(hq, m, exponent):
    """Activations across the range of bfloat16, rows of different magnitude beside one another, one element far above its row."""
    g = gen(7)
    n, k, group = 96, 512, 64
    q, s, w = random_w4(g, n, k, group, BF16)
    x = normal(g, m, k) * 2.0 ** exponent
    x[0] *= 2.0 ** 12
    x[m - 1, 7] *= 2.0 ** 14
    x = x.to(BF16)
    out = out_matrix(m, n, BF16)
    assert hq.linear_w4(x, q, s, group, None, out) == 0
    hq.sync()
    ref, magnitude = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    # (besides the usual: values far below the largest of their 128 inputs are held to 2^-36 of it, integers up to 15 and as many terms)
    beyond = x.double().abs().amax(dim=1, keepdim=True) * 2.0 ** -36 * 16 * k * float(s.double().max())
    err = (out.double() - ref).abs()
    bound = u(BF16) * ref.abs() * 1.01 + magnitude * (u(BF16) * rounds_weights(m, k, group) + (k + 16) * 2.0 ** -24) + beyond + 2.0 ** -133
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("m", [1, 40])
def test_linear_w4_offsets_beyond_32_bits(hq, m):
    """Packed weights of more than 2^32 values and outputs that lie behind them."""
    n, k, group = 140000, 32768, 128
    g = gen(3)
    q = torch.zeros((n, k // 2), dtype=torch.uint8, device="cuda")
    s = torch.full((n, k // group), 0.25, dtype=BF16, device="cuda")
    rows = [0, 1, 65535, 65536, 131071, 131072, n - 1]
    v = torch.randint(-8, 8, (len(rows), k), generator=g, device="cuda", dtype=torch.int32)
    q[rows] = ((v[:, 0::2] & 15) | ((v[:, 1::2] & 15) << 4)).to(torch.uint8)
    x = normal(g, m, k).to(BF16)
    out = out_matrix(m, n, BF16)
    assert hq.linear_w4(x, q, s, group, None, out) == 0
    hq.sync()
    w = v.double() * 0.25
    check_product(out[:, rows], x.double() @ w.t(), x.double().abs() @ w.abs().t(), k, BF16, rounds_weights(m, k, group))
    others = torch.ones(n, dtype=torch.bool)
    others[rows] = False
    assert bool((out[:, others.cuda()] == 0).all())


# ------------------------------------------------------------------------------------------------ hq_linear_w4_dgrad
DGRAD = [
    (1, 8, 32, 32), (1, 64, 128, 64), (5, 100, 96, 32), (16, 128, 256, 128), (17, 64, 128, 128), (33, 200, 160, 96), (64, 1000, 288, 64),
    (129, 136, 512, 256), (256, 256, 256, 128), (257, 72, 1056, 32), (300, 520, 384, 4096), (700, 64, 2048, 128), (128, 4096, 64, 32),
    # plain kernel only: rows of dy or of the weights off their 16 bytes
    (3, 1, 64, 32), (20, 33, 100, 64), (70, 129, 128, 32), (40, 64, 50, 32),
]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("m,n,k,group", DGRAD)
def test_linear_w4_dgrad(hq, m, n, k, group, dtype):
    g = gen(2000 + m + n)
    q, s, w = random_w4(g, n, k, group, dtype)
    dy = normal(g, m, n).to(dtype)
    dx = out_matrix(m, k, dtype)
    assert hq.linear_w4_dgrad(dy, q, s, group, dx) == 0
    hq.sync()
    check_product(dx, dy.double() @ w, dy.double().abs() @ w.abs(), n, dtype, True)


@pytest.mark.parametrize("dy_stride,dx_stride", [(136, 264), (129, 259)])
def test_linear_w4_dgrad_strided_rows(hq, dy_stride, dx_stride):
    g = gen(78)
    q, s, w = random_w4(g, 128, 256, 64, BF16)
    dy = strided(normal(g, 50, 128).to(BF16), dy_stride)
    dx = out_matrix(50, 256, BF16, dx_stride)
    assert hq.linear_w4_dgrad(dy, q, s, 64, dx) == 0
    hq.sync()
    check_product(dx, dy.double() @ w, dy.double().abs() @ w.abs(), 128, BF16, True)
    assert unwritten_between(dx)


def test_linear_w4_dgrad_against_differences(hq):
    """The layer is linear: <dout, f(x + v) - f(x - v)> / 2 = <dx, v> for every v."""
    g = gen(79)
    m, n, k, group = 64, 256, 384, 64
    q, s, w = random_w4(g, n, k, group, FP16)
    x, v = normal(g, m, k), normal(g, m, k)
    dout = normal(g, m, n).to(FP16)
    dx = out_matrix(m, k, FP16)
    assert hq.linear_w4_dgrad(dout, q, s, group, dx) == 0
    hq.sync()
    difference = float((dout.double() * ((x + v) @ w.t() - (x - v) @ w.t())).sum() / 2)
    # two roundings of every term's share in dx, independent: u * |dx| * |v| each
    assert abs(float((dx.double() * v).sum()) - difference) <= 8 * u(FP16) * float((dx.double() * v).norm())


# ------------------------------------------------------------------------------------------------ hq_act_save8, hq_act_backward8
def saved_pair(rows, cols, group):
    from paper_2011_10680_b200 import binding
    q = binding.alloc_out(1, 1, rows, cols, 8, 1).view(rows, cols)
    s = binding.alloc_out(1, 1, rows, groups(cols, group), 32, 1).view(rows, groups(cols, group)).view(FP32)
    return q, s


def quantized(x, group):
    """The definition in 64 bits on the scale in 32: integers and scales."""
    rows, cols = x.shape
    padded = torch.nn.functional.pad(x.double(), (0, groups(cols, group) * group - cols))
    s = (padded.view(rows, -1, group).abs().amax(dim=2) / 127).float()      # (torch divides 32-bit values by a number inexactly)
    wide = s.double().repeat_interleave(group, dim=1)[:, :cols]
    return torch.where(wide > 0, torch.round(x.double() / wide), 0.0).to(torch.int8), s, wide


def f_df(act, x):
    if act == "relu":
        return torch.where(x < 0, 0.0, x), (x > 0).double()
    if act == "gelu":
        phi = 0.5 * torch.erfc(-x * math.sqrt(0.5))
        return x * phi, phi + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return x * p, p + x * p * (1 - p)
    return x, torch.ones_like(x)


def check_values(got, ref, scale, dtype):
    """One rounding to the type, and 2^-19 of `scale` (the magnitude of what enters the last operation) for the 32-bit functions:
    a handful of operations of 2^-24 each and a function good to 2^-21."""
    err = (got.double() - ref).abs()
    bound = 1.01 * u(dtype) * ref.abs() + 2.0 ** -19 * scale + torch.finfo(dtype).smallest_normal
    worst = float((err / bound).max()) if err.numel() else 0.0
    assert worst <= 1, f"{worst} times the bound"


ACT = [(1, 32, 32), (1, 8, 256), (3, 128, 128), (5, 100, 32), (4, 256, 256), (7, 264, 64), (33, 1000, 128), (2, 1, 32), (6, 77, 64), (19, 2051, 256),
       (64, 520, 256), (300, 96, 64)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_act_save_and_backward(hq, dtype, act, gated):
    for rows, cols, group in ACT:
        g = gen(rows * 31 + cols)
        x = (normal(g, rows, cols) * torch.exp2(torch.rand((rows, 1), generator=g, device="cuda") * 6 - 3)).to(dtype)
        x[0, : min(cols, group)] = 0                              # a group of zeros
        x[-1, cols // 2] = -12.5                                  # far in the tail
        gate = normal(g, rows, cols).to(dtype) if gated else None
        y, (xq, xs) = out_matrix(rows, cols, dtype), saved_pair(rows, cols, group)
        gq, gs = saved_pair(rows, cols, group) if gated else (None, None)
        assert hq.act_save8(x, gate, act, group, y, xq, xs, gq, gs) == 0
        hq.sync()
        want_q, want_s, wide = quantized(x, group)
        assert torch.equal(xs, want_s)
        assert torch.equal(xq, want_q)
        f, _ = f_df(act, x.double())
        check_values(y, f * gate.double() if gated else f, (x.double() * gate.double()).abs() if gated else x.double().abs(), dtype)
        kept = want_q.double() * wide
        dy = normal(g, rows, cols).to(dtype)
        dx, dgate = out_matrix(rows, cols, dtype), out_matrix(rows, cols, dtype) if gated else None
        assert hq.act_backward8(dy, xq, xs, gq, gs, act, group, dx, dgate) == 0
        hq.sync()
        f, df = f_df(act, kept)
        if not gated:
            check_values(dx, dy.double() * df, dy.double().abs() * (1 + kept.abs()), dtype)
            continue
        want_gq, want_gs, gwide = quantized(gate, group)
        assert torch.equal(gs, want_gs) and torch.equal(gq, want_gq)
        gkept = want_gq.double() * gwide
        check_values(dx, dy.double() * gkept * df, (dy.double() * gkept).abs() * (1 + kept.abs()), dtype)
        check_values(dgate, dy.double() * f, (dy.double() * kept).abs(), dtype)


@pytest.mark.parametrize("x_stride,out_stride", [(264, 272), (263, 257)])
def test_act_strided_rows(hq, x_stride, out_stride):
    g = gen(9)
    rows, cols, group = 37, 256, 64
    x, gate, dy = (strided(normal(g, rows, cols).to(BF16), x_stride) for _ in range(3))
    y, dx, dgate = (out_matrix(rows, cols, BF16, out_stride) for _ in range(3))
    (xq, xs), (gq, gs) = saved_pair(rows, cols, group), saved_pair(rows, cols, group)
    assert hq.act_save8(x, gate, "silu", group, y, xq, xs, gq, gs) == 0
    assert hq.act_backward8(dy, xq, xs, gq, gs, "silu", group, dx, dgate) == 0
    hq.sync()
    f, _ = f_df("silu", x.double())
    check_values(y, f * gate.double(), (x.double() * gate.double()).abs(), BF16)
    kept, gkept = (quantized(t, group)[0].double() * quantized(t, group)[2] for t in (x, gate))
    f, df = f_df("silu", kept)
    check_values(dx, dy.double() * gkept * df, (dy.double() * gkept).abs() * (1 + kept.abs()), BF16)
    check_values(dgate, dy.double() * f, (dy.double() * kept).abs(), BF16)
    assert unwritten_between(y) and unwritten_between(dx) and unwritten_between(dgate)


def test_act_saves_without_an_output(hq):
    x = normal(gen(10), 9, 200).to(FP16)
    xq, xs = saved_pair(9, 200, 128)
    assert hq.act_save8(x, None, "none", 128, None, xq, xs) == 0
    hq.sync()
    want_q, want_s, _ = quantized(x, 128)
    assert torch.equal(xq, want_q) and torch.equal(xs, want_s)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_act_every_rounding_border(hq, dtype):
    """Groups whose values lie on, just above and just below the borders between two integers, for many scales; and the smallest scales."""
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
    if dtype == FP32:                                            # neighbours of the borders in 32 bits
        x[:, 3::8] = torch.nextafter(x[:, 3::8], torch.zeros_like(x[:, 3::8]))
    x[:, 0] = top.to(dtype)
    xq, xs = saved_pair(rows, group, group)
    assert hq.act_save8(x, None, "none", group, None, xq, xs) == 0
    hq.sync()
    want_q, want_s, _ = quantized(x, group)
    assert torch.equal(xs, want_s)
    assert torch.equal(xq, want_q)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_act_a_group_with_an_infinity_is_restored_as_nan(hq, dtype, bad):
    x = normal(gen(12), 3, 256).to(dtype)
    x[1, 70] = bad
    y, dx, (xq, xs) = out_matrix(3, 256, dtype), out_matrix(3, 256, dtype), saved_pair(3, 256, 64)
    assert hq.act_save8(x, None, "silu", 64, y, xq, xs) == 0
    assert hq.act_backward8(torch.ones_like(x), xq, xs, None, None, "silu", 64, dx) == 0
    hq.sync()
    hit = torch.zeros((3, 4), dtype=torch.bool, device="cuda")
    hit[1, 1] = True
    wide = hit.repeat_interleave(64, dim=1)
    assert torch.equal(torch.isnan(xs), hit) and bool((xq[wide] == 0).all())
    assert torch.equal(torch.isnan(dx), wide)
    rest = torch.ones_like(wide)
    rest[1, 70] = False
    assert bool(torch.isfinite(y[rest]).all())                   # the forward pass is element by element


def test_act_backward_against_differences(hq):
    """dx against central differences of the activation at the restored values, in 64 bits."""
    g = gen(13)
    rows, cols, group = 16, 512, 64
    x, dy = normal(g, rows, cols).float(), normal(g, rows, cols).float()
    for act in ("gelu", "silu"):
        dx, (xq, xs) = out_matrix(rows, cols, FP32), saved_pair(rows, cols, group)
        assert hq.act_save8(x, None, act, group, None, xq, xs) == 0
        assert hq.act_backward8(dy, xq, xs, None, None, act, group, dx) == 0
        hq.sync()
        kept, step = xq.double() * xs.double().repeat_interleave(group, dim=1), 1e-4
        slope = (f_df(act, kept + step)[0] - f_df(act, kept - step)[0]) / (2 * step)
        # the differences' own error: step^2 / 6 times a third derivative below 2, and 64-bit cancellation
        assert bool(((dx.double() - dy.double() * slope).abs() <= dy.double().abs() * (2.0 ** -19 * (1 + kept.abs()) + 1e-8) + 1e-30).all())


def test_act_offsets_beyond_32_bits(hq):
    rows, cols, group = 70000, 32768, 256                        # 2.3e9 values
    x = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    last = normal(gen(14), 8, cols).to(BF16)
    x[-8:] = last
    y = torch.empty_like(x)
    xq, xs = torch.empty((rows, cols), dtype=torch.int8, device="cuda"), torch.empty((rows, cols // group), dtype=FP32, device="cuda")
    assert hq.act_save8(x, None, "gelu", group, y, xq, xs) == 0
    hq.sync()
    want_q, want_s, wide = quantized(last, group)
    assert torch.equal(xq[-8:], want_q) and torch.equal(xs[-8:], want_s)
    check_values(y[-8:], f_df("gelu", last.double())[0], last.double().abs(), BF16)
    dx = y
    assert hq.act_backward8(x, xq, xs, None, None, "gelu", group, dx) == 0
    hq.sync()
    kept = want_q.double() * wide
    check_values(dx[-8:], last.double() * f_df("gelu", kept)[1], last.double().abs() * (1 + kept.abs()), BF16)
    assert not bool(xq[:-8].any()) and not bool(dx[:-8].any())


# ------------------------------------------------------------------------------------------------ hq_linear_wgrad8
WGRAD = [
    (1, 8, 32, 32), (2, 16, 128, 128), (64, 8, 256, 64), (63, 16, 144, 32), (100, 64, 400, 256), (129, 128, 128, 128), (200, 264, 272, 64),
    (333, 16, 1040, 128), (512, 256, 256, 32), (1000, 72, 640, 64), (2048, 8, 128, 32), (4100, 32, 256, 128), (700, 520, 96, 256),
    # plain kernel only
    (3, 1, 32, 32), (50, 33, 100, 64), (77, 64, 77, 32), (130, 129, 128, 128),
]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("m,n,k,group", WGRAD)
def test_linear_wgrad8(hq, m, n, k, group, dtype):
    g = gen(3000 + m + n)
    xq = torch.randint(-127, 128, (m, k), generator=g, device="cuda").to(torch.int8)
    xs = torch.exp2(torch.rand((m, groups(k, group)), generator=g, device="cuda") * 4 - 9)
    x = xq.double() * xs.double().repeat_interleave(group, dim=1)[:, :k]
    dy = normal(g, m, n).to(dtype)
    dw = out_matrix(n, k, dtype)
    assert hq.linear_wgrad8(dy, xq, xs, group, dw) == 0
    hq.sync()
    check_product(dw, dy.double().t() @ x, dy.double().abs().t() @ x.abs(), m, dtype, True)


@pytest.mark.parametrize("dy_stride,dw_stride", [(72, 272), (65, 257)])
def test_linear_wgrad8_strided_rows(hq, dy_stride, dw_stride):
    g = gen(80)
    m, n, k, group = 150, 64, 256, 64
    xq, xs, wide = quantized(normal(g, m, k).float(), group)
    dy = strided(normal(g, m, n).to(BF16), dy_stride)
    dw = out_matrix(n, k, BF16, dw_stride)
    assert hq.linear_wgrad8(dy, xq, xs, group, dw) == 0
    hq.sync()
    x = xq.double() * wide
    check_product(dw, dy.double().t() @ x, dy.double().abs().t() @ x.abs(), m, BF16, True)
    assert unwritten_between(dw)


def test_linear_wgrad8_of_no_tokens_is_zero(hq):
    dw = out_matrix(16, 64, BF16)
    dy = torch.empty((0, 16), dtype=BF16, device="cuda")
    assert hq.linear_wgrad8(dy, torch.empty((0, 64), dtype=torch.int8, device="cuda"), torch.empty((0, 1), dtype=FP32, device="cuda"), 64, dw) == 0
    hq.sync()
    assert not bool(dw.any())


def test_linear_wgrad8_a_nan_group_reaches_its_columns_only(hq):
    g = gen(81)
    m, n, k, group = 130, 24, 256, 64
    xq, xs, _ = quantized(normal(g, m, k).float(), group)
    xs[50, 2], xq[50, 128:192] = float("nan"), 0
    dw = out_matrix(n, k, BF16)
    assert hq.linear_wgrad8(normal(g, m, n).to(BF16), xq, xs, group, dw) == 0
    hq.sync()
    want = torch.zeros((n, k), dtype=torch.bool, device="cuda")
    want[:, 128:192] = True
    assert torch.equal(torch.isnan(dw), want)


def test_linear_wgrad8_against_differences(hq):
    """The loss <dout, x V^T> is linear in V: its differences along a direction D are <dV, D>."""
    g = gen(82)
    m, n, k, group = 200, 64, 128, 64
    xq, xs, wide = quantized(normal(g, m, k).float(), group)
    x, dout, d = xq.double() * wide, normal(g, m, n).to(FP16), normal(g, n, k)
    dw = out_matrix(n, k, FP16)
    assert hq.linear_wgrad8(dout, xq, xs, group, dw) == 0
    hq.sync()
    difference = float((dout.double() * (x @ d.t())).sum())
    assert abs(float((dw.double() * d).sum()) - difference) <= 8 * u(FP16) * float((dw.double() * d).norm())


# ------------------------------------------------------------------------------------------------ together
def block(hq, state):
    """One gated feed-forward block with frozen 4-bit weights, forward and backward, and a trained matrix behind its input."""
    t = state
    assert hq.linear_w4(t["x"], *t["w_up"], 64, None, t["a"]) == 0
    assert hq.linear_w4(t["x"], *t["w_gate"], 64, None, t["b"]) == 0
    assert hq.act_save8(t["a"], t["b"], "silu", 128, t["y"], t["aq"], t["as"], t["bq"], t["bs"]) == 0
    assert hq.linear_w4(t["y"], *t["w_down"], 32, t["bias"], t["out"]) == 0
    assert hq.act_save8(t["x"], None, "none", 64, None, t["xq"], t["xs"]) == 0
    assert hq.linear_w4_dgrad(t["dout"], *t["w_down"], 32, t["dy"]) == 0
    assert hq.act_backward8(t["dy"], t["aq"], t["as"], t["bq"], t["bs"], "silu", 128, t["da"], t["db"]) == 0
    assert hq.linear_w4_dgrad(t["da"], *t["w_up"], 64, t["dx"]) == 0
    assert hq.linear_wgrad8(t["da"], t["xq"], t["xs"], 64, t["dv"]) == 0


def block_state(tokens, seed, dtype=BF16, wide=640, narrow=256):
    g = gen(seed)
    t = {}
    for name, n, k, group in (("w_up", wide, narrow, 64), ("w_gate", wide, narrow, 64), ("w_down", narrow, wide, 32)):
        q, s, w = random_w4(g, n, k, group, dtype)
        t[name], t[name + "_64"] = (q, s), w
    t["x"], t["dout"], t["bias"] = normal(g, tokens, narrow).to(dtype), normal(g, tokens, narrow).to(dtype), normal(g, narrow).to(dtype)
    for name, cols in (("a", wide), ("b", wide), ("y", wide), ("out", narrow), ("dy", wide), ("da", wide), ("db", wide), ("dx", narrow)):
        t[name] = out_matrix(tokens, cols, dtype)
    t["dv"] = out_matrix(wide, narrow, dtype)
    (t["aq"], t["as"]), (t["bq"], t["bs"]), (t["xq"], t["xs"]) = saved_pair(tokens, wide, 128), saved_pair(tokens, wide, 128), saved_pair(tokens, narrow, 64)
    return t


RESULTS = ("a", "b", "y", "out", "dy", "da", "db", "dx", "dv", "aq", "as", "bq", "bs", "xq", "xs")


@pytest.mark.parametrize("tokens", [1, 13, 200])
def test_block_forward_and_backward(hq, tokens):
    t = block_state(tokens, 500 + tokens)
    block(hq, t)
    hq.sync()

    def near(name, ref, roundings):
        # every stored tensor on the way rounds once (and a tensor-core product its weights): u of the whole, each
        got = t[name].double()
        assert float((got - ref).norm()) <= roundings * u(BF16) * float(ref.norm()), name
    x, up, gate, down = t["x"].double(), t["w_up_64"], t["w_gate_64"], t["w_down_64"]
    a, b = x @ up.t(), x @ gate.t()
    near("a", a, 2), near("b", b, 2)
    # element by element the activation's relative error is at most (1 + |x f'(x) / f(x)|) times its input's, and silu's is below
    # 1 + |x|: what the large values of `a` lose is bounded by the largest of them
    spread = 2 + float(t["a"].double().abs().max())
    y = f_df("silu", a)[0] * b
    near("y", y, 2 + 2 * spread)
    near("out", y @ down.t() + t["bias"].double(), 4 + 2 * spread)
    # the backward pass, from what the forward pass stored
    dy = t["dout"].double() @ down
    near("dy", dy, 2)
    kept_a, kept_b = (t[q].double() * t[s].double().repeat_interleave(128, dim=1) for q, s in (("aq", "as"), ("bq", "bs")))
    f, df = f_df("silu", kept_a)
    da, db = t["dy"].double() * kept_b * df, t["dy"].double() * f
    near("da", da, 1.01), near("db", db, 1.01)
    near("dx", t["da"].double() @ up, 2)
    near("dv", t["da"].double().t() @ (t["xq"].double() * t["xs"].double().repeat_interleave(64, dim=1)), 2)


def test_block_is_reproducible_captured_and_on_another_stream(hq):
    """The same bits from a second run, from another stream, and from a graph replayed on new inputs; two handles at once."""
    from paper_2011_10680_b200 import binding
    for tokens in (3, 150):
        t = block_state(tokens, 700)
        block(hq, t)
        hq.sync()
        first = {k: t[k].clone() for k in RESULTS}
        block(hq, t)
        hq.sync()
        assert all(torch.equal(t[k].view(torch.uint8), first[k].view(torch.uint8)) for k in RESULTS)
        other = block_state(tokens, 700)
        hq2 = binding.Handle(0)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for _ in range(3):
                block(hq, other)
        t2 = block_state(tokens, 701)
        for _ in range(3):
            block(hq2, t2)                                       # meanwhile, on the current stream
        torch.cuda.synchronize()
        assert all(torch.equal(other[k].view(torch.uint8), first[k].view(torch.uint8)) for k in RESULTS)
        second = {k: t2[k].clone() for k in RESULTS}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block(hq, other)
        for k in ("x", "dout", "bias"):
            other[k].copy_(t2[k])
        for name in ("w_up", "w_gate", "w_down"):
            for mine, new in zip(other[name], t2[name]):
                mine.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(other[k].view(torch.uint8), second[k].view(torch.uint8)) for k in RESULTS)
        hq2.close()


def test_block_from_several_host_threads(hq):
    """One handle, four threads with a stream each: calls overlap on the host and on the GPU, and every result keeps its bits."""
    import threading
    want = block_state(70, 702)
    block(hq, want)
    hq.sync()
    states = [block_state(70, 702) for _ in range(4)]
    torch.cuda.synchronize()
    done = []

    def worker(t):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                block(hq, t)
        stream.synchronize()
        done.append(t)
    threads = [threading.Thread(target=worker, args=(t,)) for t in states]
    for thread in threads:
        thread.start()
    for thread in threads:
        thread.join()
    hq.sync()
    assert len(done) == 4
    for t in states:
        assert all(torch.equal(t[k].view(torch.uint8), want[k].view(torch.uint8)) for k in RESULTS)


def test_first_calls_of_a_process_can_be_captured():
    """No call has to run once before a capture: a new process whose first call of every operator and kernel is captured."""
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    program = """
import torch
import test_gpu_float_ops as ops
from paper_2011_10680_b200 import binding
hq = binding.Handle(0)
t = ops.block_state(70, 702)
odd_q, odd_s, _ = ops.random_w4(ops.gen(1), 96, 70, 32, ops.BF16)
odd_x, odd_out = ops.normal(ops.gen(2), 9, 70).to(ops.BF16), ops.out_matrix(9, 96, ops.BF16)
few_x, few_out = t["x"][:3], ops.out_matrix(3, 640, ops.BF16)
graph = torch.cuda.CUDAGraph()
def calls():
    ops.block(hq, t)
    assert hq.linear_w4(odd_x, odd_q, odd_s, 32, None, odd_out) == 0
    assert hq.linear_w4(few_x, *t["w_up"], 64, None, few_out) == 0
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
results = [t[k] for k in ops.RESULTS] + [odd_out, few_out]
captured = [r.clone() for r in results]
for r in results:
    r.zero_()
calls()
hq.sync()
assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(captured, results))
print("same")
"""
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(here), here, os.environ.get("PYTHONPATH", "")]))
    run = subprocess.run([sys.executable, "-c", program], env=env, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "same" in run.stdout, run.stderr[-2000:]


def test_quantized_by_the_offline_tool(hq):
    """A float matrix through the offline quantizer: the layer's result is that of the quantized weights, near the float one."""
    import numpy as np
    from paper_2011_10680_b200 import inputs, offline
    g = np.random.default_rng(4)
    w = g.normal(size=(192, 256)) / 16
    q, s = offline.quantize_weights_grouped(w, 64, "bf16")
    x = normal(gen(15), 33, 256).to(BF16)
    out = out_matrix(33, 192, BF16)
    packed, scale = torch.from_numpy(inputs.pack4(q)).cuda(), torch.from_numpy(s).cuda().to(BF16)
    assert torch.equal(scale.float().cpu(), torch.from_numpy(s))                    # the scales are bf16 values already
    assert hq.linear_w4(x, packed, scale, 64, None, out) == 0
    hq.sync()
    wq = torch.from_numpy(q * np.repeat(s.astype(np.float64), 64, axis=1)).cuda()
    check_product(out, x.double() @ wq.t(), x.double().abs() @ wq.abs().t(), 256, BF16, True)
    # a step of the 4-bit grid is max / 7: at most half of it is lost per weight
    assert float((wq.cpu() - torch.from_numpy(w)).abs().max()) <= 0.51 * float(s.max())
