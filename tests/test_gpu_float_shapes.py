"""Every launch shape of the products and of the activations at sizes that take it, against plain implementations in 64 bits.

Each case names the shape it is there for and asks the library's plan whether it takes it.  Tolerances: see test_gpu_float_ops.
"""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import test_gpu_float_ops as ops  # noqa: E402
from test_gpu_float_ops import BF16, FP16, FP32, check_product, gen, groups, hq, normal, out_matrix, random_w4, rounds_weights  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def plan_of(product, m, n, k, group):
    from paper_2011_10680_b200 import binding
    return binding.linear_plan(product, m, n, k, group, torch.cuda.get_device_properties(0).multi_processor_count)


def usual_gpu():
    """The cases' shapes are those of 148 SMs; on another number the results still have to be right."""
    return torch.cuda.get_device_properties(0).multi_processor_count == 148


def product_case(product, m, n, k, group, dtype, seed):
    """(call, output, reference, magnitude, terms, rounded) of a product on random data."""
    g = gen(seed)
    if product == "wgrad":
        q = torch.randint(-127, 128, (m, k), generator=g, device="cuda").to(torch.int8)
        s = torch.exp2(torch.rand((m, groups(k, group)), generator=g, device="cuda") * 4 - 9)
        w = q.double() * s.double().repeat_interleave(group, dim=1)[:, :k]
        b, out = normal(g, m, n).to(dtype), out_matrix(n, k, dtype)
        left = b.double().t()
        return (lambda h: h.linear_wgrad8(b, q, s, group, out)), out, left @ w, left.abs() @ w.abs(), m, True
    q, s, w = random_w4(g, n, k, group, dtype)
    if product == "dgrad":
        b, out = normal(g, m, n).to(dtype), out_matrix(m, k, dtype)
        return (lambda h: h.linear_w4_dgrad(b, q, s, group, out)), out, b.double() @ w, b.double().abs() @ w.abs(), n, True
    b, out, bias = normal(g, m, k).to(dtype), out_matrix(m, n, dtype), normal(g, n).to(dtype)
    ref, magnitude = b.double() @ w.t() + bias.double(), b.double().abs() @ w.abs().t() + bias.double().abs()
    return (lambda h: h.linear_w4(b, q, s, group, bias, out)), out, ref, magnitude, k, rounds_weights(m, k, group)


# product, m, n, k, group; columns of a tile, parts of its reduction, tiles one after another.  Seventeen and eighteen stages go round
# every ring, and leave a unit of the forward product half empty.
TENSOR = [
    ("linear", 17, 20000, 1056, 64, 32, 1, 2), ("linear", 60, 19000, 1056, 32, 64, 1, 2), ("linear", 600, 200, 1056, 64, 64, 4, 1),
    ("linear", 200, 5000, 1056, 128, 128, 1, 1), ("linear", 120, 20000, 1056, 64, 128, 1, 2), ("linear", 2500, 96, 1056, 64, 128, 4, 1),
    ("linear", 513, 8200, 1056, 64, 256, 1, 2), ("linear", 2000, 5000, 1056, 96, 256, 1, 3), ("linear", 2500, 200, 1056, 128, 256, 4, 1),
    ("dgrad", 17, 1000, 96, 64, 32, 4, 1), ("dgrad", 30, 1032, 20000, 64, 32, 1, 2), ("dgrad", 600, 1000, 160, 64, 64, 4, 1),
    ("dgrad", 60, 1032, 20000, 32, 64, 1, 2), ("dgrad", 4000, 1032, 1056, 96, 128, 1, 2), ("dgrad", 600, 2048, 160, 64, 128, 8, 1),
    ("dgrad", 2500, 1032, 4096, 128, 256, 1, 3), ("dgrad", 2500, 1000, 160, 64, 256, 4, 1),
    ("wgrad", 1100, 24, 20000, 64, 32, 1, 2), ("wgrad", 1100, 48, 20000, 32, 64, 1, 2), ("wgrad", 2000, 200, 352, 64, 64, 8, 1),
    ("wgrad", 1100, 120, 20000, 128, 128, 1, 2), ("wgrad", 2000, 200, 544, 64, 128, 8, 1),
    ("wgrad", 1100, 1032, 8224, 64, 256, 1, 3), ("wgrad", 1000, 1000, 544, 256, 256, 4, 1),
]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("product,m,n,k,group,columns,splits,rounds", TENSOR)
def test_products_on_tensor_memory(hq, product, m, n, k, group, columns, splits, rounds, dtype):  # noqa: F811
    plan = plan_of(product, m, n, k, group)
    if usual_gpu():
        assert (plan["kernel"], plan["columns"], plan["splits"], plan["rounds"]) == ("tensor_memory", columns, splits, rounds)
    call, out, ref, magnitude, terms, rounded = product_case(product, m, n, k, group, dtype, 4000 + m + n + k)
    assert call(hq) == 0
    hq.sync()
    check_product(out, ref, magnitude, terms, dtype, rounded)
    first = out.clone()
    for _ in range(20):                                            # copies land in another order every time; the bits stay
        out.zero_()
        assert call(hq) == 0
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))
    hq.sync()


@pytest.mark.parametrize("steps", [1, 2, 3, 5, 7, 12, 13, 23])
@pytest.mark.parametrize("m,n", [(17, 20000), (120, 20000), (513, 8200)])
def test_linear_w4_units_that_are_not_full(hq, m, n, steps):  # noqa: F811
    """Tiles whose last unit of packed weights holds fewer stages than others, several tiles one after another."""
    k, group = steps * 64 - 32 * (steps % 2), 32
    call, out, ref, magnitude, terms, rounded = product_case("linear", m, n, k, group, FP16, 4100 + m + steps)
    if usual_gpu():
        plan = plan_of("linear", m, n, k, group)
        assert plan["kernel"] == "tensor_memory" and plan["rounds"] > 1 and plan["steps"] == steps
    assert call(hq) == 0
    hq.sync()
    check_product(out, ref, magnitude, terms, FP16, rounded)


# few rows: m, n, k, group; columns of the matrix instruction, outputs per warp, CTAs of a tile, warps of a team
FEW = [
    (1, 4096, 4096, 128, 8, 32, 1, 16), (1, 4096, 4096, 32, 8, 32, 1, 16), (1, 5000, 2048, 128, 8, 32, 1, 8), (2, 5000, 2048, 64, 8, 32, 1, 8),
    (1, 9473, 1024, 128, 8, 32, 1, 4), (1, 9473, 1024, 32, 8, 32, 1, 4), (8, 32001, 512, 128, 8, 32, 1, 2), (1, 32001, 512, 32, 8, 32, 1, 2),
    (1, 9473, 4096, 128, 8, 32, 1, 16), (1, 9473, 4096, 32, 8, 32, 1, 16), (7, 32001, 4096, 64, 16, 32, 1, 2), (5, 32001, 8192, 128, 8, 16, 1, 8),
    (9, 32001, 512, 128, 16, 32, 1, 2), (16, 9473, 1024, 256, 16, 32, 1, None), (9, 5000, 2048, 128, 16, 32, 1, 8), (3, 32001, 512, 32, 16, 32, 1, 2),
    (8, 9473, 1024, 64, 16, 32, 1, None), (3, 4096, 4096, 32, 16, 32, 1, 16), (4, 32001, 8192, 32, 16, 16, 1, 8), (9, 5000, 8192, 128, 16, 16, 1, 16),
    (11, 4096, 8192, 128, 16, 16, 2, 16),
]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("m,n,k,group,columns,outputs,splits,team", FEW)
def test_few_rows_of_real_layers(hq, m, n, k, group, columns, outputs, splits, team, dtype):  # noqa: F811
    plan = plan_of("linear", m, n, k, group)
    if usual_gpu():
        assert (plan["kernel"], plan["columns"], plan["outputs"], plan["splits"]) == ("few_rows", columns, outputs, splits), plan
        assert team is None or plan["groups"] == team
    call, out, ref, magnitude, terms, rounded = product_case("linear", m, n, k, group, dtype, 4200 + m + n + k)
    assert call(hq) == 0
    hq.sync()
    check_product(out, ref, magnitude, terms, dtype, rounded)
    first = out.clone()
    for _ in range(5):
        out.zero_()
        assert call(hq) == 0
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))
    hq.sync()


# rows that are no multiple of a thread's pieces; enough of them for several pieces
SEVERAL_PIECES = [(2051, 1304, 128), (4097, 1000, 256), (2999, 2048, 32), (1027, 5000, 64)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("rows,cols,group", SEVERAL_PIECES)
def test_activations_of_several_pieces_per_thread(hq, rows, cols, group, dtype, gated):  # noqa: F811
    g = gen(4300 + rows)
    act = "silu" if rows % 2 else "gelu"
    x = (normal(g, rows, cols) * torch.exp2(torch.rand((rows, 1), generator=g, device="cuda") * 6 - 3)).to(dtype)
    gate = normal(g, rows, cols).to(dtype) if gated else None
    dy = normal(g, rows, cols).to(dtype)
    y, dx, dgate = out_matrix(rows, cols, dtype), out_matrix(rows, cols, dtype), out_matrix(rows, cols, dtype) if gated else None
    xq, xs = ops.saved_pair(rows, cols, group)
    gq, gs = ops.saved_pair(rows, cols, group) if gated else (None, None)
    assert hq.act_save8(x, gate, act, group, y, xq, xs, gq, gs) == 0
    assert hq.act_backward8(dy, xq, xs, gq, gs, act, group, dx, dgate) == 0
    hq.sync()
    want_q, want_s, wide = ops.quantized(x, group)
    assert torch.equal(xs, want_s) and torch.equal(xq, want_q)
    kept, f = want_q.double() * wide, ops.f_df(act, x.double())[0]
    ops.check_values(y, f * gate.double() if gated else f, (x.double() * gate.double()).abs() if gated else x.double().abs(), dtype)
    f, df = ops.f_df(act, kept)
    if not gated:
        ops.check_values(dx, dy.double() * df, dy.double().abs() * (1 + kept.abs()), dtype)
        return
    want_gq, want_gs, gwide = ops.quantized(gate, group)
    assert torch.equal(gs, want_gs) and torch.equal(gq, want_gq)
    gkept = want_gq.double() * gwide
    ops.check_values(dx, dy.double() * gkept * df, (dy.double() * gkept).abs() * (1 + kept.abs()), dtype)
    ops.check_values(dgate, dy.double() * f, (dy.double() * kept).abs(), dtype)
