"""The operators on floating-point activations without a GPU: structure layouts, refusals of the C entry points, checks of the
binding, the grouped 4-bit quantizer of the offline tool."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest

from paper_2011_10680_b200 import binding, build, inputs, offline

OK, INVALID, UNSUPPORTED, ALIGNMENT, CUDA = 0, 1, 2, 3, 6
A16 = 1 << 20                       # stands for device memory: aligned, not NULL, never read by a call that is refused
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def handle():
    # a refused call does not look into its handle, and a handle cannot be made here without a GPU
    return C.create_string_buffer(256)


def matrix(rows, cols, stride=None, t=BF16, data=A16):
    return binding._PACK_MATRIX(data, rows, cols, cols if stride is None else stride, t)


def w4(n=64, k=128, group=64, q=A16, scale=A16):
    return binding._PACK_W4(q, scale, n, k, group)


def saved(rows, cols, group=128, q=A16, scale=A16):
    return binding._PACK_SAVED8(q, scale, rows, cols, group)


def test_structures_match_the_header():
    assert C.sizeof(binding.hq_matrix) == 40 and C.sizeof(binding.hq_w4) == 32 and C.sizeof(binding.hq_saved8) == 40
    assert matrix(3, 5, 7, F16) == bytes(binding.hq_matrix(A16, 3, 5, 7, F16))
    assert w4(3, 64, 32, 16, 32) == bytes(binding.hq_w4(16, 32, 3, 64, 32))
    assert saved(1 << 33, 5, 32, 16, 32) == bytes(binding.hq_saved8(16, 32, 1 << 33, 5, 32))


LINEAR = [
    (matrix(4, 128), w4(), None, matrix(4, 64), None),                         # accepted
    (None, w4(), None, matrix(4, 64), INVALID),
    (matrix(4, 128), None, None, matrix(4, 64), INVALID),
    (matrix(4, 128), w4(), None, None, INVALID),
    (matrix(4, 128, data=0), w4(), None, matrix(4, 64), INVALID),
    (matrix(4, 128, t=F32), w4(), None, matrix(4, 64, t=F32), INVALID),        # 32-bit activations
    (matrix(4, 128, t=F16), w4(), None, matrix(4, 64, t=BF16), INVALID),       # mixed types
    (matrix(4, 128, t=7), w4(), None, matrix(4, 64, t=7), INVALID),
    (matrix(4, 128, t=-1), w4(), None, matrix(4, 64), INVALID),
    (matrix(4, 96), w4(), None, matrix(4, 64), INVALID),                       # k differs
    (matrix(4, 128), w4(), None, matrix(4, 65), INVALID),                      # n differs
    (matrix(4, 128), w4(), None, matrix(5, 64), INVALID),                      # rows differ
    (matrix(-1, 128), w4(), None, matrix(-1, 64), INVALID),
    (matrix(4, 128, 127), w4(), None, matrix(4, 64), INVALID),                 # overlapping rows
    (matrix(4, 128, 0), w4(), None, matrix(4, 64), INVALID),                   # a broadcast row
    (matrix(4, 128, -128), w4(), None, matrix(4, 64), INVALID),
    (matrix(4, 128), w4(group=16), None, matrix(4, 64), INVALID),
    (matrix(4, 128), w4(group=48), None, matrix(4, 64), INVALID),
    (matrix(4, 128), w4(group=0), None, matrix(4, 64), INVALID),
    (matrix(4, 128), w4(group=-32), None, matrix(4, 64), INVALID),
    (matrix(4, 127), w4(k=127), None, matrix(4, 64), INVALID),                 # an odd number of packed values
    (matrix(4, 128), w4(n=0), None, matrix(4, 0), INVALID),
    (matrix(4, 128), w4(q=0), None, matrix(4, 64), INVALID),
    (matrix(4, 128), w4(scale=0), None, matrix(4, 64), INVALID),
    (matrix(4, 128, data=A16 + 8), w4(), None, matrix(4, 64), ALIGNMENT),
    (matrix(4, 128), w4(q=A16 + 4), None, matrix(4, 64), ALIGNMENT),
    (matrix(4, 128), w4(scale=A16 + 1), None, matrix(4, 64), ALIGNMENT),
    (matrix(4, 128), w4(), A16 + 1, matrix(4, 64), ALIGNMENT),
    (matrix(4, 128), w4(), None, matrix(4, 64, data=A16 + 2), ALIGNMENT),
    (matrix((1 << 31), 128), w4(), None, matrix(1 << 31, 64), UNSUPPORTED),
    (matrix(4, 128, 1 << 41), w4(), None, matrix(4, 64), UNSUPPORTED),
]


@pytest.mark.parametrize("case", range(len(LINEAR)))
def test_linear_refusals(L, handle, case):
    x, w, bias, out, want = LINEAR[case]
    if want is None:
        pytest.importorskip("torch")
        import torch
        if torch.cuda.is_available():
            pytest.skip("an accepted call would run")
        want = CUDA                                             # it passes every check and finds no device
    assert L.hq_linear_w4(handle, x, w, bias, out, None) == want
    if want != CUDA and bias is None:                           # the gradient has the two matrices the other way round
        assert L.hq_linear_w4_dgrad(handle, out, w, x, None) == want


def test_null_handle_and_empty_batches(L, handle):
    assert L.hq_linear_w4(None, matrix(4, 128), w4(), None, matrix(4, 64), None) == INVALID
    assert L.hq_linear_w4_dgrad(None, matrix(4, 64), w4(), matrix(4, 128), None) == INVALID
    assert L.hq_act_save8(None, matrix(4, 128), None, 0, None, saved(4, 128), None, None) == INVALID
    assert L.hq_act_backward8(None, matrix(4, 128), saved(4, 128), None, 0, matrix(4, 128), None, None) == INVALID
    assert L.hq_linear_wgrad8(None, matrix(4, 64), saved(4, 128), matrix(64, 128), None) == INVALID
    # no rows: nothing to do, and the empty tensors' pointers may be NULL
    assert L.hq_linear_w4(handle, matrix(0, 128, data=0), w4(), None, matrix(0, 64, data=0), None) == OK
    assert L.hq_linear_w4_dgrad(handle, matrix(0, 64, data=0), w4(), matrix(0, 128, data=0), None) == OK
    assert L.hq_act_save8(handle, matrix(0, 128, data=0), None, 2, matrix(0, 128, data=0), saved(0, 128, q=0, scale=0), None, None) == OK
    assert L.hq_act_backward8(handle, matrix(0, 128, data=0), saved(0, 128, q=0, scale=0), None, 2, matrix(0, 128, data=0), None, None) == OK


@pytest.mark.parametrize("args,want", [
    ((matrix(4, 100), None, 4, matrix(4, 100), saved(4, 100), None), INVALID),                    # no such activation
    ((matrix(4, 100), None, -1, matrix(4, 100), saved(4, 100), None), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100), None, None), INVALID),                             # nowhere to save
    ((matrix(4, 100), matrix(4, 100), 1, matrix(4, 100), saved(4, 100), None), INVALID),          # a gate that is not saved
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(4, 100), saved(4, 100)), INVALID),
    ((matrix(4, 100), matrix(4, 99), 1, matrix(4, 100), saved(4, 100), saved(4, 100)), INVALID),
    ((matrix(4, 100), matrix(4, 100, t=F16), 1, matrix(4, 100), saved(4, 100), saved(4, 100)), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100, t=F32), saved(4, 100), None), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(5, 100), None), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(4, 101), None), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(4, 100, 96), None), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(4, 100, 512), None), INVALID),
    ((matrix(4, 100), matrix(4, 100), 1, matrix(4, 100), saved(4, 100, 64), saved(4, 100, 32)), INVALID),
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(4, 100, q=A16 + 8), None), ALIGNMENT),
    ((matrix(4, 100), None, 1, matrix(4, 100), saved(4, 100, scale=A16 + 2), None), ALIGNMENT),
    ((matrix(4, 100, data=A16 + 2), None, 1, matrix(4, 100), saved(4, 100), None), ALIGNMENT),
    ((matrix(4, 100, t=3), None, 1, None, saved(4, 100), None), INVALID),
])
def test_act_refusals(L, handle, args, want):
    assert L.hq_act_save8(handle, *args, None) == want
    x, gate, act, y, sx, sg = args
    if y is not None and sx is not None and (gate is None) == (sg is None):
        assert L.hq_act_backward8(handle, y, sx, sg, act, x, gate, None) == want


@pytest.mark.parametrize("args,want", [
    ((matrix(9, 64), saved(9, 128), matrix(64, 127)), INVALID),
    ((matrix(9, 64), saved(8, 128), matrix(64, 128)), INVALID),
    ((matrix(9, 64), saved(9, 128), matrix(63, 128)), INVALID),
    ((matrix(9, 64), saved(9, 128), matrix(64, 128, t=F16)), INVALID),
    ((matrix(9, 64), saved(9, 128), matrix(64, 128, t=F32)), INVALID),
    ((matrix(9, 64, t=F32), saved(9, 128), matrix(64, 128, t=F32)), INVALID),
    ((matrix(9, 64), None, matrix(64, 128)), INVALID),
    ((matrix(9, 64), saved(9, 128, group=48), matrix(64, 128)), INVALID),
    ((matrix(9, 64), saved(9, 128, q=A16 + 1), matrix(64, 128)), ALIGNMENT),
    ((matrix(9, 64), saved(9, 128), matrix(64, 128, data=A16 + 2)), ALIGNMENT),
])
def test_wgrad_refusals(L, handle, args, want):
    assert L.hq_linear_wgrad8(handle, *args, None) == want


class FakeTensor:
    """What the binding asks of a tensor, without a device."""

    def __init__(self, shape, stride, dtype, device=0):
        self.shape, self._stride, self.dtype, self._device = shape, stride, dtype, device

    def stride(self):
        return self._stride

    def get_device(self):
        return self._device

    def data_ptr(self):
        return A16


def test_binding_describes_strided_rows_and_refuses_what_it_cannot_describe():
    torch = pytest.importorskip("torch")
    t = FakeTensor((3, 8), (24, 1), torch.float16)
    assert binding._packed_matrix(t, 0) == matrix(3, 8, 24, F16)
    assert binding._packed_matrix(FakeTensor((1, 8), (0, 1), torch.bfloat16), 0) == matrix(1, 8, 8)      # one row: its stride means nothing
    assert binding._packed_matrix(FakeTensor((4, 8), (8, 1), torch.float64), 0) == matrix(4, 8, 8, -1)   # refused by the library
    with pytest.raises(ValueError):
        binding._packed_matrix(FakeTensor((3, 8), (1, 3), torch.float16), 0)                            # columns of a transposed view
    with pytest.raises(ValueError):
        binding._packed_matrix(FakeTensor((3, 8), (8, 1), torch.float16, device=1), 0)
    q, s = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.float16)
    half = torch.float16
    for bad_q, bad_s, group in ((q, s, 128), (q, s[:3], 64), (q.t(), s, 64), (q.view(-1), s, 64), (q, s.float(), 64), (q.short(), s, 64), (q, s, 0),
                                (q, torch.zeros(2, 4, dtype=half).t(), 64)):
        with pytest.raises(ValueError):
            binding._grouped(bad_q, bad_s, group, 2, half, -1)
    assert binding._grouped(q, s, 64, 2, half, -1) == (4, 128)
    with pytest.raises(ValueError):
        binding._grouped(q, s, 64, 2, half, 0)                                                          # host memory


@pytest.mark.parametrize("scale_type", ["bf16", "fp16"])
@pytest.mark.parametrize("n,k,group", [(3, 64, 32), (5, 100, 64), (2, 32, 4096)])
def test_grouped_weights_are_the_nearest_representable(n, k, group, scale_type):
    g = inputs.rng(77)
    w = g.normal(size=(n, k)) * g.uniform(0.01, 3, size=(n, 1))
    w[0, :32] = 0
    q, s = offline.quantize_weights_grouped(w, group, scale_type)
    assert s.dtype == np.float32 and s.shape == (n, -(-k // group)) and q.shape == (n, k)
    assert np.abs(q).max() <= 7
    eps = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[scale_type]                 # half a step of the scales' type
    for i in range(n):
        for j in range(s.shape[1]):
            part = slice(j * group, min(k, (j + 1) * group))
            top = np.abs(w[i, part]).max()
            assert abs(s[i, j] - top / 7) <= (eps + 2.0 ** -23) * top / 7
            # half a step, and what the scale's rounding takes from the largest values (clamped at 7 steps)
            assert np.all(np.abs(w[i, part] - q[i, part] * s[i, j]) <= 0.5 * s[i, j] * (1 + 1e-6) + top * eps)
    assert np.array_equal(inputs.unpack4(inputs.pack4(q), True), q)


def test_grouped_weights_refuse_what_cannot_be_kept():
    with pytest.raises(ValueError):
        offline.quantize_weights_grouped(np.full((1, 32), np.inf), 32)
    with pytest.raises(ValueError):
        offline.quantize_weights_grouped(np.full((1, 32), 1e6), 32, "fp16")
    with pytest.raises(ValueError):
        offline.quantize_weights_grouped(np.zeros((2, 2, 2)), 32)
