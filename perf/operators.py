"""Performance cases of the floating-point operators: linear layers with 4-bit weights and group scales, their gradient, and
activations saved in 8 bits for the backward pass.

Each operator has a plain form here (elementary torch operations in 32 bits) and the call a user makes of the library
(`binding.Handle`); `own` chooses.  Four kinds of case:
  - "linear": out = x W^T (+ bias), W = 4-bit integers times a scale per group of inputs; from one token to a long prompt;
  - "dgrad":  dx = dy W of the same weights, for training through a frozen layer;
  - "act":    an activation's forward pass, which saves its input in 8 bits, and the backward pass from what was saved;
  - "wgrad":  the gradient of a weight matrix whose input was saved in 8 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# --------------------------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------------------------
def _linear(name, m, n, k, group, dtype, bias=False):
    return {"name": name, "kind": "linear", "m": m, "n": n, "k": k, "group": group, "dtype": dtype, "bias": bias}


def _dgrad(name, m, n, k, group, dtype):
    return {"name": name, "kind": "dgrad", "m": m, "n": n, "k": k, "group": group, "dtype": dtype}


def _act(name, rows, cols, group, dtype, act, gate):
    return {"name": name, "kind": "act", "rows": rows, "cols": cols, "group": group, "dtype": dtype, "act": act, "gate": gate}


def _wgrad(name, m, n, k, group, dtype):
    return {"name": name, "kind": "wgrad", "m": m, "n": n, "k": k, "group": group, "dtype": dtype}


def listed():
    return [
        # generating for one user: a single token through a square projection; latency counts
        _linear("linear_token1_4096x4096", 1, 4096, 4096, 128, "bf16"),
        # a few sequences at once through the output projection of an odd vocabulary
        _linear("linear_token7_32001x4096_fp16", 7, 32001, 4096, 64, "fp16"),
        # continuous batching: some dozens of sequences, one token each, fine groups
        _linear("linear_token48_8192x8192_g32", 48, 8192, 8192, 32, "bf16"),
        # a prompt of odd length through the widening projection of a feed-forward block
        _linear("linear_prompt4001_16384x4096", 4001, 16384, 4096, 128, "bf16", bias=True),
        # tuning with a small batch: the gradient of a square projection's input
        _dgrad("dgrad_333_4096x4096", 333, 4096, 4096, 64, "bf16"),
        # tuning with a full batch: the gradient through the widening projection
        _dgrad("dgrad_8192_16384x4096_fp16", 8192, 16384, 4096, 128, "fp16"),
        # a micro-batch of the smallest kind: two launches, latency counts
        _act("act_silu_32x4096", 32, 4096, 128, "bf16", "silu", False),
        # full-precision training of a smaller block
        _act("act_gelu_1000x2048_fp32", 1000, 2048, 32, "fp32", "gelu", False),
        # a width that fills no whole group at the end of a row
        _act("act_gelu_4095x5000_fp16", 4095, 5000, 128, "fp16", "gelu", False),
        # the gated feed-forward block of a full batch: both inputs saved
        _act("act_silu_gated_8192x16384", 8192, 16384, 128, "bf16", "silu", True),
        # the inner factor of a low-rank adapter: few outputs, long sum over the tokens
        _wgrad("wgrad_adapter_8192_16x4096", 8192, 16, 4096, 128, "bf16"),
        # a whole square matrix trained, a batch of odd length
        _wgrad("wgrad_8191_4096x4096_fp16", 8191, 4096, 4096, 64, "fp16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "dgrad", "act", "act", "wgrad"])
    dtype = rng.choice(["bf16", "fp16"])
    while True:
        if kind == "act":
            # widths of real blocks: multiples of 8, filling their last group or not
            c = {"kind": kind, "rows": _log_uniform(rng, 1, 16384), "cols": _log_uniform(rng, 64, 20000) // 8 * 8,
                 "group": rng.choice([32, 64, 128, 256]), "dtype": rng.choice(["bf16", "fp16", "fp32"]),
                 "act": rng.choice(["none", "relu", "gelu", "silu"]), "gate": rng.random() < 0.5}
            if c["rows"] * c["cols"] * (2 if c["dtype"] == "fp32" else 1) * (2 if c["gate"] else 1) <= 2 * 8192 * 16384:
                return c
            continue
        # inputs: whole 32-value blocks (the weights' rows are packed); outputs and tokens: any number in the forward pass
        k = max(8, _log_uniform(rng, 256, 16384) // 32) * 32
        if kind == "linear":
            m, n = _log_uniform(rng, 1, 8192), _log_uniform(rng, 200, 40000)
        elif kind == "dgrad":
            m, n = _log_uniform(rng, 16, 8192), _log_uniform(rng, 200, 16384) // 8 * 8
        else:
            m, n = _log_uniform(rng, 64, 16384), _log_uniform(rng, 8, 8192) // 8 * 8
        if m * n * k <= 8192 * 16384 * 4096:
            c = {"kind": kind, "m": m, "n": n, "k": k, "group": rng.choice([32, 64, 128] if kind == "wgrad" else [32, 64, 128, 256]), "dtype": dtype}
            if kind == "linear":
                c["bias"] = rng.random() < 0.3
            return c


# --------------------------------------------------------------------------------------------
# State
# --------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _activations(gen, rows, cols, dtype):
    """Hidden states: normal, with one column in about 128 ten times as large as the others."""
    loud = torch.rand((cols,), generator=gen, device="cuda") < 1.0 / 128
    return (_normal(gen, rows, cols) * torch.where(loud, 10.0, 1.0)).to(dtype)


def _groups(cols, group):
    return (cols + group - 1) // group


def _group_amax(x, group):
    """Largest magnitude of every `group` columns of a row (the last group may be shorter)."""
    rows, cols = x.shape
    padded = torch.nn.functional.pad(x, (0, _groups(cols, group) * group - cols))
    return padded.view(rows, -1, group).abs().amax(dim=2)


def _spread(s, group, cols):
    """A value per group as a value per column."""
    return s.repeat_interleave(group, dim=1)[:, :cols]


def _weights(gen, n, k, group, dtype):
    """A trained matrix's values quantized to 4 bits: (packed integers, scales of the activations' type)."""
    w = _normal(gen, n, k) / math.sqrt(k)
    scale = (_group_amax(w, group) / 7).to(dtype)
    q = torch.round(w / _spread(scale.float(), group, k)).clamp_(-7, 7).to(torch.int32) & 15
    return (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, group = TYPES[case["dtype"]], case["group"]
    s = {"case": case}
    if case["kind"] == "act":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _activations(gen, rows, cols, dtype)
        s["dy"] = (_normal(gen, rows, cols) * 1e-2).to(dtype)
        s["gate"] = _activations(gen, rows, cols, dtype) if case["gate"] else None
        s["y"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["dgate"] = torch.empty_like(s["x"]) if case["gate"] else None
        s["xq"], s["xs"] = _saved(rows, cols, group)
        s["gq"], s["gs"] = _saved(rows, cols, group) if case["gate"] else (None, None)
        return s
    m, n, k = case["m"], case["n"], case["k"]
    if case["kind"] == "wgrad":
        s["dy"] = (_normal(gen, m, n) * 1e-2).to(dtype)
        s["xq"], s["xs"] = _quantize8(_activations(gen, m, k, dtype).float(), group)
        s["dw"] = torch.empty((n, k), dtype=dtype, device="cuda")
        return s
    s["q"], s["scale"] = _weights(gen, n, k, group, dtype)
    if case["kind"] == "linear":
        s["x"] = _activations(gen, m, k, dtype)
        s["bias"] = _normal(gen, n).to(dtype) if case["bias"] else None
        s["out"] = torch.empty((m, n), dtype=dtype, device="cuda")
    else:
        s["dy"] = (_normal(gen, m, n) * 1e-2).to(dtype)
        s["dx"] = torch.empty((m, k), dtype=dtype, device="cuda")
    return s


def _saved(rows, cols, group):
    """What a saved activation is kept in: 8-bit integers and a 32-bit scale per group."""
    return (torch.empty((rows, cols), dtype=torch.int8, device="cuda"),
            torch.empty((rows, _groups(cols, group)), dtype=torch.float32, device="cuda"))


# --------------------------------------------------------------------------------------------
# Plain form
# --------------------------------------------------------------------------------------------
def _dequantized(q, scale, group):
    """The 4-bit weights as 32-bit values."""
    n, k = q.shape[0], q.shape[1] * 2
    v = torch.stack((q & 15, q >> 4), dim=2).view(n, k).to(torch.float32)
    return torch.where(v > 7, v - 16, v) * _spread(scale.float(), group, k)


def _quantize8(x, group):
    """8-bit integers and their scales: s = max|x| / 127 in 32 bits, q = x / s rounded to the nearest integer, ties to even.
    The quotient is taken in 64 bits: many inputs lie next to a border (half of a group's largest value does)."""
    s = (_group_amax(x, group).double() / 127).to(torch.float32)
    wide = _spread(s, group, x.shape[1]).double()
    q = torch.where(wide > 0, torch.round(x.double() / wide), torch.zeros_like(wide))
    return q.to(torch.int8), s


def _f(act, x):
    if act == "relu":
        return torch.clamp(x, min=0)
    if act == "gelu":
        return 0.5 * x * torch.erfc(x * -math.sqrt(0.5))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _df(act, x):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(x * -math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return p * (1 + x * (1 - p))
    return torch.ones_like(x)


def _plain(s):
    case, group = s["case"], s["case"]["group"]
    dtype = TYPES[case["dtype"]]
    if case["kind"] == "linear":
        out = s["x"].float() @ _dequantized(s["q"], s["scale"], group).t()
        return (out if s["bias"] is None else out + s["bias"].float()).to(dtype)
    if case["kind"] == "dgrad":
        return (s["dy"].float() @ _dequantized(s["q"], s["scale"], group)).to(dtype)
    if case["kind"] == "wgrad":
        x = s["xq"].float() * _spread(s["xs"], group, case["k"])
        return (s["dy"].float().t() @ x).to(dtype)
    act, cols = case["act"], case["cols"]
    x, dy = s["x"].float(), s["dy"].float()
    q, scale = _quantize8(x, group)
    saved = q.float() * _spread(scale, group, cols)
    if s["gate"] is None:
        return _f(act, x).to(dtype), (dy * _df(act, saved)).to(dtype)
    g = s["gate"].float()
    gq, gscale = _quantize8(g, group)
    gsaved = gq.float() * _spread(gscale, group, cols)
    return ((_f(act, x) * g).to(dtype), (dy * gsaved * _df(act, saved)).to(dtype), (dy * _f(act, saved)).to(dtype))


# --------------------------------------------------------------------------------------------
# The library's calls
# --------------------------------------------------------------------------------------------
_LIBRARY = []


def _library():
    """The program's handle, kept for all calls, and the binding's status check."""
    if not _LIBRARY:
        from paper_2011_10680_b200 import binding
        _LIBRARY.extend((binding.Handle(0), binding))
    return _LIBRARY


def _calls(s):
    hq, binding = _library()
    case, group = s["case"], s["case"]["group"]
    if case["kind"] == "linear":
        st, out = hq.linear_w4(s["x"], s["q"], s["scale"], group, s["bias"], s["out"]), s["out"]
    elif case["kind"] == "dgrad":
        st, out = hq.linear_w4_dgrad(s["dy"], s["q"], s["scale"], group, s["dx"]), s["dx"]
    elif case["kind"] == "wgrad":
        st, out = hq.linear_wgrad8(s["dy"], s["xq"], s["xs"], group, s["dw"]), s["dw"]
    else:
        st = hq.act_save8(s["x"], s["gate"], case["act"], group, s["y"], s["xq"], s["xs"], s["gq"], s["gs"])
        st = st or hq.act_backward8(s["dy"], s["xq"], s["xs"], s["gq"], s["gs"], case["act"], group, s["dx"], s["dgate"])
        out = (s["y"], s["dx"]) if s["gate"] is None else (s["y"], s["dx"], s["dgate"])
    if st != 0:
        raise RuntimeError(binding.status_string(st))
    return out


def run(s):
    return _calls(s) if own else _plain(s)


# --------------------------------------------------------------------------------------------
# Least work, and the results in 64 bits
# --------------------------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "act":
        values = case["rows"] * case["cols"]
        tensors = 2 if case["gate"] else 1
        saved = values + 4 * case["rows"] * _groups(case["cols"], case["group"])
        # forward: the inputs, y and what is saved; backward: dy, what was saved and the gradients
        return {"bytes": (2 * tensors + 2) * values * size + 2 * tensors * saved, "flops": 40 * tensors * values}
    m, n, k = case["m"], case["n"], case["k"]
    groups = _groups(k, case["group"])
    if case["kind"] == "wgrad":
        matrix, scales = m * k, 4 * m * groups
        small = size * (m * n + n * k)
    else:
        matrix, scales = n * k // 2, size * n * groups
        small = size * (m * k + m * n + (n if case.get("bias") else 0))
    return {"bytes": matrix + scales + small, "flops": 2 * m * n * k}


def exact(case, seed):
    s = prepare(case, seed)
    group = case["group"]
    columns = torch.arange(case["cols"] if case["kind"] == "act" else case["k"], device="cuda")
    of_column = torch.div(columns, group, rounding_mode="floor")
    if case["kind"] in ("linear", "dgrad"):
        nibbles = torch.where(columns % 2 == 0, s["q"][:, columns // 2] % 16, s["q"][:, columns // 2] // 16).to(torch.float64)
        w = (torch.remainder(nibbles + 8, 16) - 8) * s["scale"].double()[:, of_column]
        if case["kind"] == "dgrad":
            return torch.matmul(s["dy"].double(), w)
        out = torch.matmul(s["x"].double(), w.transpose(0, 1))
        return out + s["bias"].double() if case["bias"] else out
    if case["kind"] == "wgrad":
        x = s["xq"].double() * s["xs"].double()[:, of_column]
        return torch.matmul(s["dy"].double().transpose(0, 1), x)

    def restored(x):
        index = of_column.expand(x.shape[0], -1)
        top = torch.zeros((x.shape[0], _groups(case["cols"], group)), device="cuda", dtype=torch.float64)
        top.scatter_reduce_(1, index, x.double().abs(), "amax")
        step = (top / 127).to(torch.float32).double().gather(1, index)      # the scale is kept in 32 bits
        return torch.where(step > 0, torch.round(x.double() / step) * step, 0.0)

    def f_and_df(x):
        if case["act"] == "relu":
            return torch.where(x > 0, x, 0.0), torch.where(x > 0, 1.0, 0.0).double()
        if case["act"] == "gelu":
            phi = torch.special.ndtr(x)
            return x * phi, phi + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        if case["act"] == "silu":
            p = torch.sigmoid(x)
            return x * p, p + x * p * (1 - p)
        return x, torch.ones_like(x)

    dy = s["dy"].double()
    y, (kept, slope) = f_and_df(s["x"].double())[0], f_and_df(restored(s["x"]))
    if not case["gate"]:
        return y, dy * slope
    return y * s["gate"].double(), dy * slope * restored(s["gate"]), dy * kept
