"""bpe_linear on every one of its tiles (linear_cases.py; test_linear_plan_rule.py holds the sizes to them): rows of sixteen-byte groups and
rows at odd addresses, whole tiles and edges, k whole and in parts, bias, activation and residual in the epilogue, separate and in place.

x and weight are whole numbers up to 3, weight's over 64, so every sum of products is exact in 32 bits in whatever order (at most 9 k
of 2^-6, below 2^24 of them), and so are bias, relu and residual: the outputs have to be equal to the exact value rounded once.
The other activations are held to the header's bounds on the exact argument, the residual's addition to one rounding more."""
import numpy as np
import pytest

import linear_cases
import linear_plan
from test_gpu_activations import U, _exact

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _whole(torch, seed, rows, cols, most):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, (rows, cols), generator=g, device="cuda", dtype=torch.int16)


def _inside(torch, values, dtype, pad, offset):
    """The matrix with rows `pad` elements further apart, `offset` elements into a buffer that holds NaN everywhere else."""
    rows, cols = values.shape
    t = torch.full((rows * (cols + pad) + offset + 64,), float("nan"), dtype=dtype, device="cuda")
    view = t[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(values)
    return t, view


def _half_unit(v, out):
    return {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[out] * np.abs(v) + (2.0 ** -25 if out == "float16" else 0.0)


@pytest.mark.parametrize("dtype,out", [("bfloat16", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16"), ("float16", "float32")])
@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "odd"])
@pytest.mark.parametrize("case", linear_cases.CASES, ids=lambda c: "-".join(map(str, c)))
def test_every_tile(B, case, aligned, dtype, out):
    import torch
    tile, parts, m, n, k = case
    got_tile, splits = linear_plan.plan(m, n, k, aligned)
    assert (got_tile, splits > 1) == (tile, parts)
    print(f"[case] linear tile {case} {aligned} {dtype} {out}", flush=True)
    out_type, in_type = getattr(torch, out), getattr(torch, dtype)
    pad = -k % 8 if aligned else (-k % 8) + 1
    _, x = _inside(torch, _whole(torch, 1, m, k, 3), in_type, pad, 0 if aligned else 1)
    _, w = _inside(torch, _whole(torch, 2, n, k, 3).float() / 64, in_type, pad, 0 if aligned else 3)
    bias = (_whole(torch, 3, 1, n, 200)[0].float() / 64).to(in_type)
    residual_buffer, residual = _inside(torch, _whole(torch, 4, m, n, 200).float() / 64, out_type, 5, 1)
    out_buffer, got = _inside(torch, torch.zeros(m, n, device="cuda"), out_type, 3, 2)
    outside, residual_outside = torch.isnan(out_buffer), torch.isnan(residual_buffer)
    exact = x.double() @ w.double().t()                     # in 64 bits: whole numbers over 64
    ws = torch.full((B.bpe_linear_workspace_bytes(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda")
    B.bpe_linear(x, w, got, workspace=ws)
    assert torch.equal(got, exact.float().to(out_type))
    with_bias = exact + bias.double()
    want = (with_bias.clamp(min=0) + residual.double()).float().to(out_type)
    got.fill_(7.0)
    B.bpe_linear(x, w, got, bias=bias, residual=residual, activation="relu", workspace=ws)
    assert torch.equal(got, want)
    act = ("gelu", "gelu_tanh", "silu")[(m + n + k) % 3]
    got.fill_(7.0)
    B.bpe_linear(x, w, got, bias=bias, residual=residual, activation=act, workspace=ws)
    some = torch.arange(0, m * n, max(m * n // 300000, 1), device="cuda")         # (scipy's erfc on the host: a part of the result, edges among it)
    some = torch.unique(torch.cat([some, m * n - 1 - torch.arange(min(n, 4000), device="cuda")]))
    v, units = _exact(with_bias.view(-1)[some].cpu().numpy(), act)
    r = residual.reshape(-1)[some].double().cpu().numpy()
    off = np.abs(got.reshape(-1)[some].double().cpu().numpy() - (v + r))
    assert (off <= units * U * np.abs(v) + 2.0 ** -119 + U * (np.abs(v) + np.abs(r)) + _half_unit(v + r, out)).all(), act
    B.bpe_linear(x, w, residual, bias=bias, residual=residual, activation=act, workspace=ws)           # in place: the same bits
    assert torch.equal(residual, got)
    assert torch.equal(torch.isnan(out_buffer), outside) and torch.equal(torch.isnan(residual_buffer), residual_outside), "written outside the matrix"


@pytest.mark.parametrize("which", ["x", "weight", "out", "residual"])
@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "odd"])
def test_offsets_beyond_32_bits_in_tiles(B, which, aligned):
    """Rows as far apart as the tiles allow, the last of them behind element 2^32."""
    import torch
    far_in = (1 << 21) - (8 if aligned else 7)
    m, n, k = {"x": (2100, 300, 72), "weight": (300, 2100, 72), "out": (140, 600, 72), "residual": (140, 600, 72)}[which]
    assert linear_plan.plan(m, n, k, aligned)[0] not in (linear_plan.ROWS, linear_plan.SIMPLE)
    print(f"[case] linear far {which} {aligned}", flush=True)
    rows = {"x": m, "weight": n, "out": m, "residual": m}[which]
    stride = far_in if which in ("x", "weight") else (1 << 25) - 8
    assert (rows - 1) * stride > 1 << 32
    whole = torch.empty((rows - 1) * stride + 4096, dtype=torch.bfloat16, device="cuda")

    def place(name, values):
        if name != which:
            return _inside(torch, values, torch.bfloat16, 0 if aligned else 1, 0)[1]
        far = torch.as_strided(whole, values.shape, (stride, 1), 0)
        far.copy_(values)
        return far

    x, w = place("x", _whole(torch, 1, m, k, 3)), place("weight", _whole(torch, 2, n, k, 3))
    residual, out = place("residual", _whole(torch, 3, m, n, 100)), place("out", torch.zeros(m, n, device="cuda"))
    ws = torch.empty(B.bpe_linear_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda")
    B.bpe_linear(x, w, out, residual=residual, workspace=ws)
    assert torch.equal(out, (x.double() @ w.double().t() + residual.double()).float().bfloat16())
