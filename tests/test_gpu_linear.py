"""bpe_linear against the formula in 64 bits.

Tolerance of an element, from the arithmetic alone: a sum of k products in 32 bits, in whatever order, is off by at most
about k 2^-24 times the sum of the products' absolute values S (twice that is allowed, and 16 terms more for bias and
residual); the activations have a slope of at most 1.13 and functions good to a few units in the last place (4e-6 of the
value); the result is rounded once to its type (half a unit: 2^-24, 2^-11, 2^-8 of the value, which is 2^-9 for bf16 and
is doubled here, and 2^-25 below the smallest normal f16)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _act(v, name):
    if name == "relu":
        return np.where(v > 0, v, 0.0)
    if name == "gelu":
        from scipy.special import erf
        return 0.5 * v * (1 + erf(v / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + np.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1 + np.exp(-v))
    return v


def _half_unit(v, out):
    return {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[out] * np.abs(v) + (2.0 ** -25 if out == "float16" else 0.0)


def _check(got, x, w, bias, residual, act, out):
    x, w = x.double().cpu().numpy(), w.double().cpu().numpy()
    v, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        b = bias.double().cpu().numpy()
        v, size = v + b, size + np.abs(b)
    tol = 1.13 * 2 * (x.shape[1] + 16) * 2.0 ** -24 * size
    v = _act(v, act)
    tol += 4e-6 * np.abs(v)
    if residual is not None:
        r = residual.double().cpu().numpy()
        tol += 2.0 ** -24 * (np.abs(v) + np.abs(r))
        v = v + r
    tol += _half_unit(v, out)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - v) - tol) if v.size else -1.0
    assert worst <= 0, (worst, float(np.max(np.abs(got - v))))


def _rand(torch, seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _call(B, torch, x, w, out, **kw):
    m, k = x.shape
    n = w.shape[0]
    ws = torch.full((B.bpe_linear_workspace_bytes(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda")
    B.bpe_linear(x, w, out, workspace=ws, **kw)
    return out


SHAPES = [(1, 1, 1), (1, 17, 5), (2, 33, 8), (3, 1256, 64), (5, 100, 100), (15, 48, 129), (16, 16, 32), (17, 31, 33), (1, 2048, 1024), (33, 1000, 512),
          (47, 513, 2048), (64, 128, 256), (64, 4099, 96), (65, 130, 96), (100, 257, 1031), (127, 255, 200), (128, 128, 128), (129, 64, 40), (200, 1256, 512),
          (256, 256, 64), (257, 513, 264), (300, 77, 4096), (513, 1031, 72), (700, 1300, 128), (1031, 300, 520)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,out", [("bfloat16", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16")])
def test_sizes(B, shape, dtype, out):
    import torch
    m, n, k = shape
    print(f"[case] linear {shape} {dtype} {out}", flush=True)
    x = _rand(torch, 1, m, k, dtype=getattr(torch, dtype))
    w = _rand(torch, 2, n, k, dtype=getattr(torch, dtype))
    got = torch.full((m, n), float("nan"), dtype=getattr(torch, out), device="cuda")
    _call(B, torch, x, w, got)
    _check(got, x, w, None, None, "none", out)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("shape", [(3, 70, 48), (50, 512, 256), (140, 300, 96)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,out,bias_dtype", [("bfloat16", "float32", "float32"), ("float16", "float16", "float16"), ("bfloat16", "bfloat16", "bfloat16"),
                                                  ("float16", "float32", "bfloat16")])
def test_epilogue(B, act, shape, dtype, out, bias_dtype):
    import torch
    m, n, k = shape
    x = _rand(torch, 3, m, k, dtype=getattr(torch, dtype))
    w = (_rand(torch, 4, n, k, dtype=torch.float32) * k ** -0.5 * 3).to(getattr(torch, dtype))
    bias = _rand(torch, 5, n, dtype=getattr(torch, bias_dtype))
    res = _rand(torch, 6, m, n, dtype=getattr(torch, out))
    got = torch.full((m, n), float("nan"), dtype=getattr(torch, out), device="cuda")
    _call(B, torch, x, w, got, bias=bias, residual=res, activation=act)
    _check(got, x, w, bias, res, act, out)
    # in place, and the same bits
    both = res.clone()
    _call(B, torch, x, w, both, bias=bias, residual=both, activation=act)
    assert torch.equal(both, got)


def test_activations_of_large_values(B):
    """Arguments at which exp and tanh run out of their range: no NaN, the limits of the formulas."""
    import torch
    x = torch.tensor([[1.0]], dtype=torch.bfloat16, device="cuda").expand(1, 8).contiguous()
    values = torch.tensor([-1e30, -1e4, -200.0, -100.0, -30.0, 0.0, 30.0, 1e4, 1e30], device="cuda")
    w = torch.zeros(9, 8, dtype=torch.bfloat16, device="cuda")
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        out = torch.empty(1, 9, device="cuda")
        _call(B, torch, x, w, out, bias=values, activation=act)
        got = out.cpu().numpy()[0]
        want = np.where(values.cpu().numpy() >= 30, values.cpu().numpy(), 0.0)
        assert np.abs(got - want).max() <= 1e-6 * 1e30 and np.isfinite(got).all()
        assert np.abs(got[2:8] - want[2:8]).max() <= 1e-2 + 4e-6 * 1e4, (act, got)


@pytest.mark.parametrize("m", [1, 16, 40, 64, 65, 150, 400])
@pytest.mark.parametrize("k,offset,pad", [(64, 0, 8), (64, 1, 0), (96, 4, 4), (100, 3, 7), (257, 5, 2), (30, 2, 1)])
def test_strides_and_alignment(B, m, k, offset, pad):
    """Rows inside larger buffers that hold NaN everywhere else, at every alignment that the type allows."""
    import torch
    n = 150

    def inside(seed, rows, cols, dtype):
        t = torch.full((rows * (cols + pad) + offset + 64,), float("nan"), dtype=dtype, device="cuda")
        view = t[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        view.copy_(_rand(torch, seed, rows, cols, dtype=dtype))
        return t, view

    for dtype, out in ((torch.bfloat16, torch.float32), (torch.float16, torch.float16)):
        _, x = inside(7, m, k, dtype)
        _, w = inside(8, n, k, dtype)
        whole, got = inside(9, m, n, out)
        got.zero_()
        res_whole, res = inside(10, m, n, out)
        bias = _rand(torch, 11, n + 1, dtype=dtype)[1:]
        mark = torch.isnan(whole)
        _call(B, torch, x, w, got, bias=bias, residual=res)
        _check(got, x, w, bias, res, "none", str(out).replace("torch.", ""))
        assert torch.equal(torch.isnan(whole), mark), "written outside the matrix"


def test_nan_and_infinity_stay_in_their_rows(B):
    import torch
    for m, n, k in ((5, 100, 72), (90, 100, 72)):
        x, w = _rand(torch, 1, m, k, dtype=torch.bfloat16), _rand(torch, 2, n, k, dtype=torch.bfloat16)
        x[m - 1, 3] = float("nan")
        x[m - 2, 0] = float("inf")
        w[7, k - 1] = float("nan")
        out = torch.empty(m, n, device="cuda")
        _call(B, torch, x, w, out)
        got = out.cpu().numpy()
        assert np.isnan(got[m - 1]).all() and np.isnan(got[:, 7]).all()
        rest = np.delete(got[:m - 2], 7, axis=1)
        assert np.isfinite(rest).all()
        assert not np.isfinite(got[m - 2]).any()


@pytest.mark.parametrize("m,n", [(0, 5), (5, 0), (3, 7), (70, 90)])
def test_empty_sizes(B, m, n):
    import torch
    x, w = torch.empty(m, 0, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((m, n), 7.0, device="cuda")
    bias = torch.arange(n, dtype=torch.float32, device="cuda")
    B.bpe_linear(x, w, out, bias=bias, activation="relu")
    assert torch.equal(out, bias[None].expand(m, n))


@pytest.mark.parametrize("m", [2, 70])
def test_offsets_beyond_32_bits(B, m):
    """The last row of out, of the residual and of x starts behind element 2^32."""
    import torch
    n, k = 64, 64
    stride = (1 << 32) // (m - 1) + 8
    whole = torch.empty((m - 1) * stride + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(whole, (m, k), (stride, 1), 0)
    out = torch.as_strided(whole, (m, n), (stride, 1), 1024)
    res = torch.as_strided(whole, (m, n), (stride, 1), 2048)
    x.copy_(_rand(torch, 1, m, k, dtype=torch.bfloat16))
    res.copy_(_rand(torch, 2, m, n, dtype=torch.bfloat16))
    w = _rand(torch, 3, n, k, dtype=torch.bfloat16)
    _call(B, torch, x, w, out, residual=res)
    _check(out, x, w, None, res, "none", "bfloat16")


def test_same_bits_again_on_another_stream_and_in_a_graph(B):
    import torch
    for m, n, k in ((9, 700, 640), (90, 300, 2000), (300, 300, 300)):
        x, w = _rand(torch, 1, m, k, dtype=torch.bfloat16), _rand(torch, 2, n, k, dtype=torch.bfloat16)
        ws = torch.empty(B.bpe_linear_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda")
        outs = [torch.zeros(m, n, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        B.bpe_linear(x, w, outs[0], workspace=ws)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        B.bpe_linear(x, w, outs[1], workspace=ws, stream=side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.bpe_linear(x, w, outs[2], workspace=ws)
        for _ in range(3):
            outs[2].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], outs[2])
        assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("k", [1, 7, 8, 9, 15, 57, 63, 65, 71, 72, 100, 127, 129, 184, 197, 263, 321])
@pytest.mark.parametrize("stride", ["rows of sixteen bytes", "rows next to each other"])
def test_rows_that_end_inside_a_block(B, k, stride):
    """Every way for k to end inside 64 columns, few blocks and many, NaN right behind a row, on tiles of every size."""
    import torch
    for m, n in ((3, 900), (30, 2000), (60, 5000), (130, 20000), (500, 700), (1100, 9000)):
        print(f"[case] linear cut {m} {n} {k} {stride}", flush=True)
        pad = -k % 8 if stride == "rows of sixteen bytes" else 0

        def inside(seed, rows):
            t = torch.full((rows * (k + pad) + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
            view = t[:rows * (k + pad)].view(rows, k + pad)[:, :k]
            view.copy_(_rand(torch, seed, rows, k, dtype=torch.bfloat16))
            return view

        x, w = inside(1, m), inside(2, n)
        got = torch.full((m, n), float("nan"), device="cuda")
        _call(B, torch, x, w, got)
        _check(got, x, w, None, None, "none", "float32")


def test_activations_of_infinity_and_nan(B):
    """Their limits at both ends, which all four have; NaN stays NaN."""
    import torch
    x, w = torch.zeros(40, 16, dtype=torch.float16, device="cuda"), torch.zeros(70, 16, dtype=torch.float16, device="cuda")
    bias = torch.zeros(70, device="cuda")
    bias[3], bias[4], bias[5] = float("inf"), float("-inf"), float("nan")
    bias[69] = float("-inf")
    for m in (1, 40):
        for act in ("relu", "gelu", "gelu_tanh", "silu"):
            out = torch.empty(m, 70, device="cuda")
            _call(B, torch, x[:m], w, out, bias=bias, activation=act)
            got = out.cpu().numpy()
            assert np.isposinf(got[:, 3]).all() and (got[:, 4] == 0).all() and np.isnan(got[:, 5]).all(), act
            assert (np.delete(got, [3, 5], axis=1) == 0).all(), act


def test_activations_over_their_range(B):
    """Of 40,000 values from -30 to 30: the sum is exact here, so the tolerance is the functions' and the rounding alone (the cut
    series for gelu is good to 1.5e-7 / 2 of the argument)."""
    import torch
    n = 40000
    x, w = torch.zeros(2, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    bias = torch.linspace(-30, 30, n, device="cuda")
    v = bias.double().cpu().numpy()
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        out = torch.empty(2, n, device="cuda")
        _call(B, torch, x, w, out, bias=bias, activation=act)
        want = _act(v, act)
        tol = 4e-6 * np.abs(want) + 2.0 ** -24 * np.abs(want) + (0.75e-7 + 2 * 2.0 ** -24) * np.abs(v)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all(), act


@pytest.mark.parametrize("which", ["out", "residual", "both"])
def test_far_rows_of_the_result(B, which):
    """Rows of out or of the residual 2^25 elements apart and more, of x and weight next to each other."""
    import torch
    m, n, k = 20, 600, 64
    stride = (1 << 25) + 8
    x, w = _rand(torch, 1, m, k, dtype=torch.bfloat16), _rand(torch, 2, n, k, dtype=torch.bfloat16)
    whole = torch.empty((m - 1) * stride + 4096, dtype=torch.bfloat16, device="cuda")
    near = _rand(torch, 3, m, n, dtype=torch.bfloat16)
    far = torch.as_strided(whole, (m, n), (stride, 1), 0)
    out = torch.as_strided(whole, (m, n), (stride, 1), 1024) if which != "residual" else torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    far.copy_(near)
    _call(B, torch, x, w, out, residual=near if which == "out" else far)
    _check(out, x, w, None, near, "none", "bfloat16")
