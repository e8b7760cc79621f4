"""The activations of bpe_linear against their formulas in 64 bits, relative to their value: small results count too.

The sums are exact here, so what is left is the functions' arithmetic, in units u = 2^-24 (a rounding is at most one, the hardware's 2^x
and reciprocal at most two):
  silu, v / (1 + e), e = exp(-v): the exponent v log2 e rounded and its constant 1.25 |v|, 2^x 2, the sum 1, the reciprocal 2, the product 1
  gelu by tanh, v / (1 + exp(-x)): four roundings and constants in the exponent, so 5 x, and the same 6
  gelu, max(v, 0) - |v| q: the series 4, its argument t good to 3 and q's slope in it at most 2.7, so 8, its terms 4, 2^x 2, the
  products 2; the exponent v^2 / 2 twice rounded and its constant 1.7 v^2
Where 2^x or the reciprocal fall below the smallest normal number, a factor of |v| < 128 of that may be lost: 2^-119."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _exact(v, act):
    """(value, error allowed in units of 2^-24 of it)"""
    from scipy.special import erfc
    if act == "gelu":
        return 0.5 * v * erfc(-v / np.sqrt(2.0)), 20 + 2 * v * v
    x = v if act == "silu" else 2 * np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-x)), 6 + 6 * np.abs(x)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("m", [2, 40])
def test_relative_to_the_value(B, act, m):
    import torch
    rng = np.random.default_rng(1)
    near = rng.choice([-1.0, 1.0], 20000) * 10.0 ** rng.uniform(-30, 0, 20000)
    v = np.concatenate([np.linspace(-13, 13, 60001), near, np.linspace(-100, 100, 20001), [0.0]]).astype(np.float32)
    n = v.size
    x, w = torch.zeros(m, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(m, n, device="cuda")
    ws = torch.empty(B.bpe_linear_workspace_bytes(m, n, 8), dtype=torch.uint8, device="cuda")
    B.bpe_linear(x, w, out, bias=torch.from_numpy(v).cuda(), activation=act, workspace=ws)
    v = v.astype(np.float64)
    want, units = _exact(v, act)
    off = np.abs(out.double().cpu().numpy() - want)
    allowed = units * U * np.abs(want) + 2.0 ** -119
    bad = np.argwhere(~(off <= allowed))
    assert bad.size == 0, (act, len(bad), v[bad[0, 1]], off[tuple(bad[0])], want[bad[0, 1]])


def test_gelu_on_ordinary_arguments(B):
    """Not worse on average than the formula with erf rounded to 32 bits: rms of 2.5e-8 on normal arguments, 3.4e-8 on -6 .. -2."""
    import torch
    rng = np.random.default_rng(2)
    for v, most in ((rng.standard_normal(200000), 2.5e-8), (rng.uniform(-6, -2, 200000), 3.4e-8)):
        v = v.astype(np.float32)
        x, w = torch.zeros(1, 8, dtype=torch.float16, device="cuda"), torch.zeros(v.size, 8, dtype=torch.float16, device="cuda")
        out = torch.empty(1, v.size, device="cuda")
        B.bpe_linear(x, w, out, bias=torch.from_numpy(v).cuda(), activation="gelu")
        off = out[0].double().cpu().numpy() - _exact(v.astype(np.float64), "gelu")[0]
        assert np.sqrt((off * off).mean()) <= most
