"""bpe_linear_mx with the smallest and the largest weights that the format holds.

Tolerances as in test_gpu_linear_mx; a product or sum below 2^-126 may leave nothing, so 2 (k + 1) times that is allowed besides.  For x in 16 bits weights
are 16 bits too: those above the largest number (2^128 and more: codes of 2 and above with the scale byte 254, of 4 and above with 253) are infinities."""
import numpy as np
import pytest

import linear_mx_plan as P
import mx4_reference as R
from test_gpu_linear_mx import B, KINDS, _call, torch  # noqa: F401

pytestmark = pytest.mark.gpu
# f16 through every kernel: of few columns, of few rows (by 128 and by 256 columns), in tiles; whole ones and others
SIZES = [(5, 40, 7), (1, 33, 300), (3, 96, 512), (60, 300, 544), (100, 96, 512), (300, 1300, 320), (45, 16388, 16), (4576, 1598, 17)]


def _weights(B, torch, codes, scales):  # noqa: F811
    return B.Mx4(*codes.shape, torch.from_numpy(R.pack(codes, scales)).cuda())


def _close(got, x, w):
    got, k = got.double().cpu().numpy(), x.shape[1]
    tol = 2 * (k + 16) * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T) + 2 * (k + 1) * 2.0 ** -126
    assert np.isfinite(got).all()
    assert (np.abs(got - x @ w.T) <= tol).all(), np.max(np.abs(got - x @ w.T) - tol)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("low,high", [(0, 4), (0, 30), (226, 252), (249, 252)])
def test_first_and_last_scales(B, torch, kind, m, n, k, low, high):  # noqa: F811
    """Rows of weights of one size each, x of a size that makes results of ordinary size, or as near to it as f16 comes."""
    rng = np.random.default_rng(m + low)
    codes, scales = rng.integers(0, 16, (n, k), dtype=np.uint8), np.repeat(rng.integers(low, high + 1, (n, 1)), (k + 31) // 32, 1).astype(np.uint8)
    w, wv = _weights(B, torch, codes, scales), R.values(codes, scales)
    if kind == "mx4":
        xc, xs = R.random(rng, m, k, center=220 if low == 0 else 40)
        x, xv = _weights(B, torch, xc, xs), R.values(xc, xs)
    else:
        size = {"bfloat16": 100, "float16": 13}[kind] if low == 0 else {"bfloat16": -100, "float16": -13}[kind]
        x = torch.from_numpy(rng.standard_normal((m, k)) * 2.0 ** size).to(getattr(torch, kind)).cuda()
        xv = x.double().cpu().numpy()
    got = torch.empty(m, n, device="cuda")
    _call(B, torch, x, w, got)
    _close(got, xv, wv)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("kind", ("bfloat16", "float16"))
def test_subnormal_x(B, torch, kind, m, n, k):  # noqa: F811
    rng = np.random.default_rng(m)
    x = torch.from_numpy(rng.standard_normal((m, k)) * (2.0 ** -129 if kind == "bfloat16" else 2.0 ** -18)).to(getattr(torch, kind)).cuda()
    assert (x.abs() < torch.finfo(x.dtype).smallest_normal).float().mean() > 0.9
    codes, scales = R.random(rng, n, k, center=220)
    got = torch.empty(m, n, device="cuda")
    _call(B, torch, x, _weights(B, torch, codes, scales), got)
    _close(got, x.double().cpu().numpy(), R.values(codes, scales))


@pytest.mark.parametrize("aligned", (True, False))
@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("kind", ("bfloat16", "float16"))
def test_weights_that_are_infinities(B, torch, kind, m, n, k, aligned):  # noqa: F811
    """One in some rows of weight, times x of any sign and of as many bits as the type has: an infinity of the product's sign."""
    rng = np.random.default_rng(k)
    codes, scales = R.random(rng, n, k)
    rows = rng.choice(n, n // 2, replace=False)
    place = rng.integers(0, k, n)
    for j in rows:
        of_block = slice(place[j] // 32 * 32, place[j] // 32 * 32 + 32)
        codes[j, of_block] = 0                             # the others of the block
        top = rng.integers(0, 2)
        scales[j, place[j] // 32] = (253, 254)[top]
        codes[j, place[j]] = 8 * rng.integers(0, 2) + rng.integers((6, 4)[top], 8)
    w32 = R.values(codes, scales)
    w32[np.abs(w32) >= 2.0 ** 128] *= np.inf
    assert np.isinf(w32).sum() == len(rows)
    # (1 and 3 fit 8 bits, the others of f16 do not; the largest one is rounded up by a conversion to 8 bits)
    many = [1.0, -3.0, 1 + 2.0 ** -7, -1.9921875] if kind == "bfloat16" else [1.0, -3.0, 1 + 2.0 ** -10, -1 - 2.0 ** -8, 2047.0, -65504.0, 65504.0, 2.0 ** -24, -65280.0]
    whole = torch.full((m, k + 8 + (-k) % 8 if aligned else k + 3), float("nan"), dtype=getattr(torch, kind), device="cuda")
    x = whole[:, :k] if aligned else whole[:, 1:1 + k]
    values = rng.choice([v for v in many if abs(v) < 4], (m, k))
    for j in rows:
        values[:, place[j]] = rng.choice(many, m)
    x.copy_(torch.from_numpy(values))
    assert np.array_equal(x.double().cpu().numpy(), values)
    got = torch.empty(m, n, device="cuda")
    _call(B, torch, x, _weights(B, torch, codes, scales), got)
    got = got.cpu().numpy()
    for j in rows:
        want = np.sign(values[:, place[j]]) * w32[j, place[j]]
        assert np.array_equal(got[:, j], want.astype(np.float32)), (j, got[:, j][got[:, j] != want][:3])
    assert np.isfinite(np.delete(got, rows, 1)).all()


@pytest.mark.parametrize("m,n,k", [(3, 96, 512), (100, 96, 512), (300, 1300, 320)])
def test_four_bits_by_four_bits_have_no_such_end(B, torch, m, n, k):  # noqa: F811
    """Both operands keep their scales: 2^127 by 2^-100 is what it is."""
    rng = np.random.default_rng(n)
    codes, scales = rng.integers(0, 16, (n, k), dtype=np.uint8), rng.integers(253, 255, (n, (k + 31) // 32)).astype(np.uint8)
    xc, xs = R.random(rng, m, k, center=30)
    got = torch.empty(m, n, device="cuda")
    _call(B, torch, _weights(B, torch, xc, xs), _weights(B, torch, codes, scales), got)
    _close(got, R.values(xc, xs), R.values(codes, scales))


def test_sizes_take_the_kernels_that_they_are_here_for():
    tiles = {P.plan(m, n, k, "f16")[0] for m, n, k in SIZES if k >= 8}
    assert {1, 3, 4} <= tiles, tiles
