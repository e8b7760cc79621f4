"""bpe_norm at widths that are no multiple of eight: what a thread holds behind a row's end is no part of a mean.  Tolerances as in test_gpu_norm."""
import numpy as np
import pytest

from test_gpu_norm import B, _close, _reference, torch  # noqa: F401

pytestmark = pytest.mark.gpu
WIDTHS = (2, 7, 33, 100, 1001, 4100, 8195, 16383)


@pytest.mark.parametrize("bias", (False, True))
@pytest.mark.parametrize("residual", (False, True))
@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("layer", "rms"), ("rms", "layer"), ("none", "layer"), ("layer", "none")])
@pytest.mark.parametrize("width", WIDTHS)
def test_norms_without_weights(B, torch, width, post, pre, residual, bias):  # noqa: F811
    rng = np.random.default_rng(width)
    rows = 5
    t = lambda a: torch.from_numpy(a).float().cuda()
    d = lambda a: None if a is None else a.double().cpu().numpy()
    y = t(rng.standard_normal((rows, width)) * 3 + np.array([0, 3, -30, 30, 1])[:, None])
    h = t(rng.standard_normal((rows, width)) + 1) if residual else None
    pb = t(rng.standard_normal(width)) if bias and post != "none" else None
    b = t(rng.standard_normal(width)) if bias and pre != "none" else None
    total, out = torch.empty_like(y), torch.empty_like(y)
    B.bpe_norm(y, out, post=post, post_bias=pb, residual=h, total=total, residual_scale=0.75, branch_scale=0.5, pre=pre, pre_bias=b, eps=1e-3)
    v, tol, o, o_tol = _reference(d(y), post, 1e-3, None, d(pb), None, "none", d(h), 0.75, 0.5, pre, 1e-3, None, d(b))
    _close(total, v, tol)
    _close(out, o, o_tol)


def test_a_row_of_one_element(B, torch):  # noqa: F811
    """An element is its own mean, and x * 1 is x: what a layer norm leaves is 0, and then its bias, exactly."""
    y = torch.tensor([[3.0], [-2.5e10], [1e-30], [0.0]], device="cuda")
    h = torch.tensor([[1.0], [2.0], [-3.0], [0.5]], device="cuda")
    w, pb, b = (torch.tensor([v], device="cuda") for v in (1.5, 0.25, -0.75))
    total, out = torch.empty_like(y), torch.empty_like(y)
    B.bpe_norm(y, out, post="layer", post_weight=w, post_bias=pb, residual=h, total=total, residual_scale=2.0, branch_scale=4.0, pre="layer", pre_weight=w, pre_bias=b)
    assert torch.equal(total, 2 * h + 1) and (out == -0.75).all()
    B.bpe_norm(y, out, post="layer", residual=h, total=total, pre="layer")
    assert torch.equal(total, h) and (out == 0).all()


def test_squares_beyond_32_bits(B, torch):  # noqa: F811
    """A sum of squares that passes the largest float leaves the bias, and the total is what it is."""
    y = torch.full((3, 300), 1e25, device="cuda")
    y[1] = 2.0
    b = torch.randn(300, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    total, out = torch.empty_like(y), torch.empty_like(y)
    B.bpe_norm(y, out, total=total, pre="rms", pre_bias=b, eps=0.0)
    assert torch.equal(total, y) and torch.equal(out[[0, 2]], b.expand(2, 300))
    assert (out[1] - (1 + b)).abs().max() <= 4 * 2.0 ** -24 * (1 + b.abs().max())
