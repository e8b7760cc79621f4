"""bpe_sample_tokens at logits that stand on the border of a bin of logits.

With filters the library counts a row's logits in bins, whole parts of x * scale, and looks for those of a bin again.  Taken here are the logits whose
product with the scale lies just below a whole number and becomes that number when it is rounded to 32 bits: every place that
computes the product has to round it, or one counts a logit that another does not find.  300 such values at temperatures in steps of 0.01 (bf16, which
has fewer: 0.001), all of them where there are no more; as the best logit, and as the one that a border falls on, with equal ones.  Ids and shares against the definition in 64 bits, as in
test_gpu_sample."""
import numpy as np
import pytest

from test_gpu_sample import B, TYPES, _check, torch  # noqa: F401

pytestmark = pytest.mark.gpu
N = 8 * 1024 + 61                                          # two parts of a row


def _scale(t):
    return np.float32(min(8 * (1.4426950408889634074 / float(t)), 1e30))


def _on_borders(dtype, near_zero):
    """(temperature, logit) of float32, up to 100 in size or above."""
    if dtype == "float16":
        x = np.arange(1, 0x7C00, dtype=np.uint16).view(np.float16).astype(np.float32)
    elif dtype == "bfloat16":
        x = (np.arange(1, 0x7F80, dtype=np.uint32) << 16).view(np.float32)
    else:
        x = np.random.default_rng(1).uniform(0.1, 100 if near_zero else 100000, 60000).astype(np.float32)
    x = np.concatenate([x, -x])
    x = x[(np.abs(x) >= 2.0 ** -6) & ((np.abs(x) < 100) == near_zero)]
    found = []
    steps = 1000 if dtype == "bfloat16" else 100
    for i in range(1, 2 * steps + 1):
        t = np.float32(i / steps)
        product = x.astype(np.float64) * np.float64(_scale(t))          # exact: at most 48 bits
        with np.errstate(over="ignore"):
            rounded = product.astype(np.float32)
        found += [(t, v) for v in x[(product < rounded) & (rounded == np.floor(rounded)) & (np.abs(rounded) < 4e6)]]
    rng = np.random.default_rng(2)
    if len(found) > 300:
        found = [found[i] for i in rng.choice(len(found), 300, replace=False)]
    return np.array([t for t, _ in found], dtype=np.float32), np.array([v for _, v in found], dtype=np.float32)


def test_there_are_such_logits():
    for dtype in TYPES:
        for near_zero in (True, False):
            assert len(_on_borders(dtype, near_zero)[0]) >= 20, (dtype, near_zero)
    t, x = _on_borders("float16", True)
    assert any(a == np.float32(0.33) and b == np.float32(12.5234375) for a, b in zip(t, x))      # 437.999994 becomes 438


def _rows(dtype, torch, values):  # noqa: F811
    """Rows of the type's lowest value, and what makes a tensor of them."""
    x = np.full((len(values), N), -3e38 if dtype != "float16" else -65504.0)
    return x, lambda: torch.from_numpy(x).to(getattr(torch, dtype)).cuda()


@pytest.mark.parametrize("near_zero", (True, False))
@pytest.mark.parametrize("dtype", TYPES)
def test_the_best_token_alone_in_its_bin(B, torch, dtype, near_zero):  # noqa: F811
    t, values = _on_borders(dtype, near_zero)
    rng = np.random.default_rng(3)
    rows = len(values)
    x, given = _rows(dtype, torch, values)
    at = rng.integers(0, N, rows)
    x[np.arange(rows), at] = values
    logits, u = given(), rng.random(rows)
    for kw in (dict(top_k=np.ones(rows)), dict(top_k=np.full(rows, 700)), dict(top_k=np.full(rows, 1200)), dict(top_p=np.full(rows, 0.5)), dict(min_p=np.full(rows, 0.5)),
               dict(top_k=np.full(rows, 3), top_p=np.full(rows, 0.7), min_p=np.full(rows, 0.1)), dict(top_p=np.full(rows, 0.9), min_p=np.full(rows, 1.0))):
        assert np.array_equal(_check(B, torch, logits, u, t, **kw), at)


@pytest.mark.parametrize("near_zero", (True, False))
@pytest.mark.parametrize("dtype", TYPES)
def test_a_border_among_equal_logits(B, torch, dtype, near_zero):  # noqa: F811
    """Three better tokens some bins above, 1,400 of the value, as many some bins below."""
    t, values = _on_borders(dtype, near_zero)
    rng = np.random.default_rng(4)
    keep = rng.choice(len(values), min(len(values), 60), replace=False)
    t, values = t[keep], values[keep]
    rows = len(values)
    x, given = _rows(dtype, torch, values)
    to_type = lambda v: torch.tensor(float(v), dtype=torch.float64).to(getattr(torch, dtype)).double().item()
    for r in range(rows):
        step = 12.0 / float(_scale(t[r]))
        above, below = to_type(values[r] + step), to_type(values[r] - step)
        grow = 1.0
        while above == values[r] or below == values[r]:                  # (fewer bits than the step has)
            grow *= 2
            above, below = to_type(values[r] + grow * step), to_type(values[r] - grow * step)
        places = rng.permutation(N)
        x[r, places[:3]], x[r, places[3:1403]], x[r, places[1403:2803]] = above, values[r], below
    logits, u = given(), rng.random(rows)
    k = lambda low, high: rng.integers(low, high, rows)
    ratio = np.exp((values.astype(np.float64) - logits.double().cpu().numpy().max(1)) / t)
    for kw in (dict(top_k=k(4, 1000)), dict(top_k=k(1030, 1400)), dict(top_p=rng.uniform(0.1, 0.9, rows)), dict(min_p=np.minimum(ratio * 0.99, 1)), dict(min_p=ratio * 1.01),
               dict(top_k=k(4, 1000), top_p=rng.uniform(0.1, 0.9, rows), min_p=ratio * 0.5), dict(top_k=k(1030, 2800), top_p=rng.uniform(0.1, 0.9, rows), min_p=ratio * 0.5)):
        _check(B, torch, logits, u, t, **kw)
