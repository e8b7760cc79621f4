"""bpe_top_tokens on rows that one workgroup goes through in several rounds (more rows than are cut into parts, each of more than 8,192
logits), against a sort on the same device; and k above 128 on rows in parts.

lse: as in test_gpu_logits, and a thread's additions one after the other: n_vocab / 256 of them."""
import pytest

from test_gpu_logits import U, _top

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _rows(torch, kind, rows, vocab, k, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab + k)
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    place = torch.arange(vocab, device="cuda", dtype=torch.float32)
    if kind == "rising":
        x = (place * 1e-3).expand(rows, vocab).clone()
    elif kind == "falling":
        x = (-place * 1e-3).expand(rows, vocab).clone()
    elif kind == "mostly equal":
        x = (torch.rand(rows, vocab, generator=g, device="cuda") < 1e-3).float()
    elif kind == "few left":                             # nothing above -infinity but some, in some rows none
        keep = torch.rand(rows, vocab, generator=g, device="cuda") < k / 2 / vocab
        keep[::7] = False
        x = torch.where(keep, x, torch.full_like(x, float("-inf")))
    elif kind == "last ones":                            # the best ones come in the last round
        x[:, -k // 2:] += 40
    elif kind == "steps":                                # every round is above the ones before
        x = x * 0.1 + (place // 8192)
    return x.to(getattr(torch, dtype))


def _check(B, torch, logits, k):
    rows, vocab = logits.shape
    ids, lp, lse = _top(B, torch, logits, k)
    want, order = torch.sort(logits.float(), dim=1, descending=True, stable=True)       # (stable: equal ones by their index)
    want, order = want[:, :k], order[:, :k]
    gone = want == float("-inf")
    assert torch.equal(ids.long(), torch.where(gone, torch.full_like(order, -1), order))
    exact = torch.logsumexp(logits.double(), 1)
    some = torch.isfinite(exact)
    assert torch.equal(lse[~some].double(), exact[~some])
    bound = (600 + vocab / 256) * U + 4 * U * exact[some].abs()
    assert ((lse[some].double() - exact[some]).abs() <= bound).all()
    want_lp = torch.where(gone, torch.full_like(want, float("-inf")).double(), want.double() - exact[:, None])
    fine = torch.isfinite(want_lp)
    assert torch.equal(lp[~fine].double(), want_lp[~fine])
    bound = (600 + vocab / 256) * U + 4 * U * (exact.abs()[:, None] + want_lp.abs())
    assert ((lp.double() - want_lp).abs() <= bound)[fine].all()


KINDS = ["random", "rising", "falling", "mostly equal", "few left", "last ones", "steps"]


@pytest.mark.parametrize("rows,vocab,kind", [(600, 20011, kind) for kind in KINDS] +
                         [(rows, vocab, kind) for rows, vocab in ((1024, 50257), (1030, 8193), (520, 100000)) for kind in ("random", "steps")])
@pytest.mark.parametrize("k", [1, 20, 128, 129, 256])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_in_several_rounds(B, rows, vocab, kind, k, dtype):
    import torch
    print(f"[case] top rounds {rows} {vocab} {k} {kind} {dtype}", flush=True)
    assert B.bpe_top_tokens_workspace_bytes(rows, vocab, k) == 0                 # one part per row
    _check(B, torch, _rows(torch, kind, rows, vocab, k, dtype), k)


@pytest.mark.parametrize("rows,vocab", [(1, 50256), (64, 100256), (9, 300007)])
@pytest.mark.parametrize("k", [64, 128, 129, 200, 256])
@pytest.mark.parametrize("kind", ["random", "rising", "mostly equal", "few left", "last ones"])
@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_many_best_of_rows_in_parts(B, rows, vocab, k, kind, dtype):
    import torch
    print(f"[case] top parts {rows} {vocab} {k} {kind} {dtype}", flush=True)
    assert B.bpe_top_tokens_workspace_bytes(rows, vocab, k) > 0
    _check(B, torch, _rows(torch, kind, rows, vocab, k, dtype), k)


@pytest.mark.parametrize("k", [1, 40, 256])
def test_nan_in_some_rounds(B, k):
    """NaN ranks above everything, by index, wherever its rounds are; the row's statistics are NaN, other rows' are not."""
    import torch
    rows, vocab = 600, 30000
    x = torch.randn(rows, vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k))
    place = torch.arange(vocab, device="cuda")
    x[0] = float("nan")
    x[1, 29000::3] = float("nan")                        # more than k, in the last round
    x[2, 9000] = x[2, 100] = float("nan")
    x[3, 8192:16384] = float("nan")
    x[4, 5] = float("inf")
    x[4, 29999] = float("nan")
    assert B.bpe_top_tokens_workspace_bytes(rows, vocab, k) == 0
    ids, lp, lse = _top(B, torch, x, k)
    for r in range(5):
        nan = torch.isnan(x[r])
        first = place[nan]
        rest = torch.argsort(torch.where(nan, torch.full_like(x[r], float("-inf")), x[r]), descending=True, stable=True)
        want = torch.cat([first, rest])[:k]
        assert torch.equal(ids[r].long(), want), r
        assert torch.isnan(lse[r]) and torch.isnan(lp[r]).all()
    assert torch.isfinite(lse[5:]).all() and torch.isfinite(lp[5:]).all()
    _, order = torch.sort(x[5:], dim=1, descending=True, stable=True)
    assert torch.equal(ids[5:].long(), order[:, :k])
