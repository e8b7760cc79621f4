"""bpe_linear with more columns than one launch of fewer than 2^32 threads makes, for a few rows.  Small whole numbers, so
that sums are exact in whatever order."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


@pytest.mark.parametrize("m,n,k", [(1, (1 << 28) + 5, 8), (3, (1 << 28) - 15, 16), (1, (1 << 28) - 16, 8), (5, (1 << 28) + 1, 0), (1, (1 << 30) - 1, 0)])
def test_columns_beyond_a_launch(B, m, n, k):
    import torch
    print(f"[case] linear columns {m} {n} {k}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(n)
    w = torch.randint(-3, 4, (n, k), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    x = torch.randint(-3, 4, (m, k), generator=g, device="cuda").bfloat16()
    bias = torch.randint(-9, 10, (n,), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    out = torch.randint(-9, 10, (m, n), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    before = out.clone()
    assert B.bpe_linear_workspace_bytes(m, n, k) == 0
    B.bpe_linear(x, w, out, bias=bias, residual=out, activation="relu")          # in place
    step = 1 << 25
    for a in range(0, n, step):
        b = min(a + step, n)
        for i in range(m):
            want = (w[a:b].float() * x[i].float()).sum(1) + bias[a:b].float()
            want = (want.clamp(min=0) + before[i, a:b].float()).bfloat16()
            assert torch.equal(out[i, a:b], want), (i, a)
