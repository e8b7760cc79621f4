"""bpe_adjust_logits with tables of few masks, down to none: a mask index that is too large allows no token, a negative one all."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


@pytest.mark.parametrize("n_masks", [0, 1, 2])
@pytest.mark.parametrize("lists", [False, True])
def test_tables_of_few_masks(B, n_masks, lists):
    import torch
    vocab = 70
    index = torch.tensor([0, -1, 1, 5, -7, 2**31 - 1], dtype=torch.int32, device="cuda")
    logits = torch.randn(6, vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    masks = torch.full((n_masks, 3), -1, dtype=torch.int32, device="cuda")
    kw = {}
    if lists:                                              # a bias of 0 for one token: the other form of the kernel, and its way for such tokens
        kw = dict(bias_ids=torch.full((6,), 9, dtype=torch.int32, device="cuda"), bias_values=torch.zeros(6, device="cuda"),
                  bias_offsets=torch.arange(7, dtype=torch.int32, device="cuda"))
    out = torch.empty_like(logits)
    B.bpe_adjust_logits(logits, out, masks=masks, mask_index=index, **kw)
    for r, i in enumerate(index.tolist()):
        want = logits[r] if i < n_masks else torch.full_like(logits[r], float("-inf"))
        assert torch.equal(out[r], want), (r, i)


@pytest.mark.parametrize("n_masks", [0, 1, 5])
def test_too_few_masks_for_the_rows_are_refused(B, n_masks):
    import torch
    logits, masks = torch.zeros(6, 70, device="cuda"), torch.full((n_masks, 3), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(B.BpeError) as e:
        B.bpe_adjust_logits(logits, torch.empty_like(logits), masks=masks)
    assert e.value.code == -2
    B.bpe_adjust_logits(logits[:0], torch.empty_like(logits[:0]), masks=masks)             # no rows need none


def test_no_masks_are_no_table(B):
    import torch
    logits = torch.zeros(6, 70, device="cuda")
    out = torch.ones_like(logits)
    B.bpe_adjust_logits(logits, out)
    assert torch.equal(out, logits)
    with pytest.raises(ValueError):
        B.bpe_adjust_logits(logits, out, mask_index=torch.zeros(6, dtype=torch.int32, device="cuda"))
