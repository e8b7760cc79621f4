"""A mask index without a table of masks is refused, not read as `no masks`: no GPU is needed."""
from test_answer_refusals import P, _adjust, lib  # noqa: F401


def test_an_index_without_masks(lib):  # noqa: F811
    for n_masks in (0, 4):
        assert _adjust(lib, rules=dict(mask_index=P, n_masks=n_masks, mask_stride=4)) == -1
        assert b"mask_index" in lib.bpe_last_error()
