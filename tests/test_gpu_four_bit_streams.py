"""The product with 4-bit weights and drawn tokens on two streams at once, every call with inputs and outputs of its own: a call that leaves
something unwritten, or takes another's, shows."""
import pytest

from test_gpu_answers import example  # noqa: F401
from test_gpu_four_bit_answers import _answerer

pytestmark = pytest.mark.gpu


def test_every_call_writes_its_own(example):  # noqa: F811
    import torch
    B, calls, rows = example.B, 12, 21
    streams, sides = [torch.cuda.Stream() for _ in range(2)], [_answerer(example, seed) for seed in (7, 8)]
    generator = torch.Generator(device="cuda").manual_seed(1)
    hidden = torch.randn(2, calls, *sides[0].hidden.shape, generator=generator, device="cuda").to(sides[0].hidden.dtype)
    uniform = torch.rand(2, calls, rows, generator=generator, device="cuda")

    def outputs():
        return (torch.full((2, calls, *sides[0].logits.shape), float("nan"), dtype=sides[0].logits.dtype, device="cuda"),
                torch.full((2, calls, rows), -77, dtype=torch.int32, device="cuda"), torch.full((2, calls, rows), float("nan"), device="cuda"))

    def call(s, c, out, stream=None):
        a, (logits, chosen, logprobs) = sides[s], out
        B.bpe_linear_mx(hidden[s, c], a.head4, logits[s, c], workspace=a.head4_ws, stream=stream)
        B.bpe_sample_tokens(logits[s, c], uniform[s, c], chosen[s, c], top_p=a.top_p, logprobs=logprobs[s, c], workspace=a.draw_ws, stream=stream)

    wanted, got = outputs(), outputs()
    for s in range(2):
        for c in range(calls):
            call(s, c, wanted)
            torch.cuda.synchronize()
    for c in range(calls):
        for s in range(2):
            call(s, c, got, streams[s])
    torch.cuda.synchronize()
    assert torch.isfinite(wanted[0].float()).all() and (wanted[1] >= 0).all() and torch.isfinite(wanted[2]).all()
    assert len(torch.unique(wanted[1], dim=1).unbind(1)) > 1             # the inputs do make a difference
    for want, have in zip(wanted, got):
        assert torch.equal(have, want)
