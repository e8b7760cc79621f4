"""The operators together, as examples/constrained_answers.py runs them: every answer keeps to the grammar."""
import importlib.util
import os
import re

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("constrained_answers", os.path.join(ROOT, "examples", "constrained_answers.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


_parts = [re.escape(c).encode() for c in "city "] + [b"[a-z]+;?"] + [re.escape(c).encode() for c in " year "] + [b"[0-9]+;?"] + [re.escape(c).encode() for c in " name "] + [b"[a-z]+;?"]
PREFIX = re.compile(b"(" .join([b""] + _parts) + b")?" * len(_parts))
WHOLE = re.compile(rb"city [a-z]+; year [0-9]+; name [a-z]+;")


@pytest.mark.parametrize("rows,table", [(1, "t1k"), (37, "t1k"), (6, "t50k")])
def test_answers_keep_to_the_grammar(example, rows, table):
    texts, done, logprobs = example.answer(rows=rows, steps=30, table=table, seed=rows)
    assert len(texts) == rows and np.isfinite(logprobs).all() and max(logprobs) <= 0
    for text, complete in zip(texts, done):
        assert PREFIX.fullmatch(text) and len(text) > 0, text
        assert not complete or WHOLE.fullmatch(text), text
    assert rows < 30 or any(done)
    assert example.answer(rows=rows, steps=30, table=table, seed=rows)[0] == texts        # nothing depends on the order of execution


def test_a_step_against_the_formulas(example):
    """One step's tokens and log-probabilities, restated in 64 bits from the step's own hidden states."""
    import torch
    from workloads import configs
    a = example.Answerer(configs.load_merges("t1k"), example.record_grammar(example.FIELDS), 5, 4, seed=3)
    for t in range(4):
        hidden, state, history = a.hidden.double().cpu().numpy(), a.state.cpu().numpy(), a.history.cpu().numpy().copy()
        z = hidden @ a.block.double().cpu().numpy().T + a.block_bias.double().cpu().numpy()
        mixed = torch.from_numpy(z / (1 + np.exp(-z)) + hidden)
        a.step(t, torch.full((5,), 0.5, device="cuda"))
        got = a.mixed.double().cpu()
        assert float((got - mixed).abs().max()) <= 2.0 ** -8 * float(mixed.abs().max()) + 1e-4      # half a unit of bf16, doubled
        logits = got.numpy() @ a.head.double().cpu().numpy().T
        masks = a.masks.cpu().numpy()
        for r in range(5):
            x = logits[r]
            seen, c = np.unique(history[r][history[r] >= 0], return_counts=True)
            y = x[seen]
            x[seen] = np.where(y > 0, y / np.float32(1.2), y * np.float32(1.2)) - np.float32(0.1) * c - np.float32(0.3)
            x[ord(";")] += 6.0
            bits = np.unpackbits(masks[state[r]].view(np.uint8), bitorder="little")[:a.n_vocab]
            x[bits == 0] = -np.inf
            lse = np.log(np.exp(x - x.max()).sum()) + x.max()
            n = min(a.k, int(bits.sum()))
            want = np.sort(x)[::-1][:n] - lse
            lp = a.logprobs[r].double().cpu().numpy()
            # sums of 256 products of about unit size in 32 bits, and the bound on lse of the tests of bpe_top_tokens
            assert np.abs(lp[:n] - want).max() <= 2 * 272 * 2.0 ** -24 * 40 + 600 * 2.0 ** -24
            assert (lp[n:] == -np.inf).all() and (a.ids[r, n:] == -1).all()
