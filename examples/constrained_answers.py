"""Answers under a grammar, from hidden states to text: the operators between a model and the tokenizer, run together.

Every step takes the hidden states of a batch of requests through a residual block (bpe_linear with SiLU and the residual in
its epilogue) and the projection onto the vocabulary (bpe_linear), applies each request's penalties, biases and the mask of
the state that its grammar is in (bpe_adjust_logits; the masks of all states are made once, by bpe_grammar_masks), takes the
k best tokens with their log-probabilities (bpe_top_tokens), chooses one of them by a uniform number, and moves the grammar on
(bpe_grammar_advance).  bpe_decode turns the ids into text.  The model is a stand-in with random weights: the next hidden
state is the last one mixed with the embedding of the chosen token.

    python examples/constrained_answers.py [--rows 8] [--steps 24] [--table t1k] [--seed 0]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2603_02597_amd as B  # noqa: E402
from workloads import configs  # noqa: E402


def record_grammar(fields):
    """Automaton of `name value;` for every field in turn: name literally, a space, then a word of letters or a number of digits,
    then a semicolon.  The answer may end behind the last semicolon."""
    rows = []

    def state():
        rows.append([-1] * 256)
        return len(rows) - 1

    at = state()
    for name, kind in fields:
        for byte in name.encode() + b" ":
            to = state()
            rows[at][byte] = to
            at = to
        value, after = state(), state()
        for byte in (b"abcdefghijklmnopqrstuvwxyz" if kind == "word" else b"0123456789"):
            rows[at][byte] = value
            rows[value][byte] = value
        rows[value][ord(";")] = after
        at = after
    accepting = np.zeros(len(rows), dtype=np.uint8)
    accepting[at] = 1
    return np.array(rows, dtype=np.int32), accepting


class Answerer:
    """Buffers and weights that a serving loop keeps."""

    def __init__(self, merges, grammar, rows: int, max_steps: int, width: int = 256, k: int = 16, seed: int = 0):
        import torch
        self.torch, self.rows, self.k, self.width = torch, rows, k, width
        dev = torch.device("cuda")
        self.vocab = B.Vocab(merges)
        self.grammar = B.Grammar(*grammar)
        self.end_id = self.vocab.info["n_ids"]                 # one more logit than the vocabulary has ids: the end of the answer
        self.n_vocab = self.end_id + 1
        g = torch.Generator(device=dev).manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)
        self.block = (normal(width, width) * width ** -0.5).bfloat16()
        self.block_bias = (normal(width) * 0.1).bfloat16()
        self.head = (normal(self.n_vocab, width) * width ** -0.5 * 3).bfloat16()
        self.embedding = normal(self.n_vocab, width).bfloat16()
        self.hidden = normal(rows, width).bfloat16()
        self.mixed = torch.empty_like(self.hidden)
        self.logits = torch.empty(rows, self.n_vocab, device=dev)
        self.ids = torch.empty(rows, k, dtype=torch.int32, device=dev)
        self.logprobs = torch.empty(rows, k, device=dev)
        bytes_ = lambda n: torch.empty(n, dtype=torch.uint8, device=dev)
        self.block_ws = bytes_(B.bpe_linear_workspace_bytes(rows, width, width))
        self.head_ws = bytes_(B.bpe_linear_workspace_bytes(rows, self.n_vocab, width))
        self.top_ws = bytes_(B.bpe_top_tokens_workspace_bytes(rows, self.n_vocab, k))
        n_states = self.grammar.info["n_states"]
        self.masks = torch.empty(n_states + 1, (self.n_vocab + 31) // 32, dtype=torch.int32, device=dev)
        every = torch.arange(n_states + 1, dtype=torch.int32, device=dev)      # the last one is none of the grammar's: it allows nothing
        B.bpe_grammar_masks(self.vocab, self.grammar, every, self.masks, n_vocab=self.n_vocab, end_id=self.end_id)
        self.state = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.done = torch.zeros(rows, dtype=torch.bool, device=dev)
        # histories of equal length here, row by row: what has been answered so far
        self.history = torch.full((rows, max_steps), -1, dtype=torch.int32, device=dev)
        self.offsets = (torch.arange(rows + 1, dtype=torch.int32, device=dev) * max_steps)
        self.repetition = torch.full((rows,), 1.2, device=dev)
        self.presence = torch.full((rows,), 0.3, device=dev)
        self.frequency = torch.full((rows,), 0.1, device=dev)
        # the semicolon is one token of many: a bias keeps values short
        self.bias_ids = torch.full((rows,), ord(";"), dtype=torch.int32, device=dev)
        self.bias_values = torch.full((rows,), 6.0, device=dev)
        self.bias_offsets = torch.arange(rows + 1, dtype=torch.int32, device=dev)

    def step(self, t: int, uniform):
        """One token for every request; uniform: float32 [rows] in [0, 1).  Returns (ids, log-probabilities), -1 for requests that are done."""
        torch = self.torch
        B.bpe_linear(self.hidden, self.block, self.mixed, bias=self.block_bias, residual=self.hidden, activation="silu", workspace=self.block_ws)
        B.bpe_linear(self.mixed, self.head, self.logits, workspace=self.head_ws)
        index = torch.where(self.done | (self.state < 0), torch.full_like(self.state, self.masks.shape[0] - 1), self.state)
        B.bpe_adjust_logits(self.logits, self.logits, history=self.history.view(-1), history_offsets=self.offsets, repetition=self.repetition,
                            frequency=self.frequency, presence=self.presence, bias_ids=self.bias_ids, bias_values=self.bias_values,
                            bias_offsets=self.bias_offsets, masks=self.masks, mask_index=index)
        B.bpe_top_tokens(self.logits, self.ids, self.logprobs, self.top_ws)
        share = torch.cumsum(torch.exp(self.logprobs), 1)
        at = (uniform[:, None] * share[:, -1:] >= share).sum(1).clamp(max=self.k - 1)
        chosen = self.ids.gather(1, at[:, None])[:, 0]
        logprob = self.logprobs.gather(1, at[:, None])[:, 0]
        over = self.done | (chosen < 0)
        chosen = torch.where(over, torch.full_like(chosen, -1), chosen)
        moved = torch.empty_like(self.state)
        B.bpe_grammar_advance(self.vocab, self.grammar, self.state, chosen, moved, end_id=self.end_id)
        self.state = torch.where(over, self.state, moved)
        self.done = over | (chosen == self.end_id)
        self.history[:, t] = chosen
        mix = self.mixed.float() + self.embedding[chosen.clamp(min=0).long()].float()
        self.hidden = (mix / mix.square().mean(1, keepdim=True).sqrt()).bfloat16()
        return chosen, logprob

    def text(self):
        """The answers so far, as bytes."""
        torch = self.torch
        flat = self.history.view(-1)
        keep = (flat >= 0) & (flat != self.end_id)
        ids = flat[keep].contiguous()
        counts = keep.view(self.rows, -1).sum(1).cpu().numpy()
        if ids.numel() == 0:
            return [b""] * self.rows
        out = torch.empty(ids.numel() * self.vocab.info["max_token_bytes"], dtype=torch.uint8, device="cuda")
        at = torch.empty(ids.numel() + 1, dtype=torch.int32, device="cuda")
        ws = torch.empty(B.bpe_decode_workspace_bytes(ids.numel()), dtype=torch.uint8, device="cuda")
        B.bpe_decode(self.vocab, ids, out, ws, token_byte_offsets=at)
        if (st := B.bpe_encode_status(ws)) != 0:
            raise B.BpeError(st, "decode")
        starts = at.cpu().numpy()[np.concatenate([[0], np.cumsum(counts)])]
        data = out.cpu().numpy().tobytes()
        return [data[a:b] for a, b in zip(starts, starts[1:])]


FIELDS = [("city", "word"), (" year", "number"), (" name", "word")]


def answer(rows: int = 8, steps: int = 24, table: str = "t1k", seed: int = 0):
    """(texts, whether each is complete, log-probability of each)"""
    import torch
    a = Answerer(configs.load_merges(table), record_grammar(FIELDS), rows, steps, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    total = torch.zeros(rows, device="cuda")
    for t in range(steps):
        ids, logprob = a.step(t, torch.rand(rows, generator=g, device="cuda"))
        total += torch.where(ids >= 0, logprob, torch.zeros_like(logprob))
    return a.text(), a.done.cpu().tolist(), total.cpu().tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=8)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--table", default="t1k")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    for text, done, logprob in zip(*answer(a.rows, a.steps, a.table, a.seed)):
        print(f"{logprob:9.2f}  {'complete' if done else 'cut off '}  {text.decode('utf-8', 'replace')}", flush=True)


if __name__ == "__main__":
    main()
