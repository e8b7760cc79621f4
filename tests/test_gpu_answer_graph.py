"""A whole step from hidden states to the next state of the grammar in one graph: buffers that stay, no host in between.  Replayed
several times, with other work and synchronisations in between, every replay has to give what the same calls give one by one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _program(torch, B, seed, rows=21, width=136, k=5, table="t1k"):
    from test_gpu_answers import ROOT
    import importlib.util
    import os
    from workloads import configs
    spec = importlib.util.spec_from_file_location("constrained_answers", os.path.join(ROOT, "examples", "constrained_answers.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    vocab, grammar = B.Vocab(configs.load_merges(table)), B.Grammar(*example.record_grammar(example.FIELDS))
    n_vocab = vocab.info["n_ids"] + 1
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    empty = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    block, head = (normal(width, width) * width ** -0.5).bfloat16(), (normal(n_vocab, width) * width ** -0.5 * 3).bfloat16()
    bias_ids, bias_values = torch.full((rows,), ord(";"), dtype=torch.int32, device="cuda"), torch.full((rows,), 6.0, device="cuda")
    bias_offsets = torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    history = torch.full((rows, 9), -1, dtype=torch.int32, device="cuda")
    offsets = torch.arange(rows + 1, dtype=torch.int32, device="cuda") * 9
    rep, freq, pres = (torch.full((rows,), v, device="cuda") for v in (1.2, 0.1, 0.3))
    hidden, mixed, logits = normal(rows, width).bfloat16(), torch.empty(rows, width, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, n_vocab, device="cuda")
    state, masks = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, (n_vocab + 31) // 32, dtype=torch.int32, device="cuda")
    ids, logprobs = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
    chosen, lse = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    block_ws, head_ws = empty(B.bpe_linear_workspace_bytes(rows, width, width)), empty(B.bpe_linear_workspace_bytes(rows, n_vocab, width))
    top_ws = empty(B.bpe_top_tokens_workspace_bytes(rows, n_vocab, k))

    def step():
        B.bpe_linear(hidden, block, mixed, residual=hidden, activation="silu", workspace=block_ws)
        B.bpe_linear(mixed, head, logits, workspace=head_ws)
        B.bpe_grammar_masks(vocab, grammar, state, masks, n_vocab=n_vocab, end_id=n_vocab - 1)
        B.bpe_adjust_logits(logits, logits, history=history.view(-1), history_offsets=offsets, repetition=rep, frequency=freq, presence=pres,
                            bias_ids=bias_ids, bias_values=bias_values, bias_offsets=bias_offsets, masks=masks)
        B.bpe_top_tokens(logits, ids, logprobs, top_ws, lse=lse)
        chosen.copy_(ids[:, 0])
        B.bpe_grammar_advance(vocab, grammar, state, chosen, state, end_id=n_vocab - 1)
        history.copy_(torch.cat([history[:, 1:], chosen[:, None]], 1))
        hidden.copy_(mixed.flip(1))

    return step, dict(hidden=hidden, logits=logits, masks=masks, ids=ids, logprobs=logprobs, lse=lse, state=state, history=history), (vocab, grammar)


def test_a_step_in_one_graph():
    import torch
    import paper_2603_02597_amd as B
    eager, want, _keep = _program(torch, B, 5)
    replayed, got, _keep_too = _program(torch, B, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    start = {name: t.clone() for name, t in got.items()}
    with torch.cuda.stream(side):
        replayed()                                       # (what is loaded at first use is loaded before the capture)
    torch.cuda.current_stream().wait_stream(side)
    for name, t in got.items():
        t.copy_(start[name])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed()
    seen = []
    for _ in range(8):
        eager()
        torch.cuda.synchronize()
        graph.replay()
        for name in want:
            bits = torch.int16 if want[name].element_size() == 2 else torch.int32
            assert torch.equal(got[name].view(bits), want[name].view(bits)), name
        seen.append(want["ids"][:, 0].cpu().numpy().copy())
        torch.randn(1000, 1000, device="cuda").sum().item()
    assert (np.array(seen)[0] >= 0).all() and len({s.tobytes() for s in seen}) > 1
