"""bpe_grammar_masks for so many states that tiles of tokens are walked together, against the restatement of test_gpu_grammar:
fields of literal words (few classes of bytes go on) and of free text (many do), tables in and beyond on-chip memory, long
tokens, shares of states that are larger than what a workgroup holds at a time."""
import numpy as np
import pytest

from test_gpu_grammar import _after, _grammar, _masks, _merges, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _fields(rng, n_states):
    """Literal words, then letters that loop or digits, round and round."""
    table = np.full((n_states, 256), -1, dtype=np.int32)
    for s in range(n_states):
        if rng.random() < 0.8:
            table[s, rng.integers(97, 123, int(rng.integers(1, 4)))] = (s + 1) % n_states
        elif rng.random() < 0.5:
            table[s, 97:123] = s
            table[s, 32] = (s + 1) % n_states
        else:
            table[s, 48:58] = s
            table[s, 59] = (s + 1) % n_states
    table[0] = -1                                         # a state that nothing leads on from
    return table, (rng.random(n_states) < 0.5).astype(np.uint8)


@pytest.mark.parametrize("table_name,n,n_vocab", [("t50k", 170, 50257), ("t100k", 90, 100256), ("t1k", 7000, 1256), ("t1k", 7000, 1300), ("t50k", 300, 30011), ("t50k", 500, 60001)])
@pytest.mark.parametrize("kind", ["fields", "dense", "sparse"])
def test_many_states(B, table_name, n, n_vocab, kind):
    rng = np.random.default_rng([n, n_vocab])
    assert n * n_vocab > 8000000
    n_states = 230
    if kind == "fields":
        table, accepting = _fields(rng, n_states)
    else:
        table, accepting = _grammar(rng, n_states, 0.6 if kind == "dense" else 0.02)
    after = _after(_merges(table_name), table)
    states = rng.integers(-2, n_states + 2, n)
    print(f"[case] mask tiles {table_name} {n} {n_vocab} {kind}", flush=True)
    for end_id in (-1, n_vocab - 1, 77):
        got = _run(B, _merges(table_name), table, accepting, states, n_vocab, end_id, extra_words=1)
        assert np.array_equal(got, _masks(after, accepting, states, n_vocab, end_id)), end_id


def test_output_ids(B):
    rng = np.random.default_rng(3)
    numbering = rng.permutation(2500)[:1256].astype(np.int32)
    table, accepting = _fields(rng, 60)
    states = rng.integers(0, 60, 4000)
    after = _after(_merges("t1k"), table)
    got = _run(B, _merges("t1k"), table, accepting, states, 2501, 2500, output_ids=numbering)
    assert np.array_equal(got, _masks(after, accepting, states, 2501, 2500, numbering))


@pytest.mark.parametrize("n_states", [190, 200, 9000])
def test_all_bytes_told_apart(B, n_states):
    """256 classes: tables of 48,896, 51,456 and 2.3 M transitions, the first of which is kept on chip."""
    rng = np.random.default_rng(n_states)
    table = rng.integers(-n_states // 2, n_states, (n_states, 256)).astype(np.int32)
    accepting = (rng.random(n_states) < 0.5).astype(np.uint8)
    after = _after(_merges("t1k"), table)
    states = rng.integers(0, n_states, 6500)
    got = _run(B, _merges("t1k"), table, accepting, states, 1256, 9)
    assert np.array_equal(got, _masks(after, accepting, states, 1256, 9))


def test_more_states_than_a_workgroup_holds(B):
    import torch
    rng = np.random.default_rng(5)
    table, accepting = _fields(rng, 50)
    after = _after(_merges("t1k"), table)
    every = _masks(after, accepting, np.arange(50), 300, 299)
    states = rng.integers(0, 50, 600011).astype(np.int32)
    vocab, grammar = B.Vocab(_merges("t1k")), B.Grammar(table, accepting)
    st = torch.from_numpy(states).cuda()
    masks = torch.zeros(states.size, 10, dtype=torch.int32, device="cuda")
    B.bpe_grammar_masks(vocab, grammar, st, masks, n_vocab=300, end_id=299)
    assert torch.equal(masks, torch.from_numpy(every.copy()).cuda()[st.long()])
