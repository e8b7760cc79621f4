"""bpe_grammar_masks and bpe_grammar_advance against the definition, restated through the merge rules: what a merged
token does to a state is what its two parts do one after the other.  Whole numbers: equal bit for bit."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _after(merges, table):
    """int32 [n_ids, n_states + 1]: state behind every token from every state; n_states = the walk has ended."""
    n = table.shape[0]
    after = np.full((256 + len(merges), n + 1), n, dtype=np.int32)
    after[:256, :n] = np.where(table < 0, n, table).T
    for i, (a, b) in enumerate(np.asarray(merges).tolist()):
        after[256 + i] = after[b][after[a]]
    return after


def _masks(after, accepting, states, n_vocab, end_id, numbering=None):
    n_ids, n = after.shape[0], after.shape[1] - 1
    bits = np.zeros((len(states), (n_vocab + 31) // 32 * 32), dtype=np.uint8)
    at = np.arange(n_ids) if numbering is None else numbering
    fits = at < n_vocab
    for i, s in enumerate(states):
        if 0 <= s < n:
            bits[i, at[fits]] = after[fits, s] != n
            if end_id >= 0:
                bits[i, end_id] = accepting[s]
    return np.packbits(bits, axis=1, bitorder="little").view(np.int32)


def _grammar(rng, n_states, density, bytes_used=256):
    table = np.full((n_states, 256), -1, dtype=np.int32)
    on = rng.random((n_states, bytes_used)) < density
    table[:, :bytes_used][on] = rng.integers(0, n_states, int(on.sum()))
    table[rng.random((n_states, 256)) < 0.01] = -7          # any negative value ends the walk
    return table, (rng.random(n_states) < 0.5).astype(np.uint8)


def _merges(name, n=None):
    from workloads import configs as C
    return C.load_merges(name)[:n]


def _run(B, merges, table, accepting, states, n_vocab, end_id, output_ids=None, extra_words=0):
    import torch
    vocab, grammar = B.Vocab(merges, output_ids=output_ids), B.Grammar(table, accepting)
    words = (n_vocab + 31) // 32
    masks = torch.full((len(states), words + extra_words), 0x55555555, dtype=torch.int32, device="cuda")
    st = torch.tensor(np.asarray(states, dtype=np.int32), device="cuda")
    B.bpe_grammar_masks(vocab, grammar, st, masks[:, :words] if extra_words else masks, n_vocab=n_vocab, end_id=end_id, ids_are_output_ids=output_ids is not None)
    got = masks.cpu().numpy()
    assert (got[:, words:] == 0x55555555).all(), "written behind the row"
    vocab.free()
    grammar.free()
    return got[:, :words]


@pytest.mark.parametrize("table_name,n_states,density", [(t, n, d) for t in ("t1k", "t50k", "t100k") for n, d in ((1, 1.0), (2, 0.5), (7, 0.9), (300, 0.3))] +
                         [("t1k", 3000, 0.7), ("t50k", 900, 0.7)])
def test_masks_of_random_automata(B, table_name, n_states, density):
    rng = np.random.default_rng([1, n_states])
    merges = _merges(table_name)
    table, accepting = _grammar(rng, n_states, density)
    n_vocab = 256 + len(merges) + 1
    after = _after(merges, table)
    states = rng.integers(0, n_states, 9)
    print(f"[case] masks {table_name} {n_states}", flush=True)
    got = _run(B, merges, table, accepting, states, n_vocab, n_vocab - 1)
    assert np.array_equal(got, _masks(after, accepting, states, n_vocab, n_vocab - 1))


@pytest.mark.parametrize("n", [1, 2, 3, 5, 8, 13, 16, 17, 33, 64, 100, 300])
def test_numbers_of_states(B, n):
    rng = np.random.default_rng([2, n])
    merges = _merges("t1k")
    table, accepting = _grammar(rng, 40, 0.6)
    states = rng.integers(0, 40, n)
    after = _after(merges, table)
    got = _run(B, merges, table, accepting, states, 1256, -1)
    assert np.array_equal(got, _masks(after, accepting, states, 1256, -1))


@pytest.mark.parametrize("n_vocab", [1, 31, 32, 33, 63, 64, 65, 255, 256, 257, 1000, 1256, 1300, 5000])
def test_more_or_fewer_logits_than_ids(B, n_vocab):
    rng = np.random.default_rng([3, n_vocab])
    merges = _merges("t1k")
    table, accepting = _grammar(rng, 20, 0.8)
    states = [0, -1, 19, 20, 2**31 - 1, -2**31, 5]
    after = _after(merges, table)
    for end_id in (-1, 0, n_vocab - 1):
        got = _run(B, merges, table, accepting, states, n_vocab, end_id, extra_words=2)
        assert np.array_equal(got, _masks(after, accepting, states, n_vocab, end_id)), end_id


def test_output_ids_with_gaps(B):
    rng = np.random.default_rng(4)
    merges = _merges("t1k")
    numbering = rng.permutation(2500)[:1256].astype(np.int32)
    table, accepting = _grammar(rng, 50, 0.7)
    states = rng.integers(0, 50, 21)
    after = _after(merges, table)
    for n_vocab in (2500, 1700, 3001):
        got = _run(B, merges, table, accepting, states, n_vocab, 11, output_ids=numbering)
        want = _masks(after, accepting, states, n_vocab, 11, numbering)
        assert np.array_equal(got, want)


def test_long_tokens(B):
    """Tokens of 1 to 300 bytes, whose walks end at every place of them."""
    merges, n = [(97, 97)], 256
    for k in range(60):                                     # a^3, a^4, ... then doublings
        merges.append((n, 97))
        n += 1
    for k in range(2):
        merges.append((n, n))
        n += 1
    for n_states in (1, 5, 12, 13, 14, 59, 61, 62, 130, 247, 248, 249, 400):
        table = np.full((n_states, 256), -1, dtype=np.int32)
        for s in range(n_states - 1):
            table[s, 97] = s + 1
        accepting = np.zeros(n_states, dtype=np.uint8)
        after = _after(merges, table)
        states = [0, n_states // 2, n_states - 1]
        got = _run(B, merges, table, accepting, states, after.shape[0], -1)
        assert np.array_equal(got, _masks(after, accepting, states, after.shape[0], -1)), n_states


@pytest.mark.parametrize("n_states", [9000, 65534])
def test_many_states_and_classes(B, n_states):
    """Automata that are too large for on-chip memory, all 256 bytes told apart."""
    import torch
    rng = np.random.default_rng(6)
    merges = _merges("t1k")
    table = rng.integers(-n_states // 2, n_states, (n_states, 256)).astype(np.int32)
    accepting = (rng.random(n_states) < 0.5).astype(np.uint8)
    states = np.concatenate([rng.integers(0, n_states, 20), [n_states - 1, n_states]])
    grammar = B.Grammar(table, accepting)
    assert grammar.info["n_classes"] == 256 and grammar.info["n_states"] == n_states
    grammar.free()
    closed = np.concatenate([np.where(table < 0, n_states, table), np.full((1, 256), n_states)])
    from helpers import expand_ids
    want = np.zeros((len(states), 1280), dtype=np.uint8)
    for v in range(1256):
        s = states.copy()
        for b in expand_ids([v], merges):
            s = closed[s, b]
        want[:, v] = s != n_states
    want[:-1, 5] = accepting[states[:-1]]
    want[-1] = 0
    got = _run(B, merges, table, accepting, states, 1256, 5)
    assert np.array_equal(got, np.packbits(want, axis=1, bitorder="little").view(np.int32)[:, :got.shape[1]])
    assert torch.cuda.is_available()


@pytest.mark.parametrize("end_id", [-1, 1256, 40])
def test_advance(B, end_id):
    import torch
    rng = np.random.default_rng(7)
    merges = _merges("t1k")
    table, accepting = _grammar(rng, 30, 0.8)
    after = _after(merges, table)
    states = rng.integers(-2, 33, 2000).astype(np.int32)
    ids = rng.integers(-3, 1260, 2000).astype(np.int32)
    ids[:200] = end_id
    want = np.full(2000, -1, dtype=np.int32)
    for i, (s, v) in enumerate(zip(states.tolist(), ids.tolist())):
        if 0 <= s < 30:
            if end_id >= 0 and v == end_id:
                want[i] = s if accepting[s] else -1
            elif 0 <= v < 1256 and after[v, s] < 30:
                want[i] = after[v, s]
    vocab, grammar = B.Vocab(merges), B.Grammar(table, accepting)
    st, v = torch.from_numpy(states).cuda(), torch.from_numpy(ids).cuda()
    out = torch.zeros_like(st)
    B.bpe_grammar_advance(vocab, grammar, st, v, out, end_id=end_id)
    assert np.array_equal(out.cpu().numpy(), want)
    B.bpe_grammar_advance(vocab, grammar, st, v, st, end_id=end_id)          # in place
    assert np.array_equal(st.cpu().numpy(), want)
    # without a list of accepting states no answer may end
    none = B.Grammar(table)
    B.bpe_grammar_advance(vocab, none, torch.arange(30, dtype=torch.int32, device="cuda"), torch.full((30,), 1256, dtype=torch.int32, device="cuda"), out[:30], end_id=1256)
    assert (out[:30] == -1).all()


def test_a_token_is_allowed_where_advance_goes_on(B):
    """Masks and advance agree on every token of a large vocabulary, on a stream of their own and in a graph."""
    import torch
    rng = np.random.default_rng(8)
    merges = _merges("t50k")
    table, accepting = _grammar(rng, 64, 0.5)
    vocab, grammar = B.Vocab(merges), B.Grammar(table, accepting)
    V = 50256
    side = torch.cuda.Stream()
    states = torch.arange(10, dtype=torch.int32, device="cuda")
    masks = torch.zeros(10, (V + 31) // 32, dtype=torch.int32, device="cuda")
    every = torch.arange(V, dtype=torch.int32, device="cuda")
    out = torch.empty_like(every)
    torch.cuda.synchronize()
    B.bpe_grammar_masks(vocab, grammar, states, masks, stream=side)
    side.synchronize()
    for s in range(10):
        B.bpe_grammar_advance(vocab, grammar, torch.full_like(every, s), every, out)
        bits = ((masks[s][:, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).view(-1)[:V]
        assert torch.equal(bits != 0, out >= 0)
    again = torch.zeros_like(masks)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.bpe_grammar_masks(vocab, grammar, states, again)
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, masks)
