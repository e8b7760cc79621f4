"""Cases for timing the operators that lead from a model's hidden states to the next token ids.

  linear   bpe_linear: act(x w^T + bias) + residual, the projection onto the vocabulary and the blocks before it
  masks    bpe_grammar_masks: which tokens keep a byte automaton alive, one bit per token
  adjust   bpe_adjust_logits: penalties for repeated tokens, biases and masks on logits
  top      bpe_top_tokens: the best tokens of every row with their log-probabilities

Each has a plain form in elementary torch operations, in 32 bits, rounded once at the end, and a definition in 64 bits that is
written apart from it.  Vocabularies are those of the merge tables under workloads/tables; widths are generic.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MERGES = {"t1k": 1000, "t50k": 50000, "t100k": 100000}
TOKEN_BYTES = {"t1k": 4322, "t50k": 294041}          # of all tokens of a vocabulary
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # one request's next token: the vocabulary's weights are read for a single row
        dict(name="linear_one_row", op="linear", m=1, n=50256, k=1024, dtype="bf16", out="f32", act="none", bias=False, residual=False),
        # a serving batch's next tokens over the large vocabulary
        dict(name="linear_batch", op="linear", m=64, n=100256, k=4096, dtype="bf16", out="f32", act="none", bias=True, residual=False),
        # a small residual block in front of the projection, for a batch of odd size
        dict(name="linear_block", op="linear", m=47, n=2048, k=2048, dtype="f16", out="f16", act="silu", bias=True, residual=True),
        # logits of every position of a batch of prompts, for their log-probabilities
        dict(name="linear_prompts", op="linear", m=4001, n=50256, k=4096, dtype="bf16", out="bf16", act="none", bias=False, residual=False),
        # the masks of a few requests that stand in different states of one grammar
        dict(name="masks_step", op="masks", table="t50k", states=96, n=7),
        # the masks of all states of a grammar, made once when it is loaded
        dict(name="masks_all", op="masks", table="t50k", states=1500, n=1500),
        # one request: a short history, a few biases, no grammar
        dict(name="adjust_one_row", op="adjust", rows=1, vocab=50256, dtype="f32", out="f32", history=700, biases=10, masks=0),
        # a batch with a grammar, 16-bit logits and histories of up to 8,000 tokens
        dict(name="adjust_batch", op="adjust", rows=64, vocab=100256, dtype="bf16", out="bf16", history=8000, biases=100, masks=24),
        # the largest batch, long histories, a vocabulary whose rows are not aligned
        dict(name="adjust_large", op="adjust", rows=512, vocab=100257, dtype="f32", out="f32", history=30000, biases=30, masks=200),
        # the best token of one row
        dict(name="top_one_row", op="top", rows=1, vocab=50256, dtype="f32", k=1),
        # a batch: the candidates to sample from
        dict(name="top_batch", op="top", rows=64, vocab=100256, dtype="bf16", k=64),
        # log-probabilities of the 20 best tokens at every position of some prompts
        dict(name="top_prompts", op="top", rows=1024, vocab=50257, dtype="f32", k=20),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("linear", "masks", "adjust", "top"))
    if op == "linear":
        n, k = _log(rng, 256, 100256), _log(rng, 64, 4096)
        if rng.random() < 0.6:                       # most widths are multiples of eight, not all
            k = max(64, k // 8 * 8)
        dtype = rng.choice(("bf16", "f16"))
        most = 4001 * 50256 * 4096 // (n * k)
        m = _log(rng, 1, min(4001, most))
        if m * n > 4001 * 50256 // 2:
            m = max(1, 4001 * 50256 // 2 // n)
        return dict(op="linear", m=m, n=n, k=k, dtype=dtype, out=rng.choice(("f32", dtype)), act=rng.choice(ACTIVATIONS),
                    bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    if op == "masks":
        table = rng.choice(("t1k", "t50k", "t50k"))
        states = _log(rng, 8, 1500)
        return dict(op="masks", table=table, states=states, n=_log(rng, 1, states))
    if op == "adjust":
        rows = _log(rng, 1, 512)
        vocab = rng.choice((1256, 50256, 100256)) + rng.choice((0, 0, 0, 1, 2, 8, 13))
        dtype = rng.choice(("f32", "bf16", "f16"))
        return dict(op="adjust", rows=rows, vocab=vocab, dtype=dtype, out=rng.choice(("f32", dtype)), history=rng.choice((0, _log(rng, 1, 30000), _log(rng, 1, 30000))),
                    biases=rng.choice((0, _log(rng, 1, 300))), masks=rng.choice((0, _log(rng, 1, rows))))
    return dict(op="top", rows=_log(rng, 1, 1024), vocab=rng.choice((1256, 50256, 50257)) + rng.choice((0, 0, 0, 3)), dtype=rng.choice(("f32", "bf16", "f16")),
                k=_log(rng, 1, 128))


# ---------------------------------------------------------------------------
# What the inputs consist of.

@functools.lru_cache(maxsize=None)
def _merges(table):
    return np.fromfile(f"workloads/tables/{table}.merges.i32", dtype="<i4").reshape(-1, 2)


@functools.lru_cache(maxsize=None)
def _tokens(table):
    """The bytes of every token, padded, and their lengths: host arrays."""
    expansions = [bytes([b]) for b in range(256)]
    for a, b in _merges(table).tolist():
        expansions.append(expansions[a] + expansions[b])
    lengths = np.array([len(e) for e in expansions], dtype=np.int64)
    padded = np.zeros((len(expansions), int(lengths.max())), dtype=np.int64)
    for i, e in enumerate(expansions):
        padded[i, :len(e)] = list(e)
    return padded, lengths


def _grammar(states, seed):
    """A byte automaton of so many states: a ring of fields, each a literal word (one state per letter), then
    free text of letters and spaces that loops, or digits, until a separator."""
    rng = np.random.default_rng([7, states, seed])
    table = np.full((states, 256), -1, dtype=np.int32)
    accepting = np.zeros(states, dtype=np.uint8)
    letters = np.frombuffer(b"abcdefghijklmnopqrstuvwxyz", dtype=np.uint8)
    s = 0
    while s < states:
        for _ in range(min(int(rng.integers(3, 12)), states - s - 1)):
            table[s, rng.choice(letters)] = s + 1
            if rng.random() < 0.2:
                table[s, rng.choice(letters)] = s + 1
            s += 1
        after = (s + 1) % states
        if rng.random() < 0.6:
            table[s, letters] = s
            table[s, 32] = s
        else:
            table[s, 48:58] = s
        for b in b",.;:":
            table[s, b] = after
        accepting[s] = rng.random() < 0.5
        s += 1
    return table, accepting


def _lengths(case):
    """Tokens that came before, of every row: none in the first of many, up to the case's number in others."""
    rows, most = case["rows"], case["history"]
    if rows == 1:
        return np.array([most], dtype=np.int64)
    return most * ((np.arange(rows, dtype=np.int64) * 37) % rows) // (rows - 1)


def _words(vocab):
    return (vocab + 31) // 32


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=g, device=DEVICE, dtype=dtype)
    if own:
        import paper_2603_02597_amd as B
    s = dict(case)
    if case["op"] == "linear":
        m, n, k, dtype, out = case["m"], case["n"], case["k"], DTYPES[case["dtype"]], DTYPES[case["out"]]
        s["x"] = normal(m, k, dtype=dtype)
        s["weight"] = normal(n, k, dtype=dtype).mul_(k ** -0.5)
        s["bias_"] = normal(n, dtype=dtype) if case["bias"] else None
        s["residual_"] = normal(m, n, dtype=out) if case["residual"] else None
        s["result"] = torch.empty(m, n, dtype=out, device=DEVICE)
        if own:
            s["workspace"] = torch.empty(B.bpe_linear_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEVICE)
    elif case["op"] == "masks":
        padded, lengths = _tokens(case["table"])
        table, accepting = _grammar(case["states"], seed)
        vocab = padded.shape[0] + 1                          # one more than the vocabulary: the end of the answer
        pick = np.random.default_rng(seed).permutation(case["states"])[:case["n"]]
        s["start"] = torch.from_numpy(pick.astype(np.int32)).to(DEVICE)
        s["end_id"] = vocab - 1
        s["result"] = torch.empty(case["n"], _words(vocab), dtype=torch.int32, device=DEVICE)
        if own:
            s["vocab"], s["grammar"] = B.Vocab(_merges(case["table"])), B.Grammar(table, accepting)
        else:
            dead = case["states"]
            closed = np.full((dead + 1, 256), dead, dtype=np.int64)
            closed[:dead] = np.where(table < 0, dead, table)
            s["table_"] = torch.from_numpy(closed).to(DEVICE)
            s["accepting"] = torch.from_numpy(accepting).to(DEVICE)
            s["bytes"], s["lengths"] = torch.from_numpy(padded).to(DEVICE), torch.from_numpy(lengths).to(DEVICE)
        s["seed"] = seed
    elif case["op"] == "adjust":
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = (normal(rows, vocab) * 4).to(DTYPES[case["dtype"]])
        s["result"] = torch.empty(rows, vocab, dtype=DTYPES[case["out"]], device=DEVICE)
        uniform = lambda low, high: torch.rand(rows, generator=g, device=DEVICE) * (high - low) + low
        s["repetition"], s["frequency"], s["presence"] = uniform(1.0, 1.5), uniform(0.0, 0.6), uniform(-0.5, 1.0)
        total = int(_lengths(case).sum())
        # words come again and again: ids crowd at the front, as they do in a vocabulary ordered by frequency
        s["history_"] = (torch.rand(total, generator=g, device=DEVICE) ** 4 * vocab).to(torch.int32)
        s["history_offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(_lengths(case))]).astype(np.int32)).to(DEVICE)
        if case["biases"]:
            per_row = min(case["biases"], vocab)
            step = vocab // per_row                          # distinct ids: one in each of so many stretches
            at = torch.arange(per_row, device=DEVICE) * step + (torch.rand(rows, per_row, generator=g, device=DEVICE) * step).long()
            s["bias_ids"] = at.to(torch.int32).reshape(-1)
            s["bias_values"] = normal(rows * per_row) * 3
            s["bias_offsets"] = torch.arange(rows + 1, dtype=torch.int32, device=DEVICE) * per_row
        if case["masks"]:
            # a grammar leaves a few of all tokens, or most: words of random bits, thinned out by a factor of their own
            raw = lambda: torch.randint(-2**31, 2**31, (case["masks"], _words(vocab)), generator=g, device=DEVICE).to(torch.int32)
            masks = raw()
            for depth in range(1, 6):
                thin = torch.arange(case["masks"], device=DEVICE) % 6 >= depth
                masks = torch.where(thin[:, None], masks & raw(), masks)
            if case["masks"] > 2:
                masks[2] = 0                                 # a state that no token leads on from
            s["masks_"] = masks
            s["mask_index"] = (torch.arange(rows, device=DEVICE) * 11 % (case["masks"] + 1) - 1).to(torch.int32)
    else:
        rows, vocab = case["rows"], case["vocab"]
        x = normal(rows, vocab) * 3
        # every third row has been through a grammar mask; one has fewer tokens left than are asked for, one has none
        keep = torch.rand(rows, 1, generator=g, device=DEVICE) ** 3
        keep[torch.arange(rows, device=DEVICE) % 3 != 1] = 2
        if rows > 4:
            keep[4] = 0
            keep[1] = 0.5 * case["k"] / vocab
        x.masked_fill_(torch.rand(rows, vocab, generator=g, device=DEVICE) >= keep, -math.inf)
        s["logits"] = x.to(DTYPES[case["dtype"]])
        s["ids"] = torch.empty(rows, case["k"], dtype=torch.int32, device=DEVICE)
        s["logprobs"] = torch.empty(rows, case["k"], dtype=torch.float32, device=DEVICE)
        s["lse"] = torch.empty(rows, dtype=torch.float32, device=DEVICE)
        if own:
            s["workspace"] = torch.empty(B.bpe_top_tokens_workspace_bytes(rows, vocab, case["k"]), dtype=torch.uint8, device=DEVICE)
    return s


# ---------------------------------------------------------------------------
# One pass.

def run(s):
    if own:
        return _run_own(s)
    return {"linear": _linear, "masks": _masks, "adjust": _adjust, "top": _top}[s["op"]](s)


def _run_own(s):
    import paper_2603_02597_amd as B
    op = s["op"]
    if op == "linear":
        B.bpe_linear(s["x"], s["weight"], s["result"], bias=s["bias_"], residual=s["residual_"], activation=s["act"], workspace=s["workspace"])
        return s["result"]
    if op == "masks":
        B.bpe_grammar_masks(s["vocab"], s["grammar"], s["start"], s["result"], n_vocab=s["end_id"] + 1, end_id=s["end_id"])
        return s["result"]
    if op == "adjust":
        B.bpe_adjust_logits(s["logits"], s["result"], history=s["history_"], history_offsets=s["history_offsets"], repetition=s["repetition"],
                            frequency=s["frequency"], presence=s["presence"], bias_ids=s.get("bias_ids"), bias_values=s.get("bias_values"),
                            bias_offsets=s.get("bias_offsets"), masks=s.get("masks_"), mask_index=s.get("mask_index"))
        return s["result"]
    B.bpe_top_tokens(s["logits"], s["ids"], s["logprobs"], s["workspace"], lse=s["lse"])
    return s["ids"], s["logprobs"], s["lse"]


def _linear(s):
    y = s["x"].float() @ s["weight"].float().t()
    if s["bias_"] is not None:
        y = y + s["bias_"].float()
    act = s["act"]
    if act == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    elif act == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    elif act == "gelu_tanh":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    elif act == "silu":
        y = y / (1 + torch.exp(-y))
    if s["residual_"] is not None:
        y = y + s["residual_"].float()
    return y.to(s["result"].dtype)


def _masks(s):
    state = s["start"].long()[:, None].expand(-1, s["bytes"].shape[0])
    for j in range(s["bytes"].shape[1]):                     # a token's bytes one after the other
        state = torch.where(j < s["lengths"], s["table_"][state, s["bytes"][:, j]], state)
    alive = state != s["table_"].shape[0] - 1
    end = s["accepting"][s["start"].long()] != 0
    words = s["result"].shape[1]
    bits = torch.zeros(alive.shape[0], words * 32, dtype=torch.int64, device=alive.device)
    bits[:, :alive.shape[1]] = alive
    bits[:, s["end_id"]] = end
    return (bits.view(-1, words, 32) << torch.arange(32, device=alive.device)).sum(2).to(torch.int32)


def _adjust(s):
    rows, vocab = s["logits"].shape
    x = s["logits"].float()
    offsets = s["history_offsets"].long()
    row = torch.repeat_interleave(torch.arange(rows, device=x.device), offsets[1:] - offsets[:-1], output_size=s["history_"].numel())
    count = torch.zeros(rows * vocab, dtype=torch.float32, device=x.device)
    count.index_add_(0, row * vocab + s["history_"].long(), torch.ones(row.numel(), dtype=torch.float32, device=x.device))
    count = count.view(rows, vocab)
    repetition, frequency, presence = (s[key][:, None] for key in ("repetition", "frequency", "presence"))
    punished = torch.where(x > 0, x / repetition, x * repetition) - frequency * count - presence
    x = torch.where(count > 0, punished, x)
    if s["biases"]:
        row = torch.arange(rows, device=x.device)[:, None]
        at = s["bias_ids"].long().view(rows, -1)
        x[row, at] = x[row, at] + s["bias_values"].view(rows, -1)
    if s["masks"]:
        bits = (s["masks_"][:, :, None] >> torch.arange(32, device=x.device, dtype=torch.int32)) & 1
        allowed = bits.view(s["masks"], -1)[:, :vocab] != 0
        index = s["mask_index"].long()
        x = torch.where((index < 0)[:, None] | allowed[index.clamp(min=0)], x, torch.full_like(x, -math.inf))
    return x.to(s["result"].dtype)


def _top(s):
    x, k = s["logits"].float(), s["k"]
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    value, index = value[:, :k], index[:, :k]
    none = value == -math.inf
    top = value[:, :1]
    total = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top)).sum(1, keepdim=True)
    lse = top + torch.log(total)
    logprobs = torch.where(none, value, value - lse)
    return torch.where(none, torch.full_like(index, -1), index).to(torch.int32), logprobs, lse[:, 0]


# ---------------------------------------------------------------------------
# What one pass cannot do without.

def work(case):
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        size, out = SIZE[case["dtype"]], SIZE[case["out"]]
        return {"bytes": size * (m * k + n * k + (n if case["bias"] else 0)) + out * m * n * (2 if case["residual"] else 1), "flops": 2 * m * n * k}
    if case["op"] == "masks":
        vocab, n = MERGES[case["table"]] + 256, case["n"]
        return {"bytes": 4 * n * _words(vocab + 1) + TOKEN_BYTES[case["table"]] + 4 * vocab + 2 * 256 * case["states"] + 4 * n, "flops": n * vocab}
    if case["op"] == "adjust":
        rows, vocab = case["rows"], case["vocab"]
        size = SIZE[case["dtype"]] + SIZE[case["out"]]
        more = 4 * int(_lengths(case).sum()) + 8 * rows * min(case["biases"], vocab) + 4 * case["masks"] * _words(vocab) + 24 * rows
        return {"bytes": rows * vocab * size + more, "flops": rows * vocab}
    rows, vocab = case["rows"], case["vocab"]
    return {"bytes": rows * vocab * SIZE[case["dtype"]] + rows * (8 * case["k"] + 4), "flops": 3 * rows * vocab}


# ---------------------------------------------------------------------------
# The definitions in 64 bits.

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "masks": _exact_masks, "adjust": _exact_adjust, "top": _exact_top}[case["op"]](case, s)


def _exact_linear(case, s):
    w = s["weight"].to(torch.float64).t().contiguous()
    parts = []
    for rows in torch.split(torch.arange(case["m"], device=DEVICE), 512):
        z = torch.mm(s["x"][rows].to(torch.float64), w)
        if case["bias"]:
            z += s["bias_"].to(torch.float64)[None]
        if case["act"] == "relu":
            z = z.clamp(min=0)
        elif case["act"] == "gelu":
            z = z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
        elif case["act"] == "gelu_tanh":
            z = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        elif case["act"] == "silu":
            z = z * torch.sigmoid(z)
        if case["residual"]:
            z += s["residual_"][rows].to(torch.float64)
        parts.append(z)
    return torch.cat(parts)


def _exact_masks(case, s):
    """What a merged token does to a state is what its two parts do one after the other."""
    table, accepting = _grammar(case["states"], s["seed"])
    merges = _merges(case["table"])
    dead = case["states"]
    after = np.full((256 + len(merges), dead + 1), dead, dtype=np.int32)
    after[:256, :dead] = np.where(table < 0, dead, table).T
    for i, (a, b) in enumerate(merges.tolist()):
        after[256 + i] = after[b][after[a]]
    start = s["start"].cpu().numpy()
    bits = np.zeros((case["n"], _words(s["end_id"] + 1) * 32), dtype=np.uint8)
    bits[:, :after.shape[0]] = after[:, start].T != dead
    bits[:, s["end_id"]] = accepting[start]
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy())


def _exact_adjust(case, s):
    rows, vocab = case["rows"], case["vocab"]
    out = np.empty((rows, vocab), dtype=np.float64)
    host = {key: value.cpu().numpy() for key, value in s.items() if isinstance(value, torch.Tensor) and key not in ("logits", "result")}
    logits = s["logits"].double().cpu().numpy()
    per_row = len(host["bias_ids"]) // rows if case["biases"] else 0
    for r in range(rows):
        x = logits[r].copy()
        before = host["history_"][host["history_offsets"][r]:host["history_offsets"][r + 1]]
        seen, times = np.unique(before, return_counts=True)
        rep, freq, pres = (float(host[key][r]) for key in ("repetition", "frequency", "presence"))
        y = x[seen]
        x[seen] = np.where(y > 0, y / rep, y * rep) - freq * times - pres
        if per_row:
            x[host["bias_ids"][r * per_row:(r + 1) * per_row]] += host["bias_values"][r * per_row:(r + 1) * per_row]
        if case["masks"] and host["mask_index"][r] >= 0:
            bits = np.unpackbits(host["masks_"][host["mask_index"][r]].view(np.uint8), bitorder="little")[:vocab]
            x[bits == 0] = -np.inf
        out[r] = x
    return torch.from_numpy(out)


def _exact_top(case, s):
    rows, k = case["rows"], case["k"]
    ids = np.full((rows, k), -1, dtype=np.int32)
    logprobs = np.full((rows, k), -np.inf)
    lse = np.full(rows, -np.inf)
    logits = s["logits"].float().cpu().numpy()
    for r in range(rows):
        x = logits[r]
        left = np.nonzero(x > -np.inf)[0]
        if not left.size:
            continue
        most = float(x[left].max())
        lse[r] = most + math.log(float(np.exp(x[left].astype(np.float64) - most).sum()))
        if left.size > k:
            bound = np.partition(x[left], left.size - k)[left.size - k]
            left = left[x[left] >= bound]
        best = left[np.lexsort((left, -x[left]))][:k]
        ids[r, :best.size] = best
        logprobs[r, :best.size] = x[best].astype(np.float64) - lse[r]
    return torch.from_numpy(ids), torch.from_numpy(logprobs), torch.from_numpy(lse)
