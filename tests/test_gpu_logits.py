"""bpe_adjust_logits and bpe_top_tokens against their definitions in 64 bits.

Adjusting: at most five operations, each rounded by itself, so an element is off by at most 6 * 2^-24 of the sum of the
absolute values that enter, and by half a unit of the output's type; what no rule touches keeps its bits.
Best tokens: ids are equal (ties by index).  lse: exp and its argument are good to 16 units of 2^-24 on the weighted mean
and a sum in 32 bits by at most 512 additions one after the other, so 600 * 2^-24, and 4 * 2^-24 of the values that are
subtracted and rounded."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _lists(rng, rows, lengths, vocab, skew=3):
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    return (rng.random(off[-1]) ** skew * vocab).astype(np.int32), off


def _reference(x, vocab, history=None, bias=None, masks=None, index=None, rep=None, freq=None, pres=None):
    """(values, tolerances before the last rounding, touched) in 64 bits."""
    rows = x.shape[0]
    v, tol, touched = x.astype(np.float64).copy(), np.zeros(x.shape), np.zeros(x.shape, dtype=bool)
    for r in range(rows):
        if history is not None:
            h = history[0][history[1][r]:history[1][r + 1]]
            h = h[(h >= 0) & (h < vocab)]
            ids, c = np.unique(h, return_counts=True)
            a, f, p = (d if arr is None else float(arr[r]) for arr, d in ((rep, 1.0), (freq, 0.0), (pres, 0.0)))
            y = np.where(v[r, ids] > 0, v[r, ids] / a, v[r, ids] * a)
            tol[r, ids] = 6 * U * (np.abs(y) + np.abs(f * c) + abs(p))
            v[r, ids] = y - f * c - p
            touched[r, ids] = True
        if bias is not None:
            last = {}
            for i in range(bias[2][r], bias[2][r + 1]):
                if 0 <= bias[0][i] < vocab:
                    last[int(bias[0][i])] = float(bias[1][i])
            for i, b in last.items():
                tol[r, i] += 6 * U * (abs(v[r, i]) + abs(b))
                v[r, i] += b
                touched[r, i] = True
        if masks is not None:
            i = r if index is None else int(index[r])
            if i >= 0:
                bits = np.zeros(vocab, dtype=np.uint8) if i >= masks.shape[0] else np.unpackbits(masks[i].view(np.uint8), bitorder="little")[:vocab]
                v[r, bits == 0] = -np.inf
                touched[r, bits == 0] = True
    return v, tol, touched


def _check_adjusted(got, logits, want, out):
    v, tol, touched = want
    g = got.double().cpu().numpy()
    fine = np.isfinite(v)
    assert np.array_equal(np.isnan(g), np.isnan(v))
    assert np.array_equal(g[~fine & ~np.isnan(v)], v[~fine & ~np.isnan(v)])
    limit = tol + HALF[out] * np.abs(np.where(fine, v, 0)) + 2.0 ** -25 * (out == "float16")
    bad = fine & ~(np.abs(np.where(fine, g, 0) - np.where(fine, v, 0)) <= limit)
    assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], v[bad][:5])
    same = logits.to(got.dtype).float().cpu().numpy()
    assert np.array_equal(same[~touched], got.float().cpu().numpy()[~touched], equal_nan=True)


def _adjust(B, torch, logits, out_dtype, vocab, history=None, bias=None, masks=None, index=None, rep=None, freq=None, pres=None, out=None):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if out is None:
        out = torch.full(logits.shape, 123.0, dtype=getattr(torch, out_dtype), device="cuda")
    h, b = history or (None, None), bias or (None, None, None)
    B.bpe_adjust_logits(logits, out, history=dev(h[0]), history_offsets=dev(h[1]), repetition=dev(rep), frequency=dev(freq), presence=dev(pres),
                        bias_ids=dev(b[0]), bias_values=dev(b[1]), bias_offsets=dev(b[2]), masks=dev(masks), mask_index=dev(index))
    return out


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 50256), (2, 31), (3, 33), (5, 4095), (5, 4096), (5, 4097), (4, 8193), (33, 1256), (3, 100257), (2, 16385), (1, 65537), (700, 40)])
@pytest.mark.parametrize("dtype,out", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16"), ("bfloat16", "float32")])
def test_all_rules_together(B, rows, vocab, dtype, out):
    import torch
    rng = np.random.default_rng([rows, vocab])
    print(f"[case] adjust {rows} {vocab} {dtype} {out}", flush=True)
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32) * 5).cuda().to(getattr(torch, dtype))
    lengths = rng.integers(0, 900, rows)
    lengths[rows // 2] = 0
    history = _lists(rng, rows, lengths, vocab)
    n_b = rng.integers(0, 20, rows)
    ids, off = _lists(rng, rows, n_b, vocab, 1)
    bias = (ids, rng.standard_normal(ids.size).astype(np.float32) * 4, off)
    n_masks = max(1, rows // 2)
    masks = rng.integers(-2**31, 2**31, (n_masks, (vocab + 31) // 32)).astype(np.int32)
    masks[0] = 0
    index = rng.integers(-1, n_masks + 1, rows).astype(np.int32)             # none, one of them, one that is not there
    rep = rng.uniform(0.6, 1.9, rows).astype(np.float32)
    freq = rng.uniform(-0.3, 0.7, rows).astype(np.float32)
    pres = rng.uniform(-0.5, 1.5, rows).astype(np.float32)
    got = _adjust(B, torch, logits, out, vocab, history, bias, masks, index, rep, freq, pres)
    want = _reference(logits.float().cpu().numpy(), vocab, history, bias, masks, index, rep, freq, pres)
    _check_adjusted(got, logits, want, out)
    if dtype == out:                                                           # in place: the same bits
        again = _adjust(B, torch, logits, out, vocab, history, bias, masks, index, rep, freq, pres, out=logits)
        assert torch.equal(again.view(torch.int32 if out == "float32" else torch.int16), got.view(torch.int32 if out == "float32" else torch.int16))


@pytest.mark.parametrize("which", ["none", "history", "repetition", "frequency", "presence", "bias", "masks", "masks_by_row"])
@pytest.mark.parametrize("rows,vocab", [(1, 5003), (6, 20000)])
def test_one_rule_at_a_time(B, which, rows, vocab):
    import torch
    rng = np.random.default_rng(5)
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).cuda()
    kw = {}
    if which in ("history", "repetition", "frequency", "presence"):
        kw["history"] = _lists(rng, rows, rng.integers(1, 5000, rows), vocab)
    if which in ("repetition", "frequency", "presence"):
        kw[{"repetition": "rep", "frequency": "freq", "presence": "pres"}[which]] = rng.uniform(0.5, 2, rows).astype(np.float32)
    if which == "bias":
        ids, off = _lists(rng, rows, rng.integers(0, 300, rows), vocab)
        kw["bias"] = (ids, rng.standard_normal(ids.size).astype(np.float32), off)
    if which.startswith("masks"):
        kw["masks"] = rng.integers(-2**31, 2**31, (rows, (vocab + 31) // 32)).astype(np.int32)
    if which == "masks":
        kw["index"] = np.arange(rows, dtype=np.int32)[::-1].copy()
    got = _adjust(B, torch, logits, "float32", vocab, **kw)
    _check_adjusted(got, logits, _reference(logits.cpu().numpy(), vocab, **kw), "float32")


@pytest.mark.parametrize("length", [0, 1, 1023, 70000, 400000])
def test_long_histories_count_right(B, length):
    """One token 400,000 times, others a few times; every row's history ends where the next begins."""
    import torch
    rng = np.random.default_rng(length)
    vocab, rows = 3001, 3
    logits = torch.zeros(rows, vocab, device="cuda")
    history = _lists(rng, rows, [length, 0, 17], vocab)
    history[0][:length * 3 // 4] = 2999
    freq = np.array([1.0, 1.0, 1.0], dtype=np.float32)
    got = _adjust(B, torch, logits, "float32", vocab, history, freq=freq).cpu().numpy()
    want = np.zeros((rows, vocab))
    for r in range(rows):
        want[r] -= np.bincount(history[0][history[1][r]:history[1][r + 1]], minlength=vocab)
    assert np.array_equal(got, want)               # counts below 2^24 are exact


def test_infinities_and_nan(B):
    """What a mask takes out is -infinity whatever it was; what it leaves keeps its infinity or NaN, touched or not."""
    import torch
    x = torch.tensor([[float("nan"), float("inf"), -float("inf"), 3e38, -3e38, 0.0, -0.0, 1.0]] * 3, device="cuda")
    history = (np.tile(np.array([0, 1, 2, 3, 5], dtype=np.int32), 3), np.array([0, 5, 10, 15], dtype=np.int32))
    masks = np.array([[0], [0xFF], [0x81]], dtype=np.int32)
    rep = np.full(3, 1.5, dtype=np.float32)
    got = _adjust(B, torch, x, "float32", 8, history, masks=masks, rep=rep).cpu().numpy()
    assert (got[0] == -np.inf).all()
    assert np.isnan(got[1, 0]) and got[1, 1] == np.inf and got[1, 2] == -np.inf and got[1, 7] == 1.0 and got[1, 4] == np.float32(-3e38)
    assert np.isnan(got[2, 0]) and (got[2, 1:7] == -np.inf).all() and got[2, 7] == 1.0
    lowest = torch.full((1, 8), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(lowest)
    B.bpe_adjust_logits(lowest, out)
    assert torch.equal(out, lowest)


def test_offsets_and_ids_out_of_range_touch_nothing(B):
    """Offsets are clamped to the list; ids outside the vocabulary count for nothing."""
    import torch
    rows, vocab = 4, 100
    logits = torch.zeros(rows, vocab, device="cuda")
    ids = np.array([3, -1, 100, 2**31 - 1, -2**31, 7, 7, 9], dtype=np.int32)
    off = np.array([-5, 6, 4, 8, 900], dtype=np.int32)          # decreasing once, beyond the end at last
    freq = np.ones(rows, dtype=np.float32)
    got = _adjust(B, torch, logits, "float32", vocab, (ids, off), freq=freq, bias=(ids, np.full(8, 0.5, dtype=np.float32), off)).cpu().numpy()
    want = np.zeros((rows, vocab))
    for r, part in enumerate((ids[0:6], ids[6:6], ids[4:8], ids[8:8])):
        part = part[(part >= 0) & (part < vocab)]
        want[r] -= np.bincount(part, minlength=vocab)
        want[r, np.unique(part)] += 0.5
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset,pad", [(0, 4), (1, 0), (3, 5), (2, 1)])
def test_adjust_strides_and_alignment(B, dtype, offset, pad):
    import torch
    rng = np.random.default_rng(11)
    rows, vocab = 5, 9001
    dt = getattr(torch, dtype)

    def inside(fill):
        t = torch.full((rows * (vocab + pad) + offset + 16,), fill, dtype=dt, device="cuda")
        return t, t[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]

    _, logits = inside(float("nan"))
    logits.copy_(torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)))
    whole, out = inside(77.0)
    history = _lists(rng, rows, [10, 0, 3000, 1, 200], vocab)
    masks = rng.integers(-2**31, 2**31, (rows, (vocab + 31) // 32 + 3)).astype(np.int32)
    pres = np.ones(rows, dtype=np.float32)
    _adjust(B, torch, logits, dtype, vocab, history, masks=masks, pres=pres, out=out)
    _check_adjusted(out, logits, _reference(logits.float().cpu().numpy(), vocab, history, masks=masks, pres=pres), dtype)
    out.fill_(77.0)
    assert (whole == 77.0).all(), "written outside the rows"


def _top_reference(x, k):
    rows, vocab = x.shape
    ids, lp, lse = np.full((rows, k), -1, dtype=np.int64), np.full((rows, k), -np.inf), np.full(rows, -np.inf)
    for r in range(rows):
        left = np.nonzero(x[r] > -np.inf)[0]
        if left.size:
            most = float(x[r][left].max())
            lse[r] = most + np.log(np.exp(x[r][left].astype(np.float64) - most).sum())
            best = left[np.lexsort((left, -x[r][left]))][:k]
            ids[r, :best.size] = best
            lp[r, :best.size] = x[r][best].astype(np.float64) - lse[r]
    return ids, lp, lse


def _top(B, torch, logits, k, with_lse=True, stream=None):
    rows, vocab = logits.shape
    ids = torch.full((rows, k), -9, dtype=torch.int32, device="cuda")
    lp = torch.full((rows, k), 9.0, device="cuda")
    lse = torch.full((rows,), 9.0, device="cuda") if with_lse else None
    ws = torch.full((B.bpe_top_tokens_workspace_bytes(rows, vocab, k),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    B.bpe_top_tokens(logits, ids, lp, ws, lse=lse, stream=stream)
    torch.cuda.synchronize()
    return ids, lp, lse


def _check_top(B, torch, logits, k):
    ids, lp, lse = _top(B, torch, logits, k)
    x = logits.float().cpu().numpy()
    want_ids, want_lp, want_lse = _top_reference(x, k)
    assert np.array_equal(ids.cpu().numpy(), want_ids), np.argwhere(ids.cpu().numpy() != want_ids)[:5]
    for got, want in ((lp.double().cpu().numpy(), want_lp), (lse.double().cpu().numpy(), want_lse)):
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine], want[~fine])
        scale = np.abs(np.where(np.isfinite(want_lse), want_lse, 0))[(...,) + (None,) * (want.ndim - 1)] + np.abs(np.where(fine, want, 0))
        assert (np.abs(got[fine] - want[fine]) <= (600 * U + 4 * U * np.broadcast_to(scale, want.shape))[fine]).all()


@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (1, 2, 2), (3, 7, 7), (2, 64, 10), (1, 255, 255), (4, 256, 256), (2, 1000, 256), (5, 1256, 20), (1, 4096, 64), (3, 4097, 1), (1, 50256, 1),
                                          (2, 50257, 200), (65, 8191, 5), (1, 100256, 256), (300, 1256, 50), (2, 16384, 128), (1500, 300, 3), (1, 1000003, 100)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_best_tokens(B, rows, vocab, k, dtype):
    import torch
    rng = np.random.default_rng([rows, vocab, k])
    print(f"[case] top {rows} {vocab} {k} {dtype}", flush=True)
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32) * 3).cuda().to(getattr(torch, dtype))
    _check_top(B, torch, logits, k)


@pytest.mark.parametrize("kind", ["all_equal", "two_values", "few_left", "none_left", "rising", "falling", "zeros", "lowest", "one_huge", "clusters", "first_block", "subnormal"])
@pytest.mark.parametrize("rows,vocab,k", [(1, 50256, 33), (7, 3001, 200), (2, 100, 100), (40, 20011, 1), (1, 200000, 256)])
def test_best_tokens_of_hard_rows(B, kind, rows, vocab, k):
    import torch
    rng = np.random.default_rng(3)
    x = np.zeros((rows, vocab), dtype=np.float32)
    if kind == "two_values":
        x = (rng.random((rows, vocab)) < 0.3).astype(np.float32)
    elif kind == "few_left":
        x[:] = -np.inf
        for r in range(rows):
            x[r, rng.integers(0, vocab, max(1, k // 2))] = rng.standard_normal(max(1, k // 2))
    elif kind == "none_left":
        x[:] = -np.inf
        x[rows // 2, vocab - 1] = -5.0
    elif kind == "rising":
        x[:] = np.arange(vocab) * 1e-3
    elif kind == "falling":
        x[:] = -np.arange(vocab) * 1e-3
    elif kind == "zeros":
        x = np.where(rng.random((rows, vocab)) < 0.5, np.float32(0.0), np.float32(-0.0))
    elif kind == "lowest":
        x[:] = np.finfo(np.float32).min
        x[:, ::3] = -np.inf
    elif kind == "one_huge":
        x = rng.standard_normal((rows, vocab)).astype(np.float32)
        x[:, vocab // 3] = 3e38
    elif kind == "clusters":                             # the best ones are neighbours
        x = rng.standard_normal((rows, vocab)).astype(np.float32)
        x[:, vocab // 2: vocab // 2 + k] += 50
    elif kind == "first_block":                          # the best ones come at equal distances
        x = rng.standard_normal((rows, vocab)).astype(np.float32)
        x[:, ::max(1, vocab // k)] += 50
    elif kind == "subnormal":
        x = rng.standard_normal((rows, vocab)).astype(np.float32) * np.float32(1e-40)
    _check_top(B, torch, torch.from_numpy(np.ascontiguousarray(x)).cuda(), k)


def test_best_tokens_with_nan_and_infinity(B):
    import torch
    x = torch.randn(4, 3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[0, 700] = float("nan")
    x[1, 5] = float("inf")
    x[2, 10] = float("inf")
    x[2, 2000] = float("inf")
    ids, lp, lse = (t.cpu().numpy() for t in _top(B, torch, x, 5))
    assert ids[0, 0] == 700 and np.isnan(lse[0]) and np.isnan(lp[0]).all()
    assert ids[1, 0] == 5 and lse[1] == np.inf and np.isnan(lp[1, 0]) and (lp[1, 1:] == -np.inf).all()
    assert list(ids[2, :2]) == [10, 2000] and lse[2] == np.inf
    want, _, _ = _top_reference(x[3:].cpu().numpy(), 5)
    assert np.array_equal(ids[3:], want)


@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 5), (0, 8)])
@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_top_strides_streams_and_graphs(B, offset, pad, dtype):
    import torch
    rows, vocab, k = 6, 10007, 30
    t = torch.full((rows * (vocab + pad) + offset,), float("inf"), dtype=getattr(torch, dtype), device="cuda")
    logits = t[offset:].view(rows, vocab + pad)[:, :vocab]
    logits.copy_(torch.randn(rows, vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)))
    _check_top(B, torch, logits, k)
    first = _top(B, torch, logits, k)
    side = torch.cuda.Stream()
    other = _top(B, torch, logits, k, stream=side)
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    ids, lp = torch.zeros_like(first[0]), torch.zeros_like(first[1])
    ws = torch.empty(B.bpe_top_tokens_workspace_bytes(rows, vocab, k), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.bpe_top_tokens(logits, ids, lp, ws)
    for _ in range(3):
        ids.zero_()
        lp.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, first[0]) and torch.equal(lp, first[1])


def test_rows_beyond_32_bits(B):
    """The last row starts behind element 2^32 of the logits."""
    import torch
    rows, vocab = 3, 40000
    stride = (1 << 31) + 24
    whole = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    logits = torch.as_strided(whole, (rows, vocab), (stride, 1))
    rng = np.random.default_rng(1)
    logits.copy_(torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)))
    _check_top(B, torch, logits, 12)
    history = _lists(rng, rows, [5, 6, 700], vocab)
    pres = np.ones(rows, dtype=np.float32)
    want = _reference(logits.float().cpu().numpy(), vocab, history, pres=pres)
    before = logits.clone()
    _adjust(B, torch, logits, "bfloat16", vocab, history, pres=pres, out=logits)
    _check_adjusted(logits, before, want, "bfloat16")


def test_no_rows(B):
    import torch
    empty = torch.empty(0, 50, device="cuda")
    B.bpe_adjust_logits(empty, torch.empty(0, 50, device="cuda"))
    B.bpe_top_tokens(empty, torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, 3, device="cuda"),
                     torch.empty(B.bpe_top_tokens_workspace_bytes(0, 50, 3), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_biases_of_few_tokens(B, dtype):
    """Lists of up to 5,000 entries for 300 tokens: the last entry of a token counts, in place too, with penalties and masks."""
    import torch
    rng = np.random.default_rng(21)
    rows, vocab = 4, 20000
    lengths = [5000, 0, 1025, 1024]
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    ids = (rng.integers(0, 300, off[-1]) * 61).astype(np.int32)
    ids[::97] = -4
    bias = (ids, rng.standard_normal(ids.size).astype(np.float32), off)
    history = _lists(rng, rows, [4000, 10, 0, 600], vocab)
    masks = rng.integers(-2**31, 2**31, (rows, (vocab + 31) // 32)).astype(np.int32)
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).cuda().to(getattr(torch, dtype))
    rep, pres = np.full(rows, 1.3, dtype=np.float32), np.full(rows, 0.7, dtype=np.float32)
    want = _reference(logits.float().cpu().numpy(), vocab, history, bias, masks, None, rep, None, pres)
    got = _adjust(B, torch, logits, dtype, vocab, history, bias, masks, None, rep, None, pres)
    _check_adjusted(got, logits, want, dtype)
    again = _adjust(B, torch, logits, dtype, vocab, history, bias, masks, None, rep, None, pres, out=logits)
    assert torch.equal(again, got)


def test_more_rows_than_a_launch_holds(B):
    """A launch has fewer than 2^32 threads: the rows behind that many go into another one."""
    import torch
    rows, vocab = 4200000, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(rows, vocab, generator=g, device="cuda").bfloat16()
    masks = torch.tensor([[0x5A]], dtype=torch.int32, device="cuda")
    out = torch.empty_like(logits)
    B.bpe_adjust_logits(logits, out, masks=masks, mask_index=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    keep = torch.tensor([0x5A >> v & 1 for v in range(vocab)], dtype=torch.bool, device="cuda")
    assert torch.equal(out, torch.where(keep, logits, torch.full_like(logits, float("-inf"))))
    rows = 16800000
    logits = torch.randint(0, 100, (rows, 4), generator=g, device="cuda").bfloat16()
    ids = torch.empty(rows, 1, dtype=torch.int32, device="cuda")
    lp = torch.empty(rows, 1, device="cuda")
    B.bpe_top_tokens(logits, ids, lp, torch.empty(B.bpe_top_tokens_workspace_bytes(rows, 4, 1), dtype=torch.uint8, device="cuda"))
    best = logits.max(1, keepdim=True)
    first = (logits == best.values).int().argmax(1, keepdim=True)
    assert torch.equal(ids.long(), first)
    want = logits.float().log_softmax(1).gather(1, first)
    assert float((lp - want).abs().max()) <= 600 * U + 4 * U * 110


def test_nan_in_many_places(B):
    """Rows of mostly NaN: the lowest indexes of NaN come first, and everything is NaN."""
    import torch
    x = torch.randn(3, 30000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    x[0] = float("nan")
    x[1, 7::2] = float("nan")
    ids, lp, lse = (t.cpu().numpy() for t in _top(B, torch, x, 40))
    assert np.array_equal(ids[0], np.arange(40)) and np.array_equal(ids[1], 7 + 2 * np.arange(40))
    assert np.isnan(lp[:2]).all() and np.isnan(lse[:2]).all() and np.isfinite(lp[2]).all()
