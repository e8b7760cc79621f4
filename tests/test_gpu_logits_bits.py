"""bpe_adjust_logits to the bit: the formula in 32 bits, one operation after the other, each rounded by itself, and rounded once more
to the type of the output."""
import numpy as np
import pytest

from test_gpu_logits import _adjust, _lists

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2603_02597_amd as B
    return B


def _formula(x, history, bias, masks, index, rep, freq, pres):
    """float32 [rows, vocab], every operation in np.float32."""
    v = x.copy()
    rows, vocab = x.shape
    assert v.dtype == rep.dtype == freq.dtype == pres.dtype == np.float32
    for r in range(rows):
        h = history[0][history[1][r]:history[1][r + 1]]
        ids, c = np.unique(h[(h >= 0) & (h < vocab)], return_counts=True)
        y = v[r, ids]
        y = np.where(y > 0, y / rep[r], y * rep[r])
        y = y - freq[r] * c.astype(np.float32)
        v[r, ids] = y - pres[r]
        last = {int(bias[0][i]): bias[1][i] for i in range(bias[2][r], bias[2][r + 1]) if 0 <= bias[0][i] < vocab}
        for i, b in last.items():
            v[r, i] = v[r, i] + b
        if index[r] >= 0:
            bits = np.unpackbits(masks[index[r]].view(np.uint8), bitorder="little")[:vocab]
            v[r, bits == 0] = -np.inf
    return v


@pytest.mark.parametrize("rows,vocab,most", [(1, 1, 5), (1, 50256, 700), (5, 4097, 3000), (33, 1256, 900), (3, 100257, 20000), (130, 9001, 400)])
@pytest.mark.parametrize("dtype,out", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("spread", [5.0, 1e-38, 3e4])
def test_every_bit(B, rows, vocab, most, dtype, out, spread):
    import torch
    rng = np.random.default_rng([rows, vocab])
    print(f"[case] adjust bits {rows} {vocab} {dtype} {out} {spread}", flush=True)
    logits = torch.from_numpy((rng.standard_normal((rows, vocab)) * spread).astype(np.float32)).to(getattr(torch, dtype))
    history = _lists(rng, rows, rng.integers(0, most, rows), vocab)
    ids, off = _lists(rng, rows, rng.integers(0, max(most // 4, 2), rows), vocab, 2)
    bias = (ids, rng.standard_normal(ids.size).astype(np.float32) * np.float32(spread), off)
    masks = rng.integers(-2**31, 2**31, (3, (vocab + 31) // 32)).astype(np.int32)
    masks[1] = -1
    index = rng.integers(-1, 3, rows).astype(np.int32)
    rep = rng.uniform(0.6, 1.9, rows).astype(np.float32)
    freq = (rng.uniform(-0.3, 0.7, rows) * spread).astype(np.float32)
    pres = (rng.uniform(-0.5, 1.5, rows) * spread).astype(np.float32)
    got = _adjust(B, torch, logits.cuda(), out, vocab, history, bias, masks, index, rep, freq, pres).cpu()
    want = torch.from_numpy(_formula(logits.float().numpy(), history, bias, masks, index, rep, freq, pres)).to(getattr(torch, out))
    bits = torch.int32 if out == "float32" else torch.int16
    differ = got.view(bits) != want.view(bits)
    assert not differ.any(), (int(differ.sum()), got[differ][:4], want[differ][:4])
