"""The choice of tiles of bpe_linear, restated from its description: which kernel a product of given sizes takes."""
import math
import os
import re

from conftest import ROOT

SOURCE = os.path.join(ROOT, "paper_2603_02597_amd", "csrc", "bpe_linear.hip")
ROWS, SIMPLE = "rows", "simple"          # linear_rows_kernel, linear_tile_kernel


def tiles():
    """(bm, bn, resident, us for a block, us for a tile, TFLOP/s) of every tile, as the source has them."""
    text = open(SOURCE).read()
    rows = re.findall(r"\{(\d+), (\d+), (\d+), ([\d.]+), ([\d.]+), (\d+)\}", text[text.index("kLinearTiles[] = {"):])
    return [(int(a), int(b), int(c), float(d), float(e), float(f)) for a, b, c, d, e, f in rows]


def plan(m, n, k, aligned=True):
    """(tile's index or ROWS or SIMPLE, parts of k)"""
    best, least, blocks = (0, 1), math.inf, max((k + 63) // 64, 1)
    if m <= 4 or (m <= 16 and n * k <= 1 << 24):
        best = (ROWS, 1)
    else:
        for t, (bm, bn, resident, block_us, tile_us, tflops) in enumerate(tiles()):
            count = -(-m // bm) * -(-n // bn)
            for splits in (1, 2, 4, 8, 16):
                if splits > 1 and (count * splits > 768 or blocks < 2 * splits):
                    break
                groups, per = count * splits, math.ceil(blocks / splits)
                compute = math.ceil(groups / 256) * per * (2 * bm * bn * 64) / (tflops * 1e6 / 256)
                rounds = groups / (256 * resident)
                wait = math.ceil(rounds) * per * block_us
                spread = 1 + (384 - groups) / 1230 if groups < 384 else 1.0
                memory = (2 * (n * k + m * k) * spread + 3.1 * m * n) / 4.55e6 + 2 * count * (bm + bn) * k / 2.46e7
                join = 3.8 + splits * m * n * 8 / 6.7e6 if splits > 1 else 0.0
                us = max(compute, wait, memory) + max(rounds, 1.0) * tile_us + join
                if us < least:
                    best, least = (t, splits), us
    if best[0] == ROWS and not aligned and n * k > 1 << 24:
        best = (0, 1)
    if best[0] != ROWS and k < 8:
        return SIMPLE, 1
    return best


def workspace_bytes(m, n, k):
    splits = plan(m, n, max(k, 8))[1] if k >= 8 else 1
    return 4 * splits * m * (-(-n // 4) * 4) if splits > 1 else 0
