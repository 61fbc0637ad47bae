"""Pins of the oracles of the draws and the block matrices that do not depend on them."""
import math

import numpy as np
import pytest
import torch

from oracle import blocks, draws


def test_e4m3_table():
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every, blocks.E4M3) and blocks.E4M3[-1] == 448


def test_rounding_against_the_type():
    t = np.concatenate([np.linspace(-448, 448, 20001), (blocks.E4M3[1:] + blocks.E4M3[:-1]) / 2, [2.0 ** -10, 3 * 2.0 ** -11]])
    want = torch.from_numpy(t).to(torch.float64).to(torch.float32).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(blocks.to_e4m3(t.astype(np.float32).astype(np.float64)), want)


def test_dense_is_near_its_source():
    x = np.random.default_rng(0).normal(size=(130, 200)).astype(np.float32)
    for group in (1, 128):
        for trans in (False, True):
            v, s = blocks.quantize(x, group, trans)
            want = x.T if trans else x
            top = np.abs(want).max()
            assert np.abs(blocks.dense(v, s, want.shape[1]) - want).max() <= top * (2.0 ** -4 + 1e-6)


def test_draw_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    assert draws.draw_row(x, 0.0)[::2] == (0, 4)
    assert draws.draw_row(x, 0.55)[0] == 2 and draws.draw_row(x, 0.75)[0] == 3
    tok, lp, kept = draws.draw_row(x, 0.5, top_k=2)          # columns 1 and 3, 4/7 and 3/7
    assert (tok, kept) == (1, 2) and math.isclose(lp, math.log(4 / 7))
    assert draws.draw_row(x, 0.6, top_k=2)[0] == 3
    assert draws.draw_row(x, 0.9, top_p=0.65)[2] == 2        # 0.4 + 0.3
    assert draws.draw_row(x, 0.9, top_p=0.75)[2] == 3
    assert draws.draw_row(x, 0.9, min_p=0.6)[::2] == (3, 2)
    assert draws.draw_row(x, 0.9, top_k=3, top_p=0.7)[2] == 2  # 0.7 of 0.9
    assert draws.draw_row(x, 0.9, temp=0.0) == (1, 0.0, 1)


@pytest.mark.parametrize("p", (0.1, 0.5, 0.9))
def test_equal_logits_keep_the_first(p):
    tok, lp, kept = draws.draw_row(np.zeros(100), 0.999, top_p=p)
    assert kept == math.ceil(float(np.float32(p)) * 100) and tok == kept - 1 and math.isclose(lp, -math.log(kept))


def test_rows_out_of_play():
    inf = math.inf
    assert draws.draw_row([-inf, -inf], 0.5) == (-1, 0.0, 0)
    assert draws.draw_row([1.0, math.nan], 0.5)[0] == -1
    assert draws.draw_row([1.0, inf, 2.0, inf], 0.6)[::2] == (3, 4)
    assert draws.draw_row([1.0], 1.0) == (-1, 0.0, 0)


def test_frequencies():
    x = np.random.default_rng(1).normal(size=12)
    u = (np.arange(4000) + 0.5) / 4000
    toks = [draws.draw_row(x, v, temp=0.7, top_k=5)[0] for v in u]
    top = np.argsort(-x)[:5]
    q = np.exp(x[top] / 0.7) / np.exp(x[top] / 0.7).sum()
    assert np.abs(np.bincount(toks, minlength=12)[top] / 4000 - q).max() < 1e-3
