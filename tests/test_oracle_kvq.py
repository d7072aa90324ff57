"""Pins of the 8-bit cache's oracle: closed forms of the rounding and the scale, and attention on textbook cases."""
import numpy as np
import pytest
import torch

from oracle import kvq as O
from oracle import logprobs as L


def test_rounding_matches_the_type():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    values = np.unique(codes[np.isfinite(codes)])
    assert np.array_equal(O.round_e4m3(values), values)
    mid = (values[1:] + values[:-1]) / 2
    got = O.round_e4m3(mid)
    assert np.array_equal(got, torch.from_numpy(mid).float().to(torch.float8_e4m3fn).double().numpy())    # midpoints are exact in float32
    x = np.random.default_rng(0).uniform(-448, 448, 4000)
    assert np.all(np.abs(O.round_e4m3(x) - x) <= np.abs(x[:, None] - values).min(1) * (1 + 1e-12))


@pytest.mark.parametrize("a,e", [(0.0, -15), (448.0, 0), (448.0001, 1), (447.9, 0), (224.0, -1), (1.75, -8), (1.76, -7), (57344.0, 7), (1e-9, -15)])
def test_exponent(a, e):
    assert O.exponent(a) == e


def test_values_are_exact_in_float16_and_bfloat16():
    grid = np.unique(np.concatenate([O.round_e4m3(np.linspace(-448, 448, 5001)) * 2.0 ** e for e in range(O.E_MIN, O.E_MAX + 1)]))
    t = torch.from_numpy(grid)
    assert torch.equal(t.half().double(), t) and torch.equal(t.bfloat16().double(), t)


def test_a_larger_scale_keeps_older_rows_up_to_subnormals():
    s = O.Slot(1, 4, 64)
    s.write(0, np.array([[[1.0, 0.3, 1e-3, -2.0]]]))
    before = s.read(0, 1).copy()
    s.write(1, np.full((1, 1, 4), 100.0))
    assert s.e[0, 0] == -2
    big = np.abs(before) >= 2.0 ** -6 * 2.0 ** -2
    assert np.array_equal(s.read(0, 1)[big], before[big])
    assert np.abs(s.read(0, 1) - before).max() <= 2.0 ** -10 * 2.0 ** -2


def test_attention_of_equal_scores_is_the_mean_of_what_is_visible():
    v = np.random.default_rng(1).normal(size=(5, 2, 4))
    out, mag, _ = O.attention(np.zeros((2, 4, 4)), np.ones((5, 2, 4)), v, 3)
    assert np.allclose(out[0, 3], v[:4, 1].mean(0)) and np.allclose(out[1, 0], v[:5, 0].mean(0))
    assert np.allclose(mag[1, 0], np.abs(v[:5, 0]).mean(0))


def test_logprobs_against_torch_and_closed_forms():
    z = np.random.default_rng(2).normal(size=50)
    lp = torch.log_softmax(torch.from_numpy(z) / 0.7, 0).numpy()
    a, h, top, lt = L.row(z, 7, 0.7, 5)
    assert np.isclose(a, lp[7]) and np.isclose(h, -(np.exp(lp) * lp).sum()) and np.allclose(lt, np.sort(lp)[::-1][:5])
    assert L.row(np.zeros(8), 3, 2.0, 3)[1] == pytest.approx(np.log(8)) and list(L.row(np.zeros(8), 3, 2.0, 3)[2]) == [0, 1, 2]
    a, h, top, lt = L.row([-np.inf, 1.0, -np.inf], 0, 1.0, 2)
    assert a == -np.inf and h == 0.0 and list(top) == [1, -1] and lt[0] == 0.0 and lt[1] == -np.inf
    a, h, top, lt = L.row([-np.inf] * 3, 1, 1.0, 1)
    assert a == -np.inf and h == 0.0 and list(top) == [-1]
    assert np.isnan(L.row([0.0, np.nan], 0, 1.0, 1)[0])
