"""The float64 oracle of the serving path against definitions written another way."""
import numpy as np
import pytest
import torch

from oracle import serving as so


def test_round_e4m3_is_the_nearest_value_with_ties_to_even():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    values = np.unique(codes[np.isfinite(codes)])
    assert values.max() == 448.0 and len(values) == 253   # 254 finite codes, two of them zero
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(-448, 448, 2000), np.exp2(rng.uniform(-14, 8, 2000)), values, (values[1:] + values[:-1]) / 2])
    got = so.round_e4m3(x)
    off = np.abs(x[:, None] - values[None])
    assert np.array_equal(np.abs(x - got), off.min(1))
    # of two values equally far, the one with the even mantissa
    tied = (off == off.min(1, keepdims=True)).sum(1) == 2
    assert tied.sum() >= len(values) - 1
    bits = torch.from_numpy(got[tied]).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert not (bits & 1).any()
    assert np.isnan(so.round_e4m3(np.array([np.nan, np.inf, -np.inf]))).all()


@pytest.mark.parametrize("scale", [1.0, 1e-30, 1e30, 2.0 ** -133])
def test_quantise_rows_takes_the_smallest_power_of_two(scale):
    rng = np.random.default_rng(2)
    x = np.float32(rng.standard_normal((200, 24)) * scale).astype(np.float64)
    x[0] = 0.0
    x[1] = 448.0 * 2.0 ** -20
    x[2] = np.nextafter(np.float32(448.0 * 2.0 ** -20), np.float32(1)).astype(np.float64)
    x[3, 5] = np.nan
    x[4, 7] = np.inf
    codes, e = so.quantise_rows(x)
    top = np.where(np.isfinite(x), np.abs(x), 0).max(-1)
    assert (top <= 448.0 * 2.0 ** (e - 127.0)).all()
    assert ((e == 0) | (top > 448.0 * 2.0 ** (e - 128.0))).all()
    assert e[0] == 0 and e[1] == 107 and e[2] == 108
    back = so.dequantise_rows(codes, e)
    fine = np.isfinite(x)
    assert np.isnan(back[~fine]).all() and (~fine).sum() == 2
    # half a step: 2^-4 of the value, or of the smallest normal 2^-6
    bound = np.maximum(np.abs(x), 2.0 ** -6 * 2.0 ** (e[:, None] - 127.0)) * 2.0 ** -4
    assert (np.abs(back - x)[fine] <= bound[fine]).all()


def test_attention_against_scalar_loops():
    rng = np.random.default_rng(3)
    heads, hk, d = 4, 2, 8
    offsets, length, tokens = [0, 3, 3, 4, 9], [5, 2, 1, 3], 10
    Q = rng.standard_normal((tokens, heads, d))
    keys = [rng.standard_normal((m, hk, d)) for m in (5, 2, 1, 3)]
    values = [rng.standard_normal((m, hk, d)) for m in (5, 2, 1, 3)]
    for causal in (True, False):
        O, A, reach, top = so.attention(Q, keys, values, offsets, length, causal, 0.0)
        for s in range(4):
            n = offsets[s + 1] - offsets[s]
            for i in range(n):
                t, pos = offsets[s] + i, length[s] - n + i
                for h in range(heads):
                    see = [j for j in range(len(keys[s])) if not causal or j <= pos]
                    num, den = np.zeros(d), 0.0
                    for j in see:
                        w = np.exp(sum(Q[t, h, c] * keys[s][j, h // 2, c] for c in range(d)) / d ** 0.5)
                        num, den = num + w * values[s][j, h // 2], den + w
                    want = num / den if see else np.zeros(d)
                    assert np.allclose(O[t, h], want, rtol=1e-12, atol=1e-14)
        assert np.isnan(O[9]).all()          # outside every sequence
        if causal:
            assert (O[4:6] == 0).all()       # 5 new tokens, 3 positions: the first two have none


def test_places_and_bounds():
    assert so.bounds([0, 4, 2, 99, -3], 10) == [(0, 4), (4, 0), (2, 8), (10, 0)]
    assert so.place([3, -1, 9], 5, 4, 9) is None and so.place([3, 1, 9], 5, 4, 9) == (1, 1)
    assert so.place([3, 1, 9], 8, 4, 9) is None and so.place([3], 4, 4, 9) is None and so.place([3], -1, 4, 9) is None
