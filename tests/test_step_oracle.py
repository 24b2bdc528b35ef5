"""Pins of the reference of the quantised cache and of the sampling (no GPU)."""
import itertools

import numpy as np
import pytest
import torch

from oracle import step_oracle as so


def test_the_e4m3_numbers():
    v = so.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, t, equal_nan=True)
    assert v[0x7e] == 448 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6


def test_nearest_code_against_every_code():
    v = so.e4m3_values()
    for y in np.concatenate([v[:127], (v[:126] + v[1:127]) / 2, np.linspace(0, 470, 4001), [1e9]]):
        for s in (y, -y):
            c = int(so.nearest_code(np.array([s]))[0])
            off = np.abs(np.abs(v[:127]) - min(abs(s), 448.0))
            assert np.isclose(abs(abs(v[c]) - min(abs(s), 448.0)), off.min(), atol=0)
            if (off == off.min()).sum() == 2:
                assert c % 2 == 0
            assert (c >= 128) == bool(np.signbit(s))
    assert so.nearest_code(np.array([np.nan]))[0] == 0x7f


def test_row_exponent_is_the_smallest_that_holds_the_row():
    rng = np.random.default_rng(1)
    for a in [448.0, 448.0001, 224.0, 1.75, 1.76, 0.0, 2.0 ** -126, 3.38e38, 2.0 ** 119 * 448] + list(2.0 ** rng.uniform(-100, 120, 40)):
        e = int(so.row_exponents(np.array([[a, -a / 3, 0.0]]))[0])
        assert e == so.E_MAX or a <= 448 * 2.0 ** e
        assert e == so.E_MIN or a > 448 * 2.0 ** (e - 1)


def test_read_back_is_within_half_a_step_and_exact_in_bfloat16():
    rng = np.random.default_rng(2)
    x = torch.tensor(rng.standard_normal((50, 64)) * np.exp(rng.uniform(-20, 20, (50, 1)))).to(torch.bfloat16).double().numpy()
    codes, exps = so.quantise_rows(x)
    back = so.read_rows(codes, exps)
    assert np.array_equal(back, torch.tensor(back).to(torch.bfloat16).double().numpy())
    unit = np.abs(x).max(1, keepdims=True)
    assert (np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, unit * 2.0 ** -17)).all()
    again = so.quantise_rows(back)
    assert np.array_equal(so.read_rows(*again), back)  # what has been read back is held exactly


def test_non_finite_values_take_the_nan_code_and_leave_the_others_alone():
    codes, exps = so.quantise_rows(np.array([[1.0, np.inf, np.nan, -np.inf, -0.5]]))
    assert int(exps[0]) - 127 == -8 and list(codes[0, 1:4]) == [0x7f] * 3
    assert so.read_rows(codes, exps)[0, [0, 4]].tolist() == [1.0, -0.5]


def _brute(z, u, T, k, p, m):
    """Subsets and sums spelled out."""
    n = len(z)
    order = sorted(range(n), key=lambda i: (-z[i], i))
    if T <= 0:
        return order[0]
    w = {i: np.exp((z[i] - max(z)) / T) for i in range(n)}
    kept = order[:k] if k > 0 else list(order)
    if p < 1:
        total, mass, prefix = sum(w[i] for i in kept), 0.0, []
        for i in kept:
            prefix.append(i)
            mass += w[i]
            if mass >= p * total:
                break
        kept = prefix
    kept = [i for i in kept if w[i] >= m or i == order[0]]
    total, mass = sum(w[i] for i in kept), 0.0
    for i in sorted(kept):
        mass += w[i]
        if mass > u * total:
            return i
    return max(kept)


def test_sampling_against_spelled_out_sums():
    rng = np.random.default_rng(3)
    for T, k, p, m in itertools.product((0.0, 0.5, 1.3), (0, 1, 3, 40), (1.0, 0.9, 0.37, 1e-9), (0.0, 0.1, 1.0)):
        z = np.round(rng.standard_normal(12) * 2, 1)  # with ties
        u = float(rng.random())
        assert so.sample_token(z, u, T, k, p, m)[0] == _brute(z.tolist(), u, T, k, p, m), (T, k, p, m)


def test_sampling_frequencies_and_borders():
    z = np.array([0.0, np.log(3.0), -np.inf, np.log(6.0)])
    hits = [so.sample_token(z, (i + 0.5) / 1000)[0] for i in range(1000)]
    assert [hits.count(t) for t in range(4)] == [100, 300, 0, 600]
    assert so.sample_token(z, 0.0)[0] == 0 and so.sample_token(z, np.nextafter(1.0, 0.0))[0] == 3
    t, conf, prob = so.sample_token(z, 0.99, top_k=2)
    assert t == 3 and prob == pytest.approx(6 / 9) and conf == pytest.approx(0.6)


def test_sampling_of_rows_without_a_number():
    assert so.sample_token(np.full(5, -np.inf), 0.3) == (-1, 0.0, 0.0)
    assert so.sample_token(np.array([np.nan, -np.inf, 2.0]), 0.3)[0] == 2
    t = [so.sample_token(np.array([np.inf, 0.0, np.inf]), u)[0] for u in (0.2, 0.7)]
    assert t == [0, 2]
