"""Pins of the oracle for the 8-bit floating-point products and the beam search: against torch's e4m3 type, closed forms and
brute force (no GPU)."""
import itertools

import numpy as np
import pytest

import oracle


def test_e4m3_values_and_codes_against_torch():
    import torch
    codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.e4m3_values(), ref, equal_nan=True)
    r = np.random.default_rng(1)
    v = np.concatenate([r.standard_normal(20000) * 10.0 ** r.uniform(-4, 2.4, 20000), ref[np.isfinite(ref)]]).astype(np.float32)
    fin = np.sort(ref[:127])
    v = np.concatenate([v, (fin[1:] + fin[:-1]).astype(np.float32) / 2, -(fin[1:] + fin[:-1]).astype(np.float32) / 2])  # ties
    v = np.clip(v, -448, 448)
    got = oracle.e4m3_codes(v)
    assert np.array_equal(got, torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_quantizer_scales_and_error():
    r = np.random.default_rng(2)
    x = (r.standard_normal((150, 300)) * np.exp(r.standard_normal((150, 1)))).astype(np.float32)
    for br in (1, 128):
        codes, scales = oracle.quantize_fp8(x, br)
        assert scales.shape == (-(-150 // br), 3)
        v = oracle.dequantize_fp8(codes, scales, br)
        s = np.repeat(np.repeat(scales, br, 0)[:150], 128, 1)[:, :300]
        # half a step of 3 mantissa bits, or of the smallest step 2^-9
        assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-6)).all()
        for i, j in itertools.product(range(scales.shape[0]), range(3)):
            assert np.abs(codes[i * br:(i + 1) * br, j * 128:(j + 1) * 128] & 127).max() == 126   # 448 is reached
    codes, scales = oracle.quantize_fp8(np.array([[0.0, -0.0], [1e-44, 0.0], [np.inf, 1.0], [np.nan, 1.0]], np.float32), 1)
    assert np.array_equal(codes[:2], [[0, 128], [0, 0]]) and np.array_equal(scales[:2, 0], [1, 1])
    assert (codes[2:] == 127).all() and np.isnan(scales[2:]).all()


def test_matmul_on_whole_numbers():
    r = np.random.default_rng(3)
    a, b = r.integers(-8, 9, (5, 259)), r.integers(-8, 9, (133, 259))
    x, w = oracle.e4m3_codes(a.astype(float)), oracle.e4m3_codes(b.astype(float))
    xs, ws = 2.0 ** r.integers(-2, 3, (5, 3)), 2.0 ** r.integers(-2, 3, (2, 3))
    y, top = oracle.ref_fp8_matmul(x, xs, w, ws)
    for i, j in itertools.product(range(5), (0, 1, 127, 128, 132)):
        want = sum(xs[i, k // 128] * ws[j // 128, k // 128] * int(a[i, k]) * int(b[j, k]) for k in range(259))
        assert y[i, j] == want and top[i, j] >= abs(want)


def test_select_against_brute_force():
    r = np.random.default_rng(4)
    for trial in range(20):
        b, K, V, count = 2, int(r.integers(1, 4)), int(r.integers(1, 7)), int(r.integers(1, 9))
        x = r.integers(-2, 3, (b, K, V)).astype(np.float32)      # ties in plenty
        x[r.random(x.shape) < 0.2] = -np.inf
        scores = r.integers(-3, 1, (b, K)).astype(np.float32)
        scores[r.random(scores.shape) < 0.2] = -np.inf
        fin = r.random((b, K)) < 0.3
        values, parents, tokens = oracle.ref_beam_select(x, scores, fin, 0, count)
        for i in range(b):
            cands = []
            for k, v in itertools.product(range(K), range(V)):
                if np.isinf(scores[i, k]):
                    continue
                if fin[i, k]:
                    if v == 0:
                        cands.append((-float(scores[i, k]), k, v))
                elif x[i, k, v] > -np.inf:
                    p = np.exp(x[i, k].astype(float))
                    cands.append((-float(scores[i, k] + np.log(p[v] / p.sum())), k, v))
            # equal values may differ in the last place between the two formulas
            cands.sort(key=lambda c: (round(c[0], 9), c[1], c[2]))
            for j in range(count):
                if j < len(cands):
                    assert abs(values[i, j] + cands[j][0]) < 1e-12
                else:
                    assert values[i, j] == -np.inf and parents[i, j] == j % K and tokens[i, j] == 0


def test_select_rows_without_a_distribution_offer_nothing():
    x = np.zeros((1, 5, 3), np.float32)
    x[0, 1, 2], x[0, 2, 0], x[0, 3] = np.nan, np.inf, -np.inf
    values, parents, tokens = oracle.ref_beam_select(x, np.array([[-1.0, 0, 0, 0, np.nan]]), None, 0, 4)
    assert np.allclose(values[0, :3], -1 - np.log(3)) and list(tokens[0]) == [0, 1, 2, 0]
    assert list(parents[0]) == [0, 0, 0, 3] and values[0, 3] == -np.inf


@pytest.mark.parametrize("parents", [[1, 2, 0], [2, 2, 2], [0, 1, 2], [0, 0, 1], [7, 0, -1]])
def test_reorder_by_hand(parents):
    cache = np.arange(6).reshape(1, 3, 2)
    got = oracle.ref_beam_reorder(cache, np.array([parents]))
    for k, p in enumerate(parents):
        assert list(got[0, k]) == list(cache[0, p if 0 <= p < 3 else k])
