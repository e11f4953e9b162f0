"""Pins of the attention oracle: torch's own e4m3 conversion, brute force over the scale, an orthogonal rotation, a softmax by hand."""
import numpy as np
import torch

from oracle import attention as oracle


def test_codes_are_those_of_torch():
    v = oracle.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(v, t)
    fine = v[~np.isnan(v)]
    middles = (np.sort(fine)[1:] + np.sort(fine)[:-1]) / 2
    x = np.concatenate([fine, middles, np.random.default_rng(0).normal(size=5000) * 100]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    np.testing.assert_array_equal(oracle.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert (oracle.e4m3([np.nan, np.inf]) == 127).all()


def test_the_scale_is_the_smallest_power_of_two():
    x = np.concatenate([np.exp(np.random.default_rng(1).normal(size=200) * 20), 448 * 2.0 ** np.arange(-30, 30), np.nextafter(448 * 2.0 ** np.arange(-30, 30), np.inf)])
    s = oracle.scale_for(x)
    assert (x <= 448 * s).all() and ((x > 448 * s / 2) | (s == 2.0 ** -100)).all() and (np.log2(s) % 1 == 0).all()
    assert oracle.scale_for(0.0) == 2.0 ** -100


def test_rotation_keeps_lengths_and_depends_on_differences_only():
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=(2, 64))
    freq = 10000.0 ** (-np.arange(16) / 16)
    for interleaved in (False, True):
        turn = lambda x, p: oracle.rotate(x, np.cos(p * freq), np.sin(p * freq), interleaved)
        assert np.isclose(turn(q, 9) @ turn(k, 4), turn(q, 25) @ turn(k, 20))
        assert np.isclose(np.linalg.norm(turn(q, 7)), np.linalg.norm(q)) and np.array_equal(turn(q, 7)[32:], q[32:])


def test_layouts_and_their_inverses():
    c = np.arange(64 * 128).reshape(64, 128)
    k, v = oracle.keys_page(c), oracle.values_page(c)
    assert k[1 * 4096 + 5 * 64 + 3] == c[5, 67] and v[2 * 2048 + 100 * 16 + 7] == c[39, 100]
    np.testing.assert_array_equal(oracle.from_keys_page(k, 128), c)
    np.testing.assert_array_equal(oracle.from_values_page(v, 128), c)


def test_attention_by_hand():
    q, k, v = np.array([[[1.0, 0.0]], [[0.0, 1.0]]]), np.array([[[0.0, 0.0]], [[0.0, np.log(3.0)]]]), np.array([[[2.0, 4.0]], [[6.0, -4.0]]])
    out, mass, _ = oracle.attention(q, k, v, 1.0)
    np.testing.assert_allclose(out[:, 0], [[2.0, 4.0], [5.0, -2.0]])
    np.testing.assert_allclose(mass[1, 0], [5.0, 4.0])
    assert (oracle.attention(q, k[:1], v[:1], 1.0)[0][0] == 0).all()
