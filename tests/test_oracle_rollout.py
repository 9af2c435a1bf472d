"""The rollout oracle against independent forms: rotation matrices, relative positions, a plain masked softmax."""
import numpy as np
import pytest

from oracle import rollout_oracle as ro


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_is_a_rotation_of_each_pair(interleaved):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 12))
    theta, _ = ro.frequencies(8)
    pos = np.array([0, 1, 7, 1000, -3])
    out = ro.rotary(x, pos, theta, interleaved, amplitude=2.0)
    for r in range(5):
        for i in range(4):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 4)
            t = pos[r] * theta[i]
            m = np.array([[np.cos(t), -np.sin(t)], [np.sin(t), np.cos(t)]])
            assert np.allclose(out[r][:, [a, b]].T, 2.0 * m @ x[r][:, [a, b]].T)
    assert np.array_equal(out[..., 8:], x[..., 8:])
    assert np.allclose(ro.rotary(out, pos, theta, interleaved, 0.5, inverse=True), x)


def test_scores_depend_on_distances_only():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 16))
    theta, _ = ro.frequencies(16, scaling=3, factor=8.0, original_len=100.0)
    dot = lambda i, j: float((ro.rotary(q, [i], theta) * ro.rotary(k, [j], theta)).sum())
    assert np.isclose(dot(5, 3), dot(1005, 1003)) and not np.isclose(dot(5, 3), dot(5, 4))


def test_scaled_frequencies():
    plain, _ = ro.frequencies(64)
    assert np.isclose(plain[0], 1.0) and np.isclose(plain[16], 10000.0 ** -0.5)
    linear, _ = ro.frequencies(64, scaling=1, factor=4.0)
    assert np.allclose(linear * 4, plain)
    stretched, _ = ro.frequencies(64, scaling=2, factor=4.0)
    assert np.isclose(stretched[0], plain[0]) and np.isclose(stretched[-1] * 4, plain[-1])
    parts, amp = ro.frequencies(64, scaling=3, factor=4.0, original_len=4096.0)
    assert np.isclose(parts[0], plain[0]) and np.isclose(parts[-1] * 4, plain[-1]) and np.isclose(amp, 0.1 * np.log(4.0) + 1)
    assert np.all((parts <= plain + 1e-15) & (parts >= plain / 4 - 1e-15))


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (5, 2), (100, 3), (4, 50)])
def test_attention_over_pages_is_attention_over_the_sequence(window, sinks):
    rng = np.random.default_rng(2)
    lens, new, page, kv, group, dim = [9, 1, 0, 17], [9, 1, 0, 3], 4, 2, 3, 8
    n_pages = [-(-a // page) for a in lens]
    order = rng.permutation(sum(n_pages))
    table, used = np.full((4, 6), 999), 0
    keys, values = [], []
    k_pages, v_pages = np.full((sum(n_pages), page, kv, dim), np.nan), np.full((sum(n_pages), page, kv, dim), np.nan)
    for s, a in enumerate(lens):
        table[s, :n_pages[s]] = order[used:used + n_pages[s]]
        used += n_pages[s]
        keys.append(rng.standard_normal((a, kv, dim)))
        values.append(rng.standard_normal((a, kv, dim)))
        q_off = np.array([0, a])
        k_pages, v_pages = ro.append(keys[-1], values[-1], k_pages, v_pages, table[s:s + 1], [a], q_off)
    q = rng.standard_normal((sum(new), kv * group, dim))
    q_off = np.concatenate([[0], np.cumsum(new)])
    out, lse, mass, reach = ro.attend(q, k_pages, v_pages, table, lens, q_off, 0.3, window, sinks)
    for s in range(4):
        for i in range(new[s]):
            p = lens[s] - new[s] + i
            j = np.arange(lens[s])
            see = (j <= p) & ((j > p - window) | (j < sinks) if window else True)
            for h in range(kv * group):
                z = np.where(see, 0.3 * keys[s][:, h // group] @ q[q_off[s] + i, h], -np.inf)
                w = np.exp(z - z.max()) / np.exp(z - z.max()).sum()
                assert np.allclose(out[q_off[s] + i, h], w @ values[s][:, h // group])
                assert np.isclose(lse[q_off[s] + i, h], np.log(np.exp(z).sum()))
                assert np.all(mass[q_off[s] + i, h] >= np.abs(out[q_off[s] + i, h]) - 1e-12)


def test_rows_that_see_nothing():
    pages = np.zeros((1, 4, 1, 8))
    out, lse, _, _ = ro.attend(np.ones((3, 1, 8)), pages, pages, np.zeros((1, 1), int), [1], np.array([0, 3]), 1.0)
    assert np.all(out[:2] == 0) and np.all(np.isneginf(lse[:2])) and np.isfinite(lse[2]).all()
