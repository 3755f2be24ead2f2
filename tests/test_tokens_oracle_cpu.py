"""The oracle's token operators against closed forms and against loops over their definitions."""
import math

import numpy as np
import pytest

import oracle


def test_activations_at_known_values():
    v = np.array([-40.0, -1.0, 0.0, 0.5, 1.0, 30.0])
    assert np.array_equal(oracle.activation(v, "none"), v)
    assert np.array_equal(oracle.activation(v, "relu"), [0, 0, 0, 0.5, 1, 30])
    assert abs(oracle.activation(np.array([1.0]), "gelu")[0] - 0.8413447460685429) < 1e-15        # the normal distribution at 1
    assert abs(oracle.activation(np.array([1.0]), "silu")[0] - 1 / (1 + math.exp(-1))) < 1e-15
    for act in ("gelu", "gelu_tanh", "silu"):
        y = oracle.activation(v, act)
        assert y[2] == 0.0 and abs(y[0]) < 1e-15 and abs(y[5] - 30.0) < 1e-11
        d = oracle.activation(np.linspace(-6, 6, 101), act) - oracle.activation(-np.linspace(-6, 6, 101), act)
        assert np.allclose(d, np.linspace(-6, 6, 101), atol=1e-14)                                 # a(v) - a(-v) = v


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_linear_against_loops(act):
    rng = np.random.default_rng(1)
    x, w, b, r = rng.normal(size=(3, 5)), rng.normal(size=(4, 5)), rng.normal(size=4), rng.normal(size=(3, 4))
    got = oracle.linear(x, w, b, r, act)
    for m in range(3):
        for n in range(4):
            v = b[n] + math.fsum(x[m, k] * w[n, k] for k in range(5))
            assert abs(got[m, n] - (oracle.activation(np.array([v]), act)[0] + r[m, n])) < 1e-13


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_turns_pairs(interleaved):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(2, 3, 2, 10))
    pos = rng.integers(-50, 50, size=(2, 3, 2))
    freq, sections = np.array([1.0, 0.3, 0.01, 0.5]), [3, 1]
    y = oracle.rope_axes(x, pos, freq, sections, interleaved)
    assert np.array_equal(y[..., 8:], x[..., 8:])                                                  # beyond the pairs: copied
    for b in range(2):
        for l in range(3):
            for p in range(4):
                u, v = (2 * p, 2 * p + 1) if interleaved else (p, 4 + p)
                z = (x[b, l, :, u] + 1j * x[b, l, :, v]) * np.exp(1j * pos[b, l, 0 if p < 3 else 1] * freq[p])
                assert np.allclose(y[b, l, :, u], z.real, atol=1e-13) and np.allclose(y[b, l, :, v], z.imag, atol=1e-13)
    assert np.allclose(oracle.rope_axes(y, pos, -freq, sections, interleaved), x, atol=1e-13)      # turned back


def test_rope_scores_depend_on_differences_of_positions():
    rng = np.random.default_rng(3)
    q, k = rng.normal(size=(1, 1, 1, 8)), rng.normal(size=(1, 1, 1, 8))
    f = np.array([1.0, 0.1, 1.0, 0.1])
    turn = lambda t, p: oracle.rope_axes(t, np.array([[p]]), f, [2, 2], False)
    a = (turn(q, (5, 9)) * turn(k, (2, 30))).sum()
    b = (turn(q, (105, 2)) * turn(k, (102, 23))).sum()
    assert abs(a - b) < 1e-12


def test_attention_against_loops():
    rng = np.random.default_rng(4)
    B, Lq, Lk, Hq, Hkv, D = 2, 3, 7, 4, 2, 8
    q, k, v = rng.normal(size=(B, Lq, Hq, D)), rng.normal(size=(B, Lk, Hkv, D)), rng.normal(size=(B, Lk, Hkv, D))
    lens, mask = np.array([5, 7]), rng.random((B, Lk)) < 0.6
    mask[0, 0] = mask[1, 6] = True
    got = oracle.attention(q, k, v, 0.3, lens, mask)
    for b in range(B):
        for i in range(Lq):
            for h in range(Hq):
                seen = [j for j in range(lens[b]) if mask[b, j]]
                e = [math.exp(0.3 * math.fsum(q[b, i, h] * k[b, j, h // 2])) for j in seen]
                want = sum(w * v[b, j, h // 2] for w, j in zip(e, seen)) / math.fsum(e)
                assert np.allclose(got[b, i, h], want, atol=1e-13)


def test_attention_masks():
    rng = np.random.default_rng(5)
    q, k, v = rng.normal(size=(3, 2, 1, 8)), rng.normal(size=(3, 4, 1, 8)), rng.normal(size=(3, 4, 1, 8))
    k[:, 3], v[:, 3] = np.nan, np.inf                                                              # not visible: no influence
    got = oracle.attention(q, k, v, 1.0, [0, 1, 3])
    assert not got[0].any()                                                                        # nothing visible
    assert np.allclose(got[1], np.broadcast_to(v[1, 0], got[1].shape))                             # one key: its value
    assert np.isfinite(got[2]).all()
    assert not oracle.attention(q, k, v, 1.0, None, np.zeros((3, 4), bool)).any()
    same = np.broadcast_to(rng.normal(size=(3, 1, 1, 8)), (3, 4, 1, 8))
    assert np.allclose(oracle.attention(q, same, v[:, :3][:, [0, 1, 2, 0]], 1.0)[:, 0, 0], (2 * v[:, 0, 0] + v[:, 1, 0] + v[:, 2, 0]) / 4)
