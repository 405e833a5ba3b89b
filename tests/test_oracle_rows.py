"""Pins of the oracle of rows without a tree, and of the library's host side for them (no GPU)."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import rows as O
from paper_2510_13161_b200 import binding


def rope(head_dim=128, rotary_dim=0, interleaved=0, theta=1e4, scaling=0, factor=1.0, original_len=0.0, low=1.0, high=32.0, amplitude=0.0):
    out = binding.Rope()
    code = binding.load_library().mirror_rope_init(C.byref(out), head_dim, rotary_dim, interleaved, theta, scaling, factor, original_len, low, high, amplitude)
    return code, out


@pytest.mark.parametrize("scaling", ["none", "linear", "turns", "pairs"])
@pytest.mark.parametrize("head_dim,rotary", [(64, 0), (64, 16), (128, 0), (128, 96)])
def test_frequencies(head_dim, rotary, scaling):
    r = rotary or head_dim
    code, got = rope(head_dim, rotary, 1, 5e5, binding.ROPE_SCALINGS[scaling], 8.0, 8192.0, 1.0, 4.0 if scaling == "turns" else 32.0, 1.25)
    assert code == 0 and got.rotary_dim == r and got.interleaved == 1 and got.amplitude == 1.25
    want = O.rope_frequencies(r, 5e5, scaling, 8.0, 8192.0, 1.0, 4.0 if scaling == "turns" else 32.0)
    # both are a few correctly rounded double operations and one pow (a few ulps at exponents up to 13)
    np.testing.assert_allclose(list(got.freq)[:r // 2], want, rtol=1e-14)
    assert not any(list(got.freq)[r // 2:])


def test_frequencies_by_hand():
    _, got = rope(64, 0, 0, 10000.0)
    assert got.freq[0] == 1.0 and abs(got.freq[16] - 0.01) < 1e-16 and got.amplitude == 1.0
    # wavelengths far within the lengths seen keep their frequency, far beyond them lose the whole factor
    _, got = rope(128, 0, 0, 1e6, 2, 8.0, 8192.0, 1.0, 4.0)
    assert got.freq[0] == 1.0 and abs(got.freq[63] * 8 / 1e6 ** (-126 / 128) - 1) < 1e-14


def test_rope_refusals():
    lib = binding.load_library()
    assert lib.mirror_rope_init(None, 128, 0, 0, 1e4, 0, 1.0, 0.0, 1.0, 32.0, 0.0) == 1
    assert rope(96)[0] == 3
    for rotary in (-16, 8, 24, 144):
        assert rope(128, rotary)[0] == 2
    assert rope(64, 80)[0] == 2
    for theta in (1.0, 0.0, -5.0, math.inf, math.nan):
        assert rope(theta=theta)[0] == 1
    assert rope(scaling=4)[0] == 1 and rope(scaling=-1)[0] == 1
    for factor in (0.0, -2.0, math.inf, math.nan):
        assert rope(scaling=1, factor=factor)[0] == 1
    for kind in (2, 3):
        assert rope(scaling=kind, factor=4.0, original_len=0.0)[0] == 1
        assert rope(scaling=kind, factor=4.0, original_len=8192.0, low=4.0, high=4.0)[0] == 1
        assert rope(scaling=kind, factor=4.0, original_len=8192.0, low=0.0, high=4.0)[0] == 1
        assert rope(scaling=kind, factor=4.0, original_len=8192.0, low=1.0, high=4.0)[0] == 0
    assert rope(amplitude=-1.0)[0] == 1 and rope(amplitude=math.nan)[0] == 1


def test_null_arguments_are_refused_without_a_gpu():
    lib = binding.load_library()
    assert lib.mirror_kv_append(None, None, None, None, None, 0, 0, None, None, None, 0, 0, None) == 1
    assert lib.mirror_attn_causal(None, None, None, 0, 0, None, None, None, None) == 1
    assert lib.mirror_sample(None, None, 0, 0, *[None] * 11) == 1
    assert lib.mirror_rows_workspace_bytes(None, None, None) == 1


def test_a_turn_keeps_lengths_and_composes():
    rng = np.random.default_rng(0)
    f = O.rope_frequencies(32, 1e4)
    x = rng.standard_normal((5, 2, 64))
    for inter in (False, True):
        a = O.turn(x, [0, 1, 2, 300, 5], f, inter)
        np.testing.assert_allclose(np.linalg.norm(a, axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-13)
        np.testing.assert_array_equal(a[0], x[0])
        np.testing.assert_array_equal(a[..., 32:], x[..., 32:])
        b = O.turn(O.turn(x, [7] * 5, f, inter), [11] * 5, f, inter)
        np.testing.assert_allclose(b, O.turn(x, [18] * 5, f, inter), atol=1e-12)


def test_attention_by_hand():
    """Two tokens ahead, one row; equal scores: the mean of what is seen."""
    k = np.zeros((3, 1, 16, 64))
    v = np.arange(3 * 16, dtype=np.float64).reshape(3, 1, 16, 1) * np.ones(64)
    q = np.ones((2, 2, 64))
    table = np.array([[2, 0]])
    out, lse = O.causal_attention(q, k, v, table, [20], [0, 2], 0, 0, 0.125)
    tokens = np.concatenate([np.arange(32, 48), np.arange(0, 6)])
    assert np.allclose(out[0, 0], tokens[:21].mean()) and np.allclose(out[1, 1], tokens[:22].mean())
    assert np.allclose(lse, [[math.log(21)] * 2, [math.log(22)] * 2])
    out, lse = O.causal_attention(q, k, v, table, [20], [0, 2], 3, 2, 0.125)
    assert np.allclose(out[0, 0], tokens[[0, 1, 18, 19, 20]].mean()) and np.allclose(out[1, 0], tokens[[0, 1, 19, 20, 21]].mean())


def test_sampling_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert O.sample_row(x, u=0.05)[0] == 0 and O.sample_row(x, u=0.11)[0] == 1 and O.sample_row(x, u=0.99)[0] == 3
    t, n, ids, p = O.sample_row(x, top_k=2, u=0.6)
    assert t == 3 and n == 2 and list(ids) == [1, 3] and np.allclose(p, [4 / 7, 3 / 7])
    assert O.sample_row(x, top_p=0.69)[1] == 2 and O.sample_row(x, top_p=0.71)[1] == 3 and O.sample_row(x, top_p=0.0)[1] == 1
    assert O.sample_row(x, min_p=0.51)[1] == 2 and O.sample_row(x, min_p=2.0)[1] == 1
    assert O.sample_row(x, top_k=3, top_p=0.7, min_p=0.1)[1] == 2            # 4/9 + 3/9 = 7/9 >= 0.7
    assert O.sample_row(x, temperature=0.0, u=0.9)[:2] == (1, 1)
    assert O.sample_row(np.full(4, -np.inf))[0] == -1
    assert O.sample_row(np.array([1.0, 1.0, 1.0, 0.0]), top_k=2)[2].tolist() == [0, 1]
    assert O.sample_row(np.array([np.nan, 1.0, np.inf, np.inf]), u=0.7)[:2] == (3, 2)
