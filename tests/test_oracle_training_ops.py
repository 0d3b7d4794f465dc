"""Pins of the oracle's dropout, LayerNorm and relative-bias attention: published vectors of the generator, central differences, closed forms."""
import math

import numpy as np
import pytest

from oracle import training_ops as T


def test_generator_gives_the_published_vectors():
    f = lambda c, k: [int(w) for w in T.philox4x32(c, k)]  # noqa: E731
    assert f((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    m = 0xFFFFFFFF
    assert f((m, m, m, m), (m, m)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_kept_share_and_independence_of_site_step_and_seed():
    n = 1 << 18
    masks = [T.keep_mask(512, 512, 0.25, seed, step, site) for seed, step, site in ((1, 0, 0), (2, 0, 0), (1, 1, 0), (1, 0, 1), (1 << 32, 0, 0))]
    sd = math.sqrt(0.25 * 0.75 / n)
    for m in masks:
        assert abs(m.mean() - 0.75) < 5 * sd
    for i in range(len(masks)):
        for j in range(i):
            assert abs((masks[i] & masks[j]).mean() - 0.75 ** 2) < 5 * math.sqrt(0.5625 * 0.4375 / n)


def test_a_slice_drops_what_the_whole_drops():
    whole = T.keep_mask(40, 37, 0.3, 77, 5, 2)
    assert np.array_equal(T.keep_mask(9, 37, 0.3, 77, 5, 2, first_row=13), whole[13:22])
    assert np.array_equal(T.keep_mask(40, 20, 0.3, 77, 5, 2), whole[:, :20])
    assert T.keep_mask(3, 9, 0.0, 1, 1, 1).all() and not T.keep_mask(3, 9, 1.0, 1, 1, 1).any()


def _difference(f, x, dy, eps=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + eps
        hi = (f() * dy).sum()
        x[i] = old - eps
        lo = (f() * dy).sum()
        x[i] = old
        g[i] = (hi - lo) / (2 * eps)
    return g


def test_layernorm_gradients_against_differences():
    r = np.random.default_rng(0)
    s, gamma, beta, dy = r.normal(size=(3, 7)) + 1.0, r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    f = lambda: T.layernorm_fwd(s, gamma, beta, 1e-3)[0]  # noqa: E731
    _, mean, rstd = T.layernorm_fwd(s, gamma, beta, 1e-3)
    for got, x in zip(T.layernorm_bwd(dy, s, mean, rstd, gamma), (s, gamma, beta)):
        assert np.abs(got - _difference(f, x, dy)).max() < 1e-7


def test_buckets_of_known_distances():
    # 32 buckets, both directions, 128: distances 0..7 one each, then doublings in two steps: 8, 12 (11.3), 16, 23 (22.6), 32, 46 (45.3), 64, 91 (90.5)
    b = lambda n: T.bucket(n, 32, 128, True)  # noqa: E731
    starts = [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]
    for k, n in enumerate(starts):
        assert b(-n) == k and (k == 0 or b(-n + 1) == k - 1)
        assert n == 0 or b(n) == 16 + k
    assert b(-100000) == 15 and b(100000) == 31
    # one direction: keys behind the query share bucket 0
    assert [T.bucket(n, 32, 128, False) for n in (5, 1, 0, -1, -15, -16, -127, -128, -5000)] == [0, 0, 0, 1, 15, 16, 31, 31, 31]


@pytest.mark.parametrize("causal,query0,key_len", [(False, 0, None), (True, 0, None), (True, -2, None), (False, 3, [5, 0]), (True, 2, [4, 7])])
def test_attention_gradients_against_differences(causal, query0, key_len):
    r = np.random.default_rng(1)
    q, k, v = (r.normal(size=(2, 2, n, 3)) for n in (5, 7, 7))
    table, do = r.normal(size=(6, 2)), r.normal(size=(2, 2, 5, 3))
    bk = T.buckets(5, 7, query0, 6, 9, True)
    call = lambda: T.attention_relbias_fwd(q, k, v, 0.6, table, bk, causal, query0, key_len)  # noqa: E731
    o, lse = call()
    got = T.attention_relbias_bwd(q, k, v, o, lse, do, 0.6, table, bk, causal, query0, key_len)
    for g, x in zip(got, (q, k, v, table)):
        assert np.abs(g - _difference(lambda: call()[0], x, do)).max() < 1e-7
    if query0 == -2:
        assert (o[:, :, :2] == 0).all() and np.isneginf(lse[:, :, :2]).all()
    if key_len == [5, 0]:
        assert (o[1] == 0).all() and (got[1][0, :, 5:] == 0).all() and (got[1][1] == 0).all()


def test_entries_of_minus_65536_and_less_mask():
    r = np.random.default_rng(3)
    q, k, v = (r.normal(size=(1, 1, 4, 3)) for _ in range(3))
    bk = T.buckets(4, 4, 0, 4, 8, True)
    table = r.normal(size=(4, 1))
    for x in (-65536.0, -1e30, -np.inf):
        table[3] = x
        o, lse = T.attention_relbias_fwd(q, k, v, 0.5, table, bk)
        s = np.where(bk == 3, -np.inf, 0.5 * q[0, 0] @ k[0, 0].T + table[bk][..., 0])
        w = np.exp(s) / np.exp(s).sum(-1, keepdims=True)
        np.testing.assert_allclose(o[0, 0], w @ v[0, 0], rtol=1e-13)
