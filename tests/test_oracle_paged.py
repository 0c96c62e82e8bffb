"""Pins of the oracle over caches of pages, and of the frequencies that the library computes on the host.  CPU only."""
import cmath
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from oracle import seka_oracle


def _pool(seed, pages=9, ps=4, H=2, D=6):
    g = np.random.default_rng(seed)
    return g, g.standard_normal((pages, ps, H, D)), g.standard_normal((pages, ps, H, D)), g.random((pages, H, ps))


def test_rotary_is_a_complex_product():
    g = np.random.default_rng(0)
    x, f = g.standard_normal((3, 2, 8)), [0.5, 0.01, 2.0]
    for interleaved in (False, True):
        y = orc.rotary(x, [0, 5, -7], f, interleaved, 1.5)
        for t, p in enumerate([0, 5, -7]):
            for i in range(3):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, 3 + i)
                z = complex(x[t, 1, a], x[t, 1, b]) * 1.5 * cmath.exp(1j * p * f[i])
                assert abs(complex(y[t, 1, a], y[t, 1, b]) - z) < 1e-12
        assert (y[..., 6:] == x[..., 6:]).all()


def test_rotated_scores_depend_on_the_distance_alone():
    g = np.random.default_rng(1)
    q, k = g.standard_normal((1, 1, 8)), g.standard_normal((1, 1, 8))
    f = orc.rope_frequencies(8, 10000.0)
    dots = [(orc.rotary(q, [p + 3], f) * orc.rotary(k, [p], f)).sum() for p in (0, 10, 1000)]
    assert max(dots) - min(dots) < 1e-10


def test_chunk_attention_equals_the_causal_one():
    g, K, V, W = _pool(2)
    table = np.array([[3, 1, 8], [0, 5, 2]])
    lens, cu = [9, 11], np.array([0, 4, 15])
    Q = g.standard_normal((15, 4, 6))
    O, L, _, _ = orc.chunk_attention(Q, K, V, table, lens, cu)
    for b, n in ((0, 4), (1, 11)):
        k, v = orc.cached(K, table, b, lens[b])[None], orc.cached(V, table, b, lens[b])[None]
        q = np.zeros((1, lens[b], 4, 6))
        q[0, lens[b] - n:] = Q[cu[b]:cu[b + 1]]
        o, lse = seka_oracle.causal_attention(q, k, v)
        assert np.abs(o[0, lens[b] - n:] - O[cu[b]:cu[b + 1]]).max() < 1e-12
        assert np.abs(lse[0][:, lens[b] - n:] - L[:, cu[b]:cu[b + 1]]).max() < 1e-12


def test_weights_are_column_sums_of_the_softmax():
    g, K, V, W = _pool(3)
    table, lens, cu = np.array([[3, 1, 8]]), [10], np.array([0, 3])
    Q = g.standard_normal((3, 4, 6))
    _, L, _, _ = orc.chunk_attention(Q, K, V, table, lens, cu)
    out, sums = orc.attention_weights(Q, L, K, W, W, table, lens, cu, 3, 0.5)
    w = orc.cached_weights(sums, table, 0, 10)
    assert np.allclose(w.sum(0), 6)                        # two heads, three tokens
    x = torch.from_numpy(np.einsum("ihd,jhd->hij", Q, np.repeat(orc.cached(K, table, 0, 10), 2, 1)) / math.sqrt(6))
    hidden = torch.ones(3, 10).triu(8).bool()
    p = torch.softmax(x.masked_fill(hidden, -math.inf), -1).sum(1)      # [head, key]
    assert np.allclose(w, (p[0::2] + p[1::2]).numpy().T)
    assert np.allclose(orc.cached_weights(out, table, 0, 10), w + 0.5 * orc.cached_weights(W, table, 0, 10))
    last, _ = orc.attention_weights(Q, L, K, W, None, table, lens, cu, 1, 1.0)
    assert np.allclose(orc.cached_weights(last, table, 0, 10).sum(0), 2)


def test_kept_tokens_by_hand():
    inf, nan = math.inf, math.nan
    assert orc.kept_tokens(np.array([1.0, 2, 3]), 3, 3, 0) == [0, 1, 2]
    assert orc.kept_tokens(np.array([5.0, 1, 5, 5, 0]), 5, 3, 1) == [0, 2, 4]          # ties to the earlier one
    assert orc.kept_tokens(np.array([0.0, inf, 2, 1, 9]), 5, 2, 0) == [1, 4]
    assert orc.kept_tokens(np.array([nan, -inf, nan, 0.0]), 4, 3, 1) == [0, 1, 3]
    assert orc.kept_tokens(np.array([nan, nan, -1.0]), 3, 1, 0) == [2]
    assert orc.kept_tokens(np.array([7.0, 7, 7, 7]), 4, 2, 2) == [2, 3]


def test_evicted_rows_by_hand():
    g, K, V, W = _pool(4)
    table, to = np.array([[3, 1, 8]]), np.array([[0, 2]])
    out = orc.evict(K, V, W, K, V, W, table, to, [10], 5, 2)
    assert (out[3][0, 0, 3:] == [8, 9]).all() and out[4] == [5]
    for k, j in enumerate(out[3][0, 1]):
        assert (out[0][to[0, k // 4], k % 4, 1] == K[table[0, j // 4], j % 4, 1]).all()
        assert out[2][to[0, k // 4], 1, k % 4] == W[table[0, j // 4], 1, j % 4]


@pytest.mark.parametrize("scaling,name", [(0, "plain"), (1, "linear"), (2, "base"), (3, "parts"), (4, "turns")])
@pytest.mark.parametrize("dim,base", [(128, 10000.0), (64, 500000.0), (4, 1e6)])
def test_library_frequencies(scaling, name, dim, base):
    from paper_2603_01281_amd import binding as seka
    got = seka.seka_rope_frequencies(dim, base, scaling, stretch=8.0, original=8192.0, fast=4.0, slow=1.0)
    want = orc.rope_frequencies(dim, base, name, 8.0, 8192.0, 4.0, 1.0)
    assert np.allclose(got, want, rtol=1e-12, atol=0)


def test_frequencies_at_the_ends():
    """Pairs that turn often keep their frequency, slow ones are stretched by the whole factor, and stretch 1 changes nothing."""
    for name in ("parts", "turns"):
        f, g = orc.rope_frequencies(128, 10000.0), orc.rope_frequencies(128, 10000.0, name, 8.0)
        assert g[0] == f[0] and abs(g[-1] - f[-1] / 8) < 1e-18
        assert np.allclose(orc.rope_frequencies(128, 10000.0, name, 1.0), f)
    f, g = orc.rope_frequencies(64, 10000.0), orc.rope_frequencies(64, 10000.0, "base", 8.0)
    assert g[0] == f[0] and abs(g[-1] * 8 / f[-1] - 1) < 1e-12      # the base was chosen for this
