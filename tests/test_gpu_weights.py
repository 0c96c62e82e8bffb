"""seka_attention_weights against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import paged_helpers as P

pytestmark = pytest.mark.gpu


def check(seka, x, what, window=None, decay=1.0, with_in=True, in_place=False, scale=0.0):
    print(what, flush=True)
    s = scale or None
    _, L, _, size = orc.chunk_attention(x.Q, x.K, x.V, x.table, x.lens, x.cu, scale=s)
    L32 = L.astype(np.float32)
    win = window or max(x.new)
    W0 = x.W if in_place else np.full_like(x.W, 5.0)
    cache = x.cache(seka, W=W0)
    W_in = None
    if with_in:
        W_in = cache.W if in_place else torch.from_numpy(x.W).cuda()
    seka.seka_attention_weights(x.dev(x.Q), torch.from_numpy(L32).cuda(), cache, x.cu_dev, max(max(x.new), 1), window=window, W_in=W_in, decay=decay, scale=scale)
    got = P.f64(cache.W)
    want, sums = orc.attention_weights(x.Q, L32.astype(np.float64), x.K, W0.astype(np.float64), x.W.astype(np.float64) if with_in else None, x.table, x.lens,
                                       x.cu, win, decay, scale=s)
    # an exponential is off by its argument's error: the score's, and two steps of lse and of their difference; and by 2^-21 itself.  Sums and the
    # decayed old weight: fp32, chains of at most a few hundred terms
    top = np.abs(L[np.isfinite(L)]).max() if np.isfinite(L).any() else 0.0
    rel = 2 * P.score_error(size.max(), x.D) + 2.0 ** -22 * (top + 1) * 1.5 + 2.0 ** -21 + (16 + max(x.new) * x.Hq / x.Hkv / 4) * 2.0 ** -24
    bound = rel * sums + 2.0 ** -22 * np.abs(want)
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), f"{what}: off by {np.abs(got - want).max():.3g}, {off.max():.3g} more than it may be"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (7, 1), (3, 3), (40, 2)])
def test_single_tokens(seka, dtype, D, Hq, Hkv):
    lens = [1, 2, 16, 17, 63, 64, 65, 255, 256, 257, 700]
    check(seka, P.Pages(dtype, [1] * len(lens), lens, Hq, Hkv, D, 16, seed=D), f"weights of single tokens {dtype} {D} {Hq}/{Hkv}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [8, 32, 256])
@pytest.mark.parametrize("new,lens", [([1], [1]), ([64], [64]), ([33, 1, 100], [33, 400, 260]), ([130, 7], [200, 64]), ([0, 20], [70, 400])])
def test_chunks(seka, dtype, ps, new, lens):
    for Hq, Hkv, D in ((4, 1, 128), (6, 2, 64)):
        check(seka, P.Pages(dtype, new, lens, Hq, Hkv, D, ps, seed=sum(lens)), f"weights of chunks {dtype} {ps} {new} {lens} {Hq}/{Hkv}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 7, 16, 64, 1000])
def test_windows(seka, dtype, window):
    check(seka, P.Pages(dtype, [90, 3], [300, 80], 4, 2, 64, 16, seed=2), f"window {window} {dtype}", window=window)


@pytest.mark.parametrize("kw", [dict(decay=0.5), dict(decay=0.0), dict(with_in=False), dict(in_place=True, decay=0.9), dict(scale=0.3)])
def test_decay_and_places(seka, kw):
    check(seka, P.Pages("bf16", [1, 30, 80], [99, 30, 333], 4, 2, 128, 16, seed=3), f"weights {kw}", **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_that_see_nothing_count_nothing(seka, dtype):
    check(seka, P.Pages(dtype, [20, 3, 70], [7, 0, 64], 4, 2, 128, 16, seed=4), f"weights of nothing {dtype}")


def test_infinite_weights_stay(seka):
    """+inf of highlighted tokens stays +inf; decay 0 forgets it without reading."""
    x = P.Pages("bf16", [1], [50], 2, 1, 64, 16, seed=5)
    x.W[x.table[0, 1], 0, 3] = np.inf
    cache = x.cache(seka, W=np.zeros_like(x.W))
    q, lse = x.dev(x.Q), torch.zeros((2, 1), device="cuda")
    W_in = torch.from_numpy(x.W).cuda()
    seka.seka_attention_weights(q, lse, cache, x.cu_dev, 1, W_in=W_in, decay=0.9)
    assert torch.isinf(cache.W).sum() == 1
    seka.seka_attention_weights(q, lse, cache, x.cu_dev, 1, W_in=W_in, decay=0.0)
    assert torch.isfinite(cache.W).all()


@pytest.mark.parametrize("new", [1, 60])
def test_sums_to_the_number_of_queries(seka, new):
    """With the attention's own lse, a request's weights add up to its queries: heads of the group times tokens."""
    x = P.Pages("bf16", [new, 2], [900, 300], 8, 2, 128, 16, seed=6)
    cache = x.cache(seka, W=np.zeros_like(x.W))
    q = x.dev(x.Q)
    O, L = torch.empty_like(q), torch.empty((8, x.total), device="cuda")
    seka.seka_attention_chunk(q, O, cache, x.cu_dev, max(new, 2), lse=L)
    seka.seka_attention_weights(q, L, cache, x.cu_dev, max(new, 2))
    for b, n in ((0, new), (1, 2)):
        got = orc.cached_weights(P.f64(cache.W), x.table, b, x.lens[b]).sum(0)
        assert np.abs(got - 4 * n).max() <= 4 * n * 1e-5


def test_lengths_out_of_range(seka):
    x = P.Pages("bf16", [1, 1], [60, 40], 2, 1, 64, 16, seed=7, wild=False)
    x.lens, x.table[:] = [1 << 30, -1], 1 << 30
    x.cu = np.array([-4, 1 << 30, 7], np.int32)
    cache = x.cache(seka, W=x.W)
    seka.seka_attention_weights(x.dev(x.Q), torch.zeros((2, 2), device="cuda"), cache, x.cu_dev, 1)
    torch.cuda.synchronize()


def test_replays_from_a_graph(seka):
    x = P.Pages("bf16", [1, 40], [500, 300], 8, 2, 128, 16, seed=8, wild=False)
    cache = x.cache(seka, W=np.zeros_like(x.W))
    q, L = x.dev(x.Q), torch.full((8, x.total), 6.0, device="cuda")
    call = lambda: seka.seka_attention_weights(q, L, cache, x.cu_dev, 40)      # noqa: E731
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    for lens in ([500, 300], [16, 40], [333, 290]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        q.neg_()
        cache.W.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = cache.W.clone()
        cache.W.fill_(3.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, cache.W)
