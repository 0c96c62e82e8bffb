"""seka_cache_evict against the oracle: whole numbers and copies, compared bit for bit."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import paged_helpers as P

pytestmark = pytest.mark.gpu


def target(x, budget, ps, seed, pool=None):
    """Pages for what stays: a pool of its own, or free pages (numbers) of x's."""
    g = np.random.default_rng(seed)
    pages = [-(-min(n, budget) // ps) for n in x.lens]
    most = max(-(-min(budget, x.max_pages * x.ps) // ps), 1)
    table = np.full((x.B, most), 1 << 30, np.int32)
    order = g.permutation(sum(pages) + 2) if pool is None else np.asarray(pool)
    first = 0
    for b, k in enumerate(pages):
        table[b, :k] = order[first:first + k]
        first += k
    return table, sum(pages) + 2


def check(seka, x, budget, recent, what, ps_to=None, seed=0):
    print(what, flush=True)
    ps_to = ps_to or x.ps
    table_to, n_to = target(x, budget, ps_to, seed)
    K_to, V_to, W_to = x.values(n_to, ps_to, x.Hkv, x.D), x.values(n_to, ps_to, x.Hkv, x.D), np.zeros((n_to, x.Hkv, ps_to), np.float32)
    want = orc.evict(x.K, x.V, x.W, K_to, V_to, W_to, x.table, table_to, x.lens, budget, recent)
    cache = x.cache(seka, W=x.W)
    to = seka.paged_cache(x.dev(K_to), x.dev(V_to), x.dev(table_to), torch.full((x.B,), 99, dtype=torch.int32, device="cuda"), W=torch.from_numpy(W_to).cuda())
    kept = torch.full((x.B, x.Hkv, budget), 77, dtype=torch.int32, device="cuda")
    seka.seka_cache_evict(cache, to, kept, recent)
    compare((to.K, to.V, to.W, kept, to.lens), want, what)
    # the same in place
    want = orc.evict(x.K, x.V, x.W, x.K, x.V, x.W, x.table, x.table, x.lens, budget, recent)
    lens = torch.empty(x.B, dtype=torch.int32, device="cuda")
    kept.fill_(77)
    seka.seka_cache_evict(cache, cache, kept, recent, lens_out=lens)
    compare((cache.K, cache.V, cache.W, kept, lens), want, what + " in place")


def compare(got, want, what):
    for name, a, b in zip(("K", "V", "W", "kept", "lens"), got, want):
        a = a.cpu().numpy() if not a.is_floating_point() else P.f64(a)
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f"), f"{what}: {name}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (16, 0), (50, 17), (64, 64), (257, 100), (3000, 10)])
def test_budgets(seka, dtype, D, budget, recent):
    x = P.Pages(dtype, [0] * 6, [0, 1, 16, 65, 300, 1500], 3, 3, D, 16, seed=budget)
    check(seka, x, budget, recent, f"evict {dtype} {D} {budget} {recent}")


@pytest.mark.parametrize("ps,ps_to", [(8, 8), (8, 64), (64, 8), (256, 16)])
def test_page_sizes(seka, ps, ps_to):
    check(seka, P.Pages("bf16", [0, 0], [777, 100], 2, 2, 128, ps, seed=1), 99, 20, f"pages of {ps} to {ps_to}", ps_to=ps_to)


@pytest.mark.parametrize("kind", ["equal", "few values", "infinities", "nan", "negative", "zeros", "rising", "falling", "denormal"])
def test_weights_of_all_kinds(seka, kind):
    x = P.Pages("bf16", [0, 0], [900, 500], 2, 2, 64, 16, seed=2)
    g = np.random.default_rng(3)
    if kind == "equal":
        x.W[:] = 0.25
    elif kind == "few values":
        x.W[:] = g.integers(0, 3, x.W.shape)
    elif kind == "infinities":
        x.W[g.random(x.W.shape) < 0.3] = np.inf
        x.W[g.random(x.W.shape) < 0.3] = -np.inf
    elif kind == "nan":
        x.W[g.random(x.W.shape) < 0.8] = np.nan
    elif kind == "negative":
        x.W -= 0.5
    elif kind == "zeros":
        x.W[:] = np.where(g.random(x.W.shape) < 0.5, np.float32(-0.0), np.float32(0.0))
    elif kind == "denormal":
        x.W[:] = (g.integers(0, 200, x.W.shape) * np.float32(1e-44)).astype(np.float32)
    else:
        for b, n in enumerate(x.lens):
            j = np.arange(n)
            x.W[x.table[b, j // 16], :, j % 16] = (j if kind == "rising" else n - j)[:, None]
    check(seka, x, 123, 11, f"weights: {kind}")


@pytest.mark.parametrize("kind", ["any", "equal", "few values", "infinities and nan"])
@pytest.mark.parametrize("budget,recent", [(12, 11), (30, 11), (200, 11), (9, 0)])
def test_few_candidates(seka, kind, budget, recent):
    x = P.Pages("f32", [0] * 7, [40, 13, 266, 267, 268, 75, 331], 2, 2, 64, 16, seed=8)
    g = np.random.default_rng(9)
    if kind == "equal":
        x.W[:] = 0.25
    elif kind == "few values":
        x.W[:] = g.integers(0, 3, x.W.shape)
    elif kind != "any":
        x.W[g.random(x.W.shape) < 0.3] = np.inf
        x.W[g.random(x.W.shape) < 0.3] = -np.inf
        x.W[g.random(x.W.shape) < 0.3] = np.nan
    check(seka, x, budget, recent, f"few candidates: {kind} {budget} {recent}")


def test_more_tokens_than_shared_memory_holds(seka):
    x = P.Pages("bf16", [0], [40001], 1, 1, 64, 64, seed=4)
    x.W[:] = np.round(x.W * 500) / 500                     # many ties
    check(seka, x, 9000, 77, "a long cache")


def test_free_pages_of_the_same_pool(seka):
    x = P.Pages("bf16", [0, 0], [200, 333], 2, 2, 128, 16, seed=5, spare=20)
    owned = {int(p) for b, n in enumerate(x.lens) for p in x.table[b, :-(-n // 16)]}
    table_to, _ = target(x, 100, 16, 6, pool=[p for p in range(x.num_pages) if p not in owned])
    want = orc.evict(x.K, x.V, x.W, x.K, x.V, x.W, x.table, table_to, x.lens, 100, 30)
    cache = x.cache(seka, W=x.W)
    to = seka.paged_cache(cache.K, cache.V, x.dev(table_to), torch.zeros(2, dtype=torch.int32, device="cuda"), W=cache.W)
    kept = torch.empty((2, 2, 100), dtype=torch.int32, device="cuda")
    seka.seka_cache_evict(cache, to, kept, 30)
    compare((to.K, to.V, to.W, kept, to.lens), want, "free pages of the pool")


def test_limits(seka):
    """max_len cuts first; lengths and page numbers out of range stay in the pool."""
    x = P.Pages("f32", [0], [300], 2, 2, 64, 16, seed=7, wild=False)
    cache = x.cache(seka, W=x.W)
    kept = torch.empty((1, 2, 50), dtype=torch.int32, device="cuda")
    lens = torch.empty(1, dtype=torch.int32, device="cuda")
    want = orc.evict(x.K, x.V, x.W, x.K, x.V, x.W, x.table, x.table, [128], 50, 10)
    seka.seka_cache_evict(cache, cache, kept, 10, lens_out=lens, max_len=128)
    compare((cache.K, cache.V, cache.W, kept, lens), want, "max_len")
    x.lens = [1 << 30]
    x.table[:] = -9
    cache = x.cache(seka, W=x.W)
    seka.seka_cache_evict(cache, cache, kept, 10, lens_out=lens)
    torch.cuda.synchronize()
    assert int(lens) == 50


def test_replays_from_a_graph(seka):
    x = P.Pages("bf16", [0, 0], [500, 300], 2, 2, 128, 16, seed=8, wild=False)
    cache = x.cache(seka, W=x.W)
    K, V, W = cache.K.clone(), cache.V.clone(), cache.W.clone()
    kept, lens = torch.empty((2, 2, 64), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    call = lambda: seka.seka_cache_evict(cache, cache, kept, 16, lens_out=lens)     # noqa: E731

    def restore(turn):
        cache.K.copy_(K)
        cache.V.copy_(V)
        cache.W.copy_(W.roll(turn, 0))
        kept.fill_(5)

    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    for turn in range(3):
        restore(turn)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (cache.K, cache.V, cache.W, kept, lens)]
        restore(turn)
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (cache.K, cache.V, cache.W, kept, lens)))
