"""seka_attention_chunk against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import paged_helpers as P

pytestmark = pytest.mark.gpu


def run(seka, x, lse=True, max_q=None, max_len=None, scale=0.0, workspace=None, Q=None):
    cache = x.cache(seka)
    q = x.dev(x.Q if Q is None else Q)
    O = torch.full_like(q, 7.0)
    L = torch.full((x.Hq, x.total), 7.0, device="cuda") if lse else None
    seka.seka_attention_chunk(q, O, cache, x.cu_dev, max_q or max(max(x.new), 1), max_len=max_len, lse=L, scale=scale, workspace=workspace)
    torch.cuda.synchronize()
    return O, L


def check(seka, x, what, **kw):
    print(what, flush=True)
    used = int(x.cu[-1])
    ref = orc.chunk_attention(x.Q, x.K, x.V, x.table, x.lens, x.cu, scale=kw.get("scale") or None)
    ref = (ref[0][:used], ref[1][:, :used], ref[2][:used], ref[3][:, :used])
    # chunks that are long enough for it: also with the kernel of long chunks, which a bound on the cached tokens asks for
    far = max(x.new) * x.Hq // x.Hkv > 64 and "max_len" not in kw
    for more in ({}, dict(max_len=min(100000, (1 << 31) // (x.Hq * x.D) - 1))) if far else ({},):
        O, L = run(seka, x, **kw, **more)
        P.check_attention(P.f64(O)[:used], P.f64(L)[:, :used] if L is not None else None, ref, x.dtype, f"{what} {more}", lse=L is not None)
        assert (O[used:] == 7.0).all() and (L is None or (L[:, used:] == 7.0).all()), f"{what}: rows behind the last request were written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (7, 1), (3, 3), (40, 2)])
def test_single_tokens(seka, dtype, D, Hq, Hkv):
    lens = [1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 300, 777]
    check(seka, P.Pages(dtype, [1] * len(lens), lens, Hq, Hkv, D, 16, seed=D + Hq), f"single {dtype} {D} {Hq}/{Hkv}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [8, 16, 32, 64, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_page_sizes(seka, dtype, ps, D):
    x = P.Pages(dtype, [5, 1, 33, 70, 16], [600, 333, 33, 71, 1025], 4, 2, D, ps, seed=ps)
    check(seka, x, f"pages of {ps} {dtype} {D}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,lens", [
    ([1], [1]), ([2], [2]), ([3], [500]), ([64], [64]), ([65], [65]), ([63], [64]), ([130], [130]), ([200], [457]),
    ([1, 100, 1, 17], [900, 100, 1, 333]), ([0, 40, 0], [50, 90, 0]), ([129, 1, 256], [129, 700, 300]), ([31, 32, 33], [95, 64, 34]),
])
def test_chunks(seka, dtype, new, lens):
    for Hq, Hkv, D in ((4, 1, 128), (6, 2, 64)):
        check(seka, P.Pages(dtype, new, lens, Hq, Hkv, D, 16, seed=sum(lens)), f"chunks {dtype} {new} {lens} {Hq}/{Hkv} {D}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_that_see_nothing(seka, dtype):
    """More new tokens than cached ones: those before the first cached token see no key."""
    check(seka, P.Pages(dtype, [20, 3, 70], [7, 0, 64], 4, 2, 128, 16, seed=4), f"nothing to see {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_behind_the_last_request_and_scale(seka, dtype):
    check(seka, P.Pages(dtype, [9, 1], [40, 222], 4, 2, 64, 32, seed=5, tail=6), f"tail {dtype}", scale=0.31, lse=False)
    check(seka, P.Pages(dtype, [9, 90], [40, 222], 4, 2, 64, 32, seed=5, tail=6), f"tail {dtype}", scale=0.31)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 70])
def test_many_requests(seka, dtype, new):
    g = np.random.default_rng(8)
    n = [int(v) for v in g.integers(0, new + 1, 150)]
    lens = [int(max(v, k)) for v, k in zip(g.integers(0, 200, 150), n)]
    check(seka, P.Pages(dtype, n, lens, 2, 1, 64, 8, seed=9), f"150 requests {dtype} {new}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_cache_in_many_ranges(seka, dtype):
    check(seka, P.Pages(dtype, [1, 2, 20], [5000, 9, 3001], 8, 2, 128, 16, seed=10), f"ranges {dtype}")


@pytest.mark.parametrize("Hq,Hkv,n,S", [(256, 64, 300, 900), (256, 64, 520, 1101), (256, 64, 256, 520), (1024, 64, 17, 150), (192, 64, 300, 700)])
def test_long_chunk_of_many_heads(seka, Hq, Hkv, n, S):
    """Few workgroups per head: a single request takes blocks of rows whole, and cuts the ones left over."""
    check(seka, P.Pages("bf16", [n], [S], Hq, Hkv, 64, 16, seed=n), f"whole blocks {Hq}/{Hkv} {n} {S}")


@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 64), (6, 2, 128), (7, 1, 64), (5, 5, 128), (9, 1, 128), (20, 1, 64), (32, 32, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_of_any_size(seka, Hq, Hkv, D, dtype):
    """A wave's 32 rows are a few positions and all heads of a group: first new tokens at any place in 32 positions, blocks with few rows."""
    new = [n for n in (1, 2, 11, 33, 70, 100) if n * Hq // Hkv <= 1000]
    lens = [n + c for n, c in zip(new, (31, 64, 45, 0, 95, 300))]
    check(seka, P.Pages(dtype, new, lens, Hq, Hkv, D, 16, seed=Hq + D), f"groups {Hq}/{Hkv} {D} {dtype}")
    check(seka, P.Pages(dtype, new[-1:], [lens[-1] + 500], Hq, Hkv, D, 32, seed=Hq), f"one request {Hq}/{Hkv} {D} {dtype}")


@pytest.mark.parametrize("Hq,Hkv,n,S", [(256, 64, 300, 900), (192, 64, 130, 700)])
def test_long_chunk_of_many_heads_f32(seka, Hq, Hkv, n, S):
    check(seka, P.Pages("f32", [n], [S], Hq, Hkv, 64, 16, seed=n), f"whole blocks {Hq}/{Hkv} {n} {S}")


@pytest.mark.parametrize("dtype,Hq,Hkv,n,S", [("f32", 768, 48, 81, 185), ("f32", 1024, 64, 69, 180), ("bf16", 256, 16, 296, 772)])
def test_few_blocks_left_over(seka, dtype, Hq, Hkv, n, S):
    """A single request whose blocks go to the workgroups whole, but for one or three that all of them share: pieces of no tile at all
    (the second and third), and a last block that costs half (the first)."""
    check(seka, P.Pages(dtype, [n], [S], Hq, Hkv, 64, 16, seed=n), f"left over {dtype} {Hq}/{Hkv} {n} {S}")


def test_blocks_cut_by_many_workgroups_f32(seka):
    check(seka, P.Pages("f32", [33], [9000], 4, 1, 128, 16, seed=1), "pieces of one block")
    check(seka, P.Pages("f32", [100, 1, 0, 17, 1], [5000, 3, 700, 1200, 2000], 4, 1, 64, 32, seed=2), "pieces of mixed requests")


def test_blocks_cut_by_many_workgroups(seka):
    """One head: every block of rows is cut into many pieces; requests of very different lengths share workgroups."""
    check(seka, P.Pages("bf16", [33], [9000], 4, 1, 128, 16, seed=1), "pieces of one block")
    check(seka, P.Pages("bf16", [100, 1, 0, 17, 1], [5000, 3, 700, 1200, 2000], 4, 1, 64, 32, seed=2), "pieces of mixed requests")
    check(seka, P.Pages("bf16", [90, 300], [90, 2300], 7, 1, 128, 8, seed=3), "pieces, seven heads")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_grow(seka, dtype):
    """Every block of keys outgrows the reference of the one before: references are raised all along a row."""
    x = P.Pages(dtype, [1, 50], [700, 600], 4, 2, 64, 16, seed=11)
    for b, n in enumerate(x.lens):
        j = np.arange(n)
        k = x.K[x.table[b, j // 16], j % 16]
        x.K[x.table[b, j // 16], j % 16] = torch.from_numpy(k * (j[:, None, None] / 40.0)).to(x.t).double().numpy()
    check(seka, x, f"growing scores {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_limits_of_lengths(seka, dtype):
    """max_len cuts caches to their first tokens; lens and cu out of range are clamped; page numbers out of range stay in the pool."""
    x = P.Pages(dtype, [1, 1], [300, 200], 4, 2, 64, 16, seed=12, wild=False)
    O, L = run(seka, x, max_len=128)
    y = P.Pages(dtype, [1, 1], [300, 200], 4, 2, 64, 16, seed=12, wild=False)
    y.lens = [128, 128]
    ref = orc.chunk_attention(y.Q, y.K, y.V, y.table, y.lens, y.cu)
    P.check_attention(P.f64(O), P.f64(L), ref, dtype, "max_len")
    x.lens = [1 << 30, -5]
    x.table[0, :] = -7                                    # page 0 everywhere
    x.table[1, :] = 1 << 30
    O, L = run(seka, x)
    x.lens, x.table = [x.max_pages * 16, 0], np.zeros_like(x.table)
    ref = orc.chunk_attention(x.Q, x.K, x.V, x.table, x.lens, x.cu)
    P.check_attention(P.f64(O), P.f64(L), ref, dtype, "clamped")
    x.cu = np.array([0, 900, -3], np.int32)
    run(seka, x)                                          # no content of cu leaves the tensors


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strong_cache_and_infinite_values_elsewhere(seka, dtype):
    """Values of +-inf and NaN of another request's pages do not reach a request's rows."""
    x = P.Pages(dtype, [1, 30], [100, 90], 4, 2, 128, 16, seed=13)
    clean = run(seka, x)
    x.V[x.table[1, 0]] = np.inf
    x.K[x.table[1, 1]] = np.nan
    dirty = run(seka, x)
    assert torch.equal(clean[0][:1], dirty[0][:1]) and torch.equal(clean[1][:, :1], dirty[1][:, :1])
    assert not torch.isfinite(dirty[0][1:]).all()


def test_same_bits_twice_and_on_another_stream(seka):
    x = P.Pages("bf16", [1, 90, 3], [4000, 500, 1000], 8, 2, 128, 16, seed=14)
    O, L = run(seka, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        O2, L2 = run(seka, x)
    assert torch.equal(O, O2) and torch.equal(L, L2)


def test_workspace_is_scratch(seka):
    """Whatever the workspace holds, and where a smaller call used it before."""
    x = P.Pages("bf16", [1, 1], [3000, 5000], 8, 2, 128, 16, seed=15)
    need = seka.seka_chunk_workspace_bytes(2, x.max_pages * 16, 8, 2, 128, seka.SEKA_BF16, 2, 1)
    assert need > 0
    a = run(seka, x)
    b = run(seka, x, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    with pytest.raises(seka.SekaError) as e:
        run(seka, x, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 8


def test_replays_from_a_graph(seka):
    """Captured once; replayed with other lengths, tables and queries in the same tensors."""
    x = P.Pages("bf16", [1, 40], [500, 300], 8, 2, 128, 16, seed=16, wild=False)
    cache = x.cache(seka)
    q = x.dev(x.Q)
    O, L = torch.empty_like(q), torch.empty((x.Hq, x.total), device="cuda")
    ws = torch.empty(seka.seka_chunk_workspace_bytes(2, cache.capacity, 8, 2, 128, seka.SEKA_BF16, x.total, 40), dtype=torch.uint8, device="cuda")
    call = lambda: seka.seka_attention_chunk(q, O, cache, x.cu_dev, 40, lse=L, workspace=ws)   # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    for lens in ([500, 300], [16, 40], [333, 290]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        q.neg_()
        O.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone(), L.clone()
        O.fill_(9.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], O) and torch.equal(got[1], L), lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_agrees_with_the_prefill_and_the_generation_step(seka, dtype):
    """A whole prompt as one chunk is the plain prefill; a single token over the same keys is the generation step (each within its rounding)."""
    x = P.Pages(dtype, [300], [300], 8, 2, 128, 16, seed=17)
    O, L = run(seka, x)
    K = x.dev(orc.cached(x.K, x.table, 0, 300)[None])
    V = x.dev(orc.cached(x.V, x.table, 0, 300)[None])
    Q = x.dev(x.Q[None])
    O2 = torch.empty_like(Q)
    seka.seka_attention_plain(Q, K, V, O2)
    tol = 2e-2 if dtype == "bf16" else 1e-4
    assert (O.float() - O2[0].float()).abs().max() <= tol
    q = Q[:, -1].contiguous()
    O3 = torch.empty_like(q)
    seka.seka_attention_decode(q, K, V, O3)
    assert (O[-1].float() - O3[0].float()).abs().max() <= tol
