"""seka_rotary and seka_cache_append against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import paged_helpers as P

pytestmark = pytest.mark.gpu


def bound(x, ref, freq, interleaved, factor, dtype):
    """Half a step of the result, and in front of it: the angle (in turns, rounded to 2^-26: 2 pi 2^-26 radians), sine and cosine (2 steps),
    their factor, two products and a sum in fp32: below 6e-7 of |x| + |y| together."""
    n = len(freq)
    size = np.zeros(x.shape)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return P.HALF[dtype] * 1.01 * np.abs(ref) + 6e-7 * abs(factor) * size


def close(got, x, positions, freq, interleaved, factor, dtype, what):
    ref = orc.rotary(x, positions, freq, interleaved, factor)
    off = np.abs(P.f64(got) - ref) - bound(x, ref, freq, interleaved, factor, dtype)
    assert (off <= 0).all(), f"{what}: {off.max():.3g} further off than it may be"
    n = 2 * len(freq)
    assert (P.f64(got)[..., n:] == x[..., n:]).all(), f"{what}: the part behind the rotated one"


def values(shape, dtype, seed):
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).to(P.TYPES[dtype])
    return x.cuda(), x.double().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,dim", [(64, 64), (128, 128), (128, 64), (128, 96), (64, 20), (128, 2), (64, 36), (128, 126)])
def test_layouts_and_parts(seka, dtype, interleaved, D, dim):
    print(f"rotary {dtype} {D} {dim} {interleaved}", flush=True)
    freq = orc.rope_frequencies(dim, 10000.0)
    rope = seka.rope(freq, interleaved=interleaved, factor=1.25)
    pos = np.random.default_rng(1).integers(-1000, 200000, (2, 9)).astype(np.int32)
    Q, q = values((2, 9, 6, D), dtype, 2)
    K, k = values((2, 9, 3, D), dtype, 3)
    p = torch.from_numpy(pos).cuda()
    Qo, Ko = torch.empty_like(Q), torch.empty_like(K)
    seka.seka_rotary(Q, Qo, rope, K=K, K_out=Ko, positions=p)
    close(Qo, q, pos, freq, interleaved, 1.25, dtype, "Q")
    close(Ko, k, pos, freq, interleaved, 1.25, dtype, "K")
    seka.seka_rotary(Q, Q, rope, K=K, K_out=K, positions=p)          # in place: the same bits
    assert torch.equal(Q, Qo) and torch.equal(K, Ko)


@pytest.mark.parametrize("B,S,Hq", [(1, 1, 1), (3, 1, 40), (1, 1000, 5), (2, 33, 64)])
def test_sizes_and_default_positions(seka, B, S, Hq):
    freq = orc.rope_frequencies(128, 500000.0)
    Q, q = values((B, S, Hq, 128), "bf16", 4)
    out = torch.empty_like(Q)
    seka.seka_rotary(Q, out, seka.rope(freq))
    close(out, q, np.broadcast_to(np.arange(S), (B, S)), freq, False, 1.0, "bf16", f"{B} {S} {Hq}")


def test_far_positions(seka):
    """Angles of positions up to 2^31 - 1, and whole turns: a frequency of 2 pi leaves everything as it is."""
    pos = np.array([[0, 1, 12345678, 2**24 + 1, 2**31 - 1, -2**31]], np.int64)
    Q, q = values((1, 6, 2, 64), "f32", 5)
    out = torch.empty_like(Q)
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    freq = orc.rope_frequencies(64, 1e6)
    # in 64 bits p f / 2 pi carries 2^-52 of itself: at 2^31 / 2 pi turns 2 pi 2^28.4 2^-52 = 5e-7 radians more, and as much in the oracle's product
    seka.seka_rotary(Q, out, seka.rope(freq), positions=p)
    ref = orc.rotary(q, pos, freq)
    size = np.abs(q[..., :32]) + np.abs(q[..., 32:])
    assert (np.abs(P.f64(out) - ref) <= 2e-6 * np.concatenate([size, size], -1) + 2.0 ** -23 * np.abs(ref)).all()
    seka.seka_rotary(Q, out, seka.rope([2 * np.pi] * 32), positions=p)
    assert (np.abs(P.f64(out) - q) <= 2e-6 * np.concatenate([size, size], -1) + 2.0 ** -23 * np.abs(q)).all()


def test_backwards(seka):
    freq = orc.rope_frequencies(128, 10000.0)
    Q, q = values((1, 50, 4, 128), "f32", 6)
    mid, back = torch.empty_like(Q), torch.empty_like(Q)
    seka.seka_rotary(Q, mid, seka.rope(freq))
    seka.seka_rotary(mid, back, seka.rope([-f for f in freq]))
    size = np.abs(q[..., :64]) + np.abs(q[..., 64:])
    assert (np.abs(P.f64(back) - q) <= 4 * 6e-7 * np.concatenate([size, size], -1)).all()


@pytest.mark.parametrize("scaling,name", [(0, "plain"), (1, "linear"), (2, "base"), (3, "parts"), (4, "turns")])
def test_scaled_frequencies_turn(seka, scaling, name):
    freq = seka.seka_rope_frequencies(128, 10000.0, scaling, stretch=8.0, original=4096.0, fast=4.0, slow=1.0)
    want = orc.rope_frequencies(128, 10000.0, name, 8.0, 4096.0, 4.0, 1.0)
    Q, q = values((1, 40, 2, 128), "bf16", 7)
    pos = np.arange(40)[None] * 777
    out = torch.empty_like(Q)
    seka.seka_rotary(Q, out, seka.rope(freq), positions=torch.from_numpy(pos.astype(np.int32)).cuda())
    close(out, q, pos, want, False, 1.0, "bf16", name)


# ---- append -------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [8, 16, 64, 256])
@pytest.mark.parametrize("positions", [False, True])
def test_append(seka, dtype, ps, positions):
    print(f"append {dtype} {ps} {positions}", flush=True)
    new, lens = [1, 0, 33, 100, 5], [1, 50, 33, 260, 3]             # the last one has more new tokens than places
    x = P.Pages(dtype, new, lens, 6, 3, 128, ps, seed=ps, tail=4, wild=False)
    k, v = x.values(x.total, 3, 128), x.values(x.total, 3, 128)
    pos = x.g.integers(0, 100000, x.total).astype(np.int32)
    mask = (x.g.random(x.total) < 0.3).astype(np.uint8) * 3
    cache = x.cache(seka, W=x.W)
    before = cache.K.clone(), cache.V.clone()
    freq = orc.rope_frequencies(96, 10000.0)
    q_out = torch.full_like(x.dev(x.Q), 7.0)
    seka.seka_cache_append(x.dev(k), x.dev(v), cache, x.cu_dev, 100, rope=seka.rope(freq, interleaved=True), positions=x.dev(pos) if positions else None,
                           Q=x.dev(x.Q), Q_out=q_out, mask=x.dev(mask))
    torch.cuda.synchronize()
    used = int(x.cu[-1])
    place = np.concatenate([lens[b] - new[b] + np.arange(new[b]) for b in range(5)])
    p = pos[:used] if positions else place
    close(q_out[:used], x.Q[:used], p, freq, True, 1.0, dtype, "Q")
    assert (q_out[used:] == 7.0).all()
    req = np.repeat(np.arange(5), new)
    there = place >= 0
    page, slot = x.table[req[there], place[there] // ps], place[there] % ps
    close(cache.K[page, slot], k[:used][there], p[there], freq, True, 1.0, dtype, "K")
    assert (P.f64(cache.V)[page, slot] == v[:used][there]).all()
    assert (cache.W.cpu().numpy()[page, :, slot] == np.where(mask[:used][there] != 0, np.inf, 0.0)[:, None]).all()
    rest = np.ones((x.num_pages, ps), bool)
    rest[page, slot] = False
    assert torch.equal(cache.K.cpu()[rest], before[0].cpu()[rest]) and torch.equal(cache.V.cpu()[rest], before[1].cpu()[rest])
    w = np.moveaxis(cache.W.cpu().numpy(), 1, 2)
    assert (w[rest] == np.moveaxis(x.W, 1, 2)[rest]).all()


def test_append_without_rotation_and_weights(seka):
    x = P.Pages("bf16", [3, 70], [40, 70], 4, 2, 64, 16, seed=3)
    k, v = x.values(x.total, 2, 64), x.values(x.total, 2, 64)
    cache = x.cache(seka)
    seka.seka_cache_append(x.dev(k), x.dev(v), cache, x.cu_dev, 70)
    for got, was, rows in ((cache.K, x.K, k), (cache.V, x.V, v)):
        assert np.array_equal(P.f64(got), orc.append(was, rows, x.table, x.lens, x.cu), equal_nan=True)


def test_append_many_requests_and_limits(seka):
    """More requests than a workgroup has threads; tokens beyond max_len and beyond max_q are not written."""
    new = [1] * 600
    x = P.Pages("f32", new, [20] * 600, 2, 1, 64, 8, seed=4, wild=False)
    k, v = x.values(600, 1, 64), x.values(600, 1, 64)
    cache = x.cache(seka)
    seka.seka_cache_append(x.dev(k), x.dev(v), cache, x.cu_dev, 1)
    assert (P.f64(cache.K) == orc.append(x.K, k, x.table, x.lens, x.cu)).all()
    x = P.Pages("f32", [10], [30], 2, 1, 64, 8, seed=5, wild=False)
    k, v = x.values(10, 1, 64), x.values(10, 1, 64)
    cache = x.cache(seka)
    seka.seka_cache_append(x.dev(k), x.dev(v), cache, x.cu_dev, 4, max_len=26)     # a cache cut to 26 tokens, a chunk cut to four
    want = orc.append(x.K, k, x.table, [26], np.array([0, 4]))
    assert (P.f64(cache.K) == want).all()


def test_append_replays_from_a_graph(seka):
    x = P.Pages("bf16", [1, 6], [30, 40], 4, 2, 128, 16, seed=6, wild=False)
    cache, k, v, q = x.cache(seka, W=x.W), x.dev(x.values(7, 2, 128)), x.dev(x.values(7, 2, 128)), x.dev(x.Q)
    q_out, rope = torch.empty_like(q), seka.rope(orc.rope_frequencies(128, 10000.0))
    start = cache.K.clone()
    call = lambda: seka.seka_cache_append(k, v, cache, x.cu_dev, 6, rope=rope, Q=q, Q_out=q_out)      # noqa: E731
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    for lens in ([30, 40], [17, 6], [25, 47]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        k.neg_()
        cache.K.copy_(start)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = cache.K.clone(), q_out.clone()
        cache.K.copy_(start)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], cache.K) and torch.equal(got[1], q_out)
