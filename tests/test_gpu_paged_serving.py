"""The calls over caches of pages as a serving program strings them together: two conversations, one highlighted.  A chunk's keys are edited,
turned and appended, its queries attend, the attention adds up, the caches are cut, and generation goes on over what is left.  Every
step is compared with the fp64 oracle on the inputs that the step really had."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from oracle import seka_oracle
from tests import paged_helpers as P
from tests.test_gpu_rotary import bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,ps", [(8, 2, 128, 16), (3, 3, 64, 8)])
def test_two_conversations(seka, dtype, Hq, Hkv, D, ps):
    print(f"serving {dtype} {Hq}/{Hkv} {D} {ps}", flush=True)
    t, B, pages, most = P.TYPES[dtype], 2, 60, 25
    g = np.random.default_rng(5)
    values = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).to(t).cuda()      # noqa: E731
    K, V = torch.full((pages, ps, Hkv, D), float("nan"), dtype=t, device="cuda"), torch.full((pages, ps, Hkv, D), float("nan"), dtype=t, device="cuda")
    W = torch.full((pages, Hkv, ps), float("nan"), device="cuda")
    table = torch.from_numpy(g.permutation(pages)[:B * most].reshape(B, most).astype(np.int32)).cuda()
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache = seka.paged_cache(K, V, table, lens, W=W)
    freq = seka.seka_rope_frequencies(D, 10000.0, seka.SEKA_ROPE_TURNS, stretch=4.0, original=64.0, fast=4.0, slow=1.0)
    rope = seka.rope(freq)
    U = torch.from_numpy(np.linalg.qr(g.standard_normal((Hkv, 1, D, 8)))[0].astype(np.float32)).to(t).cuda()
    gain, tab = [1.5] * Hkv, table.cpu().numpy()
    positions_seen = np.zeros(B, np.int64)

    def step(new, highlight, window, decay):
        cu_h = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        total, cu = int(cu_h[-1]), torch.from_numpy(cu_h).cuda()
        pos = np.concatenate([positions_seen[b] + np.arange(new[b]) for b in range(B)]).astype(np.int32)
        positions_seen[:] += new
        q, k, v = values(total, Hq, D), values(total, Hkv, D), values(total, Hkv, D)
        mask = torch.zeros(total, dtype=torch.uint8, device="cuda")
        if highlight:
            mask[2:9] = 1
        edited = k.clone()
        seka.seka_edit_keys_packed(edited, edited, cu, max(new), U, gain, mask)
        ref = seka_oracle.edit_keys(P.f64(k)[None], P.f64(U), gain, mask.cpu().numpy()[None])[0]
        assert np.abs(P.f64(edited) - ref).max() <= (2.0 ** -8 * np.abs(ref) + 9e-3).max()
        lens.add_(torch.tensor(new, dtype=torch.int32, device="cuda"))
        n = lens.cpu().numpy()
        seka.seka_cache_append(edited, v, cache, cu, max(new), rope=rope, positions=torch.from_numpy(pos).cuda(), Q=q, Q_out=q_out(q), mask=mask)
        for b in range(B):
            rows = slice(cu_h[b], cu_h[b + 1])
            for x, got in ((edited, orc.cached(P.f64(K), tab, b, n[b])[n[b] - new[b]:]), (q, P.f64(turned)[rows])):
                x = P.f64(x)[rows]
                want = orc.rotary(x, pos[rows], freq)
                assert (np.abs(got - want) <= bound(x, want, freq, False, 1.0, dtype)).all()
            assert (orc.cached(P.f64(V), tab, b, n[b])[n[b] - new[b]:] == P.f64(v)[rows]).all()
            assert (orc.cached_weights(P.f64(W), tab, b, n[b])[n[b] - new[b]:] == np.where(mask.cpu().numpy()[rows] != 0, np.inf, 0.0)[:, None]).all()
        O, L = torch.empty_like(q), torch.empty((Hq, total), device="cuda")
        seka.seka_attention_chunk(turned, O, cache, cu, max(new), lse=L)
        P.check_attention(P.f64(O), P.f64(L), orc.chunk_attention(P.f64(turned), P.f64(K), P.f64(V), tab, n, cu_h), dtype, f"chunk {new}")
        before = P.f64(W)
        seka.seka_attention_weights(turned, L, cache, cu, max(new), window=window, W_in=W, decay=decay)
        want, sums = orc.attention_weights(P.f64(turned), P.f64(L), P.f64(K), before, before, tab, n, cu_h, window, decay)
        for b in range(B):
            got, ref = orc.cached_weights(P.f64(W), tab, b, n[b]), orc.cached_weights(want, tab, b, n[b])
            assert (np.isinf(got) == np.isinf(ref)).all()
            fine = np.isfinite(ref)
            assert (np.abs(got[fine] - ref[fine]) <= 2e-4 * (1 + np.abs(ref[fine]))).all()      # (tight bounds: the operator's own tests)

    turned = None

    def q_out(q):
        nonlocal turned
        turned = torch.empty_like(q)
        return turned

    step([50, 37], True, 16, 1.0)
    step([40, 1], False, 40, 0.9)
    # the caches are cut in place; highlighted tokens stay
    n, budget, recent = lens.cpu().numpy(), 40, 12
    before = [P.f64(x) for x in (K, V, W)]
    kept, lens_out = torch.empty((B, Hkv, budget), dtype=torch.int32, device="cuda"), torch.empty_like(lens)
    seka.seka_cache_evict(cache, cache, kept, recent, lens_out=lens_out)
    want = orc.evict(*before, *before, tab, tab, n, budget, recent)
    for got, ref in zip((K, V, W, kept, lens_out), want):
        assert np.array_equal(P.f64(got), ref, equal_nan=True)
    held = kept.cpu().numpy()[0]
    assert all(set(range(2, 9)) <= set(held[h]) for h in range(Hkv)), "highlighted tokens were dropped"
    lens.copy_(lens_out)
    for _ in range(3):
        step([1, 1], False, 1, 0.99)
    step([20, 3], False, 8, 0.5)
    assert lens.tolist() == [63, 44]
