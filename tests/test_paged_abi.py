"""Refusals of the calls over caches of pages: host checks, before any GPU work.  CPU only."""
import ctypes
import math

import pytest

MB = 1 << 20
AT = lambda n: (n + 1) << 32          # noqa: E731  far apart, aligned, never dereferenced

NULL, SHAPE, DTYPE, ALIGN, ALIAS, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5, 6, 8


@pytest.fixture(scope="module")
def B():
    from paper_2603_01281_amd import binding
    return binding


def shape(lib, **kw):
    d = dict(B=2, S=128, Hq=4, Hkv=2, D=64, dtype=lib.SEKA_BF16, scale=0.0)
    d.update(kw)
    return lib.seka_shape(d["B"], d["S"], d["Hq"], d["Hkv"], d["D"], d["dtype"], d["scale"])


def paged(B, **kw):
    d = dict(K=AT(0), V=AT(1), W=AT(2), table=AT(3), lens=AT(4), num_pages=32, page_size=16, max_pages=8)
    d.update(kw)
    return B.seka_paged(*[d[k] for k in ("K", "V", "W", "table", "lens", "num_pages", "page_size", "max_pages")])


def rope(B, dim=64, freq=None, factor=1.0):
    f = (ctypes.c_double * 64)(*([0.1] * 64)) if freq is None else freq
    r = B.seka_rope(dim, 0, ctypes.cast(f, ctypes.POINTER(ctypes.c_double)) if f else None, factor)
    r._keep = f
    return r


ref = ctypes.byref


def test_rotary_refuses(B):
    def call(Q=AT(5), Qo=AT(6), K=AT(7), Ko=AT(8), sh=None, r=None, pos=AT(9)):
        return B.lib.seka_rotary(Q, Qo, K, Ko, ref(sh or shape(B)), ref(r or rope(B)), pos, None)
    assert call(Q=None) == NULL and call(Qo=None) == NULL and call(K=None) == NULL and call(Ko=None) == NULL
    assert B.lib.seka_rotary(AT(5), AT(6), None, None, ref(shape(B)), None, None, None) == NULL
    assert B.lib.seka_rotary(AT(5), AT(6), None, None, None, ref(rope(B)), None, None) == NULL
    assert call(r=B.seka_rope(64, 0, None, 1.0)) == NULL
    for dim in (0, 3, 66, -2):
        assert call(r=rope(B, dim=dim)) == SHAPE
    for bad in (math.inf, math.nan):
        assert call(r=rope(B, factor=bad)) == SHAPE
        assert call(r=rope(B, freq=(ctypes.c_double * 64)(*([0.1] * 31 + [bad] + [0.1] * 32)))) == SHAPE
    assert call(sh=shape(B, D=96)) == SHAPE and call(sh=shape(B, dtype=5)) == DTYPE and call(sh=shape(B, Hq=3)) == SHAPE
    assert call(sh=shape(B, B=1 << 30, S=8)) == SHAPE
    assert call(Q=AT(5) + 8) == ALIGN and call(Ko=AT(8) + 2) == ALIGN and call(pos=AT(9) + 2) == ALIGN
    assert call(Qo=AT(5) + 16) == ALIAS and call(Ko=AT(5)) == ALIAS and call(Qo=AT(7)) == ALIAS and call(Ko=AT(6)) == ALIAS and call(pos=AT(6)) == ALIAS


def test_frequencies_refuse(B):
    out = (ctypes.c_double * 64)()
    call = lambda dim=64, base=1e4, kind=0, stretch=2.0, original=4096.0, fast=32.0, slow=1.0, o=out: B.lib.seka_rope_frequencies(   # noqa: E731
        dim, base, kind, stretch, original, fast, slow, o)
    assert call() == 0 and call(o=None) == NULL
    assert call(dim=0) == SHAPE and call(dim=7) == SHAPE and call(dim=130) == SHAPE
    assert call(base=1.0) == SHAPE and call(base=math.nan) == SHAPE and call(base=math.inf) == SHAPE
    assert call(kind=-1) == UNSUPPORTED and call(kind=5) == UNSUPPORTED
    assert call(kind=1, stretch=0.5) == SHAPE and call(kind=1, stretch=math.nan) == SHAPE and call(stretch=math.nan) == 0
    assert call(kind=2, dim=2) == SHAPE
    for kind in (3, 4):
        assert call(kind=kind, original=0.0) == SHAPE and call(kind=kind, fast=1.0) == SHAPE and call(kind=kind, slow=0.0) == SHAPE
        assert call(kind=kind, fast=math.inf) == SHAPE


def bad_caches(B):
    return [(paged(B, K=None), NULL), (paged(B, V=None), NULL), (paged(B, table=None), NULL), (paged(B, num_pages=0), SHAPE), (paged(B, max_pages=0), SHAPE),
            (paged(B, page_size=0), SHAPE), (paged(B, page_size=4), SHAPE), (paged(B, page_size=24), SHAPE), (paged(B, page_size=1 << 17), SHAPE),
            (paged(B, K=AT(0) + 8), ALIGN), (paged(B, V=AT(1) + 2), ALIGN), (paged(B, W=AT(2) + 4), ALIGN), (paged(B, table=AT(3) + 2), ALIGN),
            (paged(B, lens=AT(4) + 1), ALIGN)]


def test_append_refuses(B):
    def call(K=AT(5), V=AT(6), Q=AT(7), Qo=AT(8), sh=None, c=None, r=True, pos=AT(9), mask=AT(10), cu=AT(11), total=10, max_q=5):
        return B.lib.seka_cache_append(K, V, Q, Qo, ref(sh or shape(B)), ref(c or paged(B)), ref(rope(B)) if r is True else r, pos, mask, cu, total, max_q, None)
    assert call(K=None) == NULL and call(V=None) == NULL and call(Q=None) == NULL and call(Qo=None) == NULL and call(cu=None) == NULL
    for c, code in bad_caches(B) + [(paged(B, lens=None), NULL)]:
        assert call(c=c) == code
    assert call(r=None) == UNSUPPORTED
    assert call(r=ref(rope(B, dim=66))) == SHAPE
    assert call(total=0) == SHAPE and call(total=1 << 31) == SHAPE and call(max_q=0) == SHAPE and call(max_q=129) == SHAPE
    assert call(sh=shape(B, B=70000)) == SHAPE and call(sh=shape(B, D=80)) == SHAPE and call(sh=shape(B, dtype=9)) == DTYPE
    assert call(K=AT(5) + 4) == ALIGN and call(cu=AT(11) + 2) == ALIGN and call(pos=AT(9) + 1) == ALIGN
    assert call(K=AT(0) + 64) == ALIAS and call(Q=AT(2)) == ALIAS and call(Qo=AT(0)) == ALIAS and call(Qo=AT(5)) == ALIAS and call(Qo=AT(7) + 16) == ALIAS
    assert call(mask=AT(1) + 3) == ALIAS and call(c=paged(B, V=AT(0) + 1024)) == ALIAS and call(c=paged(B, table=AT(0) + 16)) == ALIAS


def test_chunk_refuses(B):
    def call(Q=AT(5), O=AT(6), lse=AT(7), sh=None, c=None, cu=AT(8), total=10, max_q=5, ws=AT(9), n=64 * MB):
        return B.lib.seka_attention_chunk(Q, O, lse, ref(sh or shape(B, S=4096)), ref(c or paged(B)), cu, total, max_q, ws, n, None)
    assert call(Q=None) == NULL and call(O=None) == NULL and call(cu=None) == NULL
    for c, code in bad_caches(B) + [(paged(B, lens=None), NULL)]:
        assert call(c=c) == code
    assert call(total=0) == SHAPE and call(max_q=0) == SHAPE and call(max_q=4097) == SHAPE and call(sh=shape(B, scale=math.nan)) == SHAPE
    assert call(sh=shape(B, dtype=-1)) == DTYPE and call(sh=shape(B, Hq=5)) == SHAPE
    assert call(Q=AT(5) + 8) == ALIGN and call(O=AT(6) + 4) == ALIGN and call(lse=AT(7) + 2) == ALIGN and call(ws=AT(9) + 8) == ALIGN
    assert call(O=AT(5)) == ALIAS and call(O=AT(0)) == ALIAS and call(O=AT(1) + 32) == ALIAS and call(lse=AT(6)) == ALIAS and call(lse=AT(5)) == ALIAS and call(lse=AT(0)) == ALIAS
    need = B.seka_chunk_workspace_bytes(2, 4096, 4, 2, 64, B.SEKA_BF16, 10, 5)
    assert need > 0 and call(ws=None) == WORKSPACE and call(n=need - 1) == WORKSPACE
    assert B.seka_chunk_workspace_bytes(2, 4096, 4, 2, 64, B.SEKA_BF16, 10, 4097) == 0 and B.seka_chunk_workspace_bytes(2, 4096, 4, 2, 65, B.SEKA_BF16, 10, 5) == 0


def test_more_new_tokens_than_a_grid_holds(B):
    s, one, n = shape(B), shape(B, Hq=1, Hkv=1, B=1 << 12, S=1 << 12), 1 << 24
    assert B.lib.seka_rotary(AT(5), AT(6), None, None, ref(one), ref(rope(B)), None, None) == SHAPE
    assert B.lib.seka_cache_append(AT(5), AT(6), None, None, ref(s), ref(paged(B)), None, None, None, AT(11), n, 5, None) == SHAPE
    assert B.lib.seka_attention_chunk(AT(5), AT(6), None, ref(s), ref(paged(B)), AT(8), n, 5, AT(9), 64 * MB, None) == SHAPE
    assert B.lib.seka_attention_weights(AT(5), AT(6), ref(s), ref(paged(B)), None, AT(8), n, 5, 5, ctypes.c_float(1.0), None) == SHAPE
    assert B.seka_chunk_workspace_bytes(2, 128, 4, 2, 64, B.SEKA_BF16, n, 5) == 0


def test_weights_refuse(B):
    def call(Q=AT(5), lse=AT(6), sh=None, c=None, W_in=AT(7), cu=AT(8), total=10, max_q=5, window=5, decay=1.0):
        return B.lib.seka_attention_weights(Q, lse, ref(sh or shape(B)), ref(c or paged(B)), W_in, cu, total, max_q, window, decay, None)
    assert call(Q=None) == NULL and call(lse=None) == NULL and call(cu=None) == NULL
    for c, code in bad_caches(B) + [(paged(B, lens=None), NULL), (paged(B, W=None), NULL)]:
        assert call(c=c) == code
    assert call(total=0) == SHAPE and call(max_q=129) == SHAPE and call(window=0) == SHAPE and call(decay=math.inf) == SHAPE and call(decay=math.nan) == SHAPE
    assert call(Q=AT(5) + 8) == ALIGN and call(lse=AT(6) + 1) == ALIGN and call(W_in=AT(7) + 8) == ALIGN
    assert call(W_in=AT(2) + 16) == ALIAS and call(Q=AT(2)) == ALIAS and call(lse=AT(2) + 64) == ALIAS and call(c=paged(B, W=AT(0))) == ALIAS


def test_evict_refuses(B):
    to = lambda **kw: paged(B, **{**dict(K=AT(10), V=AT(11), W=AT(12), table=AT(13), lens=None), **kw})      # noqa: E731

    def call(sh=None, src=None, dst=None, budget=40, recent=8, kept=AT(20), lens=AT(21)):
        return B.lib.seka_cache_evict(ref(sh or shape(B)), ref(src or paged(B)), ref(dst or to()), budget, recent, kept, lens, None)
    for c, code in bad_caches(B) + [(paged(B, W=None), NULL)]:
        assert call(src=c) == code and call(dst=c) == code
    assert call(src=paged(B, lens=None)) == NULL and call(kept=None) == NULL and call(lens=None) == NULL
    assert call(budget=0) == SHAPE and call(recent=-1) == SHAPE and call(recent=41) == SHAPE
    assert call(dst=to(max_pages=2)) == SHAPE                                   # 32 tokens of 40
    assert call(kept=AT(20) + 2) == ALIGN and call(lens=AT(21) + 1) == ALIGN
    assert call(dst=to(K=AT(0))) == ALIAS and call(dst=to(K=AT(0) + 16)) == ALIAS and call(dst=to(V=AT(0))) == ALIAS
    assert call(dst=paged(B, table=AT(13), num_pages=16)) == ALIAS and call(dst=paged(B, table=AT(13), page_size=8)) == ALIAS
    assert call(lens=AT(4)) == ALIAS and call(kept=AT(0)) == ALIAS and call(kept=AT(3)) == ALIAS and call(lens=AT(20)) == ALIAS and call(kept=AT(10)) == ALIAS


def test_binding_refuses(B):
    """Shapes and types that the C side could not see."""
    import torch
    with pytest.raises(ValueError):
        B.paged_cache(torch.zeros(2, 8, 1, 64), torch.zeros(2, 8, 1, 64), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))   # host tensors
    with pytest.raises(ValueError):
        B.paged_cache(torch.zeros(2, 8, 64), torch.zeros(2, 8, 64), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.paged_cache(torch.zeros(2, 8, 1, 64), torch.zeros(2, 8, 1, 64), torch.zeros(1, 1, dtype=torch.int64), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.paged_cache(torch.zeros(2, 8, 1, 64), torch.zeros(2, 8, 1, 64), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), W=torch.zeros(2, 8, 1))
