"""The key/value cache's host side: sizes, steps of rotations, refusals.  Nothing is launched: every refusal comes before the
first call into HIP, so the pointers are never followed."""
import ctypes as C
import math

import pytest

from cache_reference import frequencies


@pytest.fixture(scope="module")
def comet():
    from paper_2111_09562_amd import build, comet as libcomet
    build.build()
    libcomet.lib()
    return libcomet


@pytest.mark.parametrize("how", [{}, {"scaling": "linear", "factor": 4.0}, {"scaling": "base", "factor": 8.0},
                                 {"scaling": "parts", "factor": 16.0, "original_len": 8192, "beta_fast": 24.0, "beta_slow": 2.0}])
@pytest.mark.parametrize("rot", [2, 64, 96, 256])
def test_steps(comet, rot, how):
    steps, amp = comet.comet_rope_steps(rot, base=50000.0, **how)
    f, want = frequencies(rot, base=50000.0, **how)
    assert len(steps) == rot // 2 and abs(amp - want) <= 2.0 ** -24 * want
    for a, b in zip(steps, f):              # the reference has 53 bits, its powers a few units of the last
        assert abs(a - b / (2 * math.pi) * 2.0 ** 64) <= 2.0 ** -48 * a + 1


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=3), dict(rot=4098), dict(rot=64, base=1.0), dict(rot=64, base=float("nan")), dict(rot=64, factor=0.5),
                                 dict(rot=64, factor=float("inf")), dict(rot=64, scaling="parts", factor=2.0, original_len=0),
                                 dict(rot=64, scaling="parts", factor=2.0, beta_fast=1.0)])
def test_steps_refused(comet, bad):
    with pytest.raises(comet.CometError) as ei:
        comet.comet_rope_steps(**bad)
    assert ei.value.code == comet.ERR_INVALID


def test_unknown_scaling(comet):
    with pytest.raises(ValueError):
        comet.comet_rope_steps(64, scaling="twice")


def test_bytes(comet):
    for pages, page, slots, heads, dim in [(1, 32, 1, 1, 32), (7, 160, 3, 5, 96), (70000, 256, 512, 8, 128)]:
        n = pages * heads * page // 32
        assert comet.comet_cache_bytes(pages, page, slots, heads, dim) == n * 64 * dim + -(-8 * n // 256) * 256 + slots * heads * 2 * (128 * dim + 256)
    for bad in [(0, 32, 1, 1, 64), (1, 0, 1, 1, 64), (1, 33, 1, 1, 64), (1, 32, 0, 1, 64), (1, 32, 1, 0, 64), (1, 32, 1, 1, 0), (1, 32, 1, 1, 48),
                (1, 32, 1, 1, 288), (2 ** 31 - 1, 1 << 20, 1, 4096, 256), (1, 32, 2 ** 31 - 1, 4096, 256)]:
        assert comet.comet_cache_bytes(*bad) == 0, bad


FAKE = 0x1000                                # 16-byte aligned, never followed


def _batch(comet, **over):
    return comet.CacheBatch(**{**dict(n_seqs=2, table_width=4, dev_starts=FAKE, dev_lens=FAKE, dev_table=FAKE, dev_slots=FAKE), **over})


def test_refusals_of_the_c_interface(comet):
    L = comet.lib()
    ok_shape, rows = comet.CacheShape(4, 64, 2, 2, 64), comet.CacheRows(FAKE, 128, 64)
    queries, results = comet.CacheRows(FAKE, 256, 64), comet.CacheRows(FAKE + 4096, 256, 64)
    plan = comet.RopePlan(64, 0, 1.0, FAKE)

    def append(cache=FAKE, shape=ok_shape, batch=None, n=3, k=rows, v=rows, q=queries, qo=queries, qh=4, dt=comet.F16, p=plan, pos=FAKE, status=None):
        return L.comet_cache_append(cache, shape, C.byref(batch or _batch(comet)), n, k, v, q, qo, qh, dt, C.byref(p), pos, None, status)

    def attend(cache=FAKE, shape=ok_shape, batch=None, n=3, q=queries, qh=4, dt=comet.F16, scale=0.1, out=results, lse=None, work=FAKE, size=1 << 40):
        return L.comet_cache_attend(cache, shape, C.byref(batch or _batch(comet)), n, q, qh, dt, scale, 1, out, lse, work, size, None, None)

    def fetch(cache=FAKE, shape=ok_shape, batch=None, n=3, k=rows, v=rows, dt=comet.F16):
        return L.comet_cache_fetch(cache, shape, C.byref(batch or _batch(comet)), n, k, v, dt, None, None)

    none, odd = comet.CacheRows(None, 128, 64), comet.CacheRows(FAKE + 1, 128, 64)
    for call in (append, attend, fetch):
        assert call(n=0) == comet.OK         # nothing to do
        for bad in [dict(cache=None), dict(cache=FAKE + 8), dict(shape=comet.CacheShape(4, 48, 2, 2, 64)), dict(dt=0), dict(dt=3),
                    dict(batch=_batch(comet, n_seqs=0)), dict(batch=_batch(comet, dev_starts=None)), dict(batch=_batch(comet, dev_lens=None)),
                    dict(batch=_batch(comet, dev_table=None)), dict(batch=_batch(comet, table_width=0)), dict(batch=_batch(comet, dev_slots=FAKE + 2)),
                    dict(n=0x80000000)]:
            assert call(**bad) == comet.ERR_INVALID, (call, bad)
    for call in (append, fetch):
        for bad in [dict(k=none), dict(v=none), dict(k=odd), dict(v=odd)]:
            assert call(**bad) == comet.ERR_INVALID
    for bad in [dict(q=none), dict(qo=odd), dict(qo=comet.CacheRows(FAKE, 512, 64)), dict(qh=20000), dict(p=comet.RopePlan(66, 0, 1.0, FAKE)),
                dict(p=comet.RopePlan(64, 2, 1.0, FAKE)), dict(p=comet.RopePlan(64, 0, float("nan"), FAKE)), dict(p=comet.RopePlan(64, 0, 1.0, None)),
                dict(p=comet.RopePlan(0, 0, 1.0, FAKE)), dict(pos=FAKE + 1), dict(status=FAKE + 3)]:
        assert append(**bad) == comet.ERR_INVALID, bad
    for bad in [dict(q=none), dict(out=odd), dict(out=queries), dict(qh=0), dict(qh=3), dict(scale=float("nan")), dict(scale=-1.0), dict(scale=float("inf")), dict(lse=FAKE + 2),
                dict(work=None), dict(work=FAKE + 4), dict(n=0x7fffffff)]:
        assert attend(**bad) == comet.ERR_INVALID, bad
    assert attend(size=L.comet_cache_attend_work(ok_shape, 2, 3, 4) - 1) == comet.ERR_NOMEM

    def rope(p=plan, x=rows, y=comet.CacheRows(FAKE + 4096, 128, 64), n=3, heads=2, dim=64, dt=comet.F32, pos=None):
        return L.comet_rope(C.byref(p) if p else None, x, y, n, heads, dim, dt, pos, 0, None)

    assert rope(n=0) == comet.OK
    for bad in [dict(p=None), dict(dt=3), dict(dt=-1), dict(heads=0), dict(dim=62), dict(dim=5000), dict(x=none), dict(y=odd), dict(pos=FAKE + 2), dict(n=0x80000000),
                dict(y=comet.CacheRows(FAKE, 64, 64))]:
        assert rope(**bad) == comet.ERR_INVALID, bad


def test_work_bytes(comet):
    """Room for the pieces of tiles that are cut, whose number does not grow with the sequences, and 8 bytes per tile."""
    L = comet.lib()
    few = comet.CacheShape(4, 64, 2, 8, 128)
    small, large = L.comet_cache_attend_work(few, 64, 64, 32), L.comet_cache_attend_work(few, 4096, 4096, 32)
    assert 768 * 16 * (128 + 3) * 4 <= small < 64 << 20 and large - small < 16 * 4096 * 4
    assert L.comet_cache_attend_work(few, 1, 8192, 32) >= 512 * 128 * (128 + 3) * 4
    for bad in [(few, 1, 1, 12), (few, 1, 1, 0), (few, (1 << 22) + 1, 1, 32), (comet.CacheShape(4, 64, 2, 1, 128), 1, 1 << 30, 16),
                (comet.CacheShape(4, 64, 2, 4096, 128), 8192, 8192, 4096)]:
        assert L.comet_cache_attend_work(*bad) == 0, bad


def test_results_must_not_overlap(comet):
    """Tensors that are written: rows closer to each other than they are long are refused, in either direction; those that are read may be."""
    L, shape, batch = comet.lib(), comet.CacheShape(4, 64, 2, 2, 64), C.byref(_batch(comet))
    rows, plan = comet.CacheRows(FAKE, 128, 64), comet.RopePlan(64, 0, 1.0, FAKE)
    for token, head in [(0, 64), (128, 0), (63, 64), (128, -63), (-1, 64)]:
        bad = comet.CacheRows(FAKE + 4096, token, head)
        assert L.comet_rope(C.byref(plan), rows, bad, 3, 2, 64, comet.F32, None, 0, None) == comet.ERR_INVALID
        assert L.comet_cache_fetch(FAKE, shape, batch, 3, bad, rows, comet.F16, None, None) == comet.ERR_INVALID
        assert L.comet_cache_fetch(FAKE, shape, batch, 3, rows, bad, comet.F16, None, None) == comet.ERR_INVALID
        assert L.comet_cache_append(FAKE, shape, batch, 3, rows, rows, rows, bad, 4, comet.F16, None, None, None, None) == comet.ERR_INVALID
        assert L.comet_cache_attend(FAKE, shape, batch, 3, rows, 4, comet.F16, 0.1, 1, bad, None, FAKE, 1 << 40, None, None) == comet.ERR_INVALID


def test_results_must_not_interleave(comet):
    """Rows that are apart from their neighbours can still lie on those of another token's other head; attention's result not on its queries."""
    L, shape, batch = comet.lib(), comet.CacheShape(4, 64, 2, 2, 64), C.byref(_batch(comet))
    rows, plan = comet.CacheRows(FAKE, 128, 64), comet.RopePlan(64, 0, 1.0, FAKE)
    low = -(1 << 63)
    for tokens, heads, token, head in [(2, 2, 64, 64), (3, 2, 128, 128), (3, 4, 191, 64), (2, 3, 64, 127), (3, 2, -128, 128), (3, 2, 64, 191), (3, 2, low, low)]:
        bad = comet.CacheRows(FAKE + 4096, token, head)
        assert L.comet_rope(C.byref(plan), rows, bad, tokens, heads, 64, comet.F32, None, 0, None) == comet.ERR_INVALID, (tokens, heads, token, head)
    bad = comet.CacheRows(FAKE + 4096, 64, 64)
    assert L.comet_cache_fetch(FAKE, shape, batch, 3, bad, rows, comet.F16, None, None) == comet.ERR_INVALID
    assert L.comet_cache_append(FAKE, shape, batch, 3, rows, rows, rows, bad, 4, comet.F16, None, None, None, None) == comet.ERR_INVALID
    assert L.comet_cache_attend(FAKE, shape, batch, 3, rows, 4, comet.F16, 0.1, 1, bad, None, FAKE, 1 << 40, None, None) == comet.ERR_INVALID
    assert L.comet_cache_attend(FAKE, shape, batch, 3, comet.CacheRows(FAKE, 256, 64), 4, comet.F16, 0.1, 1, comet.CacheRows(FAKE, 256, 64), None, FAKE, 1 << 40,
                                None, None) == comet.ERR_INVALID


def test_binding_refuses_host_tensors(comet):
    import torch
    x = torch.zeros(2, 2, 64)
    rope = comet.Rope(64, device="cpu")
    with pytest.raises(ValueError):
        comet.comet_rope(x, rope)
    with pytest.raises(ValueError):
        comet.Batch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        comet.Cache(1, 32, 1, 1, 32, buf=torch.zeros(1 << 16, dtype=torch.uint8))
