"""What calls on the key/value cache refuse about how their tensors lie to one another, and the host side of rotations.  Nothing is launched: every
refusal comes before the first call into HIP, so the pointers are never followed."""
import ctypes as C
import itertools

import pytest

from test_cache_cpu import FAKE, _batch, comet  # noqa: F401


def overlap(a, ha, b, hb, tokens, dim):
    """By going through all rows; (address in elements, token stride, head stride) each."""
    rows = lambda r, heads: {r[0] + t * r[1] + h * r[2] for t in range(tokens) for h in range(heads)}  # noqa: E731
    return any(abs(x - y) < dim for x in rows(a, ha) for y in rows(b, hb))


def lies(comet, r, size):  # noqa: F811
    return comet.CacheRows(FAKE * 16 + r[0] * size, r[1], r[2])


def attend(comet, q, out, heads, tokens, dim):  # noqa: F811
    """NOMEM: everything but the workspace is fine."""
    shape = comet.CacheShape(4, 64, 2, 1, dim)
    return comet.lib().comet_cache_attend(FAKE, shape, C.byref(_batch(comet)), tokens, lies(comet, q, 2), heads, comet.F16, 0.1, 1, lies(comet, out, 2), None, FAKE, 0,
                                          None, None)


def test_attention_on_its_queries(comet):  # noqa: F811
    """Same strides: exactly those results are refused of which a row meets one of the queries."""
    dim = 32
    for tokens, heads, token, head in [(1, 1, 64, 64), (3, 2, 64, 32), (3, 2, 256, 64), (2, 3, -512, 96), (4, 2, 32, 300), (3, 4, 500, -100)]:
        q = (0, token, head)
        for at in list(range(-700, 701, 31)) + [0, 1, 31, 32, -32, 64, token, head, token + head, token - 1, 10 ** 6]:
            got = attend(comet, q, (at, token, head), heads, tokens, dim)
            assert got == (comet.ERR_INVALID if overlap(q, heads, (at, token, head), heads, tokens, dim) else comet.ERR_NOMEM), (tokens, heads, token, head, at)


def test_attention_with_other_strides(comet):  # noqa: F811
    """Other head strides as well; other token strides only where neither lies in the range of the other."""
    dim = 32
    for tokens, heads, token, head, head2 in [(3, 2, 256, 64, 32), (2, 3, 512, 32, 96), (1, 4, 7, 64, 32)]:
        for at in range(-600, 601, 16):
            q, out = (0, token, head), (at, token, head2)
            got = attend(comet, q, out, heads, tokens, dim)
            assert got == (comet.ERR_INVALID if overlap(q, heads, out, heads, tokens, dim) else comet.ERR_NOMEM), (token, head, head2, at)
    q = (0, 128, 64)
    for at, good in [(64, False), (4 * 128, True), (-256, True), (16, False)]:
        out = (at, 64, 32)
        assert not good or not overlap(q, 2, out, 2, 4, dim)
        assert attend(comet, q, out, 2, 4, dim) == (comet.ERR_NOMEM if good else comet.ERR_INVALID)
    # queries that all tokens share (no token stride)
    assert attend(comet, (0, 0, 32), (64, 64, 32), 2, 4, dim) == comet.ERR_NOMEM
    assert attend(comet, (0, 0, 32), (32, 64, 32), 2, 4, dim) == comet.ERR_INVALID


def test_turned_queries_on_what_is_read(comet):  # noqa: F811
    L, shape, rope = comet.lib(), comet.CacheShape(4, 64, 2, 2, 32), comet.RopePlan(32, 0, 1.0, FAKE)

    def append(k, v, q, q_out):
        k, v, q, q_out = (lies(comet, r, 2) for r in (k, v, q, q_out))
        return L.comet_cache_append(FAKE, shape, C.byref(_batch(comet)), 3, k, v, q, q_out, 4, comet.F16, C.byref(rope), None, None, None)

    k, v, q = (0, 256, 32), (64, 256, 32), (128, 256, 32)
    for q_out in [k, v, (96, 256, 32), (-96, 256, 32), (256, 256, 32), (-64, 256, 32), (160, 256, 32), (0, 128, 32)]:
        assert append(k, v, q, q_out) == comet.ERR_INVALID, q_out


def test_results_on_one_another(comet):  # noqa: F811
    L, shape = comet.lib(), comet.CacheShape(4, 64, 2, 2, 32)
    k = (0, 64, 32)
    for v in [k, (32, 64, 32), (-32, 64, 32), (128, 64, 32), (31, 64, 32), (0, 128, 32)]:
        assert L.comet_cache_fetch(FAKE, shape, C.byref(_batch(comet)), 3, lies(comet, k, 2), lies(comet, v, 2), comet.F16, None, None) == comet.ERR_INVALID, v
    plan = comet.RopePlan(32, 0, 1.0, FAKE)
    for dtype, size in ((comet.F32, 4), (comet.BF16, 2)):
        for y in [(32, 64, 32), (-64, 64, 32), (1, 64, 32), (64, 32, 96), (0, 128, 32), (63, 128, 32)]:
            assert L.comet_rope(C.byref(plan), lies(comet, k, size), lies(comet, y, size), 3, 2, 32, dtype, None, 0, None) == comet.ERR_INVALID, y


def test_far_strides_do_not_overflow(comet):  # noqa: F811
    low, high = -(1 << 63), (1 << 63) - 1
    for token, head in itertools.product((low, -1, 0, 1, high), repeat=2):
        for at in (64, -64):
            assert attend(comet, (0, token, head), (at, 64, 32), 2, 4, 32) in (comet.ERR_INVALID, comet.ERR_NOMEM)
    assert attend(comet, (0, high, 32), (64, 64, 32), 2, 1, 32) == comet.ERR_NOMEM        # (one token has no stride)


def test_rotation_refuses_what_asks_for_a_gradient(comet):  # noqa: F811
    import torch
    rope = comet.Rope(64, device="cpu")
    for kw in (dict(), dict(out=torch.zeros(2, 2, 64, requires_grad=True))):
        with pytest.raises(RuntimeError, match="gradient"):
            comet.comet_rope(torch.zeros(2, 2, 64, requires_grad=not kw), rope, **kw)
    with torch.no_grad(), pytest.raises(ValueError):                                      # (a host tensor)
        comet.comet_rope(torch.zeros(2, 2, 64, requires_grad=True), rope)


def test_amplitude_of_a_rotation(comet):  # noqa: F811
    how = dict(scaling="parts", factor=8.0, original_len=8192, beta_fast=4.0, device="cpu")
    natural, given = comet.Rope(128, **how), comet.Rope(128, amp=1.0, **how)
    assert natural.amp > 1.2 and given.amp == 1.0 and given._plan.amp == 1.0 and given.steps.equal(natural.steps)
    for bad in (float("nan"), float("inf"), -float("inf"), 1e39):
        with pytest.raises(ValueError):
            comet.Rope(128, amp=bad, device="cpu")
