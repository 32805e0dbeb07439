"""The compressed key/value cache where values lie next to a border: pages that are none, lengths set back more than once, values half way between
two steps, weights next to a rounding, tensors that autograd knows.  Against 64 bits, as in test_gpu_cache."""
import math

import pytest

torch = pytest.importorskip("torch")
import cache_reference as ref  # noqa: E402
from test_gpu_cache import DT, U32, Sequences, check_attend, check_held, comet, gen, rope_bound, u  # noqa: E402, F401

pytestmark = pytest.mark.gpu


# ---- pages that are none ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("stray", [math.inf, -math.inf, math.nan, 0.0, -1.0, 1.0])
@pytest.mark.parametrize("dtype,group,new", [("bf16", 1, 1), ("fp16", 4, 1), ("bf16", 2, 7), ("fp16", 1, 16), ("bf16", 5, 5), ("fp16", 2, 32), ("bf16", 1, 64),
                                             ("bf16", 3, 70), ("fp16", 1, 200)])
def test_missing_pages(comet, dtype, group, new, stray):  # noqa: F811
    """Tokens of a page that is none are not seen, however few the rows are, whatever lies in the cache where nobody has written."""
    s = Sequences(comet, DT[dtype], 2, 64, 1, 1024, seed=new)
    s.table = torch.arange(2, 2 + s.table.shape[1], dtype=torch.int32)[None]          # page 0 is nobody's
    s.grow([900])
    blocks = s.pages * 2 * 2
    s.cache.buf[blocks * 64 * 64:blocks * (64 * 64 + 8)].view(torch.float32).view(s.pages, -1)[:2] = stray
    q = s.tokens(new, 2 * group)
    k, v = s.held(0)
    for missing in ([0], [5], [3, 4, 12], [13]):                                     # the first, in the middle, several, the last with complete blocks
        good = s.table.clone()
        s.table[0, missing] = -1
        s.status.zero_()
        out, lse = s.cache.comet_cache_attend(s.batch([new]), q.cuda(), lse=True, status=s.status)
        assert int(s.status.item()) == comet.ERR_FORMAT
        s.table = good
        keep = torch.ones(900, dtype=torch.bool)
        for p in missing:
            keep[64 * p:min(64 * p + 64, 896)] = False                               # (the open block is in the ring)
        for i in sorted({0, new // 2, new - 1}):
            seen = keep[:900 - new + i + 1].nonzero().flatten()
            o, want, size, top = ref.attention(q[i:i + 1], k[:, seen], v[:, seen], 0.125, False)
            d = 72 * U32 * top
            assert ((lse[i].cpu().double() - want[0]).abs() <= d + 2.0 ** -18).all()
            assert ((out[i].cpu().double() - o[0]).abs() <= ((u(torch.float16) + 2 * d + 2.0 ** -19) * size + u(s.dt) * o.abs() + 2.0 ** -24)[0]).all()


# ---- lengths that are set back ------------------------------------------------------------------------------------


def test_set_back_again(comet):  # noqa: F811
    """Set back, grown, set back once more, never below 32 tokens under the greatest length: the open block is the tokens that came."""
    for most, path in ((65, ((3, 1), (30, 40))), (70, ((20, 2), (13, 1), (1, 70))), (96, ((32, 5), (4, 40))), (127, ((1, 1), (32, 0), (0, 3), (3, 90)))):
        s = Sequences(comet, torch.bfloat16, 2, 64, 1, 256, seed=most)
        s.grow([most])
        greatest = most
        for back, new in path:
            s.lens[0] -= back
            assert s.lens[0] >= greatest - 32
            s.k[0], s.v[0] = s.k[0][:s.lens[0]], s.v[0][:s.lens[0]]
            check_held(s, 0)
            q = s.tokens(1, 4)
            out, lse = s.cache.comet_cache_attend(s.batch([1]), q.cuda(), lse=True, status=s.status)
            check_attend(s, [1], q, out, lse)
            if new:
                s.grow([new])
            greatest = max(greatest, s.lens[0])
            check_held(s, 0)
        assert s.ok()


# ---- whole numbers half way between two ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("cuts", [[256], [16, 200, 40], [31, 1, 224], [1] * 33 + [223]])
def test_whole_numbers(comet, dtype, cuts):  # noqa: F811
    """x / s with s = max|x| / 127 rounded to the nearest whole number, ties to even, for all of a type's significands as the largest value.  In 64
    bits 127 x and ties are exact, and everything else is at least 2^-19 of itself away from one: with x = m 2^e and a = n 2^f, m and n of at most 11 bits,
    |254 x / a - odd| is a multiple of 2^(e - f) / n, and 2^e is at least x 2^-11.  (There are ties at x = a / 2, and others where n is a multiple of 127.)"""
    heads, dim = 128, 32
    s = Sequences(comet, DT[dtype], heads, dim, 1, 256, seed=7)
    bits = 10 if dtype == "fp16" else 7
    g = gen(70)
    order = torch.randperm(8 * heads, generator=g)                                    # block and head -> significand of its largest value
    largest = ((2.0 ** bits + order % 2 ** bits) * 2.0 ** -bits * 2.0 ** torch.randint(-10, 11, order.shape, generator=g)).view(8, 1, heads, 1)

    def some():
        x = ((torch.rand(8, 32, heads, dim, generator=g) * 2 - 1) * largest).to(DT[dtype]).double()
        pick = torch.rand(x.shape, generator=g)
        sign = torch.where(torch.rand(x.shape, generator=g) < 0.5, -1.0, 1.0)
        x = torch.where(pick < 0.3, sign * largest / 2, x)                            # half way between 63 and 64
        x = torch.where(pick > 0.98, sign * largest, x)
        steps = torch.randint(-127, 128, x.shape, generator=g) + 0.5
        x = torch.where((pick > 0.9) & (pick < 0.98), (steps * largest / 127.5).to(DT[dtype]).double(), x)
        half = (sign * (torch.randint(0, 127, x.shape, generator=g) + 0.5) * largest / 127).to(DT[dtype]).double()
        x = torch.where((pick > 0.5) & (pick < 0.8) & (254 * half % largest == 0), half, x)          # (where that is a number of the type)
        x[:, 5, :, 3] = largest[:, 0, :, 0]
        return x.view(256, heads, dim)

    k, v = some(), some()
    at = 0
    for n in cuts:
        s.grow([n], k=k[at:at + n].to(s.dt), v=v[at:at + n].to(s.dt))
        at += n
    scales = (largest / 127).expand(8, 32, heads, 1).reshape(256, heads, 1)
    for got, x in zip(s.held(0), (k, v)):
        got = got.transpose(0, 1) / scales                                            # (the cache's scale is off by 2^-24 of itself)
        assert torch.equal(got.round(), torch.round(127 * x.view(8, 32, heads, dim) / largest).view_as(x))


# ---- weights next to a rounding -----------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,group,new", [(32, 1, [1, 1]), (32, 4, [1, 4]), (32, 1, [20, 40]), (64, 2, [9, 30]), (96, 3, [7, 12]), (32, 8, [5, 8]), (128, 4, [8, 16]),
                                           (160, 1, [33, 17]), (256, 2, [16, 30])])
def test_weights_of_float16_results(comet, dim, group, new):  # noqa: F811
    """Up to 64 rows: results in float16 are as exact as float32 sums rounded once.  What rounding a weight to float16 leaves is multiplied too, so a
    weight is off by 2^-22 of itself and by 2^-25, where the largest is 2^7 at least: 2^-32 of it for each of 100 tokens, together below 2^-25
    of the largest value.  Scores are below 2 in magnitude, so d (see test_gpu_cache) is below (dim + 8) 2^-23."""
    s = Sequences(comet, torch.float16, 2, dim, 2, 160, seed=dim + group)
    held = [100 - n for n in new]
    s.grow(held)
    s.grow(new)
    q = (s.tokens(sum(new), 2 * group) * (0.5 / math.sqrt(dim))).half()
    out = s.cache.comet_cache_attend(s.batch(new), q.cuda())
    at = 0
    for b, n in enumerate(new):
        k, v = s.held(b)
        o, _, size, top = ref.attention(q[at:at + n], k, v, dim ** -0.5, True)
        assert top < 2
        d = (dim + 8) * U32 * top
        tol = (2.0 ** -22 + 2 * d + 2.0 ** -20) * size + u(s.dt) * o.abs() + 2.0 ** -25 * v.abs().max() + 2.0 ** -25
        off = (out[at:at + n].cpu().double() - o).abs()
        assert (off <= tol).all(), float((off / tol).max())
        at += n


# ---- operands in one buffer ----------------------------------------------------------------------------------------


def test_operands_side_by_side(comet):  # noqa: F811
    """Results between the operands in one buffer, where rows do not meet, give what they give elsewhere."""
    s = Sequences(comet, torch.float16, 2, 64, 2, 128, rope=comet.Rope(64), seed=8)
    s.grow([50, 20])
    new, tokens = [3, 1], 4
    fused = torch.randn(tokens, 4 + 2 + 2 + 4, 64, generator=s.g).half().cuda()          # queries, keys, values, room for the results
    q, k, v, room = fused[:, :4], fused[:, 4:6], fused[:, 6:8], fused[:, 8:]
    for b, n in enumerate(new):
        s.lens[b] += n
    batch = s.batch(new)
    want = s.cache.comet_cache_append(batch, k, v, rope=s.rope, q=q)
    s.cache.comet_cache_append(batch, k, v, rope=s.rope, q=q, q_out=room)
    assert torch.equal(room, want)
    want = s.cache.comet_cache_attend(batch, q)
    s.cache.comet_cache_attend(batch, q, out=room)
    assert torch.equal(room, want)
    pairs = torch.randn(tokens, 2, 4, 64, generator=s.g).half().cuda()                    # head by head: keys of the strides of the values
    wk, wv = s.cache.comet_cache_fetch(batch, dtype=s.dt, tokens=tokens)
    s.cache.comet_cache_fetch(batch, pairs[:, :, 0], pairs[:, :, 2])
    assert torch.equal(pairs[:, :, 0], wk) and torch.equal(pairs[:, :, 2], wv)
    want = comet.comet_rope(q, s.rope)
    comet.comet_rope(q, s.rope, out=room)
    assert torch.equal(room, want)
    by_head = torch.zeros(4, 16, 64, dtype=s.dt, device="cuda")                           # [head][token], other strides than the input's
    comet.comet_rope(q, s.rope, out=by_head[:, :tokens].transpose(0, 1))
    assert torch.equal(by_head[:, :tokens].transpose(0, 1), want)


# ---- tensors that autograd knows ----------------------------------------------------------------------------------


def test_gradients_are_not_lost(comet):  # noqa: F811
    """Calls that have no gradient refuse tensors that ask for one; what they write is known to autograd as written."""
    from paper_2111_09562_amd import autograd
    s = Sequences(comet, torch.bfloat16, 2, 64, 2, 128, rope=comet.Rope(64), seed=3)
    s.grow([40, 3])
    batch = s.batch([1, 1])
    asks = lambda heads: s.tokens(2, heads).cuda().requires_grad_()  # noqa: E731
    plain = lambda heads: s.tokens(2, heads).cuda()  # noqa: E731
    before = s.cache.buf.clone()
    k, q = plain(2), plain(4)
    for call in (lambda: comet.comet_rope(asks(2), s.rope), lambda: comet.comet_rope(k, s.rope, out=asks(2)),
                 lambda: s.cache.comet_cache_append(batch, asks(2), k), lambda: s.cache.comet_cache_append(batch, k, asks(2)),
                 lambda: s.cache.comet_cache_append(batch, k, k, q=asks(4)), lambda: s.cache.comet_cache_append(batch, k, k, q=q, q_out=asks(4)),
                 lambda: s.cache.comet_cache_fetch(batch, asks(2), k), lambda: s.cache.comet_cache_fetch(batch, k, asks(2)),
                 lambda: s.cache.comet_cache_attend(batch, asks(4)), lambda: s.cache.comet_cache_attend(batch, q, out=asks(4)),
                 lambda: s.cache.comet_cache_attend(batch, q, lse=torch.zeros(2, 4, device="cuda", requires_grad=True))):
        with pytest.raises(RuntimeError, match="gradient"):
            call()
    assert torch.equal(s.cache.buf, before)
    x = asks(2)
    with torch.no_grad():                     # where nobody asks for gradients they go through
        y = comet.comet_rope(x, s.rope)
        s.cache.comet_cache_attend(batch, asks(4))
    assert not y.requires_grad and autograd.rotate(x, s.rope).requires_grad
    with torch.inference_mode():
        a, b = s.tokens(2, 2).cuda(), s.tokens(2, 4).cuda()
        comet.comet_rope(a, s.rope, out=a)
        s.cache.comet_cache_fetch(batch, a, torch.empty_like(a))
        s.cache.comet_cache_append(batch, a, a, q=b, q_out=b)
        s.cache.comet_cache_attend(batch, b, out=torch.empty_like(b), lse=torch.empty(2, 4, device="cuda"))

    def written(t):
        """Saves t for a backward pass, writes it with the call that is given back's argument, and says whether the pass is refused."""
        w = torch.ones_like(t, requires_grad=True)
        z = (w * t).sum()
        yield t
        with pytest.raises(RuntimeError, match="inplace"):
            z.backward()

    out, lse, x = plain(4), torch.zeros(2, 4, device="cuda"), plain(2)
    for tensors, call in (([x], lambda: comet.comet_rope(x, s.rope, out=x)), ([x, k], lambda: s.cache.comet_cache_fetch(batch, x, k)),
                          ([out], lambda: s.cache.comet_cache_append(batch, k, k, q=q, q_out=out)), ([q], lambda: s.cache.comet_cache_append(batch, k, k, q=q, q_out=q)),
                          ([out, lse], lambda: s.cache.comet_cache_attend(batch, q, out=out, lse=lse))):
        open_graphs = [written(t) for t in tensors]
        for graph in open_graphs:
            next(graph)
        call()
        for graph in open_graphs:
            assert next(graph, None) is None


# ---- a rotation with an amplitude of its own -----------------------------------------------------------------------


def test_rope_amplitude(comet):  # noqa: F811
    """Frequencies scaled by parts, values kept as large as they are (or made as large as is asked for)."""
    g = gen(1)
    x = torch.randn(70, 3, 64, generator=g)
    positions = torch.randint(0, 30000, (70,), generator=g, dtype=torch.int32)
    how = dict(scaling="parts", factor=8.0, original_len=8192, beta_fast=4.0, beta_slow=1.0)
    y, tol = rope_bound(x, positions, 64, False, how)
    _, natural = ref.frequencies(64, **how)
    for amp in (1.0, 0.25, -2.0, natural):
        got = comet.comet_rope(x.cuda(), comet.Rope(64, amp=amp, **how), positions.cuda())
        assert ((got.cpu().double() - y * (amp / natural)).abs() <= tol * abs(amp / natural) + U32 * y.abs() * abs(amp)).all()
    assert comet.Rope(64, **how).amp == pytest.approx(natural, rel=2.0 ** -24)
