"""The compressed key/value cache on the GPU against its definition in 64 bits (cache_reference): rotations with their gradients, what
the cache holds after an append, what a fetch gives back, attention over it, and a serving run of all of them.

Tolerances.  u(t) = finfo(t).eps / 2 is half a step of type t.  A rotation in float32 does six roundings on values of at most
amp * (|a| + |b|), sines and cosines included: 6 u(float32) of that, and u(t) of the result.  A compressed value is off by half its
scale.  Attention: scores are sums of dim products in float32, so off by at most d = (dim + 8) u(float32) times the largest sum of
|q k| scale, which changes every weight by at most a factor 1 + 2d; a weight is rounded to float16 once; the result to t once."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")
import cache_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
DT = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def comet():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2111_09562_amd import comet as libcomet
    libcomet.lib()
    return libcomet


def u(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- rotation -----------------------------------------------------------------------------------------------------


def rope_bound(x, positions, rot, interleaved, how, sign=1.0):
    """Where every value of a rotation may lie: (value, tolerance) in 64 bits.  (Half a step is one of the value itself: a rotation
    the other way has other values.)"""
    y = ref.rotated(x, positions, rot, interleaved, sign=sign, **how)
    _, amp = ref.frequencies(rot, **how)
    ia = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    size = torch.zeros_like(y)
    size[..., ia] = size[..., ib] = amp * (x.double()[..., ia].abs() + x.double()[..., ib].abs())
    return y, 6 * U32 * size + u(x.dtype) * y.abs() * (1 + 8 * U32) + torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps


@pytest.mark.parametrize("dtype,tokens,heads,dim,rot,interleaved,how,strided", [
    ("fp32", 1, 1, 2, 2, False, {}, False),
    ("fp32", 257, 3, 34, 34, True, {}, False),
    ("fp32", 65, 5, 96, 64, True, {"scaling": "parts", "factor": 8.0}, True),
    ("bf16", 1, 32, 128, 128, False, {}, False),
    ("bf16", 1000, 7, 128, 64, False, {"scaling": "linear", "factor": 3.0}, True),
    ("bf16", 77, 40, 192, 192, True, {"scaling": "base", "factor": 4.0}, False),
    ("bf16", 19, 3, 100, 50, False, {}, False),
    ("fp16", 513, 2, 64, 32, True, {}, True),
    ("fp16", 33, 65, 80, 80, False, {}, False),
    ("fp16", 5, 130, 256, 16, False, {}, False),
    ("bf16", 4099, 9, 64, 64, False, {}, True)])
def test_rope(comet, dtype, tokens, heads, dim, rot, interleaved, how, strided):
    g = gen(tokens + heads)
    whole = torch.randn(tokens, heads + (3 if strided else 0), dim, generator=g).to(DT[dtype])
    x = whole[:, :heads]
    positions = torch.randint(-5, 1 << 20, (tokens,), generator=g, dtype=torch.int32)
    positions[0] = 2 ** 31 - 1 if tokens > 4 else 77
    rope = comet.Rope(rot, interleaved=interleaved, **how)
    xd, pd = whole.cuda()[:, :heads], positions.cuda()
    for sign in (1.0, -1.0):
        y, tol = rope_bound(x, positions, rot, interleaved, how, sign)
        got = comet.comet_rope(xd, rope, pd, backward=sign < 0)
        assert got.dtype == x.dtype and got.shape == x.shape
        # the reference's angles have 53 bits: at 2^31 radians 2^-22 of one, what is left of them there is compared with room for that
        far = (positions.double().abs() * 2.0 ** -52)[:, None, None]
        size = x.double().abs().amax() * 4
        assert ((got.cpu().double() - y).abs() <= tol + far * size).all()
    # no positions: 0, 1, ..; in place; the part behind rot is untouched
    y, tol = rope_bound(x, torch.arange(tokens), rot, interleaved, how)
    inp = xd.clone()
    assert comet.comet_rope(inp, rope, out=inp) is inp
    assert ((inp.cpu().double() - y).abs() <= tol).all()
    assert torch.equal(inp.cpu()[..., rot:], x[..., rot:])


def test_rope_gradient(comet):
    """Against the formula (the transposed rotation) and against differences of the forward pass in the direction of a random change."""
    from paper_2111_09562_amd import autograd
    g = gen(3)
    x = torch.randn(50, 6, 64, generator=g, dtype=torch.float32)
    w, d = torch.randn(50, 6, 64, generator=g), torch.randn(50, 6, 64, generator=g)
    positions = torch.randint(0, 5000, (50,), generator=g, dtype=torch.int32)
    rope = comet.Rope(48, interleaved=True, scaling="parts", factor=4.0)
    xd = x.cuda().requires_grad_()
    y = autograd.rotate(xd, rope, positions.cuda())
    (y * w.cuda()).sum().backward()
    how = {"scaling": "parts", "factor": 4.0}
    want, tol = rope_bound(w, positions, 48, True, how, -1.0)
    assert ((xd.grad.cpu().double() - want).abs() <= tol + 1e-9).all()
    # linear in x, so a difference of any step is exact but for roundings: |x| + |d| at most 6, 64 * 300 values at 6 u each
    f = lambda t: float((comet.comet_rope(t.cuda(), rope, positions.cuda()).cpu().double() * w.double()).sum())  # noqa: E731
    lhs, rhs = f(x + d) - f(x), float((xd.grad.cpu().double() * d.double()).sum())
    assert abs(lhs - rhs) <= 8 * U32 * float(((x.abs() + d.abs()).double() * 4 * w.abs().double()).sum())
    # a gradient with strides of its own, and a half of it without any
    z = autograd.rotate(xd.to(torch.bfloat16), rope, positions.cuda())
    z.transpose(0, 1).float().sum().backward()
    assert torch.isfinite(xd.grad).all()


def test_rope_second_gradient_and_capture(comet):
    """Positions 0, 1, ..; the gradient of the gradient (a rotation again); a training step captured in a graph follows its inputs."""
    from paper_2111_09562_amd import autograd
    rope = comet.Rope(64)
    g = gen(11)
    x, w, z = (torch.randn(40, 3, 64, generator=g, device="cpu") for _ in range(3))
    xd, wd = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    (dx,) = torch.autograd.grad(autograd.rotate(xd, rope), xd, wd, create_graph=True)
    (dw,) = torch.autograd.grad(dx, wd, z.cuda())
    positions = torch.arange(40)
    y, tol = rope_bound(w, positions, 64, False, {}, -1.0)
    assert ((dx.detach().cpu().double() - y).abs() <= tol).all()
    y, tol = rope_bound(z, positions, 64, False, {})
    assert ((dw.cpu().double() - y).abs() <= tol).all()

    pos = torch.zeros(40, dtype=torch.int32, device="cuda")
    static, grad = torch.zeros(40, 3, 64, device="cuda"), torch.zeros(40, 3, 64, device="cuda")

    def step():
        leaf = static.detach().requires_grad_()
        out = autograd.rotate(leaf, rope, pos)
        return out.detach(), torch.autograd.grad(out, leaf, grad)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, dleaf = step()
    for i in range(5):
        static.copy_(torch.randn(static.shape, generator=g))
        grad.copy_(torch.randn(static.shape, generator=g))
        pos.copy_(torch.randint(0, 1 << 16, (40,), generator=g, dtype=torch.int32))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(dleaf, want[1])


# ---- sequences in a cache -----------------------------------------------------------------------------------------


class Sequences:
    """Sequences that grow in a cache, with what they hold on the CPU: the 16-bit keys (rotated by the library, checked apart) and values."""

    def __init__(self, comet, dtype, heads, dim, seqs, most, page=64, rope=None, seed=0, slots=None):
        self.comet, self.dt, self.heads, self.dim, self.n, self.page = comet, dtype, heads, dim, seqs, page
        self.g = gen(seed)
        per_seq = -(-most // page)
        self.pages = seqs * per_seq + 2
        self.cache = comet.Cache(self.pages, page, seqs + 1, heads, dim)
        self.cache.buf.fill_(0xFF)                                        # NaN wherever nobody has written
        self.table = torch.randperm(self.pages, generator=self.g)[:seqs * per_seq].to(torch.int32).view(seqs, per_seq)
        self.slots = torch.randperm(seqs + 1, generator=self.g)[:seqs].to(torch.int32)
        self.lens = [0] * seqs
        self.k = [torch.zeros(0, heads, dim) for _ in range(seqs)]
        self.v = [torch.zeros(0, heads, dim) for _ in range(seqs)]
        self.rope = rope
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def batch(self, new, lens=None):
        starts = torch.tensor([0] + list(itertools.accumulate(new)), dtype=torch.int32)
        lens = self.lens if lens is None else lens
        return self.comet.Batch(starts.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), self.table.cuda(), self.slots.cuda())

    def tokens(self, n, heads):
        return torch.randn(n, heads, self.dim, generator=self.g).to(self.dt)

    def grow(self, new, pad=0, odd=False, k=None, v=None, **kw):
        total = sum(new)
        k = self.tokens(total, self.heads) * 2 if k is None else k
        v = self.tokens(total, self.heads) if v is None else v
        room = torch.full((total + pad, self.heads + 1, self.dim + (1 if odd else 0)), float("nan"), dtype=self.dt)   # odd: rows that begin anywhere
        kd, vd = room.clone().cuda(), room.clone().cuda()
        kd[:total, :self.heads, :self.dim], vd[:total, :self.heads, :self.dim] = k.cuda(), v.cuda()
        at = 0
        for b, n in enumerate(new):
            self.lens[b] += n
            self.k[b], self.v[b] = torch.cat((self.k[b], k[at:at + n].float())), torch.cat((self.v[b], v[at:at + n].float()))
            at += n
        batch = self.batch(new)
        got = self.cache.comet_cache_append(batch, kd[:, :self.heads, :self.dim], vd[:, :self.heads, :self.dim], rope=self.rope, status=self.status, **kw)
        return batch, got

    def held(self, b):
        return ref.held(self.cache, self.table, self.lens, self.slots, b)

    def ok(self):
        return int(self.status.item()) == 0


def check_held(s, b, keys=None):
    """What the cache holds of a sequence against the 16-bit values that came (keys: those of the rotated keys, with a tolerance)."""
    k, v = s.held(b)
    whole = s.lens[b] // 32 * 32
    want_k, tol_k = (s.k[b].double(), torch.zeros_like(s.k[b], dtype=torch.float64)) if keys is None else keys
    for got, want, tol in ((k, want_k, tol_k), (v, s.v[b].double(), torch.zeros_like(s.v[b], dtype=torch.float64))):
        got = got.transpose(0, 1)
        assert got.shape == want.shape
        if whole:
            w = want[:whole].view(-1, 32, s.heads, s.dim)
            t = tol[:whole].view_as(w)
            # scale: the largest of the block / 127; half of it, with room for the quotient's and the scale's roundings, and for what the
            # largest value itself may be off
            top = w.abs().amax((1, 3), keepdim=True)
            off = (got[:whole].view_as(w) - w).abs()
            assert (off <= ((top + t.amax((1, 3), keepdim=True)) / 254).clamp_min(2.0 ** -101) * (1 + 2.0 ** -14) + t).all()
        # 16 bits: the values themselves (float16 times a power of two of the token: exact down to 2^-39 of its largest value)
        top = want[whole:].abs().amax(-1, keepdim=True)
        assert ((got[whole:] - want[whole:]).abs() <= tol[whole:] + top * 2.0 ** -38).all()


def check_attend(s, q_new, q, out, lse, causal=True, scale=None, lens=None):
    scale = s.dim ** -0.5 if scale is None else scale
    at = 0
    for b, n in enumerate(q_new):
        if n == 0:
            continue
        total = (s.lens if lens is None else lens)[b]
        k, v = ref.held(s.cache, s.table, s.lens if lens is None else lens, s.slots, b)
        o, want_lse, size, top = ref.attention(q[at:at + n], k, v, scale, causal)
        d = (s.dim + 8) * U32 * top
        tol = (u(torch.float16) + 2 * d + 2.0 ** -19) * size + u(s.dt) * o.abs() + 2.0 ** -24
        got = out[at:at + n].cpu().double()
        assert ((got - o).abs() <= tol).all(), (b, n, total, float(((got - o).abs() - tol).max()))
        got = lse[at:at + n].cpu().double()
        finite = want_lse > -math.inf
        assert torch.equal(got > -math.inf, finite)
        assert ((got - want_lse)[finite].abs() <= d + 2.0 ** -20 * (1 + want_lse[finite].abs())).all()
        at += n


@pytest.mark.parametrize("dtype,heads,dim,page,odd", [("bf16", 2, 128, 64, False), ("fp16", 3, 64, 32, False), ("bf16", 1, 32, 160, True), ("fp16", 2, 96, 64, True),
                                                      ("bf16", 5, 160, 96, False), ("fp16", 1, 192, 32, False), ("bf16", 2, 224, 64, True), ("fp16", 2, 256, 128, False)])
def test_append_and_fetch(comet, dtype, heads, dim, page, odd):
    """Tokens in pieces of every kind: none, one, up to a block's end, over several blocks from the middle of one, a whole prompt."""
    s = Sequences(comet, DT[dtype], heads, dim, 5, 512, page, seed=dim)
    for new in ([3, 0, 64, 1, 200], [29, 1, 0, 0, 1], [0, 31, 5, 98, 140], [1, 32, 27, 30, 0], [130, 1, 64, 97, 1], [32, 33, 1, 2, 31]):
        batch, _ = s.grow(new, pad=2, odd=odd)
        for b in range(s.n):
            check_held(s, b)
        total = sum(new)
        room = torch.full((total + 3, heads, dim + (1 if odd else 0)), 7.0, dtype=s.dt, device="cuda")
        k, v = room.clone()[..., :dim], room.clone()[..., :dim]
        s.cache.comet_cache_fetch(batch, k, v, status=s.status)
        assert (k[total:] == 7).all() and (v[total:] == 7).all()          # rows behind the last sequence
        at = 0
        for b, n in enumerate(new):
            for got, want in zip((k, v), s.held(b)):
                want = want[:, s.lens[b] - n:].transpose(0, 1)
                # one product in float32, one rounding to the type
                assert ((got[at:at + n].cpu().double() - want).abs() <= (u(s.dt) + 2 * U32) * want.abs() + 2.0 ** -25).all()
            at += n
    assert s.ok()


@pytest.mark.parametrize("dtype,heads,q_heads,dim,rot,interleaved,how", [("bf16", 2, 8, 128, 128, False, {}), ("fp16", 3, 3, 64, 32, True, {"scaling": "linear", "factor": 2.0}),
                                                                         ("bf16", 1, 17, 96, 34, False, {}), ("fp16", 2, 2, 256, 256, True, {"scaling": "parts", "factor": 8.0})])
def test_append_turns_keys_and_queries(comet, dtype, heads, q_heads, dim, rot, interleaved, how):
    s = Sequences(comet, DT[dtype], heads, dim, 3, 300, rope=comet.Rope(rot, interleaved=interleaved, **how), seed=rot)
    for new in ([40, 1, 100], [1, 3, 61], [90, 0, 1]):
        q = s.tokens(sum(new), q_heads)
        before = list(s.lens)
        _, got = s.grow(new, q=q.cuda())
        positions = torch.cat([torch.arange(a, a + n) for a, n in zip(before, new)])
        y, tol = rope_bound(q, positions, rot, interleaved, how)
        assert ((got.cpu().double() - y).abs() <= tol).all()
        for b in range(s.n):
            y, tol = rope_bound(s.k[b].to(s.dt), torch.arange(s.lens[b]), rot, interleaved, how)
            check_held(s, b, (y, tol))
    # positions given, queries turned in place
    new = [2, 2, 2]
    positions = torch.tensor([5, 100000, 7, 7, 0, 1], dtype=torch.int32)
    q = s.tokens(6, q_heads).cuda()
    y, tol = rope_bound(q.cpu(), positions, rot, interleaved, how)
    _, got = s.grow(new, q=q, q_out=q, positions=positions.cuda())
    assert got is q and ((q.cpu().double() - y).abs() <= tol).all()
    assert s.ok()


def test_bytes_do_not_depend_on_how_tokens_came(comet):
    """A prompt at once, in pieces, token by token: the same complete blocks, bit for bit, and the same open block."""
    total, outs = 150, []
    for cuts in ([150], [32, 64, 54], [7, 50, 1, 92], [1] * 150, [149, 1]):
        s = Sequences(comet, torch.bfloat16, 2, 64, 1, 192, rope=comet.Rope(64), seed=9)
        g = gen(5)
        k, v = torch.randn(total, 2, 64, generator=g).bfloat16(), torch.randn(total, 2, 64, generator=g).bfloat16()
        at = 0
        for n in cuts:
            s.grow([n], k=k[at:at + n], v=v[at:at + n])
            at += n
        outs.append([x.clone() for x in s.held(0)])
        # set back into the block before, the last 20 tokens once more: nothing changes
        s.lens[0] -= 20
        s.k[0], s.v[0] = s.k[0][:-20], s.v[0][:-20]
        short = s.held(0)
        assert all(torch.equal(a[:, :128], b[:, :128]) for a, b in zip(short, outs[-1]))
        s.grow([20], k=k[130:], v=v[130:])
        assert all(torch.equal(a, b) for a, b in zip(s.held(0), outs[-1]))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_set_back_over_a_block(comet):
    """Drafted tokens that complete a block and are not taken: the open block of the shorter length is still there in 16 bits."""
    s = Sequences(comet, torch.float16, 2, 64, 1, 192, seed=4)
    s.grow([94])
    for back, new in ((0, 5), (5, 3), (31, 40)):                          # 99 -> 94 + 3 = 97 -> 66 + 40
        s.lens[0] -= back
        s.k[0], s.v[0] = s.k[0][:s.lens[0]], s.v[0][:s.lens[0]]
        check_held(s, 0)
        s.grow([new])
        check_held(s, 0)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,group,dim,new,causal", [
    (2, 4, 128, [1, 1, 1, 1], True), (1, 1, 64, [1, 0, 5, 33], True), (3, 8, 32, [2, 4, 1, 0], True), (2, 3, 96, [11, 7, 64, 1], False), (1, 40, 64, [1, 2, 3, 1], True),
    (2, 1, 160, [100, 3, 1, 40], True), (1, 16, 192, [1, 1, 9, 2], False), (2, 2, 224, [17, 1, 1, 1], True), (1, 4, 256, [9, 1, 70, 31], True), (4, 1, 128, [130, 65, 1, 128], True)])
def test_attend(comet, dtype, heads, group, dim, new, causal):
    s = Sequences(comet, DT[dtype], heads, dim, 4, 1400, seed=dim + heads)
    s.grow([700, 31, 1, 1096])
    s.grow(new)
    q = s.tokens(sum(new) + 2, heads * group) * 2
    batch = s.batch(new)
    out = torch.full_like(q, 5.0, device="cuda")
    out, lse = s.cache.comet_cache_attend(batch, q.cuda(), out=out, lse=True, causal=causal, status=s.status)
    check_attend(s, new, q, out, lse, causal)
    assert (out[sum(new):] == 5).all()                                    # rows behind the last sequence
    assert s.ok()
    # the same again, bit for bit: nothing depends on the order in which workgroups end
    out2, lse2 = s.cache.comet_cache_attend(batch, q.cuda(), lse=True, causal=causal)
    assert torch.equal(out2[:sum(new)], out[:sum(new)]) and torch.equal(lse2[:sum(new)], lse[:sum(new)])


@pytest.mark.parametrize("dtype,heads,group,dim,held,new,causal", [
    ("bf16", 2, 4, 128, [0, 0, 0], [300, 1, 130], True), ("fp16", 1, 1, 64, [0, 700, 33], [700, 200, 0], True), ("bf16", 1, 16, 32, [2500, 5], [40, 9], True),
    ("fp16", 2, 3, 96, [100, 3000], [257, 64], False), ("bf16", 1, 5, 160, [64, 31], [100, 33], True), ("fp16", 1, 8, 192, [2000], [70], True),
    ("bf16", 1, 2, 224, [500, 0], [129, 300], False), ("fp16", 2, 2, 256, [96, 1500], [256, 65], True), ("bf16", 3, 1, 128, [4000], [128], True)])
def test_attend_many_rows(comet, dtype, heads, group, dim, held, new, causal):
    """Prompts and pieces of prompts: tiles of rows, blocks that some of a tile's rows see, long ranges that are cut."""
    s = Sequences(comet, DT[dtype], heads, dim, len(new), 4300, page=128, seed=dim + heads)
    s.grow(held)
    s.grow(new)
    q = s.tokens(sum(new) + 1, heads * group) * 2
    batch = s.batch(new)
    out = torch.full_like(q, 5.0, device="cuda")
    out, lse = s.cache.comet_cache_attend(batch, q.cuda(), out=out, lse=True, causal=causal, status=s.status)
    check_attend(s, new, q, out, lse, causal)
    assert (out[sum(new):] == 5).all() and s.ok()
    out2, lse2 = s.cache.comet_cache_attend(batch, q.cuda(), lse=True, causal=causal)
    assert torch.equal(out2[:sum(new)], out[:sum(new)]) and torch.equal(lse2[:sum(new)], lse[:sum(new)])
    if causal:                                # fewer tokens held than queries: the first rows see nothing
        lens = [n - n // 2 for n in new]
        out, lse = s.cache.comet_cache_attend(s.batch(new, lens=lens), q.cuda(), lse=True)
        full = [n % 32 == 0 for n in lens]    # (an open block of that length is not in the ring any more)
        at = 0
        for b, n in enumerate(new):
            assert not out[at:at + n // 2].any() and (lse[at:at + n // 2] == -math.inf).all()
            if full[b] and n:
                one = Sequences.__new__(Sequences)
                one.__dict__.update(s.__dict__, lens=lens)
                k, v = one.held(b)
                o, _, size, top = ref.attention(q[at:at + n], k, v, dim ** -0.5, True)
                d = (dim + 8) * U32 * top
                assert ((out[at:at + n].cpu().double() - o).abs() <= (u(torch.float16) + 2 * d + 2.0 ** -19) * size + u(s.dt) * o.abs() + 2.0 ** -24).all()
            at += n


def test_many_rows_and_missing_pages(comet):
    """A page that is none in the middle of a prompt's cache, and a block of NaN: the same values as with few rows at a time, where every call
    goes another way through the library."""
    s = Sequences(comet, torch.bfloat16, 1, 64, 1, 1024, seed=14)
    k, v = s.tokens(900, 1), s.tokens(900, 1)
    v[777] = float("nan")
    s.grow([900], k=k, v=v)
    q = s.tokens(300, 4)
    s.table[0, 5] = -1                                                    # tokens 320 .. 383
    out, lse = s.cache.comet_cache_attend(s.batch([300]), q.cuda(), lse=True, status=s.status)
    assert int(s.status.item()) == comet.ERR_FORMAT
    k, v = ref.held(s.cache, s.table.clamp_min(0), s.lens, s.slots, 0)
    keep = torch.ones(900, dtype=torch.bool)
    keep[320:384] = False
    for i in (0, 100, 167, 168, 250, 299):
        seen = keep[:601 + i]
        o, want, size, top = ref.attention(q[i:i + 1], k[:, :601 + i][:, seen], v[:, :601 + i][:, seen], 0.125, False)
        d = 72 * U32 * top
        assert ((lse[i].cpu().double() - want).abs() <= d + 2.0 ** -18).all()
        if 601 + i > 768:
            assert out[i].isnan().all()
        else:
            assert ((out[i].cpu().double() - o).abs() <= (u(torch.float16) + 2 * d + 2.0 ** -19) * size + u(s.dt) * o.abs()).all()


@pytest.mark.parametrize("lens,new", [([1], [1]), ([32], [1]), ([33], [33]), ([31, 1, 64], [31, 1, 2]), ([0, 5, 0], [2, 3, 0]), ([3, 40], [9, 50])])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_short(comet, lens, new, causal):
    """One token, whole blocks, nothing held at all, more queries than tokens (rows that see nothing)."""
    s = Sequences(comet, torch.bfloat16, 2, 64, len(lens), 128, seed=1)
    s.grow(lens)
    q = s.tokens(sum(new), 6)
    out, lse = s.cache.comet_cache_attend(s.batch(new), q.cuda(), lse=True, causal=causal, status=s.status)
    check_attend(s, new, q, out, lse, causal)
    assert s.ok()


@pytest.mark.parametrize("seqs,most_new,group", [(65, 1, 2), (300, 1, 4), (1000, 2, 1), (300, 40, 4), (40, 90, 2)])
def test_many_sequences(comet, seqs, most_new, group):
    """More sequences than a wavefront has lanes and than a workgroup has threads, some without tokens."""
    g = gen(seqs)
    s = Sequences(comet, torch.bfloat16, 1, 32, seqs, 320, seed=seqs)
    s.grow(torch.randint(0, 200, (seqs,), generator=g).tolist())
    new = torch.randint(0, most_new + 1, (seqs,), generator=g).tolist()
    new[0], new[-1] = 0, most_new
    s.grow(new)
    q = s.tokens(sum(new), group)
    out, lse = s.cache.comet_cache_attend(s.batch(new), q.cuda(), lse=True, status=s.status)
    check_attend(s, new, q, out, lse)
    k, v = s.cache.comet_cache_fetch(s.batch(new), dtype=s.dt, tokens=sum(new))
    at = 0
    for b, n in enumerate(new):
        check_held(s, b)
        want = s.held(b)[1][:, s.lens[b] - n:].transpose(0, 1)
        assert ((v[at:at + n].cpu().double() - want).abs() <= (u(s.dt) + 2 * U32) * want.abs() + 2.0 ** -25).all()
        at += n
    assert s.ok()


def test_attend_strides_and_options(comet):
    s = Sequences(comet, torch.float16, 2, 96, 2, 200, seed=2)
    s.grow([100, 50])
    new = [3, 1]
    q = s.tokens(4, 4)
    wide = torch.zeros(4, 9, 97, dtype=torch.float16, device="cuda")      # rows of 97: no 16-byte loads or stores
    wide[:, 2:6, :96] = q.cuda()
    out = torch.zeros(4, 5, 99, dtype=torch.float16, device="cuda")
    lse = torch.zeros(4, 4, device="cuda")
    work = torch.full((comet.comet_cache_attend_work(s.cache, 2, 4, 4),), 0xFF, dtype=torch.uint8, device="cuda")
    got = s.cache.comet_cache_attend(s.batch(new), wide[:, 2:6, :96], out=out[:, 1:, :96], lse=lse, scale=0.3, work=work)
    check_attend(s, new, q, got[0], got[1], scale=0.3)
    assert not out[:, 0].any() and not out[..., 96:].any()
    plain = s.cache.comet_cache_attend(s.batch(new), q.cuda(), scale=0.3)
    assert torch.equal(plain, out[:, 1:, :96])
    zero, _ = s.cache.comet_cache_attend(s.batch(new), q.cuda(), scale=0.0, lse=True, causal=False)
    for b, rows in enumerate((zero[:3], zero[3:])):                       # scale 0: the mean of the values
        want = s.held(b)[1].mean(1).repeat_interleave(2, 0)
        assert ((rows.cpu().double() - want).abs() <= 2.0 ** -10).all()


def test_scales_far_apart(comet):
    """Blocks whose values differ by factors of 2^60, keys of next to nothing, a huge query: weights and sums keep their place."""
    s = Sequences(comet, torch.bfloat16, 1, 64, 1, 256, seed=6)
    k, v = s.tokens(160, 1), s.tokens(160, 1)
    for j, f in enumerate((2.0 ** 30, 2.0 ** -30, 1.0, 2.0 ** -30, 2.0 ** 20)):
        v[32 * j:32 * j + 32] *= f
    k[:32] *= 2.0 ** -40
    v[70:72] = 0
    s.grow([150], k=k[:150], v=v[:150])
    check_held(s, 0)
    for f in (1.0, 2.0 ** -50, 2.0 ** 5):
        q = (s.tokens(2, 2) * f).bfloat16()
        out, lse = s.cache.comet_cache_attend(s.batch([2]), q.cuda(), lse=True)
        check_attend(s, [2], q, out, lse)
    # a hundred thousand equal weights of 2^-24 beside one of 1 are not lost: tokens with scores 24 ln 2 below the first
    s = Sequences(comet, torch.float16, 1, 32, 1, 1 << 17, page=1024, seed=6)
    n = 100000
    k, v = torch.zeros(n, 1, 32, dtype=torch.float16), torch.full((n, 1, 32), 64.0, dtype=torch.float16)
    k[:, 0, 0] = -24 * math.log(2.0)
    k[:32, 0, 0] = 0.0
    v[:32] = 0.25
    k[1:32, 0, 0] = -24 * math.log(2.0)
    s.grow([n], k=k, v=v)
    q = torch.zeros(1, 1, 32, dtype=torch.float16)
    q[..., 0] = 1.0
    out, lse = s.cache.comet_cache_attend(s.batch([1]), q.cuda(), lse=True, scale=1.0)
    check_attend(s, [1], q, out, lse, scale=1.0)


def test_inf_and_nan(comet):
    """A token with NaN makes NaN of its block and head for those that see the block, and of nothing else."""
    for where in (5, 33, 66):                                             # a complete block, another, the open one
        s = Sequences(comet, torch.bfloat16, 2, 64, 2, 128, seed=where)
        k, v = s.tokens(70 + 20, 2), s.tokens(70 + 20, 2)
        bad_k, bad_v = k.clone(), v.clone()
        bad_v[where, 0, 3] = float("nan")
        bad_k[where, 1, 9] = float("inf")
        s.grow([70, 20], k=bad_k, v=bad_v)
        clean = Sequences(comet, torch.bfloat16, 2, 64, 2, 128, seed=where)
        clean.grow([70, 20], k=k, v=v)
        q = s.tokens(72, 4)
        new = [70, 2]
        out, lse = s.cache.comet_cache_attend(s.batch(new), q.cuda(), lse=True)
        want, want_lse = clean.cache.comet_cache_attend(clean.batch(new), q.cuda(), lse=True)
        first = where // 32 * 32 if where < 64 else where                 # the open block's tokens have scales of their own
        assert torch.equal(out[:first], want[:first]) and torch.equal(out[70:], want[70:]) and torch.equal(lse[:first], want_lse[:first])
        assert out[first:70].isnan().all()
        # The values' NaN is no score's.  (Poisoned blocks take the way of blocks that not all rows see, which rounds in another order: each of both
        # is off by at most (dim + 8) u(float32) times sum |q k| scale, here below 32, and 2^-20 of the sum's logarithm, here below 7.)
        assert ((lse[first:70, :2] - want_lse[first:70, :2]).abs() <= 2 * (72 * U32 * 32 + 2.0 ** -20 * 8)).all() and lse[first:70, 2:].isnan().all()
        fk, fv = s.cache.comet_cache_fetch(s.batch([70, 20]), dtype=torch.bfloat16, tokens=90)
        end = min(70, first + 32) if where < 64 else where + 1
        assert fv[first:end, 0].isnan().all() and fk[first:end, 1].isnan().all()
        assert fk[:, 0].isfinite().all() and fv[:, 1].isfinite().all() and fv[:first].isfinite().all() and fv[end:].isfinite().all()
    # a query with NaN or Inf: its own row alone
    s = Sequences(comet, torch.float16, 1, 64, 1, 128, seed=8)
    s.grow([100])
    q = s.tokens(6, 2)
    want = s.cache.comet_cache_attend(s.batch([6]), q.cuda())
    q[2, 1, 0], q[4, 0, 63] = float("nan"), float("inf")
    out = s.cache.comet_cache_attend(s.batch([6]), q.cuda())
    bad = torch.zeros(6, 2, dtype=torch.bool)
    bad[2, 1] = bad[4, 0] = True
    assert out[bad.cuda()].isnan().all() and torch.equal(out[~bad.cuda()], want[~bad.cuda()])


def test_numbers_that_make_no_sense(comet):
    """Pages, slots, starts and lengths that are none: reported, skipped, nothing else is touched.  (Every such number is caught by the
    kernels' own checks before an address is made of it.)"""
    s = Sequences(comet, torch.float16, 2, 64, 3, 256, seed=3)
    s.grow([100, 64, 40])
    before = s.cache.buf.clone()
    good = s.table.clone()

    def attempt(what):
        s.status.zero_()
        what()
        torch.cuda.synchronize()
        assert int(s.status.item()) == comet.ERR_FORMAT

    k = torch.ones(3, 2, 64, dtype=torch.float16, device="cuda")
    q = torch.ones(3, 2, 64, dtype=torch.float16, device="cuda")
    for page in (-1, s.pages, 2 ** 31 - 1, -2 ** 31):
        s.table = good.clone()
        s.table[0, 1] = page                                              # tokens 64 .. of sequence 0
        batch = s.batch([1, 1, 1])
        attempt(lambda: s.cache.comet_cache_attend(batch, q, status=s.status))
        out, lse = s.cache.comet_cache_attend(batch, q, lse=True)
        assert out.isfinite().all()
        attempt(lambda: s.cache.comet_cache_fetch(s.batch([100, 0, 0]), dtype=torch.float16, tokens=100, status=s.status))
    s.table = good
    slots = s.slots.clone()
    for slot in (-1, 4, 2 ** 31 - 1):
        s.slots = slots.clone()
        s.slots[2] = slot
        attempt(lambda: s.cache.comet_cache_append(s.batch([0, 0, 1]), k[:1], k[:1], status=s.status))
        attempt(lambda: s.cache.comet_cache_attend(s.batch([1, 1, 1]), q, status=s.status))
    s.slots = slots
    for starts in ([0, 1, 2, 4], [0, 2, 1, 3], [-1, 1, 2, 3], [0, 2 ** 31 - 1, 2, 3]):
        b = comet.Batch(torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(s.lens, dtype=torch.int32).cuda(), s.table.cuda(), s.slots.cuda())
        s.cache.comet_cache_attend(b, q)                                  # rows that belong to no sequence have no values: only ends
        torch.cuda.synchronize()
    attempt(lambda: s.cache.comet_cache_append(s.batch([1, 0, 0], lens=[0, 64, 40]), k[:1], k[:1], status=s.status))     # one token of none
    attempt(lambda: s.cache.comet_cache_append(s.batch([0, 0, 1], lens=[100, 64, -7]), k[:1], k[:1], status=s.status))
    attempt(lambda: s.cache.comet_cache_append(s.batch([1, 0, 0], lens=[2 ** 31 - 1, 64, 40]), k[:1], k[:1], status=s.status))
    assert torch.equal(s.cache.buf, before)
    # the table ends before the sequence does: the block cannot be put anywhere, the others are
    narrow = comet.Batch(torch.tensor([0, 0, 0, 32], dtype=torch.int32).cuda(), torch.tensor([100, 64, 72], dtype=torch.int32).cuda(),
                         s.table[:, :1].contiguous().cuda(), s.slots.cuda())
    kk = torch.ones(32, 2, 64, dtype=torch.float16, device="cuda")
    s.status.zero_()
    s.cache.comet_cache_append(narrow, kk, kk, status=s.status)           # completes block 1 of page 0, the rest stays open
    assert int(s.status.item()) == 0
    longer = comet.Batch(torch.tensor([0, 0, 0, 32], dtype=torch.int32).cuda(), torch.tensor([100, 64, 104], dtype=torch.int32).cuda(),
                         s.table[:, :1].contiguous().cuda(), s.slots.cuda())
    attempt(lambda: s.cache.comet_cache_append(longer, kk, kk, status=s.status))


def test_graph_follows_the_lengths(comet):
    """A step captured once, replayed while the sequences grow: every replay equals the eager calls."""
    def step(s, batch, k, v, q, out, q_out):
        s.cache.comet_cache_append(batch, k, v, rope=s.rope, q=q, q_out=q_out)
        s.cache.comet_cache_attend(batch, q_out, out=out)

    runs = []
    for captured in (False, True):
        s = Sequences(comet, torch.bfloat16, 2, 64, 3, 256, rope=comet.Rope(64), seed=12)
        s.grow([60, 3, 0])
        g = gen(77)
        k, v = (torch.zeros(3, 2, 64, dtype=s.dt, device="cuda") for _ in range(2))
        q, out, q_out = (torch.zeros(3, 8, 64, dtype=s.dt, device="cuda") for _ in range(3))
        batch = s.batch([1, 1, 1])
        lens = batch.tensors[1]
        graph = None
        outs = []
        if captured:
            graph = torch.cuda.CUDAGraph()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):                                 # (the append of places that are overwritten by the replays)
                lens.add_(1)
                step(s, batch, k, v, q, out, q_out)
                lens.sub_(1)
            torch.cuda.current_stream().wait_stream(side)
            with torch.cuda.graph(graph):
                step(s, batch, k, v, q, out, q_out)
        for i in range(40):
            for t in (k, v, q):
                t.copy_(torch.randn(t.shape, generator=g))
            lens.add_(1)
            if captured:
                graph.replay()
            else:
                step(s, batch, k, v, q, out, q_out)
            if i % 7 == 0:
                torch.cuda.synchronize()
                torch.randn(1000, 1000, device="cuda").sum().item()       # other work between the replays
            outs.append(out.clone())
        runs.append(torch.stack(outs))
        torch.cuda.synchronize()
    assert torch.equal(runs[0], runs[1]) and runs[0].isfinite().all()


def test_streams(comet):
    """Two calls at once on streams of their own, each with a workspace of its own, on the same cache."""
    s = Sequences(comet, torch.bfloat16, 4, 128, 4, 4096, seed=21)
    s.grow([4000, 3000, 100, 2])
    qs = [s.tokens(4, 16).cuda() for _ in range(2)]
    want = [s.cache.comet_cache_attend(s.batch([1, 1, 1, 1]), q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    batch = s.batch([1, 1, 1, 1])
    torch.cuda.synchronize()
    for _ in range(5):
        got = [s.cache.comet_cache_attend(batch, q, stream=st) for q, st in zip(qs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    y = comet.comet_rope(qs[0], comet.Rope(128), stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(y, comet.comet_rope(qs[0], comet.Rope(128)))


def test_offsets_beyond_32_bits(comet):
    """A cache of more than 4 GB: blocks at its end are where they should be."""
    heads, dim, page = 8, 128, 1024
    pages = (5 << 30) // (heads * page * dim * 2)
    cache = comet.Cache(pages, page, 1, heads, dim)
    assert cache.nbytes > 1 << 32
    g = gen(2)
    k, v = torch.randn(70, heads, dim, generator=g).half(), torch.randn(70, heads, dim, generator=g).half()
    starts, lens = torch.tensor([0, 70], dtype=torch.int32).cuda(), torch.tensor([70], dtype=torch.int32).cuda()
    outs = []
    q = torch.randn(70, 8, dim, generator=g).half().cuda()
    for p in (0, pages - 1):
        b = comet.Batch(starts, lens, torch.tensor([[p]], dtype=torch.int32).cuda())
        cache.comet_cache_append(b, k.cuda(), v.cuda())
        outs.append((cache.comet_cache_attend(b, q), *cache.comet_cache_fetch(b, dtype=torch.float16, tokens=70)))
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    assert ((outs[0][2].cpu().float() - v.float()).abs() <= v.float().abs().max() / 250).all()


def test_serving_run(comet):
    """Prompts, then steps of one token, then drafted tokens of which some are taken back, then a piece of a prompt: the attention of every
    call against 64 bits over what the cache holds, and the whole run against attention over the tokens as they came."""
    rope = comet.Rope(64, scaling="parts", factor=4.0)
    s = Sequences(comet, torch.bfloat16, 2, 128, 4, 600, rope=rope, seed=31)
    back = [0, 0, 0, 0]
    for new in ([130, 1, 300, 0], [1, 1, 1, 40], [1, 1, 1, 1], [5, 4, 3, 2], [1, 1, 1, 1], [3, 64, 96, 1], [1, 1, 1, 1]):
        for b in range(4):
            s.lens[b] -= back[b]
            s.k[b], s.v[b] = s.k[b][:s.lens[b]], s.v[b][:s.lens[b]]
        back = [3, 0, 2, 1] if new == [5, 4, 3, 2] else [0] * 4
        q = s.tokens(sum(new), 8)
        before = list(s.lens)
        batch, turned = s.grow(new, q=q.cuda(), pad=0)
        out, lse = s.cache.comet_cache_attend(batch, turned, lse=True, status=s.status)
        check_attend(s, new, turned.cpu(), out, lse)
        at = 0
        for b, n in enumerate(new):
            if n:                                                         # against keys and values that were never compressed
                k = ref.rotated(s.k[b], torch.arange(s.lens[b]), 64, scaling="parts", factor=4.0).transpose(0, 1)
                qt = ref.rotated(q[at:at + n], torch.arange(before[b], s.lens[b]), 64, scaling="parts", factor=4.0)
                o, _, _, _ = ref.attention(qt, k, s.v[b].double().transpose(0, 1), 128 ** -0.5, True)
                off = float((out[at:at + n].cpu().double() - o).norm() / o.norm())
                # keys off by half a step in 127 of the largest of 4096 (about 8): scores by 8/127/sqrt(12) |q| / sqrt(128) ~ 0.02 |q_i|
                # ~ 0.02 to 0.03, values by 4/127/sqrt(12) ~ 0.01 of their size: a few per cent together
                assert off < 0.06, (new, b, off)
            at += n
    for b in range(4):
        y, tol = rope_bound(s.k[b].to(s.dt), torch.arange(s.lens[b]), 64, False, {"scaling": "parts", "factor": 4.0})
        check_held(s, b, (y, tol))
    assert s.ok()
