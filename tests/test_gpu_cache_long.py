"""Attention of long prompts over the compressed cache, against 64 bits in a sample of its rows: every kernel that takes two tiles of rows per
wavefront, and pieces of more than the 64 blocks whose places are looked up at once.  Tolerances as in test_gpu_cache."""
import math

import pytest

torch = pytest.importorskip("torch")
import cache_reference as ref  # noqa: E402
from test_gpu_cache import DT, U32, Sequences, comet, u  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def check_sample(s, new, q, out, lse, causal, count=12):
    """First and last rows of every sequence, those around the ends of tiles and blocks, and some anywhere."""
    at = 0
    for b, n in enumerate(new):
        k, v = s.held(b)
        total = s.lens[b]
        rows = {0, 1, 31, 32, 33, 63, 64, 127, 128, 255, 256, n // 2, n - 33, n - 2, n - 1} | set(torch.randint(0, n, (count,), generator=s.g).tolist())
        for i in sorted(r for r in rows if 0 <= r < n):
            seen = total - n + i + 1 if causal else total
            o, want, size, top = ref.attention(q[at + i:at + i + 1], k[:, :seen], v[:, :seen], s.dim ** -0.5, False)
            d = (s.dim + 8) * U32 * top
            tol = (u(torch.float16) + 2 * d + 2.0 ** -19) * size + u(s.dt) * o.abs() + 2.0 ** -24
            assert ((out[at + i].cpu().double() - o[0]).abs() <= tol[0]).all(), (b, i)
            assert ((lse[at + i].cpu().double() - want[0]).abs() <= d + 2.0 ** -20 * (1 + want[0].abs())).all(), (b, i)
        at += n


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,group,dim,held,new,causal", [
    (2, 2, 128, [0], [4097], True), (1, 3, 128, [777], [4100], True), (2, 1, 128, [33, 4000], [4099, 4200], False), (1, 2, 96, [0], [4500], True),
    (3, 1, 96, [1000], [4111], True), (1, 1, 96, [64], [4096], False), (16, 2, 128, [1000], [4129], True), (16, 1, 96, [3000], [4101], True),
    (12, 3, 64, [2500], [1500], True), (16, 4, 32, [2000], [1030], False), (16, 4, 128, [5000], [300], True), (12, 2, 256, [4000], [513], True)])
def test_long_prompts(comet, dtype, heads, group, dim, held, new, causal):  # noqa: F811
    s = Sequences(comet, DT[dtype], heads, dim, len(new), max(a + b for a, b in zip(held, new)), page=128, seed=dim + heads)
    s.grow(held)
    s.grow(new)
    q = s.tokens(sum(new) + 1, heads * group) * 2
    batch, qd = s.batch(new), q.cuda()
    out = torch.full_like(q, 5.0, device="cuda")
    out, lse = s.cache.comet_cache_attend(batch, qd, out=out, lse=True, causal=causal, status=s.status)
    check_sample(s, new, q, out, lse, causal)
    assert (out[sum(new):] == 5).all() and s.ok()
    for _ in range(4):                       # bit for bit, whatever else the GPU has just done
        out2, lse2 = s.cache.comet_cache_attend(batch, qd, lse=True, causal=causal)
        assert torch.equal(out2[:sum(new)], out[:sum(new)]) and torch.equal(lse2[:sum(new)], lse[:sum(new)])
        torch.randn(512, 512, device="cuda").sum()


def test_open_block_that_no_row_sees(comet):  # noqa: F811
    """Causal queries in front of the end of what is held leave the last blocks unseen; a set of rows that sees nothing at all is 0."""
    s = Sequences(comet, torch.bfloat16, 2, 96, 1, 4400, page=128, seed=5)
    s.grow([4200])
    q = s.tokens(4150, 2)
    lens = [4096]                                     # 54 rows in front of the first token
    out, lse = s.cache.comet_cache_attend(s.batch([4150], lens=lens), q.cuda(), lse=True)
    assert not out[:54].any() and (lse[:54] == -math.inf).all() and out[54:].isfinite().all()
    k, v = ref.held(s.cache, s.table, lens, s.slots, 0)
    for i in (54, 55, 86, 2000, 4149):
        o, _, size, top = ref.attention(q[i:i + 1], k[:, :i - 53], v[:, :i - 53], 96 ** -0.5, False)
        d = 104 * U32 * top
        assert ((out[i].cpu().double() - o[0]).abs() <= ((u(torch.float16) + 2 * d + 2.0 ** -19) * size + u(s.dt) * o.abs() + 2.0 ** -24)[0]).all()
