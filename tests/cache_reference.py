"""The compressed key/value cache from its definition, in 64 bits on the CPU: what a sequence holds after its tokens came, the
attention over it, and a reader of the cache's bytes.  Shares no code with the library."""
import math

import torch

BLOCK = 32


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_len=4096, beta_fast=32.0, beta_slow=1.0):
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2) if rot > 2 else 1.0)
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    amp = 1.0
    if scaling == "parts":
        amp = 0.1 * math.log(factor) + 1.0
        g = [min(1.0, max(0.0, (original_len * x / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow))) for x in f]
        f = [x * (k + (1.0 - k) / factor) for x, k in zip(f, g)]
    return f, amp


def rotated(x, positions, rot, interleaved=False, sign=1.0, **how):
    """x [tokens, heads, dim] in 64 bits, turned."""
    f, amp = frequencies(rot, **how)
    y = x.double().clone()
    angle = positions.double()[:, None] * torch.tensor(f, dtype=torch.float64)
    c, s = angle.cos()[:, None] * amp, angle.sin()[:, None] * amp * sign
    ia = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    a, b = y[..., ia].clone(), y[..., ib].clone()
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    return y


def place(t):
    u, w, h, i = t >> 4, (t >> 3) & 1, (t >> 2) & 1, t & 3
    return 16 * h + 8 * u + 4 * w + i


def held(cache, table, lens, slots, b):
    """(keys, values) [head, token, dim] of sequence b as the cache's bytes have them, in 64 bits; all arguments on the CPU."""
    shape, buf = cache.shape, cache.buf.cpu()
    per, dim, heads = shape.page_tokens // BLOCK, shape.dim, shape.heads
    n = shape.n_pages * heads * per
    blocks = buf[:n * 64 * dim].view(torch.int8).view(shape.n_pages, heads, per, 64 * dim)
    scales = buf[n * 64 * dim:n * 64 * dim + 8 * n].view(torch.float32).view(shape.n_pages, heads, per, 2)
    at = n * 64 * dim + -(-8 * n // 256) * 256
    ring = buf[at:at + shape.n_slots * heads * 2 * (128 * dim + 256)].view(shape.n_slots, heads, 2, 128 * dim + 256)
    places = [place(t) for t in range(BLOCK)]
    ks, vs = [], []
    for j in range(-(-int(lens[b]) // BLOCK)):
        if j < int(lens[b]) // BLOCK:
            page = int(table[b, j // per])
            rec, e = blocks[page, :, j % per].double(), scales[page, :, j % per].double()
            ke, ve = e[:, :1, None], e[:, 1:, None]
        else:
            half = ring[int(slots[b]), :, j % 2]
            rec, e = half[:, :128 * dim].contiguous().view(torch.float16).double(), half[:, 128 * dim:].contiguous().view(torch.float32).double()
            ke, ve = e[:, :32, None], e[:, 32:, None]
        k = rec[:, :32 * dim].reshape(heads, dim // 32, BLOCK, 32).permute(0, 2, 1, 3).reshape(heads, BLOCK, dim)
        v = rec[:, 32 * dim:].reshape(heads, dim, BLOCK)[:, :, places].transpose(1, 2)
        left = min(BLOCK, int(lens[b]) - BLOCK * j)
        ks.append((k * ke)[:, :left])
        vs.append((v * ve)[:, :left])
    if not ks:
        return torch.zeros(heads, 0, dim, dtype=torch.float64), torch.zeros(heads, 0, dim, dtype=torch.float64)
    return torch.cat(ks, 1), torch.cat(vs, 1)


def attention(q, k, v, scale, causal):
    """(out, lse, sum of p |v|, largest sum of |q k|) for q [token, query head, dim], k and v [head, token, dim] in 64 bits."""
    n, hq, dim = q.shape
    group, total = hq // k.shape[0], k.shape[1]
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    s = torch.einsum("nhd,htd->nht", q.double(), k) * scale
    size = torch.einsum("nhd,htd->nht", q.double().abs(), k.abs()) * scale
    if causal:
        s = s.masked_fill(torch.arange(total)[None, None] >= (total - n + torch.arange(n) + 1)[:, None, None], -math.inf)
    if not total:
        return torch.zeros_like(q, dtype=torch.float64), torch.full((n, hq), -math.inf, dtype=torch.float64), torch.zeros_like(q, dtype=torch.float64), 0.0
    lse = torch.logsumexp(s, -1)
    p = torch.where(s == -math.inf, 0.0, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None]))
    return torch.einsum("nht,htd->nhd", p, v), lse, torch.einsum("nht,htd->nhd", p, v.abs()), float(size.max())
