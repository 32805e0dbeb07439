"""Workloads of the compressed key/value cache: what a program that trains or serves a language model has it do.

Three kinds of cases, each one pass through the public entry points of ``paper_2111_09562_amd``:

rope     queries or keys rotated by their positions (``comet_rope``), with the gradient in training (``autograd.rotate``)
append   new keys and values rotated and compressed into a paged cache, the queries rotated on the way
         (``comet_cache_append``), and the new tokens read back as the cache holds them (``comet_cache_fetch``)
attend   attention of the new tokens' queries over the compressed cache (``comet_cache_attend``)

The cache is one buffer.  A block is 32 tokens of one head of one sequence; complete blocks are held in 8 bits with a
scale for the keys and one for the values, the last, incomplete one in 16 bits.  Sections of the buffer, in bytes, for
``pages`` pages of ``per`` blocks, ``heads`` heads, ``slots`` slots and heads of ``dim`` values:

  blocks  [pages][heads][per][64 * dim]: keys int8 [dim/32][token][32], values int8 [dim/32][32][place of the token]
  scales  [pages][heads][per][2] float32: of the keys, of the values
  ring    [slots][heads][2][128 * dim + 256]: the block in 16 bits, as above but in float16, then 32 scales for the keys'
          tokens and 32 for the values'; block j of a sequence is in the half j % 2
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 32
_DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}


def _rope(name, tokens, heads, dim, dtype, rot=0, interleaved=False, scaling="none", factor=1.0, far=4096, backward=False, fused=0):
    return dict(name=name, op="rope", tokens=tokens, heads=heads, dim=dim, dtype=dtype, rot=rot or dim, interleaved=interleaved,
                scaling=scaling, factor=factor, far=far, backward=backward, fused=fused)


def _append(name, seqs, new_lo, new_hi, held_lo, held_hi, heads, q_heads, dim, dtype, rot=0, interleaved=False, scaling="none",
            factor=1.0, page=64, mix=1):
    return dict(name=name, op="append", seqs=seqs, new_lo=new_lo, new_hi=new_hi, held_lo=held_lo, held_hi=held_hi, heads=heads,
                q_heads=q_heads, dim=dim, dtype=dtype, rot=rot or dim, interleaved=interleaved, scaling=scaling, factor=factor,
                page=page, mix=mix)


def _attend(name, seqs, new_lo, new_hi, held_lo, held_hi, heads, q_heads, dim, dtype, causal=True, page=64, mix=1):
    return dict(name=name, op="attend", seqs=seqs, new_lo=new_lo, new_hi=new_hi, held_lo=held_lo, held_hi=held_hi, heads=heads,
                q_heads=q_heads, dim=dim, dtype=dtype, causal=causal, page=page, mix=mix)


def listed():
    return [
        # The queries of sixteen sequences in one step of decoding.
        _rope("rope_step", 16, 32, 128, "bfloat16"),
        # A training step's queries, a slice of the fused projection, and their gradient.
        _rope("rope_training", 16384, 32, 128, "bfloat16", backward=True, fused=48),
        # A part of odd heads in single precision, pairs side by side, far positions of a model stretched to long contexts.
        _rope("rope_stretched", 4099, 20, 96, "float32", rot=64, interleaved=True, scaling="parts", factor=8.0, far=1 << 20, backward=True),
        # One token of each of 64 sequences, anywhere in their blocks.
        _append("append_step", 64, 1, 1, 1, 4096, 8, 32, 128, "bfloat16"),
        # Drafted tokens of 24 sequences, no shared heads, half of every head rotated.
        _append("append_drafts", 24, 1, 6, 1, 2000, 12, 12, 64, "float16", rot=32, interleaved=True, page=32, mix=2),
        # Whole prompts of different lengths, packed.
        _append("append_prompts", 9, 600, 8000, 0, 0, 8, 32, 128, "bfloat16", scaling="linear", factor=2.0, page=256, mix=3),
        # One sequence, one token: the latency of a step.
        _attend("attend_one", 1, 1, 1, 701, 701, 8, 32, 128, "bfloat16"),
        # One token of each of 64 sequences of very different lengths.
        _attend("attend_batch", 64, 1, 1, 400, 16384, 8, 32, 128, "bfloat16", mix=4),
        # Two long contexts.
        _attend("attend_long", 2, 1, 1, 100000, 131071, 8, 64, 128, "float16", page=256, mix=5),
        # Drafted tokens checked in one pass, heads of 64, none shared.
        _attend("attend_drafts", 48, 1, 8, 8, 4096, 12, 12, 64, "float16", page=32, mix=6),
        # Whole prompts of different lengths, causal.
        _attend("attend_prompts", 5, 500, 4096, 0, 0, 8, 32, 128, "bfloat16", mix=7),
        # A piece of a long prompt over what is held of it, one head of keys for all queries, wide heads.
        _attend("attend_piece", 1, 2048, 2048, 30720, 30720, 1, 16, 256, "float16", page=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend"])
    dim = rng.choice([32, 64, 64, 96, 128, 128, 128, 160, 192, 256])
    rot = rng.choice([dim, dim, dim // 2])
    interleaved = rng.random() < 0.4
    scaling, factor = rng.choice([("none", 1.0), ("none", 1.0), ("linear", 4.0), ("parts", 16.0), ("base", 8.0)])
    if op == "rope":
        dtype = rng.choice(["float32", "float16", "bfloat16", "bfloat16"])
        heads = _log_int(rng, 1, 64)
        tokens = max(1, int(_log_int(rng, 64, 60_000_000) / (heads * dim)))
        case = _rope("", tokens, heads, dim, dtype, rot, interleaved, scaling, factor, _log_int(rng, 16, 1 << 20), rng.random() < 0.5,
                     heads + rng.choice([0, 1, 16]) if rng.random() < 0.5 else 0)
    else:
        dtype = rng.choice(["float16", "bfloat16"])
        heads = rng.choice([1, 2, 4, 5, 8, 8, 12])
        group = rng.choice([1, 1, 2, 3, 4, 4, 6, 8, 16])
        page = 32 * rng.choice([1, 2, 2, 4, 5, 8])
        mix = rng.randrange(1, 1 << 20)
        kind = rng.choice(["step", "step", "drafts", "prompts"] + (["piece"] if op == "attend" else []))
        seqs = _log_int(rng, 1, 128)
        if kind in ("step", "drafts"):
            new_hi = 1 if kind == "step" else rng.randint(2, 12)
            room = int(1e8 / (heads * dim))                                # tokens held in all: 100 M values of keys
            held_hi = min(131072, max(12, room // seqs))
            held_hi = _log_int(rng, 12, held_hi)
            shape = (seqs, 1, new_hi, rng.choice([1, held_hi // 2 + 1]), held_hi)
        elif kind == "prompts":
            seqs = min(seqs, 16)
            most = int(min(4000, 4000 * math.sqrt(128 / (heads * group * seqs)), 8e6 / (heads * group * dim * math.sqrt(seqs))))
            hi = _log_int(rng, 2, max(3, most))
            shape = (seqs, rng.choice([1, hi]), hi, 0, 0)
        else:
            new = _log_int(rng, 13, max(14, int(8192 / (heads * group))))
            held = 32 * _log_int(rng, 1, max(2, int(2e6 / (heads * dim)) // 32))
            shape = (1, new, new, held, held)
        if op == "append":
            case = _append("", *shape, heads, heads * group, dim, dtype, rot, interleaved, scaling, factor, page, mix)
        else:
            case = _attend("", *shape, heads, heads * group, dim, dtype, rng.random() < 0.8, page, mix)
    del case["name"]
    return case


# ---- sizes ------------------------------------------------------------------------------------------------------


def _lengths(case):
    """(new tokens, held tokens behind them) of every sequence: of the case alone, so that work() knows them."""
    rng = random.Random(case["mix"])
    pick = lambda lo, hi: lo if lo == hi else min(hi, max(lo, _log_int(rng, max(lo, 1), hi)))  # noqa: E731
    got = []
    for b in range(case["seqs"]):
        n = pick(case["new_lo"], case["new_hi"])
        got.append((n, pick(case["held_lo"], case["held_hi"]) + n))
    return got


def work(case):
    size = _DTYPES[case["dtype"]].itemsize
    d = case["dim"]
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"]
        passes = 2 if case["backward"] else 1
        return {"bytes": passes * (2 * size * n * d + 4 * case["tokens"]), "flops": passes * 3 * n * case["rot"]}
    lens = _lengths(case)
    new = sum(n for n, _ in lens)
    held_bytes = 2 * (d + 4 / BLOCK)                                      # of one token and head, keys and values
    if case["op"] == "append":
        kv = new * case["heads"]
        q = new * case["q_heads"] * d * size
        # there: keys, values and queries read, the cache and the queries written; back: the cache read, keys and values written
        return {"bytes": 2 * (kv * 2 * d * size + kv * held_bytes) + 2 * q,
                "flops": kv * (3 * case["rot"] + 8 * d) + new * case["q_heads"] * 3 * case["rot"]}
    pairs = sum(sum(h - n + i + 1 for i in range(n)) if case["causal"] else n * h for n, h in lens)
    held = sum(h for _, h in lens)
    return {"bytes": held * case["heads"] * held_bytes + 2 * new * case["q_heads"] * d * size + 4 * new * case["q_heads"],
            "flops": 4 * d * case["q_heads"] * pairs}


# ---- inputs -----------------------------------------------------------------------------------------------------


def _frequencies(case):
    """Radians per position of every pair, and the factor on the rotated values.  "linear" divides the positions, "base"
    stretches the base, "parts" divides the frequencies whose waves are long against 4096 positions and keeps the short ones
    (arXiv 2309.00071)."""
    rot, base, f = case["rot"], 10000.0, case["factor"]
    if case["scaling"] == "base":
        base *= f ** (rot / (rot - 2)) if rot > 2 else f
    theta = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if case["scaling"] == "linear":
        theta = [t / f for t in theta]
    if case["scaling"] == "parts":
        turns = [4096 * t / (2 * math.pi) for t in theta]
        keep = [min(1.0, max(0.0, (r - 1.0) / 31.0)) for r in turns]
        theta = [t * (k + (1.0 - k) / f) for t, k in zip(theta, keep)]
        return theta, 0.1 * math.log(f) + 1.0
    return theta, 1.0


def _own_rope(case):
    from paper_2111_09562_amd import comet
    return comet.Rope(case["rot"], base=10000.0, interleaved=case["interleaved"], scaling=case["scaling"], factor=case["factor"],
                      original_len=4096)


def _k_natural(raw, dim):
    """[..., dim/32, token, 32] -> [..., token, dim]"""
    x = raw.unflatten(-1, (dim // 32, 32, 32)).transpose(-3, -2)
    return x.flatten(-2)


def _k_raw(x):
    return x.unflatten(-1, (x.shape[-1] // 32, 32)).transpose(-3, -2).flatten(-3)


def _v_natural(raw, dim):
    """[..., dim/32, 32, place] -> [..., token, dim]: token 16u + 8w + 4h + i is in place 16h + 8u + 4w + i."""
    x = raw.unflatten(-1, (dim, 2, 2, 2, 4))                               # d, h, u, w, i
    n = x.dim()
    return x.permute(*range(n - 5), n - 3, n - 2, n - 4, n - 1, n - 5).flatten(-5, -2)


def _v_raw(x):
    y = x.unflatten(-2, (2, 2, 2, 4))                                      # u, w, h, i, d
    n = y.dim()
    return y.permute(*range(n - 5), n - 1, n - 3, n - 5, n - 4, n - 2).flatten(-5)


def _sections(s):
    """Views of the cache's sections."""
    c, buf = s["case"], s["buf"]
    per, pages, heads, dim, slots = c["page"] // BLOCK, s["n_pages"], c["heads"], c["dim"], c["seqs"]
    a = pages * heads * per * 64 * dim
    b = a + -(-pages * heads * per * 8 // 256) * 256
    blocks = buf[:a].view(torch.int8).view(pages, heads, per, 64 * dim)
    scales = buf[a:a + pages * heads * per * 8].view(torch.float32).view(pages, heads, per, 2)
    ring = buf[b:].view(slots, heads, 2, 128 * dim + 256)
    return blocks, scales, ring


def prepare(case, seed):
    dt = _DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    d = case["dim"]

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    theta, amp = _frequencies(case) if "rot" in case else ([], 1.0)
    s = {"case": case, "theta": torch.tensor(theta, dtype=torch.float64, device="cuda"), "amp": amp}
    if case["op"] == "rope":
        t, h = case["tokens"], case["heads"]
        whole = normal(t, max(h, case["fused"]), d).to(dt)
        s["x"] = whole[:, :h]
        s["grad"] = normal(t, h, d).to(dt)
        # positions of packed sequences: runs that begin anywhere below the farthest position
        run = 1 + t // 4
        begin = torch.randint(0, max(1, case["far"]), (4 + 1,), device="cuda", generator=g)
        i = torch.arange(t, device="cuda")
        s["positions"] = ((begin[i // run] + i % run) % case["far"]).to(torch.int32)
        if own:
            s["rope"] = _own_rope(case)
        return s
    lens = _lengths(case)
    per = case["page"] // BLOCK
    need = [-(-total // case["page"]) for _, total in lens]
    n_pages = sum(need) + 3                                                # a few pages belong to nobody
    order = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32)
    table = table.cuda()
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    s.update(n_pages=n_pages, table=table, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
             lens=torch.tensor([x for _, x in lens], dtype=torch.int32, device="cuda"),
             slots=torch.randperm(len(lens), device="cuda", generator=g).to(torch.int32),
             most_new=max(n for n, _ in lens), most_held=max(x for _, x in lens),
             most_blocks=max((x - 1) // BLOCK - (x - n) // BLOCK + 1 for n, x in lens))
    heads, q_heads, slots, tokens = case["heads"], case["q_heads"], len(lens), starts[-1]
    # keys have a few channels that are larger than the others, values have not
    wide = 1.0 + 4.0 * (torch.rand(heads, 1, d, device="cuda", generator=g) < 0.04).float()
    a = n_pages * heads * per * 64 * d
    b = a + -(-n_pages * heads * per * 8 // 256) * 256
    s["buf"] = torch.zeros(b + slots * heads * 2 * (128 * d + 256), dtype=torch.uint8, device="cuda")
    blocks, scales, ring = _sections(s)
    for p in range(0, n_pages, 1 + (1 << 26) // (heads * case["page"] * d)):          # a part of the pages at a time
        some = slice(p, p + 1 + (1 << 26) // (heads * case["page"] * d))
        for j, (natural_to_raw, spread) in enumerate(((_k_raw, wide), (_v_raw, torch.ones_like(wide)))):
            x = normal(*blocks[some].shape[:3], BLOCK, d) * spread.unsqueeze(1)
            scale = x.abs().amax((-1, -2)) / 127
            scales[some][..., j] = scale
            blocks[some][..., 32 * d * j:32 * d * (j + 1)] = natural_to_raw((x / scale[..., None, None]).round_().to(torch.int8))
    for j, (natural_to_raw, spread) in enumerate(((_k_raw, wide), (_v_raw, torch.ones_like(wide)))):
        x = (normal(slots, heads, 2, BLOCK, d) * spread.unsqueeze(1)).to(dt).float()
        e = torch.exp2(torch.floor(torch.log2(x.abs().amax(-1).clamp_min(1e-30))) - 14)
        ring[..., 64 * d * j:64 * d * (j + 1)] = natural_to_raw((x / e[..., None]).half()).contiguous().view(torch.uint8)
        ring[..., 128 * d + 128 * j:128 * d + 128 * (j + 1)] = e.contiguous().view(torch.uint8)
    # queries, keys and values as a fused projection leaves them
    if case["op"] == "append":
        x = normal(tokens, q_heads + 2 * heads, d)
        x[:, q_heads:q_heads + heads] *= wide.squeeze(1)
        x = x.to(dt)
        s.update(q=x[:, :q_heads], k=x[:, q_heads:q_heads + heads], v=x[:, q_heads + heads:])
    else:
        s["q"] = normal(tokens, q_heads, d).to(dt)
    if own:
        from paper_2111_09562_amd import comet
        s["cache"] = comet.Cache(n_pages, case["page"], slots, heads, d, buf=s["buf"])
        s["batch"] = comet.Batch(s["starts"], s["lens"], s["table"], s["slots"])
        if case["op"] == "append":
            s["rope"] = _own_rope(case)
    return s


# ---- the operators ----------------------------------------------------------------------------------------------


def _rotate(x, positions, s, sign):
    """The plain rotation, in 32 bits with angles from 64."""
    c = s["case"]
    rot = c["rot"]
    angle = positions.double()[:, None] * s["theta"]
    cos, sin = (angle.cos() * s["amp"]).float()[:, None], (angle.sin() * (sign * s["amp"])).float()[:, None]
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((u, v), -1).flatten(-2) if c["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _ring_values(ring, dim):
    """Keys and values of the ring's blocks, [..., token, dim] in 32 bits."""
    e = ring[..., 128 * dim:].contiguous().view(torch.float32)
    k = _k_natural(ring[..., :64 * dim].contiguous().view(torch.float16), dim).float() * e[..., :32, None]
    v = _v_natural(ring[..., 64 * dim:128 * dim].contiguous().view(torch.float16), dim).float() * e[..., 32:, None]
    return k, v


def _append_plain(s):
    c = s["case"]
    dim, per, dt = c["dim"], c["page"] // BLOCK, s["k"].dtype
    blocks, scales, ring = _sections(s)
    starts, lens, slots = s["starts"].long(), s["lens"].long(), s["slots"].long()
    tokens = s["k"].shape[0]
    t = torch.arange(tokens, device="cuda")
    seq = torch.bucketize(t, starts[1:], right=True)
    before = lens - (starts[1:] - starts[:-1])
    positions = before[seq] + t - starts[seq]
    k, q = _rotate(s["k"], positions, s, 1.0), _rotate(s["q"], positions, s, 1.0)
    # every block that gets a token: [sequence, block, token], what the ring holds of it and what is new
    j = (before // BLOCK)[:, None] + torch.arange(s["most_blocks"], device="cuda")
    p = j[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")
    new = (p >= before[:, None, None]) & (p < lens[:, None, None])
    old = (p < before[:, None, None])[..., None, None]
    source = (starts[:-1, None, None] + p - before[:, None, None]).clamp(0, tokens - 1)
    held = [x.permute(0, 2, 3, 1, 4) for x in _ring_values(ring[slots], dim)]         # [sequence, half, token, head, dim]
    complete = j < (lens // BLOCK)[:, None]
    page = torch.gather(s["table"].long(), 1, (j // per).clamp_max(s["table"].shape[1] - 1))
    done = complete.nonzero(as_tuple=True)
    keep = ((j <= (lens // BLOCK)[:, None]) & (j >= (lens // BLOCK)[:, None] - 1)).nonzero(as_tuple=True)
    out = []
    for i, (x, to_raw) in enumerate(((k, _k_raw), (s["v"], _v_raw))):
        first = torch.gather(held[i], 1, (j[:, :1] % 2)[..., None, None, None].expand(-1, 1, *held[i].shape[2:]))
        y = torch.where(new[..., None, None], x.float()[source], 0.0)
        y = torch.where(old, first, y).transpose(2, 3)                    # [sequence, block, head, token, dim]
        scale = (y.abs().amax((-1, -2)) / 127).clamp_min(2.0 ** -100)
        whole = (y / scale[..., None, None]).round().clamp(-127, 127)
        at = (page[done][:, None], torch.arange(c["heads"], device="cuda"), (j % per)[done][:, None])
        scales[at + (torch.tensor(i, device="cuda"),)] = scale[done]
        blocks[..., 32 * dim * i:32 * dim * (i + 1)][at] = to_raw(whole[done].to(torch.int8))
        # the ring: the last complete block and the open one
        mine = new[keep][:, None, :, None]
        e = torch.exp2(torch.floor(torch.log2(y.abs().amax(-1).clamp_min(1e-38))) - 14)[keep]
        where = (slots[keep[0]][:, None], torch.arange(c["heads"], device="cuda"), (j % 2)[keep][:, None])
        was = ring[where]
        half = (y[keep] / e[..., None]).half()
        sel = lambda raw: raw.contiguous().view(torch.uint8)  # noqa: E731
        mask = sel(to_raw(mine.expand_as(half).half().view(torch.int16).ne(0).to(torch.int16).neg()))
        body, at_e = slice(64 * dim * i, 64 * dim * (i + 1)), slice(128 * dim + 128 * i, 128 * dim + 128 * (i + 1))
        ring[..., body][where] = torch.where(mask.ne(0), sel(to_raw(half)), was[..., body])
        ring[..., at_e][where] = torch.where(sel(mine.squeeze(-1).expand_as(e).int().neg()).ne(0), sel(e), was[..., at_e])
        values = torch.where(complete[:, :, None, None, None], whole * scale[..., None, None], y)
        back = values.transpose(2, 3)[seq, positions // BLOCK - (before // BLOCK)[seq], positions % BLOCK]
        out.append(back.to(dt))
    return {"q": q, "k": out[0], "v": out[1]}


def _attend_plain(s):
    c = s["case"]
    dim, per, heads, group = c["dim"], c["page"] // BLOCK, c["heads"], c["q_heads"] // c["heads"]
    blocks, scales, ring = _sections(s)
    starts, lens = s["starts"].long(), s["lens"].long()
    seqs, most, n = c["seqs"], s["most_new"], starts[1:] - starts[:-1]
    j = torch.arange(-(-s["most_held"] // BLOCK), device="cuda")
    page = s["table"].long()[:, j // per].clamp_min(0)                     # [sequence, block]
    at = (page[:, None], torch.arange(heads, device="cuda")[:, None], (j % per))
    raw, scale = blocks[at], scales[at]                                    # [sequence, head, block, ...]
    k = _k_natural(raw[..., :32 * dim], dim).float() * scale[..., 0, None, None]
    v = _v_natural(raw[..., 32 * dim:], dim).float() * scale[..., 1, None, None]
    open_at = (lens // BLOCK).clamp_max(len(j) - 1)
    is_open = (lens % BLOCK > 0) & (lens // BLOCK < len(j))
    tail = ring[s["slots"].long()[:, None], torch.arange(heads, device="cuda"), (lens // BLOCK % 2)[:, None]]
    b = torch.arange(seqs, device="cuda")
    for whole, last in zip((k, v), _ring_values(tail, dim)):
        whole[b, :, open_at] = torch.where(is_open[:, None, None, None], last, whole[b, :, open_at])
    k, v = k.flatten(2, 3), v.flatten(2, 3)                                # [sequence, head, token, dim]
    i = torch.arange(most, device="cuda")
    token = (starts[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"].float()[token].unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [sequence, head, query and group, dim]
    limit = (lens - n)[:, None] + i + 1 if c["causal"] else lens[:, None].expand(-1, most)
    seen = torch.arange(k.shape[2], device="cuda") < limit.repeat_interleave(group, 1)[:, None, :, None]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * dim ** -0.5
    score = score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-3e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / total
    lse = (top + total.log()).squeeze(-1)
    here = (i < n[:, None]).nonzero(as_tuple=True)
    rows = lambda x: x.unflatten(2, (most, group)).permute(0, 2, 1, 3, *range(4, x.dim() + 1))[here].flatten(1, 2)  # noqa: E731
    return {"out": rows(o).to(s["q"].dtype), "lse": rows(lse)}


def run(state):
    s, op = state, state["case"]["op"]
    if op == "rope":
        if own:
            from paper_2111_09562_amd import autograd, comet
            if not s["case"]["backward"]:
                return {"y": comet.comet_rope(s["x"], s["rope"], s["positions"])}
            x = s["x"].detach().requires_grad_()
            y = autograd.rotate(x, s["rope"], s["positions"])
            (dx,) = torch.autograd.grad(y, x, s["grad"])
            return {"y": y.detach(), "dx": dx}
        y = {"y": _rotate(s["x"], s["positions"], s, 1.0)}
        if s["case"]["backward"]:
            y["dx"] = _rotate(s["grad"], s["positions"], s, -1.0)
        return y
    if op == "append":
        if own:
            q = s["cache"].comet_cache_append(s["batch"], s["k"], s["v"], rope=s["rope"], q=s["q"])
            k, v = s["cache"].comet_cache_fetch(s["batch"], dtype=s["k"].dtype, tokens=s["k"].shape[0])
            return {"q": q, "k": k, "v": v}
        return _append_plain(s)
    if own:
        out, lse = s["cache"].comet_cache_attend(s["batch"], s["q"], causal=s["case"]["causal"], lse=True)
        return {"out": out, "lse": lse}
    return _attend_plain(s)


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------------


def _turn(x, positions, case, sign):
    """Every pair as a complex number times amp * exp(i * sign * position * theta)."""
    theta, amp = _frequencies(case)
    w = torch.polar(torch.full((len(positions), len(theta)), amp, dtype=torch.float64, device=x.device),
                    sign * torch.outer(positions.double(), torch.tensor(theta, dtype=torch.float64, device=x.device)))
    y = x.double().clone()
    rot = case["rot"]
    first = slice(0, rot, 2) if case["interleaved"] else slice(0, rot // 2)
    second = slice(1, rot, 2) if case["interleaved"] else slice(rot // 2, rot)
    z = torch.complex(y[..., first], y[..., second]) * w[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _places():
    """Token -> its place among the 32 of a row of the values."""
    return [16 * ((t >> 2) & 1) + 8 * (t >> 4) + 4 * ((t >> 3) & 1) + (t & 3) for t in range(BLOCK)]


def _spread(flat, dim, places):
    """Keys and values [..., 32, dim] of a block's elements in the order of the cache."""
    k = torch.cat([flat[..., 1024 * c:1024 * (c + 1)].reshape(*flat.shape[:-1], 32, 32) for c in range(dim // 32)], -1)
    v = flat[..., 32 * dim:].reshape(*flat.shape[:-1], dim, 32)[..., places].transpose(-1, -2)
    return k, v


def _open_block(s, b, j):
    """The block j of sequence b in the ring, [head, token, dim] in 64 bits."""
    dim = s["case"]["dim"]
    rec = _sections(s)[2][int(s["slots"][b]), :, j % 2]
    e = rec[:, 128 * dim:].contiguous().view(torch.float32).double()
    k, v = _spread(rec[:, :128 * dim].contiguous().view(torch.float16).double(), dim, _places())
    return k * e[:, :32, None], v * e[:, 32:, None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        y = {"y": _turn(s["x"], s["positions"], case, 1.0)}
        if case["backward"]:
            y["dx"] = _turn(s["grad"], s["positions"], case, -1.0)
        return y
    dim, lens, begin = case["dim"], _lengths(case), 0
    if case["op"] == "append":
        q, k, v = torch.empty_like(s["q"], dtype=torch.float64), torch.empty_like(s["k"], dtype=torch.float64), torch.empty_like(s["v"], dtype=torch.float64)
        for b, (n, total) in enumerate(lens):
            rows = slice(begin, begin + n)
            at = torch.arange(total - n, total, device="cuda")
            q[rows] = _turn(s["q"][rows], at, case, 1.0)
            # the cache holds keys and values of the 16-bit type: what it compresses is the rotated key in that type
            new = [_turn(s["k"][rows], at, case, 1.0).to(s["k"].dtype).double(), s["v"][rows].double()]
            lead = (total - n) % BLOCK
            if lead:
                old = _open_block(s, b, (total - n) // BLOCK)
                new = [torch.cat((o[:, :lead].transpose(0, 1), x)) for o, x in zip(old, new)]
            full = len(new[0]) // BLOCK * BLOCK
            for x, to in zip(new, (k, v)):
                y = x.clone()
                w = x[:full].unflatten(0, (-1, BLOCK))
                if full:
                    step = w.abs().amax((1, 3), keepdim=True) / 127
                    y[:full] = (torch.round(w / step.clamp_min(2.0 ** -100)) * step).flatten(0, 1)
                to[rows] = y[lead:]
            begin += n
        return {"q": q, "k": k, "v": v}
    blocks, scales, _ = _sections(s)
    per, group = case["page"] // BLOCK, case["q_heads"] // case["heads"]
    out = torch.empty_like(s["q"], dtype=torch.float64)
    lse = torch.empty(out.shape[:2], dtype=torch.float64, device="cuda")
    for b, (n, total) in enumerate(lens):
        ids = s["table"][b].long()
        which = torch.arange(total // BLOCK, device="cuda")
        for h in range(case["heads"]):
            flat = blocks[ids[which // per], h, which % per].double()
            k, v = _spread(flat, dim, _places())
            step = scales[ids[which // per], h, which % per].double()
            k, v = (k * step[:, 0, None, None]).flatten(0, 1), (v * step[:, 1, None, None]).flatten(0, 1)
            if total % BLOCK:
                ko, vo = _open_block(s, b, total // BLOCK)
                k, v = torch.cat((k, ko[h, :total % BLOCK])), torch.cat((v, vo[h, :total % BLOCK]))
            for part in range(0, n, 512):
                rows = slice(part, min(n, part + 512))
                q = s["q"][begin:begin + n][rows, h * group:(h + 1) * group].double()
                score = (q.flatten(0, 1) @ k.T.contiguous()).unflatten(0, (-1, group)) / math.sqrt(dim)
                if case["causal"]:
                    last = torch.arange(total - n, total, device="cuda")[rows]
                    score = score.masked_fill(torch.arange(total, device="cuda") > last[:, None, None], -math.inf)
                lse[begin:begin + n][rows, h * group:(h + 1) * group] = torch.logsumexp(score, -1)
                p = torch.softmax(score, -1).flatten(0, 1)
                out[begin:begin + n][rows, h * group:(h + 1) * group] = (p @ v).unflatten(0, (-1, group))
        begin += n
    return {"out": out, "lse": lse}
