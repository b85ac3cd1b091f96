"""Cases for timing the operators of a paged 8-bit K/V cache on one GPU: rotary positions, appending tokens, attention over the
cache, and the upkeep of its pages (reserving, forking, freeing, compacting, copying).

``run`` computes an operator in its plain form, elementary torch operations in 32 bits, or, where ``own`` is true, calls the
framework as a user's program does.

The cache.  Tokens stand in pages of ``page`` tokens; a sequence lives in a slot, whose row of the page table names its pages in
order (-1: none).  A page holds, per K/V head, blocks of 64 tokens in 8 bits with one scale each for K and V: the value is code * scale,
``int8`` codes are stored with 128 added (scale = max|x| / 127), ``e4m3`` codes as they are (scale = max|x| / 448).  The bytes of a block
stand in the order in which a wavefront's lanes take the operands of their matrix instructions:

  K  byte ((t * d/64 + c) * 64 + 16 g + r) * 16 + e         is token 16 t + r, channel 64 c + 16 g + e
  V  byte (c * 64 + 16 g + r) * 16 + 8 u + 4 h + i          is token 32 u + 16 h + 4 g + i, channel 16 c + r

Tokens behind the last of a sequence are zeros in its last block.  Beside the pages each slot keeps the last tokens in 16 bits (token p
at p % 128 of its tail), so that a block that grows is quantised from the tokens themselves: its codes do not depend on how many calls
filled it.
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
RANGE = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100  # a block whose largest value is below is held as zeros
BLOCK, TAIL = 64, 128


# ---- cases --------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # rotary positions of Q and K, views of a packed projection: one token of each of 64 conversations, launch-bound
        _rope("rope_step", 64, 32, 8, 128, 128, "half", "none", 1.0, 4000, "bf16"),
        # the prompts of a batch, positions far beyond the trained length, half of each head rotated: streams
        _rope("rope_prompt", 16384, 32, 8, 128, 64, "interleaved", "yarn", 16.0, 131072, "bf16"),
        # the gradient of a training step with an odd number of tokens
        _rope("rope_grad", 4099, 24, 24, 64, 64, "half", "bands", 8.0, 65536, "fp16", transposed=True),
        # one token of each of 64 conversations into the cache, K rotated and shifted on the way
        _append("append_step", 64, 8, 128, 1, 200, 1, 1, "int8", "bf16", page=128, rot=128, shift=True),
        # ragged prompts into an empty cache
        _append("append_prompts", 10, 8, 128, 0, 0, 300, 2500, "e4m3", "fp16", page=256, rot=64),
        # one token of two short conversations: launch-bound
        _attn("attn_short", 2, 32, 8, 128, 700, 1500, 1, False, "int8", "bf16", page=64),
        # one token of a batch of conversations of all lengths: streams the cache
        _attn("attn_batch", 48, 32, 8, 128, 1000, 8192, 1, False, "int8", "bf16", page=128),
        # five drafted tokens of a few long conversations, eight query heads to a K/V head
        _attn("attn_draft", 4, 32, 4, 64, 20000, 32768, 5, False, "e4m3", "fp16", page=256),
        # chunks of prompts and single tokens of conversations in one ragged batch: matrix products
        _attn("attn_chunks", 6, 32, 8, 128, 2000, 16384, 512, True, "int8", "bf16", page=128),
        # 16 prompts, four continuations each
        _pages("pages_fork", "fork", 16, 8, 128, 300, 2000, page=128, more=4),
        # a pool after many conversations have come and gone
        _pages("pages_compact", "compact", 96, 8, 128, 300, 6000, page=128, more=0),
        # the table between two steps: eight conversations of 256 end, the others get a few tokens each
        _pages("pages_turn", "turn", 256, 8, 128, 100, 8000, page=64, more=8),
    ]


def _rope(name, tokens, Hq, Hkv, d, rot, layout, scaling, factor, far, dtype, transposed=False):
    return _named(name, op="rope", tokens=tokens, Hq=Hq, Hkv=Hkv, d=d, rot=rot, layout=layout, scaling=scaling, factor=factor, far=far,
                  dtype=dtype, transposed=transposed)


def _append(name, B, Hkv, d, old_lo, old_hi, new_lo, new_hi, fmt, dtype, page, rot, shift=False):
    return _named(name, op="append", B=B, Hkv=Hkv, d=d, old_lo=old_lo, old_hi=old_hi, new_lo=new_lo, new_hi=new_hi, fmt=fmt, dtype=dtype,
                  page=page, rot=rot, shift=shift)


def _attn(name, B, Hq, Hkv, d, lo, hi, new, ragged, fmt, dtype, page, causal=True):
    return _named(name, op="attn", B=B, Hq=Hq, Hkv=Hkv, d=d, lo=lo, hi=hi, new=new, ragged=ragged, fmt=fmt, dtype=dtype, page=page,
                  causal=causal)


def _pages(name, what, B, Hkv, d, lo, hi, page, more):
    return _named(name, op="pages", what=what, B=B, Hkv=Hkv, d=d, lo=lo, hi=hi, page=page, more=more)


def _named(name, **c):
    return dict(c, name=name) if name else c


def _log(rng, lo, hi):
    """Whole number, spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["rope", "append", "append", "attn", "attn", "attn", "pages"])
    d, dtype, fmt = rng.choice([64, 128]), rng.choice(["fp16", "bf16"]), rng.choice(["int8", "e4m3"])
    Hkv, group, page = _log(rng, 1, 16), rng.choice([1, 2, 3, 4, 6, 8, 16]), 64 * rng.choice([1, 1, 2, 3, 4, 8])
    while True:
        if op == "rope":
            scaling = rng.choice(["none", "linear", "ntk", "yarn", "bands"])
            c = _rope(None, _log(rng, 1, 16384), Hkv * group, Hkv, d, rng.choice([d, d, d // 2, d // 4, d - 16]),
                      rng.choice(["half", "interleaved"]), scaling, 1.0 if scaling == "none" else rng.uniform(1.5, 32.0),
                      _log(rng, 100, 1000000), dtype, rng.random() < 0.3)
            if c["tokens"] * (Hkv + Hkv * group) * d <= 16384 * 40 * 128:
                return c
        elif op == "append":
            # a step of conversations (a few tokens each), or whole prompts
            step = rng.random() < 0.6
            lo, hi = (1, _log(rng, 1, 8)) if step else (_log(rng, 1, 300), _log(rng, 301, 4000))
            c = _append(None, _log(rng, 1, 128 if step else 16), Hkv, d, 0, _log(rng, 1, 500) if step else 0, lo, hi, fmt, dtype, page,
                        rng.choice([0, d, d // 2]), rng.random() < 0.5)
            if sum(_lens(c)) * Hkv * d <= 14000 * 8 * 128:
                return c
        elif op == "attn":
            lo = _log(rng, 1, 4000)
            c = _attn(None, _log(rng, 1, 64), Hkv * group, Hkv, d, lo, _log(rng, lo, 32768), rng.choice([1, 1, 1, _log(rng, 2, 16), _log(rng, 17, 512)]),
                      rng.random() < 0.5, fmt, dtype, page, rng.random() < 0.8)
            w = work(c)
            if w["flops"] <= 1.5e11 and w["bytes"] <= 4e8 and c["B"] * Hkv * group * c["new"] * c["hi"] <= 3e9 and c["B"] * Hkv * c["hi"] * d <= 1e9:
                return c
        else:
            lo, B = _log(rng, 1, 3000), _log(rng, 1, 96)
            what = rng.choice(["fork", "compact", "turn"])
            c = _pages(None, what, B, Hkv, d, lo, _log(rng, lo, 8000), page, {"fork": rng.randint(1, 4), "compact": 0, "turn": rng.randint(1, max(1, B // 4))}[what])
            if B * (lo + c["hi"]) * Hkv * d <= 600000 * 8 * 128:
                return c


def _spread(lo, hi, n, phase=0.0):
    """n whole numbers of [lo, hi], evenly spread and out of order, the first of them hi: a case's own, whatever the seed."""
    return [hi if b == 0 else min(hi, lo + int((hi - lo + 1) * ((b * 0.6180339887498949 + phase) % 1.0))) for b in range(n)]


def _lens(c):
    """Tokens per sequence, with the new ones."""
    if c["op"] == "append":
        return [a + b for a, b in zip(_spread(c["old_lo"], c["old_hi"], c["B"]), _news(c))]
    return _spread(c["lo"], c["hi"], c["B"])


def _news(c):
    """New tokens per sequence."""
    if c["op"] == "append":
        return _spread(c["new_lo"], c["new_hi"], c["B"], 0.37)
    if not c["ragged"]:
        return [min(c["new"], c["lo"])] * c["B"]
    # half of the sequences bring one token, the others up to `new`
    return [min(n, 1 if b % 2 else m) for b, (n, m) in enumerate(zip(_lens(c), _spread(1, c["new"], c["B"], 0.37)))]


def work(case):
    c = case
    if c["op"] == "rope":
        return dict(bytes=4 * c["tokens"] * (c["Hq"] + c["Hkv"]) * c["d"], flops=3 * c["tokens"] * (c["Hq"] + c["Hkv"]) * c["rot"])
    H, d = c["Hkv"], c["d"]
    lens = _lens(c)
    if c["op"] == "append":
        news = _news(c)
        first = [(n - m) % BLOCK for n, m in zip(lens, news)]   # tokens of a block begun before, read again in 16 bits
        blocks = [-(-n // BLOCK) - (n - m) // BLOCK for n, m in zip(lens, news)]
        kept = [min(m, n - max(0, (n - 1) // BLOCK - 1) * BLOCK) for n, m in zip(lens, news)]
        there = sum(-(-n // BLOCK) for n in lens)               # the whole cache is read back
        nbytes = 2 * H * (2 * d * (sum(news) + sum(first)) + BLOCK * d * sum(blocks) + 2 * d * sum(kept) + BLOCK * d * there + 2 * d * sum(lens))
        return dict(bytes=nbytes, flops=4 * H * d * sum(blocks) * BLOCK)
    if c["op"] == "attn":
        news = _news(c)
        T = sum(news)
        pairs = sum(m * n - (m * (m - 1) // 2 if c["causal"] else 0) for n, m in zip(lens, news))
        return dict(bytes=4 * T * c["Hq"] * d + 2 * H * d * sum(-(-n // BLOCK) * BLOCK for n in lens), flops=4 * c["Hq"] * d * pairs)
    page, B = c["page"], c["B"]
    one = 2 * H * page * d
    if c["what"] == "fork":
        return dict(bytes=B * c["more"] * (2 * one + 2 * 2 * 2 * H * TAIL * d), flops=0)
    if c["what"] == "compact":
        n_pages, live, moved = _fragments(c)
        return dict(bytes=2 * moved * one + 8 * n_pages, flops=0)
    return dict(bytes=4 * (sum(-(-n // page) for n in lens[:c["more"]]) * 2 + 4 * B + _pool(c)), flops=0)


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _pool(c):
    """Pages of the pool: those of the sequences, those of their continuations, and as many more as a program keeps in hand."""
    used = sum(-(-n // c["page"]) for n in _lens(c))
    if c["op"] != "pages":
        return used + 3
    return used + (c["B"] * c["more"] if c["what"] == "fork" else c["B"]) + 5


def _fragments(c):
    """(pages of the pool, live ones, live ones that stand behind as many) of a compaction: every third sequence has gone, the order of the
    pages is that in which _order gives them out."""
    n_pages, at, live = _pool(c), 0, set()
    order = _order(n_pages)
    for b, n in enumerate(_lens(c)):
        k = -(-n // c["page"])
        if b % 3:
            live.update(order[at:at + k])
        at += k
    return n_pages, len(live), sum(p >= len(live) for p in live)


def _order(n):
    """The pages of a pool in the order in which sequences got them: neighbours in a sequence are none in memory."""
    step = next(s for s in range(int(n * 0.6180339887498949) | 1, 4 * n + 3) if math.gcd(s, n) == 1)
    return [(i * step + n // 3) % n for i in range(n)]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return _ints(at)


def _table(c, slots, spare=0):
    """The page table and the lengths of _lens(c) in `slots` slots (sequence b in slot b), and the pages' reference counts."""
    lens, page, n_pages = _lens(c), c["page"], _pool(c)
    wide = max(-(-n // page) for n in lens) + spare
    order, at, table, refs = _order(n_pages), 0, [], [0] * n_pages
    for n in lens:
        k = -(-n // page)
        table.append(order[at:at + k] + [-1] * (wide - k))
        for p in order[at:at + k]:
            refs[p] = 1
        at += k
    table += [[-1] * wide] * (slots - len(lens))
    return _ints(table), _ints(lens + [0] * (slots - len(lens))), _ints(refs)


def _empty_pool(c, n_pages, slots, dtype):
    H, d, per = c["Hkv"], c["d"], c["page"] // BLOCK
    zero = 128 if c["fmt"] == "int8" else 0
    s = {}
    for x in "kv":
        s[x] = torch.full((n_pages, H, per, BLOCK * d), zero, dtype=torch.uint8, device="cuda")
        s[x + "_scale"] = torch.zeros((n_pages, H, per), device="cuda")
        s[x + "_tail"] = torch.zeros((slots, H, TAIL, d), dtype=dtype, device="cuda")
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case=c)
    d, H = c["d"], c["Hkv"]
    if c["op"] == "rope":
        dt = DTYPES[c["dtype"]]
        # Q and K are the first heads of a packed projection [T, Hq + 2 Hkv, d]; a gradient comes as two tensors of its own
        T, Hq = c["tokens"], c["Hq"]
        qkv = normal(T, Hq + (0 if c["transposed"] else 2) * H, d).to(dt)
        s["q"], s["k"] = (qkv, normal(T, H, d).to(dt)) if c["transposed"] else (qkv[:, :Hq], qkv[:, Hq:Hq + H])
        s["positions"] = torch.randint(0, c["far"], (T,), generator=g, device="cuda", dtype=torch.int32)
        return s
    if c["op"] == "attn":
        dt, lens, news = DTYPES[c["dtype"]], _lens(c), _news(c)
        s["table"], s["lens"], s["refs"] = _table(c, c["B"])
        s.update(_empty_pool(c, _pool(c), c["B"], dt))
        for x in "kv":  # a page's blocks as the cache holds them: the codes of normal values, in any order, and their scales
            _fill(s[x], s[x + "_scale"], normal, c["fmt"])
        # the last block's rows behind the last token are zeros
        _clear_ends(s, c)
        s["q"] = normal(sum(news), c["Hq"], d).to(dt)
        s["q_start"] = _starts(news) if c["ragged"] else None
        return s
    if c["op"] == "append":
        dt, lens, news, B = DTYPES[c["dtype"]], _lens(c), _news(c), c["B"]
        s["table"], s["lens"], s["refs"] = _table(c, B)
        s.update(_empty_pool(c, _pool(c), B, dt))
        s["shift"] = 3.0 * normal(H, d) if c["shift"] else None
        old = [n - m for n, m in zip(lens, news)]
        if max(old):
            wide = -(-max(old) // BLOCK) * BLOCK
            at, n_old = torch.arange(wide, device="cuda"), _ints(old)
            for x in "kv":
                y = normal(B, wide, H, d)
                if x == "k" and c["shift"]:
                    y += s["shift"]
                y = y.to(dt)
                codes, scales = _quantise(_blocks(y.float(), n_old, s["shift"] if x == "k" else None), c["fmt"])
                codes = _block_k(codes) if x == "k" else _block_v(codes)
                b, j = torch.nonzero(at[::BLOCK][None] < n_old[:, None], as_tuple=True)
                p = s["table"][b, j * BLOCK // c["page"]].long()
                s[x][p, :, j % (c["page"] // BLOCK)] = codes[b, j]
                s[x + "_scale"][p, :, j % (c["page"] // BLOCK)] = scales[b, j]
                b, i = torch.nonzero((at[None] < n_old[:, None]) & (at[None] >= n_old[:, None] - TAIL), as_tuple=True)
                s[x + "_tail"][b, :, i % TAIL] = y[b, i]
        s["new_k"], s["new_v"] = normal(sum(news), H, d), normal(sum(news), H, d).to(dt)
        if c["shift"]:
            s["new_k"] += s["shift"]
        s["new_k"] = s["new_k"].to(dt)
        s["q_start"] = None if min(news) == max(news) else _starts(news)
        s["k_start"], s["total"] = _starts(lens), sum(lens)
        return s
    # pages: e4m3 codes of a pool in use
    B, what = c["B"], c["what"]
    slots = B * (1 + c["more"]) if what == "fork" else B
    table, lens, refs = _table(c, slots, spare=1)
    if what == "compact":
        gone = torch.arange(slots, device="cuda") % 3 == 0
        table[gone], lens[gone] = -1, 0
        refs = torch.bincount(table[table >= 0].long(), minlength=refs.numel()).to(torch.int32)
    s.update(table0=table, lens0=lens, refs0=refs, table=table.clone(), lens=lens.clone(), refs=refs.clone())
    if what == "turn":
        s["gone"] = _ints(list(range(c["more"])))
        s["stay"] = _ints(list(range(c["more"], B)))
        s["stay"] = s["stay"][torch.randperm(s["stay"].numel(), generator=g, device="cuda")]
        s["n_new"] = torch.randint(1, 9, s["stay"].shape, generator=g, device="cuda", dtype=torch.int32)
        return s
    s.update(_empty_pool(dict(c, fmt="e4m3"), refs.numel(), slots, torch.bfloat16))
    for x in "kv":
        _fill(s[x], s[x + "_scale"], normal, "e4m3")
        s[x + "_tail"].copy_(normal(*s[x + "_tail"].shape))
    if what == "fork":
        s["src"] = _ints([b for b in range(B) for _ in range(c["more"])])
        s["dst"] = _ints(list(range(B, slots)))
    else:
        s["most"] = refs.numel() // 2
    return s


def _fill(pool, scales, normal, fmt):
    """Blocks of normal values in 8 bits with the scales that their largest values give, piece by piece."""
    flat, sc = pool.view(-1, pool.shape[-1]), scales.view(-1)
    for i in range(0, flat.shape[0], 8192):
        codes, a = _quantise(normal(*flat[i:i + 8192].shape)[:, None], fmt)
        flat[i:i + 8192], sc[i:i + 8192] = codes[:, 0], a


def _clear_ends(s, c):
    zero, per = 128 if c["fmt"] == "int8" else 0, c["page"] // BLOCK
    lens = s["lens"].long()
    b = torch.arange(c["B"], device="cuda")
    j = (lens - 1) // BLOCK
    p, j = s["table"][b, j // per].long(), j % per
    behind = torch.arange(BLOCK, device="cuda")[None] >= ((lens - 1) % BLOCK + 1)[:, None]
    for x, unblock, block in (("k", _unblock_k, _block_k), ("v", _unblock_v, _block_v)):
        y = unblock(s[x][p, :, j])
        y[behind[:, None, :, None].expand_as(y)] = zero
        s[x][p, :, j] = block(y)


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _block_k(x):
    """[..., 64, d] by token and channel -> [..., 64 d] in the order of the cache."""
    d, lead = x.shape[-1], x.shape[:-2]
    n = len(lead)
    return x.reshape(*lead, 4, 16, d // 64, 4, 16).permute(*range(n), n, n + 2, n + 3, n + 1, n + 4).reshape(*lead, BLOCK * d)


def _unblock_k(x):
    d, lead = x.shape[-1] // BLOCK, x.shape[:-1]
    n = len(lead)
    return x.reshape(*lead, 4, d // 64, 4, 16, 16).permute(*range(n), n, n + 3, n + 1, n + 2, n + 4).reshape(*lead, BLOCK, d)


def _block_v(x):
    d, lead = x.shape[-1], x.shape[:-2]
    n = len(lead)
    return x.reshape(*lead, 2, 2, 4, 4, d // 16, 16).permute(*range(n), n + 4, n + 2, n + 5, n, n + 1, n + 3).reshape(*lead, BLOCK * d)


def _unblock_v(x):
    d, lead = x.shape[-1] // BLOCK, x.shape[:-1]
    n = len(lead)
    return x.reshape(*lead, d // 16, 4, 16, 2, 2, 4).permute(*range(n), n + 3, n + 4, n + 1, n + 5, n, n + 2).reshape(*lead, BLOCK, d)


def _quantise(x, fmt):
    """[..., 64, d] -> (codes, scales [...])"""
    a = x.abs().amax((-2, -1))
    some = a >= TINY
    y = x * torch.where(some, RANGE[fmt] / a, torch.zeros_like(a))[..., None, None]
    codes = (y.round() + 128).to(torch.uint8) if fmt == "int8" else y.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, torch.where(some, a / RANGE[fmt], torch.zeros_like(a))


def _values(codes, fmt):
    return codes.float() - 128 if fmt == "int8" else codes.view(torch.float8_e4m3fn).float()


def _blocks(x, lens, shift):
    """[B, L, H, d] -> [B, L / 64, H, 64, d], minus the shift, zeros behind the last token."""
    B, L, H, d = x.shape
    if shift is not None:
        x = x - shift
    x = torch.where((torch.arange(L, device=x.device)[None] < lens[:, None])[:, :, None, None], x, torch.zeros((), device=x.device))
    return x.view(B, L // BLOCK, BLOCK, H, d).transpose(2, 3)


def _freqs(c, like=torch.float64):
    """Radians per position of each pair of channels, and the factor on the result."""
    rot, base, s, trained = c["rot"], 10000.0, c["factor"], 8192.0
    i = torch.arange(0, rot, 2, dtype=like, device="cuda")
    if c["scaling"] == "ntk":
        return (base * s ** (rot / (rot - 2.0))) ** (-i / rot), 1.0
    f = base ** (-i / rot)
    if c["scaling"] == "linear":
        return f / s, 1.0
    if c["scaling"] == "yarn":
        # pairs that turn more than 32 times over the trained length stay, those below one turn are stretched
        low, high = (rot * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (32.0, 1.0))
        low, high = max(math.floor(low), 0), min(math.ceil(high), rot - 1)
        ramp = ((i / 2 - low) / max(high - low, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / s * ramp, 0.1 * math.log(s) + 1.0
    if c["scaling"] == "bands":
        # the same by wavelength: below a quarter of the trained length, above it, between
        keep = ((trained * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f * keep + f / s * (1 - keep), 1.0
    return f, 1.0


def _rotate(x, positions, f, factor, layout, transposed=False):
    """x [T, H, d] in 32 bits, the angles in 64: far positions need them."""
    rot = 2 * f.numel()
    angle = positions.double()[:, None] * f * (-1.0 if transposed else 1.0)
    cos, sin = (angle.cos() * factor).float()[:, None], (angle.sin() * factor).float()[:, None]
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


APPEND_ROPE = dict(scaling="none", factor=1.0)  # plain rotation, by halves


def _plain_rope(s):
    c = s["case"]
    f, factor = _freqs(c)
    return tuple(_rotate(s[x].float(), s["positions"], f, factor, c["layout"], c["transposed"]).to(s[x].dtype) for x in "qk")


def _plain_read(s, c, lens, fmt):
    """K and V of every sequence in 32 bits, [B, L, H, d] with L whole blocks, as the table names their pages."""
    per = c["page"] // BLOCK
    j = torch.arange(-(-max(lens) // BLOCK), device="cuda")
    p = s["table"][:len(lens)][:, j // per].long().clamp(min=0)
    out = []
    for x, unblock in (("k", _unblock_k), ("v", _unblock_v)):
        y = _values(unblock(s[x][p, :, (j % per)[None].expand_as(p)]), fmt) * s[x + "_scale"][p, :, (j % per)[None].expand_as(p)][..., None, None]
        out.append(y.transpose(2, 3).reshape(len(lens), j.numel() * BLOCK, c["Hkv"], c["d"]))
    return out


def _plain_append(s):
    c = s["case"]
    B, dt, page, per = c["B"], s["new_k"].dtype, c["page"], c["page"] // BLOCK
    lens, news = _lens(c), _news(c)
    end = s["lens"].long()
    q_start = s["q_start"].long() if s["q_start"] is not None else torch.arange(B + 1, device="cuda") * news[0]
    start = end - (q_start[1:] - q_start[:-1])
    wide = max(-(-n // BLOCK) - (n - m) // BLOCK for n, m in zip(lens, news)) * BLOCK
    at = (start // BLOCK * BLOCK)[:, None] + torch.arange(wide, device="cuda")          # positions that the touched blocks hold
    new = (at >= start[:, None]) & (at < end[:, None])
    row = torch.where(new, q_start[:-1, None] + at - start[:, None], torch.zeros_like(at))
    seq = torch.arange(B, device="cuda")
    for x in "kv":
        fresh = s["new_" + x]
        if x == "k" and c["rot"]:
            position = torch.zeros(fresh.shape[0], dtype=torch.int64, device="cuda")
            position[row[new]] = at[new]
            fresh = _rotate(fresh.float(), position, *_freqs(dict(c, **APPEND_ROPE)), "half").to(dt)
        tail = s[x + "_tail"]
        held = tail[seq[:, None], :, at % TAIL]
        y = torch.where(new[:, :, None, None], fresh[row], held)
        b, i = torch.nonzero(new & (at >= ((end - 1) // BLOCK * BLOCK - BLOCK)[:, None]), as_tuple=True)
        tail[b, :, at[b, i] % TAIL] = y[b, i]
        codes, scales = _quantise(_blocks(y.float(), end - start // BLOCK * BLOCK, s["shift"] if x == "k" else None), c["fmt"])
        codes = _block_k(codes) if x == "k" else _block_v(codes)
        b, i = torch.nonzero(at[:, ::BLOCK] < end[:, None], as_tuple=True)
        j = at[b, i * BLOCK] // BLOCK
        p = s["table"][b, j // per].long()
        s[x][p, :, j % per], s[x + "_scale"][p, :, j % per] = codes[b, i], scales[b, i]
    k, v = _plain_read(s, c, lens, c["fmt"])
    k = k + s["shift"] if s["shift"] is not None else k
    token = torch.arange(s["total"], device="cuda")
    b = torch.searchsorted(s["k_start"][1:].long(), token, right=True)
    i = token - s["k_start"].long()[b]
    return k[b, i].to(dt), v[b, i].to(dt), s["k_tail"], s["v_tail"]


def _plain_attn(s):
    c, q = s["case"], s["q"]
    B, Hq, H, d, T = c["B"], c["Hq"], c["Hkv"], c["d"], s["q"].shape[0]
    group, news = Hq // H, _news(c)
    n = max(news)
    k, v = _plain_read(s, c, _lens(c), c["fmt"])
    L = k.shape[1]
    q_start = s["q_start"].long() if s["q_start"] is not None else torch.arange(B + 1, device="cuda") * n
    count, lens = q_start[1:] - q_start[:-1], s["lens"].long()
    i = torch.arange(n, device="cuda")
    rows = q[(q_start[:-1, None] + i).clamp(max=T - 1)].float()                                   # [B, n, Hq, d]
    rows = rows.view(B, n, H, group, d).permute(0, 2, 3, 1, 4).reshape(B, H, group * n, d)
    scores = torch.matmul(rows, k.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(d)).view(B, H, group, n, L)
    last = lens[:, None] - 1 + (i[None] - count[:, None] + 1 if c["causal"] else torch.zeros_like(i)[None])
    seen = torch.arange(L, device="cuda")[None, None] <= last[:, :, None]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    l = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, H, group * n, L), v.transpose(1, 2)).view(B, H, group, n, d) / torch.where(l > 0, l, torch.ones_like(l))
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, d)
    token = torch.arange(T, device="cuda")
    b = torch.searchsorted(q_start[1:].contiguous(), token, right=True)
    return out[b, token - q_start[b]].to(q.dtype)


def _plain_reserve(s, slots, n_new):
    """n_new more tokens for each of `slots`: the lowest free pages, in the order of the list."""
    page, slots = s["case"]["page"], slots.long()
    old, new = s["lens"][slots].long(), s["lens"][slots].long() + n_new
    have, need = (old + page - 1) // page, (new + page - 1) // page - (old + page - 1) // page
    upto = need.cumsum(0)
    free = torch.sort((s["refs"] != 0).to(torch.int8), stable=True).indices
    ok = (need == 0) | ((upto <= (s["refs"] == 0).sum()) & (have + need <= s["table"].shape[1]))
    b, w = torch.nonzero((torch.arange(s["table"].shape[1], device="cuda")[None] < need[:, None]) & ok[:, None], as_tuple=True)
    pages = free[upto[b] - need[b] + w]
    s["table"][slots[b], have[b] + w] = pages.to(torch.int32)
    s["refs"][pages] = 1
    s["lens"][slots] = torch.where(ok, new, old).to(torch.int32)
    return torch.where(ok, 0, -1).to(torch.int32)


def _plain_pages(s):
    c = s["case"]
    table, lens, refs, page = s["table"], s["lens"], s["refs"], c["page"]
    if c["what"] == "turn":
        gone = s["gone"].long()
        held = table[gone]
        refs -= torch.bincount(held[held >= 0].long(), minlength=refs.numel()).to(torch.int32)
        table[gone], lens[gone] = -1, 0
        return _plain_reserve(s, s["stay"], s["n_new"])
    if c["what"] == "fork":
        src, dst = s["src"].long(), s["dst"].long()
        n = lens[src].long()
        full, part = n // page, n % page != 0
        upto = part.cumsum(0)
        free = torch.sort((refs != 0).to(torch.int8), stable=True).indices
        at = torch.arange(table.shape[1], device="cuda")[None]
        rows = torch.where(at < full[:, None], table[src], torch.full_like(table[src], -1))
        shared = rows[rows >= 0].long()
        refs += torch.bincount(shared, minlength=refs.numel()).to(torch.int32)
        b = torch.nonzero(part)[:, 0]
        to = free[upto[b] - 1]
        rows[b, full[b]] = to.to(torch.int32)
        refs[to] = 1
        table[dst], lens[dst] = rows, lens[src]
        moved = table[src[b], full[b]].long()
        for x in ("k", "v", "k_scale", "v_scale"):
            s[x][to] = s[x][moved]
        for x in ("k_tail", "v_tail"):
            s[x][dst] = s[x][src]
        return torch.zeros_like(s["src"])
    live = refs > 0
    used = live.sum()
    at = torch.arange(refs.numel(), device="cuda")
    src, dst = at[live & (at >= used)], at[~live & (at < used)]
    src, dst = src[:s["most"]], dst[:s["most"]]
    to = at.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].to(torch.int32), table))
    refs[dst] = refs[src]
    refs[src] = 0
    for x in ("k", "v", "k_scale", "v_scale"):
        s[x][dst] = s[x][src]
    return torch.stack([used, used * 0 + src.numel()]).to(torch.int32)


def run(state):
    s, c = state, state["case"]
    if c["op"] == "rope":
        return _own_rope(s) if own else _plain_rope(s)
    if c["op"] == "append":
        return _own_append(s) if own else _plain_append(s)
    if c["op"] == "attn":
        return _own_attn(s) if own else _plain_attn(s)
    # a program's table goes from state to state; here every pass begins at the same one
    s["table"].copy_(s["table0"])
    s["lens"].copy_(s["lens0"])
    s["refs"].copy_(s["refs0"])
    said = _own_pages(s) if own else _plain_pages(s)
    out = dict(said=said, table=s["table"], lens=s["lens"], refs=s["refs"])
    if c["what"] != "turn":
        out.update(k=s["k"].view(torch.float8_e4m3fn), v=s["v"].view(torch.float8_e4m3fn),
                   **{x: s[x] for x in ("k_scale", "v_scale", "k_tail", "v_tail")})
    return out


# ---- the framework's calls ----------------------------------------------------------------------------------------------

def _kept(s, what, make):
    """A handle that a program makes once and keeps."""
    if what not in s:
        import paper_2505_21136_amd as sage
        s["sage"] = sage
        s[what] = make(sage)
    return s["sage"], s[what]


def _plan(c):
    return lambda sage: sage.rope_plan(c["rot"], base=10000.0, layout=c.get("layout", "half"), scaling=c["scaling"], factor=c["factor"],
                                       trained_len=8192)


def _own_rope(s):
    sage, plan = _kept(s, "plan", _plan(s["case"]))
    return sage.sage_rope(s["q"], s["positions"], plan, k=s["k"], transposed=s["case"]["transposed"])


def _handles(s):
    c = s["case"]

    def make(sage):
        pages = sage.PageTable(table=s["table"], lens=s["lens"], refs=s["refs"], page_tokens=c["page"])
        if "k" not in s:
            return pages, None
        return pages, sage.PagedCache(pages, k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"], k_tail=s["k_tail"],
                                      v_tail=s["v_tail"], fmt=c.get("fmt", "e4m3"), k_shift=s.get("shift"))

    return _kept(s, "handles", make)


def _own_append(s):
    c = s["case"]
    sage, (_, cache) = _handles(s)
    plan = _kept(s, "plan", _plan(dict(c, **APPEND_ROPE)))[1] if c["rot"] else None
    sage.sage_paged_append(cache, s["new_k"], s["new_v"], q_start=s["q_start"], rope=plan)
    k, v = sage.sage_paged_gather(cache, s["k_start"], s["total"])
    return k, v, s["k_tail"], s["v_tail"]


def _own_attn(s):
    c = s["case"]
    sage, (_, cache) = _handles(s)
    if "workspace" not in s:
        s["workspace"] = torch.empty(sage.paged_workspace_bytes(s["q"].shape[0], c["B"], c["Hq"], c["Hkv"], c["d"], c["hi"]), dtype=torch.uint8,
                                     device="cuda")
    return sage.sage_attn_fwd_paged(s["q"], cache, causal=c["causal"], max_len=c["hi"], q_start=s["q_start"], workspace=s["workspace"])


def _own_pages(s):
    c = s["case"]
    sage, (pages, cache) = _handles(s)
    if c["what"] == "turn":
        sage.sage_pages_free(pages, s["gone"])
        return sage.sage_pages_reserve(pages, s["n_new"], slots=s["stay"])
    if c["what"] == "fork":
        status, moves, slot_moves = sage.sage_pages_fork(pages, s["src"], s["dst"])
        sage.sage_pages_copy(cache, moves, slot_moves)
        return status
    moves, counts = sage.sage_pages_compact(pages, s["most"])
    sage.sage_pages_copy(cache, moves)
    return counts


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None  # whole numbers and copies
    s = prepare(c, seed)
    return {"rope": _exact_rope, "append": _exact_append, "attn": _exact_attn}[c["op"]](c, s)


def _exact_turn(x, positions, f, factor, layout, sign):
    """Each pair of channels as a complex number times factor e^(i angle)."""
    rot, x = 2 * f.numel(), x.double()
    turn = torch.polar(torch.full((positions.numel(), f.numel()), factor, dtype=torch.float64, device="cuda"), sign * positions.double()[:, None] * f)
    pair = (torch.arange(f.numel(), device="cuda"), torch.arange(f.numel(), device="cuda") + f.numel()) if layout == "half" else \
        (torch.arange(0, rot, 2, device="cuda"), torch.arange(1, rot, 2, device="cuda"))
    z = torch.complex(x[..., pair[0]], x[..., pair[1]]) * turn[:, None]
    y = x.clone()
    y[..., pair[0]], y[..., pair[1]] = z.real, z.imag
    return y


def _exact_rope(c, s):
    f, factor = _freqs(c)
    return tuple(_exact_turn(s[x], s["positions"], f, factor, c["layout"], -1.0 if c["transposed"] else 1.0) for x in "qk")


def _byte(c, which, r, ch):
    """Where token r (of 64), channel ch of a block stands."""
    if which == "k":
        return ((r // 16 * (c["d"] // 64) + ch // 64) * 64 + ch % 64 // 16 * 16 + r % 16) * 16 + ch % 16
    return (ch // 16 * 64 + r % 16 // 4 * 16 + ch % 16) * 16 + r // 32 * 8 + r % 32 // 16 * 4 + r % 4


def _exact_tokens(c, s, which, b, n):
    """The first n tokens of sequence b, [H, n, d], byte by byte."""
    at = torch.arange(n, device="cuda")
    p = s["table"][b].long()[at // c["page"]]
    j = at % c["page"] // BLOCK
    pool, scale = s[which], s[which + "_scale"]
    H = pool.shape[1]
    first = ((p * H)[None] + torch.arange(H, device="cuda")[:, None]) * pool.shape[2] + j[None]                        # [H, n] blocks
    offset = first[..., None] * pool.shape[3] + _byte(c, which, at % BLOCK, torch.arange(c["d"], device="cuda")[:, None]).T[None]
    code = pool.view(-1)[offset]
    value = code.double() - 128 if c["fmt"] == "int8" else code.view(torch.float8_e4m3fn).double()
    return value * scale.view(-1)[first].double()[..., None]


def _exact_attn(c, s):
    lens, news, group, d = _lens(c), _news(c), c["Hq"] // c["Hkv"], c["d"]
    out, at = [], 0
    for b, (n, m) in enumerate(zip(lens, news)):
        k, v = (_exact_tokens(c, s, x, b, n) for x in "kv")
        q = s["q"][at:at + m].double().view(m, c["Hkv"], group, d).permute(1, 2, 0, 3).reshape(c["Hkv"], group * m, d)
        x = (q @ k.transpose(1, 2) / math.sqrt(d)).view(c["Hkv"], group, m, n)
        if c["causal"]:
            x = x + torch.full((m, n), -math.inf, dtype=torch.float64, device="cuda").triu(n - m + 1)
        y = torch.softmax(x, -1).view(c["Hkv"], group * m, n) @ v
        out.append(y.view(c["Hkv"], group, m, d).permute(2, 0, 1, 3).reshape(m, c["Hq"], d))
        at += m
    return torch.cat(out)


def _exact_append(c, s):
    """Block by block over all tokens of a sequence: what the 16-bit tokens give, however they came."""
    lens, news, dt = _lens(c), _news(c), s["new_k"].dtype
    # (tokens that stood in whole blocks before are there in 8 bits alone: their blocks stay)
    got, tails, at = {"k": [], "v": []}, {}, 0
    for x in "kv":
        tails[x] = s[x + "_tail"].double()
    for b, (n, m) in enumerate(zip(lens, news)):
        old, begun = n - m, (n - m) // BLOCK * BLOCK
        for x in "kv":
            new = s["new_" + x][at:at + m]
            if x == "k" and c["rot"]:
                new = _exact_turn(new, torch.arange(old, n, device="cuda"), _freqs(dict(c, **APPEND_ROPE))[0], 1.0, "half", 1.0)
            p = torch.arange(old, n, device="cuda")
            late = p >= (n - 1) // BLOCK * BLOCK - BLOCK
            held = s[x + "_tail"][b][:, torch.arange(begun, old, device="cuda") % TAIL].transpose(0, 1).double()
            tails[x][b, :, p[late] % TAIL] = new.double()[late].transpose(0, 1)
            y = torch.cat([held, new.to(dt).double()])
            shift = s["shift"].double() if x == "k" and s["shift"] is not None else 0.0
            y = torch.nn.functional.pad((y - shift).float().double(), (0, 0, 0, 0, 0, -len(y) % BLOCK)).view(-1, BLOCK, c["Hkv"], c["d"])
            a = y.abs().amax((1, 3), keepdim=True)
            step = a / RANGE[c["fmt"]]
            # (a code is defined by two binary32 operations, the factor range / a and its product with a value, as the
            # framework's other quantisers define theirs: values that fall between two codes go by them)
            factor = torch.where(a >= TINY, (RANGE[c["fmt"]] / a).float().double(), torch.zeros_like(a))
            z = (y * factor).float()
            z = z.round().double() if c["fmt"] == "int8" else z.to(torch.float8_e4m3fn).double()
            z = (z * step).flatten(0, 1)[:n - begun] + shift
            whole = _exact_tokens(c, s, x, b, begun).transpose(0, 1) + shift
            got[x].append(torch.cat([whole, z]))
        at += m
    return torch.cat(got["k"]), torch.cat(got["v"]), tails["k"], tails["v"]
