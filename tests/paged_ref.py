"""The paged 8-bit cache in plain steps on the CPU: where a token's bytes stand, the quantiser's binary32 steps, attention in 64 bits with a bound
on what the kernel's roundings can move, and the page table's upkeep as loops.  Written from include/sage.h alone."""
import math

import numpy as np
import torch

import paper_2505_21136_amd as sage

BLOCK, TAIL = 64, 128
EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def byte_of(which, r, ch, d):
    """Byte of token r (of 64), channel ch in a block of K or V."""
    if which == "k":
        return ((r // 16 * (d // 64) + ch // 64) * 64 + 16 * (ch % 64 // 16) + r % 16) * 16 + ch % 16
    return (ch // 16 * 64 + 16 * (r % 16 // 4) + ch % 16) * 16 + 8 * (r // 32) + 4 * (r % 32 // 16) + r % 4


def byte_table(which, d):
    return torch.tensor([[byte_of(which, r, c, d) for c in range(d)] for r in range(BLOCK)])


def code_values(codes, fmt):
    """uint8 codes -> what they stand for without the scale, float64."""
    return codes.double() - 128 if fmt == "int8" else codes.view(torch.float8_e4m3fn).double()


def sequence(cache, which, slot, n):
    """The first n tokens of a slot as the cache holds them, float64 [n, Hkv, d] (CPU copies of everything)."""
    pt = cache.pages
    table, per = pt.table.cpu(), pt.page_tokens // BLOCK
    pool, scale = (getattr(cache, which).cpu(), getattr(cache, which + "_scale").cpu())
    where, out = byte_table(which, cache.d), torch.empty((n, cache.Hkv, cache.d), dtype=torch.float64)
    for j in range(-(-n // BLOCK)):
        p = int(table[slot, j // per])
        for h in range(cache.Hkv):
            block = code_values(pool[p, h, j % per], cache.fmt)[where] * scale[p, h, j % per].double()
            m = min(BLOCK, n - j * BLOCK)
            out[j * BLOCK:j * BLOCK + m, h] = block[:m]
    return out


def quantise(x, fmt):
    """One block and head, x float32 [<= 64, d]: (codes uint8 [64, d] with the values' zero behind the last token, scale) by the header's binary32 steps."""
    x = np.asarray(x, dtype=np.float32)
    R = np.float32(127.0 if fmt == "int8" else 448.0)
    y = np.zeros((BLOCK, x.shape[1]), dtype=np.float32)
    if not np.isfinite(x).all():
        scale = np.float32("nan")
    else:
        a = np.float32(np.abs(x).max())
        scale = np.float32(0)
        if a >= 2.0 ** -100:
            scale = a / R
            y[:len(x)] = x * (R / a)
    t = torch.from_numpy(y)
    codes = (t.round() + 128).to(torch.uint8) if fmt == "int8" else t.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scale


def make_cache(lens, *, Hkv, d, dtype, fmt, page_tokens, seed, slots=None, spare=3, garbage=True, device="cuda"):
    """A cache with random contents for the given lengths (sequence b in slot b), its pages in random order; what no call may read -- pages
    that nobody has, blocks behind a sequence's last -- holds NaN codes and NaN scales where the format has them."""
    g = torch.Generator().manual_seed(seed)
    slots = slots or len(lens)
    per = page_tokens // BLOCK
    need = [-(-n // page_tokens) for n in lens]
    n_pages, width = sum(need) + spare, max(need + [1]) + 1
    order = torch.randperm(n_pages, generator=g).tolist()
    table, refs = torch.full((slots, width), -1, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32)
    shape = (n_pages, Hkv, per)
    pool, scale = {}, {}
    for x in "kv":
        pool[x] = torch.full(shape + (BLOCK * d,), 127 if fmt == "e4m3" else 255, dtype=torch.uint8)
        scale[x] = torch.full(shape, float("nan") if garbage else 0.0)
    where = {x: byte_table(x, d).flatten() for x in "kv"}
    zero = 128 if fmt == "int8" else 0
    for b, n in enumerate(lens):
        table[b, :need[b]] = torch.tensor(order[:need[b]], dtype=torch.int32)
        refs[order[:need[b]]] = 1
        for j in range(-(-n // BLOCK)):
            p, m = int(table[b, j // per]), min(BLOCK, n - j * BLOCK)
            for h in range(Hkv):
                for x in "kv":
                    v = torch.randn(m, d, generator=g) * torch.rand(1, generator=g).mul(3).exp()
                    codes, s = quantise(v.numpy(), fmt)
                    codes[m:] = zero
                    pool[x][p, h, j % per][where[x]] = codes.flatten()
                    scale[x][p, h, j % per] = float(s)
        order = order[need[b]:]
    pages = sage.PageTable(table=table.to(device), lens=torch.tensor(list(lens) + [0] * (slots - len(lens)), dtype=torch.int32, device=device),
                           refs=refs.to(device), page_tokens=page_tokens)
    tail = lambda: torch.full((slots, Hkv, TAIL, d), float("nan"), dtype=dtype, device=device)  # noqa: E731
    return sage.PagedCache(pages, k=pool["k"].to(device), v=pool["v"].to(device), k_scale=scale["k"].to(device), v_scale=scale["v"].to(device),
                           k_tail=tail(), v_tail=tail(), fmt=fmt)


def attention(q, k, v, *, causal, sm_scale=None):
    """q [n, Hq, d], k, v float64 [N, Hkv, d] -> (out, bound on |kernel - out| before the last rounding), float64.

    The bound: a score is a binary32 sum of d products and two more roundings, e = (d + 8) 2^-24 sum|q k| off at most (in log units), the weight's
    exponential adds 2^-20, its rounding to binary16 2^-11 and, below 2^-14, at most 2^-25 of the largest V step instead; numerator and denominator both carry the
    first two.  With A = sum p|v| / l: A (2 (e + 2^-20) + 2^-11 + (N/64 + 8) 2^-23) + N 2^-25 max|v| 448."""
    n, Hq, d = q.shape
    N, Hkv = k.shape[0], k.shape[1]
    q = q.double()
    sm = sm_scale or 1.0 / math.sqrt(d)
    out, err = torch.zeros(n, Hq, d, dtype=torch.float64), torch.zeros(n, Hq, d, dtype=torch.float64)
    if N == 0:
        return out, err
    for h in range(Hq):
        kk, vv = k[:, h * Hkv // Hq], v[:, h * Hkv // Hq]
        s = q[:, h] @ kk.T * sm
        big = (q[:, h].abs() @ kk.abs().T * sm)
        if causal:
            hidden = torch.arange(N)[None] > torch.arange(n)[:, None] + N - n
            s = s.masked_fill(hidden, -math.inf)
            big = big.masked_fill(hidden, 0.0)
        m = s.amax(-1, keepdim=True)
        p = torch.where(m > -math.inf, (s - m).exp(), torch.zeros_like(s))
        l = p.sum(-1, keepdim=True)
        p = torch.where(l > 0, p / l, p)
        out[:, h] = p @ vv
        e = (d + 8) * 2.0 ** -24 * big.amax(-1, keepdim=True)
        err[:, h] = (p @ vv.abs()) * (2 * (e + 2.0 ** -20) + 2.0 ** -11 + (N / 64 + 8) * 2.0 ** -23) + N * 2.0 ** -25 * vv.abs().max()
    return out, err


def assert_attention(got, want, err, dtype, what):
    got = got.double().cpu()
    tol = err + EPS[dtype] * (want.abs() + err) + 2.0 ** -24
    assert torch.isfinite(got).all(), what
    worst = ((got - want).abs() / tol).max().item() if got.numel() else 0.0
    print(f"   {what}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


class Table:
    """The page table's upkeep as loops over lists."""

    def __init__(self, pages):
        self.table, self.lens, self.refs = pages.table.cpu().tolist(), pages.lens.cpu().tolist(), pages.refs.cpu().tolist()
        self.page, self.width = pages.page_tokens, pages.width

    def same(self, pages):
        assert pages.lens.cpu().tolist() == self.lens
        assert pages.table.cpu().tolist() == self.table
        assert pages.refs.cpu().tolist() == self.refs

    def count(self):
        """refs as the table says them."""
        n = [0] * len(self.refs)
        for row in self.table:
            for p in row:
                if p >= 0:
                    n[p] += 1
        return n

    def reserve(self, slots, n_new):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        total, seen, status, at = len(free), set(), [], 0
        for s, m in zip(slots, n_new):
            if not 0 <= s < len(self.lens) or s in seen or m < 0 or self.lens[s] + m > self.width * self.page:
                status.append(-1)
                seen.add(s)
                continue
            seen.add(s)
            has = -(-self.lens[s] // self.page)
            while has < self.width and self.table[s][has] >= 0:
                has += 1
            need = max(0, -(-(self.lens[s] + m) // self.page) - has)
            at += need
            if need and at > total:
                status.append(-1)
                continue
            for w in range(need):
                p = free[at - need + w]
                self.table[s][has + w], self.refs[p] = p, 1
            self.lens[s] += m
            status.append(0)
        return status

    def fork(self, src, dst):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        total, seen, status, pm, sm, at = len(free), set(), [], [], [], 0
        rows, lens = [r[:] for r in self.table], self.lens[:]
        for s, t in zip(src, dst):
            ok = 0 <= t < len(lens) and t not in seen and 0 <= s < len(lens) and s not in dst and lens[t] == 0 and rows[t][0] < 0
            seen.add(t)
            need = int(ok and lens[s] % self.page != 0)
            at += need
            if not ok or (need and at > total):
                status.append(-1), pm.append([-1, -1]), sm.append([-1, -1])
                continue
            full = lens[s] // self.page
            self.table[t] = rows[s][:full] + [-1] * (self.width - full)
            for p in rows[s][:full]:
                self.refs[p] += 1
            if need:
                p = free[at - 1]
                self.table[t][full], self.refs[p] = p, 1
                pm.append([rows[s][full], p])
            else:
                pm.append([-1, -1])
            self.lens[t] = lens[s]
            status.append(0), sm.append([s, t])
        return status, pm, sm

    def free(self, slots):
        for s in slots:
            if 0 <= s < len(self.lens):
                for p in self.table[s]:
                    if p >= 0:
                        self.refs[p] -= 1
                self.table[s], self.lens[s] = [-1] * self.width, 0

    def compact(self, most):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        M = len(live)
        moves = list(zip([p for p in live if p >= M], [p for p in range(M) if self.refs[p] == 0]))[:most]
        to = dict(moves)
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return [list(m) for m in moves] + [[-1, -1]] * (most - len(moves)), [M, len(moves)]
