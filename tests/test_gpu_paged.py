"""The paged cache: codes and scales of appended tokens bit for bit, whatever calls brought them; reading back; the page table's upkeep
against loops; attention within the bound that its roundings allow; and a serving loop of all of them."""
import pytest
import torch

import paper_2505_21136_amd as sage
from paged_ref import (BLOCK, TAIL, Table, assert_attention, attention, byte_table, code_values, make_cache, quantise,
                       sequence)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def empty(slots, Hkv, d, dtype, fmt, page, width, n_pages=None, shift=None):
    pages = sage.PageTable.empty(n_pages or slots * width, page_tokens=page, slots=slots, width=width, device=DEV)
    cache = sage.PagedCache.empty(pages, Hkv, d, dtype, fmt=fmt, k_shift=shift)
    for t in (cache.k, cache.v):
        t.fill_(0x7f)                              # NaN codes, where the format has them
    for t in (cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail):
        t.fill_(float("nan"))
    return pages, cache


def check_blocks(cache, slot, tokens, shift=None, shortened=False):
    """Every block of a slot, bit for bit: tokens = {'k': [n, Hkv, d], 'v': ...} in 16 bits on the CPU, K as rotated; and the tail, which holds the
    last two blocks (of a sequence that has been longer: the one that goes on)."""
    pt = cache.pages
    table, per, n = pt.table.cpu(), pt.page_tokens // BLOCK, tokens["k"].shape[0]
    for x in "kv":
        pool, scale, where = getattr(cache, x).cpu(), getattr(cache, x + "_scale").cpu(), byte_table(x, cache.d)
        for j in range(-(-n // BLOCK)):
            p = int(table[slot, j // per])
            for h in range(cache.Hkv):
                y = tokens[x][j * BLOCK:(j + 1) * BLOCK, h].float()
                if x == "k" and shift is not None:
                    y = y - shift[h].cpu()
                codes, s = quantise(y.numpy(), cache.fmt)
                got = scale[p, h, j % per]
                assert got.view(torch.int32) == torch.tensor(s).view(torch.int32) or (got.isnan() and s != s), (x, j, h)
                a, b = code_values(pool[p, h, j % per][where], cache.fmt), code_values(codes, cache.fmt)
                assert torch.equal(a, b), (x, j, h, (a != b).sum())
        tail = getattr(cache, x + "_tail").cpu()[slot]
        for i in range(n // BLOCK * BLOCK if shortened else max(0, ((n - 1) // BLOCK - 1) * BLOCK), n):
            assert torch.equal(tail[:, i % TAIL].view(torch.int16), tokens[x][i].view(torch.int16)), (x, i)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,page,rot,layout,shifted", [(64, 64, 0, "half", False), (128, 192, 64, "half", True), (64, 128, 48, "interleaved", True),
                                                      (128, 64, 128, "interleaved", False), (128, 256, 112, "half", False)])
def test_codes_do_not_depend_on_the_calls(fmt, dtype, d, page, rot, layout, shifted):
    dt, Hkv, B = DTYPES[dtype], 2, 4
    g = torch.Generator().manual_seed(d + rot)
    shift = (torch.randn(Hkv, d, generator=g) * 3).to(DEV) if shifted else None
    plan = sage.rope_plan(rot, layout=layout) if rot else None
    pages, cache = empty(B + 1, Hkv, d, dt, fmt, page, -(-700 // page), shift=shift)
    slots = ints(3, 0, 4, 1)
    # ragged calls, an empty one among them: from single tokens to several blocks, starts and ends inside blocks and on their borders
    steps = [(1, 64, 0, 130), (1, 0, 63, 1), (62, 1, 1, 200), (130, 63, 65, 0), (1, 1, 1, 1), (5, 300, 64, 3), (7, 1, 127, 64)]
    k = torch.randn(sum(map(sum, steps)), Hkv, d, generator=g).to(dt)
    v = (torch.randn(sum(map(sum, steps)), Hkv, d, generator=g) * 5).to(dt)
    k[3] *= 50
    have, at = [{"k": [], "v": []} for _ in range(B)], 0
    for step in steps:
        T = sum(step)
        n_new, starts = ints(*step), ints(0, *torch.tensor(step).cumsum(0).tolist())
        assert bool((sage.sage_pages_reserve(pages, n_new, slots) == 0).all())
        # K as every other head of a wider tensor, V head-major
        wide = torch.zeros(T, 2 * Hkv, d, dtype=dt, device=DEV)
        wide[:, ::2] = k[at:at + T].to(DEV)
        vv = v[at:at + T].to(DEV).transpose(0, 1).contiguous().transpose(0, 1)
        sage.sage_paged_append(cache, wide[:, ::2], vv, q_start=starts, slots=slots, rope=plan)
        i = at
        for b, n in enumerate(step):
            if n:
                kb = k[i:i + n]
                if plan is not None:
                    old = sum(len(x) for x in have[b]["k"])
                    kb = sage.sage_rope(kb.to(DEV), torch.arange(old, old + n, dtype=torch.int32, device=DEV), plan).cpu()
                have[b]["k"].append(kb)
                have[b]["v"].append(v[i:i + n])
            i += n
        at += T
    for b, slot in enumerate(slots.tolist()):
        tokens = {x: torch.cat(have[b][x]) for x in "kv"}
        assert int(pages.lens[slot]) == tokens["k"].shape[0]
        check_blocks(cache, slot, tokens, shift)
    # the whole sequences in one call give the same bytes
    pages2, cache2 = empty(B + 1, Hkv, d, dt, fmt, page, -(-700 // page), shift=shift)
    n_all = [sum(len(x) for x in h["k"]) for h in have]
    sage.sage_pages_reserve(pages2, ints(*n_all), slots)
    raw, i = [], [[] for _ in range(B)]
    at = 0
    for step in steps:
        for b, n in enumerate(step):
            i[b].append((k[at:at + n], v[at:at + n]))
            at += n
    raw = [torch.cat([x[j] for h in i for x in h]).to(DEV) for j in (0, 1)]
    sage.sage_paged_append(cache2, raw[0], raw[1], q_start=ints(0, *torch.tensor(n_all).cumsum(0).tolist()), slots=slots, rope=plan)
    starts = ints(0, *torch.tensor(n_all).cumsum(0).tolist())
    one = sage.sage_paged_gather(cache, starts, sum(n_all), slots=slots)
    two = sage.sage_paged_gather(cache2, starts, sum(n_all), slots=slots)
    for x, y in zip(one, two):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_a_shortened_sequence_goes_on():
    """Drafted tokens are taken back, up to 64 of them and across a block's border, and others come: as if the first had never been."""
    d, Hkv, dt = 64, 1, torch.bfloat16
    pages, cache = empty(1, Hkv, d, dt, "int8", 64, 6)
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(400, Hkv, d, generator=g).to(dt) for _ in "kv")
    keep = {"k": [], "v": []}
    at, n = 0, 0
    for add, back in ((100, 0), (64, 64), (30, 29), (63, 63), (1, 0), (27, 5), (1, 0)):
        sage.sage_pages_reserve(pages, ints(add))
        sage.sage_paged_append(cache, k[at:at + add].to(DEV), v[at:at + add].to(DEV))
        pages.lens.sub_(back)
        for x, t in (("k", k), ("v", v)):
            keep[x].append(t[at:at + add - back])
        at, n = at + add, n + add - back
    sage.sage_pages_reserve(pages, ints(3))
    sage.sage_paged_append(cache, k[at:at + 3].to(DEV), v[at:at + 3].to(DEV))
    tokens = {x: torch.cat(keep[x] + [t[at:at + 3]]) for x, t in (("k", k), ("v", v))}
    check_blocks(cache, 0, tokens, shortened=True)
    t = Table(pages)
    assert t.count() == t.refs                      # the pages kept by the shortened sequence were used, not lost


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_values_that_are_not_finite_show_and_heal(fmt):
    d, dt = 128, torch.float16
    pages, cache = empty(2, 2, d, dt, fmt, 64, 4)
    k, v = (torch.randn(2 * 100, 2, d, device=DEV).to(dt) for _ in "kv")
    k[70, 0, 5], v[170, 1, 7] = float("inf"), float("nan")
    v[0, 0, 0] = 65504.0
    sage.sage_pages_reserve(pages, ints(100, 100))
    sage.sage_paged_append(cache, k, v)
    kk, vv = sage.sage_paged_gather(cache, ints(0, 100, 200), 200)
    bad_k, bad_v = torch.zeros(200, 2, dtype=torch.bool), torch.zeros(200, 2, dtype=torch.bool)
    bad_k[64:100, 0], bad_v[164:200, 1] = True, True
    assert torch.equal(kk.isnan().all(-1).cpu(), bad_k) and torch.equal(kk.isnan().any(-1).cpu(), bad_k)
    assert torch.equal(vv.isnan().all(-1).cpu(), bad_v) and torch.equal(vv.isnan().any(-1).cpu(), bad_v)
    q = torch.randn(2 * 36, 4, d, device=DEV).to(dt)
    out = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=100).view(2, 36, 2, 2, d)
    # rows 0 .. 35 are tokens 64 .. 99: all see the block; the other sequence and head do not
    assert out[0, :, 0].isnan().all() and out[1, :, 1].isnan().all() and out[0, :, 1].isfinite().all() and out[1, :, 0].isfinite().all()
    # the tokens from the bad one on are taken back, and good ones come
    pages.lens.copy_(ints(70, 70))
    sage.sage_pages_reserve(pages, ints(1, 1))
    sage.sage_paged_append(cache, torch.ones(2, 2, d, device=DEV, dtype=dt), torch.ones(2, 2, d, device=DEV, dtype=dt))
    kk, vv = sage.sage_paged_gather(cache, ints(0, 71, 142), 142)
    assert kk.isfinite().all() and vv.isfinite().all()


def test_rows_that_do_not_see_a_bad_block_stay_clean():
    """Causal rows in front of a block with a NaN scale, in one tile with rows that see it."""
    d, dt = 64, torch.bfloat16
    for fmt in ("int8", "e4m3"):
        cache = make_cache([200], Hkv=1, d=d, dtype=dt, fmt=fmt, page_tokens=64, seed=4)
        p = int(cache.pages.table[0, 3])
        cache.v_scale[p], cache.k_scale[p] = float("nan"), float("nan")    # tokens 192 ..
        q = torch.randn(12, 1, d, device=DEV).to(dt)
        out = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=200)
        assert out[:4].isfinite().all() and out[4:].isnan().all()


def test_tiny_and_zero_blocks():
    d, dt = 64, torch.bfloat16
    pages, cache = empty(1, 1, d, dt, "e4m3", 64, 2)
    k, v = torch.zeros(70, 1, d, device=DEV, dtype=dt), torch.full((70, 1, d), 1e-38, device=DEV, dtype=dt)
    sage.sage_pages_reserve(pages, ints(70))
    sage.sage_paged_append(cache, k, v)
    kk, vv = sage.sage_paged_gather(cache, ints(0, 70), 70)
    assert bool((kk == 0).all()) and bool((vv == 0).all())
    out = sage.sage_attn_fwd_paged(torch.randn(1, 1, d, device=DEV).to(dt), cache, causal=True, max_len=70)
    assert bool((out == 0).all())


def test_gather_pads_skips_and_refuses():
    cache = make_cache([100, 0, 65], Hkv=2, d=64, dtype=torch.float16, fmt="int8", page_tokens=64, seed=1, slots=4)
    starts, slots = ints(2, 132, 132, 140, 150, 160), ints(0, 1, 2, 3, -1)
    k, v = sage.sage_paged_gather(cache, starts, 170, slots=slots)
    for x, y in (("k", k), ("v", v)):
        y = y.double().cpu()
        assert torch.equal(y[2:102], sequence(cache, x, 0, 100).half().double()) and bool((y[102:132] == 0).all())
        assert torch.equal(y[132:140], sequence(cache, x, 2, 8).half().double()) and bool((y[140:150] == 0).all())
    # rows of no sequence and of padding are left as they are: through the C call, into a marked buffer
    k.fill_(3.0), v.fill_(3.0)
    assert sage.lib().sage_paged_gather(cache.pages.ref, cache.ref, k.data_ptr(), v.data_ptr(), starts.data_ptr(), slots.data_ptr(), 5, 170,
                                        torch.cuda.current_stream().cuda_stream) == 0
    for y in (k, v):
        assert bool((y[:2] == 3).all()) and bool((y[150:] == 3).all()) and not bool((y[2:150] == 3).all(-1).any())
    cache.pages.table[0, 1] = 999                       # no such page
    k, _ = sage.sage_paged_gather(cache, ints(0, 100), 100, slots=ints(0))
    assert k[:64].isfinite().all() and k[64:].isnan().all()


# ---- pages --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("seed,n_pages,slots,width,page", [(0, 7, 5, 4, 64), (1, 300, 40, 12, 128), (2, 40000, 300, 140, 64), (3, 17001, 64, 300, 192)])
def test_the_tables_upkeep(seed, n_pages, slots, width, page):
    """Random calls, among them the ones that are refused, against loops over lists."""
    g = torch.Generator().manual_seed(seed)
    pages = sage.PageTable.empty(n_pages, page_tokens=page, slots=slots, width=width, device=DEV)
    sim = Table(pages)
    pick = lambda lo, hi, n: torch.randint(lo, hi, (n,), generator=g).tolist()  # noqa: E731
    for step in range(24):
        what = ("reserve", "reserve", "fork", "free", "reserve", "compact")[step % 6]
        n = pick(1, slots + 3, 1)[0]
        if what == "reserve":
            s, m = pick(-1, slots + 1, n), pick(-1, width * page // 3 + 2, n)
            got = sage.sage_pages_reserve(pages, ints(*m), ints(*s)).tolist()
            assert got == sim.reserve(s, m), step
        elif what == "fork":
            src, dst = pick(-1, slots + 1, n), pick(-1, slots + 1, n)
            status, pm, sm = sage.sage_pages_fork(pages, ints(*src), ints(*dst))
            want = sim.fork(src, dst)
            assert (status.tolist(), pm.tolist(), sm.tolist()) == want, step
        elif what == "free":
            s = pick(-1, slots + 1, n)
            sage.sage_pages_free(pages, ints(*(s + s[:2])))
            sim.free(s)
        else:
            most = pick(1, n_pages, 1)[0] if step % 2 else pick(1, 4, 1)[0]
            moves, counts = sage.sage_pages_compact(pages, most)
            assert (moves.tolist(), counts.tolist()) == sim.compact(most), step
        sim.same(pages)
        assert sim.count() == sim.refs
        if step % 5 == 4:                               # sequences are shortened now and then
            cut = torch.tensor([x // 2 if x % 3 == 0 else x for x in sim.lens])
            pages.lens.copy_(cut.to(torch.int32))
            sim.lens = cut.tolist()
    sage.sage_pages_reserve(pages)                       # one token for every slot
    sim.reserve(list(range(slots)), [1] * slots)
    sim.same(pages)


@pytest.mark.parametrize("d,Hkv,page,fmt", [(64, 1, 64, "int8"), (128, 3, 192, "e4m3")])
def test_copies_follow_forks_and_compaction(d, Hkv, page, fmt):
    dt = torch.bfloat16
    pages, cache = empty(12, Hkv, d, dt, fmt, page, 5, n_pages=40)
    _, other = empty(12, Hkv, d, dt, fmt, page, 5, n_pages=40)
    other = sage.PagedCache(pages, k=other.k, v=other.v, k_scale=other.k_scale, v_scale=other.v_scale, k_tail=other.k_tail, v_tail=other.v_tail, fmt=fmt)
    lens = [page * 2, page + 1, 3 * page - 1, 5, 64]
    T = sum(lens)
    sage.sage_pages_reserve(pages, ints(*lens), ints(*range(5)))
    starts = ints(0, *torch.tensor(lens).cumsum(0).tolist())
    kv = [torch.randn(T, Hkv, d, device=DEV).to(dt) for _ in range(4)]
    for c, (k, v) in ((cache, kv[:2]), (other, kv[2:])):     # two layers of one table
        sage.sage_paged_append(c, k, v, q_start=starts, slots=ints(*range(5)))
    status, moves, slot_moves = sage.sage_pages_fork(pages, ints(0, 1, 1, 2, 3), ints(5, 6, 7, 8, 9))
    assert bool((status == 0).all())
    for c in (cache, other):
        sage.sage_pages_copy(c, moves, slot_moves)

    def both(c, slots, n):
        return [sage.sage_paged_gather(c, ints(0, *torch.tensor(n).cumsum(0).tolist()), sum(n), slots=ints(*slots))]

    n = [lens[i] for i in (0, 1, 1, 2, 3)]
    for c in (cache, other):
        for a, b in zip(both(c, (0, 1, 1, 2, 3), n), both(c, (5, 6, 7, 8, 9), n)):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # children grow on their own: parents and siblings keep their tokens
    before = [both(c, (0, 1, 2, 3, 7), [lens[0], lens[1], lens[2], lens[3], lens[1]])[0] for c in (cache, other)]
    sage.sage_pages_reserve(pages, ints(3, 70, 1), ints(5, 6, 8))
    for c in (cache, other):
        more = torch.randn(74, Hkv, d, device=DEV).to(dt)
        sage.sage_paged_append(c, more, -more, q_start=ints(0, 3, 73, 74), slots=ints(5, 6, 8))
    after = [both(c, (0, 1, 2, 3, 7), [lens[0], lens[1], lens[2], lens[3], lens[1]])[0] for c in (cache, other)]
    for a, b in zip(before, after):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # the first slots go; what is left moves to the front and reads as before
    left, n = (4, 5, 6, 7, 8, 9), [int(pages.lens[s]) for s in (4, 5, 6, 7, 8, 9)]
    before = [both(c, left, n)[0] for c in (cache, other)]
    sage.sage_pages_free(pages, ints(0, 1, 2, 3))
    for most in (1, 40):
        moves, counts = sage.sage_pages_compact(pages, most)
        for c in (cache, other):
            sage.sage_pages_copy(c, moves)
    live = int((pages.refs > 0).sum())
    assert counts[0] == live and bool((pages.refs[:live] > 0).all()) and int(pages.table.max()) < live
    for a, b in zip(before, [both(c, left, n)[0] for c in (cache, other)]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # moves outside the pool are passed over
    k = cache.k.clone()
    sage.sage_pages_copy(cache, ints(-1, 3, 2, 40, 1 << 30, 1, 3, -7).view(4, 2), ints(-1, 0, 12, 1).view(2, 2))
    assert torch.equal(k, cache.k)


# ---- attention ----------------------------------------------------------------------------------------------------------

def run_case(lens, news, *, Hq, Hkv, d, dtype, fmt, page, causal, seed, split=0, max_len=None, uniform=False, sm_scale=0.0, scale_q=1.0):
    dt = DTYPES[dtype]
    cache = make_cache(lens, Hkv=Hkv, d=d, dtype=dt, fmt=fmt, page_tokens=page, seed=seed)
    T = sum(news)
    q = (torch.randn(T + 2, Hq, d, generator=torch.Generator().manual_seed(seed)) * scale_q).to(dt)
    # rows behind the last sequence are left as they are
    out = torch.full((T + 2, Hq, d), 5.0, dtype=dt, device=DEV)
    starts = None if uniform else ints(0, *torch.tensor(news).cumsum(0).tolist())
    rows = slice(0, T) if uniform else slice(0, T + 2)
    sage.sage_attn_fwd_paged(q.to(DEV)[rows], cache, causal=causal, max_len=max_len or max(lens + [1]), q_start=starts, out=out[rows], split_keys=split,
                             sm_scale=sm_scale)
    assert bool((out[T:] == 5).all())
    at = 0
    for b, (n, m) in enumerate(zip(lens, news)):
        want, err = attention(q[at:at + m], sequence(cache, "k", b, n), sequence(cache, "v", b, n), causal=causal, sm_scale=sm_scale)
        assert_attention(out[at:at + m], want, err, dt, f"sequence {b} of {n} tokens, {m} rows")
        at += m
    return cache, q, out


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens(fmt, dtype, d):
    lens = [1, 63, 64, 65, 200, 0, 515]
    run_case(lens, [1] * 7, Hq=6, Hkv=2, d=d, dtype=dtype, fmt=fmt, page=128, causal=True, seed=d, uniform=True)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (16, 1), (17, 1), (40, 2), (6, 3), (128, 1)])
@pytest.mark.parametrize("split", [0, 64, 192])
def test_head_groups_and_ranges(Hq, Hkv, split):
    # 1 to 384 packed rows: one wavefront, shared keys, rows of their own; more ranges than some sequences have blocks
    run_case([300, 65, 7, 450], [1, 3, 2, 1], Hq=Hq, Hkv=Hkv, d=64, dtype="bf16", fmt="int8", page=64, causal=True, seed=Hq + split, split=split)


@pytest.mark.parametrize("fmt,dtype,d", [("int8", "bf16", 128), ("e4m3", "fp16", 64), ("e4m3", "bf16", 128), ("int8", "fp16", 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks_and_single_tokens_together(fmt, dtype, d, causal):
    run_case([400, 129, 77, 1, 260, 64], [130, 1, 77, 1, 33, 0], Hq=4, Hkv=2, d=d, dtype=dtype, fmt=fmt, page=192, causal=causal, seed=9, split=128)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_long_chunks(fmt, dtype, causal):
    # tiles of 128 rows over an odd and an even number of blocks, in one range and in three; the last tile is short
    for lens, split in (([705, 1024], 0), ([705, 1024], 384)):
        run_case(lens, [150, 200], Hq=6, Hkv=2, d=128, dtype=dtype, fmt=fmt, page=64, causal=causal, seed=21, split=split)


@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "fp16"), ("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_between_the_tiles_of_32(fmt, dtype, causal):
    # 33 to 48 and 65 to 96 packed rows on average, d 64: one, two and four groups of rows, two tiles, rows beyond a sequence's length
    for lens, news, split in (([300, 5, 64], [5, 5, 5], 0), ([300, 129, 70, 515], [9, 1, 4, 8], 64), ([260, 1, 130, 64], [20, 1, 1, 1], 128),
                              ([450, 12], [12, 12], 192), ([705, 64, 3, 65, 200], [44, 1, 1, 1, 1], 256), ([705, 40, 3, 65, 0], [44, 1, 1, 1, 1], 0)):
        run_case(lens, news, Hq=16, Hkv=2, d=64, dtype=dtype, fmt=fmt, page=128, causal=causal, seed=sum(news), split=split)


@pytest.mark.parametrize("d,rows,split", [(128, 1, 0), (128, 40, 256), (64, 3, 64), (64, 10, 0)])
def test_large_values(d, rows, split):
    # V of 2^127 / (number of keys) and a scale of its own per block, equal weights: no sum passes the range
    n, Hkv = 1024, 2
    cache = make_cache([n], Hkv=Hkv, d=d, dtype=torch.bfloat16, fmt="int8", page_tokens=64, seed=d)
    v = sequence(cache, "v", 0, n)
    cache.v_scale.mul_(2.0 ** 116 / float(v.abs().max()))
    q = (torch.randn(rows, 8, d, generator=torch.Generator().manual_seed(3)) * 2.0 ** -60).bfloat16()
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=False, max_len=n, split_keys=split)
    want, err = attention(q, sequence(cache, "k", 0, n), sequence(cache, "v", 0, n), causal=False)
    assert_attention(out, want, err, torch.bfloat16, f"{rows} rows")


def test_rows_that_see_nothing_are_zeros():
    # more rows than tokens: the first ones lie in front of the sequence
    for split in (0, 64):
        for Hq in (2, 64):
            _, _, out = run_case([3, 0, 70], [9, 4, 100], Hq=Hq, Hkv=2, d=64, dtype="fp16", fmt="e4m3", page=64, causal=True, seed=2, split=split)
            assert bool((out[:6] == 0).all()) and bool((out[9:13] == 0).all()) and bool((out[13:43] == 0).all())


def test_bounds_that_are_too_low_and_other_scales():
    run_case([700, 10], [2, 2], Hq=8, Hkv=2, d=64, dtype="bf16", fmt="int8", page=64, causal=True, seed=5, max_len=1, uniform=True)
    run_case([700, 10], [2, 2], Hq=8, Hkv=2, d=64, dtype="bf16", fmt="int8", page=64, causal=True, seed=5, max_len=130, split=64, sm_scale=0.3)
    run_case([700, 10], [2, 2], Hq=8, Hkv=2, d=128, dtype="bf16", fmt="e4m3", page=64, causal=False, seed=6, max_len=1 << 20, scale_q=40.0)


@pytest.mark.parametrize("exponent", [-60, 60])
def test_bfloat16_rows_beyond_the_range_of_binary16(exponent):
    cache = make_cache([130], Hkv=1, d=64, dtype=torch.bfloat16, fmt="int8", page_tokens=64, seed=8)
    q = torch.randn(3, 2, 64).bfloat16()
    scaled = (q.double() * 2.0 ** exponent).bfloat16()
    a = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=True, max_len=130, sm_scale=0.125)
    b = sage.sage_attn_fwd_paged(scaled.to(DEV), cache, causal=True, max_len=130, sm_scale=0.125 * 2.0 ** -exponent)
    assert torch.equal(a, b)                           # powers of two all the way


def test_views_padding_and_shared_slots():
    cache = make_cache([150, 90], Hkv=2, d=64, dtype=torch.float16, fmt="int8", page_tokens=64, seed=3, slots=4)
    q = torch.randn(5, 4, 64, device=DEV).half()
    want = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=150, slots=ints(1, 0, 0, 1, 1))
    qkv = torch.randn(5, 8, 64, device=DEV).half()
    qkv[:, 2:6] = q
    room = torch.full((4, 7, 64), 9.0, device=DEV).half().transpose(0, 1)     # [7, 4, 64], head-major
    out = sage.sage_attn_fwd_paged(qkv[:, 2:6], cache, causal=True, max_len=150, slots=ints(1, 0, 0, 1, 1), out=room[1:6])
    assert torch.equal(out, want) and bool((room[0] == 9).all()) and bool((room[6] == 9).all())
    # slots outside the table are padding: those rows stay, the others do not change
    out = torch.full_like(q, 9.0)
    sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=150, slots=ints(1, -1, 0, 4, 1), out=out)
    assert torch.equal(out[[0, 2, 4]], want[[0, 2, 4]]) and bool((out[[1, 3]] == 9).all())
    lens = cache.pages.lens.clone()
    k = cache.k.clone()
    sage.sage_paged_append(cache, q[:2, :2], q[:2, :2], slots=ints(-1, 4))
    assert torch.equal(k, cache.k) and torch.equal(lens, cache.pages.lens)


def test_missing_pages_and_wild_lengths_give_nan_and_nothing_worse():
    cache = make_cache([150, 90, 20], Hkv=1, d=64, dtype=torch.float16, fmt="e4m3", page_tokens=64, seed=3)
    q = torch.randn(3, 2, 64, device=DEV).half()
    good = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=150)
    cache.pages.table[0, 1], cache.pages.lens[1] = 1 << 30, 2 ** 31 - 1
    for split in (0, 64):
        out = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=150, split_keys=split)
        assert out[:2].isnan().all() and torch.equal(out[2], good[2])
    cache.pages.lens[1] = -5
    out = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=150)
    assert bool((out[1] == 0).all())
    # row starts that go back or beyond the rows: nothing outside is touched
    room = torch.full((5, 2, 64), 9.0, device=DEV).half()
    sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=150, q_start=ints(2, 1, 50, -7), out=room[1:4])
    assert bool((room[0] == 9).all()) and bool((room[4] == 9).all())
    k = cache.k.clone()
    cache.pages.lens.fill_(0)
    sage.sage_paged_append(cache, q[:, :1], q[:, :1])
    cache.pages.lens.fill_(2 ** 31 - 1)
    cache.pages.table.fill_(-1)
    sage.sage_paged_append(cache, q[:, :1], q[:, :1])
    torch.cuda.synchronize()
    assert torch.equal(k, cache.k)


def test_many_sequences_and_a_long_one():
    # more sequences than a workgroup has threads, ragged; then a cache beyond 4 GiB of codes, read at its end
    lens = [1 + (37 * b) % 90 for b in range(300)]
    news = [1 + b % 2 for b in range(300)]
    run_case(lens, [min(a, b) for a, b in zip(lens, news)], Hq=2, Hkv=1, d=64, dtype="bf16", fmt="int8", page=64, causal=True, seed=1)


def test_a_pool_beyond_four_gib():
    Hkv, d, page = 8, 128, 1024
    n_pages = (5 << 30) // (Hkv * d * page)
    pages = sage.PageTable.empty(n_pages, page_tokens=page, slots=1, width=2, device=DEV)
    cache = sage.PagedCache.empty(pages, Hkv, d, torch.bfloat16, fmt="int8")
    pages.refs[:n_pages - 2] = 1
    assert sage.sage_pages_reserve(pages, ints(1500)).tolist() == [0] and pages.table.tolist() == [[n_pages - 2, n_pages - 1]]
    k, v = (torch.randn(1500, Hkv, d, device=DEV).bfloat16() for _ in "kv")
    sage.sage_paged_append(cache, k, v)
    q = torch.randn(1, 2 * Hkv, d).bfloat16()
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=True, max_len=1500)
    kk, vv = (t.double().cpu() for t in sage.sage_paged_gather(cache, ints(0, 1500), 1500))
    # the gathered values carry one more rounding to bfloat16: compared with what they are off, not with the kernel's bound
    want, err = attention(q, kk, vv, causal=True)
    assert (out.double().cpu() - want).norm() <= 2.0 ** -6 * want.norm()
    small = sage.PagedCache.empty(sage.PageTable.empty(2, page_tokens=page, slots=1, width=2, device=DEV), Hkv, d, torch.bfloat16, fmt="int8")
    sage.sage_pages_reserve(small.pages, ints(1500))
    sage.sage_paged_append(small, k, v)
    assert torch.equal(out, sage.sage_attn_fwd_paged(q.to(DEV), small, causal=True, max_len=1500))


def test_results_do_not_depend_on_the_batch():
    lens = [300, 900, 65, 500]
    cache = make_cache(lens, Hkv=2, d=64, dtype=torch.bfloat16, fmt="int8", page_tokens=64, seed=11)
    q = torch.randn(4, 8, 64, device=DEV).bfloat16()
    all_ = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=900, split_keys=128)
    for b in range(4):
        one = sage.sage_attn_fwd_paged(q[b:b + 1], cache, causal=True, max_len=900, split_keys=128, slots=ints(b))
        assert torch.equal(one[0], all_[b])
    again = sage.sage_attn_fwd_paged(q, cache, causal=True, max_len=900, split_keys=128)
    assert torch.equal(again, all_)


# ---- together -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "fp16")])
def test_a_serving_loop(fmt, dtype):
    """Prompts in chunks, then tokens one by one with a fork, a sequence that ends and a compaction in between: attention over all tokens so
    far in 64 bits, within what 8 bits lose; and over the cache's own values, within the kernel's bound."""
    dt, Hq, Hkv, d = DTYPES[dtype], 4, 2, 64
    g = torch.Generator().manual_seed(12)
    shift = torch.randn(Hkv, d, generator=g) * 2
    pages, cache = empty(6, Hkv, d, dt, fmt, 64, 6, n_pages=20, shift=shift.to(DEV))
    plan = sage.rope_plan(d, scaling="linear", factor=2.0)
    held = {}

    def step(slots, news):
        T = sum(news)
        q, k, v = (torch.randn(T, h, d, generator=g).to(dt) for h in (Hq, Hkv, Hkv))
        k = (k.float() + shift).to(dt)
        starts = ints(0, *torch.tensor(news).cumsum(0).tolist())
        assert bool((sage.sage_pages_reserve(pages, ints(*news), ints(*slots)) == 0).all())
        lens = [int(pages.lens[s]) for s in slots]
        pos = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, news)]).to(torch.int32).to(DEV)
        qr = sage.sage_rope(q.to(DEV), pos, plan)
        kr = sage.sage_rope(k.to(DEV), pos, plan).cpu()
        sage.sage_paged_append(cache, k.to(DEV), v.to(DEV), q_start=starts, slots=ints(*slots), rope=plan)
        out = sage.sage_attn_fwd_paged(qr, cache, causal=True, max_len=384, q_start=starts, slots=ints(*slots))
        at = 0
        for s, n, m in zip(slots, lens, news):
            old = held.get(s, (kr[:0], v[:0]))
            held[s] = (torch.cat([old[0], kr[at:at + m]]), torch.cat([old[1], v[at:at + m]]))
            kk, vv = sequence(cache, "k", s, n), sequence(cache, "v", s, n)
            want, err = attention(qr[at:at + m].cpu(), kk, vv, causal=True)
            assert_attention(out[at:at + m], want, err, dt, f"slot {s}: {n} tokens")
            assert held[s][0].shape[0] == n
            check_blocks(cache, s, {"k": held[s][0], "v": held[s][1]}, shift)
            # the rotated K's constant part turns with the position: the shift takes off what it can
            exact, _ = attention(qr[at:at + m].cpu(), held[s][0].double(), held[s][1].double(), causal=True)
            assert (out[at:at + m].double().cpu() - exact).norm() <= 0.1 * exact.norm()
            at += m

    step([0, 1, 2], [70, 5, 130])
    step([1, 2], [64, 60])
    step([0, 1, 2], [1, 1, 1])
    status, moves, slot_moves = sage.sage_pages_fork(pages, ints(0, 2, 2), ints(3, 4, 5))
    assert status.tolist() == [0, 0, 0]
    sage.sage_pages_copy(cache, moves, slot_moves)
    for s, t in ((0, 3), (2, 4), (2, 5)):
        held[t] = held[s]
    step([0, 1, 2, 3, 4, 5], [1, 1, 1, 2, 3, 1])
    sage.sage_pages_free(pages, ints(0, 2))
    moves, counts = sage.sage_pages_compact(pages)
    sage.sage_pages_copy(cache, moves)
    held.pop(0), held.pop(2)
    step([5, 4, 3, 1], [1, 64, 1, 2])
    step([2, 1], [100, 1])


def test_a_captured_step_replays_as_sequences_grow():
    """One token of every slot, reserve to attention, captured once: every replay against the same calls made eagerly on a second cache."""
    Hq, Hkv, d, dt, B = 8, 2, 64, torch.bfloat16, 3
    plan = sage.rope_plan(d)
    pages, cache = empty(B, Hkv, d, dt, "int8", 64, 8)
    pages2, cache2 = empty(B, Hkv, d, dt, "int8", 64, 8)
    lens = [62, 190, 5]
    k, v = (torch.randn(sum(lens), Hkv, d, device=DEV).to(dt) for _ in "kv")
    for p, c in ((pages, cache), (pages2, cache2)):
        sage.sage_pages_reserve(p, ints(*lens))
        sage.sage_paged_append(c, k, v, q_start=ints(0, *torch.tensor(lens).cumsum(0).tolist()), rope=plan)
    q, k1, v1 = (torch.zeros(B, h, d, device=DEV, dtype=dt) for h in (Hq, Hkv, Hkv))
    ws = torch.empty(max(256, sage.paged_workspace_bytes(B, B, Hq, Hkv, d, 512)), dtype=torch.uint8, device=DEV)
    slots, out = ints(*range(B)), torch.zeros(B, Hq, d, device=DEV, dtype=dt)

    def step(p, c, out):
        sage.sage_pages_reserve(p, slots=slots)
        pos = p.lens - 1
        qr = sage.sage_rope(q, pos, plan)
        sage.sage_paged_append(c, k1, v1, rope=plan)
        return sage.sage_attn_fwd_paged(qr, c, causal=True, max_len=512, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pages, cache, out)
    for i in range(70):                                  # across blocks and pages
        for t in (q, k1, v1):
            t.copy_(torch.randn(t.shape, device=DEV).to(dt))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = step(pages2, cache2, torch.zeros_like(out))   # shares the workspace, between the replays
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(pages.lens, pages2.lens) and torch.equal(pages.table, pages2.table), i
    n = [int(x) for x in pages.lens]
    for a, b in zip(sage.sage_paged_gather(cache, ints(0, *torch.tensor(n).cumsum(0).tolist()), sum(n)),
                    sage.sage_paged_gather(cache2, ints(0, *torch.tensor(n).cumsum(0).tolist()), sum(n))):
        assert torch.equal(a, b)


def test_captured_upkeep():
    """Fork, copy, free, compaction and reading back in one graph: every replay, from a table that changed in between, against the eager calls."""
    B, Hkv, d, dt = 3, 2, 64, torch.float16
    slots, n_pages = 8, 24
    sets = [empty(slots, Hkv, d, dt, "e4m3", 64, 6, n_pages=n_pages) for _ in range(2)]
    src, dst, gone, starts = ints(1, 2, 1), ints(4, 5, 6), ints(1, 0), ints(0, 200, 300, 400)

    def work(pages, cache):
        status, moves, slot_moves = sage.sage_pages_fork(pages, src, dst)
        sage.sage_pages_copy(cache, moves, slot_moves)
        sage.sage_pages_free(pages, gone)
        moves, counts = sage.sage_pages_compact(pages)
        sage.sage_pages_copy(cache, moves)
        return status, counts, *sage.sage_paged_gather(cache, starts, 400, slots=dst)

    def fill(pages, cache, lens, k):
        sage.sage_pages_free(pages, torch.arange(slots, dtype=torch.int32, device=DEV))
        sage.sage_pages_reserve(pages, ints(*lens), ints(0, 1, 2))
        sage.sage_paged_append(cache, k, -k, q_start=ints(0, *torch.tensor(lens).cumsum(0).tolist()), slots=ints(0, 1, 2))

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    first = torch.randn(150, Hkv, d, device=DEV).to(dt)
    fill(*sets[0], [10, 70, 70], first)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = work(*sets[0])
    for lens in ([10, 70, 70], [300, 128, 1], [64, 200, 90], [10, 70, 70]):
        k = torch.randn(sum(lens), Hkv, d, device=DEV).to(dt)
        for s in sets:
            fill(*s, lens, k)
        graph.replay()
        torch.cuda.synchronize()
        want = work(*sets[1])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), lens
        assert torch.equal(sets[0][0].table, sets[1][0].table) and torch.equal(sets[0][0].refs, sets[1][0].refs)


def test_two_graphs_share_a_workspace_and_two_streams_do_not():
    cache = make_cache([700, 300], Hkv=2, d=64, dtype=torch.bfloat16, fmt="int8", page_tokens=64, seed=5)
    q = [torch.randn(2, 8, 64, device=DEV).bfloat16() for _ in range(2)]
    kw = dict(causal=True, max_len=700, split_keys=64)
    want = [sage.sage_attn_fwd_paged(x, cache, **kw) for x in q]
    ws = torch.empty(sage.paged_workspace_bytes(2, 2, 8, 2, 64, 700, 64), dtype=torch.uint8, device=DEV)
    outs, graphs, side = [torch.zeros_like(x) for x in q], [torch.cuda.CUDAGraph() for _ in q], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for x, o, g in zip(q, outs, graphs):
        with torch.cuda.graph(g, stream=side):
            sage.sage_attn_fwd_paged(x, cache, out=o, workspace=ws, **kw)
    for i in (0, 1, 1, 0, 1):
        outs[i].zero_()
        ws.fill_(255)                                     # nothing in it has to be initialised
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = sage.sage_attn_fwd_paged(q[i], cache, **kw)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals_on_the_device():
    cache = make_cache([5], Hkv=1, d=64, dtype=torch.float16, fmt="int8", page_tokens=64, seed=1)
    q = torch.zeros(2, 2, 64, device=DEV, dtype=torch.float16)
    attn = lambda q=q, **kw: sage.sage_attn_fwd_paged(q, cache, **dict(dict(causal=True, max_len=64), **kw))  # noqa: E731
    for call in (lambda: attn(q.bfloat16()), lambda: attn(torch.zeros(2, 2, 128, device=DEV).half()), lambda: attn(q[..., ::2]), lambda: attn(q[0]),
                 lambda: attn(q_start=ints(0)), lambda: attn(q_start=torch.zeros(2, device=DEV)), lambda: attn(slots=ints(0, 0, 0)), lambda: attn(max_len=0),
                 lambda: attn(split_keys=100), lambda: attn(out=q[:1]), lambda: attn(workspace=torch.zeros(16, device=DEV)[1:], split_keys=64, max_len=640),
                 lambda: sage.sage_paged_append(cache, q, q), lambda: sage.sage_paged_append(cache, q[:, :1], q[:1, :1]),
                 lambda: sage.sage_paged_append(cache, q[:, :1], q[:, :1], slots=ints(0, 0, 0)), lambda: sage.sage_paged_gather(cache, ints(0), 4),
                 lambda: sage.sage_paged_gather(cache, ints(0, 4).long(), 4), lambda: sage.sage_paged_gather(cache, ints(0, 4), 0),
                 lambda: sage.sage_pages_reserve(cache.pages, ints(1, 2)), lambda: sage.sage_pages_fork(cache.pages, ints(0), ints(0, 1)),
                 lambda: sage.sage_pages_compact(cache.pages, 0), lambda: sage.sage_pages_copy(cache, ints(0, 1)),
                 lambda: sage.PagedCache(cache.pages, k=cache.k, v=cache.v, k_scale=cache.k_scale, v_scale=cache.v_scale, k_tail=cache.k_tail,
                                         v_tail=cache.v_tail[:, :, :64], fmt="int8"),
                 lambda: sage.PageTable(table=cache.pages.table, lens=cache.pages.lens.long(), refs=cache.pages.refs, page_tokens=64)):
        with pytest.raises(sage.SageError):
            call()
