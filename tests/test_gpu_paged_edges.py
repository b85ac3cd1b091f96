"""The paged cache where calls meet what goes wrong in a serving program: lengths beyond the table's row, pages that two sequences share, V blocks of
very different sizes, missing pages, starts that go back; and the sizes at which the kernels change their ways."""
import math

import pytest
import torch

import paper_2505_21136_amd as sage
from paged_ref import EPS, Table, attention, byte_table, make_cache, sequence
from test_gpu_paged import DEV, DTYPES, check_blocks, empty, ints, run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,Hq", [(64, 2), (64, 32), (128, 16)])
def test_starts_that_claim_the_same_tiles_stay_within_the_call(d, Hq):
    """Row starts have to be ascending; with others it is open what a row gets, but nothing outside the call's rows is touched: sequences far enough
    apart that different wavefronts find the same tile."""
    dt, T, B = torch.float16, 640, 300
    cache = make_cache([130] * B, Hkv=1, d=d, dtype=dt, fmt="int8", page_tokens=64, seed=2)
    starts = ints(*[(0, T, 9, T - 4)[i % 4] for i in range(B + 1)])
    q = torch.randn(2 * T, Hq, d, device=DEV).to(dt)
    for split in (0, 64):
        room = torch.full((2 * T, Hq, d), 9.0, device=DEV, dtype=dt)
        sage.sage_attn_fwd_paged(q[:T], cache, causal=True, max_len=130, q_start=starts, out=room[:T], split_keys=split)
        assert bool((room[T:] == 9).all()) and bool((room[:T] != 9).any())
    room = torch.full((2, 2 * T, 1, d), 9.0, device=DEV, dtype=dt)
    assert sage.lib().sage_paged_gather(cache.pages.ref, cache.ref, room[0].data_ptr(), room[1].data_ptr(), starts.data_ptr(), None, B, T,
                                        torch.cuda.current_stream().cuda_stream) == 0
    assert bool((room[:, T:] == 9).all()) and bool((room[:, :T] != 9).any())
    sage.sage_paged_append(cache, q[:T, :1], q[:T, :1], q_start=starts)
    torch.cuda.synchronize()


def _everything(pages, cache):
    """Copies of all that an append may write."""
    return [t.clone().view(torch.uint8) for t in (pages.table, pages.lens, pages.refs, cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail)]


@pytest.mark.parametrize("length", [129, 130, 200, 2 ** 31 - 1])
@pytest.mark.parametrize("rotated", [False, True])
def test_a_length_beyond_the_row_appends_nothing(length, rotated):
    """The row is full and its pages are there, so the tokens would have a place to go: the last of the row's, which other tokens have."""
    d, Hkv, dt = 64, 2, torch.bfloat16
    pages, cache = empty(2, Hkv, d, dt, "int8", 64, 2)
    plan = sage.rope_plan(d) if rotated else None
    k, v = (torch.randn(128 + 70 + 6, Hkv, d, device=DEV).to(dt) for _ in "kv")
    sage.sage_pages_reserve(pages, ints(128, 70))
    sage.sage_paged_append(cache, k[:198], v[:198], q_start=ints(0, 128, 198), rope=plan)
    pages.lens[0] = length
    sage.sage_pages_reserve(pages, ints(3), ints(1))
    before = _everything(pages, cache)
    sage.sage_paged_append(cache, k[198:201], v[198:201], q_start=ints(0, 3, 3), rope=plan)
    for x, y in zip(before, _everything(pages, cache)):
        assert torch.equal(x, y)
    # another sequence of the same call gets its tokens
    sage.sage_paged_append(cache, k[198:], v[198:], q_start=ints(0, 3, 6), rope=plan)
    pages.lens[0] = 128
    for slot, rows in ((0, list(range(128))), (1, list(range(128, 198)) + [201, 202, 203])):
        kk = k[rows]
        if rotated:
            kk = sage.sage_rope(kk, torch.arange(len(rows), dtype=torch.int32, device=DEV), plan)
        check_blocks(cache, slot, {"k": kk.cpu(), "v": v[rows].cpu()})


@pytest.mark.parametrize("back", [1, 3, 64])
def test_an_append_leaves_shared_pages_as_they_are(back):
    """Two sequences share whole pages, one is shortened into them and goes on (back = 64: from a page's first token): the other one's tokens
    stay.  Forked into a slot of its own first, the shortened one goes on as if it had been alone."""
    d, Hkv, dt, n = 64, 2, torch.float16, 128
    pages, cache = empty(4, Hkv, d, dt, "e4m3", 64, 4)
    k, v = (torch.randn(n + 5, Hkv, d, device=DEV).to(dt) for _ in "kv")
    sage.sage_pages_reserve(pages, ints(n), ints(0))
    sage.sage_paged_append(cache, k[:n], v[:n], slots=ints(0))
    status, moves, slot_moves = sage.sage_pages_fork(pages, ints(0, 0), ints(1, 2))
    assert status.tolist() == [0, 0]
    sage.sage_pages_copy(cache, moves, slot_moves)
    both = {"k": k[:n].cpu(), "v": v[:n].cpu()}
    pages.lens[1].sub_(back)
    assert pages.table[1, :2].tolist() == pages.table[2, :2].tolist()
    sage.sage_pages_reserve(pages, ints(5), ints(1))
    sage.sage_paged_append(cache, k[n:], v[n:], slots=ints(1))
    for slot in (0, 2):
        check_blocks(cache, slot, both)
    # slot 2 goes on after taking as many tokens back, by way of slot 3
    pages.lens[2].sub_(back)
    status, moves, slot_moves = sage.sage_pages_fork(pages, ints(2), ints(3))
    assert status.tolist() == [0]
    sage.sage_pages_copy(cache, moves, slot_moves)
    sage.sage_pages_free(pages, ints(2))
    sage.sage_pages_reserve(pages, ints(5), ints(3))
    sage.sage_paged_append(cache, k[n:], v[n:], slots=ints(3))
    check_blocks(cache, 0, both)
    rows = list(range(n - back)) + list(range(n, n + 5))
    check_blocks(cache, 3, {"k": k[rows].cpu(), "v": v[rows].cpu()}, shortened=True)
    t = Table(pages)
    assert t.count() == t.refs


def _bounded_by_own_blocks(got, q, k, v, dtype, what, causal=True):
    """Attention against 64 bits with a bound in which every key counts with its own V alone.

    As paged_ref.attention's, with another last term: a weight's rounding to binary16 is 2^-11 of it or, where it is small, half the spacing of
    the smallest numbers, 2^-25.  The weight is multiplied by 2^14 and by its block's V scale over a power of two that is at
    most 2^8 times the scale, so that this is at most 2^-25 2^-14 2^8 = 2^-31 |v|, where the row's largest weight is 1 and the sum that all is
    divided by at least 1 - 2^-20; nor more than the weight itself: min(p, 2^-30) |v| is granted."""
    want, _ = attention(q, k, v, causal=causal)
    n, Hq, d = q.shape
    N, Hkv = k.shape[0], k.shape[1]
    err = torch.zeros_like(want)
    for h in range(Hq):
        kk, vv = k[:, h * Hkv // Hq], v[:, h * Hkv // Hq]
        s, big = q[:, h].double() @ kk.T / math.sqrt(d), q[:, h].double().abs() @ kk.abs().T / math.sqrt(d)
        seen = torch.arange(N)[None] <= (torch.arange(n)[:, None] + N - n if causal else torch.full((n, 1), N))
        s, big = s.masked_fill(~seen, -math.inf), big.masked_fill(~seen, 0.0)
        p = torch.softmax(s, -1)
        e = (d + 8) * 2.0 ** -24 * big.amax(-1, keepdim=True)
        err[:, h] = (p @ vv.abs()) * (2 * (e + 2.0 ** -20) + 2.0 ** -11 + (N / 64 + 8) * 2.0 ** -23) + p.clamp(max=2.0 ** -30) @ vv.abs()
    tol = err + EPS[dtype] * (want.abs() + err) + 2.0 ** -24
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    worst = ((got - want).abs() / tol).max().item()
    print(f"   {what}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


# the packed rows of a sequence: one wavefront of 16, of 48 (d 64), of 32, rows of their own (d 64) and with shared conversions (d 128)
ROWS = [(64, 1), (64, 12), (64, 40), (64, 8), (128, 1), (128, 8), (128, 40)]


@pytest.mark.parametrize("d,rows", ROWS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("where", ["first", "middle", "in turn", "shrinking"])
@pytest.mark.parametrize("ratio", [12, 16, 24])
def test_blocks_of_large_v_take_no_precision_from_the_others(d, rows, dtype, where, ratio):
    """Blocks with 2^ratio times the others' V and next to none of the weight: what the row gives the others comes out as it does without them."""
    n, Hq, Hkv, dt, fmt = 64 * 18 - 9, 8, 2, DTYPES[dtype], "int8" if rows % 3 else "e4m3"
    cache = make_cache([n], Hkv=Hkv, d=d, dtype=dt, fmt=fmt, page_tokens=64, seed=rows + d)
    table = cache.pages.table[0].tolist()
    loud = {"first": [0], "middle": [7, 8], "in turn": list(range(0, 17, 2)), "shrinking": range(0, 17)}[where]
    cache.v_scale.clamp_(min=0.01, max=0.012)
    cache.k_scale.clamp_(max=0.004 if fmt == "int8" else 0.0012)
    # the first channel of K says how loud a block is: nothing else of it has any weight; q sees it with 2^6, so its keys lose 2^6 * 8 / sqrt(d) at least
    where_k = byte_table("k", d)
    none, low = (128, 0) if fmt == "int8" else (0, 0xfe)     # 0, and -128 or -448 times the scale
    cache.k[:, :, 0, where_k[:, 0].to(DEV)] = none
    for j in loud:
        p = table[j]
        if where == "shrinking":                             # each a little smaller than the one before; all that counts is in the last
            cache.v_scale[p] *= 2.0 ** (ratio * (17 - j) / 17.0)
        else:
            cache.v_scale[p] *= 2.0 ** ratio
        cache.k[p, :, 0, where_k[:, 0].to(DEV)] = low
    q = torch.randn(rows, Hq, d, generator=torch.Generator().manual_seed(rows))
    q[..., 0] = 512.0 if d == 64 else 700.0
    q = q.to(dt)
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=True, max_len=n)
    k, v = sequence(cache, "k", 0, n), sequence(cache, "v", 0, n)
    _bounded_by_own_blocks(out, q, k, v, dt, f"{rows} rows")


@pytest.mark.parametrize("d,rows", ROWS)
@pytest.mark.parametrize("loud", [[0], [9], [17], [3, 11, 12]])
def test_blocks_of_v_very_far_apart_stay_finite(d, rows, loud):
    # equal weights: the large blocks are the result, and the sums of them pass by those that are 2^112 below
    n, dt = 64 * 18 - 9, torch.bfloat16
    cache = make_cache([n], Hkv=2, d=d, dtype=dt, fmt="int8", page_tokens=64, seed=rows)
    cache.v_scale.fill_(0.01)
    for j in loud:
        cache.v_scale[int(cache.pages.table[0, j])] *= 2.0 ** 112
    q = (torch.randn(rows, 8, d, generator=torch.Generator().manual_seed(rows)) * 2.0 ** -40).to(dt)
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=False, max_len=n)
    _bounded_by_own_blocks(out, q, sequence(cache, "k", 0, n), sequence(cache, "v", 0, n), dt, f"{rows} rows", causal=False)


@pytest.mark.parametrize("d,rows", ROWS)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("zeros", [[0], [0, 1, 2, 3, 4], [9, 17], list(range(0, 18, 2)), list(range(18))])
def test_blocks_of_zeros_among_others(d, rows, fmt, zeros):
    # V's scale is 0 there, and K's in some: their keys have weight like others
    n, dt = 64 * 18 - 9, torch.float16
    cache = make_cache([n], Hkv=2, d=d, dtype=dt, fmt=fmt, page_tokens=64, seed=rows)
    for j in zeros:
        p = int(cache.pages.table[0, j])
        cache.v[p], cache.v_scale[p] = 128 if fmt == "int8" else 0, 0.0
        if j % 4 == 0:
            cache.k[p], cache.k_scale[p] = 128 if fmt == "int8" else 0, 0.0
    q = torch.randn(rows, 8, d, generator=torch.Generator().manual_seed(rows)).to(dt)
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=True, max_len=n)
    _bounded_by_own_blocks(out, q, sequence(cache, "k", 0, n), sequence(cache, "v", 0, n), dt, f"{rows} rows")
    assert len(zeros) < 18 or bool((out == 0).all())


@pytest.mark.parametrize("exponent", [8, 16, 22, 23, 24, 25, 26, 27])
@pytest.mark.parametrize("d,rows,fmt", [(64, 1, "int8"), (64, 12, "e4m3"), (64, 40, "int8"), (128, 1, "e4m3"), (128, 8, "int8"), (128, 40, "e4m3")])
def test_scores_of_all_sizes_that_one_key_wins(exponent, d, rows, fmt):
    """Scores up to 2^exponent, in powers of two: where the largest is ahead by more than what binary32 sums of d products leave open, and 40 more,
    the row is that key's V: P~'s and the output's rounding off, and what n others can weigh."""
    n, dt = 300, torch.bfloat16
    cache = make_cache([n], Hkv=2, d=d, dtype=dt, fmt=fmt, page_tokens=64, seed=d + rows)
    q = torch.randn(rows, 8, d, generator=torch.Generator().manual_seed(3)).to(dt)
    k, v = sequence(cache, "k", 0, n), sequence(cache, "v", 0, n)
    raw = torch.stack([q[:, h].double() @ k[:, h // 4].T for h in range(8)], 1)
    sm = 2.0 ** exponent * math.log(2) / float(raw.abs().max())
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=False, max_len=n, sm_scale=sm).double().cpu()
    two = (raw * sm).topk(2, -1)
    big = torch.stack([q[:, h].double().abs() @ k[:, h // 4].abs().T for h in range(8)], 1).amax(-1) * sm
    sure = two.values[..., 0] - two.values[..., 1] > 40 + 2 * (d + 8) * 2.0 ** -24 * big
    assert bool(sure.any()) and bool(out.isfinite().all())
    at = two.indices[..., 0]
    want = torch.stack([v[at[:, h], h // 4] for h in range(8)], 1)
    tol = want.abs() * (2.0 ** -11 + 2.0 ** -19 + EPS[dt]) * (1 + 2.0 ** -8) + n * math.exp(-40) * float(v.abs().max())
    assert bool(((out - want).abs() <= tol)[sure].all())


@pytest.mark.parametrize("d,n,rows,Hq,block", [(64, 200, 12, 1, 3), (64, 300, 48, 1, 4), (64, 300, 60, 1, 4), (64, 300, 130, 2, 4), (128, 260, 10, 1, 4),
                                              (128, 300, 60, 1, 4), (128, 300, 130, 1, 4), (128, 300, 130, 1, 3), (128, 300, 299, 1, 0)])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_rows_that_do_not_see_a_missing_page_stay_clean(d, n, rows, Hq, block, fmt):
    """Causal rows in front of a block without a page, in one tile with rows that see it: whatever the pool's first page holds."""
    dt = torch.float16
    cache = make_cache([n], Hkv=1, d=d, dtype=dt, fmt=fmt, page_tokens=64, seed=0, spare=40)
    table = cache.pages.table[0].tolist()
    assert 0 not in table                                 # nobody's: NaN codes, where the format has them
    q = torch.randn(rows, Hq, d, generator=torch.Generator().manual_seed(1)).to(dt)
    want, err = attention(q, sequence(cache, "k", 0, n), sequence(cache, "v", 0, n), causal=True)
    cache.pages.table[0, block] = -1
    out = sage.sage_attn_fwd_paged(q.to(DEV), cache, causal=True, max_len=n).double().cpu()
    clean = max(0, 64 * block - (n - rows + 1) + 1)       # row i sees n - rows + i + 1 tokens
    assert clean < rows and out[clean:].isnan().all()
    tol = err + EPS[dt] * (want.abs() + err) + 2.0 ** -24
    assert bool(((out - want).abs() <= tol)[:clean].all())


def test_a_chain_of_forks_in_one_call():
    """A slot that a call fills cannot be copied by the same call: the entry with that source is refused, the one that fills it is not."""
    pages, cache = empty(4, 1, 64, torch.float16, "int8", 64, 2)
    sage.sage_pages_reserve(pages, ints(70, 64), ints(0, 3))
    status, moves, slot_moves = sage.sage_pages_fork(pages, ints(0, 1, 3), ints(1, 2, 2))
    assert status.tolist() == [0, -1, -1]                 # (the last one's destination is listed before)
    assert slot_moves.tolist() == [[0, 1], [-1, -1], [-1, -1]] and moves[1:].tolist() == [[-1, -1], [-1, -1]]
    assert pages.lens.tolist() == [70, 70, 0, 64] and pages.table[2].tolist() == [-1, -1]
    # a slot that is not empty is not filled, and its name as a destination still bars it as a source
    status, _, _ = sage.sage_pages_fork(pages, ints(0, 1), ints(1, 2))
    assert status.tolist() == [-1, -1]


# ---- sizes at which the kernels change their ways -----------------------------------------------------------------------

@pytest.mark.parametrize("ranges", [17, 20, 32, 33, 257, 300])
@pytest.mark.parametrize("d,rows", [(64, 1), (128, 3)])
def test_many_ranges(ranges, d, rows):
    # up to 32 ranges are combined by each thread, more by the row's threads together, 256 at a time
    run_case([64 * ranges - 5, 64, 130], [rows, 1, 1], Hq=2, Hkv=1, d=d, dtype="bf16", fmt="int8", page=256, causal=True, seed=ranges, split=64)


@pytest.mark.parametrize("n_pages,n", [(3000, 1500), (9000, 4096), (40000, 4096)])
def test_lists_and_tables_of_the_largest_size(n_pages, n):
    g = torch.Generator().manual_seed(n)
    slots, width = 4096, 12
    pages = sage.PageTable.empty(n_pages, page_tokens=64, slots=slots, width=width, device=DEV)
    sim = Table(pages)
    perm = lambda k: torch.randperm(slots, generator=g)[:k].tolist()  # noqa: E731
    s, m = perm(slots // 2), torch.randint(0, 200, (slots // 2,), generator=g).tolist()
    assert sage.sage_pages_reserve(pages, ints(*m), ints(*s)).tolist() == sim.reserve(s, m)
    sim.same(pages)
    # sources with and without tokens, destinations of which some are in use or listed twice
    src, dst = torch.randint(0, slots, (n,), generator=g).tolist(), perm(n) if n < slots else torch.randint(0, slots, (n,), generator=g).tolist()
    dst = [-1 if i % 3 else t for i, t in enumerate(dst)] if n == slots else dst
    status, pm, sm = sage.sage_pages_fork(pages, ints(*src), ints(*dst))
    want = sim.fork(src, dst)
    assert (status.tolist(), pm.tolist(), sm.tolist()) == want and 0 in want[0] and -1 in want[0]
    sim.same(pages)
    s, m = perm(n) if n < slots else perm(slots), torch.randint(0, 300, (n,), generator=g).tolist()
    assert sage.sage_pages_reserve(pages, ints(*m), ints(*s)).tolist() == sim.reserve(s, m)
    sim.same(pages)
    assert sage.sage_pages_reserve(pages).tolist() == sim.reserve(list(range(slots)), [1] * slots)
    gone = perm(slots)[:3000]
    sage.sage_pages_free(pages, ints(*gone))
    sim.free(gone)
    moves, counts = sage.sage_pages_compact(pages, n_pages // 2)
    assert (moves.tolist(), counts.tolist()) == sim.compact(n_pages // 2)
    sim.same(pages)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling,magnitude", [("yarn", 0.0), ("none", 0.5)])
def test_an_append_with_a_magnitude(layout, scaling, magnitude):
    d, Hkv, dt, n = 128, 2, torch.bfloat16, 150
    pages, cache = empty(1, Hkv, d, dt, "int8", 128, 2)
    plan = sage.rope_plan(96, layout=layout, scaling=scaling, factor=8.0, trained_len=64, magnitude=magnitude)
    assert plan.magnitude != 1.0
    k, v = (torch.randn(n, Hkv, d, device=DEV).to(dt) for _ in "kv")
    for a, b in ((0, 70), (70, 71), (71, n)):
        sage.sage_pages_reserve(pages, ints(b - a))
        sage.sage_paged_append(cache, k[a:b], v[a:b], rope=plan)
    check_blocks(cache, 0, {"k": sage.sage_rope(k, torch.arange(n, dtype=torch.int32, device=DEV), plan).cpu(), "v": v.cpu()})
