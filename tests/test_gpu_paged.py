"""The paged cache on the GPU: rows in and out bit by bit, attention against
float64 within what the kernel rounds (oracle/paged_oracle.py), and a prompt's
way from rotary positions to a compression."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_24467_gb300 as ckv
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
NAN = float("nan")


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def make(lengths, heads, page, dtype=BF, layout="head", extra=3, slack=1, fill=NAN, seed=0):
    """A cache of a shuffled pool, its slots behind the lengths (and its spare
    pages) filled with `fill`; unused table entries are outside the pool."""
    gen = torch.Generator().manual_seed(seed)
    used = [-(-max(n, 0) // page) for n in lengths]
    pool = sum(used) + extra
    order = torch.randperm(pool, generator=gen)
    table = torch.full((len(lengths), max(max(used), 1) + slack), -7, dtype=torch.int32)
    at = 0
    for s, u in enumerate(used):
        table[s, :u] = order[at:at + u].int()
        at += u
    kv = []
    for value in (False, True):
        x = torch.full((pool, page, heads, 128), fill, dtype=dtype)
        for s, n in enumerate(lengths):
            if n > 0:
                slot = torch.arange(n)
                x[table[s, slot // page].long(), slot % page] = (
                    torch.randn((n, heads, 128), generator=gen) * (0.5 if value else 1.0)).to(dtype)
        x = x.cuda()
        kv.append(x if layout == "token" else x.transpose(1, 2).contiguous().transpose(1, 2))
    return ckv.PagedCache(*kv, table.cuda(), ints(lengths))


def packed(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def queries(n, hq, dtype, seed=1, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn((n, hq, 128), generator=gen) * size).to(dtype).cuda()


def check(cache, q, out, lse, cu, start=None, causal=True, scale=128 ** -0.5, sequences=None):
    """Every sequence (or some) against the oracle."""
    cu = [int(x) for x in cu]
    for s in sequences if sequences is not None else range(cache.batch):
        n = cu[s + 1] - cu[s]
        if n == 0:
            continue
        length = max(int(cache.lengths[s]), 0)
        first = length - n if start is None else int(start[s])
        k, v = (po.rows_of(x, cache.table[s], 0, length) for x in (cache.k_pages, cache.v_pages))
        rows = slice(cu[s], cu[s + 1])
        want, want_lse, parts = po.attend(q[rows], k, v, first, causal, scale)
        tol, ltol = po.tolerance(q.dtype, max(length, 1), want, want_lse, parts)
        off = (out[rows].double() - want).abs()
        assert (off <= tol).all(), (s, float((off / tol).max()), float(off.max()))
        got = lse[:, rows].double()
        seen = torch.isfinite(want_lse)
        assert torch.equal(seen, torch.isfinite(got)) and (got[~seen] == -float("inf")).all()
        assert ((got - want_lse)[seen].abs() <= ltol[seen]).all()


def attend(cache, q, cu=None, start=None, causal=True, ws=None, **kw):
    most = int(np.diff(cu).max()) if cu is not None else q.shape[0] // cache.batch
    ws = ckv.paged_workspace(cache, q.shape[1], most) if ws is None else ws
    out = torch.full_like(q, 7.0)
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    ckv.paged_attend(cache, q, out, ws, cu_rows=cu, start=start, lse=lse, causal=causal, **kw)
    torch.cuda.synchronize()
    status = ckv.read_device_status(ws)
    if status == 0:  # every row is written
        assert not (out == 7).all(-1).any() and not (lse == 7).any()
    return out, lse, status


def run(lengths, rows, hq, h, page=64, dtype=BF, layout="head", start=None, causal=True, seed=0):
    cache = make(lengths, h, page, dtype, layout, seed=seed)
    cu = packed(rows)
    q = queries(int(cu[-1]), hq, dtype, seed + 1)
    first = None if start is None else ints(start)
    out, lse, status = attend(cache, q, cu, first, causal)
    assert status == 0
    check(cache, q, out, lse, cu, first, causal)
    return cache, q, out, lse


# ------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("dtype, page, layout, given", [(BF, 16, "head", False), (HF, 32, "token", True),
                                                        (BF, 128, "head", True), (HF, 256, "token", False)])
@pytest.mark.parametrize("rows", [[1, 1, 1], [0, 3, 17], [16, 2, 0], [300, 1, 40]])
def test_append_and_gather(rows, dtype, page, layout, given):
    h, hq = 3, 6
    before = [5, 0, 2 * page - 1]
    after = [a + b for a, b in zip(before, rows)]
    cache = make(after, h, page, dtype, layout, fill=3.0)
    cache.lengths.copy_(ints(before))
    k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
    cu = packed(rows)
    n = int(cu[-1])
    k, v, q = queries(n, h, dtype, 1), queries(n, h, dtype, 2), queries(n, hq, dtype, 3)
    rope = ckv.Rope(128, interleaved=layout == "token")
    start = ints(before) if given else None
    q_out = torch.empty_like(q)
    status = ints([0])
    ckv.paged_append(cache, k, v, cu, start=start, rope=rope, q=q, q_out=q_out, device_status=status)
    slots = torch.cat([torch.arange(b, a) for b, a in zip(before, after)]).int().cuda()
    turned = [torch.empty_like(x) for x in (q, k)]
    if n:
        ckv.rope_apply(rope, slots, q, k, *turned)
    assert torch.equal(q_out, turned[0]) and int(status) == 0
    assert cache.lengths.tolist() == after
    for s in range(3):
        at, where = slots[cu[s]:cu[s + 1]].long(), slice(cu[s], cu[s + 1])
        pages = cache.table[s].long()[at // page]
        k0[pages, at % page], v0[pages, at % page] = turned[1][where], v[where]
    assert torch.equal(cache.k_pages, k0) and torch.equal(cache.v_pages, v0)  # and nothing else
    all_cu = packed(after)
    ko = torch.full((int(all_cu[-1]), h, 128), 9.0, dtype=dtype, device="cuda")
    vo = ko.clone()
    ckv.paged_gather(cache, ko, vo, all_cu, device_status=status)
    for s in range(3):
        where = slice(all_cu[s], all_cu[s + 1])
        assert torch.equal(ko[where], po.rows_of(cache.k_pages, cache.table[s], 0, after[s]))
        assert torch.equal(vo[where], po.rows_of(cache.v_pages, cache.table[s], 0, after[s]))
    assert int(status) == 0
    # the new rows alone, K alone
    if n:
        back = torch.empty_like(k)
        ckv.paged_gather(cache, back, None, cu, start=ints(before))
        assert torch.equal(back, turned[1])


def test_append_without_rope_and_with_positions():
    cache = make([40, 40], 2, 16, fill=0.0)
    k, v, q = queries(6, 2, BF, 1), queries(6, 2, BF, 2), queries(6, 4, BF, 3)
    ckv.paged_append(cache, k, v, start=ints([7, 30]))
    assert cache.lengths.tolist() == [10, 33]
    got = po.rows_of(cache.k_pages, cache.table[1], 30, 3)
    assert torch.equal(got, k[3:])
    rope, pos = ckv.Rope(64), ints([9, -4, 100000, 0, 5, 2 ** 31 - 1])
    wk, wq = torch.empty_like(k), torch.empty_like(q)
    ckv.rope_apply(rope, pos, q, k, wq, wk)
    ckv.paged_append(cache, k, v, start=ints([7, 30]), rope=rope, positions=pos, q=q)  # q in place
    assert torch.equal(q, wq) and torch.equal(po.rows_of(cache.k_pages, cache.table[0], 7, 3), wk[:3])
    # strided rows: K and V inside one projection
    qkv = queries(6, 8, BF, 4)
    ckv.paged_append(cache, qkv[:, 4:6], qkv[:, 6:], start=ints([1, 1]))
    assert torch.equal(po.rows_of(cache.v_pages, cache.table[1], 1, 3), qkv[3:, 6:])


@pytest.mark.parametrize("rows", [2, 40])
@pytest.mark.parametrize("given", [False, True])
def test_append_where_there_is_no_room(rows, given):
    """Absent sequences, pages outside the pool and the table's end."""
    page, h = 16, 2
    cache = make([64] * 4, h, page, slack=0, fill=0.0)
    cache.table[2, 1] = cache.num_pages
    first = [-1, 63, 15, 70]
    cache.lengths.copy_(ints(first))
    k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
    k, v = queries(4 * rows, h, BF, 1), queries(4 * rows, h, BF, 2)
    q = queries(4 * rows, 1, BF, 3)
    q_out = torch.full_like(q, 7.0)
    status = ints([0])
    ckv.paged_append(cache, k, v, start=ints(first) if given else None, rope=ckv.Rope(2), q=q, q_out=q_out,
                     device_status=status)
    assert int(status) == -8
    assert cache.lengths.tolist() == [-1, 64, min(15 + rows, 64), 64]
    pages = cache.table.long()
    for s in (1, 2):
        for i in range(rows):
            at = first[s] + i
            if at < 64 and not (s == 2 and at // page == 1):
                x = torch.empty(1, h, 128, dtype=BF, device="cuda")
                ckv.rope_apply(ckv.Rope(2), ints([at]), k[s * rows + i:s * rows + i + 1], k_out=None, q_out=x)
                k0[pages[s, at // page], at % page], v0[pages[s, at // page], at % page] = x[0], v[s * rows + i]
    assert torch.equal(cache.k_pages, k0) and torch.equal(cache.v_pages, v0)
    assert (q_out[:rows] == 7).all() and not (q_out[rows:] == 7).all(-1).any()


def test_gather_leaves_what_is_not_there():
    cache = make([20, 33, 5], 2, 16, fill=0.0)
    cache.table[1, 0] = -1
    cache.lengths[2] = -3
    out = torch.full((3 * 25, 2, 128), 9.0, dtype=BF, device="cuda")
    status = ints([0])
    ckv.paged_gather(cache, out, None, start=ints([0, 10, 0]), device_status=status)
    assert int(status) == -8
    assert torch.equal(out[:20], po.rows_of(cache.k_pages, cache.table[0], 0, 20)) and (out[20:25] == 9).all()
    assert (out[25:31] == 9).all()
    assert torch.equal(out[31:48], po.rows_of(cache.k_pages, cache.table[1], 16, 17)) and (out[48:] == 9).all()
    status.zero_()
    ckv.paged_gather(cache, out[:50], out[:50].clone(), [0, 0, 0, 50], device_status=status)
    assert int(status) == 0  # a sequence that is not there is no error


# ----------------------------------------------------------------- attention
@pytest.mark.parametrize("hq, h", [(32, 8), (28, 4), (64, 8), (5, 5), (9, 1), (128, 1)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_single_tokens(hq, h, dtype):
    run([777, 1, 64, 129, 2000], [1] * 5, hq, h, dtype=dtype, page=32, seed=hq)


@pytest.mark.parametrize("page, layout", [(16, "head"), (32, "token"), (64, "head"), (128, "token"), (256, "head")])
def test_pages(page, layout):
    run([1000, 127, 256, 257], [1, 9, 33, 130], 16, 4, page, HF, layout, seed=page)
    run([300, 15], [300, 15], 8, 2, page, BF, layout, seed=page)


@pytest.mark.parametrize("rows", [2, 3, 16, 17, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 200])
def test_chunk_sizes(rows):
    run([rows, rows + 1, rows + 127, 1024 + rows], [rows] * 4, 8, 2, seed=rows)


@pytest.mark.parametrize("hq, h", [(7, 1), (28, 4), (3, 3), (20, 2), (33, 1), (100, 1), (64, 8)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_group_sizes(hq, h, dtype):
    run([150, 40, 391], [150, 1, 70], hq, h, 16, dtype, seed=hq)


def test_ragged_with_empty_sequences():
    run([0, 5, 300, 129, 0, 77], [0, 5, 0, 100, 0, 1], 8, 2)
    run([500, 0, 300], [0, 0, 20], 8, 2)


def test_not_causal_and_given_starts():
    run([300, 40], [5, 70], 8, 2, causal=False)
    run([300, 40, 200], [5, 70, 2], 8, 2, start=[100, 0, 1000])
    run([300, 400], [130, 66], 4, 1, start=[-100, 390])


def test_tokens_that_see_nothing():
    """Chunks longer than what is in use, lengths of zero and below, absent ones."""
    _, _, out, lse = run([3, 0, 130], [10, 4, 200], 8, 2)
    assert (out[:7] == 0).all() and (out[10:14] == 0).all() and torch.isinf(lse[:, 14:84]).all()
    cache = make([50, 60], 2, 16)
    cache.lengths[0] = -5
    q = queries(6, 4, BF)
    out, lse, status = attend(cache, q)
    assert status == 0 and (out[:3] == 0).all() and (lse[:, :3] == -float("inf")).all()
    check(cache, q, out, lse, [0, 3, 6], sequences=[1])


@pytest.mark.parametrize("rows, length", [(1, 300), (6, 300), (90, 300), (90, 9000), (300, 9000), (130, 131)])
def test_what_is_not_seen_leaves_no_trace(rows, length):
    """Infinities and NaN in slots that a token does not see: of the chunk's later
    tokens, and behind the length (where make() puts NaN); in those that it sees
    they reach every channel that they are in."""
    h, hq, page = 2, 8, 32
    cache = make([length], h, page)
    q = queries(rows, hq, BF)
    clean, clean_lse, _ = attend(cache, q)
    bad = length - max(rows // 2, 1)  # seen by the tokens from slot `bad` on

    def put(pages, slot, head, channel, value):
        pages[cache.table[0, slot // page].long(), slot % page, head, channel] = value

    for value in (NAN, float("inf"), -float("inf")):
        k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
        put(cache.v_pages, bad, 0, 5, value)
        put(cache.v_pages, bad, 0, 100, value)
        out, lse, _ = attend(cache, q)
        first = bad - (length - rows)  # the first token that sees it
        assert torch.equal(out[:first], clean[:first]) and torch.equal(lse, clean_lse)
        hit = out[first:, :4]
        want = torch.full_like(hit[..., 5], value)
        assert torch.equal(torch.isnan(hit[..., 5]), torch.isnan(want))
        assert np.isnan(value) or (torch.equal(hit[..., 5], want) and torch.equal(hit[..., 100], want))
        others = [c for c in range(128) if c not in (5, 100)]
        assert torch.equal(hit[..., others], clean[first:, :4][..., others])
        assert torch.equal(out[:, 4:], clean[:, 4:])  # the other KV head
        cache.v_pages.copy_(v0)
        put(cache.k_pages, bad, 1, 7, NAN if not np.isnan(value) else value)
        out, lse, _ = attend(cache, q)
        assert torch.equal(out[:first], clean[:first]) and torch.equal(lse[:, :first], clean_lse[:, :first])
        assert torch.isnan(out[first:, 4:]).all() and torch.isnan(lse[4:, first:]).all()
        assert torch.equal(out[:, :4], clean[:, :4])
        cache.k_pages.copy_(k0)
    q2 = q.clone()
    q2[rows - 1, 3] = NAN  # one row of one token
    out, lse, _ = attend(cache, q2)
    assert torch.isnan(out[rows - 1, 3]).all() and torch.isnan(lse[3, rows - 1])
    out[rows - 1, 3] = clean[rows - 1, 3]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_growing_and_extreme_logits(dtype):
    """Logits that rise through the slots raise the reference again and again;
    huge ones put all weight on one slot; a scale of its own."""
    cache = make([2000], 1, 64, dtype)
    ramp = torch.linspace(0.0, 6.0, 2000, device="cuda")
    slot = torch.arange(2000, device="cuda")
    pages = cache.table[0].long()[slot // 64]
    cache.k_pages[pages, slot % 64] *= ramp[:, None, None].to(dtype)
    for size in (1.0, 8.0):
        for rows in (1, 70):
            q = queries(rows, 4, dtype, size=size)
            out, lse, _ = attend(cache, q)
            check(cache, q, out, lse, [0, rows])
            out, lse, _ = attend(cache, q, scale=0.5)
            check(cache, q, out, lse, [0, rows], scale=0.5)
    # one sign: every logit far below zero, or far above
    cache.k_pages[pages, slot % 64] = cache.k_pages[pages, slot % 64].abs()
    for sign in (1, -1):
        q = queries(70, 4, dtype).abs() * sign
        out, lse, _ = attend(cache, q)
        check(cache, q, out, lse, [0, 70])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("length, rows", [(700, 1), (40000, 1), (9000, 200)])
def test_values_near_the_largest_number(dtype, length, rows):
    """Averages of values near the type's largest number are finite, whatever the sum
    of their weights; small ones are kept (bf16: down to 2^(8 - 126) times the length,
    rounded up to a power of two)."""
    cache = make([length], 1, 64, dtype)
    slot = torch.arange(length, device="cuda")
    pages = cache.table[0].long()[slot // 64]
    v = cache.v_pages[pages, slot % 64]
    q = queries(rows, 4, dtype)
    least = 2.0 ** -90 if dtype == BF else torch.finfo(dtype).smallest_normal * 64
    for size in (torch.finfo(dtype).max / 4, least):
        cache.v_pages[pages, slot % 64] = (v.double().clamp(-1, 1).abs() * size).to(dtype)
        out, lse, _ = attend(cache, q)
        assert torch.isfinite(out).all()
        check(cache, q, out, lse, [0, rows])


def test_long_contexts_and_many_pieces():
    """Slots beyond 64K, shared by many CTAs; a chunk over a long context."""
    for lengths, rows, hq, h in (([70000], [1], 4, 1), ([70001, 300], [3, 1], 8, 2), ([40000], [40], 8, 1),
                                 ([33333, 20], [70, 20], 8, 2)):
        cache = make(lengths, h, 256, HF, fill=0.0)
        cu = packed(rows)
        q = queries(int(cu[-1]), hq, HF)
        out, lse, status = attend(cache, q, cu)
        assert status == 0
        check(cache, q, out, lse, cu)


def test_chunks_in_pieces_whose_tiles_see_different_blocks():
    """One head a group: the second 128 rows see a block of slots more; starts that
    are not the newest slots; many short sequences beside a long one."""
    run([20000], [260], 1, 1, 128, BF)
    run([20000, 9000], [260, 200], 2, 2, 64, HF)
    run([30000], [300], 4, 1, start=[-200])
    run([30000], [300], 4, 1, start=[20000])
    run([30000, 40], [300, 0], 4, 1, causal=False)
    cache, q, out, lse = run([9000] + [150] * 20, [200] + [100] * 20, 8, 2)
    run([9000] + [150] * 20, [1] + [100] * 20, 8, 2)


@pytest.mark.parametrize("lengths, rows, hq, h, start, causal", [
    ([60000], [140], 4, 1, None, True),                        # three items, each in some fifty pieces
    ([20000, 300, 40, 5000], [200, 150, 0, 129], 7, 1, None, True),
    ([9000, 9000, 9000], [300, 300, 300], 4, 2, [-200, 9000, 100], True),
    ([9000, 1000], [300, 200], 4, 4, None, False),
    ([700] * 40, [300] * 40, 8, 4, None, True),                # items that are whole, and few tiles
    ([3000] * 10, [256] * 10, 32, 8, None, True),              # alike: two rounds, and 16 items in runs
    ([2000] * 9 + [1, 300] * 20, [400] * 9 + [1, 130] * 20, 16, 4, None, True),
    ([130] * 70, [129] * 70, 2, 2, None, True),                # three lanes' worth of sequences, a tile or two each
])
def test_chunks_in_runs_and_in_whole_items(lengths, rows, hq, h, start, causal):
    """What is cut into runs, where runs end, and how many share an item."""
    dtype = BF if len(lengths) % 2 else HF
    cache = make(lengths, h, 64, dtype)
    cu = packed(rows)
    q = queries(int(cu[-1]), hq, dtype)
    first = None if start is None else ints(start)
    ws = ckv.paged_workspace(cache, hq, max(rows))
    out, lse, status = attend(cache, q, cu, first, causal, ws=ws)
    assert status == 0
    check(cache, q, out, lse, cu, first, causal, sequences=range(0, len(lengths), 1 + len(lengths) // 12))
    again, lse2, status = attend(cache, q, cu, first, causal, ws=ws)
    assert status == 0 and torch.equal(out, again) and torch.equal(lse, lse2)


def test_a_whole_prompt():
    run([3000], [3000], 4, 1, 128, BF)


def test_many_sequences():
    gen = np.random.default_rng(0)
    lengths = gen.integers(1, 400, 512).tolist()
    cache = make(lengths, 2, 16, BF)
    q = queries(512, 8, BF)
    out, lse, _ = attend(cache, q)
    check(cache, q, out, lse, range(513), sequences=range(0, 512, 37))
    rows = [min(n, int(r)) for n, r in zip(lengths, gen.integers(0, 40, 512))]
    cu = packed(rows)
    q = queries(int(cu[-1]), 8, BF)
    out, lse, _ = attend(cache, q, cu)
    check(cache, q, out, lse, cu, sequences=range(0, 512, 37))


@pytest.mark.parametrize("seed", range(6))
def test_random_batches_of_chunks(seed):
    """Batches of up to a hundred sequences, some of them long, some with one token:
    what CTAs share, and how the last items are cut, differ from case to case."""
    gen = np.random.default_rng(seed)
    b = int(gen.integers(1, 100))
    most = int(4000 / b) + 10
    rows = gen.integers(0, most, b)
    rows[gen.random(b) < 0.3] = 1
    rows[0] += 200
    lengths = rows + (gen.random(b) ** 6 * 20000).astype(int)
    hq, h = [(8, 2), (6, 1), (4, 4), (14, 2), (16, 2), (3, 1)][seed]
    cache = make(lengths.tolist(), h, [16, 32, 64, 128, 256, 64][seed], [BF, HF][seed % 2], seed=seed)
    cu = packed(rows)
    q = queries(int(cu[-1]), hq, [BF, HF][seed % 2], seed)
    out, lse, status = attend(cache, q, cu)
    assert status == 0
    check(cache, q, out, lse, cu, sequences=sorted({0, b - 1, *gen.integers(0, b, 6).tolist()}))


def test_strided_queries_and_outputs():
    cache = make([300, 200], 2, 32)
    qkv = queries(40, 8 + 4, BF)
    ws = ckv.paged_workspace(cache, 8, 20)
    wide = torch.full((40, 8, 264), 7.0, dtype=BF, device="cuda")
    lse = torch.empty(8, 40, device="cuda")
    ckv.paged_attend(cache, qkv[:, 2:10], wide[..., 8:136], ws, lse=lse)
    check(cache, qkv[:, 2:10], wide[..., 8:136], lse, [0, 20, 40])
    assert (wide[..., :8] == 7).all() and (wide[..., 136:] == 7).all()
    by_head = queries(8, 40, BF).transpose(0, 1)
    out = torch.empty(8, 40, 128, dtype=BF, device="cuda").transpose(0, 1)
    ckv.paged_attend(cache, by_head, out, ws, lse=lse)
    check(cache, by_head, out, lse, [0, 20, 40])
    same = torch.empty_like(out)
    ckv.paged_attend(cache, by_head, same, ws)  # without the log-sum-exp
    assert torch.equal(same, out)


def test_pages_outside_the_pool_count_as_zeros():
    for rows in (1, 50):
        cache = make([200], 2, 16)
        cache.table[0, 3], cache.table[0, 7] = cache.num_pages, -1
        q = queries(rows, 8, BF)
        out, lse, status = attend(cache, q)
        assert status == -8
        check(cache, q, out, lse, [0, rows])


def test_shared_pages_and_parts_of_a_cache():
    """Sequences with a prefix in common; some sequences of a cache; a table that is
    wider than it is used; a pool of one page."""
    page, h = 32, 2
    cache = make([200, 180, 90], h, page, slack=4)
    cache.table[1, :2] = cache.table[0, :2]
    for rows in (1, 60):
        q = queries(3 * rows, 8, BF)
        out, lse, _ = attend(cache, q)
        check(cache, q, out, lse, packed([rows] * 3))
        part = cache.sequences(1, 2)
        out2, lse2, _ = attend(part, q[rows:])
        assert torch.equal(out2, out[rows:]) and torch.equal(lse2, lse[:, rows:])
    narrow = ckv.PagedCache(cache.k_pages, cache.v_pages, cache.table[:, :7], cache.lengths)
    out3, _, _ = attend(narrow, q)
    assert torch.equal(out3, out)
    one = make([17], 1, 64, extra=0, slack=0)
    assert one.num_pages == 1
    for rows in (1, 17):
        q = queries(rows, 3, BF)
        out, lse, _ = attend(one, q)
        check(one, q, out, lse, [0, rows])


@pytest.mark.parametrize("n", [8, 64])
def test_on_a_share_of_the_sms(n):
    from test_gpu_shared_sms import GreenStream

    try:
        green = GreenStream(n)
    except (OSError, AttributeError, RuntimeError) as e:
        pytest.skip(f"no green contexts here: {e}")
    for lengths, rows in (([9000, 300], [1, 1]), ([6000, 300], [150, 40])):
        cache = make(lengths, 2, 64, fill=0.0)
        cu = packed(rows)
        q = queries(int(cu[-1]), 8, BF)
        ws = ckv.paged_workspace(cache, 8, max(rows))
        torch.cuda.synchronize()
        out, lse, status = attend(cache, q, cu, ws=ws, stream=green.stream)
        assert status == 0
        check(cache, q, out, lse, cu)


@pytest.mark.parametrize("lengths, rows", [([777], [1]), ([30000, 5000], [1, 1]), ([300, 200], [300, 130]),
                                           ([9000], [200])])
def test_a_wait_that_runs_out(lengths, rows):
    """A hook makes a CTA wait for what nothing completes: the call ends, the context
    stays usable, later calls do nothing until the workspace is set up again."""
    cache = make(lengths, 2, 64, fill=0.0)
    cu = packed(rows)
    q = queries(int(cu[-1]), 8, BF)
    ws = ckv.paged_workspace(cache, 8, max(rows))
    want, want_lse, _ = attend(cache, q, cu, ws=ws)
    ckv.debug_stall_next_paged_attend(2_000_000)
    _, _, status = attend(cache, q, cu, ws=ws)
    assert status == -7
    out, _, status = attend(cache, q, cu, ws=ws)
    assert status == -7 and (out == 7).all()
    assert ckv.load().compresskv_paged_workspace_init(ws.data_ptr(), ws.numel(), None) == 0
    for _ in range(2):
        out, lse, status = attend(cache, q, cu, ws=ws)
        assert status == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


def test_two_calls_give_the_same_bits():
    for lengths, rows in (([30000, 7], [1, 1]), ([5000, 900, 33], [100, 64, 33]), ([2500], [2500])):
        cache = make(lengths, 2, 64, fill=0.0)
        cu = packed(rows)
        q = queries(int(cu[-1]), 8, BF)
        ws = ckv.paged_workspace(cache, 8, max(rows))
        a, la, _ = attend(cache, q, cu, ws=ws)
        for _ in range(3):
            b, lb, status = attend(cache, q, cu, ws=ws)
            assert torch.equal(a, b) and torch.equal(la, lb) and status == 0


def test_a_workspace_serves_smaller_calls():
    cache = make([5000, 700], 2, 64)
    ws = ckv.paged_workspace(cache, 16, 300)
    for rows, hq in (([300, 300], 16), ([1, 1], 8), ([3, 250], 4), ([1, 1], 16), ([300, 0], 2)):
        cu = packed(rows)
        q = queries(int(cu[-1]), hq, BF)
        out, lse, status = attend(cache, q, cu, ws=ws)
        assert status == 0
        check(cache, q, out, lse, cu)


@pytest.mark.parametrize("rows", [1, 3, 80])
def test_captured_steps_follow_the_lengths(rows):
    """append and attend in one graph, replayed while the sequences grow."""
    h, hq, page = 2, 8, 16
    cache = make([1000, 1000, 1000], h, page, fill=0.0)
    cache.lengths.copy_(ints([0, 500, 130]))
    n = 3 * rows
    k, v, q = queries(n, h, BF, 1), queries(n, h, BF, 2), queries(n, hq, BF, 3)
    rope = ckv.Rope(128)
    ws = ckv.paged_workspace(cache, hq, rows)
    turned, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(hq, n, device="cuda")

    def step():
        ckv.paged_append(cache, k, v, rope=rope, q=q, q_out=turned)
        ckv.paged_attend(cache, turned, out, ws, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for x in (k, v, q):
            x.copy_(queries(n, x.shape[1], BF, 10 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert cache.lengths.tolist() == [a + (i + 2) * rows for a in (0, 500, 130)]
        check(cache, turned, out, lse, packed([rows] * 3))
    assert ckv.read_device_status(ws) == 0


def test_two_streams_with_workspaces_of_their_own():
    caches = [make([20000, 50], 2, 64, fill=0.0, seed=s) for s in (0, 1)]
    qs = [queries(2 * 70, 8, BF, s) for s in (5, 6)]
    wss = [ckv.paged_workspace(c, 8, 70) for c in caches]
    want = [attend(c, q, ws=w)[:2] for c, q, w in zip(caches, qs, wss)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(10)] for q in qs]
    torch.cuda.synchronize()
    for i in range(10):
        for j, st in enumerate(streams):
            ckv.paged_attend(caches[j], qs[j], outs[j][i], wss[j], stream=st)
    torch.cuda.synchronize()
    for j in range(2):
        assert all(torch.equal(o, want[j][0]) for o in outs[j])
        assert ckv.read_device_status(wss[j]) == 0


def test_pools_beyond_four_gigabytes():
    """Offsets that pass 32 bits, in bytes and in elements."""
    h, page = 8, 256
    pages = (5 << 30) // (page * h * 128 * 2) * 2  # 10 GiB: over 2^32 elements
    pool = torch.zeros((pages, h, page, 128), dtype=BF, device="cuda").transpose(1, 2)
    table = ints([pages - 1, 0, pages // 2, pages - 2]).view(1, 4)
    cache = ckv.PagedCache(pool, pool, table, ints([0]))
    k = queries(1000, h, BF, 1)
    ckv.paged_append(cache, k, k)  # (K and V share their memory: the same rows)
    back = torch.empty_like(k)
    ckv.paged_gather(cache, back)
    assert torch.equal(back, k)
    for rows in (1, 40):
        q = queries(rows, 16, BF)
        out, lse, status = attend(cache, q)
        assert status == 0
        check(cache, q, out, lse, [0, rows])


def test_traces_count_launches():
    cache = make([100], 2, 16, fill=0.0)
    trace = ckv.Trace(8)
    cache = ckv.PagedCache(cache.k_pages, cache.v_pages, cache.table, cache.lengths, trace)
    k, q = queries(1, 2, BF), queries(1, 4, BF)
    ckv.paged_append(cache, k, k, start=ints([99]))
    ckv.paged_gather(cache, torch.empty_like(k))
    attend(cache, q)
    kinds = [k for k, _ in trace.records()]
    assert kinds[:2] == ["paged_write", "paged_gather"] and set(kinds[2:]) == {"paged_attend"}


# ------------------------------------------------------------------ together
def test_from_rotary_positions_to_a_compression():
    """A prompt prefilled in chunks over pages: its last window's log-sum-exp and
    its rows, packed again, give the compression that float64 gives, and the
    4-bit cache decodes over it."""
    L, W, hq, h, page = 1500, 32, 8, 2, 32
    gen = torch.Generator().manual_seed(0)
    q, k, v = ((torch.randn((L, n, 128), generator=gen) * s).to(BF).cuda() for n, s in ((hq, 1.0), (h, 1.0), (h, 0.5)))
    rope = ckv.Rope(128, base=500000.0)
    cache = ckv.paged_cache(1, h, L, page)
    ws = ckv.paged_workspace(cache, hq, 700)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    lse = None
    for a, b in ((0, 700), (700, 1399), (1399, 1400), (1400, L)):
        ckv.paged_append(cache, k[a:b], v[a:b], rope=rope, q=q[a:b], q_out=turned[a:b])
        lse = torch.empty((hq, b - a), device="cuda")
        ckv.paged_attend(cache, turned[a:b], out[a:b], ws, lse=lse)
    assert cache.lengths.tolist() == [L]
    rotated = [torch.empty_like(x) for x in (q, k)]
    ckv.rope_apply(rope, torch.arange(L, dtype=torch.int32, device="cuda"), q, k, *rotated)
    assert torch.equal(turned, rotated[0])
    want, _, parts = po.attend(turned, rotated[1], v, 0, True, 128 ** -0.5)
    tol, _ = po.tolerance(BF, L, want, torch.zeros(hq, L, device="cuda"), parts)
    assert ((out.double() - want).abs() <= tol).all()
    kp, vp = torch.empty_like(k), torch.empty_like(v)
    ckv.paged_gather(cache, kp, vp)
    assert torch.equal(kp, rotated[1]) and torch.equal(vp, v)
    q_win = turned[-W:].transpose(0, 1)[None]          # [1, Hq, W, 128]
    lse_win = lse[None, :, -W:]                         # the chunk's last W tokens
    problem = ckv.Problem(q_win, kp, [0, L], W, 7)
    budgets, mask = [200], np.array([1, 0, 1, 0, 0, 1, 0, 0], np.uint8)
    res = ckv.LayerOutputs(problem, budgets, 128, BF, "cuda")
    cws = ckv.workspace(problem)
    cu_out = ckv.compress_layer_lse(problem, q_win, kp, vp, lse_win, mask, budgets, res.indices, res.k_out,
                                    res.v_out, cws, raw=res.raw, pooled=res.pooled)
    torch.cuda.synchronize()
    ref = oracle.compress_layer(q_win.float().cpu().numpy(), kp.float().cpu().numpy(), vp.float().cpu().numpy(),
                                np.array([0, L]), mask, np.array(budgets), W, 7)
    from oracle import compare

    compare.check_layer(ref, res.raw.cpu().numpy(), res.pooled.cpu().numpy(), res.indices.cpu().numpy(),
                        np.array([0, L]), W)
    q4 = ckv.q4_cache(1, h, 256)
    ckv.q4_gather(problem, q4, res.indices, cu_out, kp, vp, raw=res.raw)
    q4_ws = ckv.q4_workspace(q4, hq, 1)
    one = turned[-1:].view(1, hq, 1, 128).contiguous()
    got = torch.empty_like(one)
    ckv.q4_attend(q4, one, got, q4_ws)
    torch.cuda.synchronize()
    assert torch.isfinite(got).all() and int(q4.lengths[0, 0]) == 200
