"""What the paged cache's calls do with values on the device that are out of range: offsets, lengths and page numbers
that no check on the host sees. Nothing is followed, the status word says so, and what is in range keeps its results."""
import numpy as np
import pytest
import torch

import paged
from paper_2609_32663_gb300 import dkv
from test_gpu_chunk import Call, inputs, lens_of
from test_gpu_pages import State, dev, plan_of, slot_map, tables_of

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.int16).clone()


@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cu", [
    [4, 6, 9, 79], [1, 1, 1, 1], [-2, 2, 5, 75], [0, 5, 2, 75], [0, 2, 5, 83], [0, 2, 5, 1 << 30], [0, -1, 5, 75],
    [0, 2, 75, 5], [0, 2, 5, -(1 << 31)],
])
def test_bad_token_offsets_change_nothing(cuda, cu, dtype, append):
    """Offsets that do not start at 0 (a slice of a larger batch's), descend or pass the rows of the call."""
    tokens = [2, 3, 70]
    cache = paged.Cache(lens_of(1, 3, 2, [98, 300, 131], tokens, 1), 16, H=8, dtype=dtype)
    good, qkv = inputs(cache, tokens, 3, pad=7)
    c = Call(cache, 0, qkv, cu, append=append)
    before = bits(c.Kp), bits(c.Vp), bits(c.out)
    c.run()
    assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
    for got, old in zip((c.Kp, c.Vp, c.out), before):
        assert torch.equal(bits(got), old)
    # The same buffers with offsets that hold.
    c.cu.copy_(torch.from_numpy(good))
    c.status.zero_()
    c.run()
    k, v = (qkv[1], qkv[2]) if append else (None, None)
    want, size, _, _ = paged.attention(cache, 0, qkv[0], k, v, good, True)
    assert int(c.status) == 0
    paged.assert_attention(c.out, want, size, dtype)


def test_bad_token_offsets_of_many_slots(cuda):
    """The pair that breaks the order lies behind the CTA's first 384 slots."""
    tokens = [1] * 512
    cache = paged.Cache(lens_of(1, 512, 1, [5] * 512, tokens, 1), 16, H=2)
    good, qkv = inputs(cache, tokens, 3)
    for at in (383, 384, 385, 511, 512):
        cu = good.copy()
        cu[at] += 600 if at == 512 else -2
        c = Call(cache, 0, qkv, cu)
        before = bits(c.Kp), bits(c.Vp), bits(c.out)
        c.run()
        assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
        for got, old in zip((c.Kp, c.Vp, c.out), before):
            assert torch.equal(bits(got), old)


@pytest.mark.parametrize("over", [1, 2, 3, 100, -1])
def test_a_length_out_of_range_counts_as_empty(cuda, over):
    """A slab whose length passes its table (or is negative): none of its rows is written or read, though some of the
    new tokens' places would lie in the table."""
    tokens = [2, 3, 2]
    cache = paged.Cache(lens_of(1, 3, 1, [40, 61, 60], tokens, 1), 16, H=4, wider=0)
    cap = cache.pages.max_pages * 16
    assert cache.lens[1] == cap
    cu, qkv = inputs(cache, tokens, 3)
    want, size, Kp, Vp = paged.attention(cache, 0, *qkv, cu, True)
    c = Call(cache, 0, qkv, cu)
    c.len[1] = cap + over if over > 0 else over
    before = bits(c.Kp), bits(c.Vp)
    c.run()
    assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
    mine = torch.from_numpy(cache.rows(1))
    for got, old in zip((c.Kp, c.Vp), before):
        assert torch.equal(bits(got)[mine], old[mine])
    assert not c.out[2:5].any()
    for t in (slice(0, 2), slice(5, 7)):
        paged.assert_attention(c.out[t], want[t], size[t], cache.dtype)
    for h in (0, 2):
        assert torch.equal(c.Kp.cpu()[cache.rows(h)].double(), Kp[cache.rows(h)])


def test_a_slab_shorter_than_its_new_tokens(cuda):
    """Tokens that the slab has no row for are skipped and reported, the others are placed."""
    tokens = [5, 1]
    cache = paged.Cache(np.array([[[3], [40]]]), 16, H=4)
    cu, qkv = inputs(cache, tokens, 3)
    c = Call(cache, 0, qkv, cu).run()
    assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
    Kp = cache.Kp.clone()
    Kp[cache.rows(0)] = qkv[1][2:5, 0]
    Kp[cache.rows(1)[-1]] = qkv[1][5, 0]
    assert torch.equal(bits(c.Kp.cpu()), bits(Kp))


BAD = [-1, 1 << 30, -(1 << 31), None]  # None: the number of pages, the first that is none


def spoil(a, at, pages):
    """The entries `at` of a table or list out of range; the array, and what the definition then has in it."""
    for i, x in enumerate(at):
        a[tuple(np.atleast_1d(x))] = pages if BAD[i % 4] is None else BAD[i % 4]


def none_out_of_range(a, pages):
    return np.where((a >= 0) & (a < pages), a, -1)


@pytest.mark.parametrize("V", [4, 1])
def test_tables_pass_no_bad_page_on(cuda, V):
    """Bad entries of the free list and of the tables' last pages: -1 in the new entries and in the slot map, all else as
    it would be."""
    r = np.random.default_rng(V)
    lens = r.integers(0, 90, (3, 5, 4 if V == 4 else 3))
    tokens = [20, 0, 1, 40, 7]
    n = np.broadcast_to(np.asarray(tokens)[None, :, None], lens.shape)
    need = int((-(-(lens + n) // 16) - -(-lens // 16)).sum())
    cache = paged.Cache(lens, 16, spare=need + 3, wider=4)
    pages = cache.pages.num_pages
    spoil(cache.free, [cache.count - 1, cache.count - 4, cache.count - need, 4], pages)
    some = [h for h in range(cache.lens.size) if cache.lens[h] % 16][:9]
    spoil(cache.table, [(h, cache.lens[h] // 16) for h in some], pages)
    s = State(cache)
    cap = sum(tokens) + 2
    cu, slots = dev(np.full(6, -9)), dev(np.full((3, cap, lens.shape[2]), -3))
    s.tables(tokens=dev(tokens), cu_tokens=cu, slots=slots)
    table, free, count, ln = paged.tables_after(cache, n)
    had, has = -(-cache.lens // 16), -(-ln // 16)
    for h in range(cache.lens.size):  # only entries that the call writes are changed
        table[h, had[h]:has[h]] = none_out_of_range(table[h, had[h]:has[h]], pages)
    assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE
    s.same(table, free, count, ln)
    seen = np.where((table >= 0) & (table < pages), table, -(1 << 20))
    want = slot_map(cache, seen, tokens, cap)[1]
    want[want < -3] = -1
    assert (want == -1).any() and np.array_equal(slots.cpu().numpy(), want)


def test_release_passes_no_bad_page_on(cuda):
    lens = np.array([[[40, 17], [300, 16], [5, 5]]])
    cache = paged.Cache(lens, 16, spare=2)
    pages = cache.pages.num_pages
    spoil(cache.table, [(0, 0), (0, 2), (3, 0), (5, 0), (2, 1)], pages)
    s = State(cache)
    s.release([1, 0, 1])
    table, free, count, ln = paged.tables_after(cache, [1, 1, 0, 0, 1, 1], release=True)
    free[2:count] = none_out_of_range(free[2:count], pages)
    assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE
    s.same(table, free, count, ln)
    # What came back as -1 is no page for the next sequence either.
    s.len, s.count, s.status = s.new_len.clone(), s.new_count.clone(), torch.zeros_like(s.status)
    s.tables(tokens=dev([0, 0, 60]))
    assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE
    got = s.table.cpu().numpy()[4:6, :4]
    assert np.array_equal(got.reshape(-1), free[:count][::-1][:8]) and (got == -1).any()


@pytest.mark.parametrize("release", [False, True])
def test_bad_pages_among_many(cuda, release):
    """More pages than one a lane: runs of one slab and chunks of several."""
    r = np.random.default_rng(2)
    lens = r.integers(0, 60000, (4, 8, 6))
    lens[:, 3] = r.integers(0, 400, (4, 6))
    tokens = r.integers(0, 40000, 8)
    tokens[3] = 200
    n = np.broadcast_to(tokens[None, :, None], lens.shape)
    need = int((-(-(lens + n) // 16) - -(-lens // 16)).sum())
    cache = tables_of(lens, 16, need + 1, 40000 // 16 + 2)
    pages = cache.pages.num_pages
    had = -(-cache.lens // 16)
    if release:
        assert int(had.sum()) > 152 * 1024
        spoil(cache.table, [(h, int(x)) for h in range(cache.lens.size) for x in r.integers(0, had[h], 3) if had[h]], pages)
    else:
        assert need > 152 * 1024
        spoil(cache.free, list(r.integers(1, need + 1, 300)), pages)
    s = State(cache)
    if release:
        s.release(np.ones(8, int))
        table, free, count, ln = paged.tables_after(cache, np.ones(lens.size), release=True)
        free[need + 1:count] = none_out_of_range(free[need + 1:count], pages)
    else:
        s.tables(tokens=dev(tokens))
        table, free, count, ln = paged.tables_after(cache, n)
        has = -(-ln // 16)
        for h in range(lens.size):
            table[h, had[h]:has[h]] = none_out_of_range(table[h, had[h]:has[h]], pages)
    assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE
    s.same(table, free, count, ln)


def test_rows_of_another_type_are_not_packed(cuda):
    plan, _ = plan_of(1, 2, 1, [100])
    cache = paged.Cache(np.zeros((1, 1, 1), int), 16, spare=9, wider=9, H=2, dtype=torch.bfloat16)
    s = State(cache)
    s.tables(plan=plan)
    K = torch.ones((1, 1, 1, 100, 128), dtype=torch.float16, device="cuda")
    Kp, Vp = cache.Kp.cuda(), cache.Vp.cuda()
    with pytest.raises(dkv.DkvError, match="types"):
        dkv.dkv_page_compact(s.p, plan, K, K, s.table, s.new_len, Kp, Vp, status=s.status)
    torch.cuda.synchronize()
    assert int(s.status) == 0 and torch.isnan(Kp).all() and torch.isnan(Vp).all()
    # 16-bit words without a type go into pools of either.
    dkv.dkv_page_compact(s.p, plan, K.view(torch.int16), K.view(torch.int16), s.table, s.new_len, Kp, Vp, status=s.status)
    n = int(s.new_len[0])
    cache.table, cache.lens = s.table.cpu().numpy(), np.array([n])
    at = torch.from_numpy(cache.rows(0))
    assert n > 0 and int(s.status) == 0 and (Kp.cpu()[at].view(torch.float16) == 1).all()
    plan.close()


def test_a_layer_of_numpy(cuda):
    tokens = [1, 3]
    cache = paged.Cache(lens_of(2, 2, 1, [30, 90], tokens, 1), 16, H=2)
    cu, qkv = inputs(cache, tokens, 3)
    c = Call(cache, np.int64(1), qkv, cu).run()
    want, size, _, _ = paged.attention(cache, 1, *qkv, cu, True)
    paged.assert_attention(c.out, want, size, cache.dtype)


@pytest.mark.parametrize("name", ["page table", "page release", "paged compact", "chunk attention"])
def test_an_injected_launch_failure_is_an_error(cuda, monkeypatch, name):
    plan, _ = plan_of(1, 2, 1, [100])
    cache = paged.Cache(np.zeros((1, 1, 1), int), 16, spare=9, wider=9, H=2)
    s = State(cache)
    K = torch.ones((1, 1, 1, 100, 128), dtype=torch.bfloat16, device="cuda")
    Kp, Vp = cache.Kp.cuda(), cache.Vp.cuda()
    cu, qkv = inputs(paged.Cache(np.full((1, 1, 1), 90), 16, H=2), [3], 1)
    c = Call(paged.Cache(np.full((1, 1, 1), 90), 16, H=2), 0, qkv, cu)
    call = {
        "page table": lambda: s.tables(plan=plan),
        "page release": lambda: s.release([1]),
        "paged compact": lambda: dkv.dkv_page_compact(s.p, plan, K, K, s.table, s.len, Kp, Vp, status=s.status),
        "chunk attention": c.run,
    }[name]
    call()
    monkeypatch.setenv("DKV_FAULT", "launch")
    with pytest.raises(dkv.DkvError, match=f"{name}.*injected launch failure") as e:
        call()
    assert e.value.status == dkv.DKV_ERR_CUDA
    monkeypatch.delenv("DKV_FAULT")
    call()
    torch.cuda.synchronize()
    plan.close()


def test_rows_of_no_token_hold_anything(cuda):
    """Rows behind the last sequence: what they hold in q, k_new and v_new is not used."""
    for tokens in ([1, 3], [40, 1]):
        cache = paged.Cache(lens_of(1, 2, 2, [200, 90], tokens, 1), 16, H=8)
        cu, qkv = inputs(cache, tokens, 3, pad=30)
        qkv = [x.clone() for x in qkv]
        for x, fill in zip(qkv, (float("nan"), float("inf"), float("nan"))):
            x[cu[-1]:] = fill
        c = Call(cache, 0, qkv, cu).run()
        want, size, Kp, Vp = paged.attention(cache, 0, *qkv, cu, True)
        assert int(c.status) == 0
        paged.assert_attention(c.out, want, size, cache.dtype)
        for got, exp in ((c.Kp, Kp), (c.Vp, Vp)):
            assert torch.equal(got.double().cpu().nan_to_num(99.0), exp.nan_to_num(99.0))


def test_without_a_status_word(cuda):
    """Values out of range with nowhere to report them."""
    tokens = [2, 3]
    cache = paged.Cache(lens_of(1, 2, 1, [98, 30], tokens, 1), 16, H=4)
    cu, qkv = inputs(cache, tokens, 3, pad=7)
    c = Call(cache, 0, qkv, [4, 6, 9])
    c.status = None
    before = bits(c.Kp), bits(c.Vp), bits(c.out)
    c.run()
    for got, old in zip((c.Kp, c.Vp, c.out), before):
        assert torch.equal(bits(got), old)
    s = State(cache)
    s.status = None
    s.len[0] = -4
    s.tables(tokens=dev(tokens))
    assert torch.equal(s.new_len, s.len) and torch.equal(s.new_count, s.count)
    s = State(cache)
    s.status = None
    s.table[0, 0] = -7
    s.release([1, 0])
    assert int(s.free[cache.count]) == -1


def test_a_prompt_that_found_no_pages_is_not_packed(cuda):
    plan, _ = plan_of(2, 4, 2, [300, 200])
    cache = paged.Cache(np.zeros((2, 3, 2), int), 16, spare=9, wider=30, H=4)
    s = State(cache)
    s.new_len, s.new_count = s.len, s.count
    s.table.fill_(3)  # entries of sequences that are gone
    K = torch.ones((2, 2, 2, 300, 128), dtype=torch.bfloat16, device="cuda")
    Kp, Vp = cache.Kp.cuda(), cache.Vp.cuda()
    s.tables(plan=plan, seq=dev([0, 2]))
    dkv.dkv_page_compact(s.p, plan, K, K, s.table, s.len, Kp, Vp, seq=dev([0, 2]), status=s.status)
    assert int(s.status) == dkv.DKV_DEV_PAGES_EXHAUSTED | dkv.DKV_DEV_PAGE_RANGE
    assert torch.isnan(Kp).all() and torch.isnan(Vp).all()
    plan.close()
