"""The page tables, releases and the prune-and-pack into pages against their definitions, and a serving loop of them
with dkv_chunk_attn."""
import numpy as np
import pytest
import torch

import oracle as O
import paged
from paper_2609_32663_gb300 import dkv

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


class State:
    """A cache's tables on the GPU."""

    def __init__(self, cache):
        self.cache, self.p = cache, cache.pages
        self.table, self.free, self.len = dev(cache.table), dev(cache.free), dev(cache.lens)
        self.count = dev([cache.count])
        self.new_len = torch.full_like(self.len, -9)
        self.new_count = torch.full_like(self.count, -9)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.work = torch.full((dkv.dkv_page_workspace_bytes(self.p),), 0xa5, dtype=torch.uint8, device="cuda")

    def tables(self, **kw):
        dkv.dkv_page_tables(self.p, self.len, self.new_len, self.table, self.free, self.count, self.new_count, self.work,
                            status=self.status, **kw)

    def release(self, ended):
        dkv.dkv_page_release(self.p, dev(ended), self.len, self.new_len, self.table, self.free, self.count, self.new_count,
                             self.work, status=self.status)

    def same(self, table, free, count, ln):
        assert int(self.new_count) == count
        assert np.array_equal(self.new_len.cpu().numpy(), ln)
        assert np.array_equal(self.table.cpu().numpy(), table)
        assert np.array_equal(self.free.cpu().numpy(), free)


def slot_map(cache, table, tokens, cap):
    cu = np.concatenate([[0], np.cumsum(tokens)])
    slots = np.full((cache.L, cap, cache.Hkv), -3, np.int32)
    for h in range(cache.lens.size):
        l, b, g = h // (cache.B * cache.Hkv), h // cache.Hkv % cache.B, h % cache.Hkv
        r = cache.lens[h] + np.arange(tokens[b])
        slots[l, cu[b]:cu[b + 1], g] = table[h][r // cache.P] * cache.P + r % cache.P
    return cu, slots


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("L,B,Hkv,most,tokens", [
    (1, 1, 1, 0, [1]), (1, 1, 1, 40, [0]), (2, 3, 2, 300, [1, 0, 5]), (3, 5, 3, 200, [0, 0, 0, 0, 0]),
    (2, 4, 8, 100, [129, 16, 15, 17]), (5, 7, 4, 500, [1] * 7), (33, 17, 4, 130, list(range(17))),
    (2, 512, 1, 70, [i % 3 for i in range(512)]), (3, 2, 7, 60, [333, 1]),
])
@pytest.mark.parametrize("alias", [False, True])
def test_tables(cuda, page, L, B, Hkv, most, tokens, alias):
    r = np.random.default_rng(page + L)
    lens = r.integers(0, most + 1, (L, B, Hkv))
    n = np.broadcast_to(np.asarray(tokens)[None, :, None], lens.shape)
    need = int((-(-(lens + n) // page) - -(-lens // page)).sum())
    cache = paged.Cache(lens, page, spare=need + 2, wider=max(tokens) // page + 2)
    s = State(cache)
    if alias:
        s.new_len, s.new_count = s.len, s.count
    cap = sum(tokens) + 3
    cu, slots = dev(np.full(B + 1, -9)), dev(np.full((L, cap, Hkv), -3))
    s.tables(tokens=dev(tokens), cu_tokens=cu, slots=slots)
    table, free, count, ln = paged.tables_after(cache, n)
    want_cu, want_slots = slot_map(cache, table, tokens, cap)
    assert int(s.status) == 0
    s.same(table, free, count, ln)
    assert np.array_equal(cu.cpu().numpy(), want_cu)
    assert np.array_equal(slots.cpu().numpy(), want_slots)


def test_more_slabs_than_one_launch_takes(cuda):
    """Past 49,152 slabs the scan is a launch of its own."""
    L, B, Hkv = 2, 100, 251
    r = np.random.default_rng(1)
    lens, tokens = r.integers(0, 41, (L, B, Hkv)), [i % 4 for i in range(100)]
    n = np.broadcast_to(np.asarray(tokens)[None, :, None], lens.shape)
    cache = paged.Cache(np.zeros((1, 1, 1), int), 16)
    cache.L, cache.B, cache.Hkv, cache.lens = L, B, Hkv, lens.reshape(-1).astype(np.int64)
    pages = -(-cache.lens // 16)
    order = r.permutation(int(pages.sum()) + 20000).astype(np.int32)
    cache.table = np.full((cache.lens.size, 6), -1, np.int32)
    cache.table[np.arange(6)[None] < pages[:, None]] = order[:int(pages.sum())]
    cache.free, cache.count = np.concatenate([order[int(pages.sum()):], np.full(int(pages.sum()), -7, np.int32)]), 20000
    cache.pages = dkv.Pages(L=L, B=B, H=Hkv, H_kv=Hkv, page_rows=16, num_pages=order.size, max_pages=6)
    for alias in (False, True):
        s = State(cache)
        if alias:
            s.new_len, s.new_count = s.len, s.count
        cu, slots = dev(np.zeros(B + 1)), dev(np.full((L, sum(tokens) + 1, Hkv), -3))
        s.tables(tokens=dev(tokens), cu_tokens=cu, slots=slots)
        table, free, count, ln = paged.tables_after(cache, n)
        s.same(table, free, count, ln)
        assert np.array_equal(slots.cpu().numpy(), slot_map(cache, table, tokens, sum(tokens) + 1)[1])
        s = State(cache)
        ended = r.integers(0, 2, B)
        s.release(ended)
        s.same(*paged.tables_after(cache, np.broadcast_to(ended[None, :, None], lens.shape), release=True))


def test_tables_without_slot_map_or_offsets(cuda):
    cache = paged.Cache(np.array([[[5], [16]]]), 16, spare=4)
    for kw in ({}, {"cu_tokens": dev([7, 7, 7])}):
        s = State(cache)
        s.tables(tokens=dev([20, 1]), **kw)
        s.same(*paged.tables_after(cache, [20, 1]))


@pytest.mark.parametrize("what,bit", [
    ("short", "EXHAUSTED"), ("negative", "RANGE"), ("wide", "RANGE"), ("cap", "RANGE"), ("length", "RANGE"),
    ("count", "RANGE"), ("count_low", "RANGE"),
])
def test_tables_all_or_nothing(cuda, what, bit):
    lens = np.array([[[5, 9], [16, 40]], [[0, 1], [33, 2]]])
    cache = paged.Cache(lens, 16, spare=30, wider=2)
    s = State(cache)
    tokens = [20, 13]
    cap = 40
    if what == "short":
        s.count.fill_(3)
    elif what == "negative":
        tokens = [20, -1]
    elif what == "wide":
        tokens = [20, 80]
    elif what == "cap":
        cap = 32
    elif what == "length":
        s.len[5] = -4
    elif what == "count":
        s.count.fill_(s.p.num_pages + 1)
    else:
        s.count.fill_(-1)
    before = s.table.clone(), s.free.clone(), s.len.clone(), s.count.clone()
    cu, slots = dev([9, 9, 9]), dev(np.full((2, cap, 2), -3))
    s.tables(tokens=dev(tokens), cu_tokens=cu, slots=slots)
    assert int(s.status) == getattr(dkv, "DKV_DEV_PAGES_EXHAUSTED" if bit == "EXHAUSTED" else "DKV_DEV_PAGE_RANGE")
    assert torch.equal(s.table, before[0]) and torch.equal(s.free, before[1])
    assert torch.equal(s.new_len, before[2]) and torch.equal(s.new_count, before[3])
    assert not cu.any() and (slots == -3).all()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("L,B,Hkv,most", [(1, 1, 1, 0), (1, 1, 1, 77), (2, 5, 3, 300), (30, 70, 4, 40)])
@pytest.mark.parametrize("alias", [False, True])
def test_release(cuda, page, L, B, Hkv, most, alias):
    r = np.random.default_rng(page + L)
    cache = paged.Cache(r.integers(0, most + 1, (L, B, Hkv)), page, spare=4)
    for ended in (r.integers(0, 2, B), np.zeros(B, int), np.ones(B, int)):
        s = State(cache)
        if alias:
            s.new_len, s.new_count = s.len, s.count
        s.release(ended * 3)
        assert int(s.status) == 0
        s.same(*paged.tables_after(cache, np.broadcast_to(ended[None, :, None], (L, B, Hkv)), release=True))


def test_release_past_the_list_is_refused(cuda):
    cache = paged.Cache(np.array([[[40], [16]]]), 16, spare=4)
    s = State(cache)
    s.count.fill_(s.p.num_pages - 1)
    free = s.free.clone()
    s.release([1, 0])
    assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE
    assert torch.equal(s.new_len, s.len) and torch.equal(s.new_count, s.count) and torch.equal(s.free, free)


def plan_of(L, H, Hkv, ctx, seed=0):
    shape = dkv.Shape(L=L, H=H, H_kv=Hkv, D=9, sink=5, recent=11, bin_width=40)
    M = (np.random.default_rng(seed).random((L, H, 9)) < 0.3).astype(np.uint8)
    plan = dkv.dkv_map_pattern(M, ctx, shape)
    om = O.map_pattern(M, ctx, O.Geometry(L=L, H=H, Hkv=Hkv, D=9, sink=5, recent=11, bin_width=40))
    return plan, om


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ctx,B,seq", [([300], 1, None), ([16, 0, 222], 3, None), ([376, 1, 90], 7, [0, 2, 6])])
def test_admit(cuda, page, dtype, ctx, B, seq):
    """dkv_page_tables and dkv_page_compact with a plan: the kept rows are in their slots' pages, all else is as it was."""
    L, H, Hkv = 2, 6, 2
    plan, om = plan_of(L, H, Hkv, ctx)
    where = seq if seq is not None else list(range(len(ctx)))
    lens = np.random.default_rng(1).integers(0, 50, (L, B, Hkv))  # some slots hold rows already
    grow = np.zeros((L, B, Hkv), int)
    grow[:, where] = om.len.reshape(L, len(ctx), Hkv)
    cache = paged.Cache(lens, page, spare=200, wider=30, dtype=dtype)
    s = State(cache)
    s.tables(plan=plan, seq=None if seq is None else dev(seq))
    table, free, count, ln = paged.tables_after(cache, grow)
    s.same(table, free, count, ln)
    T = max(ctx) + 2
    K, V = (torch.randn((L, len(ctx), Hkv, T, 128), generator=torch.Generator().manual_seed(i)).to(dtype) for i in (1, 2))
    Kp, Vp = cache.Kp.cuda(), cache.Vp.cuda()
    dkv.dkv_page_compact(s.p, plan, K.cuda(), V.cuda(), s.table, s.new_len, Kp, Vp, seq=None if seq is None else dev(seq),
                         status=s.status)
    assert int(s.status) == 0
    for got, src, pool in ((Kp, K, cache.Kp), (Vp, V, cache.Vp)):
        want = pool.clone()
        for i in range(om.len.size):
            l, j, g = i // (len(ctx) * Hkv), i // Hkv % len(ctx), i % Hkv
            h = (l * B + where[j]) * Hkv + g
            r = cache.lens[h] + np.arange(om.len[i])
            want[table[h][r // page].astype(np.int64) * page + r % page] = src[l, j, g, om.idx[om.ioff[i]:om.ioff[i + 1]]]
        assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))
    plan.close()


@pytest.mark.parametrize("seq", [[1, 0], [2, 2], [-1, 0], [0, 3]])
def test_slots_out_of_order_or_range_are_refused(cuda, seq):
    plan, _ = plan_of(1, 2, 1, [100, 50])
    s = State(paged.Cache(np.zeros((1, 3, 1), int), 16, spare=40, wider=20, H=2))
    s.tables(plan=plan, seq=dev(seq))
    assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE and not s.new_len.any() and int(s.new_count) == 40
    plan.close()


def test_compact_skips_rows_without_a_place(cuda):
    """Tables that were never grown: nothing is written, and the status says so."""
    plan, _ = plan_of(1, 2, 1, [100])
    cache = paged.Cache(np.zeros((1, 1, 1), int), 16, spare=4, H=2)
    s = State(cache)
    K = torch.ones((1, 1, 1, 100, 128), dtype=torch.bfloat16, device="cuda")
    Kp, Vp = cache.Kp.cuda(), cache.Vp.cuda()
    for n in (0, 30, 1 << 30):
        s.status.zero_()
        dkv.dkv_page_compact(s.p, plan, K, K, s.table, torch.full_like(s.len, n), Kp, Vp, status=s.status)
        assert int(s.status) == dkv.DKV_DEV_PAGE_RANGE and torch.isnan(Kp).all() and torch.isnan(Vp).all()
    plan.close()


def test_serving_loop(cuda):
    """Admit two pruned prompts, take turns and tokens, end one, admit another into its slot and pages: every step's
    outputs against 64 bits, with host copies of the tables that follow the definitions."""
    L, H, Hkv, B, page = 2, 8, 2, 3, 16
    cache = paged.Cache(np.zeros((L, B, Hkv), int), page, spare=190, wider=40, H=H)
    s = State(cache)
    s.new_len, s.new_count = s.len, s.count
    Kp, Vp = cache.Kp.cuda(), cache.Vp.cuda()
    work = torch.empty(dkv.dkv_chunk_workspace_bytes(s.p), dtype=torch.uint8, device="cuda")
    gen = torch.Generator().manual_seed(3)

    def follow(n, release=False):
        cache.table, cache.free, cache.count, cache.lens = paged.tables_after(cache, n, release)
        s.same(cache.table, cache.free, cache.count, cache.lens)

    def admit(ctx, seq, seed):
        plan, om = plan_of(L, H, Hkv, ctx, seed)
        s.tables(plan=plan, seq=dev(seq))
        n = np.zeros((L, B, Hkv), int)
        n[:, seq] = om.len.reshape(L, len(ctx), Hkv)
        follow(n)
        K, V = (torch.randn((L, len(ctx), Hkv, max(ctx), 128), generator=gen).bfloat16() for _ in range(2))
        dkv.dkv_page_compact(s.p, plan, K.cuda(), V.cuda(), s.table, s.len, Kp, Vp, seq=dev(seq), status=s.status)
        cache.Kp, cache.Vp = Kp.cpu(), Vp.cpu()
        for i in range(om.len.size):
            l, j, g = i // (len(ctx) * Hkv), i // Hkv % len(ctx), i % Hkv
            h = (l * B + seq[j]) * Hkv + g
            assert torch.equal(cache.Kp[cache.rows(h)], K[l, j, g, om.idx[om.ioff[i]:om.ioff[i + 1]]])
        plan.close()

    def step(tokens):
        cu = dev(np.zeros(B + 1))
        s.tables(tokens=dev(tokens), cu_tokens=cu)
        follow(np.broadcast_to(np.asarray(tokens)[None, :, None], (L, B, Hkv)))
        T = sum(tokens)
        for layer in range(L):
            qkv = torch.randn((T, H + 2 * Hkv, 128), generator=gen).bfloat16()
            d = qkv.cuda()
            out = torch.full((T, H, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
            dkv.dkv_chunk_attn(s.p, layer, d[:, :H], d[:, H:H + Hkv], d[:, H + Hkv:], cu, s.table, s.len, Kp, Vp, out, work,
                               status=s.status)
            want, size, wK, wV = paged.attention(cache, layer, qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:],
                                                 np.concatenate([[0], np.cumsum(tokens)]), True)
            paged.assert_attention(out, want, size, torch.bfloat16, f"{tokens} layer {layer}")
            cache.Kp, cache.Vp = wK.bfloat16(), wV.bfloat16()
            assert torch.equal(Kp.cpu().nan_to_num(9.0), cache.Kp.nan_to_num(9.0))

    admit([300, 120], [0, 2], 1)
    step([20, 0, 1])
    step([1, 0, 1])
    s.release([1, 0, 0])
    follow(np.broadcast_to(np.array([1, 0, 0])[None, :, None], (L, B, Hkv)), release=True)
    admit([376], [1], 2)
    step([0, 33, 1])
    step([7, 1, 2])  # a slot that held a sequence before starts anew
    assert int(s.status) == 0


def tables_of(lens, page, spare, wider):
    """The tables of a cache without its pools."""
    cache = paged.Cache(np.zeros((1, 1, 1), int), page)
    cache.L, cache.B, cache.Hkv = lens.shape
    cache.lens = lens.reshape(-1).astype(np.int64)
    pages = -(-cache.lens // page)
    total = int(pages.sum())
    order = np.random.default_rng(5).permutation(total + spare).astype(np.int32)
    cache.table = np.full((cache.lens.size, int(pages.max()) + wider), -1, np.int32)
    cache.table[np.arange(cache.table.shape[1])[None] < pages[:, None]] = order[:total]
    cache.free, cache.count = np.concatenate([order[total:], np.full(total, -7, np.int32)]), spare
    cache.pages = dkv.Pages(L=cache.L, B=cache.B, H=cache.Hkv, H_kv=cache.Hkv, page_rows=page, num_pages=order.size,
                            max_pages=cache.table.shape[1])
    return cache


@pytest.mark.parametrize("L,Hkv,tokens,off", [
    (33, 8, [0, 1700, 0, 3001, 7], 0), (33, 8, [5, 1700, 0, 3001], 1), (33, 3, [1, 999, 1500], 0), (70, 1, [40000, 1], 0),
    (2, 33, [3, 1, 40], 0), (2, 136, [0, 9, 30], 0), (2, 260, [17, 0], 0), (1, 132, [9000], 2),
])
def test_slot_map_of_many_entries(cuda, L, Hkv, tokens, off):
    """More entries than one a lane, past ends of sequences and layers; rows of heads wider than a warp; maps off 16 bytes."""
    r = np.random.default_rng(Hkv)
    lens = r.integers(0, 90, (L, len(tokens), Hkv))
    n = np.broadcast_to(np.asarray(tokens)[None, :, None], lens.shape)
    need = int((-(-(lens + n) // 64) - -(-lens // 64)).sum())
    cache = tables_of(lens, 64, need, max(tokens) // 64 + 2)
    s = State(cache)
    cap = sum(tokens) + 5
    cu, flat = dev(np.full(len(tokens) + 1, -9)), dev(np.full(L * cap * Hkv + 8, -3))
    slots = flat[off:off + L * cap * Hkv].view(L, cap, Hkv)
    s.tables(tokens=dev(tokens), cu_tokens=cu, slots=slots)
    table, free, count, ln = paged.tables_after(cache, n)
    want_cu, want = slot_map(cache, table, tokens, cap)
    assert int(s.status) == 0
    s.same(table, free, count, ln)
    assert np.array_equal(cu.cpu().numpy(), want_cu) and np.array_equal(slots.cpu().numpy(), want)
    assert (flat[:off] == -3).all() and (flat[off + L * cap * Hkv:] == -3).all()


@pytest.mark.parametrize("L,B,Hkv,most", [(8, 8, 8, 16000), (8, 500, 10, 170), (3, 2, 7, 200000), (1, 9, 5, 120000)])
def test_many_pages(cuda, L, B, Hkv, most):
    """More pages than one a lane: runs of one slab, chunks of several slabs, slabs of none, some ended."""
    r = np.random.default_rng(B)
    lens = r.integers(0, most + 1, (L, B, Hkv))
    lens[r.integers(0, 4, lens.shape) == 0] = 0
    tokens = r.integers(0, most, B)
    n = np.broadcast_to(tokens[None, :, None], lens.shape)
    need = int((-(-(lens + n) // 16) - -(-lens // 16)).sum())
    assert need > 152 * 1024
    cache = tables_of(lens, 16, need + 1, most // 16 + 2)
    s = State(cache)
    s.tables(tokens=dev(tokens))
    assert int(s.status) == 0
    s.same(*paged.tables_after(cache, n))
    for ended in (r.integers(0, 2, B), np.ones(B, int)):
        s = State(cache)
        s.release(ended)
        assert int(s.status) == 0
        s.same(*paged.tables_after(cache, np.broadcast_to(ended[None, :, None], (L, B, Hkv)), release=True))
