"""Paged-cache operators on the GPU against plain implementations in 64 bits (paged_reference.py)."""
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2410_13344_b200 import binding

pytestmark = pytest.mark.gpu
PAGE = 16
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------- pages


def make_book(rng, B, max_pages, context, spare):
    lens = [rng.choice([0, 0, 1, 15, 16, 17, rng.randint(0, context)]) for _ in range(B)]
    lens = [min(n, max_pages * PAGE) for n in lens]
    held = [ref.pages_of(n) for n in lens]
    pool = rng.sample(range(sum(held) + spare + 3), sum(held) + spare + 3)
    table = []
    for h in held:
        table.append([pool.pop() for _ in range(h)] + [-1] * (max_pages - h))
    free = [pool.pop() for _ in range(spare)]
    return ref.Book(lens, table, free + [-1] * (sum(held) + 3), spare)


def to_gpu(book):
    return [i32(book.lens), i32(book.table).view(len(book.lens), -1), i32(book.free), i32([book.n_free])]


def same_book(book, state):
    lens, table, free, n_free = state
    assert lens.tolist() == book.lens and table.tolist() == book.table and free.tolist() == book.free and n_free.tolist() == [book.n_free]


@pytest.mark.parametrize("B,chunk,spare", [(1, 1, 0), (1, 1, 3), (1, 700, 60), (3, 40, 4), (33, 20, 30), (64, 1, 64), (300, 50, 500), (1025, 3, 300),
                                           (2049, 30, 3000), (8192, 2, 5000)])
def test_plan_and_trim_follow_the_requests(B, chunk, spare):
    rng = random.Random(B * 1000 + chunk)
    book = make_book(rng, B, 60, 300, spare)
    state = to_gpu(book)
    for step in range(3):
        n_new = [rng.choice([0, 1, 1, -2, rng.randint(0, chunk)]) for _ in range(B)]
        rows = sum(max(0, n) for n in n_new) + rng.choice([0, 1, 37, -5])
        rows = max(rows, 0)
        plan = binding.pages_plan(i32(n_new), *state, rows)
        want = book.plan(n_new, rows)
        for name, got, w in zip(plan._fields, plan, want):
            assert got.tolist() == w, (step, name)
        same_book(book, state)
        keep = [rng.choice([0, n, n + 3, max(0, n - 1), rng.randint(0, n), -1]) for n in book.lens]
        binding.pages_trim(i32(keep), *state)
        book.trim(keep)
        same_book(book, state)


def test_a_trim_behind_a_plan_restores_the_stack():
    rng = random.Random(5)
    book = make_book(rng, 200, 70, 800, 900)
    state = to_gpu(book)
    before = [t.clone() for t in state]
    binding.pages_plan(i32([rng.randint(0, 90) for _ in range(200)]), *state, 20000)
    assert not torch.equal(state[0], before[0])
    binding.pages_trim(before[0], *state)
    assert all(torch.equal(a, b) for a, b in zip(state, before))


def test_plan_of_many_rows_and_of_no_requests():
    rng = random.Random(6)
    book = make_book(rng, 7, 5000, 3, 6000)
    state = to_gpu(book)
    n_new = [20000, 1, 0, 15, 61007, 2, 1]
    rows = sum(n_new) + 3
    plan, want = binding.pages_plan(i32(n_new), *state, rows), book.plan(n_new, rows)
    for got, w in zip(plan, want):
        assert got.tolist() == w
    same_book(book, state)
    # wants past 31 bits fit nobody's table; what comes behind has its rows behind them
    book = make_book(rng, 4, 8, 3, 40)
    state = to_gpu(book)
    n_new = [2, 2 ** 31 - 1, 2 ** 31 - 1, 4]
    plan = binding.pages_plan(i32(n_new), *state, 20)
    want = book.plan(n_new, 20)
    assert plan.slot.tolist() == want[0] and plan.granted.tolist() == want[4] == [2, 0, 0, 0]
    assert plan.row_off.tolist() == [min(x, 2 ** 31 - 1) for x in want[3]]
    same_book(book, state)
    none = [torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 4, dtype=torch.int32, device="cuda"), i32([3, 4]), i32([2])]
    plan = binding.pages_plan(none[0], *none, 5)
    assert plan.slot.tolist() == [-1] * 5 and plan.row_off.tolist() == [0] and none[3].tolist() == [2]
    binding.pages_trim(none[0], *none)


def test_lengths_out_of_range_are_taken_to_the_nearest_in_range():
    lens, table, free, n_free = i32([-5, 1000, 20]), i32([[-1] * 3, [5, 6, 7], [8, 9, -1]]), i32([1, 2, 3]), i32([100])
    plan = binding.pages_plan(i32([1, 1, 1]), lens, table, free, n_free, 3)
    assert plan.granted.tolist() == [1, 0, 1] and plan.slot.tolist() == [3 * 16, -1, 9 * 16 + 4]
    assert n_free.tolist() == [2] and table.tolist() == [[3, -1, -1], [5, 6, 7], [8, 9, -1]]
    binding.pages_trim(i32([0, 0, 0]), lens, table, free, n_free)
    assert n_free.tolist() == [3] and lens.tolist() == [0, 0, 0] and bool((table == -1).all())       # (room for one of the six)


@pytest.mark.parametrize("rows", [40, 200000])                # a row to a lane, four rows to a lane
def test_what_can_be_no_page_gives_no_slot(rows):
    for page in (2 ** 27, 2 ** 28, 2 ** 31 - 1, -1, -(2 ** 28), -(2 ** 31)):
        lens, table, free, n_free = i32([3]), i32([[page] + [-1] * 12499]), i32([page] * 12500), i32([12500])
        plan = binding.pages_plan(i32([min(rows, 199990)]), lens, table, free, n_free, rows)
        assert plan.granted.tolist() == [min(rows, 199990)] and bool((plan.slot < 0).all())


# ---------------------------------------------------------------------------------------------- append


def runs_of_slots(rng, T, n_pages, decode):
    pages = rng.sample(range(n_pages), n_pages)
    slots = []
    while len(slots) < T:
        if rng.random() < 0.1:
            slots.append(rng.choice([-1, -7, n_pages * PAGE, n_pages * PAGE + 5, 2 ** 31 - 1]))
            continue
        page = pages.pop()
        start = rng.choice([0, 0, rng.randrange(PAGE)])
        n = 1 if decode else rng.choice([PAGE - start, rng.randint(1, PAGE - start)])
        slots += [page * PAGE + start + i for i in range(n)]
    return slots[:T]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hk,D,decode", [(1, 1, 64, True), (5, 3, 128, True), (64, 8, 128, True), (333, 5, 64, False), (1000, 2, 128, False), (3001, 8, 64, False)])
@pytest.mark.parametrize("summaries", [True, False])
def test_append(dtype, T, Hk, D, decode, summaries):
    rng, g = random.Random(T), torch.Generator().manual_seed(T)
    n_pages = T + 5 if decode else T // 4 + 20
    slots = runs_of_slots(rng, T, n_pages, decode)
    dt = DT[dtype]
    qkv = torch.randn(T, (2 * Hk + 3) * D, generator=g).to(dt)
    if T > 4:
        qkv[3, 3 * D:3 * D + 9] = torch.tensor([math.inf, -math.inf, math.nan, 0.0, -0.0, 1e-40, -1e-40, 3e38, -3e38]).to(dt)
    k_pool, v_pool = torch.randn(n_pages, Hk, PAGE, D, generator=g).to(dt), torch.randn(n_pages, Hk, PAGE, D, generator=g).to(dt)
    k_min, k_max = k_pool.amin(2), k_pool.amax(2)
    cpu = [k_pool, v_pool] + ([k_min, k_max] if summaries else [])
    gpu = [t.cuda() for t in cpu]
    packed = qkv.cuda()

    def split(x):
        return x[:, 3 * D:(3 + Hk) * D].unflatten(1, (Hk, D)), x[:, (3 + Hk) * D:].unflatten(1, (Hk, D))

    binding.kv_append(*split(packed), i32(slots), *gpu)
    ref.append(*split(qkv), slots, *cpu)
    for got, want in zip(gpu, cpu):
        assert torch.equal(torch.nan_to_num(got.cpu(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))


def test_append_into_pools_past_32_bits():
    n_pages, Hk, D = (1 << 31) // (4 * PAGE * 64) + 9, 4, 64
    pool = torch.zeros(n_pages, Hk, PAGE, D, dtype=torch.bfloat16, device="cuda")
    other = torch.zeros_like(pool)
    k = torch.randn(3, Hk, D, device="cuda").bfloat16()
    slots = [(n_pages - 1) * PAGE + 15, 3, (n_pages // 2) * PAGE]
    binding.kv_append(k, k + 1, i32(slots), pool, other)
    for t, s in enumerate(slots):
        assert torch.equal(pool[s // PAGE, :, s % PAGE], k[t]) and torch.equal(other[s // PAGE, :, s % PAGE], k[t] + 1)
    assert int((pool != 0).any(3).any(2).any(1).sum()) == 3
    # ... and the attention that reads them back: one key is its own average
    q = torch.randn(1, 8, D, device="cuda").bfloat16()
    out, lse = binding.paged_attention(q, pool, other, i32([[n_pages - 1]]), i32([16]), 0.125, 16, window=1)
    assert torch.equal(out.view(4, 2, D), (k[0] + 1)[:, None].expand(4, 2, D))
    s = (q[0].view(4, 2, D).double() * k[0].double()[:, None]).sum(2) * 0.125
    assert float((lse.view(4, 2).double() - s).abs().max()) < 1e-4
    del pool, other


# ---------------------------------------------------------------------------------------------- attention


class Cache:
    def __init__(self, lens, Hk, D, dtype, seed, wider=2, garbage=True):
        g, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        dt = DT[dtype]
        held = [ref.pages_of(n) for n in lens]
        n_pages = sum(held) + 3
        self.lens, self.dt = lens, dt
        self.k_pool = (0.8 * torch.randn(n_pages, Hk, PAGE, D, generator=g) + 0.6 * torch.randn(n_pages, Hk, 1, D, generator=g)).to(dt)
        self.v_pool = torch.randn(n_pages, Hk, PAGE, D, generator=g).to(dt)
        pages = rng.sample(range(n_pages), n_pages)
        mp = max(held) + wider
        self.table = torch.full((len(lens), mp), -1, dtype=torch.int32)
        self.k_min, self.k_max = self.k_pool.amin(2), self.k_pool.amax(2)
        for b, n in enumerate(lens):
            for j in range(held[b]):
                self.table[b, j] = pages.pop()
            if n % PAGE:
                last = int(self.table[b, held[b] - 1])
                self.k_min[last], self.k_max[last] = self.k_pool[last, :, :n % PAGE].amin(1), self.k_pool[last, :, :n % PAGE].amax(1)
                if garbage:
                    bad = [math.nan, math.inf, -math.inf, float(torch.finfo(dt).min)][b % 4]
                    self.k_pool[last, :, n % PAGE:], self.v_pool[last, :, n % PAGE:] = bad, bad
            # what stands behind a request's pages is not looked at
            self.table[b, held[b]:] = [-1, 2 ** 30, n_pages, -2 ** 31][b % 4]
        self.gpu = [t.cuda() for t in (self.k_pool, self.v_pool, self.table)]
        self.glens = i32(lens)

    def queries(self, H, seed, size=2.0):
        """A view into a wider product."""
        D = self.k_pool.shape[3]
        x = (size * torch.randn(len(self.lens), (H + 3) * D, generator=torch.Generator().manual_seed(seed))).to(self.dt)
        return x[:, D:(H + 1) * D].unflatten(1, (H, D)), x.cuda()[:, D:(H + 1) * D].unflatten(1, (H, D))


def check(out, lse, want):
    o, l, (to, tl) = want
    out, lse = out.double().cpu(), lse.double().cpu()
    empty = torch.isneginf(l)
    assert torch.equal(torch.isneginf(lse), empty) and bool((out[empty] == 0).all())
    assert bool(((out - o).abs() <= to).all()), float(((out - o).abs() - to).max())
    assert bool(((lse - l).abs()[~empty] <= tl[~empty]).all()), float(((lse - l).abs() - tl)[~empty].max())


LENS = [0, 1, 2, 15, 16, 17, 31, 33, 100, 640, 0, 1]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hk,G,D", [(1, 1, 64), (2, 1, 128), (3, 2, 64), (2, 3, 128), (8, 4, 128), (2, 5, 64), (1, 7, 128), (2, 8, 64), (1, 9, 128), (2, 12, 64),
                                    (1, 16, 128), (1, 17, 64), (1, 40, 128)])
@pytest.mark.parametrize("window", [0, 1, 17, 100])
def test_attention_of_ragged_batches(dtype, Hk, G, D, window):
    c = Cache(LENS, Hk, D, dtype, 7 * Hk + G)
    q, gq = c.queries(Hk * G, G)
    scale = D ** -0.5
    out, lse = binding.paged_attention(gq, *c.gpu, c.glens, scale, 640, window=window)
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, LENS, scale, window))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,window", [([9000], 0), ([4097, 12000, 0, 33], 0), ([20011], 9001), ([5000, 16], 4999)])
@pytest.mark.parametrize("hint", [1, None, 60000])
def test_attention_of_long_caches_in_splits(dtype, lens, window, hint):
    Hk, G, D = (2, 4, 128) if len(lens) > 1 else (1, 5, 64)
    c = Cache(lens, Hk, D, dtype, len(lens))
    q, gq = c.queries(Hk * G, 3)
    out, lse = binding.paged_attention(gq, *c.gpu, c.glens, 0.1, hint or max(lens), window=window)
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, lens, 0.1, window))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,Hk,G,D,longest,window", [(120, 5, 1, 64, 60, 0), (120, 5, 1, 128, 200, 50), (75, 4, 3, 128, 64, 0), (90, 8, 9, 64, 250, 0), (60, 16, 2, 64, 33, 1), (64, 4, 16, 128, 700, 0), (40, 2, 40, 64, 3000, 500),
                                                     (300, 2, 17, 128, 40, 0)])
def test_attention_of_many_short_sequences(dtype, B, Hk, G, D, longest, window):
    rng = random.Random(B)
    lens = [rng.choice([0, 1, 16, 17, longest, rng.randint(0, longest)]) for _ in range(B)]
    lens[-1] = 0
    c = Cache(lens, Hk, D, dtype, B)
    q, gq = c.queries(Hk * G, 5)
    want = ref.attention(q, c.k_pool, c.v_pool, c.table, lens, 0.2, window)
    check(*binding.paged_attention(gq, *c.gpu, c.glens, 0.2, longest, window=window), want)
    if not window:
        # (and with lists: of all pages, which is the same, in another order)
        pages = [ref.pages_of(n) for n in lens]
        lists = [[list(range(n))[::-1] + [-1] * (max(pages) - n) for _ in range(Hk)] for n in pages]
        check(*binding.paged_attention(gq, *c.gpu, c.glens, 0.2, longest, sel=i32(lists), n_sel=i32(pages)), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size,scale", [(0.0, 1.0), (30.0, 1.0), (4.0, -0.3), (2.0, 0.0)])
def test_attention_with_flat_peaked_and_negative_scores(dtype, size, scale):
    lens = [1, 50, 700]
    c = Cache(lens, 2, 64, dtype, 11)
    q, gq = c.queries(8, 12, size)
    out, lse = binding.paged_attention(gq, *c.gpu, c.glens, scale, 700)
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, lens, scale))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [0, 40])
def test_attention_over_listed_pages(dtype, window):
    lens = [0, 5, 100, 333, 2000, 16]
    Hk, G, D, K = 3, 4, 64, 21
    c = Cache(lens, Hk, D, dtype, 21)
    q, gq = c.queries(Hk * G, 5)
    rng = random.Random(1)
    lists, counts = [], []
    for n in lens:
        N = ref.pages_of(n)
        counts.append(rng.choice([min(N, K), K, 0 if n == 100 else 3]))
        # any order, pages outside the sequence among them, some twice
        lists.append([[rng.choice([rng.randrange(max(N, 1)), -1, N, 2 ** 31 - 1]) if rng.random() < 0.3 else rng.randrange(max(N, 1)) for _ in range(K)]
                      for _ in range(Hk)])
    sel = i32(lists)
    out, lse = binding.paged_attention(gq, *c.gpu, c.glens, 0.2, 2000, window=window, sel=sel, n_sel=i32(counts))
    used = [[row[:min(counts[b], K)] for row in lists[b]] for b in range(len(lens))]
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, lens, 0.2, window, used))


@pytest.mark.parametrize("G,D", [(3, 64), (4, 64), (5, 128), (8, 128), (8, 64), (11, 64), (16, 128)])
@pytest.mark.parametrize("lens,window", [([1], 0), ([24, 3, 0, 200] * 60, 0), ([9000, 0, 7000], 0), ([700, 1, 555], 99)])
def test_fp32_attention_of_many_heads_in_every_form(G, D, lens, window):
    c = Cache(lens, 2, D, "fp32", G)
    q, gq = c.queries(2 * G, D)
    out, lse = binding.paged_attention(gq, *c.gpu, c.glens, 0.1, max(lens), window=window)
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, lens, 0.1, window))
    # a list in descending order, its first page twice
    K = 30
    lists = [[[ref.pages_of(n) - 1 - max(i - 1, 0) for i in range(K)] for _ in range(2)] for n in lens]
    out, lse = binding.paged_attention(gq, *c.gpu, c.glens, 0.1, max(lens), window=window, sel=i32(lists), n_sel=i32([K] * len(lens)))
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, lens, 0.1, window, lists))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages_outside_the_pool_hold_no_keys(dtype):
    lens = [200, 40, 16]
    c = Cache(lens, 2, 64, dtype, 31)
    n_pages = c.k_pool.shape[0]
    c.table[0, 3], c.table[0, 12], c.table[1, 0], c.table[2, 0] = -1, n_pages, 2 ** 31 - 1, -9
    table = c.table.cuda()
    q, gq = c.queries(6, 5)
    out, lse = binding.paged_attention(gq, c.gpu[0], c.gpu[1], table, c.glens, 0.2, 200)
    check(out, lse, ref.attention(q, c.k_pool, c.v_pool, c.table, lens, 0.2))
    assert bool(torch.isneginf(lse[2]).all())


def test_attention_scratch_and_output_without_lse():
    c = Cache([3000, 70], 2, 128, "bf16", 41)
    _, gq = c.queries(8, 6)
    # (a cache that may be long enough for shares and a join: those need the scratch)
    a, lse = binding.paged_attention(gq, *c.gpu, c.glens, 0.1, 60000)
    scratch = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")
    b, none = binding.paged_attention(gq, *c.gpu, c.glens, 0.1, 60000, want_lse=False, scratch=scratch)
    assert none is None and torch.equal(a, b)
    with pytest.raises(binding.CerbError) as e:
        binding.paged_attention(gq, *c.gpu, c.glens, 0.1, 60000, scratch=scratch[:64])
    assert e.value.code == binding.E_NOMEM


# ---------------------------------------------------------------------------------------------- selection


def check_lists(sel, n_sel, want, K):
    for b, rows in enumerate(want):
        assert int(n_sel[b]) == len(rows[0])
        for h, row in enumerate(rows):
            assert sel[b, h].tolist() == row + [-1] * (K - len(row)), (b, h)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hk,G,D,K,n_first,n_last", [(1, 1, 64, 1, 0, 0), (2, 3, 128, 2, 1, 1), (3, 8, 64, 7, 0, 2), (1, 9, 128, 40, 3, 1), (2, 16, 64, 64, 1, 1),
                                                     (1, 33, 128, 100, 0, 0), (2, 2, 64, 5, 5, 0)])
def test_selected_pages(dtype, Hk, G, D, K, n_first, n_last):
    lens = [0, 1, 17, 100, 16 * K, 16 * K + 1, 2000, 5003]
    c = Cache(lens, Hk, D, dtype, K)
    q, gq = c.queries(Hk * G, K)
    sel, n_sel = binding.page_select(gq, c.k_min.cuda(), c.k_max.cuda(), c.gpu[2], c.glens, K, 5003, n_first, n_last)
    check_lists(sel, n_sel, ref.select(q, c.k_min, c.k_max, c.table, lens, K, n_first, n_last), K)


def score_cache(kind, dtype, N, Hk=1, D=64):
    """Summaries of N pages whose scores are hard to tell apart."""
    g = torch.Generator().manual_seed(N)
    mid, spread = torch.randn(N, Hk, D, generator=g), torch.rand(N, Hk, D, generator=g)
    lo, hi = mid - spread, mid + spread
    if kind == "equal":
        lo, hi = lo[:1].expand(N, Hk, D), hi[:1].expand(N, Hk, D)
    elif kind == "zero":
        lo = hi = torch.zeros(N, Hk, D)
    elif kind == "few values":
        pick = torch.randint(0, 5, (N,), generator=g)
        lo, hi = lo[pick], hi[pick]
    elif kind == "near":                                    # a page's scores differ in the last bits of an element
        lo, hi = lo[:1].repeat(N, 1, 1), hi[:1].repeat(N, 1, 1)
        hi[:, :, 5] += 2.0 ** -20 * torch.randint(0, 4000, (N, 1), generator=g)
    elif kind == "outliers":
        lo[7], hi[7] = 1e4, 3e4
        lo[11], hi[11] = -3e4, -1e4
        hi[N // 2, :, 3] = 1e6
    elif kind == "channel":                                  # a channel far larger than the others
        lo[:, :, 9] -= 300
        hi[:, :, 9] -= 290
    elif kind == "odd":
        hi[3, :, 0], lo[5, :, 1], hi[N - 3, :, 2], lo[9, :, 3] = math.inf, -math.inf, math.nan, math.nan
    elif kind == "huge":
        hi[::3], lo[::5] = 3e38, -3e38
    lo, hi = lo.to(DT[dtype]).contiguous(), hi.to(DT[dtype]).contiguous()
    return lo, hi


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["plain", "equal", "zero", "few values", "near", "outliers", "channel", "odd", "huge"])
@pytest.mark.parametrize("N,K", [(40, 9), (3001, 130)])
def test_selection_where_scores_are_hard_to_tell_apart(dtype, kind, N, K):
    lo, hi = score_cache(kind, dtype, N)
    table = torch.tensor([random.Random(N).sample(range(N), N)], dtype=torch.int32)
    lens = [N * PAGE - 5]
    q = torch.randn(1, 3, 64, generator=torch.Generator().manual_seed(1)).to(DT[dtype])
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32(lens), K, lens[0])
    check_lists(sel, n_sel, ref.select(q, lo, hi, table, lens, K), K)


@pytest.mark.parametrize("N,K", [(45000, 300), (131072, 2048)])
def test_selection_of_very_long_caches(N, K):
    lo, hi = score_cache("plain", "bf16", N)
    table = torch.randperm(N, generator=torch.Generator().manual_seed(3)).to(torch.int32)[None]
    q = torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16()
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32([N * PAGE]), K, 100)     # (the hint far too small)
    x, rows = q[0].double(), table[0].long()
    score = (x.clamp(min=0) @ hi[rows, 0].double().T + x.clamp(max=0) @ lo[rows, 0].double().T).amax(0)
    score[0] = score[-1] = math.inf
    want = torch.sort(torch.sort(score, descending=True, stable=True).indices[:K]).values
    assert sel[0, 0].tolist() == want.tolist() and n_sel.tolist() == [K]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hint", [1, 100, 16 * 30, 16 * 30 + 1, 60000])
def test_selection_from_caches_longer_than_was_said(dtype, hint):
    lens = [16 * 30, 16 * 30 + 1, 9000, 0, 12345]
    c = Cache(lens, 2, 64, dtype, 5)
    q, gq = c.queries(6, 5)
    sel, n_sel = binding.page_select(gq, c.k_min.cuda(), c.k_max.cuda(), c.gpu[2], c.glens, 30, hint)
    check_lists(sel, n_sel, ref.select(q, c.k_min, c.k_max, c.table, lens, 30), 30)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gone", ["one", "half", "all but few", "all but as many", "all", "all but few alike", "all but first and last"])
@pytest.mark.parametrize("N,K", [(60, 9), (700, 60), (2500, 130), (9000, 300)])
def test_selection_from_tables_with_pages_that_are_gone(dtype, gone, N, K):
    lo, hi = score_cache("equal" if gone == "all but few alike" else "plain", dtype, N)
    table = torch.tensor([random.Random(N).sample(range(N), N)], dtype=torch.int32)
    stay = {"one": N - 1, "half": N // 2, "all but few": K // 2, "all but as many": K, "all": 0, "all but few alike": K // 2, "all but first and last": 2}[gone]
    away = random.Random(K).sample(range(1, N - 1), N - 2)[:N - stay] if stay else list(range(N))
    table[0, away] = torch.tensor([[-1, N, 2 ** 31 - 1, -2 ** 31][i % 4] for i in range(len(away))], dtype=torch.int32)
    q = torch.randn(1, 3, 64, generator=torch.Generator().manual_seed(1)).to(DT[dtype])
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32([N * PAGE]), K, N * PAGE)
    at, rows = table[0].long(), ref.pages_of(N * PAGE)
    live = (at >= 0) & (at < N)
    x, a, b = q[0].double(), lo[at.clamp(0, N - 1), 0].double(), hi[at.clamp(0, N - 1), 0].double()
    score = torch.where(live, (x.clamp(min=0) @ b.T + x.clamp(max=0) @ a.T).amax(0), -math.inf)
    score[0] = score[-1] = math.inf
    want = torch.sort(torch.sort(score, descending=True, stable=True).indices[:K]).values
    assert rows == N and sel[0, 0].tolist() == want.tolist() and n_sel.tolist() == [K]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K", [(40, 9), (700, 60), (3001, 130)])
@pytest.mark.parametrize("power", [-72, -66, -60])
def test_selection_where_products_underflow(dtype, N, K, power):
    lo, hi = score_cache("plain", dtype, N)
    lo, hi = lo * 2.0 ** power, hi * 2.0 ** power
    table = torch.arange(N, dtype=torch.int32)[None]
    q = torch.randn(1, 3, 64, generator=torch.Generator().manual_seed(2)).to(DT[dtype]) * 2.0 ** power
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32([N * PAGE]), K, N * PAGE)
    check_lists(sel, n_sel, ref.select(q, lo, hi, table, [N * PAGE], K), K)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K", [(40, 9), (700, 60)])
@pytest.mark.parametrize("bad,query", [(-math.inf, 0.0), (-math.inf, -0.0), (math.nan, 0.0), (math.nan, 1.0)])
def test_selection_with_an_infinity_or_nan_on_the_side_that_does_not_count(dtype, N, K, bad, query):
    lo, hi = score_cache("plain", dtype, N)
    lo[7, :, 3] = bad
    table = torch.arange(N, dtype=torch.int32)[None]
    q = torch.randn(1, 3, 64, generator=torch.Generator().manual_seed(2)).to(DT[dtype])
    q[0, :, 3] = q[0, :, 3].abs()
    q[0, 1, 3] = query
    want = ref.select(q, lo, hi, table, [N * PAGE], K)
    assert 7 in want[0][0]
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32([N * PAGE]), K, N * PAGE)
    check_lists(sel, n_sel, want, K)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("N", [60, 700])
def test_fp32_selection_with_queries_that_are_not_finite(bad, N):
    lo, hi = score_cache("plain", "fp32", N)
    lo[5, :, 5] = hi[5, :, 5] = 0.0
    table, lens = torch.arange(N, dtype=torch.int32)[None].repeat(2, 1), [N * PAGE, N * PAGE - 3]
    q = torch.randn(2, 12, 64, generator=torch.Generator().manual_seed(1))
    q[1, 7, 5] = bad
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32(lens), 50, N * PAGE)
    check_lists(sel, n_sel, ref.select(q, lo, hi, table, lens, 50), 50)


def test_selection_with_queries_that_are_not_finite_and_pages_outside_the_pool():
    lo, hi = score_cache("plain", "bf16", 500)
    table = torch.arange(500, dtype=torch.int32)[None].repeat(2, 1)
    table[0, 100:120], table[1, 3] = -1, 500
    lens = [500 * PAGE, 300 * PAGE]
    q = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16()
    for bad in (0.0, math.nan, math.inf):
        q[1, 0, 5] = bad
        sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32(lens), 50, 8000)
        check_lists(sel, n_sel, ref.select(q, lo, hi, table, lens, 50), 50)


# ---------------------------------------------------------------------------------------------- together


class Serving:
    """A serving loop's cache on the GPU, and what it should hold as plain rows per request."""

    def __init__(self, B, Hk, D, dtype, n_pages, max_pages, seed):
        self.B, self.Hk, self.D, self.dt = B, Hk, D, DT[dtype]
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.state = [torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda"),
                      torch.randperm(n_pages, device="cuda", generator=self.g).to(torch.int32), i32([n_pages])]
        z = dict(dtype=self.dt, device="cuda")
        self.k_pool, self.v_pool = torch.full((n_pages, Hk, PAGE, D), math.nan, **z), torch.full((n_pages, Hk, PAGE, D), math.nan, **z)
        self.k_min, self.k_max = torch.full((n_pages, Hk, D), math.nan, **z), torch.full((n_pages, Hk, D), math.nan, **z)

    def normal(self, *size):
        return torch.empty(*size, dtype=self.dt, device="cuda").normal_(generator=self.g)

    def step(self, n_new, k, v, rows):
        p = binding.pages_plan(n_new, *self.state, rows)
        binding.kv_append(k, v, p.slot, self.k_pool, self.v_pool, self.k_min, self.k_max)
        return p

    def decode(self, q, n_pages, max_len):
        lens, table = self.state[:2]
        dense = binding.paged_attention(q, self.k_pool, self.v_pool, table, lens, 0.2, max_len)
        sel, n_sel = binding.page_select(q, self.k_min, self.k_max, table, lens, n_pages, max_len)
        sparse = binding.paged_attention(q, self.k_pool, self.v_pool, table, lens, 0.2, max_len, sel=sel, n_sel=n_sel)
        return dense, sel, n_sel, sparse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_serving_loop(dtype):
    """Requests come, decode, are cut back, end and come again in a pool that is too small for all of them; every step's attention, dense and over selected
    pages, against the rows that each request should have."""
    rng = random.Random(3)
    B, Hk, G, D, K = 6, 2, 4, 64, 5
    s = Serving(B, Hk, D, dtype, 60, 24, 9)
    k_rows, v_rows = [[] for _ in range(B)], [[] for _ in range(B)]
    refused = 0
    for step in range(24):
        n_new = [rng.choice([1, 1, 1, 0, rng.randint(1, 90)]) if k_rows[b] else rng.randint(0, 150) for b in range(B)]
        total = sum(n_new)
        k, v = s.normal(total + 7, Hk, D), s.normal(total + 7, Hk, D)
        p = s.step(i32(n_new), k, v, total + 7)
        granted = p.granted.tolist()
        row = 0
        for b, n in enumerate(n_new):
            if granted[b]:
                k_rows[b] += list(k[row:row + n].cpu())
                v_rows[b] += list(v[row:row + n].cpu())
            refused += n > 0 and not granted[b]
            row += n
        lens = [len(x) for x in k_rows]
        assert s.state[0].tolist() == lens
        q = s.normal(B, Hk * G, D)
        dense, sel, n_sel, sparse = s.decode(q, K, 400)
        # the rows as a cache of the plain implementation, page after page
        pages = [ref.pages_of(n) for n in lens]
        table = torch.full((B, 24), -1)
        kp, vp = torch.zeros(sum(pages) + 1, Hk, PAGE, D, dtype=s.dt), torch.zeros(sum(pages) + 1, Hk, PAGE, D, dtype=s.dt)
        at = 0
        for b in range(B):
            for j in range(pages[b]):
                table[b, j] = at
                for i, (x, y) in enumerate(zip(k_rows[b][j * PAGE:(j + 1) * PAGE], v_rows[b][j * PAGE:(j + 1) * PAGE])):
                    kp[at, :, i], vp[at, :, i] = x, y
                at += 1
        check(*dense, ref.attention(q.cpu(), kp, vp, table, lens, 0.2))
        lists = [[[x for x in sel[b, h].tolist() if x >= 0] for h in range(Hk)] for b in range(B)]
        for b in range(B):
            for h in range(Hk):
                want = min(pages[b], K)
                assert len(lists[b][h]) == want == int(n_sel[b])
                assert not want or (lists[b][h][0] == 0 and lists[b][h][-1] == pages[b] - 1)
        check(*sparse, ref.attention(q.cpu(), kp, vp, table, lens, 0.2, sel=lists))
        # the lists are those of the summaries that the appends have left
        check_lists(sel, n_sel, ref.select(q.cpu(), s.k_min.cpu(), s.k_max.cpu(), s.state[1].cpu(), lens, K), K)
        keep = [rng.choice([n, n, n, 0 if step % 5 == 4 else n, max(0, n - rng.randint(0, 20))]) for n in lens]
        binding.pages_trim(i32(keep), *s.state)
        for b in range(B):
            del k_rows[b][keep[b]:], v_rows[b][keep[b]:]
        held = sum(ref.pages_of(len(x)) for x in k_rows)
        assert int(s.state[3]) == 60 - held
    assert refused


def test_a_captured_step_replays_as_the_requests_grow():
    B, Hk, G, D = 4, 2, 8, 128
    s, t = (Serving(B, Hk, D, "bf16", 400, 100, 1) for _ in range(2))
    prompt = [700, 3, 0, 90]
    k, v = s.normal(793, Hk, D), s.normal(793, Hk, D)
    for x in (s, t):
        x.step(i32(prompt), k, v, 793)
    one = i32([1] * B)
    feed = [s.normal(B, Hk, D), s.normal(B, Hk, D), s.normal(B, Hk * G, D)]

    def run(x):
        x.step(one, feed[0], feed[1], B)
        return x.decode(feed[2], 6, 1024)

    for x in (s, t):
        run(x)                                               # (first calls set kernels up: outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(s)
    for _ in range(20):
        for f in feed:
            f.normal_(generator=s.g)
        graph.replay()
        want = run(t)
        torch.cuda.synchronize()
        flat = lambda r: [*r[0], r[1], r[2], *r[3]]
        for a, b in zip(flat(held), flat(want)):
            assert torch.equal(a, b)
        for a, b in zip(s.state + [s.k_min[s.state[1][0, :44].long()]], t.state + [t.k_min[t.state[1][0, :44].long()]]):
            assert torch.equal(a, b)
    assert s.state[0].tolist() == [n + 21 for n in prompt]


def test_tree_attention_right_behind_an_append_and_a_plan():
    """The library's tree attention reads lengths, tables and committed keys ahead of its wait for the kernel in front: behind the calls that change them
    it must find them changed."""
    B, H, D, mp = 4, 8, 128, 40
    g = torch.Generator(device="cuda").manual_seed(4)

    def normal(*size):
        return torch.empty(*size, dtype=torch.bfloat16, device="cuda").normal_(generator=g)

    k_pool, v_pool = normal(B * mp, H, PAGE, D), normal(B * mp, H, PAGE, D)
    one = torch.tensor([[1, 0, 0]], dtype=torch.int64, device="cuda")
    for step in range(12):
        state = [torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, mp, dtype=torch.int32, device="cuda"),
                 torch.randperm(B * mp, device="cuda", generator=g).to(torch.int32), i32([B * mp])]
        lens = [37 + 50 * b + step for b in range(B)]
        rows = sum(lens)
        k, v, q = normal(rows, H, D), normal(rows, H, D), normal(B, 1, H, D)
        n_new, less = i32(lens), i32([n - 1 for n in lens])
        _, _, scratch = binding.tree_attention(q, k_pool, v_pool, state[1], state[0], one, 0.1, max(lens))
        torch.cuda.synchronize()
        p = binding.pages_plan(n_new, *state, rows)
        # a tree of one node sits behind the committed keys: the last token's key is its own
        binding.kv_append(k, v, p.slot, k_pool, v_pool)
        late, _, _ = binding.tree_attention(q, k_pool, v_pool, state[1], less, one, 0.1, max(lens), scratch=scratch)
        state[0].copy_(less)
        keep = less.clone()
        torch.cuda.synchronize()
        binding.pages_plan(i32([0] * B), *state, 0)
        again, _, _ = binding.tree_attention(q, k_pool, v_pool, state[1], keep, one, 0.1, max(lens), scratch=scratch)
        own, _ = binding.paged_attention(q[:, 0], k_pool, v_pool, state[1], n_new, 0.1, max(lens))
        assert torch.equal(late, again), step
        assert float((late[:, 0].float() - own.float()).abs().max()) < 0.03, step      # (two kernels: each within 2^-8 of its weights and its result, values of 3 to 4)


def test_operands_with_strides_of_their_own():
    c = Cache([300], 1, 64, "bf16", 71)
    q, gq = c.queries(8, 6)
    want = ref.attention(q[:, ::2], c.k_pool, c.v_pool, c.table, [300], 0.1)
    check(*binding.paged_attention(gq[:, ::2], *c.gpu, c.glens, 0.1, 300), want)
    # dimensions of one: any stride will do
    odd = torch.empty(5000, dtype=torch.bfloat16, device="cuda")
    one = odd[:64].copy_(gq[0, 3]).as_strided((1, 1, 64), (3, 7, 1))
    check(*binding.paged_attention(one, *c.gpu, c.glens, 0.1, 300), ref.attention(q[:, 3:4], c.k_pool, c.v_pool, c.table, [300], 0.1))
    pool = [torch.zeros(2, 1, PAGE, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.kv_append(one, one, i32([17]), *pool)
    assert torch.equal(pool[0][1, 0, 1], gq[0, 3]) and int((pool[1] != 0).sum()) == int((gq[0, 3] != 0).sum())
    # the same key for every row of a call
    row = gq[0, 2:3][None].expand(5, 1, 64)
    binding.kv_append(row, row, i32([0, 1, 2, -1, 4]), *pool)
    assert torch.equal(pool[0][0, 0, :5], torch.stack([gq[0, 2]] * 3 + [torch.zeros_like(gq[0, 2]), gq[0, 2]]))
    # not on 16 bytes
    for bad in (odd[1:65].view(1, 1, 64), odd[:2 * 68].view(2, 1, 68)[:, :, :64]):
        with pytest.raises(binding.CerbError) as e:
            binding.kv_append(bad, bad, i32([0] * bad.shape[0]), *pool)
        assert e.value.code == binding.E_ARG


def test_calls_on_another_stream():
    c = Cache([3000, 70, 0], 2, 64, "bf16", 51)
    _, gq = c.queries(8, 6)
    lo, hi = c.k_min.cuda(), c.k_max.cuda()
    want = binding.paged_attention(gq, *c.gpu, c.glens, 0.1, 3000) + binding.page_select(gq, lo, hi, c.gpu[2], c.glens, 9, 3000)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(binding.paged_attention(gq, *c.gpu, c.glens, 0.1, 3000) + binding.page_select(gq, lo, hi, c.gpu[2], c.glens, 9, 3000))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_refusals_of_tensors_that_do_not_belong_together():
    c = Cache([40, 50], 2, 64, "bf16", 61)
    _, q = c.queries(4, 6)
    lo, hi = c.k_min.cuda(), c.k_max.cuda()
    k_pool, v_pool, table = c.gpu
    sel, n_sel = binding.page_select(q, lo, hi, table, c.glens, 2, 50)
    slot, rows = i32([0, 1]), q[:, :2]
    book = [i32([0, 0]), i32([[-1], [-1]]), i32([0, 1]), i32([2])]
    bad = [
        lambda: binding.paged_attention(q.float(), k_pool, v_pool, table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q[:, :3], k_pool, v_pool, table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q[..., :32], k_pool, v_pool, table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q.transpose(0, 1), k_pool, v_pool, table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q, k_pool, v_pool[1:], table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q, k_pool[:, :, :8], v_pool[:, :, :8], table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q, k_pool.half(), v_pool.half(), table, c.glens, 1.0, 50),
        lambda: binding.paged_attention(q, k_pool, v_pool, table[:, ::2], c.glens, 1.0, 50),
        lambda: binding.paged_attention(q, k_pool, v_pool, table, c.glens.long(), 1.0, 50),
        lambda: binding.paged_attention(q, k_pool, v_pool, table, c.glens[:1], 1.0, 50),
        lambda: binding.paged_attention(q, k_pool, v_pool, table.cpu(), c.glens, 1.0, 50),
        lambda: binding.paged_attention(q, k_pool, v_pool, table, c.glens, 1.0, 0),
        lambda: binding.paged_attention(q, k_pool, v_pool, table, c.glens, 1.0, 50, window=-1),
        lambda: binding.paged_attention(q, k_pool, v_pool, table, c.glens, 1.0, 50, sel=sel),
        lambda: binding.paged_attention(q, k_pool, v_pool, table, c.glens, 1.0, 50, sel=sel[:, :1], n_sel=n_sel),
        lambda: binding.page_select(q, lo, hi[1:], table, c.glens, 2, 50),
        lambda: binding.page_select(q, lo, hi, table, c.glens, 0, 50),
        lambda: binding.page_select(q, lo.half(), hi.half(), table, c.glens, 2, 50),
        lambda: binding.kv_append(rows, rows, slot[:1], k_pool, v_pool),
        lambda: binding.kv_append(rows, rows, slot.long(), k_pool, v_pool),
        lambda: binding.kv_append(rows, rows, slot, k_pool, v_pool, lo),
        lambda: binding.kv_append(rows, rows, slot, k_pool, v_pool, lo[1:], hi[1:]),
        lambda: binding.kv_append(q, q, slot, k_pool, v_pool),
        lambda: binding.pages_plan(i32([1]), *book, 4),
        lambda: binding.pages_plan(i32([1, 1]), *book, -1),
        lambda: binding.pages_plan(i32([1, 1]), book[0], book[1], book[2], i32([1, 2]), 4),
        lambda: binding.pages_trim(i32([1, 1]), book[0], book[1][:1], *book[2:]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.CerbError) as e:
            call()
        assert e.value.code == binding.E_ARG, i
    for call in (lambda: binding.page_select(q, lo, hi, table, c.glens, 2, 50, 2, 1), lambda: binding.pages_plan(i32([1, 1]), *book, (1 << 30) + 1)):
        with pytest.raises(binding.CerbError) as e:
            call()
        assert e.value.code == binding.E_SHAPE
