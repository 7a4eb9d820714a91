"""Paged-cache operators at the ends of their ranges, against the plain implementations in 64 bits (paged_reference.py)."""
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2410_13344_b200 import binding
from test_gpu_paged import score_cache

pytestmark = pytest.mark.gpu
PAGE = 16
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check_lists(sel, n_sel, want, K):
    for b, rows in enumerate(want):
        assert int(n_sel[b]) == len(rows[0])
        for h, row in enumerate(rows):
            assert sel[b, h].tolist() == row + [-1] * (K - len(row)), (b, h)


# ---------------------------------------------------------------------------------------------- selection


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,G,K", [(20, 8, 4), (34, 4, 20), (34, 4, 9), (40, 4, 9), (300, 2, 60), (3001, 3, 130)])
@pytest.mark.parametrize("kind", ["one each", "both ways", "one side"])
def test_selection_where_finite_scores_span_more_than_fp32_holds(dtype, N, G, K, kind):
    g = torch.Generator().manual_seed(N)
    mid, spread = torch.randn(N, 1, 64, generator=g), torch.rand(N, 1, 64, generator=g)
    lo, hi = mid - spread, mid + spread
    # one channel, in which every query is 1: scores stay finite
    if kind == "one each":
        lo[N // 3, 0, 9] = hi[N // 3, 0, 9] = 3e38
        lo[N // 2, 0, 9] = hi[N // 2, 0, 9] = -3e38
    else:
        size = 2e38 + 1.2e38 * torch.rand(N, generator=g)
        sign = torch.where(torch.rand(N, generator=g) < 0.5, -1.0, 1.0) if kind == "both ways" else 1.0
        lo[:, 0, 9] = hi[:, 0, 9] = size * sign
    lo, hi = lo.to(DT[dtype]), hi.to(DT[dtype])
    q = torch.randn(1, G, 64, generator=torch.Generator().manual_seed(1)).to(DT[dtype])
    q[:, :, 9] = 1.0
    table = torch.tensor([random.Random(N).sample(range(N), N)], dtype=torch.int32)
    x, at = q[0].double(), table[0].long()
    scores = (x.clamp(min=0) @ hi[at, 0].double().T + x.clamp(max=0) @ lo[at, 0].double().T).float()
    assert bool(torch.isfinite(scores).all())
    assert kind == "one side" or bool(torch.isinf(scores.amax() - scores.amin()))
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32([N * PAGE]), K, N * PAGE)
    check_lists(sel, n_sel, ref.select(q, lo, hi, table, [N * PAGE], K), K)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["plain", "equal", "zero", "few values", "near", "outliers", "channel", "odd", "huge"])
@pytest.mark.parametrize("G", [4, 9])                         # (three heads of forty pages are all scored in 64 bits: these are not)
def test_selection_from_few_pages_by_their_scores(dtype, kind, G):
    N, K = 40, 9
    lo, hi = score_cache(kind, dtype, N)
    table = torch.tensor([random.Random(N).sample(range(N), N)], dtype=torch.int32)
    for power in (0, -60, -66, -72):
        if power and kind != "plain":
            continue
        a, b = lo * 2.0 ** power, hi * 2.0 ** power
        q = torch.randn(1, G, 64, generator=torch.Generator().manual_seed(1)).to(DT[dtype]) * 2.0 ** power
        sel, n_sel = binding.page_select(q.cuda(), a.cuda(), b.cuda(), table.cuda(), i32([N * PAGE - 5]), K, N * PAGE - 5)
        check_lists(sel, n_sel, ref.select(q, a, b, table, [N * PAGE - 5], K), K)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad,query", [(-math.inf, 0.0), (-math.inf, -0.0), (math.nan, 0.0), (math.nan, 1.0), (math.inf, 1.0), (-math.inf, -1.0)])
def test_selection_from_few_pages_with_an_infinity_or_nan(dtype, bad, query):
    lo, hi = score_cache("plain", dtype, 40)
    lo[7, :, 3] = bad
    if bad == math.inf:
        hi[7, :, 3] = bad
    table = torch.arange(40, dtype=torch.int32)[None]
    q = torch.randn(1, 5, 64, generator=torch.Generator().manual_seed(2)).to(DT[dtype])
    q[0, :, 3] = q[0, :, 3].abs()
    q[0, 1, 3] = query
    sel, n_sel = binding.page_select(q.cuda(), lo.cuda(), hi.cuda(), table.cuda(), i32([640]), 9, 640)
    check_lists(sel, n_sel, ref.select(q, lo, hi, table, [640], 9), 9)


# ---------------------------------------------------------------------------------------------- attention


def test_attention_over_lists_of_nearly_2_to_the_32_entries():
    """Four thousand heads share a list of 2^24 - 1 entries, of which twenty are pages: 256 units, 2^32 - 256 items in all."""
    H, D, K, length = 4096, 64, (1 << 24) - 1, 16 * 20 - 3
    g = torch.Generator().manual_seed(1)
    k_pool, v_pool = (torch.randn(20, 1, PAGE, D, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(1, H, D, generator=g).bfloat16()
    table = torch.randperm(20, generator=g).to(torch.int32)[None]
    sel = torch.full((1, 1, K), -1, dtype=torch.int32)
    at = random.Random(1).sample(range(K), 16) + [0, K - 1, K // 2, 14510163]
    assert len(set(at)) == 20
    sel[0, 0, at] = torch.arange(20, dtype=torch.int32)
    out, lse = binding.paged_attention(q.cuda(), k_pool.cuda(), v_pool.cuda(), table.cuda(), i32([length]), 0.125, 1 << 28, sel=sel.cuda(), n_sel=i32([K]))
    o, l, (to, tl) = ref.attention(q, k_pool, v_pool, table, [length], 0.125)
    assert bool(((out.double().cpu() - o).abs() <= to).all()) and bool(((lse.double().cpu() - l).abs() <= tl).all())


def test_an_idle_sequence_of_2_to_the_31_outputs():
    H, D = 1 << 24, 128
    q = torch.ones(1, 1, D, dtype=torch.bfloat16, device="cuda").expand(1, H, D)
    pool = torch.ones(1, 1, PAGE, D, dtype=torch.bfloat16, device="cuda")
    before = torch.full((6 << 30,), 255, dtype=torch.uint8, device="cuda")                  # (what the results' memory may hold)
    del before
    out, lse = binding.paged_attention(q, pool, pool, i32([[0]]), i32([0]), 0.1, 60000)
    assert not bool(out.view(torch.int16).any()) and bool(torch.isneginf(lse).all())
    del out, lse
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------------------------- pages


def test_trim_of_nearly_2_to_the_31_pages():
    B, each = 33, 65075262
    total = B * each                                        # 2^31 - 2
    table = torch.arange(total, dtype=torch.int32, device="cuda").remainder_(1 << 27).view(B, each)
    free = torch.full((total + 1,), -5, dtype=torch.int32, device="cuda")
    lens, n_free = i32([each * PAGE] * B), i32([1])
    binding.pages_trim(i32([0] * B), lens, table, free, n_free)
    assert n_free.tolist() == [total + 1] and not bool(lens.any()) and int(free[0]) == -5
    assert bool((table == -1).all())
    del table
    for lo in range(0, total, 1 << 28):                     # page i of the table lies total - i above the bottom
        hi = min(total, lo + (1 << 28))
        want = torch.arange(lo, hi, dtype=torch.int32, device="cuda").remainder_(1 << 27)
        assert torch.equal(free[total - hi + 1:total - lo + 1].flip(0), want)
    del free
    torch.cuda.empty_cache()


@pytest.mark.parametrize("B,max_pages,context,gone", [(1, 3, 40, 1.0), (3, 8, 120, 0.5), (40, 30, 450, 0.3), (300, 60, 900, 0.02), (2049, 40, 600, 0.5), (5, 9000, 140000, 0.4), (3, 9000, 140000, 0.0002),
                                                      (1200, 50, 700, 0.0)])
def test_trim_passes_over_entries_that_are_no_page(B, max_pages, context, gone):
    """Requests whose old pages have been given back by hand, as behind a window: the stack has room for every page once, and gets every page once."""
    rng = random.Random(B * 7 + max_pages)
    lens = [rng.choice([0, context, rng.randint(0, context)]) for _ in range(B)]
    lens[-1] = context
    held = [ref.pages_of(n) for n in lens]
    n_pages = sum(held) + 50
    pool = rng.sample(range(n_pages), n_pages)
    table = [[pool.pop() for _ in range(h)] + [-1] * (max_pages - h) for h in held]
    free = pool
    for b, h in enumerate(held):
        for j in range(h - 1):
            if rng.random() < gone:
                free.append(table[b][j])
                table[b][j] = rng.choice([-1, -1, -2 ** 31, 2 ** 27, 2 ** 31 - 1])
    n_free = len(free)
    free = free + [-3] * (n_pages - n_free)
    state = [i32(lens), i32(table).view(B, max_pages), i32(free), i32([n_free])]
    for keep in ([rng.choice([n, max(0, n - 3), rng.randint(0, n), n // 2]) for n in lens], [0] * B):
        binding.pages_trim(i32(keep), *state)
        back = []
        for b, n in enumerate(keep):
            n = min(n, lens[b])
            for j in range(ref.pages_of(n), ref.pages_of(lens[b])):
                if 0 <= table[b][j] < 2 ** 27:
                    back.append(table[b][j])
                table[b][j] = -1
            lens[b] = n
        free[n_free:n_free + len(back)] = back[::-1]
        n_free += len(back)
        assert state[0].tolist() == lens and state[1].tolist() == table and state[3].tolist() == [n_free]
        assert state[2].tolist()[:n_free] == free[:n_free]
        # what a plan then hands out are pages
        new = [1] * B
        plan = binding.pages_plan(i32(new), *[t.clone() for t in state], B)
        whole = [b for b in range(B) if lens[b] % PAGE == 0 and int(plan.granted[b])] if B < 50 else []
        assert all(int(plan.slot[b]) >= 0 for b in whole)
    assert sorted(free) == list(range(n_pages))


@pytest.mark.parametrize("rows", [4, 600, 5000])              # one CTA of few threads, one of many, many CTAs
def test_a_plan_changes_the_lengths_of_those_that_get_tokens(rows):
    lens, table = i32([-5, 1000, 20, 7, -5, 1000]), i32([[-1] * 3, [5, 6, 7], [8, 9, -1], [10, -1, -1], [-1] * 3, [11, 12, 13]])
    free, n_free = i32([1, 2, 3]), i32([100])
    plan = binding.pages_plan(i32([0, 0, 0, 1, 1, 1]), lens, table, free, n_free, rows)
    assert plan.granted.tolist() == [0, 0, 0, 1, 1, 0] and plan.slot.tolist() == [10 * 16 + 7, 3 * 16, -1] + [-1] * (rows - 3)
    assert lens.tolist() == [-5, 1000, 20, 8, 1, 1000] and n_free.tolist() == [2]


# ---------------------------------------------------------------------------------------------- append


@pytest.mark.parametrize("dtype,T,Hk,D", [("bf16", 5003, 8, 64), ("bf16", 10007, 8, 64), ("fp32", 6001, 8, 64), ("bf16", 6001, 8, 128), ("fp32", 3001, 8, 128)])
def test_append_in_windows_of_up_to_a_page(dtype, T, Hk, D):
    """Rows of the list that a group of threads looks through at a time: as many as let all groups run at once, 9 in the first case, a page in the others."""
    lanes = D * DT[dtype].itemsize // 16
    block = min(PAGE, -(-2 * T * Hk * lanes // (148 * 512)))
    assert block == (9 if T == 5003 else PAGE)
    rng = random.Random(T)
    n_pages = T // 4
    pages, slots = rng.sample(range(n_pages), n_pages), []
    while len(slots) < T:
        kind = rng.random()
        if kind < 0.15:
            slots += [rng.choice([-1, -9, n_pages * PAGE, 2 ** 31 - 1])] * rng.choice([1, 1, 2, 5])
            continue
        page, start = pages.pop(), rng.choice([0, 0, rng.randrange(PAGE)])
        n = rng.choice([1, PAGE - start, rng.randint(1, PAGE - start)])
        slots += [page * PAGE + start + i for i in range(n)]
    slots = slots[:T]
    g = torch.Generator().manual_seed(T)
    k, v = (torch.randn(T, Hk, D, generator=g).to(DT[dtype]) for _ in range(2))
    cpu = [torch.randn(n_pages, Hk, PAGE, D, generator=g).to(DT[dtype]) for _ in range(2)]
    cpu += [cpu[0].amin(2), cpu[0].amax(2)]
    gpu = [t.cuda() for t in cpu]
    binding.kv_append(k.cuda(), v.cuda(), i32(slots), *gpu)
    ref.append(k, v, slots, *cpu)
    for got, want in zip(gpu, cpu):
        assert torch.equal(got.cpu(), want)
