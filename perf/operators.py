"""The paged-cache operators that are timed: what a serving loop calls between and inside its layers.

pages      page tables, slots and positions of a step's tokens, built on the GPU from the requests' lengths (and the trim that
           gives pages back, which makes a pass repeatable)
append     a step's keys and values into their slots, with the per-page minimum and maximum of the keys
attention  one new token per sequence over the paged cache, query heads sharing KV heads
sparse     the same over the pages that a score from those minima and maxima selects

A case is a dict of plain values.  `prepare` makes what a serving program has in hand, `run` is one pass: with `own` set
through the public entry points of paper_2410_13344_b200.binding, otherwise in elementary torch operations.  `exact` states
the operators once more in 64 bits.
"""
import math

import torch

own = False

PAGE = 16                     # tokens of a page
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ROWS_PAD = 64                 # a step's row buffers are padded to a multiple of this, as captured steps are


def listed():
    return [
        # 64 running requests, one new token each: what every decoding step starts with.  Launch latency.
        dict(name="pages decode x64", kind="pages", requests=64, context=2048, new="one", chunk=1, spare=1.0),
        # A scheduler's step of chunked prefill: most requests decode, one in eight brings up to 512 prompt tokens.
        dict(name="pages mixed x300", kind="pages", requests=300, context=1900, new="mixed", chunk=512, spare=1.0),
        # Admission of many prompts at once with too few free pages for all of them.
        dict(name="pages prompts x2000 short of pages", kind="pages", requests=2000, context=0, new="prompts", chunk=900, spare=0.8),
        # One decoding step's keys, each into a page of its own, out of a packed QKV product.
        dict(name="append decode x64", kind="append", tokens=64, kv_heads=8, head_dim=128, dtype="bf16", runs="decode"),
        # The same of a chunk of ragged prompts: runs that begin and end inside pages.
        dict(name="append prompts 16000", kind="append", tokens=16000, kv_heads=8, head_dim=128, dtype="bf16", runs="prompts"),
        # fp32, heads of 64, an odd number of tokens.
        dict(name="append prompts 1537 fp32", kind="append", tokens=1537, kv_heads=5, head_dim=64, dtype="fp32", runs="prompts"),
        # One conversation: the latency of a layer.
        dict(name="attention x1 1k", kind="attention", batch=1, heads=32, kv_heads=8, head_dim=128, dtype="bf16", context=1000, window=0),
        # A full batch of ragged conversations (some slots idle): bandwidth.
        dict(name="attention x64 8k", kind="attention", batch=64, heads=64, kv_heads=8, head_dim=128, dtype="bf16", context=8192, window=0),
        # Few long contexts behind a sliding window, five query heads to a KV head, heads of 64.
        dict(name="attention x7 window", kind="attention", batch=7, heads=40, kv_heads=8, head_dim=64, dtype="bf16", context=50001, window=16001),
        # fp32, every query head with a KV head of its own.
        dict(name="attention x4 fp32", kind="attention", batch=4, heads=32, kv_heads=32, head_dim=128, dtype="fp32", context=1500, window=0),
        # One very long context, 256 of its 8192 pages read.
        dict(name="sparse x1 128k", kind="sparse", batch=1, heads=32, kv_heads=8, head_dim=128, dtype="bf16", context=131072, pages=256),
        # A batch of long contexts, ragged, 128 pages each.
        dict(name="sparse x24 32k", kind="sparse", batch=24, heads=32, kv_heads=8, head_dim=128, dtype="bf16", context=32000, pages=128),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["pages", "append", "attention", "attention", "sparse", "sparse"])
    if kind == "pages":
        new = rng.choice(["one", "mixed", "prompts"])
        return dict(kind=kind, requests=log_int(1, 2000), context=0 if new == "prompts" else log_int(1, 8000), new=new,
                    chunk=1 if new == "one" else log_int(2, 900), spare=rng.choice([1.0, 1.0, 0.5, 0.9]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 8])
    if kind == "append":
        return dict(kind=kind, tokens=log_int(1, 8000 if dtype == "fp32" else 16000), kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
                    runs=rng.choice(["decode", "prompts"]))
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 12, 16])
    if kind == "attention" and rng.random() < 0.2:
        kv_heads, group = rng.choice([32, 40]), 1
    heads = kv_heads * group
    batch = log_int(1, 128)
    # of the keys of the largest listed cases
    keys = (64 * 8 * 8192 if kind == "attention" else 24 * 8 * 32000) // kv_heads // (2 if dtype == "fp32" else 1)
    longest = max(1, min(131072, keys // batch))
    c = dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, context=log_int(1, longest))
    if kind == "sparse":
        c["pages"] = log_int(2, 256)
    else:
        c["window"] = rng.choice([0, 0, log_int(1, max(2, c["context"]))])
    return c


# ---------------------------------------------------------------------------------------------- inputs


class _State:
    pass


def _ceil(a, b):
    return (a + b - 1) // b


def _generators(seed):
    host = torch.Generator()
    host.manual_seed(seed)
    dev = torch.Generator(device="cuda")
    dev.manual_seed(seed)
    return host, dev


def prepare(case, seed):
    host, dev = _generators(seed)
    s = _State()
    s.case = case
    {"pages": _prepare_pages, "append": _prepare_append, "attention": _prepare_attention, "sparse": _prepare_attention}[case["kind"]](s, case, host, dev)
    return s


def _prepare_pages(s, c, host, dev):
    B = c["requests"]
    lens = torch.randint(0, 2 * c["context"] + 1, (B,), generator=host)
    if c["new"] == "one":
        n_new = torch.ones(B, dtype=torch.int64)
    else:
        n_new = torch.randint(1, c["chunk"] + 1, (B,), generator=host)
        if c["new"] == "mixed":
            n_new = torch.where(torch.rand(B, generator=host) < 1 / 8, n_new, torch.ones_like(n_new))
    held = _ceil(lens, PAGE)
    need = _ceil(lens + n_new, PAGE) - held
    max_pages = _ceil(2 * c["context"] + c["chunk"], PAGE)
    n_held = int(held.sum())
    n_free = int(c["spare"] * int(need.sum()))
    pool = torch.randperm(B * max_pages, generator=host).to(torch.int32)            # (some of its pages belong to nobody)
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    table[torch.arange(max_pages)[None, :] < held[:, None]] = pool[:n_held]
    free = torch.full((pool.numel(),), -1, dtype=torch.int32)
    free[:n_free] = pool[n_held:n_held + n_free]
    # the step's row buffers: what the requests bring on average and an eighth more (a step that brings more leaves its last ones out)
    s.rows = _ceil(int(1.125 * _mean_rows(c)), ROWS_PAD) * ROWS_PAD
    s.base = lens.to(torch.int32).cuda()
    s.lens = s.base.clone()
    s.n_new = n_new.to(torch.int32).cuda()
    s.page_table = table.cuda()
    s.free_pages = free.cuda()
    s.n_free = torch.tensor([n_free], dtype=torch.int32).cuda()


def _mean_rows(c):
    return c["requests"] * {"one": 1.0, "mixed": 7 / 8 + (c["chunk"] + 1) / 16, "prompts": (c["chunk"] + 1) / 2}[c["new"]]


def _prepare_append(s, c, host, dev):
    T, Hk, D, dt = c["tokens"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    # where the runs of consecutive tokens begin inside their first pages, and how long they are
    if c["runs"] == "decode":
        start, length = torch.randint(0, 2 * PAGE, (T,), generator=host), torch.ones(T, dtype=torch.int64)
    else:
        n = max(1, T // 300)
        cuts = torch.sort(torch.randint(0, T + 1, (n - 1,), generator=host)).values
        edges = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([T])])
        length = edges[1:] - edges[:-1]
        start = torch.randint(0, 2 * PAGE, (n,), generator=host)
        start[torch.rand(n, generator=host) < 0.5] = 0            # half of them are new requests
    first = torch.cumsum(_ceil(start + length, PAGE), 0) - _ceil(start + length, PAGE)
    n_pages = T // PAGE + 4 * length.numel() + 3
    page_of = torch.randperm(n_pages, generator=host)
    run = torch.repeat_interleave(torch.arange(length.numel()), length)
    at = start[run] + torch.arange(T) - (torch.cumsum(length, 0) - length)[run]
    slot = page_of[first[run] + at // PAGE] * PAGE + at % PAGE
    rows = _ceil(T, ROWS_PAD) * ROWS_PAD
    s.slot = torch.full((rows,), -1, dtype=torch.int32)
    s.slot[:T] = slot.to(torch.int32)
    s.slot = s.slot.cuda()
    H = 4 * Hk
    qkv = torch.empty(rows, (H + 2 * Hk) * D, dtype=dt, device="cuda").normal_(generator=dev)
    s.k = qkv[:, H * D:(H + Hk) * D].unflatten(1, (Hk, D))
    s.v = qkv[:, (H + Hk) * D:].unflatten(1, (Hk, D))
    s.k_pool = torch.empty(n_pages, Hk, PAGE, D, dtype=dt, device="cuda").normal_(generator=dev)
    s.v_pool = torch.empty(n_pages, Hk, PAGE, D, dtype=dt, device="cuda").normal_(generator=dev)
    s.k_min, s.k_max = s.k_pool.amin(2), s.k_pool.amax(2)


def _lengths(c, host):
    """Between half the context and all of it, one of them all of it; an idle slot in every fourth of a batch."""
    B, L = c["batch"], c["context"]
    lens = torch.randint(max(1, L // 2), L + 1, (B,), generator=host)
    lens[0] = L
    lens[3::4] = 0
    return lens


def _prepare_attention(s, c, host, dev):
    B, H, Hk, D, dt = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    lens = _lengths(c, host)
    held = _ceil(lens, PAGE)
    max_pages = _ceil(c["context"], PAGE) + 4
    n_pages = int(held.sum()) + 3
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    table[torch.arange(max_pages)[None, :] < held[:, None]] = torch.randperm(n_pages, generator=host).to(torch.int32)[:int(held.sum())]
    s.page_table, s.lens, s.max_len = table.cuda(), lens.to(torch.int32).cuda(), c["context"]
    # keys of a page resemble one another, and the queries are long enough for a softmax with a few clear winners
    s.k_pool = torch.empty(n_pages, Hk, PAGE, D, dtype=dt, device="cuda").normal_(generator=dev)
    s.k_pool *= 0.8
    s.k_pool += torch.empty(n_pages, Hk, 1, D, dtype=dt, device="cuda").normal_(0.0, 0.6, generator=dev)
    s.v_pool = torch.empty(n_pages, Hk, PAGE, D, dtype=dt, device="cuda").normal_(generator=dev)
    qkv = torch.empty(B, (H + 2 * Hk) * D, dtype=dt, device="cuda").normal_(0.0, 2.0, generator=dev)
    s.q = qkv[:, :H * D].unflatten(1, (H, D))                     # a view into the packed product
    s.scale = D ** -0.5
    # what a request before left behind in the last pages, behind the keys
    for pool in (s.k_pool, s.v_pool):
        for b in range(min(B, 8)):
            if int(lens[b]) % PAGE:
                pool[int(table[b, int(held[b]) - 1]), :, int(lens[b]) % PAGE:] = (float("nan"), float("inf"), -3e38)[b % 3]
    if c["kind"] == "sparse":
        s.k_min, s.k_max = s.k_pool.amin(2), s.k_pool.amax(2)
        for b in range(B):
            r = int(lens[b]) % PAGE
            if r:
                page = int(table[b, int(held[b]) - 1])
                s.k_min[page], s.k_max[page] = s.k_pool[page, :, :r].amin(1), s.k_pool[page, :, :r].amax(1)


# ---------------------------------------------------------------------------------------------- one pass


def run(s):
    if own:
        return _run_own(s)
    return {"pages": _plain_pages, "append": _plain_append, "attention": _plain_attention, "sparse": _plain_sparse}[s.case["kind"]](s)


def _run_own(s):
    from paper_2410_13344_b200 import binding
    kind = s.case["kind"]
    if kind == "pages":
        # what an earlier pass has planned goes back, as a rejected draft's pages would
        binding.pages_trim(s.base, s.lens, s.page_table, s.free_pages, s.n_free)
        p = binding.pages_plan(s.n_new, s.lens, s.page_table, s.free_pages, s.n_free, s.rows)
        return [p.slot, p.pos, p.seq, p.row_off, p.granted, s.page_table, s.free_pages, s.n_free, s.lens]
    if kind == "append":
        binding.kv_append(s.k, s.v, s.slot, s.k_pool, s.v_pool, s.k_min, s.k_max)
        return [s.k_pool, s.v_pool, s.k_min, s.k_max]
    if kind == "attention":
        return list(binding.paged_attention(s.q, s.k_pool, s.v_pool, s.page_table, s.lens, s.scale, s.max_len, window=s.case["window"]))
    sel, n_sel = binding.page_select(s.q, s.k_min, s.k_max, s.page_table, s.lens, s.case["pages"], s.max_len)
    out, lse = binding.paged_attention(s.q, s.k_pool, s.v_pool, s.page_table, s.lens, s.scale, s.max_len, sel=sel, n_sel=n_sel)
    return [sel, n_sel, out, lse]


def _plain_pages(s):
    dev = s.lens.device
    cols = torch.arange(s.page_table.shape[1], device=dev)
    # trim to the base lengths
    new = torch.minimum(s.base.clamp(min=0), s.lens)
    gone = (cols >= _ceil(new, PAGE)[:, None]) & (cols < _ceil(s.lens, PAGE)[:, None])
    pages = s.page_table[gone]
    f = int(s.n_free)
    s.free_pages[f:f + pages.numel()] = pages.flip(0)
    s.page_table[gone] = -1
    s.lens.copy_(new)
    f += pages.numel()
    # plan
    n_new = s.n_new.clamp(min=0).long()
    ends = torch.cumsum(n_new, 0)
    row_off = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), ends])
    held, want = _ceil(s.lens.long(), PAGE), _ceil(s.lens + n_new, PAGE)
    fits = (s.lens + n_new <= PAGE * s.page_table.shape[1]) & (ends <= s.rows)
    need = torch.where(fits, want - held, 0)
    cum = torch.cumsum(need, 0)
    ok = fits & ((need == 0) | (cum <= f))
    granted = torch.where(ok, n_new, 0)
    take = torch.where(ok, need, 0)
    fresh = (cols >= held[:, None]) & (cols < (held + take)[:, None])
    b, j = fresh.nonzero(as_tuple=True)
    s.page_table[b, j] = s.free_pages[f - 1 - (cum - need)[b] - (j - held[b])]
    r = torch.arange(s.rows, device=dev)
    seq = torch.searchsorted(ends, r, right=True).clamp(max=s.lens.numel() - 1)
    live = (r < ends[-1]) & ok[seq]
    pos = s.lens[seq] + r - row_off[seq]
    page = s.page_table[seq, torch.where(live, pos // PAGE, 0)]
    slot = torch.where(live, page.long() * PAGE + pos % PAGE, -1).int()
    pos = torch.where(live, pos, -1).int()
    seq = torch.where(live, seq, -1).int()
    s.lens += granted.int()
    s.n_free.fill_(f - int(take.sum()))
    return [slot, pos, seq, row_off.int(), granted.int(), s.page_table, s.free_pages, s.n_free, s.lens]


def _plain_append(s):
    rows = (s.slot >= 0).nonzero()[:, 0]
    slot = s.slot[rows].long()
    page, off = slot // PAGE, slot % PAGE
    k = s.k[rows]
    s.k_pool[page, :, off] = k
    s.v_pool[page, :, off] = s.v[rows]
    pages, at = torch.unique(page, return_inverse=True)
    grid = torch.full((pages.numel(), PAGE) + k.shape[1:], float("inf"), device=k.device)
    grid[at, off] = k.float()
    lo = grid.amin(1)
    grid = torch.where(torch.isposinf(grid), -grid, grid)
    grid[at, off] = k.float()
    hi = grid.amax(1)
    fresh = torch.zeros(pages.numel(), dtype=torch.bool, device=k.device)
    fresh[at[off == 0]] = True
    fresh = fresh[:, None, None]
    s.k_min[pages] = torch.where(fresh, lo, torch.minimum(lo, s.k_min[pages].float())).to(k.dtype)
    s.k_max[pages] = torch.where(fresh, hi, torch.maximum(hi, s.k_max[pages].float())).to(k.dtype)
    return [s.k_pool, s.v_pool, s.k_min, s.k_max]


def _attend(q, k, v, scale):
    """q [Hk][G][D], k and v [Hk][keys][D], all fp32."""
    x = (q @ k.transpose(1, 2)) * scale
    m = x.amax(2, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(2, keepdim=True)
    return (e @ v) / total, (m + torch.log(total))[..., 0]


def _plain_attention(s):
    H, Hk, D = s.q.shape[1], s.k_pool.shape[1], s.q.shape[2]
    out = torch.zeros(s.q.shape, dtype=s.q.dtype, device=s.q.device)
    lse = torch.full(s.q.shape[:2], float("-inf"), device=s.q.device)
    for b, length in enumerate(s.lens.tolist()):
        if not length:
            continue
        first = max(0, length - s.case["window"]) if s.case["window"] else 0
        pages = s.page_table[b, first // PAGE:_ceil(length, PAGE)].long()
        span = slice(first % PAGE, first % PAGE + length - first)
        k = s.k_pool[pages].transpose(0, 1).flatten(1, 2)[:, span].float()
        v = s.v_pool[pages].transpose(0, 1).flatten(1, 2)[:, span].float()
        o, l = _attend(s.q[b].float().unflatten(0, (Hk, H // Hk)), k, v, s.scale)
        out[b], lse[b] = o.flatten(0, 1).to(s.q.dtype), l.flatten()
    return [out, lse]


def _plain_sparse(s):
    H, Hk, D = s.q.shape[1], s.k_pool.shape[1], s.q.shape[2]
    dev, K = s.q.device, s.case["pages"]
    out = torch.zeros(s.q.shape, dtype=s.q.dtype, device=dev)
    lse = torch.full(s.q.shape[:2], float("-inf"), device=dev)
    sel = torch.full((s.q.shape[0], Hk, K), -1, dtype=torch.int32, device=dev)
    n_sel = torch.zeros(s.q.shape[0], dtype=torch.int32, device=dev)
    offsets = torch.arange(PAGE, device=dev)
    for b, length in enumerate(s.lens.tolist()):
        if not length:
            continue
        N = _ceil(length, PAGE)
        n = min(N, K)
        table = s.page_table[b, :N].long()
        q = s.q[b].unflatten(0, (Hk, H // Hk))
        # the scores decide between neighbours: 64 bits
        q64 = q.double()
        lo, hi = s.k_min[table].double().permute(1, 2, 0), s.k_max[table].double().permute(1, 2, 0)
        score = (q64.clamp(min=0) @ hi + q64.clamp(max=0) @ lo).amax(1)
        score = torch.where(torch.isnan(score), float("inf"), score)
        score[:, 0] = score[:, N - 1] = float("inf")               # the first and the last page are always read
        best = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :n]
        best = torch.sort(best, dim=1).values
        sel[b, :, :n], n_sel[b] = best.int(), n
        heads = torch.arange(Hk, device=dev)[:, None]
        k, v = s.k_pool[table[best], heads].float(), s.v_pool[table[best], heads].float()       # [Hk][n][PAGE][D]
        live = (best[..., None] * PAGE + offsets < length)[..., None]
        k, v = torch.where(live, k, 0.0).flatten(1, 2), torch.where(live, v, 0.0).flatten(1, 2)
        x = (q.float() @ k.transpose(1, 2)) * s.scale
        x = torch.where(live.flatten(1, 2).transpose(1, 2), x, float("-inf"))
        m = x.amax(2, keepdim=True)
        e = torch.exp(x - m)
        total = e.sum(2, keepdim=True)
        out[b] = ((e @ v) / total).flatten(0, 1).to(s.q.dtype)
        lse[b] = (m + torch.log(total)).flatten()
    return [sel, n_sel, out, lse]


# ---------------------------------------------------------------------------------------------- definition, 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"pages": _exact_pages, "append": _exact_append, "attention": _exact_attention, "sparse": _exact_attention}[case["kind"]](s, case)


def _exact_pages(s, c):
    """Request after request, on lists.  (The state is as a first pass finds it: there is nothing to trim.)"""
    lens, n_new, table = s.lens.tolist(), s.n_new.tolist(), s.page_table.cpu()
    stack, f = s.free_pages.tolist(), int(s.n_free)
    slot, pos, seq, granted, row_off = [-1] * s.rows, [-1] * s.rows, [-1] * s.rows, [], [0]
    asked = 0
    for b, (length, new) in enumerate(zip(lens, n_new)):
        r0 = row_off[-1]
        row_off.append(r0 + new)
        held, want = -(-length // PAGE), -(-(length + new) // PAGE)
        ok = want <= table.shape[1] and row_off[-1] <= s.rows
        if ok and want > held:
            if asked + want - held <= f:
                for j in range(held, want):
                    table[b, j] = stack[f - 1 - asked - (j - held)]
            else:
                ok = False
            asked += want - held
        granted.append(new if ok else 0)
        if ok:
            pages = table[b].tolist()
            for i in range(new):
                p = length + i
                slot[r0 + i], pos[r0 + i], seq[r0 + i] = pages[p // PAGE] * PAGE + p % PAGE, p, b
    now = [a + b for a, b in zip(lens, granted)]
    used = sum(-(-a // PAGE) for a in now) - sum(-(-a // PAGE) for a in lens)

    def t(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    return [t(slot), t(pos), t(seq), t(row_off), t(granted), table.cuda(), s.free_pages, t([f - used]), t(now)]


def _exact_append(s, c):
    k_pool, v_pool, lo, hi = (x.double() for x in (s.k_pool, s.v_pool, s.k_min, s.k_max))
    slots = s.slot.tolist()
    heads = s.k.double(), s.v.double()
    for off in range(PAGE):                                        # a page's keys in the order of its slots: at most one each
        rows = torch.tensor([r for r, x in enumerate(slots) if x >= 0 and x % PAGE == off], dtype=torch.long, device="cuda")
        pages = torch.tensor([x // PAGE for x in slots if x >= 0 and x % PAGE == off], dtype=torch.long, device="cuda")
        k_pool[pages, :, off], v_pool[pages, :, off] = heads[0][rows], heads[1][rows]
        if off == 0:
            lo[pages], hi[pages] = heads[0][rows], heads[0][rows]
        else:
            lo[pages], hi[pages] = torch.minimum(lo[pages], heads[0][rows]), torch.maximum(hi[pages], heads[0][rows])
    return [k_pool, v_pool, lo, hi]


def _exact_attention(s, c):
    B, H, D, Hk = *s.q.shape, s.k_pool.shape[1]
    G, dev = H // Hk, s.q.device
    out = torch.zeros(B, H, D, dtype=torch.float64, device=dev)
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device=dev)
    sel = torch.full((B, Hk, c.get("pages", 1)), -1, dtype=torch.int32, device=dev)
    n_sel = torch.zeros(B, dtype=torch.int32, device=dev)
    for b in range(B):
        length = int(s.lens[b])
        if length == 0:
            continue
        N = -(-length // PAGE)
        table = s.page_table[b, :N].long()
        key = torch.arange(N * PAGE, device=dev)
        for h in range(Hk):
            q = s.q[b, h * G:(h + 1) * G].double()
            seen = key < length
            if c["kind"] == "sparse":
                lo, hi = s.k_min[table, h].double(), s.k_max[table, h].double()
                score = torch.stack([torch.maximum(x * lo, x * hi).sum(1) for x in q]).amax(0).tolist()
                score[0] = score[-1] = math.inf
                best = sorted(sorted(range(N), key=lambda p: (-score[p], p))[:c["pages"]])
                n_sel[b] = len(best)
                sel[b, h, :len(best)] = torch.tensor(best, dtype=torch.int32)
                chosen = torch.zeros(N, dtype=torch.bool, device=dev)
                chosen[torch.tensor(best, device=dev)] = True
                seen = seen & chosen[key // PAGE]
            elif c["window"]:
                seen = seen & (key >= length - c["window"])
            at = seen.nonzero()[:, 0]
            k, v = s.k_pool[table[at // PAGE], h, at % PAGE].double(), s.v_pool[table[at // PAGE], h, at % PAGE].double()
            x = s.scale * (k @ q.T)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(x, 0)
            out[b, h * G:(h + 1) * G] = torch.softmax(x, 0).T @ v
    return [sel, n_sel, out, lse] if c["kind"] == "sparse" else [out, lse]


# ---------------------------------------------------------------------------------------------- bounds


def work(case):
    """Of one pass, from the case alone: lengths at their means (three quarters of the context, a quarter of the slots idle)."""
    kind = case["kind"]
    if kind == "pages":
        # lengths, new tokens and their results a request, slot, position and sequence a row, a page of the table for every page taken and given back
        rows = _mean_rows(case)
        pages = rows / PAGE
        return {"bytes": 28 * case["requests"] + 12 * rows + 16 * pages, "flops": 0}
    e, D = 2 if case["dtype"] == "bf16" else 4, case["head_dim"]
    if kind == "append":
        T, row = case["tokens"], case["kv_heads"] * D * e
        pages = T if case["runs"] == "decode" else T / PAGE
        return {"bytes": 4 * T * row + (4 if case["runs"] == "decode" else 2) * pages * row + 4 * T, "flops": 2 * T * case["kv_heads"] * D}
    B, H, Hk, L = case["batch"], case["heads"], case["kv_heads"], case["context"]
    full = 1                                                       # the first sequence has the whole context
    rest = B - 1 - B // 4
    q_and_out = 2 * B * H * D * e + 4 * B * H
    if kind == "attention":
        w = case["window"] or L
        keys = full * min(L, w) + rest * min(0.75 * L, w)
        return {"bytes": 2 * keys * Hk * D * e + q_and_out + 4 * keys / PAGE, "flops": 4 * keys * H * D}
    K = case["pages"]
    pages = full * math.ceil(L / PAGE) + rest * 0.75 * L / PAGE
    read = full * min(K, math.ceil(L / PAGE)) + rest * min(K, 0.75 * L / PAGE)
    return {"bytes": 2 * pages * Hk * D * e + 2 * read * PAGE * Hk * D * e + q_and_out + 4 * B * Hk * K + 4 * pages,
            "flops": 4 * pages * H * D + 4 * read * PAGE * H * D}
