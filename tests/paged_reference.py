"""The paged-cache operators once more, plainly: whole numbers on lists, everything else in 64 bits on the CPU, key by key."""
import math

import torch

PAGE = 16


def pages_of(tokens):
    return -(-tokens // PAGE)


class Book:
    """Lengths, tables and the stack of free pages, as lists."""

    def __init__(self, lens, table, free, n_free):
        self.lens, self.table, self.free, self.n_free = list(lens), [list(r) for r in table], list(free), n_free

    def plan(self, n_new, rows):
        n_new = [max(0, n) for n in n_new]
        slot, pos, seq, granted, row_off = [-1] * rows, [-1] * rows, [-1] * rows, [], [0]
        cum = 0
        top = self.n_free
        for b, n in enumerate(n_new):
            r0 = row_off[-1]
            row_off.append(r0 + n)
            held, want = pages_of(self.lens[b]), pages_of(self.lens[b] + n)
            ok = want <= len(self.table[b]) and r0 + n <= rows
            if ok and want > held:
                base = cum
                cum += want - held
                ok = cum <= top
                if ok:
                    for j in range(held, want):
                        self.table[b][j] = self.free[top - 1 - base - (j - held)]
                    self.n_free -= want - held
            granted.append(n if ok else 0)
            if not ok:
                continue
            for i in range(n):
                p = self.lens[b] + i
                slot[r0 + i], pos[r0 + i], seq[r0 + i] = self.table[b][p // PAGE] * PAGE + p % PAGE, p, b
            self.lens[b] += n
        return slot, pos, seq, row_off, granted

    def trim(self, keep):
        back = []
        for b, n in enumerate(keep):
            n = min(max(n, 0), self.lens[b])
            for j in range(pages_of(n), pages_of(self.lens[b])):
                back.append(self.table[b][j])
                self.table[b][j] = -1
            self.lens[b] = n
        for page in reversed(back):
            if self.n_free < len(self.free):
                self.free[self.n_free] = page
            self.n_free = min(self.n_free + 1, len(self.free))


def append(k, v, slots, k_pool, v_pool, k_min=None, k_max=None):
    """In place, token by token."""
    in_call = {}
    n_slots = k_pool.shape[0] * PAGE
    for t, s in enumerate(slots):
        if not 0 <= s < n_slots:
            continue
        k_pool[s // PAGE, :, s % PAGE], v_pool[s // PAGE, :, s % PAGE] = k[t], v[t]
        in_call.setdefault(s // PAGE, []).append((s % PAGE, k[t]))
    if k_min is None:
        return
    for page, keys in in_call.items():
        rows = [x for _, x in keys]
        if all(off for off, _ in keys):
            lo, hi = [k_min[page]] + rows, [k_max[page]] + rows
        else:
            lo = hi = rows
        k_min[page], k_max[page] = torch.stack(lo).amin(0), torch.stack(hi).amax(0)


def select(q, k_min, k_max, table, lens, K, n_first=1, n_last=1):
    """q [B][H][D], lists of pages per (sequence, KV head)."""
    B, H, D = q.shape
    P, Hk, _ = k_min.shape
    G = H // Hk
    out = []
    for b, length in enumerate(lens):
        N = pages_of(length)
        out.append([])
        for h in range(Hk):
            score = []
            for p in range(N):
                at = int(table[b][p])
                if not 0 <= at < P:
                    score.append(-math.inf)
                    continue
                lo, hi = k_min[at, h].double(), k_max[at, h].double()
                x = q[b, h * G:(h + 1) * G].double()
                s = float(torch.maximum(x * lo, x * hi).sum(1).amax())
                score.append(math.inf if math.isnan(s) else s)
            forced = [p for p in range(N) if p < n_first or p >= N - n_last]
            rest = sorted((p for p in range(n_first, N - n_last)), key=lambda p: (-score[p], p))
            out[-1].append(list(range(N)) if N <= K else sorted(forced + rest[:K - len(forced)]))
    return out


def attention(q, k_pool, v_pool, table, lens, scale, window=0, sel=None):
    """q [B][H][D]; sel: lists of logical pages per (sequence, KV head), or None.  Returns (out, lse, tol): tol bounds what the kernels' roundings
    can do to each element of out, and (second entry) of lse.

    Of a score, S = scale sum |q||k| its largest absolute sum: bf16 products are exact, a chain is D / 32 steps of the tensor cores long, each off by at most 17
    addends x 2^-23 S, two chains, three more roundings: d <= (2 D / 32 x 17 x 2^-23 + 3 x 2^-24) S + 2^-22 for the exponential.  fp32: chains of at most D / 32
    + 5 roundings of 2^-24.  A weight is off by d and, in bf16, by 2^-8 for its rounding; with A = sum p |v| / sum p, numerator and denominator move the result
    by at most (2 d + 2^-8) A; the sums over n keys add n x 2^-24 A (fp32, each key a rounding) or n / 16 x 17 x 2^-23 A (bf16, a step for 16), and as much for joining
    and rescaling; the result is rounded once."""
    B, H, D = q.shape
    P, Hk = k_pool.shape[:2]
    G = H // Hk
    bf = q.dtype == torch.bfloat16
    out = torch.zeros(B, H, D, dtype=torch.float64)
    lse = torch.full((B, H), -math.inf, dtype=torch.float64)
    tol_o, tol_l = torch.zeros(B, H, D, dtype=torch.float64), torch.zeros(B, H, dtype=torch.float64)
    for b, length in enumerate(lens):
        lo = max(0, length - window) if window else 0
        N = pages_of(length)
        for h in range(Hk):
            pages = range(N) if sel is None else [p for p in sel[b][h] if 0 <= p < N]
            ks, vs = [], []
            for p in pages:
                at = int(table[b][p])
                if not 0 <= at < P:
                    continue
                r0, r1 = max(lo - p * PAGE, 0), min(length - p * PAGE, PAGE)
                if r0 < r1:
                    ks.append(k_pool[at, h, r0:r1])
                    vs.append(v_pool[at, h, r0:r1])
            if not ks:
                continue
            k, v = torch.cat(ks).double(), torch.cat(vs).double()
            x = q[b, h * G:(h + 1) * G].double()
            s = scale * (x @ k.T)
            w = torch.softmax(s, 1)
            o = w @ v
            A = w @ v.abs()
            S = (abs(scale) * (x.abs() @ k.abs().T)).amax(1)
            n = k.shape[0]
            if bf:
                d = (2 * D / 32 * 17 * 2.0 ** -23 + 3 * 2.0 ** -24) * S + 2.0 ** -22
                a = (2 * d + 2.0 ** -8 + 2 * n / 16 * 17 * 2.0 ** -23)[:, None] * A + 2.0 ** -8 * o.abs()
            else:
                d = (D / 32 + 8) * 2.0 ** -24 * S + 2.0 ** -22
                a = (2 * d + 2 * n * 2.0 ** -24 + 2.0 ** -23)[:, None] * A + 2.0 ** -24 * o.abs()
            sl = slice(h * G, (h + 1) * G)
            out[b, sl], lse[b, sl], tol_o[b, sl] = o, torch.logsumexp(s, 1), a
            # the logarithm of a sum of n weights off by d each, and two roundings of the result
            tol_l[b, sl] = d + n * 2.0 ** -24 + 4 * 2.0 ** -24 * (lse[b, sl].abs() + S + 1)
    return out, lse, (tol_o, tol_l)
