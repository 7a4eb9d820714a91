"""Attention over the paged cache in bf16: softmax weights keep about 16 significant bits, as in the library's tree attention.

Tolerance: a score is off by d = (2 (D / 32) 17 2^-23 + 3 2^-24) S + 2^-22, S its scaled sum of absolute products (paged_reference.py).  A weight enters its product as two bf16 terms, the
first off by at most 2^-8 of it, the second, which is the rest, by at most 2^-8 of that: 2^-16.  The sum of n weighted values takes 2 n / 16 steps of the tensor cores, each off by at most 17 2^-23 A,
A = sum p |v| / sum p, and as much again for rescaling and joining; the result is rounded once, by at most 2^-8 of itself."""
import random

import pytest
import torch

import paged_reference as ref
from paper_2410_13344_b200 import binding

pytestmark = pytest.mark.gpu
PAGE = 16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(lens, Hk, keys, values, seed):
    """Pools that hold keys[b][kv head][len][D] and values, in pages of any order."""
    held = [ref.pages_of(n) for n in lens]
    pages = random.Random(seed).sample(range(sum(held) + 2), sum(held) + 2)
    D = keys[0].shape[2]
    pools = [torch.zeros(len(pages), Hk, PAGE, D, dtype=torch.bfloat16) for _ in range(2)]
    table = torch.full((len(lens), max(held) + 1), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        for j in range(held[b]):
            at = pages.pop()
            table[b, j] = at
            m = min(PAGE, n - j * PAGE)
            for pool, rows in zip(pools, (keys, values)):
                pool[at, :, :m] = rows[b][:, j * PAGE:j * PAGE + m]
    return pools[0], pools[1], table


def weights_tolerance(q, k, v, scale, H, Hk):
    """Of one sequence, k and v [Hk][n][D], q [H][D]: the result and what the roundings above can do to it."""
    G, n, D = H // Hk, k.shape[1], k.shape[2]
    x, k, v = q.double().view(Hk, G, D), k.double(), v.double()
    w = torch.softmax(scale * (x @ k.transpose(1, 2)), 2)
    S = (abs(scale) * (x.abs() @ k.abs().transpose(1, 2))).amax(2, keepdim=True)
    d = (2 * D / 32 * 17 * 2.0 ** -23 + 3 * 2.0 ** -24) * S + 2.0 ** -22
    o, A = w @ v, w @ v.abs()
    return o.view(H, D), ((2 * d + 2.0 ** -16 + 2 * (2 * n / 16) * 17 * 2.0 ** -23) * A + 2.0 ** -8 * o.abs()).view(H, D)


def check(lens, Hk, G, D, keys, values, q, scale, max_len, seed):
    k_pool, v_pool, table = make(lens, Hk, keys, values, seed)
    out, _ = binding.paged_attention(q.cuda(), k_pool.cuda(), v_pool.cuda(), table.cuda(), i32(lens), scale, max_len)
    out = out.double().cpu()
    for b in range(len(lens)):
        o, tol = weights_tolerance(q[b], keys[b], values[b], scale, Hk * G, Hk)
        assert bool(((out[b] - o).abs() <= tol).all()), (b, float(((out[b] - o).abs() / tol).max()))


# a cluster to a unit, one of them of two pages ahead, shares with a join, a warp to a unit, and sixteen heads to a unit
FORMS = [([100], 2, 4, 64), ([1000], 2, 4, 128), ([600] * 16, 8, 8, 128), ([20000, 16, 3000], 1, 5, 64), ([9000, 7000], 8, 8, 128), ([48] * 200, 4, 8, 64), ([33] * 130, 4, 3, 128),
         ([5000] * 4, 2, 16, 64), ([5000] * 4, 4, 12, 128)]


@pytest.mark.parametrize("lens,Hk,G,D", FORMS)
def test_weights_that_one_bf16_term_would_make_equal(lens, Hk, G, D):
    """Weights 1 and e^-t, t = 3 / 2048, of values 1 and -1: tanh(t / 2).  (Rounded to bf16, both weights are 1 and the result 0.)"""
    t = 3 / 2048
    keys, values = [], []
    for b, n in enumerate(lens):
        down = torch.randint(0, 2, (Hk, n, 1), generator=torch.Generator().manual_seed(b)).bool() if n % 2 else (torch.arange(n) % 2 == 1)[None, :, None].expand(Hk, n, 1)
        keys.append(torch.cat([torch.where(down, -t, 0.0), torch.zeros(Hk, n, D - 1)], 2).bfloat16())
        values.append(torch.where(down, -1.0, 1.0).expand(Hk, n, D).bfloat16())
    q = torch.zeros(len(lens), Hk * G, D, dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    check(lens, Hk, G, D, keys, values, q, 1.0, max(lens), 1)


@pytest.mark.parametrize("lens,Hk,G,D", FORMS)
def test_random_keys_and_values(lens, Hk, G, D):
    g = torch.Generator().manual_seed(D + G)
    keys = [torch.randn(Hk, n, D, generator=g).bfloat16() for n in lens]
    values = [torch.randn(Hk, n, D, generator=g).bfloat16() for n in lens]
    q = (2 * torch.randn(len(lens), Hk * G, D, generator=g)).bfloat16()
    check(lens, Hk, G, D, keys, values, q, D ** -0.5, max(lens), 2)
