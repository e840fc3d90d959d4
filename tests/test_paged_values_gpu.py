"""What the paged calls make of values: the bits that a decode step keeps, infinities,
against the float64 oracle (oracle/paged.py).

Bounds of a decode step, per output. P multiplies V as the sum of two bfloat16, the first
cut (off by less than a step, 2^-7 of it), the second rounded (half a step of the rest,
2^-8): 2^-15 sum p |v|. The sums of products in float32 lose at most T 2^-24 of
sum p |v| more, the division and the exponential's 2 units 2^-21. O is rounded to bfloat16
once, 2^-8 |O|. A score is off by at most D (see test_paged_gpu.py), which moves O by at
most 2 D max |v|.
"""
import numpy as np
import pytest
import torch

import paper_2609_33916_amd as lib
from helpers import gpu_available, to_host64
from oracle import paged
from test_paged_gpu import BF16, NAN, Pool, ints, same, stored

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("G,n", [(1, 300), (4, 300), (4, 3000), (8, 70), (16, 300), (20, 300), (33, 3000)])
def test_probabilities_keep_their_bits(bits, d, G, n):
    """Undivided and split, every layout of the query heads, one and two columns of them."""
    lens = [n, n // 2, 17]
    pool = Pool(lens, 2, 64 if n > 100 else 16, d, bits, seed=G).fill(lens, seed=n)
    q = torch.randn(3, 2 * G, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(G + n)).to(BF16)
    ref = pool.oracle()
    O, L = lib.attn_paged_decode(q, lens=ints(lens), **pool.args())
    want, lse, A, S = ref.attend(to_host64(q), lens, d ** -0.5)
    D = S * d * 2.0 ** -24 + (4 * S + 8) * 2.0 ** -23
    top = np.array([np.abs(ref.rows(b, range(lens[b]))[2]).max() for b in range(3)])
    tol = 2.0 ** -8 * np.abs(want) + A * (2.0 ** -15 + n * 2.0 ** -24 + 2.0 ** -21) * 1.01 + (2 * D * top[:, None])[..., None]
    err = np.abs(to_host64(O) - want)
    assert np.all(err <= tol), (err - tol).max()


@pytest.mark.parametrize("n", [100, 5000])
@pytest.mark.parametrize("G", [2, 20])
def test_infinite_values(n, G):
    """An infinite value of a token makes its column of O infinite, with its sign."""
    pool = Pool([n], 1, 16, 64, 16).fill([n])
    at = int(pool.table[0, 2])
    pool.v[at, 0, 5, 9], pool.v[at, 0, 6, 11] = float("inf"), -float("inf")
    q = 0.1 * torch.randn(1, G, 64, device="cuda")
    q[0, 0] = 0   # every token with the same weight, 1
    O, L = lib.attn_paged_decode(q.to(BF16), lens=ints([n]), **pool.args())
    assert bool((O[..., 9] == float("inf")).all()) and bool((O[..., 11] == -float("inf")).all())
    O[..., 9] = O[..., 11] = 0
    assert bool(torch.isfinite(O).all()) and bool(torch.isfinite(L).all())
