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
from test_paged_gpu import BF16, Pool, ints, same, stored

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


# --------------------------------------------- pages of another writer of the format --
def all_codes(rows, d):
    """[rows, d/2] bytes in which every code stands at every scale."""
    c = (np.arange(d)[None] * 5 + np.arange(rows)[:, None]) % 16
    return torch.from_numpy((c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)).cuda()


@pytest.mark.parametrize("d", [32, 64, 128])
def test_gather_every_scale(d):
    """All 256 scale bytes with all codes: what bfloat16 holds exactly, infinities behind
    its range, NaN for 255."""
    pool = Pool([256], 1, 16, d, 4)
    for p in range(256):
        at, r = int(pool.table[0, p // 16]), p % 16
        pool.k[at, 0, r] = all_codes(256, d)[p]
        pool.v[at, 0, r] = all_codes(256, d)[255 - p]
        pool.scales["k_scales"][at, 0, r] = pool.scales["v_scales"][at, 0, r] = p
    ref = pool.oracle()
    K, V = lib.attn_paged_gather(lens=ints([256]), n=256, **pool.args())
    for got, x in ((K, ref.k), (V, ref.v)):
        want = ref.rows(0, range(256))[1 if x is ref.k else 2][0]
        want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
        assert same(to_host64(got)[0, 0], want)


@pytest.mark.parametrize("n", [5, 100, 5000])
@pytest.mark.parametrize("d,G", [(32, 2), (64, 1), (64, 20), (128, 3), (128, 8), (128, 12)])
def test_a_scale_that_is_not_a_number(n, d, G):
    """255 makes a block not a number whatever its codes: of V its 32 columns of O, of K
    everything of its heads."""
    pool = Pool([n], 2, 16, d, 4, seed=G).fill([n])
    q = torch.randn(1, 2 * G, d, device="cuda").to(BF16)
    at = int(pool.table[0, 0])
    pool.v[at, 1, 3] = torch.randint(1, 8, (d // 2,), device="cuda").to(torch.uint8) * 17   # no code is 0
    pool.scales["v_scales"][at, 1, 3, d // 32 - 1] = 255
    O, L = lib.attn_paged_decode(q, lens=ints([n]), **pool.args())
    bad = torch.zeros_like(O, dtype=torch.bool)
    bad[0, G:, d - 32:] = True
    assert torch.equal(torch.isnan(O), bad) and bool(torch.isfinite(O[~bad]).all()) and bool(torch.isfinite(L).all())
    pool.k[at, 0, 3] = pool.v[at, 1, 3]
    pool.scales["k_scales"][at, 0, 3, 0] = 255
    O, L = lib.attn_paged_decode(q, lens=ints([n]), **pool.args())
    assert bool(torch.isnan(O[0, :G]).all()) and bool(torch.isnan(L[0, :G]).all()) and bool(torch.isfinite(L[0, G:]).all())


@pytest.mark.parametrize("d,G", [(32, 2), (64, 20), (128, 3), (128, 8), (128, 12)])
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 30, 100, 126, 160, 200, 220])
def test_decode_other_scales(byte, d, G):
    """Scales far from 1, of V, then of K. V's byte 0 counts as zero (6 2^-127 at most);
    a sum of products loses what is below 2^-133, a bfloat16's last bit, per token."""
    n = 40
    pool = Pool([n], 1, 16, d, 4, seed=byte).fill([n], seed=byte)
    for i in range(3):
        at = int(pool.table[0, i])
        pool.k[at, 0], pool.v[at, 0] = all_codes(16, d), all_codes(16, d) + 16 * (i % 2)
        pool.scales["v_scales"][at] = byte
    q = torch.randn(1, G, d, device="cuda").to(BF16)
    ref = pool.oracle()
    O, L = lib.attn_paged_decode(q, lens=ints([n]), **pool.args())
    want, lse, A, S = ref.attend(to_host64(q), [n], d ** -0.5)
    D = S * d * 2.0 ** -24 + (4 * S + 8) * 2.0 ** -23
    top = 6 * 2.0 ** (byte - 127)
    tol = 2.0 ** -8 * np.abs(want) + A * (2.0 ** -15 + n * 2.0 ** -24 + 2.0 ** -21) * 1.01 + (2 * D * top)[..., None] + 2 * n * 2.0 ** -133
    tol += 6 * 2.0 ** -127 if byte == 0 else 0
    err = np.abs(to_host64(O) - want)
    assert np.all(err <= tol), (err / tol).max()
    for i in range(3):   # scores of the same size whatever the scale
        at = int(pool.table[0, i])
        pool.scales["k_scales"][at], pool.scales["v_scales"][at] = byte, 126
    ref, scale = pool.oracle(), 0.1 * 2.0 ** min(127 - byte, 100)
    O, L = lib.attn_paged_decode(q, lens=ints([n]), scale=scale, **pool.args())
    want, lse, A, S = ref.attend(to_host64(q), [n], scale)
    D = S * d * 2.0 ** -24 + (4 * S + 8) * 2.0 ** -23
    assert np.all(np.abs(to_host64(L) - lse) <= D + np.abs(lse) * 2.0 ** -22 + 2.0 ** -22)
    err, tol = np.abs(to_host64(O) - want), 2.0 ** -8 * np.abs(want) + 4 * A * (2.0 ** -15 + n * 2.0 ** -24 + 2.0 ** -21) + (6 * D)[..., None]
    assert np.all(err <= tol), (err / tol).max()


# ------------------------------------------------------- the ends of what is written --
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("amplitude", [1.0, 1.25, 0.75])
@pytest.mark.parametrize("d,r", [(32, 32), (64, 32), (128, 128), (128, 16)])
def test_smallest_values(interleaved, amplitude, d, r):
    """Every bfloat16 below 2^-125, where blocks have the smallest scale: codes of the
    rotated and of the other columns against the oracle, at position 0 (products are
    exact) and elsewhere; an append and a decode step's append store the same bytes."""
    steps = torch.arange(512, dtype=torch.int16)   # bits: 0 .. 2^-124
    g = torch.Generator().manual_seed(d + r)
    rows = torch.stack([steps[torch.randperm(512, generator=g)[:d]] for _ in range(96)])
    rows[:32] %= 256      # below 2^-125
    rows[32:64] %= 128    # below 2^-126
    x = rows.view(BF16) * torch.where(torch.rand(96, d, generator=g) < 0.5, -1, 1)
    k = x.view(1, 1, 96, d).cuda()
    freqs, _ = lib.attn_rope_freqs(r)
    for at in (0, 77):
        pos = ints([at] * 96)[None]
        rot = dict(freqs=freqs, amplitude=amplitude, interleaved=interleaved)
        pool, one = Pool([96], 1, 16, d, 4), Pool([96], 1, 16, d, 4)
        lib.attn_paged_append(k, k, lens=ints([0]), positions=pos, **rot, **pool.args())
        ref = pool.oracle().rows(0, range(96))
        y = paged.rotate(to_host64(k)[0, 0], np.full(96, at), freqs.cpu().numpy(), amplitude, interleaved)
        assert same(ref[1][0], stored(y, 4)) and same(ref[2][0], stored(to_host64(k)[0, 0], 4))
        for t in range(96):
            new = k[:, :, t].contiguous()
            lib.attn_paged_decode(new, lens=ints([t]), k_new=new, v_new=new, positions=pos[:, t].contiguous(), **rot, **one.args())
        assert all(torch.equal(a, b) for a, b in zip(pool.state(), one.state()))
