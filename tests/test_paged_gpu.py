"""The paged key/value cache on the GPU (attn_paged_append, attn_paged_gather,
attn_paged_decode) against the float64 oracle (oracle/paged.py).

Bounds of a decode step, per output. P is rounded to bfloat16 for the second product
(half a step, 2^-8 relative: 2^-8 sum p |v|), O once more (2^-8 |O|); a score is off by
at most D: the rotated query is the sum of two bfloat16 (2^-16 relative), keys are exact
as stored, and float32 sums of d products lose at most d 2^-24, of S = the largest
scale sum |q k| in both cases; a score error D moves O by at most 2 D max |v|. The
exponentials' float32 argument adds (4 |s| + 8) 2^-23 to D, |s| <= S. L is off by at
most D and its own rounding. What is stored is compared exactly.
"""
import numpy as np
import pytest
import torch

import paper_2609_33916_amd as lib
from helpers import gpu_available, to_host64
from oracle import paged

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

BF16, NAN = torch.bfloat16, float("nan")


class Pool:
    """Pages of `need` tokens per sequence in no order; everything else in the pool
    is poison (NaN, or scale 255), table entries behind a sequence's pages are junk."""

    def __init__(self, need, Hkv, page, d, bits, seed=0, width=None, spare=2):
        g = np.random.default_rng(seed)
        count = [-(-x // page) for x in need]
        self.B, self.page, self.bits, self.d, self.Hkv = len(need), page, bits, d, Hkv
        self.num = sum(count) + spare
        width = max(count + [1]) if width is None else width
        order = g.permutation(self.num)
        self.table = g.choice([-1, self.num, 2**31 - 1, -2**31], size=(self.B, width)).astype(np.int32)
        at = 0
        for b, k in enumerate(count):
            self.table[b, :k] = order[at:at + k]
            at += k
        self.t_table = torch.from_numpy(self.table).cuda()
        shape = (self.num, Hkv, page)
        if bits == 16:
            self.k, self.v = (torch.full(shape + (d,), NAN, dtype=BF16, device="cuda") for _ in range(2))
            self.scales = {}
        else:
            self.k, self.v = (torch.zeros(shape + (d // 2,), dtype=torch.uint8, device="cuda") for _ in range(2))
            self.scales = {x: torch.full(shape + (d // 32,), 255, dtype=torch.uint8, device="cuda") for x in ("k_scales", "v_scales")}

    def fill(self, lens, seed=1, sigma=1.0):
        """Random rows for the first lens[b] tokens (4 bits: random codes)."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        for b, n in enumerate(lens):
            for i in range(-(-n // self.page)):
                at, m = int(self.table[b, i]), min(self.page, n - i * self.page)
                if not 0 <= at < self.num:
                    continue
                for x in (self.k, self.v):
                    if self.bits == 16:
                        x[at, :, :m] = (torch.randn(self.Hkv, m, self.d, device="cuda", generator=g) * sigma).to(BF16)
                    else:
                        x[at, :, :m] = torch.randint(0, 256, (self.Hkv, m, self.d // 2), device="cuda", generator=g).to(torch.uint8)
                for x in self.scales.values():
                    x[at, :, :m] = torch.randint(124, 127, (self.Hkv, m, self.d // 32), device="cuda", generator=g).to(torch.uint8)
        return self

    def args(self):
        return dict(k_pages=self.k, v_pages=self.v, block_table=self.t_table, **self.scales)

    def state(self):
        return [x.clone() for x in (self.k, self.v, *self.scales.values())]

    def oracle(self):
        if self.bits == 16:
            return paged.Cache(to_host64(self.k), to_host64(self.v), self.table)
        c = [paged.from_codes(x.cpu().numpy(), s.cpu().numpy()) for x, s in zip((self.k, self.v), self.scales.values())]
        return paged.Cache(*c, self.table)


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def stored(x, bits):
    """float64 rows as a cache holds them"""
    if bits == 4:
        return paged.from_codes(*paged.to_codes(x))
    return to_host64(torch.from_numpy(x).to(BF16))


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


# ------------------------------------------------------------------ append --
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d,r,interleaved", [(32, 32, False), (64, 0, False), (64, 32, True), (64, 48, False), (128, 128, False),
                                             (128, 16, False), (128, 128, True)])
@pytest.mark.parametrize("T,page", [(1, 16), (37, 16), (50, 64)])
def test_append(bits, d, r, interleaved, T, page):
    """Rows, and nothing else, hold the tokens; counts from 0 to T, a sequence of no
    tokens, one that starts inside a page, one whose table ends early, one with a bad
    page, a negative length. Read back with attn_paged_gather."""
    Hkv = 3
    lens = [0, 5, page, 3 * page - 1, 9, -4]
    news = [T, T, 0, T, max(1, T // 2), T]
    need = [max(0, x) + t for x, t in zip(lens, news)]
    need[3] = lens[3] + 1                       # no room for more
    width = -(-(3 * page + T) // page)
    pool = Pool(need, Hkv, page, d, bits, seed=d + T, width=width)
    pool.table[1, 1 if need[1] > page else 0] = pool.num   # a number that is no page
    pool.t_table.copy_(torch.from_numpy(pool.table))
    pool.fill([max(0, x) for x in lens])
    freqs, a = lib.attn_rope_freqs(r, scaling="ramp", factor=4.0, original_length=100) if r else (None, 1.0)
    g = torch.Generator(device="cuda").manual_seed(T)
    kv = torch.randn(len(lens), T, 2 * Hkv, d, device="cuda", generator=g).to(BF16).transpose(1, 2)
    k, v = kv[:, :Hkv], kv[:, Hkv:]
    before, ref = pool.state(), pool.oracle()
    kept = kv.clone()
    assert lib.attn_paged_append(k, v, lens=ints(lens), new_lens=ints(news), freqs=freqs, amplitude=a, interleaved=interleaved,
                                 **pool.args()) is None
    torch.cuda.synchronize()
    assert torch.equal(kv, kept)
    kh, vh = to_host64(k), to_host64(v)
    if bits == 16 and r:   # the very bits of attn_rope (float32 arithmetic): compared with it, and it with the oracle
        pos = ints(range(T))[None] + ints(lens)[:, None]
        kr = to_host64(lib.attn_rope(k, None, freqs, a, interleaved, positions=pos)[0])
    touched = np.zeros(pool.k.shape[:3], dtype=bool)
    for b, n in enumerate(lens):
        for t in range(news[b] if n >= 0 else 0):
            if ref.place(b, n + t) is None:
                continue
            row = kr[b, :, t] if bits == 16 and r else stored(paged.rotate(kh[b, :, t], np.full(Hkv, n + t), freqs.cpu().numpy(), a, interleaved)
                                                              if r else kh[b, :, t], bits)
            ref.write(b, n + t, row, stored(vh[b, :, t], bits))
            touched[ref.place(b, n + t)[0], :, ref.place(b, n + t)[1]] = True
    got = pool.oracle()
    assert same(got.k, ref.k) and same(got.v, ref.v)
    keep = torch.from_numpy(~touched).cuda()
    for x, y in zip(pool.state(), before):
        assert torch.equal(x[keep].view(torch.uint8), y[keep].view(torch.uint8))
    # read back: whole sequences and a window that starts before and ends behind them
    after = [max(0, x) + (t if x >= 0 else 0) for x, t in zip(lens, news)]
    n = max(after) + 3
    for starts in (None, [0, 2, -3, page - 1, 100, 7]):
        K, V = lib.attn_paged_gather(lens=ints(after), n=n, starts=None if starts is None else ints(starts), **pool.args())
        for x, y in ((to_host64(K), ref.k), (to_host64(V), ref.v)):
            want = np.zeros(x.shape)
            for b in range(len(lens)):
                for j in range(n):
                    p = j + (0 if starts is None else starts[b])
                    at = ref.place(b, p) if p < after[b] else None
                    if at is not None:
                        want[b, :, j] = y[at[0], :, at[1]]
            assert same(x, want)


def test_append_given_positions_and_defaults():
    """Positions turn the keys, lengths place them; without new_lens all T are written."""
    freqs, a = lib.attn_rope_freqs(64)
    pool = Pool([40, 40], 2, 16, 64, 16)
    k, v = (torch.randn(2, 2, 7, 64, device="cuda").to(BF16) for _ in range(2))
    pos = ints(np.random.default_rng(0).integers(-100, 100000, 14)).view(2, 7)
    lib.attn_paged_append(k, v, lens=ints([3, 30]), freqs=freqs, amplitude=a, positions=pos, **pool.args())
    want = lib.attn_rope(k, None, freqs, a, positions=pos)[0]
    K, V = lib.attn_paged_gather(lens=ints([10, 37]), n=7, starts=ints([3, 30]), **pool.args())
    assert torch.equal(K, want) and torch.equal(V, v)


@pytest.mark.parametrize("interleaved", [False, True])
def test_one_rotation_for_all(interleaved):
    """attn_rope, an append and a decode step's append turn a key to the same bits, so a
    cache does not depend on how its rows came in."""
    B, T, d = 64, 80, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    k = torch.randn(B, 2, T, d, device="cuda", generator=g).to(BF16)
    freqs, a = lib.attn_rope_freqs(d, scaling="ramp", factor=3.0, original_length=100)
    pos = torch.randint(0, 10**6, (B, T), device="cuda", generator=g).int()
    rot = dict(freqs=freqs, amplitude=a, interleaved=interleaved)
    want = lib.attn_rope(k, None, freqs, a, interleaved, positions=pos)[0]
    rows = []
    for bits in (16, 4):
        one, all_ = (Pool([T] * B, 2, 16, d, bits, seed=2) for _ in range(2))
        lib.attn_paged_append(k, k, lens=ints([0] * B), positions=pos, **rot, **all_.args())
        for t in range(T):
            new = k[:, :, t].contiguous()
            lib.attn_paged_decode(new, lens=ints([t] * B), k_new=new, v_new=new, n=T - 1, positions=pos[:, t].contiguous(),
                                  **rot, **one.args())
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(one.state(), all_.state()))
        rows.append(lib.attn_paged_gather(lens=ints([T] * B), n=T, **all_.args())[0])
    assert torch.equal(rows[0], want)


def test_4bit_extremes():
    """Zeros, infinities, NaN, the ends of the bfloat16 range and values on the borders of
    the codes, block by block, against the oracle; a block's neighbours are not touched."""
    d = 128
    x = torch.zeros(8, d, dtype=torch.float64)
    x[1, 40] = float("inf")
    x[2, 3], x[2, 90] = float("nan"), float("-inf")
    x[3] = 3.3895313892515355e38 * torch.linspace(-1, 1, d, dtype=torch.float64)
    x[4] = 1.2e-38 * torch.linspace(-1, 1, d, dtype=torch.float64)
    x[5] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 16, dtype=torch.float64) * -1
    x[6] = torch.tensor([7.0, 6.96875, 0.0, -0.0] * 32, dtype=torch.float64)
    x[7] = 2.0 ** torch.randint(-30, 30, (d,)).double()
    x = x.to(BF16).cuda()
    pool = Pool([8], 1, 16, d, 4)
    lib.attn_paged_append(x[None, None], x[None, None], lens=ints([0]), **pool.args())
    K, V = lib.attn_paged_gather(lens=ints([8]), n=8, **pool.args())
    want = stored(to_host64(x), 4)
    assert np.isnan(want).sum() == 3 * 32
    assert same(to_host64(K)[0, 0], want) and same(to_host64(V)[0, 0], want)


# ------------------------------------------------------------------ decode --
def decode_case(lens, Hq, Hkv, page, d, bits, r=0, interleaved=False, append=True, scale=None, pos=None, n=None, seed=0,
                spoil=(), packed=False, width=None, sigma=1.0):
    B = len(lens)
    pool = Pool([x + append for x in lens], Hkv, page, d, bits, seed=seed, width=width)
    pool.fill(lens, seed=seed + 1, sigma=sigma)
    for b, i in spoil:
        pool.table[b, i] = [-1, pool.num, 2**31 - 1][(b + i) % 3]
    pool.t_table.copy_(torch.from_numpy(pool.table))
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    qkv = torch.randn(B, Hq + 2 * Hkv, d, device="cuda", generator=g).to(BF16)
    q, kn, vn = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if not packed:
        q, kn, vn = q.contiguous(), kn.contiguous(), vn.contiguous()
    freqs, a = lib.attn_rope_freqs(r, scaling="ramp", factor=4.0, original_length=100) if r else (None, 1.0)
    scale = d ** -0.5 if scale is None else scale
    ref, before = pool.oracle(), pool.state()
    O, L = lib.attn_paged_decode(q, lens=ints(lens), k_new=kn if append else None, v_new=vn if append else None, n=n, scale=scale,
                                 freqs=freqs, amplitude=a, interleaved=interleaved, positions=None if pos is None else ints(pos),
                                 **pool.args())
    torch.cuda.synchronize()
    T = [x + append for x in lens]
    at = np.array([t - 1 for t in T] if pos is None else pos)
    qh, kh, vh = to_host64(q), to_host64(kn), to_host64(vn)
    if r:
        f = freqs.cpu().numpy()
        qh = paged.rotate(qh, np.broadcast_to(at[:, None], qh.shape[:2]), f, a, interleaved)
        kr = paged.rotate(kh, np.broadcast_to(at[:, None], kh.shape[:2]), f, a, interleaved)
        if bits == 16:   # stored in bfloat16: within its half step and the rotation's own error of the oracle's
            kr = to_host64(lib.attn_rope(kn[:, :, None], None, freqs, a, interleaved, positions=ints(at)[:, None])[0][:, :, 0])
        kh = kr
    if append:
        kh, vh = stored(kh, bits), stored(vh, bits)
        touched = np.zeros(pool.k.shape[:3], dtype=bool)
        for b, x in enumerate(lens):
            ref.write(b, x, kh[b], vh[b])
            if ref.place(b, x) is not None:
                touched[ref.place(b, x)[0], :, ref.place(b, x)[1]] = True
        got = pool.oracle()
        assert same(got.k, ref.k) and same(got.v, ref.v)
        keep = torch.from_numpy(~touched).cuda()
        before = [x[keep] for x in before]
        now = [x[keep] for x in pool.state()]
    else:
        now = pool.state()
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(now, before))
    want, lse, A, S = ref.attend(qh, T, scale)
    D = S * (2.0 ** -16 * bool(r) + d * 2.0 ** -24) + (4 * S + 8) * 2.0 ** -23
    top = np.array([max([np.abs(ref.rows(b, range(T[b]))[2]).max(initial=0.0)]) for b in range(B)])
    o, l = to_host64(O), to_host64(L)
    tol = 2.0 ** -8 * (A + np.abs(want)) * 1.01 + (2 * D * top[:, None])[..., None]
    err = np.abs(o - want)
    assert np.all(err <= tol), (err - tol).max()
    empty = ~np.isfinite(lse)
    assert np.array_equal(l[empty], lse[empty]) and not np.any(o[empty])
    l, lse, D = l[~empty], lse[~empty], D[~empty]
    assert np.all(np.abs(l - lse) <= D + np.abs(lse) * 2.0 ** -22 + 2.0 ** -22)


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("d,r,interleaved,page", [(32, 32, False, 16), (64, 32, True, 32), (64, 0, False, 16), (128, 128, False, 16),
                                                  (128, 0, False, 128), (128, 64, True, 64)])
def test_decode_lengths(bits, append, d, r, interleaved, page):
    decode_case(EDGES, 8, 2, page, d, bits, r, interleaved, append, seed=d + r + page)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (16, 1), (17, 1), (32, 1), (33, 1), (64, 2), (40, 1), (70, 1)])
def test_decode_groups(bits, d, Hq, Hkv):
    decode_case([200, 3, 77], Hq, Hkv, 16, d, bits, r=d, seed=Hq, packed=True)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 8, 9, 16, 20])
def test_decode_groups_in_large_pages(bits, d, G):
    """Blocks inside one page (64 tokens and more), ends at and beside its edges."""
    decode_case([0, 63, 64, 65, 128, 200, 255, 256, 257], 2 * G, 2, 64 if G % 2 else 128, d, bits, r=d // 2, seed=G, spoil=[(5, 1)])


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_many_splits(bits, d):
    """One long sequence and short ones beside it: splits that hold nothing."""
    decode_case([9000, 1, 4097, 0], 8, 1, 64, d, bits, r=d, seed=5)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("G", [17, 32, 33])
@pytest.mark.parametrize("page", [16, 64])
def test_decode_groups_in_large_batches(bits, d, G, page):
    """Enough keys for two columns of query heads in a workgroup: split, and in one part."""
    decode_case([0, 300, 64, 33], G, 1, page, d, bits, r=32, n=40000, width=40000 // page + 1, seed=G)
    lens = [int(x) for x in np.random.default_rng(G).integers(0, 701, 200)]
    decode_case(lens, G, 1, page, d, bits, r=32, n=700, width=701 // page + 1, seed=G, packed=True)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_decode_joins_hundreds_of_splits(bits, d):
    """One cache head; the lengths fill all of the splits, a few, one, none but the new row's."""
    for x, n in ((40000, 40000), (19000, 40000), (70, 40000), (0, 40000)):
        decode_case([x], 3, 1, 16, d, bits, r=32, n=n, width=2501, seed=x + 1)
    decode_case([0], 3, 1, 16, d, bits, append=False, n=40000, width=2501)


@pytest.mark.parametrize("bits", [16, 4])
def test_decode_bad_pages(bits):
    """Numbers outside the pool inside a sequence: those tokens do not take part, the
    new row among them is not written; a sequence with none left."""
    decode_case([100, 40, 70, 15], 4, 2, 16, 64, bits, r=64, spoil=[(0, 0), (0, 3), (0, 6), (1, 2), (3, 0)], seed=3)
    decode_case([100, 40, 70, 15], 4, 2, 32, 128, bits, append=False, spoil=[(0, 0), (1, 0), (1, 1), (2, 2)], seed=4)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("bad", [float("inf"), NAN])
def test_new_row_without_a_page_stays_out(bits, page, bad):
    """The newest token has no page: its values, finite or not, do not touch the result,
    which is that of the tokens before it."""
    pool = Pool([page + 1, 1], 1, page, 64, bits).fill([page, 0])
    pool.t_table[0, 1] = pool.t_table[1, 0] = -1
    q = torch.randn(2, 4, 64, device="cuda").to(BF16)
    new = torch.full((2, 1, 64), bad, device="cuda").to(BF16)
    want = lib.attn_paged_decode(q, lens=ints([page, 0]), **pool.args())
    for k, v in ((q[:, :1], new), (new, q[:, :1]), (new, new)):
        got = lib.attn_paged_decode(q, lens=ints([page, 0]), k_new=k.contiguous(), v_new=v.contiguous(), **pool.args())
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 0.5, 3.0])
def test_decode_scales(bits, scale):
    decode_case([300, 20], 8, 2, 16, 64, bits, r=32, scale=scale, seed=8)


@pytest.mark.parametrize("bits", [16, 4])
def test_decode_positions_and_bounds(bits):
    """Given positions; n above, at and (clamping) below the lengths; a table wider than
    needed; peaked rows."""
    decode_case([300, 20, 150], 8, 2, 16, 64, bits, r=64, pos=[5, 100000, -3], seed=1)
    decode_case([300, 20, 150], 8, 2, 16, 64, bits, r=64, n=4000, width=300, seed=2)
    decode_case([300, 20, 150], 8, 2, 16, 64, bits, r=64, n=300, seed=3)
    decode_case([600, 600], 8, 2, 16, 128, bits, r=64, sigma=6.0, seed=4)


@pytest.mark.parametrize("bits", [16, 4])
def test_decode_clamps_lengths(bits):
    """Lengths past n count as n, negative ones as 0; the append follows."""
    pool = Pool([64, 64, 64], 1, 16, 64, bits).fill([60, 60, 60])
    q, k, v = (torch.randn(3, h, 64, device="cuda").to(BF16) for h in (2, 1, 1))
    want = [lib.attn_paged_decode(q, lens=ints([40, 0, 33]), **pool.args()),
            lib.attn_paged_decode(q, lens=ints([10**9, -5, 33]), n=40, **pool.args())]
    assert all(torch.equal(x, y) for x, y in zip(*want))
    before = pool.state()
    lib.attn_paged_decode(q, lens=ints([10**9, -5, 33]), k_new=k, v_new=v, n=40, **pool.args())
    K, V = lib.attn_paged_gather(lens=ints([64] * 3), n=1, starts=ints([40, 0, 33]), **pool.args())
    assert same(to_host64(K)[:, :, 0], stored(to_host64(k), bits)) and same(to_host64(V)[:, :, 0], stored(to_host64(v), bits))
    rows = [((x != y) & ~(torch.isnan(x) & torch.isnan(y))).any(-1).sum() for x, y in zip(pool.state()[:2], before)]
    assert sum(map(int, rows)) <= 6   # the three new rows of K and V


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n", [100, 5000])
def test_decode_not_a_number(bits, n):
    """A NaN inside the sequence reaches exactly the heads that read it; NaN in a query
    its own head; unsplit and split."""
    pool = Pool([n, n], 2, 16, 64, bits).fill([n, n])
    q = torch.randn(2, 4, 64, device="cuda").to(BF16)
    q[1, 3, 7] = NAN
    at = int(pool.table[0, 2])
    if bits == 16:
        pool.v[at, 1, 5, 9] = NAN
    else:
        pool.v[at, 1, 5, :16], pool.scales["v_scales"][at, 1, 5, 0] = 0, 255
    O, L = lib.attn_paged_decode(q, lens=ints([n, n]), **pool.args())
    bad = torch.isnan(O)
    cols = range(9, 10) if bits == 16 else range(32)
    assert {tuple(x) for x in bad.nonzero().tolist()} == \
        {(0, h, c) for h in (2, 3) for c in cols} | {(1, 3, c) for c in range(64)}
    assert torch.isnan(L).nonzero().tolist() == [[1, 3]]
    if bits == 16:
        pool.k[at, 0, 5, 9] = NAN
    else:
        pool.scales["k_scales"][at, 0, 5, 1] = 255
    O, L = lib.attn_paged_decode(q, lens=ints([n, n]), **pool.args())
    assert bool(torch.isnan(O[0, :2]).all()) and bool(torch.isnan(L[0, :2]).all())


@pytest.mark.parametrize("bits", [16, 4])
def test_pool_past_32_bits(bits):
    """Pages behind 2^32 bytes and 2^31 elements of a pool."""
    d, page, Hkv, n = 128, 128, 8, 300
    num = 2**31 // (d * page * Hkv) * (1 if bits == 16 else 2) + 9
    shape = (num, Hkv, page)
    far = [num - 1, num - 5, num - 3]
    small = Pool([n], Hkv, page, d, bits).fill([n - 1])
    table = ints(far)[None]
    big = {"k_pages": torch.empty(shape + (small.k.shape[3],), dtype=small.k.dtype, device="cuda")}
    big["v_pages"] = torch.empty_like(big["k_pages"])
    big.update({x: torch.empty(shape + (d // 32,), dtype=torch.uint8, device="cuda") for x in small.scales})
    for i, p in enumerate(far):
        for name, x in small.args().items():
            if name != "block_table":
                big[name][p] = x[int(small.table[0, i])]
    q, k, v = (torch.randn(1, h, d, device="cuda").to(BF16) for h in (16, Hkv, Hkv))
    freqs, a = lib.attn_rope_freqs(d)
    args = dict(lens=ints([n - 1]), k_new=k, v_new=v, freqs=freqs, amplitude=a)
    want = lib.attn_paged_decode(q, **args, **small.args())
    got = lib.attn_paged_decode(q, **args, block_table=table, **big)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    lib.attn_paged_append(k[:, :, None], v[:, :, None], lens=ints([n - 1]), freqs=freqs, amplitude=a, **small.args())
    lib.attn_paged_append(k[:, :, None], v[:, :, None], lens=ints([n - 1]), freqs=freqs, amplitude=a, block_table=table, **big)
    want = lib.attn_paged_gather(lens=ints([n]), n=n, **small.args())
    got = lib.attn_paged_gather(lens=ints([n]), n=n, block_table=table, **big)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("bits", [16, 4])
def test_shared_pages(bits):
    """Two sequences with the same prefix pages, each with its own last one."""
    pool = Pool([40, 40], 2, 16, 64, bits).fill([39, 39])
    pool.table[1, :2] = pool.table[0, :2]
    pool.t_table.copy_(torch.from_numpy(pool.table))
    q, k, v = (torch.randn(2, h, 64, device="cuda").to(BF16) for h in (4, 2, 2))
    O, L = lib.attn_paged_decode(q, lens=ints([39, 39]), k_new=k, v_new=v, **pool.args())
    for b in range(2):
        args = {**pool.args(), "block_table": pool.t_table[b:b + 1].contiguous()}
        o, l = lib.attn_paged_decode(q[b:b + 1], lens=ints([40]), n=39 + 1, **args)
        assert torch.equal(o[0], O[b]) and torch.equal(l[0], L[b])


# ------------------------------------------------------------- as they are used --
@pytest.mark.parametrize("bits", [16, 4])
def test_prompt_then_tokens(bits):
    """A prompt is rotated and attended (attn_rope, attn_fwd), written in two chunks,
    then tokens follow one by one from a captured graph that moves the lengths on.
    Every token's output against the oracle over what the cache holds (bf16: also
    attn_fwd over the whole sequence); eager work between the replays."""
    B, H, n, more, d, page = 2, 4, 75, 6, 64, 16
    freqs, a = lib.attn_rope_freqs(d)
    g = torch.Generator(device="cuda").manual_seed(0)
    qkv = torch.randn(B, n + more, 3 * H, d, device="cuda", generator=g).to(BF16).transpose(1, 2)
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    qr, kr = lib.attn_rope(q, k, freqs, a)
    full, _ = lib.attn_fwd(qr, kr, v.contiguous(), causal=True)
    pool = Pool([n + more] * B, H, page, d, bits)
    lens = ints([0] * B)
    for lo, hi in ((0, 33), (33, n)):
        lib.attn_paged_append(k[:, :, lo:hi], v[:, :, lo:hi], lens=lens, freqs=freqs, amplitude=a, **pool.args())
        lens += hi - lo
    K, V = lib.attn_paged_gather(lens=lens, n=n, **pool.args())
    if bits == 16:
        assert torch.equal(K, kr[:, :, :n]) and torch.equal(V, v[:, :, :n])
    qt, kt, vt = (torch.empty(B, H, d, dtype=BF16, device="cuda") for _ in range(3))
    O, L = torch.empty(B, H, d, dtype=BF16, device="cuda"), torch.empty(B, H, device="cuda")
    start = pool.state()

    def step():
        lib.attn_paged_decode(qt, lens=lens, k_new=kt, v_new=vt, freqs=freqs, amplitude=a, out=(O, L), **pool.args())
        lens.add_(1)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(more):
        for dst, src in ((qt, q), (kt, k), (vt, v)):
            dst.copy_(src[:, :, n + i])
        graph.replay()
        torch.cuda.synchronize()
        assert lens.tolist() == [n + i + 1] * B
        ref = pool.oracle()
        qh = paged.rotate(to_host64(qt), np.full((B, H), n + i), freqs.cpu().numpy(), a)
        want, lse, A, S = ref.attend(qh, [n + i + 1] * B, d ** -0.5)
        D = S * (2.0 ** -16 + d * 2.0 ** -24) + (4 * S + 8) * 2.0 ** -23
        tol = 2.0 ** -8 * (A + np.abs(want)) * 1.01 + (2 * D * np.abs(to_host64(v)).max() * 1.2)[..., None]
        assert np.all(np.abs(to_host64(O) - want) <= tol)
        kept = O.clone()
        o, l = lib.attn_paged_decode(qt, lens=lens, freqs=freqs, amplitude=a, **pool.args())   # the same token, already there
        torch.cuda.synchronize()
        assert torch.equal(o, kept) and torch.equal(l, L)
        if bits == 16:
            assert float((kept.float() - full[:, :, n + i].float()).abs().max()) <= 2.0 ** -6 * float(full.float().abs().max())
    assert not torch.equal(start[0].view(torch.uint8), pool.k.view(torch.uint8))


@pytest.mark.parametrize("bits", [16, 4])
def test_streams_workspaces_and_two_graphs(bits):
    """Another stream, a workspace larger than needed and reused between sizes, and two
    captured graphs that share it, replayed in turn."""
    small, large = Pool([200], 1, 16, 128, bits, seed=1).fill([200]), Pool([6000, 10], 1, 16, 128, bits, seed=2).fill([6000, 10])
    calls = []
    for pool, lens in ((small, [200]), (large, [6000, 10])):
        q = torch.randn(len(lens), 8, 128, device="cuda").to(BF16)
        calls.append(dict(q=q, lens=ints(lens), **pool.args()))
    want = [lib.attn_paged_decode(**c) for c in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [lib.attn_paged_decode(**c) for c in calls]
    side.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for c in calls:
        out = (torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda"))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lib.attn_paged_decode(**c, out=out, workspace=ws)
        graphs.append(graph)
        outs.append(out)
    for _ in range(3):
        for x in outs:
            x[0].zero_()
        ws.fill_(255)   # not-a-number in whatever is read before it is written
        graphs[0].replay()
        graphs[1].replay()
        lib.attn_paged_decode(**calls[0], workspace=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(outs, want) for x, y in zip(a, b))


@pytest.mark.parametrize("bits", [16, 4])
def test_native_and_python_forms_agree(bits, monkeypatch):
    freqs, a = lib.attn_rope_freqs(64)
    pool = Pool([300, 300], 2, 16, 64, bits).fill([290, 290])
    lens = ints([280, 17])
    q, k, v = (torch.randn(2, h, 64, device="cuda").to(BF16) for h in (8, 2, 2))
    kc = torch.randn(2, 2, 5, 64, device="cuda").to(BF16)
    p = pool.args()
    calls = [lambda: lib.attn_paged_decode(q, lens=lens, **p), lambda: lib.attn_paged_decode(q, lens=lens, k_new=k, v_new=v, n=280,
                                                                                          scale=0.3, freqs=freqs, **p),
             lambda: lib.attn_paged_append(kc, kc, lens=lens, new_lens=ints([2, 5]), freqs=freqs, interleaved=True, **p),
             lambda: lib.attn_paged_gather(lens=lens, n=9, starts=ints([275, 0]), **p),
             lambda: lib.attn_paged_decode(q, lens=lens, out=(torch.empty_like(q), None), positions=ints([3, 4]), freqs=freqs, **p)]
    bad = [lambda: lib.attn_paged_decode(q, lens=lens, n=10**6, **p), lambda: lib.attn_paged_decode(q[:, :7], lens=lens, **p),
           lambda: lib.attn_paged_decode(q, lens=lens, scale=float("nan"), **p),
           lambda: lib.attn_paged_append(kc, kc[:, :1], lens=lens, **p),
           lambda: lib.attn_paged_append(kc, kc, lens=lens, freqs=freqs[:5].clone(), **p),
           lambda: lib.attn_paged_gather(lens=lens, n=0, **p)]
    start = pool.state()
    assert lib._native is not None

    def each(call, form):
        for x, y in zip((pool.k, pool.v, *pool.scales.values()), start):
            x.copy_(y)
        with monkeypatch.context() as m:
            if not form:
                m.setattr(lib, "_native_lib", None)
            return form_call(call)

    def form_call(call):
        try:
            return call(), pool.state()
        except (ValueError, TypeError, lib.AttnError) as e:
            return type(e), str(e)

    for call in calls:
        (x, s), (y, t) = each(call, True), each(call, False)
        assert (x is None) == (y is None)
        for u, w in zip(x or (), y or ()):
            assert u is w is None or torch.equal(u, w) and u.stride() == w.stride()
        assert all(torch.equal(u.view(torch.uint8), w.view(torch.uint8)) for u, w in zip(s, t))
    for call in bad:
        x, y = each(call, True), each(call, False)
        assert isinstance(x[1], str) and x == y
