"""attn_cross_fwd and attn_cross_bwd on the GPU against the float64 oracle (oracle/cross.py), within
the bounds of cross_bounds.py."""
import itertools

import numpy as np
import pytest
import torch

import paper_2609_33916_amd as lib
from cross_bounds import bounds, check
from helpers import gpu_available, to_host64
from oracle import cross

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


class Call:
    """Seeded inputs of one call, its run on the GPU and the oracle's answer."""

    def __init__(self, B, Hq, Hkv, nq, nk, d, dtype, seed=0, causal=False, start=0, starts=None, k_lens=None, buckets=None,
                 packed=False, scale=None, sigma=1.0):
        rng = np.random.default_rng([seed, B, Hq, Hkv, nq, nk, d])
        self.dtype, self.d = dtype, d
        self.how = dict(causal=causal, start=start, starts=starts, k_lens=k_lens)
        self.scale = d ** -0.5 if scale is None else scale

        def draw(*shape):
            return torch.tensor(rng.standard_normal(shape) * sigma, dtype=dtype, device="cuda")
        if packed:   # heads behind tokens, K and V in one projection
            self.q, kv = draw(B, nq, Hq, d).transpose(1, 2), draw(B, nk, 2 * Hkv, d).transpose(1, 2)
            self.k, self.v = kv[:, :Hkv], kv[:, Hkv:]
            self.do = draw(B, nq, Hq, d).transpose(1, 2)
        else:
            self.q, self.k, self.v, self.do = draw(B, Hq, nq, d), draw(B, Hkv, nk, d), draw(B, Hkv, nk, d), draw(B, Hq, nq, d)
        self.bias = None
        if buckets:
            self.bias = draw(buckets[0], Hq)
            self.rows, self.first = lib.attn_bias_buckets(*buckets)

    def args(self):
        how = dict(self.how, starts=ints(self.how["starts"]), k_lens=ints(self.how["k_lens"]), scale=self.scale)
        if self.bias is not None:
            how.update(bias=self.bias, bias_rows=self.rows, bias_first=self.first)
        return how

    def run(self, backward=True):
        O, L = lib.attn_cross_fwd(self.q, self.k, self.v, **self.args())
        got = {"O": O, "L": L}
        if backward:
            g = lib.attn_cross_bwd(self.q, self.k, self.v, O, L, self.do, **self.args())
            got.update(zip(("dQ", "dK", "dV", "dBias"), g))
        torch.cuda.synchronize()
        return got

    def ref(self, backward=True):
        x = [to_host64(t) for t in (self.q, self.k, self.v)]
        how = dict(self.how)
        if self.bias is not None:
            how.update(bias=to_host64(self.bias), rows=self.rows.cpu().numpy(), first=self.first)
        do = to_host64(self.do) if backward else None
        ref = cross.attention(*x, self.scale, do=do, **how)
        return ref, bounds(*x, self.scale, self.dtype == BF16, ref, do=do, **how)

    def check(self, backward=True, what=""):
        got = self.run(backward)
        ref, bound = self.ref(backward)
        check({name: to_host64(x) for name, x in got.items()}, ref, bound, what)
        return got


SHAPES = [  # B, Hq, Hkv, nq, nk
    (1, 1, 1, 1, 1), (2, 2, 2, 1, 33), (1, 4, 2, 3, 64), (2, 3, 3, 31, 65), (1, 8, 1, 32, 1), (1, 2, 1, 33, 127),
    (2, 4, 4, 65, 128), (1, 6, 2, 127, 129), (1, 2, 2, 128, 200), (2, 2, 1, 129, 95), (1, 1, 1, 300, 31), (1, 12, 4, 5, 700),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(shape, d, dtype):
    for packed in (False, True):
        Call(*shape, d, dtype, packed=packed).check(what=f"packed={packed}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("G", [1, 4])
def test_large_grid(d, dtype, G):
    """More than 256 tiles of 128 queries: the kernels of large grids."""
    Call(2, 64, 64 // G, 260, 333, d, dtype, k_lens=[333, 190], packed=True).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_few_queries_on_many_keys(d, dtype):
    """128 rows a workgroup, the keys in parts: heads of a group as rows, masks, a bias."""
    Call(1, 4, 2, 101, 16500, d, dtype, k_lens=[16400], packed=True).check(False)
    Call(2, 2, 1, 150, 12000, d, dtype, causal=True, starts=[11850, 5], k_lens=[12000, 9000]).check(False)
    Call(1, 4, 2, 131, 9000, d, dtype, causal=True, start=8800, buckets=(32, 128, False)).check(False)


def some_heads(c, heads, what):
    """A call of many heads on one cache head against the oracle of some of them."""
    got = c.run(False)
    one = Call(1, 1, 1, 1, 1, c.d, c.dtype)
    one.how, one.scale = c.how, c.scale
    one.q, one.k, one.v = c.q[:, heads], c.k[:, :1], c.v[:, :1]
    ref, bound = one.ref(False)
    check({n: to_host64(got[n][:, heads]) for n in ("O", "L")}, ref, bound, what)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_large_grids_in_parts(d, dtype):
    """Grids of 256 and 290 tiles of 128 queries on keys long enough to split."""
    for B, H, nq, how in ((1, 256, 70, {}), (1, 290, 65, {"causal": True, "start": 6200 - 65})):
        c = Call(B, H, 1, nq, 6200, d, dtype, k_lens=[6170], **how)
        c.k, c.v = c.k.expand(B, H, -1, -1), c.v.expand(B, H, -1, -1)
        some_heads(c, [0, 1, H // 2, H - 1], str((H, nq)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_rows_of_a_group_undivided(d, dtype):
    """256 tiles of a group's rows and more, few queries each: 128 rows a workgroup, all keys."""
    Call(32, 16, 8, 20, 77, d, dtype, k_lens=[77 - 2 * i for i in range(32)]).check(False)
    Call(64, 16, 4, 13, 90, d, dtype, causal=True, start=77).check(False)
    Call(64, 8, 4, 33, 70, d, dtype, buckets=(32, 128)).check(False)


@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("nk", [2, 3, 5])
def test_few_keys_many_queries(nk, G):
    """dK and dV of few keys are off by their own last rounding: uniform within half a step, at most 2^-8 of the value, so
    2^-8 / sqrt(3) in the norm; the mean of n such squares lies within 3 sqrt(0.8 / n) of theirs."""
    c = Call(1, 4, 4 // G, 1892, nk, 128, BF16, packed=True)
    got, (ref, _) = c.run(), c.ref()
    for name in ("dK", "dV"):
        x, y = to_host64(got[name]), ref[name]
        most = 2.0 ** -8 * np.sqrt((1 + 3 * np.sqrt(0.8 / x.size)) / 3)
        off = np.linalg.norm(x - y) / np.linalg.norm(y)
        assert off <= most, (name, off, most)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nk,lens", [(70, 200, [200, 0, 1, 77, 128]), (1, 300, [0, 300, 1, 64, 65]), (200, 64, [64, 0, 32, 33, 63]),
                                        (5, 40, [-3, 41, 40, 7, 100])])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(nq, nk, lens, d, dtype):
    """Lengths of 0 and 1, outside [0, nk], and what lies behind them not a number."""
    c = Call(5, 4, 2, nq, nk, d, dtype, k_lens=lens)
    for b, n in enumerate(lens):
        for x in (c.k, c.v):
            x[b, :, max(n, 0):] = NAN
    got = c.run()
    clean = Call(5, 4, 2, nq, nk, d, dtype, k_lens=lens)
    ref, bound = clean.ref()
    check({name: to_host64(x) for name, x in got.items()}, ref, bound)
    for b, n in enumerate(lens):
        assert (got["dK"][b, :, max(n, 0):] == 0).all() and (got["dV"][b, :, max(n, 0):] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nk,start", [(64, 64, 0), (100, 300, 200), (100, 300, 150), (130, 40, 0), (200, 100, -120), (1, 77, 76), (1, 77, 30),
                                         (40, 90, -41), (300, 300, 0), (70, 500, 1000)])
def test_causal(nq, nk, start, dtype):
    """Chunks of a sequence, queries before the first key and behind the last one."""
    Call(2, 4, 2, nq, nk, 64, dtype, causal=True, start=start, k_lens=[nk, nk // 2]).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_causal_starts(dtype):
    lens = [300, 150, 0, 90]
    Call(4, 2, 2, 60, 300, 64, dtype, causal=True, starts=[240, 90, -60, 95], k_lens=lens).check()
    Call(4, 4, 2, 1, 300, 128, dtype, causal=True, starts=[299, 149, -1, 89], k_lens=lens).check()
    Call(4, 4, 2, 3, 300, 32, dtype, causal=True, starts=[2 ** 31 - 1, -2 ** 31, 10, 299], k_lens=lens).check()


def test_causal_large_grid():
    Call(2, 64, 16, 260, 520, 64, BF16, causal=True, start=200).check()
    Call(2, 128, 32, 130, 390, 128, BF16, causal=True, start=260, k_lens=[390, 300]).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("buckets", [(32, 128, True), (32, 128, False), (16, 20, True), (4, 5, False), (64, 700, True)], ids=str)
def test_bias(buckets, d, dtype):
    """Tiles before, among and behind the positions that have a bias of their own."""
    for nq, nk, how in [(200, 200, {}), (333, 333, {"causal": True}), (1, 500, {"start": 499}), (77, 450, {"causal": True, "start": 373}),
                        (150, 400, {"k_lens": [400, 0]}), (40, 700, {"start": -300}), (64, 640, {"start": 900})]:
        Call(2, 4, 2, nq, nk, d, dtype, buckets=buckets, **how).check(what=str((nq, nk, how)))
    Call(2, 12, 2, 7, 300, d, dtype, buckets=buckets, causal=True, start=290).check(what="grouped heads")
    Call(1, 40, 1, 3, 90, d, dtype, buckets=buckets, k_lens=[70]).check(what="40 heads on one")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_bias_large_grid(d, dtype):
    for how in ({}, {"causal": True}):
        Call(2, 96, 48, 390, 390, d, dtype, buckets=(32, 128, not how), k_lens=[390, 200], **how).check(what=str(how))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_few_queries_large_grid_of_keys(d, dtype):
    for how in ({}, {"causal": True, "start": 1500}, {"buckets": (32, 128), "start": 1000}):
        Call(2, 32, 16, 5, 1100, d, dtype, k_lens=[1100, 700], **how).check(what=str(how))
        Call(1, 16, 16, 300, 2100, d, dtype, **how).check(what=str(how))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_bias_backward_in_parts_of_queries(d, dtype):
    """Few heads, many queries: a head's queries in parts, some of which see no key of a block, or none of a short sequence."""
    for how in ({}, {"causal": True}, {"causal": True, "start": -700}, {"start": 5, "k_lens": [0]}, {"k_lens": [300]}):
        Call(1, 2, 1, 1100, 700, d, dtype, buckets=(32, 128, "causal" not in how), **how).check(what=str(how))
    Call(1, 1, 1, 600, 17000, d, dtype, buckets=(32, 128), start=8000).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bias_positions_of_all_sizes(dtype):
    """2 to 2048 positions of their own, in no order, some of no bucket, and far from the queries."""
    rng = np.random.default_rng(5)
    for R, first, start in ((2, 0, 0), (2, -70, 3), (3, 40, -20), (2048, -1000, 0), (2048, -900, 500), (700, 300, -200)):
        c = Call(2, 3, 3, 150, 330, 64, dtype, buckets=(32, 128), start=start)
        c.rows, c.first = ints(rng.integers(-2, 35, R).tolist()), first
        c.check(what=str((R, first, start)))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bias_masks(dtype):
    """Entries of -inf hide their positions, and so does the type's lowest value; a row may see nothing at all."""
    c = Call(2, 2, 2, 100, 230, 64, dtype, buckets=(32, 128))
    c.bias[3:20, 0] = -float("inf")
    c.bias[:, 1] = torch.finfo(dtype).min
    c.bias[5, 1] = 0
    c.check()
    for low in (-float("inf"), torch.finfo(dtype).min):
        c.bias[:] = low
        got = c.run()
        assert (got["O"] == 0).all() and (got["L"] == -float("inf")).all()
        assert all((got[x] == 0).all() for x in ("dQ", "dK", "dV", "dBias"))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale, dtype):
    for nq in (20, 140):
        Call(1, 4, 2, nq, 150, 64, dtype, scale=scale, buckets=(32, 128)).check()
        Call(1, 4, 2, nq, 150, 64, dtype, scale=scale, causal=True, start=10).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(dtype):
    """Every tensor a view of another kind: tokens first, batches last, gaps, keys shared by a batch, one head's."""
    B, Hq, Hkv, nq, nk, d = 3, 4, 2, 70, 150, 64
    base = Call(B, Hq, Hkv, nq, nk, d, dtype, k_lens=[150, 100, 3])
    ref, bound = base.ref()
    orders = list(itertools.permutations(range(3)))
    for i, order in enumerate(orders):
        c = Call(B, Hq, Hkv, nq, nk, d, dtype, k_lens=[150, 100, 3])

        def spread(x, order=order, gap=8 * (i % 3)):
            shape = [x.shape[a] for a in order]
            y = torch.full((*shape, d + gap), NAN, dtype=x.dtype, device="cuda")[..., :d]
            back = [order.index(a) for a in range(3)]
            y = y.permute(*back, 3)
            y.copy_(x)
            return y
        for name, o in zip(("q", "k", "v", "do"), orders[i:] + orders[:i]):
            setattr(c, name, spread(getattr(c, name), o))
        O, L = spread(torch.zeros_like(base.q)), torch.empty(B, Hq, nq, device="cuda")
        lib.attn_cross_fwd(c.q, c.k, c.v, out=(O, L), **c.args())
        out = [spread(torch.zeros_like(x), o) for x, o in zip((base.q, base.k, base.v), orders[::-1])]
        lib.attn_cross_bwd(c.q, c.k, c.v, O, L, c.do, out=out, **c.args())
        check({n: to_host64(x) for n, x in zip(("O", "L", "dQ", "dK", "dV"), (O, L, *out))}, ref, bound, str(order))
        for x in (O, *out):   # the gaps as they were
            if x.stride(-2) > d or min(s for s, n in zip(x.stride()[:3], x.shape[:3]) if n > 1) > d:
                whole = torch.as_strided(x, (x.numel() // d, min(s for s in x.stride()[:3])), (min(s for s in x.stride()[:3]), 1))
                assert whole[:, d:].isnan().all()
    # a batch's shared keys: strides of 0, gradients for every sequence
    c = Call(B, Hq, Hkv, nq, nk, d, dtype)
    c.k, c.v = c.k[:1].expand(B, -1, -1, -1), c.v[:1].expand(B, -1, -1, -1)
    got = c.check()
    assert got["dK"].shape == (B, Hkv, nk, d)


@pytest.mark.parametrize("nq", [1, 40, 200])
def test_far_offsets(nq):
    """Rows farther than 2^32 bytes from the first."""
    B, H, nk, d = 1, 2, 1100, 64
    step = 2 ** 21
    room = torch.empty(nk * step, dtype=BF16, device="cuda")
    c = Call(B, H, H, nq, nk, d, BF16, causal=True, start=nk - nq)

    def far(x, at):
        y = torch.as_strided(room, x.shape, (0, 2 * d, step, 1), at)
        y.copy_(x)
        return y
    c.k, c.v = far(c.k, 0), far(c.v, d)
    c.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_same_bits(dtype):
    """Every call gives the same bits, with sums in parts and with a bias gradient."""
    for how in (dict(B=1, Hq=4, Hkv=1, nq=90, nk=900), dict(B=2, Hq=4, Hkv=2, nq=300, nk=300, buckets=(32, 128))):
        how = dict(how)
        c = Call(**how, d=64, dtype=dtype)
        first = c.run()
        for _ in range(3):
            again = c.run()
            assert all(torch.equal(first[x], again[x]) for x in first)


def test_batches_do_not_matter():
    """A sequence's O and gradients within their rounding whatever the batch is split into."""
    c = Call(4, 4, 2, 100, 500, 64, BF16, k_lens=[500, 3, 250, 499])
    c.check()
    one = Call(4, 4, 2, 100, 500, 64, BF16, k_lens=[500, 3, 250, 499])
    ref, bound = one.ref()
    for b in range(4):
        part = Call(1, 4, 2, 100, 500, 64, BF16, k_lens=[one.how["k_lens"][b]])
        for x in ("q", "k", "v", "do"):
            setattr(part, x, getattr(one, x)[b:b + 1])
        got = part.run()
        check({n: to_host64(x) for n, x in got.items()}, {n: x[b:b + 1] for n, x in ref.items()}, {n: x[b:b + 1] for n, x in bound.items()})


def test_gradients_by_differences():
    """float32 gradients against differences of the float64 oracle's sum of O dO, bias and shared heads included."""
    c = Call(2, 4, 2, 9, 13, 32, F32, buckets=(8, 6), k_lens=[13, 8], causal=True, start=4, sigma=0.7)
    got = c.run()
    x = {n: to_host64(getattr(c, n)) for n in ("q", "k", "v", "bias")}
    do = to_host64(c.do)

    def loss(v):
        return (cross.attention(v["q"], v["k"], v["v"], c.scale, bias=v["bias"], rows=c.rows.cpu().numpy(), first=c.first, **c.how)["O"]
                * do).sum()
    rng = np.random.default_rng(1)
    for name, grad in (("q", "dQ"), ("k", "dK"), ("v", "dV"), ("bias", "dBias")):
        g = to_host64(got[grad])
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in x[name].shape)
            diff = 0.0
            for sign in (1, -1):
                y = dict(x)
                y[name] = x[name].copy()
                y[name][at] += sign * 1e-5
                diff += sign * loss(y) / 2e-5
            # differences: third derivatives times 1e-10, roundings 2^-53 of a loss below 1e3 over 1e-5;
            # the gradient: some hundred float32 roundings of terms below 10
            assert abs(diff - g[at]) < 1e-4, (name, at, diff, g[at])


def test_other_stream_and_capture():
    """On a stream of its own; captured, replayed on other inputs, with eager calls between."""
    c = Call(2, 4, 2, 90, 400, 64, BF16, buckets=(32, 128), k_lens=[400, 170])
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run()
    assert all(torch.equal(want[x], got[x]) for x in want)
    how = c.args()
    nws = lib.lib().attn_cross_bwd_workspace_bytes(2, 4, 2, 90, 400, 64, 0, len(c.rows))
    ws = torch.empty(nws, dtype=torch.uint8, device="cuda")
    out = {x: torch.empty_like(want[x]) for x in want}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.attn_cross_fwd(c.q, c.k, c.v, out=(out["O"], out["L"]), **how)
        lib.attn_cross_bwd(c.q, c.k, c.v, out["O"], out["L"], c.do, out=[out[x] for x in ("dQ", "dK", "dV", "dBias")], workspace=ws, **how)
    for seed in (1, 2, 3):
        other = Call(2, 4, 2, 90, 400, 64, BF16, buckets=(32, 128), k_lens=[400, 170], seed=seed)
        for x in ("q", "k", "v", "do", "bias"):
            getattr(c, x).copy_(getattr(other, x))
        want = other.run()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[x], out[x]) for x in want), seed


def test_bias_without_its_gradient():
    c = Call(2, 4, 2, 60, 300, 64, BF16, buckets=(32, 128))
    want = c.run()
    out = [torch.empty_like(want[x]) for x in ("dQ", "dK", "dV")] + [None]
    lib.attn_cross_bwd(c.q, c.k, c.v, want["O"], want["L"], c.do, out=out, **c.args())
    ref, bound = c.ref()
    check({n: to_host64(x) for n, x in zip(("dQ", "dK", "dV"), out)}, {n: ref[n] for n in ("dQ", "dK", "dV")}, bound)


def test_values_of_rows_behind():
    """Infinite values behind a length and a causal query's far future leave the others alone."""
    c = Call(1, 2, 2, 64, 600, 64, BF16, causal=True, start=100, k_lens=[500])
    ref, bound = c.ref()
    c.v[:, :, 300:] = float("inf")   # the last query's place is 163
    c.k[:, :, 300:] = NAN
    got = c.run()
    for name in ("O", "L", "dQ"):
        check({name: to_host64(got[name])}, {name: ref[name]}, bound)


def test_decode_steps_are_a_causal_call():
    """A sequence's tokens one by one over a growing cache, under a bias, are the rows of one causal call."""
    B, H, n, d = 2, 4, 150, 64
    c = Call(B, H, 2, n, n, d, BF16, causal=True, buckets=(32, 128, False))
    ref, bound = c.ref(False)
    how = c.args()
    rows = []
    for i in range(n):
        how.update(starts=ints([i] * B), k_lens=ints([i + 1] * B), start=0)
        rows.append(lib.attn_cross_fwd(c.q[:, :, i:i + 1], c.k, c.v, **how))
    got = {"O": torch.cat([o for o, _ in rows], 2), "L": torch.cat([l for _, l in rows], 2)}
    check({x: to_host64(y) for x, y in got.items()}, ref, bound)


def test_layer_of_an_encoder_and_a_decoder():
    """Biased self-attention, attention to padded states, and back, as a training step runs them, against
    float64 autograd of the formulas on the same bfloat16 tensors. Outputs that the next part takes are
    rounded to bfloat16 by both. Bound: each of the six roundings that a gradient passes is off by 2^-8 of
    terms whose sum of squares is at most that of the result's terms; of the largest gradient, 6 2^-8."""
    torch.manual_seed(3)
    B, H, n, m, d = 2, 4, 96, 150, 64
    lens = [150, 61]
    x, y, z = (torch.randn(B, H, n, d, device="cuda").to(BF16) for _ in range(3))
    ek, ev = (torch.randn(B, H, m, d, device="cuda").to(BF16) for _ in range(2))
    g = torch.randn(B, H, n, d, device="cuda").to(BF16)
    table = torch.randn(32, H, device="cuda").to(BF16)
    rows, first = lib.attn_bias_buckets(32, 128, False)
    bias = dict(bias=table, bias_rows=rows, bias_first=first, causal=True)
    s, sl = lib.attn_cross_fwd(x, y, z, **bias)
    o, ol = lib.attn_cross_fwd(s, ek, ev, k_lens=ints(lens))
    ds, dek, dev = lib.attn_cross_bwd(s, ek, ev, o, ol, g, k_lens=ints(lens))
    dx, dy, dz, dt = lib.attn_cross_bwd(x, y, z, s, sl, ds, **bias)

    leaf = [t.double().cpu().requires_grad_() for t in (x, y, z, ek, ev, table)]
    X, Y, Z, EK, EV, T = leaf
    r = (torch.arange(n)[None] - torch.arange(n)[:, None])
    at = rows.cpu().long()[(r - first).clamp(0, len(rows) - 1)]
    w = X @ Y.transpose(2, 3) / 8 + T[at].permute(2, 0, 1)
    S = torch.softmax(w.masked_fill(r > 0, -torch.inf), 3) @ Z
    S = S + (S.detach().to(BF16).double() - S.detach())
    w = S @ EK.transpose(2, 3) / 8
    O = torch.softmax(w.masked_fill(torch.arange(m)[None, None, None] >= torch.tensor(lens)[:, None, None, None], -torch.inf), 3) @ EV
    O.backward(g.double().cpu())
    for got, want in zip((dx, dy, dz, dek, dev, dt), leaf):
        top = want.grad.abs().max()
        assert (got.double().cpu() - want.grad).abs().max() <= 6 * 2 ** -8 * top
