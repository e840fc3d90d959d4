"""attn_prefix_decode on the GPU against the float64 oracle (oracle/cross.py).

Bounds: as cross_bounds.py, except that P multiplies V in two bfloat16 parts, the first cut (off by
less than a step, 2^-7), the second rounded to half a step of the rest: 2^-15 of P. The new token's
weight and the joining of the parts stay float32. Over the prefix of large batches P is rounded to one
bfloat16: 2^-8 of it."""
import numpy as np
import pytest
import torch

import paper_2609_33916_amd as lib
from cross_bounds import F
from helpers import gpu_available, to_host64
from oracle import cross

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

BF16 = torch.bfloat16
NAN = float("nan")


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


class Step:
    def __init__(self, B, Hq, Hkv, n_p, cap, d, lens, append=True, seed=0, sigma=1.0):
        rng = np.random.default_rng([seed, B, Hq, Hkv, n_p, cap, d])

        def draw(*shape):
            return torch.tensor(rng.standard_normal(shape) * sigma, dtype=BF16, device="cuda")
        self.q, self.k_prefix, self.v_prefix = draw(B, Hq, d), draw(Hkv, n_p, d), draw(Hkv, n_p, d)
        self.k_cache, self.v_cache = draw(B, Hkv, cap, d), draw(B, Hkv, cap, d)
        self.k_new, self.v_new = (draw(B, Hkv, d), draw(B, Hkv, d)) if append else (None, None)
        self.lens, self.d = lens, d

    def host(self):
        return {x: None if getattr(self, x) is None else to_host64(getattr(self, x))
                for x in ("q", "k_prefix", "v_prefix", "k_cache", "v_cache", "k_new", "v_new")}

    def check(self, scale=None, p_bits=2.0 ** -15, **how):
        x = self.host()
        s = self.d ** -0.5 if scale is None else scale
        B, Hq, d = self.q.shape
        cap = x["k_cache"].shape[2]
        top = how.get("n", cap - (x["k_new"] is not None))
        lens = [top if self.lens is None else min(max(n, 0), top) for n in (self.lens or [0] * B)]
        O, L, kc, vc = cross.prefix_decode(x["q"], x["k_prefix"], x["v_prefix"], x["k_cache"], x["v_cache"], lens, s, x["k_new"], x["v_new"])
        gO, gL = lib.attn_prefix_decode(self.q, self.k_prefix, self.v_prefix, self.k_cache, self.v_cache, k_new=self.k_new,
                                        v_new=self.v_new, cache_lens=ints(self.lens), scale=scale, **how)
        torch.cuda.synchronize()
        assert np.array_equal(to_host64(self.k_cache), kc, equal_nan=True) and np.array_equal(to_host64(self.v_cache), vc, equal_nan=True)
        gO, gL = to_host64(gO), to_host64(gL)
        for b in range(B):
            n = lens[b] + (x["k_new"] is not None)
            for h in range(Hq):
                g = h * x["k_prefix"].shape[0] // Hq
                k = np.concatenate((x["k_prefix"][g], kc[b, g, :n]))
                v = np.concatenate((x["v_prefix"][g], vc[b, g, :n]))
                sc = s * (k @ x["q"][b, h])
                p = np.exp(sc - L[b, h])
                dx = F * ((d + 4) * abs(s) * (np.abs(k) @ np.abs(x["q"][b, h])) + 8 * (np.abs(sc) + np.abs(sc).max()))
                e = dx + dx.max() + (len(k) + 8) * F
                bound = 1.02 * (((e + p_bits + len(k) * F) * p) @ np.abs(v) + 2.0 ** -8 * np.abs(O[b, h]))
                assert (np.abs(gO[b, h] - O[b, h]) <= bound).all(), (b, h, (np.abs(gO[b, h] - O[b, h]) / bound).max())
                assert abs(gL[b, h] - L[b, h]) <= 1.02 * (dx.max() + (len(k) + 8) * F + 4 * F * abs(L[b, h])), (b, h)
        return gO, gL


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,n_p,cap,lens", [
    (1, 1, 1, 1, 1, [0]), (2, 4, 2, 33, 5, [0, 4]), (3, 6, 3, 64, 40, [39, 0, 17]), (5, 8, 1, 200, 70, [1, 31, 32, 33, 69]),
    (9, 16, 4, 1000, 300, [299, 0, 5, 100, 128, 129, 255, 256, 64]), (33, 2, 2, 127, 20, list(range(17)) + [3] * 16), (2, 40, 1, 65, 3, [2, 1]),
])
def test_steps(B, Hq, Hkv, n_p, cap, lens, d):
    Step(B, Hq, Hkv, n_p, cap, d, lens).check()


@pytest.mark.parametrize("d", [64, 128])
def test_long_prefix_in_parts(d):
    Step(4, 8, 2, 5000, 900, d, [899, 3, 450, 0]).check()


@pytest.mark.parametrize("d", [32, 64, 128])
def test_long_prefix_of_a_large_batch(d):
    """Rows and keys enough for 128 rows of the batch to share a tile of keys."""
    Step(21, 32, 4, 8500, 40, d, [7 * i % 40 for i in range(21)]).check(p_bits=2.0 ** -8)


@pytest.mark.parametrize("n_p", [5, 70])
def test_short_prefix_of_many_heads(n_p):
    """256 tiles of the batch's rows: 128 rows a tile, the prefix whole."""
    Step(33, 256, 256, n_p, 3, 32, [i % 3 for i in range(33)]).check(p_bits=2.0 ** -8)


def test_without_append_lengths_and_defaults():
    Step(3, 4, 2, 90, 50, 64, [50, 0, 20], append=False).check()
    Step(3, 4, 2, 90, 50, 64, None).check(n=49)
    Step(3, 4, 2, 90, 50, 64, None, append=False).check(n=10)
    Step(3, 4, 2, 90, 50, 64, [-5, 100, 20]).check(n=30)
    Step(3, 4, 2, 90, 1, 64, None).check(n=0)
    Step(2, 4, 2, 90, 1, 64, None, append=False).check(n=0)
    for scale in (0.0, -0.3, 2.0):
        Step(3, 4, 2, 90, 50, 64, [49, 0, 20]).check(scale=scale)


def test_rows_behind_are_not_read():
    s = Step(3, 4, 2, 70, 200, 64, [0, 100, 33])
    for b, n in enumerate(s.lens):
        s.k_cache[b, :, n:], s.v_cache[b, :, n:] = NAN, NAN
    s.check()


def test_the_same_as_one_long_cache():
    """A generation, token by token, behind a prefix: as attn_decode on caches that hold the prefix themselves.
    Both round O once and P: within 2^-7 of the values' size, twice over."""
    B, Hq, Hkv, n_p, d, steps = 3, 8, 2, 150, 64, 40
    s = Step(B, Hq, Hkv, n_p, steps, d, None)
    kc = torch.cat((s.k_prefix.expand(B, -1, -1, -1), torch.zeros_like(s.k_cache)), 2).contiguous()
    vc = torch.cat((s.v_prefix.expand(B, -1, -1, -1), torch.zeros_like(s.v_cache)), 2).contiguous()
    rng = torch.Generator(device="cuda").manual_seed(1)
    for i in range(steps):
        q, k, v = (torch.randn(B, H, d, generator=rng, device="cuda").to(BF16) for H in (Hq, Hkv, Hkv))
        lens = ints([i] * B)
        O, L = lib.attn_prefix_decode(q, s.k_prefix, s.v_prefix, s.k_cache, s.v_cache, k, v, lens)
        O2, L2 = lib.attn_decode(q, kc, vc, k, v, lens + n_p, n=n_p + i)
        assert (O.float() - O2.float()).abs().max() <= 2 * 2 ** -7 * vc.abs().max()
        assert (L - L2).abs().max() <= 1e-4
    assert torch.equal(kc[:, :, n_p:], s.k_cache) and torch.equal(vc[:, :, n_p:], s.v_cache)


def test_capture_and_stream():
    s = Step(4, 8, 2, 500, 60, 128, None)
    lens = ints([0, 5, 30, 58])
    ws = torch.empty(lib.attn_prefix_decode_workspace_bytes(4, 8, 2, 500, 59, 128), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(s.q), torch.empty(4, 8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.attn_prefix_decode(s.q, s.k_prefix, s.v_prefix, s.k_cache, s.v_cache, s.k_new, s.v_new, lens, out=out, workspace=ws)
    side = torch.cuda.Stream()
    for seed in (1, 2, 3):
        other = Step(4, 8, 2, 500, 60, 128, None, seed=seed)
        for x in ("q", "k_prefix", "v_prefix", "k_cache", "v_cache", "k_new", "v_new"):
            getattr(s, x).copy_(getattr(other, x))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = lib.attn_prefix_decode(other.q, other.k_prefix, other.v_prefix, other.k_cache, other.v_cache, other.k_new, other.v_new, lens)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0], out[0]) and torch.equal(want[1], out[1])
        assert torch.equal(s.k_cache, other.k_cache) and torch.equal(s.v_cache, other.v_cache)
        lens.copy_((lens + 7) % 59)
