"""Attention to keys of another length and the decode step behind a shared prefix without a GPU: the oracle's
pins, the buckets of relative positions, every refusal of the C ABI and of the Python form."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_33916_amd as pkg
from oracle import cross, decode, naive
from test_binding_host import FakeLib, gpu

FAKE, MIS = 1 << 20, (1 << 20) + 2   # never dereferenced: validation fails first
BF16, F32 = 0, 1
CSRC = os.path.join(os.path.dirname(pkg.__file__), "csrc")


# ------------------------------------------------------------------ oracle --
def _inputs(B=2, Hq=4, Hkv=2, nq=5, nk=9, d=6, buckets=7, seed=0):
    rng = np.random.default_rng(seed)
    q, do = rng.standard_normal((2, B, Hq, nq, d))
    k, v = rng.standard_normal((2, B, Hkv, nk, d))
    return q, k, v, do, rng.standard_normal((buckets, Hq)), rng.integers(-1, buckets + 1, 11), -6


def test_oracle_is_attention():
    """Without a bias, of equal lengths and head counts: the fused path's oracle."""
    rng = np.random.default_rng(1)
    q, k, v, do = rng.standard_normal((4, 2, 3, 8, 4))
    for causal in (False, True):
        want = naive.attention(q, k, v, do, 0.3, causal)
        got = cross.attention(q, k, v, 0.3, do=do, causal=causal)
        for name in ("O", "L", "dQ", "dK", "dV"):
            assert np.allclose(got[name], want[name], atol=1e-12), name


@pytest.mark.parametrize("how", [{}, {"causal": True, "start": 3}, {"k_lens": [9, 4], "starts": [2, -3]}, {"causal": True, "start": -2}], ids=str)
def test_oracle_gradients_are_differences(how):
    q, k, v, do, bias, rows, first = _inputs()
    x = {"q": q, "k": k, "v": v, "bias": bias}

    def loss(x):
        return (cross.attention(x["q"], x["k"], x["v"], 0.4, bias=x["bias"], rows=rows, first=first, **how)["O"] * do).sum()
    got = cross.attention(q, k, v, 0.4, do=do, bias=bias, rows=rows, first=first, **how)
    rng = np.random.default_rng(2)
    for name, grad in (("q", "dQ"), ("k", "dK"), ("v", "dV"), ("bias", "dBias")):
        for _ in range(20):
            at = tuple(rng.integers(0, s) for s in x[name].shape)
            up, down = dict(x), dict(x)
            up[name], down[name] = x[name].copy(), x[name].copy()
            up[name][at] += 1e-5
            down[name][at] -= 1e-5
            assert abs((loss(up) - loss(down)) / 2e-5 - got[grad][at]) < 1e-8, (name, at)


def test_oracle_rows_without_keys():
    q, k, v, do, bias, rows, first = _inputs()
    got = cross.attention(q, k, v, 0.4, do=do, bias=bias, rows=rows, first=first, k_lens=[0, 3], causal=True, start=-2)
    assert (got["O"][0] == 0).all() and (got["L"][0] == -np.inf).all() and (got["O"][1, :, :2] == 0).all()
    assert all(np.isfinite(got[x]).all() for x in ("O", "dQ", "dK", "dV", "dBias"))
    assert (got["dK"][0] == 0).all() and (got["dV"][1, :, 3:] == 0).all() and (got["dQ"][1, :, :2] == 0).all()


def test_oracle_prefix_is_a_longer_cache():
    rng = np.random.default_rng(3)
    q, kp, vp = rng.standard_normal((3, 4, 6)), rng.standard_normal((2, 5, 6)), rng.standard_normal((2, 5, 6))
    kc, vc, kn, vn = rng.standard_normal((3, 2, 8, 6)), rng.standard_normal((3, 2, 8, 6)), rng.standard_normal((3, 2, 6)), rng.standard_normal((3, 2, 6))
    lens = np.array([0, 7, 3])
    O, L, k2, v2 = cross.prefix_decode(q, kp, vp, kc, vc, lens, 0.4, kn, vn)
    long_k, long_v = (np.concatenate((np.broadcast_to(p, (3, *p.shape)), c), 2) for p, c in ((kp, kc), (vp, vc)))
    K, V = decode.append_kv(long_k, long_v, kn, vn, lens + 5)
    for b in range(3):
        assert np.array_equal(k2[b, :, lens[b]], kn[b]) and np.array_equal(v2[b, :, lens[b]], vn[b])
        for h in range(4):
            o, l = decode.decode_head(q[b, h], K[b, h // 2], V[b, h // 2], int(lens[b]) + 6, 0.4)
            assert np.allclose(O[b, h], o) and np.isclose(L[b, h], l)


# ----------------------------------------------------------------- buckets --
@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("n,far", [(32, 128), (16, 64), (64, 200), (32, 1000), (4, 3), (8, 5), (320, 800)])
def test_buckets(n, far, both):
    """Against the logarithms in 64 bits; positions whose logarithm is within 1e-9 of a border by whole numbers."""
    side = n // 2 if both else n
    near = side // 2
    if far <= near:
        pytest.skip("no distance beyond the nearest")
    rows, first = pkg.attn_bias_buckets(n, far, both, device="cpu")
    rows = rows.tolist()
    for r in range(-2 * far, 2 * far + 1):
        p = abs(r) if both else max(-r, 0)
        if p < near:
            want = p
        else:
            t = np.log(p / near) / np.log(far / near) * (side - near)
            want = near + min(int(np.floor(t + 1e-9)), side - near - 1)
            k = round(t)
            if abs(t - k) < 1e-9 and 0 < k < side - near:
                assert (p ** (side - near) >= near ** (side - near - k) * far ** k) == (want >= near + k)
        want += side if both and r > 0 else 0
        assert rows[min(max(r - first, 0), len(rows) - 1)] == want, r


def test_buckets_refused():
    for args in ((31, 128), (2, 128), (32, 8), (32, 0), (32.0, 128), (32, 5000), (1, 10, False), (32, 16, False),
                 (10 ** 9, 10 ** 10), (4, 10 ** 400), (6, 2 ** 62)):
        with pytest.raises(ValueError):
            pkg.attn_bias_buckets(*args, device="cpu")


# ------------------------------------------------------------------- C ABI --
@pytest.fixture(scope="module")
def L():
    return pkg.lib()


def ll(*v):
    return (ctypes.c_longlong * len(v))(*v)


def fwd(L, strides=None, ptr=None, ws=FAKE, wsb=1 << 40, lens=None, starts=None, start=0, bias=None, rows=None, first=0, R=0, buckets=0,
        B=1, Hq=4, Hkv=2, nq=8, nk=9, d=64, scale=0.1, causal=0, dtype=BF16):
    p = {x: FAKE for x in ("q", "k", "v", "o", "L")}
    p.update(ptr or {})
    return L.attn_cross_fwd(*p.values(), strides, lens, starts, start, bias, rows, first, R, buckets, ws, wsb, B, Hq, Hkv, nq, nk, d, scale,
                            causal, dtype, None)


def bwd(L, strides=None, ptr=None, ws=FAKE, wsb=1 << 40, lens=None, starts=None, start=0, bias=None, rows=None, first=0, R=0, buckets=0,
        B=1, Hq=4, Hkv=2, nq=8, nk=9, d=64, scale=0.1, causal=0, dtype=BF16):
    p = {x: FAKE * (i + 1) for i, x in enumerate(("q", "k", "v", "o", "L", "do", "dq", "dk", "dv"))}
    p["dbias"] = None
    p.update(ptr or {})
    return L.attn_cross_bwd(*p.values(), strides, lens, starts, start, bias, rows, first, R, buckets, ws, wsb, B, Hq, Hkv, nq, nk, d, scale,
                            causal, dtype, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_refusals_of_both(L, call):
    for x in ("q", "k", "v", "o", "L"):
        assert call(L, ptr={x: None}) == -1
        assert call(L, ptr={x: MIS}) == -4
    for bad in ({"B": 0}, {"Hq": 0}, {"Hkv": 0}, {"nq": 0}, {"nk": 0}, {"nk": -1}, {"Hq": 3}, {"nq": (1 << 29) + 1}, {"nk": (1 << 29) + 1},
                {"B": 1 << 20, "nq": 1 << 10}, {"B": 1 << 30}, {"nk": 1 << 28}, {"start": (1 << 30) + 1}, {"start": -(1 << 30) - 1}):
        assert call(L, **bad) == -2, bad
    for bad in ({"d": 80}, {"d": 256}, {"d": 0}, {"dtype": 2}):
        assert call(L, **bad) == -3, bad
    for bad in ({"scale": float("nan")}, {"scale": float("inf")}, {"causal": 2}, {"causal": -1}):
        assert call(L, **bad) == -7, bad
    assert call(L, lens=MIS + 1) == -4 and call(L, starts=MIS) == -4
    some = {"bias": FAKE, "rows": FAKE, "R": 3, "buckets": 4}
    assert call(L, **{**some, "rows": None}) == -1
    for bad in ({"R": 1}, {"R": 0}, {"R": 2049}, {"R": -5}, {"buckets": 0}, {"buckets": -1}, {"first": (1 << 20) + 1}, {"first": -(1 << 31)}):
        assert call(L, **{**some, **bad}) == -2, bad
    assert call(L, **{**some, "bias": FAKE + 1}) == -4 and call(L, **{**some, "rows": MIS}) == -4
    assert call(L, **{**some, "bias": FAKE + 2}, dtype=F32) == -4


def test_refusals_of_strides(L):
    q, kv = [4 * 8 * 64, 8 * 64, 64], [2 * 9 * 64, 9 * 64, 64]
    good = q + kv + kv + q

    def one(i, v):
        s = list(good)
        s[i] = v
        return ll(*s)
    for t in range(4):
        assert fwd(L, strides=one(3 * t + 1, -64), nq=8) == -2
        assert fwd(L, strides=one(3 * t + 2, 68)) == -4          # 136 bytes
        assert fwd(L, strides=one(3 * t + 1, 65)) == -4
        assert fwd(L, strides=one(3 * t + 2, (1 << 22) + 8)) == -2
        assert fwd(L, strides=one(3 * t, 1 << 61), B=2) == -2
    assert fwd(L, strides=one(11, 0)) == -7 and fwd(L, strides=one(10, 32)) == -7   # rows of O overlap
    good += q + q + kv + kv
    for t, step in ((5, q), (6, kv), (7, kv)):
        assert bwd(L, strides=one(3 * t + 2, 0)) == -7
        assert bwd(L, strides=one(3 * t + 1, step[2])) == -7
    assert bwd(L, ptr={"dv": 8 * FAKE}) == -7   # dK's place
    assert bwd(L, ptr={"dv": 8 * FAKE + 2 * 64}) == -7
    for x in ("dk", "dv"):   # in dQ's place, behind its start, before its end
        assert bwd(L, ptr={x: 7 * FAKE}) == -7 and bwd(L, ptr={x: 7 * FAKE + 128}) == -7 and bwd(L, ptr={x: 7 * FAKE - 128}) == -7
        assert bwd(L, ptr={x: 7 * FAKE + 4 * 8 * 64 * 2}, wsb=0) == -5   # right behind it: only the workspace is wrong


def test_refusals_of_results_in_place(L):
    """An output on an input, or reaching into it."""
    apart = {x: FAKE * (i + 1) for i, x in enumerate(("q", "k", "v", "o", "L"))}
    for x in ("q", "k", "v"):
        for at in (0, 128, -128):
            assert fwd(L, ptr={**apart, "o": apart[x] + at}) == -7
    packed = ll(4 * 8 * 64, 64, 4 * 64, *([2 * 9 * 64, 9 * 64, 64] * 2), 8 * 8 * 64, 64, 8 * 64)   # with gaps, on q's first row
    assert fwd(L, strides=packed, ptr={**apart, "o": apart["q"]}) == -7
    for x in ("q", "k", "v", "o", "do"):
        i = ("q", "k", "v", "o", "L", "do").index(x)
        for y in ("dq", "dk", "dv"):
            for at in (0, 128, -128):
                assert bwd(L, ptr={y: FAKE * (i + 1) + at}) == -7, (x, y, at)
    # dQ [2, 2, 4, 64] between two sequences' dK: only the workspace is wrong
    q, kv = [2 * 4 * 64, 4 * 64, 64], [2 * 9 * 64, 9 * 64, 64]
    slots = ll(*q, *kv, *kv, *q, *q, *q, 2 * kv[0], *kv[1:], *kv)
    small = dict(B=2, Hq=2, nq=4, strides=slots, wsb=0)
    assert bwd(L, ptr={"dq": 8 * FAKE + 2 * kv[0]}, **small) == -5
    assert bwd(L, ptr={"dq": 8 * FAKE + 2 * kv[0] - 128}, **small) == -7
    assert bwd(L, ptr={"dq": 8 * FAKE + 4 * kv[0] - 2 * q[0] * 2}, **small) == -5   # right before the second
    assert bwd(L, ptr={"dq": 8 * FAKE + 4 * kv[0] - 2 * q[0] * 2 + 128}, **small) == -7


RANGES = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "strides.hpp"
using attn::Strides;
int main() {
  std::mt19937 g(11);
  auto pick = [&](int lo, int hi) { return lo + (int)(g() % (unsigned)(hi - lo + 1)); };
  int met = 0, apart = 0;
  const int d = 4;
  struct Tensor { Strides s; int H, n; bool dense; };
  auto draw = [&](int B, int gaps) {   // axes in a random order, each over the smaller ones and a gap, or not stepping at all
    Tensor x{{0, 0, 0}, pick(1, 3), pick(1, 4), true};
    int order[3] = {0, 1, 2}, size[3] = {B, x.H, x.n};
    for (int i = 2; i > 0; --i) std::swap(order[i], order[pick(0, i)]);
    long long step[3], span = d;
    for (int i : order) {
      const long long gap = gaps ? 4 * pick(0, 6) : 0;
      step[i] = gaps == 2 && pick(0, 3) == 0 ? 0 : span + gap;
      if (size[i] == 1) step[i] = 0;
      else if (step[i] != span) x.dense = false;
      if (step[i]) span = step[i] * size[i];
    }
    x.s = {step[0], step[1], step[2]};
    return x;
  };
  for (int it = 0; it < 300000; ++it) {
    const int B = pick(1, 3);
    const Tensor a = draw(B, 0), b = draw(B, it % 3);
    const bool swap = it % 2;
    const Tensor &x = swap ? b : a, &y = swap ? a : b;
    const long long delta = pick(-160, 160);
    bool want = false;
    for (int i = 0; i < B; ++i) for (int j = 0; j < x.H; ++j) for (int k = 0; k < x.n; ++k)
      for (int l = 0; l < B; ++l) for (int m = 0; m < y.H; ++m) for (int o = 0; o < y.n; ++o)
        want = want || std::llabs(delta + l * y.s.b + m * y.s.h + o * y.s.t - i * x.s.b - j * x.s.h - k * x.s.t) < d;
    if (attn::ranges_meet(x.s, x.H, x.n, y.s, y.H, y.n, B, d, delta) != want) {
      std::printf("%d: %lld %lld %lld, %lld %lld %lld, delta %lld: %d\n", it, x.s.b, x.s.h, x.s.t, y.s.b, y.s.h, y.s.t, delta, want);
      return 1;
    }
    ++(want ? met : apart);
  }
  const Strides far{1LL << 50, 128, 1LL << 20}, dense{64LL << 27, 1LL << 27, 128};   // sizes whose products pass 64 bits
  if (attn::ranges_meet(far, 64, 1 << 20, dense, 64, 1 << 20, 1 << 9, 128, -(1LL << 58))) return 1;
  if (!attn::ranges_meet(dense, 64, 1 << 20, far, 64, 1 << 20, 1 << 9, 128, 1LL << 30)) return 1;
  return met > 1000 && apart > 1000 ? 0 : 1;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_overlaps_against_all_pairs(tmp_path):
    """Of two tensors, one of them without gaps, every overlap is found and no other (csrc/strides.hpp, compiled for the CPU)."""
    (tmp_path / "ranges.cpp").write_text(RANGES)
    exe = str(tmp_path / "ranges")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-I", CSRC, str(tmp_path / "ranges.cpp"), "-o", exe], check=True)
    subprocess.run([exe], check=True, timeout=120)


def test_workspaces(L):
    assert L.attn_cross_fwd_workspace_bytes(1, 4, 2, 8, 9, 64, BF16, 0) == 0
    need = L.attn_cross_fwd_workspace_bytes(1, 4, 2, 1, 100000, 64, BF16, 0)
    assert need > 0 and need % (4 * (64 + 2) * 4) == 0
    big = dict(nq=1, nk=100000)
    assert fwd(L, ws=None, **big) == -1
    assert fwd(L, wsb=need - 1, **big) == -5
    assert fwd(L, ws=FAKE + 8, **big) == -4
    for args in ((0, 4, 2, 8, 9, 64, BF16, 0), (1, 4, 2, 8, 9, 65, BF16, 0), (1, 4, 3, 8, 9, 64, BF16, 0), (1, 4, 2, 8, 9, 64, BF16, -1)):
        assert L.attn_cross_fwd_workspace_bytes(*args) == 0 and L.attn_cross_bwd_workspace_bytes(*args) == 0
    need = L.attn_cross_bwd_workspace_bytes(1, 4, 2, 8, 9, 64, BF16, 0)
    assert need >= 2 * 4 * 8 * 4
    assert bwd(L, wsb=need - 1) == -5 and bwd(L, ws=None) == -1 and bwd(L, ws=FAKE + 4) == -4
    some = {"bias": FAKE, "rows": FAKE, "R": 300, "buckets": 4}
    with_bias = L.attn_cross_bwd_workspace_bytes(1, 4, 2, 8, 9, 64, BF16, 300)
    assert with_bias >= need + 4 * 300 * 4
    assert bwd(L, wsb=with_bias - 1, ptr={"dbias": FAKE}, **some) == -5
    assert bwd(L, ptr={"dbias": FAKE}) == -1   # no bias


def prefix(L, ptr=None, ws=FAKE, wsb=1 << 40, lens=None, B=2, Hq=4, Hkv=2, n_p=7, n=3, n_cap=4, d=64, scale=0.1, dtype=BF16):
    p = {x: FAKE for x in ("q", "k_new", "v_new", "k_prefix", "v_prefix", "k_cache", "v_cache")}
    q = {"O": FAKE, "L": FAKE}
    for x, v in (ptr or {}).items():
        (p if x in p else q)[x] = v
    return L.attn_prefix_decode(*p.values(), lens, *q.values(), ws, wsb, B, Hq, Hkv, n_p, n, n_cap, d, scale, dtype, None)


def test_refusals_of_prefix(L):
    for x in ("q", "k_new", "v_new", "k_prefix", "v_prefix", "k_cache", "v_cache", "O"):
        assert prefix(L, ptr={x: None}) == -1, x
        assert prefix(L, ptr={x: FAKE + 8}) == -4, x
    assert prefix(L, ws=None) == -1 and prefix(L, ws=FAKE + 8) == -4 and prefix(L, ptr={"L": MIS}) == -4 and prefix(L, lens=MIS) == -4
    for bad in ({"B": 0}, {"Hq": 0}, {"Hkv": 0}, {"Hq": 3}, {"n_p": 0}, {"n": -1}, {"n": 4}, {"n_cap": 3}, {"n_cap": 0, "n": 0},
                {"n_p": 1 << 28}, {"B": 1 << 26}, {"n": 1 << 26, "n_cap": 1 << 27}):
        assert prefix(L, **bad) == -2, bad
    for bad in ({"d": 96}, {"dtype": F32}, {"dtype": 5}):
        assert prefix(L, **bad) == -3, bad
    assert prefix(L, scale=float("inf")) == -7
    # written tensors that reach into another one
    names = ("q", "k_new", "v_new", "k_prefix", "v_prefix", "k_cache", "v_cache", "O")
    apart = {x: FAKE * (i + 1) for i, x in enumerate(names)}
    size = {"O": 2 * 4 * 64 * 2, "k_cache": 2 * 2 * 4 * 64 * 2, "v_cache": 2 * 2 * 4 * 64 * 2}
    for x in size:
        for y in names[1:]:
            if x != y:
                assert prefix(L, ptr={**apart, x: apart[y]}) == -7, (x, y)
                assert prefix(L, ptr={**apart, y: apart[x] + size[x] - 16}) == -7, (x, y)
    assert prefix(L, ptr={**apart, "k_new": None, "v_new": None, "O": apart["k_cache"]}) == -7
    need = L.attn_prefix_decode_workspace_bytes(2, 4, 2, 7, 3, 64)
    assert need == 2 * 2 * 4 * (64 + 2) * 4 and prefix(L, wsb=need - 1) == -5
    assert L.attn_prefix_decode_workspace_bytes(2, 4, 2, 7, 0, 64) == 2 * 4 * (64 + 2) * 4
    assert L.attn_prefix_decode_workspace_bytes(2, 4, 3, 7, 0, 64) == 0


# ------------------------------------------------------------- Python form --
class Lib(FakeLib):
    def attn_cross_fwd_workspace_bytes(self, *a):
        return 64

    def attn_cross_bwd_workspace_bytes(self, *a):
        return 64

    def attn_prefix_decode_workspace_bytes(self, *a):
        return 64


@pytest.fixture
def fake(monkeypatch):
    f = Lib()
    monkeypatch.setattr(pkg, "_lib", f)
    return f


def ints(*shape):
    return gpu(*shape, dtype=torch.int32)


def cross_case():
    return {"q": gpu(2, 4, 5, 64), "k": gpu(2, 2, 7, 64), "v": gpu(2, 2, 7, 64)}


BAD = {
    "q": (None, torch.zeros(2, 4, 5, 64), gpu(4, 5, 64), gpu(2, 4, 5, 128)[..., ::2], gpu(2, 4, 5, 32), gpu(0, 4, 5, 64)),
    "k": (None, gpu(2, 2, 7, 32), gpu(1, 2, 7, 64), gpu(2, 2, 7, 64, dtype=torch.float32), gpu(2, 2, 64)),
    "v": (None, gpu(2, 2, 8, 64), gpu(2, 4, 7, 64), torch.zeros(2, 2, 7, 64, dtype=torch.bfloat16)),
    "k_lens": (ints(3), gpu(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), ints(4)[::2]),
    "starts": (ints(1), gpu(2), ints(2, 1)),
    "bias_rows": (ints(9),),   # without a bias
}


@pytest.mark.parametrize("name,i", [(n, i) for n, v in BAD.items() for i in range(len(v))])
def test_bad_tensors(fake, name, i):
    x = {**cross_case(), name: BAD[name][i]}
    with pytest.raises(ValueError):
        pkg.attn_cross_fwd(**x)
    with pytest.raises(ValueError):
        pkg.attn_cross_bwd(o=gpu(2, 4, 5, 64), lse=gpu(2, 4, 5, dtype=torch.float32), do=gpu(2, 4, 5, 64), **x)
    assert not fake.launches


def test_bad_bias_outputs_workspace(fake):
    f32 = torch.float32
    good = dict(cross_case(), bias=gpu(8, 4), bias_rows=ints(9), out=(gpu(2, 4, 5, 64), gpu(2, 4, 5, dtype=f32)))
    for bad in ({"bias": gpu(8, 2)}, {"bias": gpu(8, 4, dtype=f32)}, {"bias": torch.zeros(8, 4)}, {"bias": gpu(4, 8).t()}, {"bias": gpu(8)},
                {"bias_rows": None}, {"bias_rows": ints(3, 3)}, {"bias_rows": gpu(9)}, {"bias_rows": ints(18)[::2]}, {"bias_first": 2 ** 31},
                {"start": 2 ** 31}, {"workspace": gpu(10, dtype=torch.uint8)}, {"workspace": torch.zeros(100)},
                {"out": (gpu(2, 4, 5, 64),)}, {"out": (gpu(2, 4, 5, 64), gpu(2, 4, 5))}, {"out": (gpu(2, 4, 7, 64), gpu(2, 4, 5, dtype=f32))},
                {"out": (torch.zeros(2, 4, 5, 64), gpu(2, 4, 5, dtype=f32))}):
        with pytest.raises(ValueError):
            pkg.attn_cross_fwd(**{**good, **bad})
    saved = dict(o=gpu(2, 4, 5, 64), lse=gpu(2, 4, 5, dtype=f32), do=gpu(2, 4, 5, 64))
    dq, dkv = gpu(2, 4, 5, 64), gpu(2, 2, 7, 64)
    good["out"] = (dq, dkv, dkv, None)
    for bad in ({"o": gpu(2, 4, 5, 32)}, {"lse": gpu(2, 4, 5)}, {"lse": gpu(2, 4, 6, dtype=f32)}, {"do": gpu(2, 4, 5, 64, dtype=f32)}, {"do": None},
                {"out": (dq, dkv, dkv)}, {"out": (dq, dkv, dkv, gpu(8, 4, dtype=f32))}, {"out": (dkv, dkv, dkv, None)},
                {"workspace": gpu(63, dtype=torch.uint8)}):
        with pytest.raises(ValueError):
            pkg.attn_cross_bwd(**{**good, **saved, **bad})
    assert not fake.launches


def test_bad_prefix_tensors(fake):
    good = dict(q=gpu(3, 4, 64), k_prefix=gpu(2, 9, 64), v_prefix=gpu(2, 9, 64), k_cache=gpu(3, 2, 5, 64), v_cache=gpu(3, 2, 5, 64),
                k_new=gpu(3, 2, 64), v_new=gpu(3, 2, 64), cache_lens=ints(3), out=(gpu(3, 4, 64), None))
    f32 = torch.float32
    for bad in ({"q": None}, {"q": gpu(3, 4, 64, dtype=f32)}, {"q": torch.zeros(3, 4, 64)}, {"q": gpu(4, 64)}, {"q": gpu(3, 8, 64)[:, ::2]},
                {"k_prefix": gpu(2, 9, 32)}, {"k_prefix": gpu(1, 2, 9, 64)}, {"v_prefix": gpu(2, 8, 64)}, {"v_prefix": gpu(9, 2, 64).transpose(0, 1)},
                {"k_cache": gpu(3, 1, 5, 64)}, {"v_cache": gpu(3, 2, 6, 64)}, {"k_cache": gpu(2, 2, 5, 64)}, {"k_new": None}, {"v_new": None},
                {"v_new": gpu(3, 4, 64)}, {"cache_lens": ints(2)}, {"cache_lens": gpu(3)}, {"cache_lens": None}, {"n": 2 ** 31},
                {"out": (gpu(3, 4, 64),)}, {"out": (gpu(3, 4, 64), gpu(3, 4))}, {"out": (gpu(3, 4, 32), None)},
                {"workspace": gpu(63, dtype=torch.uint8)}):
        with pytest.raises(ValueError):
            pkg.attn_prefix_decode(**{**good, **bad})
    assert not fake.launches
