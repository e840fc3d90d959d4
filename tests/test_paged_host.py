"""Rotary positions and the paged cache without a GPU: page addresses (csrc/pages.hpp,
compiled for the CPU), every refusal of the C ABI and of the Python form, the frequency
tables."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_33916_amd as pkg
from test_binding_host import FakeLib, gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33916_amd", "csrc")

MAIN = r"""
#include <climits>
#include <cstdio>
#include <vector>
#include "pages.hpp"
int main() {
  for (int shift : {4, 5, 7, 10}) for (int Hkv : {1, 3, 8}) for (int num : {1, 5, 1 << 20}) {
    const int ps = 1 << shift, width = 6;
    const std::vector<int> table = {num - 1, 0, -1, num, INT_MAX, num / 2};
    const attn::Pages a{nullptr, width, num, shift, Hkv};
    for (int p = -3; p < width * ps + 3; ++p) {
      const long long got = attn::page_row(a, table.data(), p);
      const int page = p < 0 || p >= width * ps ? -1 : table[p / ps];
      const long long want = page < 0 || page >= num ? -1 : (long long)page * Hkv * ps + p % ps;
      if (got != want) { std::printf("row %d: %lld, not %lld\n", p, got, want); return 1; }
      if (got >= 0 && got + (long long)(Hkv - 1) * ps >= (long long)num * Hkv * ps) { std::printf("outside\n"); return 1; }
    }
    for (int p : {INT_MAX, INT_MIN, width * ps})
      if (attn::page_row(a, table.data(), p) != -1) { std::printf("far\n"); return 1; }
  }
  std::printf("ok\n");
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_page_rows(tmp_path):
    src, exe = tmp_path / "pages.cpp", tmp_path / "pages"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok" and not out.stderr, out.stdout + out.stderr


# ----------------------------------------------------------------- C ABI --
FAKE, MIS = 1 << 20, (1 << 20) + 2   # never dereferenced: validation fails first
import ctypes  # noqa: E402


def _ll(*v):
    return (ctypes.c_longlong * len(v))(*v)


@pytest.fixture(scope="module")
def L():
    return pkg.lib()


def _rope(L, fn="attn_rope", q=FAKE, k=FAKE, qo=FAKE, ko=FAKE, strides=None, freqs=FAKE, pos=None, ps=0, start=0, B=2, Hq=4,
          Hk=2, n=8, d=64, r=64, amp=1.0, inter=0, dtype=0):
    return getattr(L, fn)(q, k, qo, ko, strides, freqs, pos, ps, start, B, Hq, Hk, n, d, r, amp, inter, dtype, None)


@pytest.mark.parametrize("fn", ["attn_rope", "attn_rope_bwd"])
def test_rope_refusals(L, fn):
    def call(**kw):
        return _rope(L, fn, **kw)
    for name in ("q", "qo", "freqs", "k", "ko"):
        assert call(**{name: None}) == -1, name
    for bad in (dict(B=0), dict(Hq=0), dict(Hk=0), dict(n=0), dict(n=-1), dict(B=1 << 16, n=1 << 15), dict(Hq=65535),
                dict(start=2**31 - 8), dict(pos=FAKE, ps=-1), dict(strides=_ll(*[-8] * 12)),
                dict(strides=_ll(*[1 << 60] * 12))):
        assert call(**bad) == -2, bad
    for bad in (dict(d=48), dict(d=256, r=64), dict(dtype=2), dict(r=8), dict(r=72), dict(r=24), dict(r=128), dict(r=0)):
        assert call(**bad) == -3, bad
    dense = [4 * 8 * 64, 8 * 64, 64, 2 * 8 * 64, 8 * 64, 64] * 2
    for bad in [dict(q=MIS), dict(ko=MIS), dict(pos=FAKE + 1), dict(freqs=FAKE + 4)] + \
            [dict(strides=_ll(*(s + (1 if i == j else 0) for j, s in enumerate(dense)))) for i in range(12)]:
        assert call(**bad) == -4, bad
    for bad in (dict(amp=math.nan), dict(amp=math.inf), dict(inter=2), dict(inter=-1)):
        assert call(**bad) == -7, bad
    # outputs whose rows overlap: token on token, head on head, heads inside a token's row
    for i, s in ((6, 0), (7, 0), (8, 0), (8, 32), (7, 64), (10, 0), (11, 56)):
        assert call(strides=_ll(*(s if i == j else x for j, x in enumerate(dense)))) == -7, (i, s)


def _append(L, kn=FAKE, vn=FAKE, strides=None, kp=FAKE, vp=FAKE, ks=None, vs=None, table=FAKE, lens=FAKE, news=None, freqs=None,
            pos=None, B=2, Hkv=2, T=3, P=9, ps=16, W=4, d=64, r=0, amp=1.0, inter=0, dtype=0):
    return L.attn_paged_append(kn, vn, strides, kp, vp, ks, vs, table, lens, news, freqs, pos, B, Hkv, T, P, ps, W, d, r, amp,
                               inter, dtype, None)


def _gather(L, kp=FAKE, vp=FAKE, ks=None, vs=None, table=FAKE, lens=FAKE, starts=None, K=FAKE, V=FAKE, B=2, Hkv=2, n=3, P=9,
            ps=16, W=4, d=64, dtype=0):
    return L.attn_paged_gather(kp, vp, ks, vs, table, lens, starts, K, V, B, Hkv, n, P, ps, W, d, dtype, None)


def _decode(L, q=FAKE, kn=FAKE, vn=FAKE, strides=None, kp=FAKE, vp=FAKE, ks=None, vs=None, table=FAKE, lens=FAKE, freqs=None,
            pos=None, O=FAKE, lse=FAKE, ws=FAKE, wsb=1 << 40, B=2, Hq=4, Hkv=2, n=63, P=9, ps=16, W=4, d=64, r=0, amp=1.0,
            inter=0, scale=0.1, dtype=0):
    return L.attn_paged_decode(q, kn, vn, strides, kp, vp, ks, vs, table, lens, freqs, pos, O, lse, ws, wsb, B, Hq, Hkv, n, P,
                               ps, W, d, r, amp, inter, scale, dtype, None)


@pytest.mark.parametrize("call", [_append, _gather, _decode])
def test_pool_refusals(L, call):
    for name in ("kp", "vp", "table", "lens"):
        assert call(L, **{name: None}) == -1, name
    assert call(L, ks=FAKE) == -1 and call(L, vs=FAKE) == -1
    for bad in (dict(B=0), dict(Hkv=0), dict(P=0), dict(W=0), dict(B=65536), dict(P=2**31 - 1, ps=1 << 20)):
        assert call(L, **bad) == -2, bad
    for bad in (dict(d=80), dict(dtype=1), dict(dtype=5), dict(ps=8), dict(ps=24), dict(ps=0), dict(ps=1 << 21)):
        assert call(L, **bad) == -3, bad
    for bad in (dict(kp=MIS), dict(vp=FAKE + 8), dict(ks=FAKE + 8, vs=FAKE), dict(ks=FAKE, vs=FAKE + 1), dict(table=MIS),
                dict(lens=FAKE + 1)):
        assert call(L, **bad) == -4, bad


def test_append_refusals(L):
    assert _append(L, kn=None) == -1 and _append(L, vn=None) == -1
    for bad in (dict(T=0), dict(B=65535, T=1 << 16), dict(strides=_ll(-8, 8, 8, 8, 8, 8))):
        assert _append(L, **bad) == -2, bad
    assert _append(L, freqs=FAKE, r=8) == -3 and _append(L, freqs=FAKE, r=80) == -3
    for bad in (dict(kn=MIS), dict(vn=FAKE + 8), dict(news=MIS), dict(pos=MIS), dict(freqs=FAKE + 4, r=64),
                dict(strides=_ll(8, 8, 8, 8, 8, 12))):
        assert _append(L, **bad) == -4, bad
    assert _append(L, inter=3) == -7 and _append(L, freqs=FAKE, r=64, amp=math.inf) == -7


def test_gather_refusals(L):
    assert _gather(L, K=None) == -1 and _gather(L, V=None) == -1
    assert _gather(L, n=0) == -2 and _gather(L, B=65535, Hkv=65535, n=1 << 20) == -2
    assert _gather(L, K=MIS) == -4 and _gather(L, starts=MIS) == -4


def test_decode_refusals(L):
    for bad in (dict(q=None), dict(O=None), dict(kn=None), dict(vn=None)):
        assert _decode(L, **bad) == -1, bad
    for bad in (dict(Hq=3), dict(Hq=0), dict(n=-1), dict(n=64), dict(kn=None, vn=None, n=65), dict(n=2**31 - 1),
                dict(B=65535, Hq=2), dict(strides=_ll(-8, 0, 0)), dict(strides=_ll(0, 0, 1 << 50))):
        assert _decode(L, **bad) == -2, bad
    assert _decode(L, freqs=FAKE, r=96) == -3
    for bad in (dict(q=MIS), dict(kn=MIS), dict(O=MIS), dict(lse=MIS), dict(pos=MIS), dict(strides=_ll(8, 8, 4))):
        assert _decode(L, **bad) == -4, bad
    for bad in (dict(scale=math.nan), dict(scale=-math.inf), dict(inter=2), dict(freqs=FAKE, r=64, amp=math.nan)):
        assert _decode(L, **bad) == -7, bad
    for bits in (16, 4):
        big = dict(B=1, n=16 * 4000 - 1, W=4000, **(dict(ks=FAKE, vs=FAKE) if bits == 4 else {}))
        need = L.attn_paged_decode_workspace_bytes(1, 4, 2, 16 * 4000 - 1, 64, 1, bits)
        assert need > 0 and need % (4 * 66 * 4) == 0
        assert _decode(L, ws=None, **big) == -1 and _decode(L, ws=FAKE + 8, **big) == -4
        assert _decode(L, wsb=need - 1, **big) == -5
    for bad in ((0, 4, 2, 5, 64, 1, 16), (1, 5, 2, 5, 64, 1, 16), (1, 4, 2, -1, 64, 1, 16), (1, 4, 2, 5, 60, 1, 16),
                (1, 4, 2, 5, 64, 1, 8)):
        assert L.attn_paged_decode_workspace_bytes(*bad) == 0


# ---------------------------------------------------------------- Python --
class Fake(FakeLib):
    def attn_paged_decode_workspace_bytes(self, *a):
        return 4096


@pytest.mark.parametrize("elem,d", [(2, 128), (2, 64), (2, 32), (4, 128), (4, 32)])
def test_launches_past_32_bits(L, elem, d):
    """More threads than a launch can have (2^32 along an axis): refused, not launched."""
    n = min(2**32 * 8 * 4 // elem // d, 2**31 - 1)   # a thread per 32 bytes
    for fn in ("attn_rope", "attn_rope_bwd"):
        assert _rope(L, fn, B=1, n=n, start=-n, d=d, r=16, dtype=0 if elem == 2 else 1) == -2
    if elem == 2:
        for four in (False, True):
            sc = dict(ks=FAKE, vs=FAKE) if four else {}
            assert _append(L, B=1, T=min(2**32 * (8 if four else 16) // d, 2**31 - 1), d=d, **sc) == -2
            assert _gather(L, B=1, Hkv=1, n=min(2**32 * 8 // d, 2**31 - 1), d=d, **sc) == -2


@pytest.fixture
def fake(monkeypatch):
    f = Fake()
    monkeypatch.setattr(pkg, "_lib", f)
    return f


def _pool(four=False):
    P, H, ps, d = 6, 2, 16, 64
    p = dict(k_pages=gpu(P, H, ps, d), v_pages=gpu(P, H, ps, d))
    if four:
        p = {k: gpu(P, H, ps, d // 2, dtype=torch.uint8) for k in p}
        p.update(k_scales=gpu(P, H, ps, 2, dtype=torch.uint8), v_scales=gpu(P, H, ps, 2, dtype=torch.uint8))
    p.update(block_table=gpu(3, 4, dtype=torch.int32), lens=gpu(3, dtype=torch.int32))
    return p


F64 = torch.float64


@pytest.mark.parametrize("bad", [
    dict(q=torch.zeros(1, 2, 8, 64)), dict(q=gpu(2, 8, 64)), dict(q="q"), dict(k=gpu(1, 2, 9, 64)), dict(k=gpu(2, 2, 8, 64)),
    dict(k=gpu(1, 2, 8, 64, dtype=torch.float32)), dict(k=gpu(1, 2, 64, 8).transpose(2, 3)), dict(freqs=None),
    dict(freqs=gpu(32, dtype=torch.float32)), dict(freqs=gpu(64, dtype=F64)), dict(freqs=torch.zeros(32, dtype=F64)),
    dict(freqs=gpu(32, 1, dtype=F64)), dict(positions=gpu(8, dtype=torch.int64)), dict(positions=gpu(9, dtype=torch.int32)),
    dict(positions=gpu(2, 8, dtype=torch.int32)), dict(positions=torch.zeros(8, dtype=torch.int32)), dict(start=2**31),
    dict(out=(gpu(1, 2, 8, 64),)), dict(out=(gpu(1, 2, 8, 64), None)), dict(out=(gpu(1, 2, 8, 64), gpu(1, 2, 8, 32))),
    dict(out=(gpu(1, 2, 8, 64, dtype=torch.float32), gpu(1, 2, 8, 64)))])
def test_rope_form_refuses(fake, bad):
    for call in (pkg.attn_rope, pkg.attn_rope_bwd):
        args = dict(q=gpu(1, 2, 8, 64), k=gpu(1, 2, 8, 64), freqs=gpu(32, dtype=F64), **{})
        args.update(bad)
        with pytest.raises(ValueError):
            call(args.pop("q"), args.pop("k"), args.pop("freqs"), **args)
    assert fake.launches == []


@pytest.mark.parametrize("four", [False, True])
def test_paged_forms_refuse(fake, four):
    """A wrong pool, table or length in each call, then each call's own arguments."""
    wrong = [dict(k_pages=torch.zeros(6, 2, 16, 64)), dict(v_pages=gpu(6, 2, 16, 16)), dict(v_pages=gpu(5, 2, 16, 64)),
             dict(k_pages=gpu(6, 2, 16, 64, dtype=torch.float32)), dict(k_pages=gpu(2, 6, 16, 64).transpose(0, 1)),
             dict(block_table=gpu(3, 4, dtype=torch.int64)), dict(block_table=gpu(3, dtype=torch.int32)),
             dict(block_table=torch.zeros(3, 4, dtype=torch.int32)), dict(block_table=gpu(4, 3, dtype=torch.int32).t()),
             dict(lens=gpu(2, dtype=torch.int32)), dict(lens=None), dict(lens=gpu(3, dtype=torch.int64)),
             dict(lens=torch.zeros(3, dtype=torch.int32))]
    wrong += [dict(k_scales=None), dict(v_scales=None), dict(k_scales=gpu(6, 2, 16, 1, dtype=torch.uint8)),
              dict(v_scales=gpu(6, 2, 16, 2))] if four else [dict(k_scales=gpu(6, 2, 16, 2, dtype=torch.uint8))]
    kv = gpu(3, 2, 5, 64)
    calls = {"append": lambda **p: pkg.attn_paged_append(p.pop("k_new", kv), p.pop("v_new", kv), **p),
             "gather": lambda **p: pkg.attn_paged_gather(n=p.pop("n", 7), **p),
             "decode": lambda **p: pkg.attn_paged_decode(p.pop("q", gpu(3, 4, 64)), **{
                 "out": (gpu(3, 4, 64), gpu(3, 4, dtype=torch.float32)), **p})}
    own = {"append": [dict(k_new=gpu(3, 2, 5, 32)), dict(v_new=gpu(3, 2, 6, 64)), dict(k_new=torch.zeros(3, 2, 5, 64)),
                      dict(k_new=gpu(3, 2, 64)), dict(v_new=gpu(3, 2, 5, 64, dtype=torch.float32)),
                      dict(new_lens=gpu(4, dtype=torch.int32)), dict(positions=gpu(3, dtype=torch.int32)),
                      dict(freqs=gpu(40, dtype=F64))],
           "gather": [dict(n=0), dict(n=-3), dict(starts=gpu(2, dtype=torch.int32)), dict(out=(gpu(3, 2, 7, 64),)),
                      dict(out=(gpu(3, 2, 7, 64), gpu(3, 2, 8, 64))), dict(out=(gpu(3, 2, 7, 64), torch.zeros(3, 2, 7, 64)))],
           "decode": [dict(q=gpu(3, 4, 32)), dict(q=gpu(2, 4, 64)), dict(q=gpu(3, 4, 1, 64)), dict(q=gpu(4, 3, 64).transpose(0, 1)),
                      dict(k_new=gpu(3, 2, 64)), dict(k_new=gpu(3, 2, 64), v_new=gpu(3, 1, 64)),
                      dict(k_new=gpu(3, 2, 64), v_new=torch.zeros(3, 2, 64)), dict(positions=gpu(3, 1, dtype=torch.int32)),
                      dict(n=2**31), dict(out=(gpu(3, 4, 64),)), dict(out=(gpu(3, 4, 64), gpu(3, 4))),
                      dict(out=(gpu(3, 5, 64), None)), dict(workspace=gpu(100, dtype=torch.uint8)),
                      dict(workspace=torch.zeros(4096, dtype=torch.uint8))]}
    for name, call in calls.items():
        for bad in wrong + own[name]:
            with pytest.raises(ValueError):
                call(**{**_pool(four), **bad})
    assert fake.launches == []


def test_native_form_declines_what_is_not_plain():
    pkg.lib()
    if pkg._native is None:
        pytest.skip("no native binding")
    x = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    t, l = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    f = torch.zeros(32, dtype=F64)
    assert pkg._native.rope(x, x, f, 1.0, False, None, 0, None, False) is NotImplemented
    assert pkg._native.paged_append(x, x, x, x, t, l, None, None, None, None, 1.0, False, None) is NotImplemented
    assert pkg._native.paged_gather(x, x, t, l, 3, None, None, None, None) is NotImplemented
    assert pkg._native.paged_decode(x[:, :, 0], x, x, t, l, None, None, None, None, None, None, None, 1.0, False, None, None,
                                    None) is NotImplemented
    for call in (pkg._native.rope, pkg._native.paged_append, pkg._native.paged_gather, pkg._native.paged_decode):
        assert call(x) is NotImplemented


# ----------------------------------------------------------- frequencies --
def test_frequencies():
    f, a = pkg.attn_rope_freqs(64, device="cpu")
    assert f.dtype == F64 and f.shape == (32,) and a == 1.0
    assert f[0] == 1.0 and math.isclose(f[16], 0.01, rel_tol=1e-14)
    g, a = pkg.attn_rope_freqs(64, scaling="linear", factor=4.0, device="cpu")
    assert torch.allclose(g * 4, f, rtol=1e-15, atol=0) and a == 1.0
    g, a = pkg.attn_rope_freqs(64, scaling="base", factor=4.0, device="cpu")
    assert g[0] == 1.0 and math.isclose(f[-1] / g[-1], 4.0, rel_tol=1e-12) and a == 1.0
    g, a = pkg.attn_rope_freqs(64, scaling="ramp", factor=4.0, original_length=4096, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1] * 4, f[turns <= 1], rtol=1e-15, atol=0)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    assert mid.any() and torch.allclose(g[mid], f[mid] * keep + f[mid] / 4 * (1 - keep), rtol=1e-14, atol=0)
    assert math.isclose(a, 0.1 * math.log(4) + 1)
    assert pkg.attn_rope_freqs(32, scaling="ramp", factor=2.0, original_length=10, amplitude=1.0, device="cpu")[1] == 1.0
    for bad in (dict(r=8), dict(r=40), dict(r=0), dict(r=64, base=0.0), dict(r=64, factor=-1.0), dict(r=64, scaling="other"),
                dict(r=64, scaling="ramp"), dict(r=64, scaling="ramp", original_length=5, low=2.0, high=2.0)):
        with pytest.raises(ValueError):
            pkg.attn_rope_freqs(device="cpu", **bad)
