"""The native form of attn_cross_fwd, attn_cross_bwd and attn_prefix_decode (csrc/binding.cpp): it declines whatever
is not plain, and where it answers, outputs, identities and errors are those of the Python form."""
import pytest
import torch

import paper_2609_33916_amd as pkg
from helpers import gpu_available
from test_native_binding import _both, native  # noqa: F401

BF16 = torch.bfloat16


def test_declines_what_is_not_plain(native):  # noqa: F811
    x, l, t = torch.zeros(1, 2, 8, 32), torch.zeros(1, 2, 8), torch.zeros(4, 2)
    assert native.cross_fwd(x, x, x, None, False, 0, None, None, None, None, 0, None, None) is NotImplemented
    assert native.cross_fwd(x, x, x) is NotImplemented
    assert native.cross_bwd(x, x, x, x, l, x, None, False, 0, None, None, t, None, 0, None, None) is NotImplemented
    assert native.prefix_decode(x[0], x[0], x[0], x, x, None, None, None, 3, None, None, None) is NotImplemented
    assert native.prefix_decode(None) is NotImplemented


def _inputs(dtype=BF16):
    q = torch.randn(2, 70, 6, 64, device="cuda", dtype=dtype).transpose(1, 2)
    kv = torch.randn(2, 90, 6, 64, device="cuda", dtype=dtype).transpose(1, 2)
    bias = torch.randn(32, 6, device="cuda", dtype=dtype)
    rows, first = pkg.attn_bias_buckets(32, 128)
    return q, kv[:, :3], kv[:, 3:], bias, rows, first


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_same_as_the_python_form(native, monkeypatch, dtype):  # noqa: F811
    q, k, v, bias, rows, first = _inputs(dtype)
    lens = torch.tensor([90, 33], dtype=torch.int32, device="cuda")
    starts = torch.tensor([20, -10], dtype=torch.int32, device="cuda")
    with_bias = dict(bias=bias, bias_rows=rows, bias_first=first)
    for how in ({}, dict(k_lens=lens, scale=0.2), dict(causal=True, start=20), dict(causal=True, starts=starts, **with_bias), with_bias):
        o, lse = pkg.attn_cross_fwd(q, k, v, **how)
        for call in (lambda: pkg.attn_cross_fwd(q, k, v, **how), lambda: pkg.attn_cross_bwd(q, k, v, o, lse, q, **how)):
            got, want = _both(monkeypatch, call)
            assert type(got) is tuple and len(got) == len(want)
            for a, b in zip(got, want):
                assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride() and torch.equal(a, b)
    if dtype == BF16:
        qd, kp, kc, new = (torch.randn(*s, device="cuda").to(BF16) for s in ((2, 6, 64), (3, 50, 64), (2, 3, 40, 64), (2, 3, 64)))
        lens = torch.tensor([39, 5], dtype=torch.int32, device="cuda")
        for call in (lambda: pkg.attn_prefix_decode(qd, kp, kp, kc, kc.clone(), new, new, lens),
                     lambda: pkg.attn_prefix_decode(qd, kp, kp, kc, kc, cache_lens=lens, n=39, scale=0.3),
                     lambda: pkg.attn_prefix_decode(qd, kp, kp, kc, kc, n=40)):
            got, want = _both(monkeypatch, call)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
def test_given_outputs_and_errors(native, monkeypatch):  # noqa: F811
    q, k, v, bias, rows, first = _inputs()
    how = dict(bias=bias, bias_rows=rows, bias_first=first)
    out = torch.zeros(2, 70, 6, 64, device="cuda", dtype=BF16).transpose(1, 2), torch.zeros(2, 6, 70, device="cuda")
    assert pkg.attn_cross_fwd(q, k, v, out=out, **how) is out
    grads = (torch.empty_like(q), torch.empty(2, 3, 90, 64, device="cuda", dtype=BF16), torch.empty(2, 3, 90, 64, device="cuda", dtype=BF16), None)
    assert pkg.attn_cross_bwd(q, k, v, *out, q, out=grads, **how) is grads
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    far = torch.empty(1, 1, 2, 1 << 23, device="cuda", dtype=BF16)[..., :64]
    for bad in (lambda: pkg.attn_cross_fwd(q.half(), k, v), lambda: pkg.attn_cross_fwd(q, k.float(), v), lambda: pkg.attn_cross_fwd(q, k[:, :, :5], v),
                lambda: pkg.attn_cross_fwd(q[..., :48], k[..., :48], v[..., :48]), lambda: pkg.attn_cross_fwd(q, k[:, :2], v[:, :2], scale=1.0, causal=True),
                lambda: pkg.attn_cross_fwd(q[:, :4], k, v), lambda: pkg.attn_cross_fwd(q, k, v, scale=float("nan")), lambda: pkg.attn_cross_fwd(q, k, v, start=2 ** 30 + 1),
                lambda: pkg.attn_cross_fwd(q, k, v, **{**how, "bias_rows": rows[:1]}), lambda: pkg.attn_cross_fwd(far, far, far),
                lambda: pkg.attn_cross_bwd(q, k, v, *out, q, workspace=ws[1:], **how), lambda: pkg.attn_cross_bwd(q, k, v, *out, q, workspace=ws[:100], **how),
                lambda: pkg.attn_cross_bwd(q, k, v, *out, q, out=(q, k, k))):
        seen = []
        for direct in (True, False):
            with monkeypatch.context() as m:
                if not direct:
                    m.setattr(pkg, "_native_lib", None)
                try:
                    bad()
                    seen.append(None)
                except (ValueError, TypeError, pkg.AttnError) as e:
                    seen.append((type(e), str(e)))
        assert seen[0] == seen[1]
        if seen[0] is None:   # the call that is fine: 6 query heads on 2
            assert bad() is not None
    torch.cuda.synchronize()
