"""A table of frequencies without entries is refused, not taken for no rotation."""
import pytest
import torch

import paper_2609_33916_amd as pkg
from test_binding_host import gpu
from test_paged_host import _pool, fake  # noqa: F401 (fixture)


@pytest.mark.parametrize("four", [False, True])
def test_empty_frequencies(fake, four):   # noqa: F811
    none = gpu(0, dtype=torch.float64)
    kv = gpu(3, 2, 5, 64)
    calls = [lambda: pkg.attn_paged_append(kv, kv, freqs=none, **_pool(four)),
             lambda: pkg.attn_paged_decode(gpu(3, 4, 64), freqs=none, out=(gpu(3, 4, 64), gpu(3, 4, dtype=torch.float32)), **_pool(four)),
             lambda: pkg.attn_rope(kv, kv, none), lambda: pkg.attn_rope_bwd(kv, kv, none)]
    for call in calls:
        with pytest.raises(ValueError, match="freqs"):
            call()
    assert fake.launches == []


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("native", [True, False])
def test_empty_frequencies_in_both_forms(native, monkeypatch):
    k = torch.zeros(1, 1, 3, 64, dtype=torch.bfloat16, device="cuda")
    pages = torch.full((1, 1, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.float64, device="cuda")
    pkg.lib()
    if not native:
        monkeypatch.setattr(pkg, "_native_lib", None)
    for call in (lambda: pkg.attn_paged_append(k, k, pages, pages, table, lens, freqs=none),
                 lambda: pkg.attn_paged_decode(k[:, :, 0], pages, pages, table, lens, k[:, :, 0], k[:, :, 0], freqs=none),
                 lambda: pkg.attn_rope(k, None, none)):
        with pytest.raises(ValueError, match="freqs"):
            call()
    assert bool((pages == 7).all())
