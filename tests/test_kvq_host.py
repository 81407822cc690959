"""The 8-bit cache's sizes and refusals that need no GPU."""
import ctypes as C

import pytest

from paper_2506_03700_amd import binding as ad
from paper_2506_03700_amd import synth


def test_sizes():
    L = ad.lib()
    s = synth.LLAMA8B
    cfg = ad.make_config(s)
    n = 1 << 17
    got, had = L.ad_kvq_bytes(C.byref(cfg), n), L.ad_kv_bytes(C.byref(cfg), n)
    entries = s.n_layers * 2 * s.n_kv_heads * n * (s.head_dim + 1)
    # entries, one layer's values in 16 bits and rows for the prompt pass, partials of 512 items, the rotary table
    assert entries < got < entries + 2 * s.n_kv_heads * n * s.head_dim * 2 + n * s.head_dim * 4 + (1 << 29)
    assert got < 0.58 * had
    # the 16-bit cache's size is what it was: entries, partials of 128 positions, table, prompt pass
    assert had > s.n_layers * 2 * s.n_kv_heads * n * s.head_dim * 2


@pytest.mark.parametrize("dtype", [synth.F32, synth.BF16, synth.F16])
@pytest.mark.parametrize("head_dim,most", [(64, 1 << 25), (128, 1 << 24)])
def test_positions(head_dim, most, dtype):
    L = ad.lib()
    cfg = ad.make_config(synth.TINY.with_(head_dim=head_dim, dtype=dtype))
    assert L.ad_kvq_bytes(C.byref(cfg), most) > 0
    assert L.ad_kvq_bytes(C.byref(cfg), most + 1) == 0 and b"more positions" in L.ad_last_error()
    assert L.ad_kvq_bytes(C.byref(cfg), 0) == 0 and L.ad_kvq_bytes(None, 8) == 0
    assert L.ad_kvq_bytes(C.byref(ad.make_config(synth.TINY.with_(head_dim=96))), 8) == 0


def test_null_arguments():
    L = ad.lib()
    assert L.ad_kvq_create(None, None, 0, 8, None, None) == ad.AD_EINVAL
    assert L.ad_kvq_append(None, None, 1, None, None, 0, 0, 1, None) == ad.AD_EINVAL
    assert L.ad_kvq_read(None, None, 1, 0, 1, None, None, 0, None) == ad.AD_EINVAL
    assert L.ad_kvq_attend(None, None, 1, None, None, 1, None, None) == ad.AD_EINVAL
