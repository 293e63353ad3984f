"""What the workspace queries of the serving calls ask for, on the CPU."""
import ctypes as C

import pytest

from paper_2403_02352_amd import binding

MB = 10 ** 6


def packed(n_seq, tokens, heads, hk, d, t):
    return binding.lib.atp_attention_packed_workspace(n_seq, tokens, heads, hk, d, t)


def paged(n_seq, positions, tokens, heads, hk, d, t, max_new=0, page=16):
    cache = binding._Cache(None, None, None, None, 1, page, hk, d, binding.ATP_CACHE_SAME)
    return binding.lib.atp_attention_paged_workspace(C.byref(cache), C.byref(binding._Batch(None, None, None, n_seq, positions // page, tokens)), heads, max_new, t)


@pytest.mark.parametrize("t", [binding.ATP_F32, binding.ATP_BF16])
@pytest.mark.parametrize("d", [8, 64, 128, 136, 256])
def test_at_most_2048_tiles_of_128_rows(t, d):
    """Partial sums are bounded by the items wanted, not by tokens, heads or lengths: 2·1024 tiles of 128 rows of the padded width and their two numbers."""
    most = 2 * 1024 * 128 * ((64 if d <= 64 else 128 if d <= 128 else 256) * 4 + 8)
    assert most <= (137 if d <= 128 else 271) * MB
    for hk in (1, 3, 8, 100, 512, 700, 1024, 5000, 65535):
        for tokens in (1, 5, 100, 127, 2000, 30000):
            for n_seq in (1, 50, 65536):
                assert packed(n_seq, tokens, hk, hk, d, t) <= most
                for positions in (512, 4096, 8192, 2 ** 20):
                    for max_new in (0, 1):
                        assert paged(n_seq, positions, tokens, hk, hk, d, t, max_new) <= most


@pytest.mark.parametrize("t", [binding.ATP_F32, binding.ATP_BF16])
def test_none_where_every_key_head_is_an_item_already(t):
    """More key heads than half the items wanted: one item a key head, nothing is cut."""
    for hk in (600, 1024, 4096):
        assert packed(1, 2000 if hk == 600 else 100, hk, hk, 64, t) == 0
        for tokens in (1, 100):
            assert paged(tokens, 2 ** 17, tokens, hk, hk, 64, t) == 0 and paged(1, 2 ** 17, tokens, 2 * hk, hk, 128, t, 1) == 0
    assert paged(1, 2 ** 17, 1, 256, 256, 64, t) > 0 or t == binding.ATP_F32
