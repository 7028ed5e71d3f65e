"""Sizes at which a grid of kvlinc_bounded.h would have 2^32 threads: refused on the host, before any launch."""
import paper_2510_05373_amd as kv
import pytest

from tests.test_bounded_api import decode, of_rows, plain, rotary, rows


# 2^26 - 1, - 2 and - 3 tokens, four to a workgroup of 256 threads
@pytest.mark.parametrize("B, T", [(8193, 8191), (37262, 1801), (5197, 12913)])
def test_rotary_of_more_tokens_than_a_grid_holds(B, T):
    assert (1 << 26) - 4 < B * T < 1 << 26
    whole = (T * 128, T * 128, 128)
    assert rotary(plain(B=B, H_q=1, H_kv=1), q=rows(at=0x100000, out=0x4000000000000, strides=whole), T=T) == kv.KVLINC_EINVAL


# A wave a slot: 2^26 slots, max_groups + 1 of every pair
@pytest.mark.parametrize("B, H_kv, max_groups", [(64, 1, (1 << 20) - 1), (1 << 12, 2, (1 << 13) - 1), (1, 1 << 21, 31)])
def test_mass_of_more_slots_than_a_grid_holds(B, H_kv, max_groups):
    c = plain(B=B, H_q=H_kv, H_kv=H_kv, max_groups=max_groups)
    assert B * H_kv * (max_groups + 1) == 1 << 26
    apart = dict(q=0x200000, mass=None, mass_out=0x400000000000)
    assert decode(c, out=0x200000000000, **apart) == of_rows(c, **apart) == kv.KVLINC_EINVAL
    assert kv.kvlinc_decode_mass_workspace_bytes(c) == kv.kvlinc_attention_mass_workspace_bytes(c, 4) == kv.kvlinc_cache_evict_workspace_bytes(c) == 0
    c = plain(B=B, H_q=H_kv, H_kv=H_kv, max_groups=max_groups - 1)
    assert min(kv.kvlinc_decode_mass_workspace_bytes(c), kv.kvlinc_attention_mass_workspace_bytes(c, 4), kv.kvlinc_cache_evict_workspace_bytes(c)) > 0
    assert decode(c, out=0x200000000000, size=0, **apart) == of_rows(c, size=0, **apart) == kv.KVLINC_EWORKSPACE
