"""Limits of the 4-bit cache on the host alone: nothing is launched and no pointer below is followed."""
import pytest

from paper_2607_20357_gb300 import svl
from tests.test_kv4_abi import D, P, UNSUPPORTED, code


@pytest.mark.parametrize("desc", [D(65535, 65535, 128, 2 ** 31 - 1), D(65535, 65535, 64, 2 ** 31 - 1),
                                  D(65535, 2 ** 15, 128, 2 ** 31 - 1)])
def test_a_cache_whose_size_is_no_64_bit_number(svl_lib, desc):
    assert desc.n_slots * desc.n_kv_heads * 2 ** 26 * 36 * desc.d_head >= 2 ** 63
    assert svl.svl_kv4_cache_size(desc) == 0
    assert svl.svl_kv4_attention_workspace_size(desc, desc.n_kv_heads, 1) == 0
    ld = desc.n_kv_heads * desc.d_head
    assert code(svl.svl_kv4_write, desc, P, P, ld, P, ld, 0, P, P, None) == UNSUPPORTED
    assert code(svl.svl_kv4_read, desc, P, 0, P, P, P, ld, P, ld) == UNSUPPORTED
    assert code(svl.svl_kv4_reorder, desc, P, 1, 1, P, None, P, None) == UNSUPPORTED


def test_the_largest_sizes_that_are(svl_lib):
    assert svl.svl_kv4_cache_size(D(65535, 256, 128, 2 ** 31 - 1)) == 65535 * 256 * 2 ** 26 * 4608
    assert svl.svl_kv4_cache_size(D(65535, 65535, 64, 32)) == 65535 ** 2 * 2304
