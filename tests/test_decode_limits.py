"""Calls just within and just behind the limits of their sizes (no GPU call is made before these return)."""
import pytest

from paper_2604_06664_amd import FDY_ERR_INVALID_ARG, FDY_OK
from paper_2604_06664_amd import decode as fdd

A = 0x10000  # an address that is aligned and never touched


def bounds(heads, row_pages, max_fresh, fresh, n_seqs):
    kv = fdd.make_kv(A, None, type=fdd.FDY_BF16, n_pages=4, page_tokens=16, n_heads=heads, head_dim=8, page_stride=128 * heads,
                     token_stride=8 * heads, head_stride=8)
    return fdd.fdy_bounds(bounds=A, table=A, lens=A, rows=None, fresh=fresh, kv=kv, n_seqs=n_seqs, n_rows=1, row_pages=row_pages,
                          max_fresh=max_fresh)


@pytest.mark.parametrize("heads,row_pages,max_fresh,fresh,rc", [
    (32, 1 << 26, 1 << 30, A, FDY_ERR_INVALID_ARG),         # 2^31 pieces of work, counted in 32 bits
    (32, (1 << 27) - 1, 0xFFFFFFFF, A, FDY_ERR_INVALID_ARG),
    (64, (1 << 27) - 1, 1 << 30, A, FDY_ERR_INVALID_ARG),   # 2^32: none of the bounds would have been written
    (32, (1 << 26) - 1, 1 << 30, A, FDY_OK),
    (64, (1 << 27) - 1, 1 << 30, None, FDY_OK),             # one new token each
    (64, (1 << 27) - 1, 1 << 20, A, FDY_OK),
])
def test_new_pages_of_all_heads_are_counted_in_32_bits(heads, row_pages, max_fresh, fresh, rc):
    # without sequences nothing is launched, but sizes are looked at first
    assert fdd.fdy_page_bounds(bounds(heads, row_pages, max_fresh, fresh, 0), stream=0, check=False) == rc
