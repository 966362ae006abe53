"""The paged cache's limits on counts, without a GPU: what the kernels' 32-bit
indexes do not hold is refused before anything is launched."""

import ctypes

from paper_2607_15105_amd import hga
from tests.test_paged_args import FAKE, _attend, _cfg, _desc


def _row_calls(desc):
    c, S = _cfg(), hga.Strides(2 * 128, 128)
    return [fn(ctypes.byref(c), ctypes.byref(desc), FAKE, S, FAKE, S, 0, FAKE, FAKE, None)
            for fn in (hga.lib().hga_cache_write, hga.lib().hga_cache_read)]


def test_more_sequences_than_their_loops_count():
    """seq_rows is looked through 64 entries at a time with a 32-bit index, which has
    to pass the last entry."""
    assert _attend(desc=_desc(n_seqs=1 << 30)) == -3  # all is right but the workspace
    for n in ((1 << 30) + 1, (1 << 31) - 64, (1 << 31) - 1):
        assert _attend(desc=_desc(n_seqs=n)) == -2, n
        assert _row_calls(_desc(n_seqs=n)) == [-2, -2], n
    assert _row_calls(_desc(n_seqs=1 << 30)) == [-1, -1]  # the rows' count, which is checked next


def test_scales_of_a_page_that_pass_32_bits():
    """The scale table's page stride, heads * page_size bytes, is held in 32 bits."""
    f8 = dict(format=hga.CACHE_E4M3, k_scale=FAKE, v_scale=FAKE, page_size=65536)
    for heads, want in ((65535, -3), (65536, -2), (131072, -2)):
        c = _cfg(hq=heads, hkv=heads)
        assert _attend(c, _desc(**f8), n_rows=1, max_rows=1, qs=hga.Strides(heads * 128, 128)) == want, heads
    c = _cfg(hq=65536, hkv=65536)
    assert _attend(c, _desc(page_size=65536), n_rows=1, max_rows=1, qs=hga.Strides(65536 * 128, 128)) == -3  # no scales
