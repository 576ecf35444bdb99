"""CPU test of the cache's calls: positions are 32-bit numbers, so a call that would write or read beyond the last of them is refused before anything is launched."""
import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF
from tests.test_target_host import _cache, _read, _write, lib  # noqa: F401

LAST = 2 ** 31 - 1


@pytest.mark.parametrize("start,rows", [(LAST, 1), (LAST - 4, 5), (LAST - 1, 1000)])
def test_positions_beyond_32_bits_are_refused(start, rows):
    huge = _cache(offsets=(0, 64, 1 << 33))
    assert VF.ps_cache_write(_write(huge, rows=rows, kv_len=(0, start), n_seq=(1, rows)), None) == B.PS_ERR_UNSUPPORTED
    assert VF.ps_cache_read(_read(huge, rows=rows, start=(0, start), n_seq=(1, rows)), None) == B.PS_ERR_UNSUPPORTED
    if rows == 5:
        assert VF.ps_cache_write(_write(huge, rows=rows, kv_len=(0, start), n_accepted=0x1000, path=0x1000, path_rows=4), None) == B.PS_ERR_UNSUPPORTED
