"""CPU checks of chunk attention's limits, before anything touches a device."""
import ctypes as C

import paper_2511_07427_b200 as P
from paper_2511_07427_b200 import rows as R

BUF = C.create_string_buffer(4096 + 64)
ADDR = (C.addressof(BUF) + 63) // 64 * 64        # an aligned host address: never read, the calls are refused


def test_tables_of_more_than_2_to_the_25_columns_are_refused():
    """Beyond 2^30 rows a window of 2^30 would not be the caller's any more, and the last stage's end would not fit 32 bits."""
    cache = R._RowCache(ADDR, ADDR, None, None, 4, 2, 128, P.BF16)
    scores = R._Scores(0.1, 0.0, 0, None, None, None)
    for columns in (2 ** 25 + 1, 2 ** 26 - 1):
        assert R._library().dynakv_attend_chunk_workspace(C.byref(cache), 4, 3, 1, 3, columns) == -1
        assert R._library().dynakv_attend_chunk(C.byref(cache), ADDR, 4, 3, ADDR, 1, 3, ADDR, columns, ADDR, C.byref(scores), ADDR, None, ADDR, 1 << 40, None, None) == -1
    # the largest that is taken: bytes on a device, another error (no device) elsewhere
    assert R._library().dynakv_attend_chunk_workspace(C.byref(cache), 4, 3, 1, 3, 2 ** 25) != -1
