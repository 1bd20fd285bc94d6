"""kv_quantize on arrays that overlap (no GPU): blocks read begin and end while others
write the new lengths, so any common entry is refused before the launch."""
import ctypes

import pytest

from test_kv8_abi import INV, P, cache, cache8, lib, needs_no_gpu  # noqa: F401


@needs_no_gpu
@pytest.mark.parametrize("B", [1, 2, 40])
def test_new_lengths_overlap_neither_begin_nor_end(lib, B):  # noqa: F811
    def call(begin, end, new):
        return lib.dreams_kv_quantize(ctypes.byref(cache()), ctypes.byref(cache8()), B, begin, end, new, None, None)

    far = P + 4096
    for off in (0, 4, 4 * (B - 1)):
        if off // 4 < B:
            for new in (P + off, P - off):
                assert call(P, far, new) == INV and call(far, P, new) == INV, off
    for new in (P + 4 * B, P - 4 * B):  # side by side (no launch succeeds here, for want of a GPU)
        assert call(P, far, new) != INV and call(far, P, new) != INV
