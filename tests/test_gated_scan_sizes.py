"""dsattn_gated_scan_workspace and the checks of a workspace, on the host: streams of up to the largest number of frames."""
import ctypes

import pytest

from paper_2406_16260_amd import binding as B

MOST = 0x7fffffff - 2 * B.DSATTN_SCAN_FRAMES


@pytest.mark.parametrize("io_dtype", [B.DSATTN_F32, B.DSATTN_BF16])
@pytest.mark.parametrize("T", [MOST, MOST - 1, 2147000000, 2146959000, 2146958712, 2000000000, 1 << 30, 1 << 24])
def test_workspaces_of_the_longest_streams(T, io_dtype):
    """One channel is one wavefront: 4,096 chunks at most, each with a product and a result in fp32, and no more than twice too few
    (a chunk's frames are rounded up to a multiple of 16)."""
    need = B.dsattn_gated_scan_workspace(1, T, 1, 1, io_dtype=io_dtype)
    assert 4096 * 8 // 2 < need <= 4096 * 8
    assert need <= B.dsattn_gated_scan_workspace(2, T, 1, 1, io_dtype=io_dtype) <= 2 * 4096 * 8


@pytest.mark.parametrize("T", [MOST, 2147000000, 1 << 30])
def test_a_workspace_that_is_too_small_is_refused(T):
    lib, p = B.load(), [k << 50 for k in range(1, 9)]
    need = B.dsattn_gated_scan_workspace(1, T, 1, 1)
    d = ctypes.byref(B.DsattnScanDesc(1, T, 1, 1, B.DSATTN_SCAN_MEAN, B.DSATTN_BF16))
    for space, size in ((None, need), (p[6], need - 1), (p[6], 0)):
        assert lib.dsattn_gated_scan(d, None, p[0], p[1], None, p[2], None, None, space, size, None) == B.DSATTN_EINVAL
        assert lib.dsattn_gated_scan_backward(d, None, p[0], p[1], p[2], p[3], None, p[4], p[5], None, space, size,
                                              None) == B.DSATTN_EINVAL
