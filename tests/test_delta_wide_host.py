"""The sizes of the wide heads' tests are cut into segments: their workspace has room for what segments leave."""
import ctypes

import pytest

from delta_wide_sizes import WIDE

nd = pytest.importorskip("paper_2607_03574_amd")


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("lens,H,Hk,dk,dv", WIDE)
def test_sequences_are_cut(dtype, packed, lens, H, Hk, dk, dv):
    if not packed and len(lens) > 1:
        pytest.skip("sequences of one length")
    n = sum(lens)
    padded, need = (dk + 7) // 8 * 8, nd._sz()
    assert nd._delta_ws(nd._DeltaShape(dtype, len(lens), n, H, Hk, dk, dv, 1.0), int(packed), 0, ctypes.byref(need)) == nd.OK
    rows = 2 * n * Hk * padded * (2 if dtype else 4) if dk % 8 else 0       # copies of q and k
    chunks = (n // 32 + len(lens) if packed else -(-n // 32)) * H * (512 + (6 + 2 * (2 if dtype else 3)) * 1024)
    # two segments at the least: what each adds to a state, and what it makes of one
    assert need.value >= rows + chunks + 2 * H * dk * (dv + padded) * 4
    # and none for the same tokens in sequences of 128 each
    assert nd._delta_ws(nd._DeltaShape(dtype, n // 128, n // 128 * 128, H, Hk, dk, dv, 1.0), 0, 0, ctypes.byref(need)) == nd.OK
    assert need.value < rows + chunks + 2 * H * dk * (dv + padded) * 4
