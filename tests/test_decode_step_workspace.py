"""paep_attend_workspace_bytes: 0 for no shape that the kernels can run split; and what a caller may rely on when it asks once: the
answer for a longer cache, a larger batch or more heads is never less than for a shorter, smaller one or fewer."""
import ctypes

import pytest

from paper_2511_10676_amd import binding as B


def _bytes(batch, max_len, mass, Hkv, G, D, dtype):
    page = 16
    wide = 1 << 20
    c = B.CacheDesc(batch, Hkv, D, D, page, 8, wide, dtype, Hkv * page * D, page * D, D, Hkv * page * D, page * D, D)
    d = B.AttendDesc(Hkv * G, max_len, 1.0, 0, Hkv * G * D, D, wide * page)
    return B.lib().paep_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(d), mass)


@pytest.mark.parametrize("Hkv,batch,max_len", [(8, 200, 16777216), (16, 61, 1 << 24), (1, 2000, 1 << 23)])
def test_attend_without_mass_is_not_refused_for_the_sake_of_the_mass(Hkv, batch, max_len):
    """Where the workgroups that add up mass would be more than a launch can hold, calls that do not ask for it still run."""
    assert _bytes(batch, max_len, 0, Hkv, 4, 128, B.BF16) > 0
    assert _bytes(batch, max_len, 1, Hkv, 4, 128, B.BF16) == 0
