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


LENGTHS = sorted({*range(1, 1400, 13), *range(241, 245), *range(1, 300000, 3989), *range(255, 9000, 256), *range(256, 9000, 256), *range(272, 9000, 256),
                  16384, 16400, 65535, 65536, 131071, 131072, 131073, 524287, 524288, 524289, 600000, 1048576, 5000000, 16777216})


@pytest.mark.parametrize("mass", [0, 1])
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("Hkv,G,D", [(1, 1, 64), (8, 4, 128), (4, 8, 128), (3, 7, 80), (16, 1, 128), (1, 40, 256)])
@pytest.mark.parametrize("batch", [1, 2, 3, 61, 200])
def test_attend_workspace_does_not_shrink_with_longer_caches(batch, Hkv, G, D, dtype, mass):
    sizes = [_bytes(batch, n, mass, Hkv, G, D, dtype) for n in LENGTHS]
    fits = [s for s in sizes if s or not mass]            # (a mass always needs some: 0 is a shape that is refused)
    assert fits == sorted(fits) and sizes[:len(fits)] == fits


@pytest.mark.parametrize("mass", [0, 1])
@pytest.mark.parametrize("Hkv,G,D", [(1, 1, 64), (8, 4, 128), (3, 7, 80), (1, 40, 256)])
@pytest.mark.parametrize("max_len", [1, 100, 241, 242, 300, 500, 1000, 2049, 4096, 16400, 131072])
def test_attend_workspace_does_not_shrink_with_larger_batches_and_more_heads(max_len, Hkv, G, D, mass):
    sizes = [_bytes(b, max_len, mass, Hkv, G, D, B.BF16) for b in range(0, 140)]
    assert sizes == sorted(sizes)
    sizes = [_bytes(3, max_len, mass, h, G, D, B.BF16) for h in range(1, 24)]
    assert sizes == sorted(sizes)
