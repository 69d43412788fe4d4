"""Rows of numbers below the smallest normal one, and next to it, into a cache in 4 bits."""
import numpy as np
import pytest
import torch

import rotate_fourbit_reference as R
from paper_2511_10676_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_subnormal_numbers_are_rounded_as_others_are(dtype):
    """The least power is 2^-125: what is above a quarter of it, 2^-127, becomes half of it, the tie 0."""
    x = np.zeros((6, 1, 128))
    x[0, 0] = np.arange(128)                              # 2^-127 is 64
    x[1, 0] = -np.arange(128)
    x[2, 0] = np.arange(64, 192)                          # into the normal numbers, 128 on: 192 is the tie of a half and one power
    x[3, 0] = np.arange(128) * (-1.0) ** np.arange(128)
    x[3, 0, ::32] = 256 * 7                               # the largest that 2^-125 takes
    x[4, 0] = np.arange(128)
    x[4, 0, ::32] = 256 * 7.5                             # the next power: a quarter of it is 128
    x[5, 0, 1::2] = 64 + (0.5 if dtype is torch.float32 else 1)
    x = (x * 2.0 ** -133).astype(np.float32)
    k = torch.from_numpy(x).to(dtype)
    assert np.array_equal(k.float().numpy(), x)
    kp, ks = torch.zeros((6, 1, 1, 64), dtype=torch.uint8, device="cuda"), torch.zeros((6, 1, 4, 1), dtype=torch.uint8, device="cuda")
    vp, vs = kp.clone(), ks.clone()
    table, pos = torch.arange(6, dtype=torch.int32, device="cuda").view(6, 1), torch.zeros(6, dtype=torch.int32, device="cuda")
    B.cache_append_fourbit(k.cuda(), k.cuda(), kp, vp, ks, vs, table, pos)
    want, byte = R.to_fourbit(x)
    assert np.any(want[0] != 0) and np.any(want[0, 0, 1:65] == 0)
    for p, s in ((kp, ks), (vp, vs)):
        assert np.array_equal(s.cpu().numpy()[:, :, :, 0], byte)
        assert np.array_equal(R.values(p.cpu().numpy()[:, :, 0], byte), want)
    for t in (torch.bfloat16, torch.float32):
        assert np.array_equal(B.cache_read_fourbit(kp, vp, ks, vs, table, pos, dtype=t).k.double().cpu().numpy(), want)
