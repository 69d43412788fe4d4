"""The Python calls of the decode step's operators at the ends of what their arguments can be."""
import pytest
import torch

from paper_2511_10676_amd import binding as B

pytestmark = pytest.mark.gpu


def _i32(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def test_evict_takes_buffers_for_an_empty_batch():
    kp = torch.zeros((4, 2, 16, 8), device="cuda")
    none = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    lengths, mass = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 2, 64), device="cuda")
    first = B.cache_evict(kp, kp.clone(), none, lengths, mass, none, 16, 4)
    again = B.cache_evict(kp, kp.clone(), none, lengths, mass, none, 16, 4, out=first)
    assert again is first and first.kept.shape == (0, 2, 16)
