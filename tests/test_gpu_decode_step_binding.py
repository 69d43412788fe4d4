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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_default_bound_of_a_table_for_more_positions_than_32_bits_count(dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    kp, vp = (torch.randn((2, 1, 65536, 8), generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.full((2, 40000), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[1, 0] = 1, 0
    q, lengths = torch.randn((2, 3, 8), generator=g, device="cuda").to(dtype), _i32(100, 65000)
    got = B.attend(q, kp, vp, table, lengths)
    want = B.attend(q, kp, vp, table, lengths, max_len=65000)
    torch.cuda.synchronize()
    assert torch.allclose(got.out.float(), want.out.float(), rtol=2 ** -7, atol=1e-5)


@pytest.mark.parametrize("wrong", [-(1 << 31) - 1, 1 << 31, (1 << 32) + 16])
def test_numbers_past_32_bits_are_refused(wrong):
    """... and not taken for what their lower 32 bits are."""
    kp, vp = torch.zeros((4, 1, 16, 8), device="cuda"), torch.zeros((4, 1, 16, 8), device="cuda")
    table, free, lengths = _i32([0, 1]), _i32([2, 3]), _i32(20)
    q, mass = torch.zeros((1, 1, 8), device="cuda"), torch.zeros((1, 1, 32), device="cuda")
    with pytest.raises(ValueError, match="max_len"):
        B.attend(q, kp, vp, table, lengths, max_len=wrong)
    with pytest.raises(ValueError, match="max_len"):
        B.cache_evict(kp, vp, table, lengths, mass, free, 16, 4, max_len=wrong)
    with pytest.raises(ValueError, match="budget"):
        B.cache_evict(kp, vp, table, lengths, mass, free, wrong, 4)
    with pytest.raises(ValueError, match="recent"):
        B.cache_evict(kp, vp, table, lengths, mass, free, 16, wrong)
    x, W = torch.zeros((0, 8), device="cuda"), torch.zeros((4, 8), device="cuda")
    with pytest.raises(ValueError, match="k must"):
        B.moe_layer(x, W, torch.zeros((4, 16, 8), device="cuda"), torch.zeros((4, 8, 8), device="cuda"), wrong)
