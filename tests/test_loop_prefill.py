"""A decode loop's prefills have its type, whatever its cache holds (no GPU)."""
import pytest
import torch

from paper_2608_08569_amd.loop import DecodeLoop


@pytest.mark.parametrize("bits", [None, 4])
@pytest.mark.parametrize("own,other", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
def test_a_prefill_of_another_type_is_refused(bits, own, other):
    loop = DecodeLoop(2, 4, 2, 64, [16, 16], [12, 12], 0.9, dtype=own, device="cpu", bits=bits)
    k, off = torch.zeros(2, 2, 8, 64, dtype=other), torch.arange(9, dtype=torch.int32)
    one = torch.zeros(2, dtype=torch.int64)
    n = torch.full((2,), 4, dtype=torch.int32)
    with pytest.raises(TypeError, match="prefill has dtype"):
        loop.fuse(k, k, one, n, off, one, n, 4)
    loop.retire(1)
    with pytest.raises(TypeError, match="prefill has dtype"):
        loop.admit(1, k, k, off)
    assert not loop.active[1] and loop.cap[1] == 0
