"""Calls of the feed-forward block and of 8-bit activations that the GPU tests of their
results do not make."""
import pytest
import torch

from paper_2608_00573_amd import abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_rows_past_32_bits_are_refused():
    """More rows than a call takes, with few in the lower 32 bits."""
    n = 2 ** 32 + 5
    x = torch.empty(n, 1, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(abi.TrimmoeError, match="checkpoint_pack"):
        abi.trimmoe_checkpoint_pack(x)
    del x
    codes = torch.empty(n, 1, dtype=torch.int8, device=DEV)
    with pytest.raises(abi.TrimmoeError, match="checkpoint_unpack"):
        abi.trimmoe_checkpoint_unpack(codes, codes.view(torch.uint8))
    del codes
    w = torch.ones(1, 1, 1, device=DEV)
    x = torch.empty(n, 1, device=DEV)
    offsets = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    with pytest.raises(abi.TrimmoeError, match="expert_ffn"):
        abi.trimmoe_expert_ffn(w, w, w, x, offsets)
    with pytest.raises(abi.TrimmoeError, match="expert_ffn_backward"):
        abi.trimmoe_expert_ffn_backward(w, None, w, x, x, (x, None), offsets, want_dx=False)
