"""Calls of the feed-forward block's binding that it refuses, with what it says (no call
below reaches the GPU)."""
import pytest
import torch

from paper_2608_00573_amd import abi


def _t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def _packed(n, c):
    return abi.Packed(_t(n, c, dtype=torch.int8), _t(n, -(-c // 32), dtype=torch.uint8))


W = dict(w_up=_t(2, 8, 4), w_gate=_t(2, 8, 4), w_down=_t(2, 4, 8))
OFFSETS = _t(3, dtype=torch.int32)


@pytest.mark.parametrize("x", [_packed(3, 4), tuple(_packed(3, 4)), None])
def test_the_forward_takes_rows_as_a_tensor_only(x):
    with pytest.raises(ValueError, match="x.*gradient alone"):
        abi.trimmoe_expert_ffn(**W, x=x, offsets=OFFSETS)


def test_the_gradient_takes_dy_as_a_tensor_only():
    with pytest.raises(ValueError, match="dy"):
        abi.trimmoe_expert_ffn_backward(**W, x=_t(3, 4), dy=_packed(3, 4), kept=(_t(3, 8), _t(3, 8)),
                                        offsets=OFFSETS)


@pytest.mark.parametrize("call", [
    lambda: abi.trimmoe_expert_ffn(**W, x=_t(3, 4), offsets=OFFSETS),
    lambda: abi.trimmoe_expert_ffn_backward(**W, x=_t(3, 4), dy=_t(3, 4), kept=(_t(3, 8), _t(3, 8)),
                                            offsets=OFFSETS),
    lambda: abi.trimmoe_checkpoint_pack(_t(2, 32)),
    lambda: abi.trimmoe_checkpoint_unpack(*_packed(2, 32)),
    lambda: abi.trimmoe_head_cross_entropy(_t(5, 4), _t(3, 4), _t(3, dtype=torch.int32)),
])
def test_host_tensors_are_refused_by_where_they_are(call):
    with pytest.raises(ValueError, match="GPU.* not on cpu") as e:
        call()
    assert "loss" not in str(e.value)


@pytest.mark.parametrize("name,dims", [
    ("trimmoe_expert_ffn", (abi.BF16, abi.ACT_SWIGLU, 4, 64, 128, 2 ** 32 + 10, 0)),
    ("trimmoe_expert_ffn", (abi.F32, abi.ACT_RELU, 1, 2 ** 32 + 1, 3, 10, 0)),
    ("trimmoe_expert_ffn_backward", (abi.F32, abi.ACT_RELU, 1, 3, 2 ** 40 + 1, 10, 0)),
    ("trimmoe_expert_ffn_backward", (abi.F32, abi.ACT_RELU, 2 ** 32 + 1, 3, 4, 10, 0)),
    ("trimmoe_head_cross_entropy", (abi.F32, 2 ** 32 + 7, 4, 8)),
    ("trimmoe_balance_loss", (abi.F32, 8, 2, 4, 2 ** 32 + 8)),
])
def test_sizes_past_32_bits_are_refused(name, dims):
    """... and not taken by their lower bits."""
    with pytest.raises(abi.TrimmoeError, match=name):
        abi._loss_ws_bytes(name, dims)
