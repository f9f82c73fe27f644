"""DecoderMlp's buffers and refusals (host logic; nothing is launched)."""
import pytest
import torch

from paper_2410_09615_amd import binding as B
from paper_2410_09615_amd.mlp import DecoderMlp


def _byte(n):
    return torch.empty(n, dtype=torch.uint8)


def _packed(n, k, rank):
    s = B.slim_packed_sizes(n, k, rank)
    none = torch.empty(0)
    return B.SlimLayer(n, k, rank, s["rank_pad"], none, none, none, none, none)


def _down(n, k):
    s = B.slim_block_fp8_weight_sizes(n, k)
    return B.SlimBlockFp8Weight(n, k, _byte(s["codes"]), torch.empty(s["scales"] // 4))


@pytest.mark.parametrize("f,k,rank,tokens", [(11008, 4096, 409, 4096), (28672, 8192, 819, 2048), (768, 512, 32, 64), (768, 512, 32, 1)])
def test_workspace_beside_a_layer_in_4_bits_covers_every_number_of_tokens(f, k, rank, tokens):
    """What a forward call needs does not grow with its tokens throughout: T = X R^T of fewer tokens is split into more ranges."""
    layer = _packed(2 * f, k, rank)
    mlp = DecoderMlp(torch.ones(k), layer, _down(k, f), tokens)
    need = [B.slim_workspace_bytes(layer, m) for m in range(1, tokens + 1)]
    assert mlp._ws.numel() >= max(need)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_takes_fp16_only(dtype):
    """Its inner matrices and what it returns are fp16: other inputs would come back in a type beside theirs."""
    mlp = DecoderMlp(torch.ones(256), _packed(512, 256, 32), _down(256, 256), 4)
    with pytest.raises(ValueError, match="float16"):
        mlp(torch.zeros(2, 256, dtype=dtype))
