"""``forward_rotary`` on the layouts of heads that a projection may leave."""

import pytest
import torch

import paper_2512_02541_b200 as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("frame", (False, True))
@pytest.mark.parametrize("shift", (0, 1, 4, 8))
def test_contiguous_heads_at_any_element(shift, frame):
    """Contiguous tensors that begin at an element that the attention's 16 bytes do not fall on: the same results as aligned ones."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    params = P.make_params(3, 6, 7, 5, 4, 64, 4)
    shape = (3 * 47, 4, 64)
    q, k, v = (torch.randn(shape, generator=gen, device="cuda").bfloat16() for _ in range(3))
    layer, rotary, positions = P.SubsampledGlobalAttention(params), P.AxialRotary(64, (16, 16)), P.token_positions(params)
    want = layer.forward_rotary(q, k, v, positions, rotary, frame=frame)
    room = torch.zeros(q.numel() + shift, dtype=torch.bfloat16, device="cuda")
    moved = []
    for t in (q, k, v):
        moved.append(room.clone()[shift:].view(shape))
        moved[-1].copy_(t)
        assert moved[-1].is_contiguous()
    got = layer.forward_rotary(*moved, positions, rotary, frame=frame)
    layer.check_status()
    assert torch.equal(got, want)
