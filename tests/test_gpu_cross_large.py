"""Attention to a prompt for so many short sequences that the form of few rows has no launch for them."""
import pytest
import torch

import block_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu


def test_many_single_queries():
    """2^19 sequences of one query and 16 heads, one shared prompt of which each reads a length of its own."""
    B, Lk, heads, d = 1 << 19, 1024, 16, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(9)

    def draw(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = draw(B, 1, heads, d), draw(1, Lk, heads, d), draw(1, Lk, heads, d)
    lengths = torch.randint(0, Lk + 1, (B,), generator=g, device="cuda").to(torch.int32)
    out = rf.rf_cross_attention(q, k.expand(B, -1, -1, -1), v.expand(B, -1, -1, -1), lengths)
    at = torch.tensor([0, 1, 7, 4095, 262143, 262144, 400001, B - 2, B - 1], device="cuda")
    want, bound = ref.cross(q[at], k.expand(len(at), -1, -1, -1), v.expand(len(at), -1, -1, -1), lengths[at].tolist())
    ref.assert_within(out[at], want, bound)
    assert bool(torch.isfinite(out).all())
    assert torch.equal((out != 0).any(-1).any(-1).any(-1), lengths > 0)
