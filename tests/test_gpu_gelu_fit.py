"""GELU of the 8-bit products and the group norm, whose tail is a fit of erfc, to the last places of its own size."""
import pytest
import torch

import block_reference as block

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
U = block.U


def bound(z):
    """gelu(z) in 64 bits, and how far z t 2^f may be off below 0, or z less that above, u = 2^-24, h = Phi(-|z|).

    f = s - 0.7213 z^2: the constant, the square and the sum are rounded once each, 3 u 0.7213 z^2 + 3.2 u as |s| is at most 3.2. s is a
    polynomial of degree 8 in t <= 1, by eight fused steps from rounded coefficients, 9 u sum |p_i| = 103 u, at a t that is off by 4 u (its
    argument by 2, the reciprocal by its last place, 2 u): 4 u sum i |p_i| = 152 u. 2^f turns an error of f into ln 2 of it and adds 2 u, the
    fit is off by 1.5 u, t by 4 u and the two products by u each: u (1.5 z^2 + 190) of h in all. Above 0 the difference and
    the product add 2 u. Below 2^-126 results may be 0."""
    z = z.double()
    h = 0.5 * torch.special.erfc(z.abs() * 0.5 ** 0.5)
    y = z * torch.where(z < 0, h, 1 - h)
    return y, z.abs() * (h * U * (1.5 * z.clamp(-40, 40) ** 2 + 190) + 2.0 ** -126) + 3 * U * y.abs()


@pytest.mark.parametrize("rows", [2, 300, 6000])
def test_tail_of_a_product(rows):
    """The bias under sums of zero: its activation."""
    z = torch.cat([torch.linspace(-14, 14, 28 * 128), torch.linspace(-1, 1, 512), torch.linspace(-60, 60, 256),
                   torch.logspace(-30, 15, 128), -torch.logspace(-30, 15, 128)]).cuda()
    n, K = z.numel(), 16
    zero = torch.zeros((max(rows, n), K), dtype=torch.int8, device="cuda")
    y = rf.rf_frame_linear_i8(zero[:rows], torch.ones(rows, device="cuda"), zero[:n], torch.ones(n, device="cuda"), z, "gelu")
    want, err = bound(z)
    block.assert_within(y, want.expand(rows, n), err.expand(rows, n))


@pytest.mark.parametrize("M,N", [(1, 9), (2, 3000)])
def test_tail_of_a_norm(M, N):
    """The bias of constant groups: its activation, in the norm of one launch and of more."""
    z = torch.cat([torch.linspace(-14, 14, 1792), torch.linspace(-1, 1, 256)]).cuda()
    x = torch.ones((M * N, z.numel()), device="cuda")
    y = rf.rf_frame_group_norm(x, 32, None, z, activation="gelu", frame_ids=range(M), T=M, rows_per_frame=N)
    want, err = bound(z)
    block.assert_within(y, want.expand(*x.shape), err.expand(*x.shape))
