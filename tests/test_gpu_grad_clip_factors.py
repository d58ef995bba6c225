"""focus_grad_clip with factors far below fp32's normal numbers: what large numbers become is right to fp32's last bit all the same."""
import pytest
import torch

from test_gpu_grad_clip import check, clip, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bound", [1e-17, 1e-19, 1e-20, 1e-23, 1e-25, 1e-27, 1e-30, 1e-36, 1e-39, 1e-43, 0.0])
@pytest.mark.parametrize("sizes", [[60, 41], [1, 0, 9000, 33]])
def test_factors(sizes, bound):
    check(tensors(sizes, scale=1e36), bound)


def test_each_number_is_rounded_once():
    """half a step of fp32, and what the norm is off; no number becomes zero"""
    g = [1e36 * torch.randn(5000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))]
    for bound in (1e-22, 1e-26, 1e-30):
        out = [torch.empty_like(g[0])]
        clip(g, bound, out)
        norm = g[0].double().square().sum().sqrt()
        by = torch.tensor(bound, dtype=torch.float32).double().item() / norm
        # (the kernel's norm is off by at most 2^-22 of itself)
        assert ((out[0].double() - g[0].double() * by).abs() <= (2.0 ** -24 + 2.0 ** -22) * (g[0].double() * by).abs()).all()
        assert (out[0] != 0).all()


def test_other_alignment_than_the_source():
    x = tensors([1000], scale=1e36)[0]
    buf = torch.full((1003,), 5.0, device="cuda")
    clip([x], 1e-28, [buf[1:1001]])
    by = torch.tensor(1e-28, dtype=torch.float32).double().item() / x.double().norm()
    assert ((buf[1:1001].double() - x.double() * by).abs() <= (2.0 ** -24 + 2.0 ** -22) * (x.double() * by).abs()).all()
    assert buf[0] == 5.0 and (buf[1001:] == 5.0).all()
