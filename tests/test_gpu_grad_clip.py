"""focus_grad_clip against the same in 64 bits."""
import math

import pytest
import torch

from paper_2604_03260_b200 import binding as fb

pytestmark = pytest.mark.gpu


def tensors(sizes, seed=0, scale=1.0):
    """of both types in turn, contiguous, at any multiple of a number's size from an aligned place"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        x = (scale * torch.randn(n + 5, generator=gen, device="cuda")).to(torch.bfloat16 if i % 2 else torch.float32)
        out.append(x[i % 5:i % 5 + n])
    return out


def clip(grads, bound, out=None, stream=None):
    norm = torch.full((1,), -1.0, device="cuda")
    ws = torch.empty(fb.focus_grad_clip_workspace_bytes(), dtype=torch.uint8, device="cuda").fill_(0xff)
    fb.focus_grad_clip(fb.make_grad_list(grads, out), bound, norm, ws, stream)
    torch.cuda.synchronize()
    return norm.item()


def check(grads, bound):
    want = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))
    before = [g.clone() for g in grads]
    out = [torch.full_like(g, math.nan) for g in grads]
    norm = clip(grads, bound, out)
    # sums of squares in fp32 in pieces, joined in 64 bits, half of whose relative error the root keeps; then one rounding
    assert abs(norm - want) <= want * 2.0 ** -22
    by = bound / want if want > bound else 1.0
    for g, x, b in zip(grads, out, before):
        assert torch.equal(g, b)
        if by == 1.0:
            assert torch.equal(x, g)
        else:
            u = 2.0 ** -8 if g.dtype == torch.bfloat16 else 2.0 ** -23     # (factor and product rounded to fp32)
            tiny = 2.0 ** -133 if g.dtype == torch.bfloat16 else 2.0 ** -149
            assert ((x.double() - g.double() * by).abs() <= u * 1.001 * (g.double() * by).abs() + tiny + g.double().abs() * by * 2.0 ** -22).all()
    assert clip(grads, bound) == norm                            # in place
    assert all(torch.equal(g, x) for g, x in zip(grads, out))


@pytest.mark.parametrize("sizes", [[1], [0], [], [7, 0, 3], [8192, 8193, 8191, 16384], [100000, 3, 65537], [1] * 350, list(range(1, 260)), [5000001, 12]])
@pytest.mark.parametrize("bound", [0.5, 1e9])
def test_sizes(sizes, bound):
    check(tensors(sizes), bound)


def test_matrices_and_a_bound_of_nothing():
    g = [torch.randn((33, 65), device="cuda"), torch.randn((4, 3, 2), device="cuda").to(torch.bfloat16)]
    check([x.clone() for x in g], 1.0)
    clip(g, 0.0)
    assert all((x == 0).all() for x in g)


def test_infinite_bound_scales_nothing():
    g = tensors([1000, 1000], scale=1e6)
    check(g, math.inf)


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e25, 1e35])
def test_squares_beyond_fp32(scale):
    check(tensors([3000, 500, 70000], scale=scale), 0.25 * scale)


def test_some_large_among_small():
    g = tensors([40000, 40000])
    g[0][17] = 1e25
    g[1][-1] = -3e24
    check(g, 1.0)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_is_reported_and_left(bad):
    g = tensors([5000, 5000, 30])
    g[1][4321] = bad
    before = [x.clone() for x in g]
    norm = clip(g, 1.0)
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    assert all(torch.equal(x.nan_to_num(), b.nan_to_num()) for x, b in zip(g, before))


def test_same_bits_captured_and_on_two_streams():
    a, b = tensors([100000, 999], 1), tensors([77777, 31, 5], 2)
    oa, ob = [torch.empty_like(x) for x in a], [torch.empty_like(x) for x in b]
    wa, wb = [torch.empty_like(x) for x in a], [torch.empty_like(x) for x in b]
    na, nb = clip(a, 1.0, wa), clip(b, 1.0, wb)
    ws = [torch.empty(fb.focus_grad_clip_workspace_bytes(), dtype=torch.uint8, device="cuda") for _ in range(2)]
    norms = [torch.zeros(1, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for g, o, w, n, st in ((a, oa, ws[0], norms[0], streams[0]), (b, ob, ws[1], norms[1], streams[1])):
        for _ in range(3):
            fb.focus_grad_clip(fb.make_grad_list(g, o), 1.0, n, w, st)
    torch.cuda.synchronize()
    assert norms[0].item() == na and norms[1].item() == nb and all(torch.equal(x, y) for x, y in zip(oa + ob, wa + wb))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.focus_grad_clip(fb.make_grad_list(a, oa), 1.0, norms[0], ws[0])
    a[0].mul_(2.0)
    want = clip(a, 1.0, wa)
    graph.replay()
    torch.cuda.synchronize()
    assert norms[0].item() == want and all(torch.equal(x, y) for x, y in zip(oa, wa))


def test_a_factor_below_normal_numbers_loses_nothing():
    check(tensors([60, 41], scale=3e37), 1e-3)


def test_a_norm_beyond_fp32_is_reported_so_and_left():
    g = [torch.full((1000,), 1e38, device="cuda")]
    assert clip(g, 1.0) == math.inf and (g[0] == 1e38).all()


def test_a_tensor_listed_twice_is_refused():
    x = torch.ones(8, device="cuda")
    with pytest.raises(AssertionError, match="twice"):
        fb.make_grad_list([x, x])
    fb.make_grad_list([x, x], [torch.empty_like(x) for _ in range(2)])
    fb.make_grad_list([torch.empty(0, device="cuda")] * 2)
