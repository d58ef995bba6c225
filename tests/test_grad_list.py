"""make_grad_list refuses lists in which what is written overlaps something else (no GPU needed: on stand-ins for its tensors)."""
import pytest
import torch

from paper_2604_03260_b200 import binding as fb


class OnGpu:
    """a CPU tensor that says it is on the GPU"""
    def __init__(self, t):
        self.t = t

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)


def tensors(dtype=torch.float32):
    base = torch.zeros(1000, dtype=dtype)
    return base, lambda lo, hi: OnGpu(base[lo:hi])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_overlaps(dtype):
    base, at = tensors(dtype)
    other, to = tensors(dtype)
    for grads, out in (([at(0, 100), at(99, 200)], None), ([at(50, 60), at(0, 1000)], None), ([at(0, 1000), at(999, 1000)], None),       # in place
                       ([at(0, 100)], [at(1, 101)]), ([at(1, 101)], [at(0, 100)]),                                                      # over itself, shifted
                       ([at(0, 100), at(100, 200)], [to(0, 100), at(50, 150)]), ([at(0, 10), at(20, 30)], [at(20, 30), to(0, 10)]),     # over another's source
                       ([at(0, 10), at(20, 30)], [to(0, 10), to(9, 19)]), ([at(0, 10), at(20, 30)], [to(9, 19), to(0, 10)])):           # over another's result
        with pytest.raises(AssertionError, match="over another"):
            fb.make_grad_list(grads, out)
    with pytest.raises(AssertionError, match="twice"):
        fb.make_grad_list([at(3, 9), at(3, 9)])


def test_pieces_of_one_buffer():
    base, at = tensors()
    other, to = tensors()
    pieces = [at(0, 1), at(1, 400), at(400, 400), at(400, 401), at(401, 1000)]
    assert fb.make_grad_list(pieces).count == 5 and fb.make_grad_list(pieces[::-1]).count == 5
    assert fb.make_grad_list(pieces, [to(0, 1), to(1, 400), to(400, 400), to(400, 401), to(401, 1000)]).count == 5
    # the same source twice, or overlapping sources, into places of their own
    assert fb.make_grad_list([at(0, 10), at(0, 10), at(5, 9)], [to(0, 10), to(10, 20), to(30, 34)]).count == 3
    assert fb.make_grad_list([], []).count == 0


def test_tensors_of_several_devices():
    """(one kernel reads them all)"""
    a, b = (OnGpu(torch.zeros(4)) for _ in range(2))
    assert fb.make_grad_list([a, b]).count == 2
    b.device = torch.device("cuda", 1)
    with pytest.raises(AssertionError, match="devices"):
        fb.make_grad_list([a, b])
