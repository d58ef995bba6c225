"""focus_gate_attn_bwd: the same bits in every call, for each way in which a tile's assignments lie in shared memory (they are copied over while other
warps are at work), long enough that every place is used many times."""
import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from test_gpu_attn_bwd import make, run_bwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [3100, 900])
@pytest.mark.parametrize("B,Hq,Hkv,D", [(1, 4, 2, 64), (1, 4, 2, 128), (1, 4, 4, 64), (1, 4, 4, 128)])
@pytest.mark.parametrize("K", [4, 8, 16, 32])
def test_same_bits(B, Hq, Hkv, n, D, K):
    t, gen = make(B, Hq, Hkv, n, D, K)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, 64, batch=B)
    g = torch.zeros((B, n, fb.focus_soft_ld(K)), device="cuda")
    g[..., :K] = torch.softmax(torch.randn((B, n, K), generator=gen, device="cuda"), -1)
    t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty((B, Hq, n), device="cuda")
    fb.focus_gate_attn_fwd(shape, t["q"], t["k"], t["v"], g, 5.0, t["o"], t["lse"])
    first = run_bwd(shape, t, g=g, lam=5.0)
    for _ in range(12):
        again = run_bwd(shape, t, g=g, lam=5.0)
        assert all(torch.equal(first[x], again[x]) for x in first)
