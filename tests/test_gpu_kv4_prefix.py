"""A cached prefix through a pass of its own: norm and rotation, groups, append, read, tiles and focus_attn_fwd over what came out of the cache,
whose queries are those of all its tokens (focus_attn_fwd has one length for queries and keys); its last row against the decode step over the
same cache, all rows against the 64-bit oracle (tolerances of the forward pass)."""
import numpy as np
import pytest
import torch

from oracle import focus_oracle as fo
from paper_2604_03260_b200 import binding as fb
from paper_2604_03260_b200 import inputs as fi
from paper_2604_03260_b200.kv4_cache import Kv4Cache
from tests.gpu_util import LSE_MAX_ABS, O_MAX_ABS, O_MEAN_ABS, as_u32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,n,layout,cap", [(128, 700, 0, 0.0), (128, 1500, 1, 0.0), (64, 333, 3, 0.0), (256, 513, 0, 30.0)])
def test_read_then_a_pass_over_the_prefix(D, n, layout, cap):
    B, Hq, Hkv, K, topk, w = 2, 8, 2, 4, 1, 40
    g = torch.Generator(device="cuda"); g.manual_seed(D + n)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    shape = fb.make_shape(Hq, Hkv, n, D, K, topk, w, 0.0, cap, batch=B)
    layer = Kv4Cache(B, Hq, Hkv, D, K, topk, w, n + 5, 2 * (n // 32 + 1), 32, softcap=cap)
    qkv = rn(B, n, Hq + 2 * Hkv, D).to(torch.bfloat16)
    q, k, v = (t.transpose(1, 2) for t in qkv.split([Hq, Hkv, Hkv], 2))
    rope, freq = fb.make_rope(D), fb.focus_rope_frequencies(D)[0]
    wq, wk = (1 + 0.1 * rn(D) for _ in range(2))
    fb.focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, None, q, k)
    cent = rn(Hkv, K, D)
    mq, mk = torch.empty((B * Hq, n), dtype=torch.int32, device="cuda"), torch.empty((B * Hkv, n), dtype=torch.int32, device="cuda")
    fb.focus_assign(shape, q, Hq, cent, mq)
    fb.focus_assign(shape, k, Hkv, cent, mk)
    layer.append(k, v, mk)
    k4, v4 = (torch.empty((B, Hkv, n, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mk4 = torch.empty_like(mk)
    layer.read(k4, v4, mk4)
    assert torch.equal(mk4, mk)
    qc = q.contiguous()
    ws = fb.alloc_workspace(shape, layout)
    fb.focus_build_tiles(shape, mq, mk4, layout, ws)
    O, lse = torch.full_like(qc, float("nan")), torch.full((B * Hq, n), float("nan"), device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    fb.focus_attn_fwd(shape, qc, k4, v4, mq, mk4, ws, layout, O, lse, status)
    o1, lse1 = torch.empty((B, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty(B * Hq, device="cuda")
    layer.decode(qc[:, :, -1].contiguous(), mq[:, -1].contiguous(), o1, lse1)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * 4 and layer.status.tolist() == [0] * 4
    err = (O[:, :, -1].float() - o1.float()).abs()
    assert err.max() <= O_MAX_ABS and err.mean() <= O_MEAN_ABS and (lse[:, -1] - lse1).abs().max() <= LSE_MAX_ABS
    m, mkn = as_u32(mq).reshape(B, Hq, n), as_u32(mk).reshape(B, Hkv, n)
    for b in range(B):
        rows = np.array([(h, r) for h in range(Hq) for r in (0, 1, n // 2, n - 2, n - 1)])
        ref = fo.attn_rows(fi.bf16_bits(qc[b]), fi.bf16_bits(k4[b]), fi.bf16_bits(v4[b]), m[b], mkn[b], w, scale=D ** -0.5, softcap=cap, rows=rows)
        got = O[b].float().cpu().numpy()[rows[:, 0], rows[:, 1]]
        assert np.abs(got - ref["O"]).max() <= O_MAX_ABS and np.abs(lse.view(B, Hq, n)[b].cpu().numpy()[rows[:, 0], rows[:, 1]] - ref["lse"]).max() <= LSE_MAX_ABS
