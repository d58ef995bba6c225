"""Norm and rotation over tensors of more than 2^31 numbers (4 GB): rows on both sides of 2^31 bytes and of 2^31 numbers from the start."""
import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from tests.test_gpu_rope import check, pair_size, reference, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rotary", [128, 70])                # (70: halves that are no whole 16 bytes)
@pytest.mark.parametrize("layout", ["token", "head"])
def test_offsets_past_32_bits(rotary, layout):
    Hq, Hkv, n, D = 40, 8, 350011, 128
    g = torch.Generator(device="cuda"); g.manual_seed(rotary)
    x = torch.randn((n, Hq + Hkv, D) if layout == "token" else (Hq + Hkv, n, D), generator=g, device="cuda", dtype=torch.bfloat16)
    assert x.numel() > 1 << 31
    heads = (lambda t: t.transpose(0, 1)) if layout == "token" else (lambda t: t)
    parts = lambda t: (heads(t)[None, :Hq], heads(t)[None, Hq:])
    y = torch.full_like(x, float("nan"))
    (q, k), (qo, ko) = parts(x), parts(y)
    # both keys and the queries' last heads lie past 2^31 numbers when the heads are apart, the last tokens when they are side by side
    wq, wk = (1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
    rope, freq = fb.make_rope(rotary), fb.focus_rope_frequencies(rotary)[0]
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16)
    fb.focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, None, qo, ko)
    edges = [e // D // (Hq + Hkv if layout == "token" else 1) for e in (1 << 30, 1 << 31)]
    rows = sorted({r for e in edges for r in range(e % n - 20, e % n + 20) if 0 <= r < n} | set(range(40)) | set(range(n - 40, n)))
    at = torch.tensor(rows, device="cuda")
    for a, b, w in ((q, qo, wq), (k, ko, wk)):
        check(b[:, :, at], reference(a[:, :, at], w, at[None], freq, rope))
    assert not torch.isnan(heads(y)[::7]).any()
    # the derivative, over the results
    ws = torch.empty(fb.focus_qk_norm_rope_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    want = [b[:, :, at].clone() for b in (qo, ko)]
    dwq, dwk = torch.empty_like(wq), torch.empty_like(wk)
    fb.focus_qk_norm_rope_bwd(shape, rope, q, k, wq, wk, freq, None, qo, ko, qo, ko, dwq, dwk, ws)
    for a, b, w, gy in ((q, qo, wq, want[0]), (k, ko, wk, want[1])):
        v = a[:, :, at].double()
        back = turned(gy.double(), at[None], freq, False, rotary, 1.0, -1.0)
        r = 1 / torch.sqrt(v.square().mean(-1, keepdim=True) + rope.eps)
        u, xhat = back * w.double(), v * r
        ref = r * (u - xhat * (u * xhat).mean(-1, keepdim=True))
        size = r * (pair_size(u) + pair_size(xhat) * (u * xhat).abs().mean(-1, keepdim=True))
        assert (b[:, :, at].double() - ref).abs().sub(2.0 ** -8 * ref.abs() + 2.0 ** -17 * size).max() <= 0
    assert not torch.isnan(heads(y)[::7]).any() and dwq.isfinite().all() and dwk.isfinite().all()
