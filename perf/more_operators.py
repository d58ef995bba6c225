"""The backward pass of training with learned groups, as measurable cases: plain forms and the framework's kernels.

* ``attn``    ``focus_attn_bwd``: from the gradient of the attention's output those of queries, keys and values, under the hard mask
              (window or a shared group) or over every causal pair.  The probabilities are worked out again from ``lse``.
* ``gate``    ``focus_gate_attn_bwd``: the same for the training-time gate (a distant pair's score times sigmoid(lambda g_i . g_j)), with
              the gradient of the soft assignments g.
* ``router``  ``focus_router_scores_bwd``: from the gradient of the scores (W_g h) . C those of h, W_g and C.
* ``clip``    ``focus_grad_clip``: the norm over all gradients of a model, and the gradients scaled where it is above a bound.

``own`` says which of the two ``run`` computes.  The plain forms are elementary torch in 32 bits; ``exact`` computes the same in 64 bits
and on its own.  What the forward pass left behind (o rounded to bf16, lse in fp32) is an input of the backward pass.
"""
import math

import torch

own = False

#: head counts and dimension (query heads, KV heads, head dimension, softcap) of the workloads of inputs.py
HEADS = {"gpt2": (12, 12, 64, 0.0), "llama": (32, 8, 128, 0.0), "llama-shard": (8, 2, 128, 0.0), "gemma": (16, 8, 256, 50.0)}


def _attn(name, heads, n, batch=1, K=4, topk=2, window=None, runs=0):
    """window None: every causal pair.  runs: mean length of the stretches of tokens that keep their groups (0: every token its own)"""
    Hq, Hkv, D, cap = HEADS[heads]
    return {"name": name, "kind": "attn", "Hq": Hq, "Hkv": Hkv, "D": D, "softcap": cap, "n": n, "batch": batch, "K": K, "topk": topk, "window": window, "runs": runs}


def _gate(name, heads, n, K, window, batch=1, lam=10.0):
    Hq, Hkv, D, _ = HEADS[heads]
    return {"name": name, "kind": "gate", "Hq": Hq, "Hkv": Hkv, "D": D, "n": n, "batch": batch, "K": K, "window": window, "lam": lam}


def _router(name, n, d_model, d_g, K, batch=1):
    return {"name": name, "kind": "router", "n": n, "d_model": d_model, "d_g": d_g, "K": K, "batch": batch}


def _clip(name, what, layers, d_model, d_g=16, K=4, bound=1.0):
    return {"name": name, "kind": "clip", "what": what, "layers": layers, "d_model": d_model, "d_g": d_g, "K": K, "bound": bound}


def listed():
    return [
        # one short sequence, small heads: where launches and the first tile's way through the kernel count
        _attn("attn-gpt2-1k", "gpt2", 1024, K=4, topk=2, window=64),
        # a training sequence of the usual length, every token with groups of its own
        _attn("attn-llama-8k", "llama", 8192, K=4, topk=2, window=512),
        # the same with topics that persist: most distant tiles hold no pair
        _attn("attn-llama-8k-runs", "llama", 8192, K=8, topk=1, window=512, runs=512),
        # a batch of odd length, every causal pair (the layers that are not grouped)
        _attn("attn-dense-odd", "llama", 1021, batch=3),
        # one rank's heads of a long sequence, every causal pair
        _attn("attn-dense-16k", "llama-shard", 16384),
        # head dimension 256 with logit softcap, one group a token
        _attn("attn-gemma-4k", "gemma", 4096, K=4, topk=1, window=1024),
        # training the groups on a small model: a batch of sequences of 1000 tokens
        _gate("gate-gpt2-1000", "gpt2", 1000, 4, 64, batch=4),
        # training the groups on a large one
        _gate("gate-llama-4k", "llama", 4096, 8, 512),
        # the router of a small model: latency
        _router("router-gpt2-1k", 1024, 768, 16, 4),
        # the router of a large one over a long sequence
        _router("router-llama-32k", 32768, 4096, 16, 8),
        # only centroids and projections are trained: many small gradients
        _clip("clip-routers-12", "router", 12, 768),
        # everything is trained: the attention weights of eight layers beside their routers
        _clip("clip-layers-8", "layer", 8, 4096, K=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the kinds in the proportion of the listed ones, lengths over their whole range"""
    kind = rng.choice(["attn", "attn", "attn", "attn", "gate", "gate", "router", "router", "clip", "clip"])
    if kind == "attn":
        heads = rng.choice(["gpt2", "llama", "llama", "llama-shard", "gemma"])
        Hq, _, D, _ = HEADS[heads]
        # (a token that attends itself alone has gradients of q and k that are zero but for rounding: where all tokens do, there is
        # nothing to compare)
        n = _log_int(rng, 2, min(16384, math.isqrt((1 << 38) // (Hq * D))))
        batch = min(rng.randint(1, 6), max(1, (1 << 38) // (Hq * D * n * n)))
        K, topk = rng.choice([(4, 1), (4, 2), (8, 1), (8, 2), (16, 2), (32, 3)])
        c = _attn("", heads, n, batch, K, topk, rng.choice([None, 0 if n >= 64 else 16, 64, 512, 2048]), rng.choice([0, 0, 256, 512]))
    elif kind == "gate":
        heads, K = rng.choice([("gpt2", 4), ("gpt2", 32), ("llama", 4), ("llama", 8), ("llama-shard", 16), ("llama", 7), ("gemma", 8)])
        Hq, _, D, _ = HEADS[heads]
        n = _log_int(rng, 2, min(8192, math.isqrt((1 << 36) // (Hq * D))))
        batch = min(rng.randint(1, 6), max(1, (1 << 36) // (Hq * D * n * n)))
        c = _gate("", heads, n, K, rng.choice([0, 64, 512]), batch, rng.choice([5.0, 10.0, 30.0]))
    elif kind == "router":
        d_model, n = 8 * _log_int(rng, 8, 512), _log_int(rng, 1, 32768)
        c = _router("", n, d_model, rng.choice([8, 16, 32, 128]), rng.choice([3, 4, 8, 16, 32]), min(rng.randint(1, 4), max(1, 32768 // n)))
    else:
        c = _clip("", rng.choice(["router", "layer"]), rng.randint(1, 8), _log_int(rng, 64, 4096), rng.choice([8, 16, 32]), rng.choice([4, 8]),
                  rng.choice([1.0, 1.0, 1e9]))
    return {k: v for k, v in c.items() if k != "name"}


def _ld(K):
    """row length of scores and assignments"""
    return 4 if K <= 4 else 8 if K <= 8 else 16 if K <= 16 else 32


def _masks(B, H, n, K, topk, runs, gen):
    """membership masks int32 [B * H, n]: topk of K groups at random, for every token or for whole stretches of tokens (those of all heads)"""
    if runs:
        first = torch.rand((B, 1, n), generator=gen, device="cuda") < 1.0 / runs
        stretch = first.int().cumsum(-1)
        pick = torch.rand((B, 1, n, K), generator=gen, device="cuda")
        pick = pick.gather(2, stretch[..., None].long().clamp(max=n - 1).expand(-1, -1, -1, K)).expand(B, H, n, K)
    else:
        pick = torch.rand((B, H, n, K), generator=gen, device="cuda")
    member = pick.argsort(-1) < topk
    return (member.int() << torch.arange(K, device="cuda", dtype=torch.int32)).sum(-1).to(torch.int32).reshape(B * H, n)


def _gradient_shapes(case):
    """(shape, type) of the gradients of a clip case"""
    d = case["d_model"]
    router = [((d, case["d_g"]), torch.float32), ((case["K"], case["d_g"]), torch.float32)]
    if case["what"] == "router":
        return router * case["layers"]
    kv = max(1, d // 4)
    return [((d, d), torch.bfloat16), ((2 * kv, d), torch.bfloat16), ((d, d), torch.bfloat16), ((d,), torch.float32)] * case["layers"] + router * case["layers"]


def prepare(case, seed):
    kind = case["kind"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    empty = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")
    s = {"case": case}
    if kind in ("attn", "gate"):
        n, B, Hq, Hkv, D, K = (case[x] for x in ("n", "batch", "Hq", "Hkv", "D", "K"))
        # token by token, as a projection leaves them
        for x, H in (("q", Hq), ("k", Hkv), ("v", Hkv), ("do", Hq)):
            s[x] = randn(B, n, H, D).to(torch.bfloat16).transpose(1, 2)
        if kind == "gate":
            s["g"] = torch.zeros((B, n, _ld(K)), device="cuda")
            s["g"][..., :K] = torch.softmax(3.0 * randn(B, n, K), -1)
        elif case["window"] is not None:
            s["mq"] = _masks(B, Hq, n, K, case["topk"], case["runs"], gen)
            # (with stretches, keys have the groups of the queries)
            s["mk"] = s["mq"].view(B, Hq, n)[:, :Hkv].reshape(B * Hkv, n).contiguous() if case["runs"] else _masks(B, Hkv, n, K, case["topk"], 0, gen)
        s["o"], s["lse"] = empty(B, Hq, n, D), empty(B, Hq, n, dtype=torch.float32)
        _forward(s)
        for x, like in (("dq", "q"), ("dk", "k"), ("dv", "v")):
            s[x] = torch.empty_like(s[like])
        if kind == "gate":
            s["dg"] = torch.empty_like(s["g"])
    elif kind == "router":
        n, B, K, d, dg = (case[x] for x in ("n", "batch", "K", "d_model", "d_g"))
        s["h"] = randn(B, n, d).to(torch.bfloat16)
        s["Wg"], s["C"] = randn(d, dg) / math.sqrt(d), randn(K, dg)
        s["ds"] = torch.zeros((B, n, _ld(K)), device="cuda")
        s["ds"][..., :K] = 1e-3 * randn(B, n, K)
        s["dh"], s["dWg"], s["dC"] = torch.empty_like(s["h"]), torch.empty_like(s["Wg"]), torch.empty_like(s["C"])
    else:
        s["grads"] = [(1e-2 * randn(*shape)).to(dtype) for shape, dtype in _gradient_shapes(case)]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        s["norm"] = empty(1, dtype=torch.float32)
    if own:
        from paper_2604_03260_b200 import binding as fb
        s["status"] = torch.zeros(4, dtype=torch.int32, device="cuda")
        if kind == "clip":
            s["list"] = fb.make_grad_list(s["grads"], s["out"])
            s["ws"] = empty(fb.focus_grad_clip_workspace_bytes(), dtype=torch.uint8)
            return s
        Hq, Hkv, D = (case.get(x, v) for x, v in (("Hq", 1), ("Hkv", 1), ("D", 64)))
        s["shape"] = fb.make_shape(Hq, Hkv, case["n"], D, case["K"], case.get("topk", 1), case.get("window") or 0, 0.0, case.get("softcap", 0.0), batch=case["batch"])
        if kind == "router":
            size = fb.focus_router_scores_bwd_workspace_bytes(s["shape"], case["d_model"], case["d_g"])
        elif kind == "gate":
            size = fb.focus_gate_attn_bwd_workspace_bytes(s["shape"])
        else:
            size = fb.focus_attn_bwd_workspace_bytes(s["shape"])
            s["tiles"] = None
            if "mq" in s:                                    # the forward pass has them
                s["tiles"] = fb.alloc_workspace(s["shape"], fb.FOCUS_LAYOUT_ORIGINAL)
                fb.focus_build_tiles(s["shape"], s["mq"], s["mk"], fb.FOCUS_LAYOUT_ORIGINAL, s["tiles"])
        s["ws"] = empty(size, dtype=torch.uint8)
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2604_03260_b200 import binding as fb
        if kind == "attn":
            fb.focus_attn_bwd(s["shape"], s["q"], s["k"], s["v"], s.get("mq"), s.get("mk"), s["tiles"], fb.FOCUS_LAYOUT_ORIGINAL, s["o"], s["lse"], s["do"],
                              s["dq"], s["dk"], s["dv"], s["ws"], s["status"])
            return {x: s[x] for x in ("dq", "dk", "dv")}
        if kind == "gate":
            fb.focus_gate_attn_bwd(s["shape"], s["q"], s["k"], s["v"], s["g"], s["case"]["lam"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], s["dg"],
                                   s["ws"], s["status"])
            return {x: s[x] for x in ("dq", "dk", "dv", "dg")}
        if kind == "router":
            fb.focus_router_scores_bwd(s["shape"], s["h"], s["Wg"], s["C"], s["ds"], s["dh"], s["dWg"], s["dC"], s["ws"])
            return {x: s[x] for x in ("dh", "dWg", "dC")}
        fb.focus_grad_clip(s["list"], s["case"]["bound"], s["norm"], s["ws"])
        return {"norm": s["norm"], "grads": s["out"]}
    if kind in ("attn", "gate"):
        return _attn_bwd(s)
    if kind == "router":
        return _router_bwd(s)
    return _clipped(s)


# ---- plain forms

def _rows(s, x):
    """[B, Hq, n, D] or [B, Hkv, n, D] in fp32, the query heads of a KV head in an axis of their own"""
    c, t = s["case"], s[x].float()
    return t.unflatten(1, (c["Hkv"], -1))


def _keep(s):
    """which pairs are attended: bool [B, Hkv, G, n, n], or [n, n] where only causality counts"""
    c, n = s["case"], s["case"]["n"]
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")
    causal = j <= i
    if "mq" not in s:
        return causal
    B, Hkv = c["batch"], c["Hkv"]
    shared = (s["mq"].view(B, Hkv, -1, n, 1) & s["mk"].view(B, Hkv, 1, 1, n)) != 0
    return shared.logical_or_(i - j <= c["window"]).logical_and_(causal)


def _factor(s):
    """the gate's factor of every pair, [B, 1, 1, n, n]"""
    c, n = s["case"], s["case"]["n"]
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")
    f = torch.sigmoid(c["lam"] * (s["g"] @ s["g"].transpose(1, 2)))
    return f.masked_fill_(i - j <= c["window"], 1.0)[:, None, None]


def _forward(s):
    """o and lse of the forward pass"""
    c = s["case"]
    k, v, q = _rows(s, "k"), _rows(s, "v"), _rows(s, "q")
    x = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(c["D"]))
    if c["kind"] == "gate":
        x.mul_(_factor(s))
    elif c["softcap"]:
        x.mul_(1.0 / c["softcap"]).tanh_().mul_(c["softcap"])
    x.masked_fill_(~_keep(s), -math.inf)
    m = x.amax(-1, keepdim=True)
    l = x.sub_(m).exp_().sum(-1, keepdim=True)
    s["o"].copy_(((x @ v) / l).flatten(1, 2))
    s["lse"].copy_((m + torch.log(l)).flatten(1, 2)[..., 0])


def _attn_bwd(s):
    """With x = scale q k (times a factor, or capped), p = exp(x - lse), dp = do v, ds = p (dp - rowsum(do o)): dv = p do, dq = scale ds k,
    dk = scale ds q, those of the query heads of a KV head added up."""
    c = s["case"]
    B, n, scale = c["batch"], c["n"], 1.0 / math.sqrt(c["D"])
    q, k, v, o, do = (_rows(s, x) for x in ("q", "k", "v", "o", "do"))
    x = (q @ k.transpose(-1, -2)).mul_(scale)
    p, cap = x, None
    if c["kind"] == "gate":
        factor = _factor(s)
        p = x * factor
    elif c["softcap"]:
        cap = x.mul_(1.0 / c["softcap"]).tanh_()
        p = cap * c["softcap"]
    p = p.sub_(s["lse"].unflatten(1, (c["Hkv"], -1))[..., None]).exp_().masked_fill_(~_keep(s), 0.0)
    out = {"dv": (p.transpose(-1, -2) @ do).sum(2)}
    ds = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    del p
    if c["kind"] == "gate":
        # the factor's gradient is ds x summed over heads, and sigmoid' = f (1 - f); pairs inside the window have none
        i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")
        da = x.mul_(ds).sum((1, 2)).mul_((c["lam"] * factor * (1.0 - factor))[:, 0, 0]).masked_fill_(i - j <= c["window"], 0.0)
        out["dg"] = da @ s["g"] + da.transpose(1, 2) @ s["g"]
        ds.mul_(factor)
    elif cap is not None:
        ds.mul_(1.0 - cap * cap)
    out["dq"] = (ds @ k).mul_(scale).flatten(1, 2)
    out["dk"] = (ds.transpose(-1, -2) @ q).mul_(scale).sum(2)
    return {x: t.to(s[x].dtype) for x, t in out.items()}


def _router_bwd(s):
    K = s["case"]["K"]
    ds, h = s["ds"][..., :K].flatten(0, 1), s["h"].float().flatten(0, 1)
    u, du = h @ s["Wg"], ds @ s["C"]
    return {"dh": (du @ s["Wg"].T).to(torch.bfloat16).view_as(s["h"]), "dWg": h.T @ du, "dC": ds.T @ u}


def _clipped(s):
    # (long sums: each tensor's in 64 bits)
    squares = torch.stack([g.double().square().sum() for g in s["grads"]])
    norm = squares.sum().sqrt()
    factor = torch.where(norm > s["case"]["bound"], s["case"]["bound"] / norm, 1.0).float()
    return {"norm": norm.float().view(1), "grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


def work(case):
    kind = case["kind"]
    if kind == "clip":
        # read, and once more where they are scaled and copied
        sizes = [(math.prod(shape), 2 if dtype == torch.bfloat16 else 4) for shape, dtype in _gradient_shapes(case)]
        return {"bytes": float(sum(2 * c * b for c, b in sizes)), "flops": float(sum(3 * c for c, _ in sizes))}
    n, B, K = (case[x] for x in ("n", "batch", "K"))
    if kind == "router":
        d, dg = case["d_model"], case["d_g"]
        # h and the scores' gradient read, dh written, the weights both; T = ds' h and dh = ds (C W') are products with K columns
        return {"bytes": 4.0 * B * n * d + 4.0 * B * n * _ld(K) + 8.0 * (d * dg + K * dg), "flops": 4.0 * B * n * d * K + 6.0 * K * d * dg}
    Hq, Hkv, D = (case[x] for x in ("Hq", "Hkv", "D"))
    w = n if case["window"] is None else min(n, case["window"] + 1)
    local = w * (w + 1) / 2 + (n - w) * w
    far = n * (n + 1) / 2 - local
    # q, o, do read and dq written; k, v read and dk, dv written; lse
    b = B * n * (8.0 * Hq * D + 8.0 * Hkv * D + 4.0 * Hq)
    if kind == "gate":
        # five products of D, and per distant pair the product of assignments and two sums of their gradients
        return {"bytes": b + 8.0 * B * n * _ld(K), "flops": B * Hq * (10.0 * D * (local + far) + 6.0 * K * far)}
    if case["window"] is not None:
        b += 4.0 * B * n * (Hq + Hkv)
        far *= 1.0 - math.comb(K - case["topk"], case["topk"]) / math.comb(K, case["topk"])
    return {"bytes": b, "flops": B * Hq * 10.0 * D * (local + far)}


# ---- the same in 64 bits

def _exact_head(s, b, h, hk, out):
    """adds what query head h contributes to the gradients of sequence b"""
    c, n = s["case"], s["case"]["n"]
    scale = c["D"] ** -0.5
    q, o, do = (s[x][b, h].double() for x in ("q", "o", "do"))
    k, v = (s[x][b, hk].double() for x in ("k", "v"))
    delta, lse = torch.einsum("id,id->i", do, o), s["lse"][b, h].double()
    # blocks of rows, the columns up to the block's last row
    step = max(1, min(n, (1 << 26) // n))
    for r0 in range(0, n, step):
        r1 = min(n, r0 + step)
        rows, cols = torch.arange(r0, r1, device="cuda")[:, None], torch.arange(r1, device="cuda")[None]
        near = rows - cols <= (n if c["window"] is None else c["window"])
        raw = torch.einsum("id,jd->ij", q[r0:r1], k[:r1]) * scale
        seen, slope, logit = cols <= rows, None, raw
        if c["kind"] == "gate":
            z = c["lam"] * torch.einsum("ik,jk->ij", s["g"][b, r0:r1].double(), s["g"][b, :r1].double())
            open_ = 1.0 / (1.0 + torch.exp(-z))
            slope = torch.where(near, 1.0, open_)
            logit = raw * slope
        elif c["softcap"]:
            t = torch.tanh(raw / c["softcap"])
            logit, slope = c["softcap"] * t, 1.0 - t ** 2
        if "mq" in s:
            mq, mk = s["mq"].view(c["batch"], -1, n)[b, h, r0:r1], s["mk"].view(c["batch"], -1, n)[b, hk, :r1]
            seen = seen & (near | ((mq[:, None] & mk[None]) != 0))
        p = torch.where(seen, torch.exp(logit - lse[r0:r1, None]), 0.0)
        out["dv"][b, hk, :r1] += torch.einsum("ij,id->jd", p, do[r0:r1])
        dx = p * (torch.einsum("id,jd->ij", do[r0:r1], v[:r1]) - delta[r0:r1, None])
        if c["kind"] == "gate":
            da = torch.where(near, 0.0, dx * raw * c["lam"] * open_ * (1.0 - open_))
            out["dg"][b, r0:r1] += torch.einsum("ij,jk->ik", da, s["g"][b, :r1].double())
            out["dg"][b, :r1] += torch.einsum("ij,ik->jk", da, s["g"][b, r0:r1].double())
        if slope is not None:
            dx = dx * slope
        out["dq"][b, h, r0:r1] = torch.einsum("ij,jd->id", dx, k[:r1]) * scale
        out["dk"][b, hk, :r1] += torch.einsum("ij,id->jd", dx, q[r0:r1]) * scale


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        total = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
        by = min(1.0, case["bound"] / total)
        return {"norm": torch.tensor([total], dtype=torch.float64), "grads": [g.double() * by for g in s["grads"]]}
    if kind == "router":
        K = case["K"]
        h, Wg, C = (s[x].double().requires_grad_() for x in ("h", "Wg", "C"))
        scores = torch.einsum("bnd,de,ke->bnk", h, Wg, C)
        dh, dWg, dC = torch.autograd.grad(scores, (h, Wg, C), s["ds"][..., :K].double())
        return {"dh": dh, "dWg": dWg, "dC": dC}
    out = {x: torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in (("dq", "dk", "dv", "dg") if kind == "gate" else ("dq", "dk", "dv"))}
    for b in range(case["batch"]):
        for h in range(case["Hq"]):
            _exact_head(s, b, h, h // (case["Hq"] // case["Hkv"]), out)
    return out
