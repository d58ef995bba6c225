"""The operators around a 4-bit cache of an attention layer, as measurable cases: plain forms and the framework's kernels.

* ``rope``      ``focus_qk_norm_rope``: the projections' query and key vectors are normalised head by head and turned by their
                positions, before the groups are assigned and attention reads them.
* ``rope_bwd``  ``focus_qk_norm_rope_bwd``: the gradients of the vectors and of the two norm weights.
* ``store``     ``focus_kv4_append``, then ``focus_kv4_read``: keys, values and key masks go into the pages of the 4-bit cache and
                come back as the values that the codes stand for.
* ``decode``    ``focus_kv4_decode_step``: one new query per sequence against its pages, under the rule of ``focus_decode_step``.
* ``copy``      ``focus_kv4_copy_pages``: pages copied to other pages (a sequence forked, a pool compacted).

``own`` says which of the two ``run`` computes.  The plain forms are elementary torch in 32 bits (angles in 64); ``exact`` computes
the same in 64 bits and on its own.

A page of the cache holds ``P`` tokens of all KV heads: ``[Hkv][P]`` rows of ``D`` bytes (4-bit codes of the key, then of the value,
two dimensions a byte, the even one in the low bits), ``[Hkv][P]`` rows of ``D / 8`` bytes (8-bit scales of blocks of 16 dimensions,
key then value), ``[Hkv][P]`` 32-bit masks.  A code is sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6; a scale is an 8-bit float with
four exponent bits, amax / 6 of its block rounded to nearest; ``k_scale`` and ``v_scale`` are powers of two on top.
"""
import math

import torch

own = False

#: head counts and dimension (query heads, KV heads, head dimension, softcap) of the workloads of inputs.py
HEADS = {"gpt2": (12, 12, 64, 0.0), "llama": (32, 8, 128, 0.0), "gemma": (16, 8, 256, 50.0)}
K_SCALE, V_SCALE = 1.0, 0.5
EPS = 1e-6


def _rope(name, heads, n, batch=1, bwd=False, rotary=1.0, interleaved=False, norm=True, base=500000.0, factor=1.0, first=0):
    Hq, Hkv, D, _ = HEADS[heads]
    return {"name": name, "kind": "rope_bwd" if bwd else "rope", "Hq": Hq, "Hkv": Hkv, "D": D, "n": n, "batch": batch, "rotary": int(rotary * D),
            "interleaved": interleaved, "norm": norm, "base": base, "factor": factor, "first": first}


def _store(name, heads, n, batch=1, page=64, first=0):
    Hq, Hkv, D, _ = HEADS[heads]
    return {"name": name, "kind": "store", "Hq": Hq, "Hkv": Hkv, "D": D, "n": n, "batch": batch, "page": page, "first": first}


def _decode(name, heads, n, K, topk, window, batch=1, page=64, ragged=False):
    Hq, Hkv, D, cap = HEADS[heads]
    return {"name": name, "kind": "decode", "Hq": Hq, "Hkv": Hkv, "D": D, "softcap": cap, "n": n, "K": K, "topk": topk, "window": window,
            "batch": batch, "page": page, "ragged": ragged}


def _copy(name, heads, count, page, pool):
    Hq, Hkv, D, _ = HEADS[heads]
    return {"name": name, "kind": "copy", "Hq": Hq, "Hkv": Hkv, "D": D, "n": 1, "batch": 1, "page": page, "count": count, "pool": pool}


def listed():
    return [
        # a generation step of 16 sequences deep in their contexts: latency
        _rope("rope-step-16", "llama", 1, batch=16, first=120000),
        # a prompt: norm and whole-head rotation, as the attention pass wants it next
        _rope("rope-llama-8k", "llama", 8192),
        # training, the layer's gradients through norm and rotation
        _rope("rope-bwd-llama-8k", "llama", 8192, bwd=True),
        # training, odd lengths in a batch, part of a small head rotated in interleaved pairs, positions stretched for a long context
        _rope("rope-bwd-gpt2-odd", "gpt2", 1021, batch=3, bwd=True, rotary=0.5, interleaved=True, base=10000.0, factor=8.0),
        # one new token of each of 32 sequences goes into the cache: latency
        _store("store-step-32", "llama", 1, batch=32, first=5000),
        # the prompt's keys and values into the cache, and back for a pass over the cached prefix
        _store("store-llama-8k", "llama", 8192),
        # generation, one sequence with a short, odd cache: latency
        _decode("decode-llama-2k", "llama", 2049, 4, 2, 512),
        # serving: sequences of all lengths from one token to 16385 in one call
        _decode("decode-ragged-24", "llama", 16385, 4, 2, 2048, batch=24, ragged=True),
        # generation at the end of a long context
        _decode("decode-llama-128k", "llama", 131072, 4, 2, 2048),
        # head dimension 256 with logit softcap, top-1: half of the distant keys fall away
        _decode("decode-gemma-64k", "gemma", 65536, 4, 1, 4096, page=32),
        # 48 sequences forked: the page that each is writing to is copied
        _copy("copy-fork-48", "llama", 48, 64, 512),
        # a pool compacted: a thousand pages moved into the holes
        _copy("copy-compact-1024", "llama", 1024, 64, 4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the kinds in the proportion of the listed ones, lengths over their whole range"""
    kind = rng.choice(["rope", "rope", "rope_bwd", "rope_bwd", "store", "store", "decode", "decode", "decode", "decode", "copy"])
    heads = rng.choice(["gpt2", "llama", "llama", "gemma"])
    page = rng.choice([16, 32, 64, 128])
    if kind in ("rope", "rope_bwd"):
        n = _log_int(rng, 1, 8192)
        c = _rope("", heads, n, min(rng.randint(1, 24), max(1, 8192 // n)), kind == "rope_bwd", rng.choice([1.0, 1.0, 0.5, 0.25]), rng.random() < 0.4,
                  rng.random() < 0.8, rng.choice([10000.0, 500000.0]), rng.choice([1.0, 8.0]), rng.randint(0, 200000))
    elif kind == "store":
        n = _log_int(rng, 1, 8192)
        c = _store("", heads, n, min(rng.randint(1, 40), max(1, 8192 // n)), page, rng.randint(0, 5000))
    elif kind == "decode":
        n = _log_int(rng, 1, 65536)
        K, topk = rng.choice([(4, 1), (4, 2), (8, 1), (8, 2)])
        batch = min(rng.randint(1, 48), max(1, 65536 // n))
        c = _decode("", heads, n, K, topk, rng.choice([0, 64, 512, 2048]), batch, page, rng.random() < 0.6)
    else:
        count = _log_int(rng, 1, 512)
        c = _copy("", heads, count, page, 3 * count + rng.randint(0, 64))
    return {k: v for k, v in c.items() if k != "name"}


def _lens(case):
    """Cached tokens of every sequence, the new one among them: equal, or spread from 1 to n"""
    n, B = case["n"], case["batch"]
    if not case.get("ragged"):
        return [n] * B
    return [n] + [max(1, int(n * ((0.618034 * b) % 1.0) ** 2)) for b in range(1, B)]


def _page_bytes(case):
    return case["Hkv"] * case["page"] * (case["D"] + case["D"] // 8 + 4)


# ---- the 4-bit form, elementary

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _codes(x, scale):
    """codes [..., D] (0..15) and scales fp32 [..., D / 16] of x [..., D]; ties go to the code whose last bit is 0"""
    y = x.float().unflatten(-1, (-1, 16)) / scale
    # (in 64 bits: a division by a number may be a product with its reciprocal, and a scale half-way between two has to stay there)
    s = (y.abs().amax(-1).double() / 6.0).float().clamp(max=448.0).to(torch.float8_e4m3fn).float()
    y = torch.where(s[..., None] > 0, y / s[..., None], torch.zeros_like(y))
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int()
    return (code + 8 * (y < 0).int()).flatten(-2), s


def _values(code, s, scale, dtype=torch.float32):
    """what codes [..., D] and scales [..., D / 16] stand for"""
    grid = torch.tensor(_GRID, dtype=dtype, device=code.device)
    v = grid[(code & 7).long()] * (1 - 2 * (code >> 3)).to(dtype)
    return (v.unflatten(-1, (-1, 16)) * (s.to(dtype) * scale)[..., None]).flatten(-2)


def _pack(k, v, mk, case):
    """pages uint8 [batch * pages a sequence, page bytes] of k, v [batch, Hkv, tokens, D] and mk [batch, Hkv, tokens] (tokens a multiple of the page)"""
    B, H, N, D = k.shape
    P = case["page"]
    rows = []
    for x, scale in ((k, K_SCALE), (v, V_SCALE)):
        code, s = _codes(x, scale)
        pair = code.unflatten(-1, (-1, 2))
        rows.append(((pair[..., 0] + 16 * pair[..., 1]).to(torch.uint8), s.to(torch.float8_e4m3fn).view(torch.uint8)))
    parts = [torch.cat([rows[0][i], rows[1][i]], -1) for i in (0, 1)] + [mk.contiguous().view(torch.uint8).view(B, H, N, 4)]
    return torch.cat([p.unflatten(2, (N // P, P)).transpose(1, 2).reshape(B * (N // P), -1) for p in parts], 1)


def _unpack(pages, case):
    """codes of key and value int8 [pages, Hkv, P, D], their scales fp32 [pages, Hkv, P, D / 16], masks int32 [pages, Hkv, P]"""
    H, P, D = case["Hkv"], case["page"], case["D"]
    a, b = H * P * D, H * P * (D + D // 8)
    c = pages[:, :a].reshape(-1, H, P, D)
    c = torch.stack([c & 15, c >> 4], -1).flatten(-2).to(torch.int8)
    s = pages[:, a:b].contiguous().view(torch.float8_e4m3fn).float().reshape(-1, H, P, D // 8)
    mk = pages[:, b:].contiguous().view(torch.int32).reshape(-1, H, P)
    return c[..., :D], c[..., D:], s[..., :D // 16], s[..., D // 16:], mk


def _masks(shape, K, topk, gen):
    """membership masks: topk of K groups at random"""
    member = torch.rand(shape + (K,), generator=gen, device="cuda").argsort(-1) < topk
    return (member.int() << torch.arange(K, device="cuda", dtype=torch.int32)).sum(-1).to(torch.int32)


def prepare(case, seed):
    kind, n, B, Hq, Hkv, D = (case[x] for x in ("kind", "n", "batch", "Hq", "Hkv", "D"))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    empty = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")
    # a few dimensions of a head stand out, as they do in projections
    loud = 1.0 + 3.0 * (torch.rand(D, generator=gen, device="cuda") < 0.05)
    s = {"case": case, "kind": kind}
    if kind in ("rope", "rope_bwd"):
        r = case["rotary"]
        # the projections' output, token by token; query and key heads are views of it
        qkv = empty(B, n, Hq + 2 * Hkv, D)
        qkv.copy_(randn(B, n, Hq + 2 * Hkv, D) * loud)
        s["q"], s["k"] = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
        s["wq"], s["wk"] = ((1 + 0.1 * randn(D) for _ in range(2)) if case["norm"] else (None, None))
        s["freq"] = case["base"] ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r) / case["factor"]
        # prompts start at 0, sequences of a batch somewhere
        s["positions"] = None
        if case["first"]:
            start = torch.randint(0, case["first"], (B, 1), generator=gen, device="cuda")
            s["positions"] = (start + torch.arange(n, device="cuda")).to(torch.int32)
        if kind == "rope":
            s["q_out"], s["k_out"] = empty(B, Hq, n, D), empty(B, Hkv, n, D)
        else:
            s["gq"], s["gk"] = randn(B, Hq, n, D).to(torch.bfloat16), randn(B, Hkv, n, D).to(torch.bfloat16)
            grads = empty(B, n, Hq + 2 * Hkv, D)
            s["dq"], s["dk"] = grads[:, :, :Hq].transpose(1, 2), grads[:, :, Hq:Hq + Hkv].transpose(1, 2)
            s["dwq"], s["dwk"] = (empty(D, dtype=torch.float32) for _ in range(2)) if case["norm"] else (None, None)
    elif kind == "copy":
        pool, count = case["pool"], case["count"]
        s["pages"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (pool, _page_bytes(case) // 4), generator=gen, device="cuda", dtype=torch.int32).view(torch.uint8)
        pick = torch.randperm(pool, generator=gen, device="cuda")[:2 * count].to(torch.int32)
        s["src"], s["dst"] = pick[:count].contiguous(), pick[count:].contiguous()
    else:
        P = case["page"]
        lens = _lens(case) if kind == "decode" else [case["first"] + n] * B
        most = max(lens)
        per = -(-most // P)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["table"] = torch.randperm(B * per, generator=gen, device="cuda").to(torch.int32).view(B, per)
        if kind == "store":
            s["k"], s["v"] = (randn(B, Hkv, n, D) * loud).to(torch.bfloat16), randn(B, Hkv, n, D).to(torch.bfloat16)
            s["mk"] = _masks((B * Hkv, n), 4, 2, gen)
            s["pages"] = torch.zeros((B * per, _page_bytes(case)), dtype=torch.uint8, device="cuda")
            s["first"] = s["lens"] - n
            s["k_out"], s["v_out"], s["mk_out"] = empty(B, Hkv, n, D), empty(B, Hkv, n, D), empty(B * Hkv, n, dtype=torch.int32)
        else:
            pages = empty(B * per, _page_bytes(case), dtype=torch.uint8)
            step = max(1, 131072 // (per * P))
            for b in range(0, B, step):                          # (a few sequences at a time)
                m = min(step, B - b)
                k, v = (randn(m, Hkv, per * P, D) * loud).to(torch.bfloat16), randn(m, Hkv, per * P, D).to(torch.bfloat16)
                mk = _masks((m, Hkv, per * P), case["K"], case["topk"], gen)
                pages[s["table"][b:b + m].long().flatten()] = _pack(k, v, mk, case)
            s["pages"] = pages
            s["q"] = randn(B, Hq, D).to(torch.bfloat16)
            s["mq"] = _masks((B * Hq,), case["K"], case["topk"], gen)
            s["o"], s["lse"] = empty(B, Hq, D), empty(B * Hq, dtype=torch.float32)
    if own:
        from paper_2604_03260_b200 import binding as fb
        s["shape"] = fb.make_shape(Hq, Hkv, n, D, case.get("K", 4), case.get("topk", 2), case.get("window", 0), 0.0, case.get("softcap", 0.0), batch=B)
        s["status"] = torch.zeros(4, dtype=torch.int32, device="cuda")
        if kind in ("rope", "rope_bwd"):
            s["rope"] = fb.make_rope(case["rotary"], case["interleaved"], eps=EPS)
            s["ws"] = empty(fb.focus_qk_norm_rope_bwd_workspace_bytes(s["shape"]), dtype=torch.uint8)
        elif kind == "copy":
            s["cache"] = fb.make_kv4(s["pages"], case["page"])
        else:
            s["cache"] = fb.make_kv4(s["pages"], case["page"], s["table"], s["lens"], K_SCALE, V_SCALE)
            s["ws"] = empty(fb.focus_kv4_decode_workspace_bytes(s["shape"]), dtype=torch.uint8)
    return s


def run(s):
    case = s["case"]
    if own:
        from paper_2604_03260_b200 import binding as fb
        if s["kind"] == "rope":
            fb.focus_qk_norm_rope(s["shape"], s["rope"], s["q"], s["k"], s["wq"], s["wk"], s["freq"], s["positions"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        if s["kind"] == "rope_bwd":
            fb.focus_qk_norm_rope_bwd(s["shape"], s["rope"], s["q"], s["k"], s["wq"], s["wk"], s["freq"], s["positions"], s["gq"], s["gk"],
                                      s["dq"], s["dk"], s["dwq"], s["dwk"], s["ws"])
            return {"dq": s["dq"], "dk": s["dk"], "dwq": s["dwq"], "dwk": s["dwk"]}
        if s["kind"] == "store":
            fb.focus_kv4_append(s["shape"], s["cache"], s["k"], s["v"], s["mk"], None, s["status"])
            fb.focus_kv4_read(s["shape"], s["cache"], s["first"], s["k_out"], s["v_out"], s["mk_out"], s["status"])
            return {"k": s["k_out"], "v": s["v_out"], "mk": s["mk_out"]}
        if s["kind"] == "decode":
            fb.focus_kv4_decode_step(s["shape"], s["cache"], s["q"], s["mq"], s["o"], s["lse"], s["ws"], s["status"])
            return {"o": s["o"], "lse": s["lse"]}
        fb.focus_kv4_copy_pages(s["shape"], s["cache"], s["src"], s["dst"], s["status"])
        return {"pages": s["pages"].view(torch.int32)}
    if s["kind"] == "rope":
        return {x: _norm_rope(s[x], s["w" + x], s) for x in ("q", "k")}
    if s["kind"] == "rope_bwd":
        (dq, dwq), (dk, dwk) = (_norm_rope_bwd(s[x], s["w" + x], s["g" + x], s) for x in ("q", "k"))
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    if s["kind"] == "store":
        k, v = (_values(*_codes(s[x], scale), scale).to(torch.bfloat16) for x, scale in (("k", K_SCALE), ("v", V_SCALE)))
        return {"k": k, "v": v, "mk": s["mk"]}
    if s["kind"] == "decode":
        return _attend(s)
    s["pages"][s["dst"].long()] = s["pages"][s["src"].long()]
    return {"pages": s["pages"].view(torch.int32)}


# ---- plain forms

def _angles(s):
    """cos and sin fp32 [batch or 1, 1, n, rotary / 2] of the tokens' angles, which are taken in 64 bits: positions reach 200000"""
    n = s["case"]["n"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(n, device="cuda")[None]
    t = pos.double()[:, None, :, None] * s["freq"]
    return torch.cos(t).float(), torch.sin(t).float()


def _turn(x, cos, sin, case):
    """the first `rotary` dimensions of x rotated pair by pair"""
    r = case["rotary"]
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., r:]], -1)
    a, b = x[..., :r // 2], x[..., r // 2:r]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)


def _norm_rope(x, w, s):
    cos, sin = _angles(s)
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w
    return _turn(y, cos, sin, s["case"]).to(torch.bfloat16)


def _norm_rope_bwd(x, w, g, s):
    """gradients of x and of w; the rotation's transpose is the rotation by the negative angle"""
    cos, sin = _angles(s)
    g = _turn(g.float(), cos, -sin, s["case"])
    if w is None:
        return g.to(torch.bfloat16), None
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xhat = x * r
    gw = g * w
    dx = r * (gw - xhat * (gw * xhat).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), (g * xhat).flatten(0, 2).sum(0)


def _attend(s):
    case = s["case"]
    B, Hq, Hkv, D, G = case["batch"], case["Hq"], case["Hkv"], case["D"], case["Hq"] // case["Hkv"]
    kc, vc, ks, vs, mk = _unpack(s["pages"], case)
    at = s["table"].long()
    # [batch, pages, Hkv, P, ...] -> [batch, Hkv, tokens, ...]
    seq = lambda x: x[at].transpose(1, 2).flatten(2, 3)
    k, mk = _values(seq(kc), seq(ks), K_SCALE), seq(mk)
    x = (s["q"].float().view(B, Hkv, G, D) @ k.transpose(-1, -2)) / math.sqrt(D)
    del k
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    j, last = torch.arange(mk.shape[-1], device="cuda"), (s["lens"].long() - 1).view(B, 1, 1, 1)
    keep = (last - j <= case["window"]) | ((mk[:, :, None] & s["mq"].view(B, Hkv, G, 1)) != 0)
    x = x.masked_fill(~keep | (j > last), -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    o = (p @ _values(seq(vc), seq(vs), V_SCALE)) / l
    return {"o": o.reshape(B, Hq, D).to(torch.bfloat16), "lse": (m + torch.log(l)).reshape(B * Hq)}


def work(case):
    kind, n, B, Hq, Hkv, D = (case[x] for x in ("kind", "n", "batch", "Hq", "Hkv", "D"))
    rows = float(B) * n * (Hq + Hkv)
    if kind == "rope":
        # vectors read and written; square, scale and weigh, and a rotation of a pair in six operations
        return {"bytes": 4.0 * D * rows, "flops": rows * (5.0 * D + 3.0 * case["rotary"])}
    if kind == "rope_bwd":
        # gradients and vectors read, gradients written (without a norm the vectors are not needed)
        return {"bytes": (6.0 if case["norm"] else 4.0) * D * rows, "flops": rows * (12.0 * D + 3.0 * case["rotary"])}
    if kind == "store":
        # read in bf16, written in 4 bits with scales and masks; read in 4 bits, written in bf16
        return {"bytes": 2.0 * B * n * Hkv * (4.0 * D + 4 + (D + D / 8.0 + 4)), "flops": 2.0 * B * n * Hkv * 2 * D}
    if kind == "copy":
        return {"bytes": 2.0 * case["count"] * _page_bytes(case), "flops": 0}
    # the share of distant keys that meet a query head in a group; a key is read when one of the heads of its KV head attends it
    share = 1.0 - math.comb(case["K"] - case["topk"], case["topk"]) / math.comb(case["K"], case["topk"])
    b = f = 0.0
    for m in _lens(case):
        local = min(m, case["window"] + 1)
        read = local + (1.0 - (1.0 - share) ** (Hq // Hkv)) * (m - local)
        b += Hkv * ((D + D / 8.0) * read + 4.0 * m) + 4.0 * D * Hq
        f += 4.0 * D * Hq * (local + share * (m - local))
    return {"bytes": b, "flops": f}


# ---- the same in 64 bits

def _exact_store(x, scale):
    """nearest values of the 4-bit form, by distance to the tables of what a scale and a code can be"""
    # the scales from 0 to 448 (made on the host, where powers of two are exact)
    table = torch.tensor([e / 512 if e < 8 else (8 + e % 8) * 2.0 ** (e // 8 - 10) for e in range(127)], dtype=torch.float64).to(x.device)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)

    def nearest(y, values):
        """index of the nearest of the ascending values, of two equally near ones the even index"""
        mid = (values[1:] + values[:-1]) / 2
        lo, hi = torch.bucketize(y, mid), torch.bucketize(y, mid, right=True)
        return torch.where(lo % 2 == 0, lo, hi)

    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for b in range(x.shape[0]):
        y = x[b].double().unflatten(-1, (-1, 16)) / scale
        s = table[nearest(y.abs().amax(-1), 6 * table)][..., None]
        a = grid[nearest(torch.where(s > 0, y.abs() / s.clamp(min=1e-30), torch.zeros_like(y)), grid)]
        out[b] = (torch.sign(y) * a * s * scale).flatten(-2)
    return out


def _exact_turn(x, s, sign):
    """x [batch, H, n, D] as complex pairs times e^(i angle)"""
    case, r = s["case"], s["case"]["rotary"]
    pos = s["positions"].double() if s["positions"] is not None else torch.arange(case["n"], device="cuda", dtype=torch.float64)[None]
    unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), sign * torch.einsum("bt,f->btf", pos, s["freq"]))[:, None]
    first = torch.arange(r // 2, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else r // 2)
    z = torch.complex(x[..., first], x[..., second]) * unit
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind == "copy":
        return None                                              # (whole numbers)
    s = prepare(case, seed)
    if kind == "store":
        return {"k": _exact_store(s["k"], K_SCALE), "v": _exact_store(s["v"], V_SCALE), "mk": None}
    if kind == "rope":
        out = {}
        for name in ("q", "k"):
            x = s[name].double()
            if case["norm"]:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["D"] + EPS) * s["w" + name].double()
            out[name] = _exact_turn(x, s, 1.0)
        return out
    if kind == "rope_bwd":
        out = {}
        for name in ("q", "k"):
            g = _exact_turn(s["g" + name].double(), s, -1.0)
            out["dw" + name] = None
            if case["norm"]:
                # by differentiating the norm itself
                x, w = s[name].double().requires_grad_(), s["w" + name].double().requires_grad_()
                y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["D"] + EPS) * w
                g, out["dw" + name] = torch.autograd.grad(y, (x, w), g)
            out["d" + name] = g
        return out
    B, Hq, Hkv, D, P = case["batch"], case["Hq"], case["Hkv"], case["D"], case["page"]
    o, lse = torch.empty((B, Hq, D), dtype=torch.float64, device="cuda"), torch.empty((B, Hq), dtype=torch.float64, device="cuda")
    # what a byte's two codes stand for
    byte = torch.arange(256, device="cuda")
    half = lambda c: torch.tensor(_GRID, dtype=torch.float64, device="cuda")[c % 8] * torch.where(c >= 8, -1.0, 1.0).double()
    two = torch.stack([half(byte % 16), half(byte // 16)], -1)
    for b, m in enumerate(_lens(case)):
        raw = s["pages"][s["table"][b, :-(-m // P)].long()]
        for h in range(Hkv):
            rows = raw[:, h * P * D:(h + 1) * P * D].reshape(-1, D)[:m]
            at = Hkv * P * D + h * P * (D // 8)
            scales = raw[:, at:at + P * (D // 8)].reshape(-1, D // 8)[:m].contiguous().view(torch.float8_e4m3fn).double()
            at = Hkv * P * (D + D // 8) + h * P * 4
            mk = raw[:, at:at + P * 4].contiguous().view(torch.int32).reshape(-1)[:m]
            kv = two[rows.long()].view(m, 2, D // 16, 16) * scales.view(m, 2, D // 16, 1)
            k, v = kv[:, 0].reshape(m, D) * K_SCALE, kv[:, 1].reshape(m, D) * V_SCALE
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            x = s["q"][b, heads].double() @ k.T / D ** 0.5
            if case["softcap"]:
                x = torch.tanh(x / case["softcap"]) * case["softcap"]
            seen = torch.arange(m, device="cuda") >= m - 1 - case["window"]
            x = torch.where(seen | ((mk & s["mq"].view(B, Hq)[b, heads, None]) != 0), x, -math.inf)
            lse[b, heads] = torch.logsumexp(x, -1)
            o[b, heads] = torch.softmax(x, -1) @ v
    return {"o": o, "lse": lse.view(B * Hq)}
