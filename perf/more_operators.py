"""The operators of an int8 expert layer whose speed is measured: router logits, routing by scores with balance bias and groups, rows to int8
behind the norm and behind a (gated) activation, and the int8 product with scales per token and channel, alone and grouped by expert.

Token counts run from one decoder token to the largest prefill preset of workloads.py; widths are those of its layers or generic.
int8 rows have one fp32 scale per row, weights one per output channel.  `own` chooses between the plain torch form and the calls of the library.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TOP, TINY, EPS = 127.0, 2.0 ** -126, 1e-6
NLLB = dict(K=2048, N=8192, E=128, k=2)


def _named(name, c):
    return c if name is None else dict(c, name=name)


def _logits(name=None, *, T, d, E, dtype="bf16", bias=False):
    return _named(name, dict(op="logits", T=T, d=d, E=E, dtype=dtype, bias=bias))


def _route(name=None, *, T, E, k, score="sigmoid", balance=True, groups=1, kept=1, top=1, renormalize=True, scale=1.0, H=-1, dtype="f32"):
    return _named(name, dict(op="route", T=T, E=E, k=k, score=score, balance=balance, groups=groups, kept=kept, top=top,
                             renormalize=renormalize, scale=scale, H=H, dtype=dtype))


def _norm(name=None, *, T, d, dtype="bf16", residual=True, normed=True):
    return _named(name, dict(op="norm", T=T, d=d, dtype=dtype, residual=residual, normed=normed))


def _act(name=None, *, rows, f, act="silu", gated=True, dtype="bf16"):
    return _named(name, dict(op="act", T=rows, f=f, act=act, gated=gated, dtype=dtype))


def _linear(name=None, *, T, N, K, act="none", bias=False, out="bf16"):
    return _named(name, dict(op="linear", T=T, N=N, K=K, act=act, bias=bias, out=out))


def _experts(name=None, *, T, N, K, E, k, act="none", bias=False, out="bf16", gather=True, zipf=0.0, H=-1):
    return _named(name, dict(op="experts", T=T, N=N, K=K, E=E, k=k, act=act, bias=bias, out=out, gather=gather, zipf=zipf, H=H))


def listed():
    return [
        # a generation batch: the router of a 128-expert layer
        _logits("logits_32_tokens", T=32, d=2048, E=128),
        # ragged prefill batch, more experts
        _logits("logits_5003_tokens", T=5003, d=2048, E=256),
        # one token being generated: sigmoid scores, balance bias, half of eight groups
        _route("route_1_token", T=1, E=128, k=8, groups=8, kept=4, top=2, scale=2.5),
        # the largest prefill batch, 256 experts
        _route("route_16384_tokens", T=16384, E=256, k=8, groups=8, kept=4, top=2, scale=2.5),
        # the norm in front of a layer, one token
        _norm("norm_1_token", T=1, d=2048),
        # the norm in front of a layer, the largest prefill batch
        _norm("norm_16384_tokens", T=16384, d=2048),
        # between the two products of a generation batch (32 tokens, two experts each)
        _act("act_64_rows", rows=64, f=8192, act="relu", gated=False),
        # between the two products of gated experts, ragged prefill batch
        _act("act_gated_20011_rows", rows=20011, f=2048),
        # ragged encoder batch, second product of a dense FFN with bias
        _linear("linear_1501_tokens", T=1501, N=1024, K=4096, bias=True),
        # long prefill, first product
        _linear("linear_16384_tokens", T=16384, N=8192, K=2048),
        # one token being generated: the first product of its two experts
        _experts("experts_1_token", T=1, act="relu", **NLLB),
        # the largest grouped product: a long prefill batch, skewed routing
        _experts("experts_16384_skewed", T=16384, act="relu", zipf=1.2, **NLLB),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return rng.choice([768, 1024, 2048, 32 * rng.randint(8, 64), rng.randint(200, 2000)])


def draw(rng):
    op = rng.choice(["logits", "route", "norm", "act", "linear", "experts", "experts"])
    T = _log_int(rng, 1, 12000)
    if op == "logits":
        return _logits(T=T, d=_ceil(_width(rng), 32) * 32, E=rng.choice([8, 64, 128, 256, rng.randint(4, 400)]),
                       dtype=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.3)
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        E = groups * rng.choice([8, 16, 32, rng.randint(4, 50)])
        kept = rng.randint((groups + 1) // 2, groups)
        return _route(T=T, E=E, k=rng.randint(1, min(8, kept * (E // groups))), score=rng.choice(["softmax", "sigmoid"]),
                      balance=rng.random() < 0.6, groups=groups, kept=kept, top=rng.choice([1, 2]), renormalize=rng.random() < 0.6,
                      scale=rng.choice([1.0, 2.5]), H=rng.choice([-1, -1, E // 4]), dtype=rng.choice(["f32", "f32", "bf16"]))
    if op == "norm":
        return _norm(T=T, d=_width(rng), dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7, normed=rng.random() < 0.7)
    act = rng.choice(["none", "relu", "gelu", "silu"])
    if op == "act":
        return _act(rows=T, f=rng.choice([_width(rng), 4 * _width(rng)]), act=act, gated=rng.random() < 0.6,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    out = rng.choice(["f32", "bf16", "bf16"])
    if op == "linear":
        d = _width(rng)
        N, K = rng.choice([(4 * d, d), (d, 4 * d)])
        return _linear(T=T, N=N, K=K, act=act, bias=rng.random() < 0.4, out=out)
    dims = rng.choice([NLLB, dict(K=1024, N=4096, E=128, k=1), dict(K=_width(rng), N=rng.randint(500, 6000), E=rng.randint(4, 128),
                                                                    k=rng.choice([1, 2]))])
    gather = rng.random() < 0.6
    if not gather:
        dims = dict(dims, N=dims["K"], K=dims["N"])
    return _experts(T=T, act=act, bias=rng.random() < 0.3, out=out, gather=gather, zipf=rng.choice([0.0, 1.1, 1.2]),
                    H=rng.choice([-1, -1, max(1, dims["E"] // 4)]), **dims)


def _ceil(n, m):
    return -(-n // m)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _codes(gen, rows, K, pitch):
    """Normal values as int8 rows of `pitch` bytes and their scales, each row's largest value at the end of the range."""
    q = torch.zeros((rows, pitch), dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, dtype=torch.float32, device="cuda")
    step = max(1, (1 << 27) // K)
    for r in range(0, rows, step):                     # a slice at a time: the temporaries stay small
        n = min(step, rows - r)
        v = torch.randn((n, K), dtype=torch.bfloat16, device="cuda", generator=gen).float()
        scales[r:r + n] = v.abs().amax(1) / TOP
        q[r:r + n, :K] = (v / scales[r:r + n, None]).round().to(torch.int8)
    return q, scales


def _weights(gen, E, N, K):
    """A checkpoint's int8 weights [E, N, K] with a scale per output channel."""
    w, scales = _codes(gen, E * N, K, K)
    spread = torch.exp(0.2 * torch.randn(E * N, device="cuda", generator=gen))
    return w.view(E, N, K), (scales * spread / math.sqrt(K)).view(E, N)


def _laid_out(w):
    """The layout that the library's products read, made once when a layer is loaded."""
    import paper_2405_18832_amd as moe

    E, N, K = w.shape
    packed = torch.empty(moe.moe_quant_weight_bytes(E, N, K), dtype=torch.int8, device="cuda")
    moe.moe_quantize_weights_int(E, N, K, "i8", w, packed, None)
    return packed


def _routing(s, c, gen):
    """What routing and moe_permute leave: the assignments in expert order and where each expert's begin."""
    T, E, k = c["T"], c["E"], c["k"]
    logits = -torch.log(-torch.log(torch.rand((T, E), dtype=torch.float64, device="cuda", generator=gen).clamp(1e-12, 1 - 1e-12)))
    if c["zipf"]:
        rank = torch.rand(E, device="cuda", generator=gen).argsort()
        logits = logits - c["zipf"] * torch.log1p(rank.double())
    flat = logits.topk(k, dim=1).indices.reshape(-1)
    s["perm"] = flat.argsort(stable=True).int()
    counts = torch.bincount(flat, minlength=E)
    s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    s["offsets"][1:] = counts.cumsum(0)
    s["mask"] = None
    run_ = torch.ones(E, dtype=torch.bool, device="cuda")
    if c["H"] >= 0:
        run_ = torch.zeros_like(run_)
        run_[counts.argsort(descending=True, stable=True)[:c["H"]]] = True
        s["mask"] = run_.to(torch.uint8)
    # the same for the host, where the plain form is a product per expert
    s["segments"] = [(e, a, b) for e, (a, b, on) in enumerate(zip(*(t.tolist() for t in (s["offsets"][:-1], s["offsets"][1:], run_)))) if on and b > a]


def _buffers_of_product(s, c):
    import paper_2405_18832_amd as moe

    A = c["T"] * c.get("k", 1)
    s["packed"] = _laid_out(s["w"])
    s["shape"] = moe.make_quant_shape(A, c["N"], c["K"], c.get("E", 1), c.get("k", 1), c["act"], c["out"])
    s["ws"] = torch.empty(max(256, moe.moe_int_workspace_bytes(s["shape"])), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    s = {"case": c}
    T = c["T"]
    if c["op"] == "logits":
        dt = DTYPES[c["dtype"]]
        s["x"] = torch.randn((T, c["d"]), device=dev, generator=gen).to(dt)
        s["w"] = (torch.randn((c["E"], c["d"]), device=dev, generator=gen) * 0.02).to(dt)
        s["bias"] = torch.randn(c["E"], device=dev, generator=gen) if c["bias"] else None
        s["out"] = torch.empty((T, c["E"]), dtype=torch.float32, device=dev)
        if own:
            import paper_2405_18832_amd as moe
            s["shape"] = moe.make_shape(T, c["d"], 32, c["E"], 1, c["dtype"], False)
        return s
    if c["op"] == "route":
        E, k = c["E"], c["k"]
        # logits of a trained router: a few experts stand out; the balance bias is small beside the scores
        s["logits"] = (torch.randn((T, E), device=dev, generator=gen) * 1.2).to(DTYPES[c["dtype"]])
        s["balance"] = 0.05 * torch.randn(E, device=dev, generator=gen) if c["balance"] else None
        i32 = torch.int32
        s["idx"] = torch.empty((T, k), dtype=i32, device=dev)
        s["weight"] = torch.empty((T, k), dtype=torch.float32, device=dev)
        s["counts"] = torch.empty(E, dtype=i32, device=dev)
        s["offsets"] = torch.empty(E + 1, dtype=i32, device=dev)
        s["hot"] = torch.empty(E, dtype=torch.uint8, device=dev) if c["H"] >= 0 else None
        if own:
            import paper_2405_18832_amd as moe
            s["shape"] = moe.make_shape(T, 32, 32, E, k, "bf16", c["renormalize"])
            s["rule"] = moe.make_routing(c["score"], c["groups"], c["kept"], c["top"], c["scale"])
            s["ws"] = torch.empty(max(256, moe.moe_workspace_bytes(s["shape"])), dtype=torch.uint8, device=dev)
        return s
    if c["op"] == "norm":
        d, dt = c["d"], DTYPES[c["dtype"]]
        s["x"] = torch.randn((T, d), device=dev, generator=gen).to(dt)
        # the residual stream is wider than a sublayer's output
        s["residual"] = (3 * torch.randn((T, d), device=dev, generator=gen)).to(dt) if c["residual"] else None
        s["weight"] = torch.exp(0.2 * torch.randn(d, device=dev, generator=gen))
        s["sum"] = torch.empty((T, d), dtype=dt, device=dev) if c["residual"] else None
        s["normed"] = torch.empty((T, d), dtype=dt, device=dev) if c["normed"] else None
        s["q"] = torch.empty((T, _ceil(d, 128) * 128), dtype=torch.int8, device=dev)
        s["scales"] = torch.empty(T, dtype=torch.float32, device=dev)
        return s
    if c["op"] == "act":
        f = c["f"]
        s["h"] = torch.randn((T, f * (1 + c["gated"])), device=dev, generator=gen)
        s["h"] *= torch.exp(0.5 * torch.randn((T, 1), device=dev, generator=gen))
        s["h"] = s["h"].to(DTYPES[c["dtype"]])
        s["q"] = torch.empty((T, _ceil(f, 128) * 128), dtype=torch.int8, device=dev)
        s["scales"] = torch.empty(T, dtype=torch.float32, device=dev)
        return s
    N, K, E, k = c["N"], c["K"], c.get("E", 1), c.get("k", 1)
    s["w"], s["w_scales"] = _weights(gen, E, N, K)
    s["bias"] = 0.25 * torch.randn((E, N), device=dev, generator=gen) if c["bias"] else None
    s["q"], s["q_scales"] = _codes(gen, T if c.get("gather", True) else T * k, K, _ceil(K, 128) * 128)
    if c["op"] == "experts":
        _routing(s, c, gen)
    s["out"] = torch.zeros((T * k, N), dtype=DTYPES[c["out"]], device=dev)
    if own:
        _buffers_of_product(s, c)
    return s


# ---- one pass, the library's calls ---------------------------------------------------------------------------------
def _run_own(s):
    import paper_2405_18832_amd as moe

    c = s["case"]
    if c["op"] == "logits":
        moe.moe_gate_logits(s["shape"], s["x"], s["w"], s["bias"], s["out"])
        return s["out"]
    if c["op"] == "route":
        moe.moe_route_logits(s["shape"], s["rule"], c["dtype"], s["logits"], s["balance"], s["idx"], s["weight"], s["counts"], s["offsets"],
                             c["H"], s["hot"], s["ws"])
        return _route_out(s["idx"], s["weight"], s["counts"], s["offsets"], s["hot"])
    if c["op"] == "norm":
        moe.moe_norm_quantize_int(c["T"], c["d"], c["dtype"], s["x"], s["residual"], s["weight"], EPS, s["sum"], s["normed"], s["q"], s["scales"])
        return _norm_out(s["sum"], s["normed"], s["q"][:, :c["d"]], s["scales"])
    if c["op"] == "act":
        moe.moe_act_quantize_int(c["T"], c["f"], c["dtype"], s["h"], c["gated"], c["act"], 0, None, None, s["q"], s["scales"])
        return {"q": s["q"][:, :c["f"]], "scales": s["scales"]}
    if c["op"] == "linear":
        moe.moe_int_linear(s["shape"], s["q"], s["q_scales"], s["packed"], s["w_scales"], s["bias"], s["out"], s["ws"])
        return s["out"]
    moe.moe_int_expert_linear(s["shape"], s["q"], s["q_scales"], s["perm"] if c["gather"] else None, s["offsets"], s["mask"], s["packed"],
                             s["w_scales"], s["bias"], s["out"], s["ws"])
    return s["out"]


def _route_out(idx, weight, counts, offsets, hot):
    out = {"idx": idx, "weight": weight, "counts": counts, "offsets": offsets}
    return out if hot is None else dict(out, hot=hot)


def _norm_out(total, normed, q, scales):
    out = {"q": q, "scales": scales}
    if total is not None:
        out["sum"] = total
    if normed is not None:
        out["normed"] = normed
    return out


# ---- one pass, in elementary torch operations ----------------------------------------------------------------------
def _activated(v, act):
    """In the precision of v."""
    if act == "relu":
        return v.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(v * -math.sqrt(0.5))
    return v / (1.0 + torch.exp(-v)) if act == "silu" else v


def _quantized(u, rho=None):
    """Codes and scales of rows u * rho; whole numbers, so in 64 bits: values next to the middle between two of them."""
    top = u.abs().amax(1, keepdim=True)
    most = top if rho is None else top * rho
    scales = (most / TOP).clamp_min(TINY)
    t = torch.where(most / TOP < TINY, (u if rho is None else u * rho) / TINY, u * TOP / torch.where(top > 0, top, torch.ones_like(top)))
    return t.round().to(torch.int8), scales[:, 0].float()


def _run_plain(s):
    c = s["case"]
    if c["op"] == "logits":
        y = s["x"].float() @ s["w"].float().T
        return y if s["bias"] is None else y + s["bias"]
    if c["op"] == "route":
        return _plain_route(s)
    if c["op"] == "norm":
        total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
        v = total.float()
        rho = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
        q, scales = _quantized(total.double() * s["weight"].double(), rho.double())
        return _norm_out(total if c["residual"] else None, (v * rho * s["weight"]).to(s["x"].dtype) if c["normed"] else None, q, scales)
    if c["op"] == "act":
        h, f = s["h"].double(), c["f"]
        v = _activated(h[:, :f], c["act"])
        q, scales = _quantized(v * h[:, f:] if c["gated"] else v)
        return {"q": q, "scales": scales}
    N, K = c["N"], c["K"]
    x = s["q"][:, :K].float()
    if c["op"] == "linear":
        y = (x @ s["w"][0].float().T) * (s["q_scales"][:, None] * s["w_scales"][0])
        return _activated(y if s["bias"] is None else y + s["bias"][0], c["act"]).to(s["out"].dtype)
    sx = s["q_scales"]
    if c["gather"]:
        token = s["perm"].long() // c["k"]
        x, sx = x[token], sx[token]
    y = torch.zeros((x.shape[0], N), device=x.device)
    for e, a, b in s["segments"]:              # the active experts, a product each
        v = (x[a:b] @ s["w"][e].float().T) * (sx[a:b, None] * s["w_scales"][e])
        y[a:b] = _activated(v if s["bias"] is None else v + s["bias"][e], c["act"])
    return y.to(s["out"].dtype)


def _plain_route(s):
    """In 64 bits: the order of scores next to each other."""
    c = s["case"]
    E, k, G = c["E"], c["k"], c["groups"]
    l = s["logits"].double()
    p = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.softmax(l, 1)
    choice = l if s["balance"] is None else p + s["balance"].double()
    if G > 1:
        value = choice if c["top"] == 1 else (p if s["balance"] is None else choice)
        of_group = value.view(-1, G, E // G).sort(2, descending=True).values[:, :, :c["top"]].sum(2)
        kept = of_group.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        allowed = torch.zeros_like(of_group, dtype=torch.bool).scatter_(1, kept, True)
        choice = choice.masked_fill(~allowed.repeat_interleave(E // G, 1), -math.inf)
    idx = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, idx)
    if c["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    counts = (idx.reshape(-1, 1) == torch.arange(E, device=idx.device)).sum(0)
    offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0))
    hot = None
    if c["H"] >= 0:
        hot = torch.zeros(E, dtype=torch.uint8, device=idx.device)
        hot[counts.sort(dim=0, descending=True, stable=True).indices[:c["H"]]] = 1
    return _route_out(idx.int(), (w * c["scale"]).float(), counts.int(), offsets.int(), hot)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the work of a pass --------------------------------------------------------------------------------------------
def _active(c):
    """Expected number of experts that run and of their rows: tokens take experts by their Zipf weights."""
    E, k, T = c["E"], c["k"], c["T"]
    p = [(1.0 + r) ** -c["zipf"] for r in range(E)]
    total = sum(p)
    share = [min(1.0, k * v / total) for v in p]
    share = share if c["H"] < 0 else share[:c["H"]]
    return sum(1.0 - (1.0 - v) ** T for v in share), T * min(float(k), sum(share))


def work(case):
    c, T = case, case["T"]
    es = DTYPES[c["dtype"]].itemsize if "dtype" in c else DTYPES[c["out"]].itemsize
    if c["op"] == "logits":
        return {"bytes": (T + c["E"]) * c["d"] * es + 4 * T * c["E"], "flops": 2.0 * T * c["d"] * c["E"]}
    if c["op"] == "route":
        return {"bytes": T * c["E"] * es + 8 * T * c["k"] + 8 * c["E"], "flops": 10.0 * T * c["E"]}
    if c["op"] == "norm":
        return {"bytes": T * c["d"] * (es * (1 + 2 * c["residual"] + c["normed"]) + 1) + 4 * T + 4 * c["d"], "flops": 8.0 * T * c["d"]}
    if c["op"] == "act":
        return {"bytes": T * c["f"] * (es * (1 + c["gated"]) + 1) + 4 * T, "flops": 10.0 * T * c["f"]}
    N, K = c["N"], c["K"]
    if c["op"] == "linear":
        return {"bytes": T * (K + 4) + N * (K + 4) + T * N * es, "flops": 2.0 * T * N * K}
    experts, rows = _active(c)
    return {"bytes": (T if c["gather"] else rows) * (K + 4) + experts * N * (K + 4) + rows * N * es, "flops": 2.0 * rows * N * K}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------
def _codes64(n):
    """n [rows, d]: whole multiples of a row's largest magnitude / 127."""
    most = torch.maximum(n.max(1).values, -n.min(1).values)
    scale = torch.maximum(most / 127, torch.full_like(most, TINY))
    safe = torch.where(most / 127 >= TINY, most, torch.full_like(most, 127 * TINY))
    return torch.round(127 * n / safe[:, None]), scale


def _act64(v, act):
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return v * torch.special.ndtr(v)
    return torch.where(v > 0, v, torch.zeros_like(v)) if act == "relu" else v


def _product64(q, sq, w, sw):
    return torch.mm(q.double(), w.double().t().contiguous()) * sq.double().unsqueeze(1) * sw.double().unsqueeze(0)


def _route64(s, c):
    """Token by token what is chosen, without sorting: the best remaining expert k times."""
    E, k, G = c["E"], c["k"], c["groups"]
    l = s["logits"].double()
    if c["score"] == "sigmoid":
        p = 1 / (1 + torch.exp(-l))
    else:
        p = torch.exp(l - l.max(1, keepdim=True).values)
        p = p / p.sum(1, keepdim=True)
    rows = torch.arange(l.shape[0], device=l.device)

    def first_best(v):
        best = v == v.max(1, keepdim=True).values
        at = torch.arange(v.shape[1], device=v.device).expand_as(v)
        return torch.where(best, at, torch.full_like(at, v.shape[1])).min(1).values

    choice = l.clone() if s["balance"] is None else p + s["balance"].double()
    if G > 1:
        v = (p if c["top"] == 2 and s["balance"] is None else choice).reshape(-1, E // G).clone()
        value = torch.zeros(v.shape[0], dtype=torch.float64, device=l.device)
        for _ in range(c["top"]):
            at = first_best(v)
            value += v[torch.arange(v.shape[0], device=l.device), at]
            v[torch.arange(v.shape[0], device=l.device), at] = -math.inf
        value = value.view(-1, G)
        allowed = torch.zeros_like(value, dtype=torch.bool)
        for _ in range(c["kept"]):
            at = first_best(value)
            allowed[rows, at] = True
            value[rows, at] = -math.inf
        choice[~allowed[:, torch.arange(E, device=l.device) // (E // G)]] = -math.inf
    idx, w = [], []
    for _ in range(k):
        at = first_best(choice)
        idx.append(at)
        w.append(p[rows, at])
        choice[rows, at] = -math.inf
    idx, w = torch.stack(idx, 1), torch.stack(w, 1)
    w = (w / w.sum(1, keepdim=True) if c["renormalize"] else w) * c["scale"]
    counts = torch.bincount(idx.reshape(-1), minlength=E)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    hot = None
    if c["H"] >= 0:
        ahead = (counts[None] > counts[:, None]) | ((counts[None] == counts[:, None]) &
                                                    (torch.arange(E, device=l.device)[None] < torch.arange(E, device=l.device)[:, None]))
        hot = (ahead.sum(1) < c["H"]).to(torch.uint8)
    return _route_out(idx.int(), w, counts.int(), offsets.int(), hot)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "logits":
        y = torch.mm(s["x"].double(), s["w"].double().t().contiguous())
        return y if s["bias"] is None else y + s["bias"].double()
    if c["op"] == "route":
        return _route64(s, c)
    if c["op"] == "norm":
        v = s["x"].double()
        if c["residual"]:
            v = (v + s["residual"].double()).to(s["x"].dtype).double()
        rms = torch.sqrt((v ** 2).sum(1, keepdim=True) / c["d"] + EPS)
        n = v * s["weight"].double()
        q, scales = _codes64(n)                        # the norm's factor does not change a row's codes
        return _norm_out(v if c["residual"] else None, n / rms if c["normed"] else None, q.to(torch.int8), scales / rms[:, 0])
    if c["op"] == "act":
        h, f = s["h"].double(), c["f"]
        v = _act64(h[:, :f], c["act"])
        q, scales = _codes64(v * h[:, f:] if c["gated"] else v)
        return {"q": q.to(torch.int8), "scales": scales}
    N, K = c["N"], c["K"]
    finish = lambda v, e: _act64(v if s["bias"] is None else v + s["bias"][e].double(), c["act"])
    if c["op"] == "linear":
        return finish(_product64(s["q"][:, :K], s["q_scales"], s["w"][0], s["w_scales"][0]), 0)
    A = c["T"] * c["k"]
    token = torch.arange(A, device="cuda")
    if c["gather"]:
        token = torch.div(s["perm"].long(), c["k"], rounding_mode="floor")
    v = torch.zeros((A, N), dtype=torch.float64, device="cuda")
    bounds = s["offsets"].tolist()
    for e in range(c["E"]):
        a, b = bounds[e], bounds[e + 1]
        if a < b and (s["mask"] is None or int(s["mask"][e])):
            v[a:b] = finish(_product64(s["q"][token[a:b], :K], s["q_scales"][token[a:b]], s["w"][e], s["w_scales"][e]), e)
    return v
