"""Cases of the 8-bit serving operators: a transformer layer's products, norms, quantisers and cached attention.

A case is a plain dict.  prepare() makes what a serving program holds before the call (activations, 8-bit weights with a scale
per output channel, a paged cache with its block table), run() is one pass through one operator, exact() the operator's
definition in 64 bits.  Where `own` is false run() computes the same in elementary 32-bit torch operations.

An 8-bit token is codes and one scale:  scale = max(max |v| / 127, 2^-126), code = round_half_even(v / scale).
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "s8": torch.int8}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "s8": 1}
TINY = 2.0 ** -126


def listed():
    return [
        # one new token through a square projection: the smallest call of a step, nothing to share the weights with
        dict(name="linear_token", kind="linear", M=1, K=4096, N=4096, x="bf16", y="bf16", bias=False),
        # a serving batch through the wide projection of an MLP: the weights are the traffic
        dict(name="linear_batch", kind="linear", M=48, K=4096, N=16384, x="bf16", y="bf16", bias=False),
        # a ragged prompt batch, sizes that fill no tile, with bias
        dict(name="linear_ragged", kind="linear", M=1531, K=4100, N=5001, x="f16", y="f16", bias=True),
        # a long prompt through the largest projection, tokens already in 8 bits (from the norm in front)
        dict(name="linear_prompt", kind="linear", M=8192, K=8192, N=8192, x="s8", y="bf16", bias=False),
        # between two blocks of one step of a serving batch: residual update and norm, the result in 8 bits for the next product
        dict(name="norm_step_codes", kind="norm", rows=64, C=4096, type="bf16", post="", pre="rms", gate="", codes=True),
        # odd rows of a small model in 32 bits, layer norm and a gate per sequence
        dict(name="norm_ragged", kind="norm", rows=777, C=1001, type="f32", post="", pre="layer", gate="sequence", codes=False),
        # a long prompt, norms on both sides of the block and a learnt gate per channel
        dict(name="norm_prompt", kind="norm", rows=16384, C=4096, type="bf16", post="rms", pre="rms", gate="channel", codes=False),
        # few tokens of an odd width, as an attention output before its projection
        dict(name="quant_step", kind="quant", rows=33, C=1111, type="f16", act=""),
        # the middle of a gated MLP over a long prompt
        dict(name="quant_gated", kind="quant", rows=8192, C=16384, type="bf16", act="silu"),
        # a short chat batch, 16-bit cache: one step, latency
        dict(name="attend_short", kind="attend", B=8, longest=300, even=False, heads=4, group=2, D=64, page=16, cache="bf16", x="bf16"),
        # one very long context in 8 bits: few rows, the length has to be shared out
        dict(name="attend_long", kind="attend", B=1, longest=131072, even=True, heads=8, group=4, D=128, page=64, cache="s8", x="bf16"),
        # a full serving batch of all lengths, one slot of it empty, 8-bit cache
        dict(name="attend_batch", kind="attend", B=64, longest=8192, even=False, heads=8, group=4, D=128, page=32, cache="s8", x="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    """A width: mostly a multiple of 128 or 16, as models have them, otherwise any number; 3072 is left out."""
    n, u = _log(rng, lo, hi), rng.random()
    step = 128 if u < 0.5 else 16 if u < 0.8 else 1
    n = max(min(step, hi), n // step * step)
    return n if n != 3072 else 3200


def draw(rng):
    u = rng.random()
    if u < 0.4:
        while True:
            x = rng.choice(("bf16", "bf16", "f16", "s8"))
            c = dict(kind="linear", M=_log(rng, 1, 8192), K=_width(rng, 32, 16384), N=_width(rng, 32, 16384), x=x,
                     y=rng.choice(("bf16", "f16", "f32") if x == "s8" else ("bf16", "f16")), bias=rng.random() < 0.3)
            if c["M"] != 3072 and work(c)["flops"] <= 2 * 8192 ** 3:
                return c
    if u < 0.55:
        return dict(kind="norm", rows=_log(rng, 1, 16383), C=_width(rng, 32, 4096), type=rng.choice(("bf16", "bf16", "f16", "f32")),
                    post=rng.choice(("", "", "rms", "layer")), pre=rng.choice(("rms", "rms", "layer")),
                    gate=rng.choice(("", "", "channel", "sequence")), codes=False)
    if u < 0.7:
        act = rng.choice(("", "silu", "gelu"))
        return dict(kind="quant", rows=_log(rng, 1, 8191), C=_width(rng, 32, 16384), type=rng.choice(("bf16", "f16") if act else ("bf16", "f16", "f32")),
                    act=act)
    while True:
        cache = rng.choice(("s8", "s8", "bf16", "f16"))
        c = dict(kind="attend", B=_log(rng, 1, 64), longest=_log(rng, 1, 131072), even=rng.random() < 0.5, heads=rng.choice((1, 2, 4, 5, 8)),
                 group=rng.choice((1, 2, 4, 5, 8, 16)), D=rng.choice((64, 128, 128, 80, 96, 192, 256)), page=rng.choice((1, 16, 16, 24, 32, 64, 128)),
                 cache=cache, x=rng.choice(("bf16", "f16")) if cache == "s8" else cache)
        if work(c)["bytes"] <= 5e8 and c["longest"] != 3072:
            return c


def _lens(case):
    """Cached tokens of each request, the new one included: a property of the case.  In a batch of all lengths the longest comes
    first, and with eight requests or more the last place of the batch is empty (a step captured for a fixed batch)."""
    B, top = case["B"], case["longest"]
    if case["even"]:
        return [top] * B
    r = random.Random(B * 131 + top)
    lens = [top] + [r.randint(1, top) for _ in range(B - 1)]
    if B >= 8:
        lens[-1] = 0
    return lens


def _tokens(g, rows, C):
    """Activations as blocks meet them: tokens of different size, a few channels far larger than the others."""
    x = torch.randn(rows, C, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    big = torch.rand(C, generator=g, device="cuda") < 0.01
    return x * torch.where(big, 8.0, 1.0)


def _quant(v):
    scale = (v.abs().amax(-1, keepdim=True) / 127).clamp_min(TINY)
    return torch.round(v / scale), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    kind = case["kind"]
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        wq, ws = _quant(rand(N, K) * 0.02)
        st = dict(w=wq.to(torch.int8), sw=ws[:, 0].contiguous(), bias=rand(N) * 0.1 if case["bias"] else None, y=TYPES[case["y"]])
        x = _tokens(g, M, K)
        if case["x"] == "s8":
            xq, xs = _quant(x)
            return dict(case=case, x=xq.to(torch.int8), sx=xs[:, 0].contiguous(), **st)
        return dict(case=case, x=x.to(TYPES[case["x"]]), **st)
    if kind == "norm":
        rows, C, t = case["rows"], case["C"], TYPES[case["type"]]
        gate, per = None, rows
        if case["gate"]:
            per = rows if case["gate"] == "channel" else max(1, -(-rows // 4))  # four sequences share the batch
            gate = (0.5 + 0.2 * rand(-(-rows // per), C)).to(t)
        weight = lambda: (1 + 0.1 * rand(C)).to(t)  # noqa: E731
        bias = lambda form: (0.1 * rand(C)).to(t) if form == "layer" else None  # noqa: E731
        return dict(case=case, a=_tokens(g, rows, C).to(t), res=(3 * rand(rows, C)).to(t), gate=gate, per=per,
                    post_w=weight() if case["post"] else None, post_b=bias(case["post"]), pre_w=weight(), pre_b=bias(case["pre"]))
    if kind == "quant":
        x = _tokens(g, case["rows"], case["C"]).to(TYPES[case["type"]])
        return dict(case=case, x=x, gate=(2 * rand(case["rows"], case["C"])).to(x.dtype) if case["act"] else None)
    # the cache of a batch: page 0 belongs to nobody, the others are dealt out in random order
    B, H, D, page, lens = case["B"], case["heads"], case["D"], case["page"], _lens(case)
    need = [-(-n // page) for n in lens]
    pages, width = sum(need) + 1, max(1, max(need))
    order = (torch.randperm(pages - 1, generator=g, device="cuda") + 1).to(torch.int32)
    at = torch.tensor([0] + need, device="cuda").cumsum(0)
    cols = torch.arange(width, device="cuda")
    used = cols[None] < torch.tensor(need, device="cuda")[:, None]
    table = torch.where(used, torch.cat([order, order[:1] * 0])[(at[:-1, None] + cols[None]).clamp_max(pages - 1)], 0).to(torch.int32)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    last = (n - 1).clamp_min(0)
    slots = table.gather(1, (last // page).long()[:, None])[:, 0].long() * page + last % page
    slots = torch.where(n > 0, slots, -1)
    kv = rand(2, pages, page, H, D)
    kv *= torch.exp(0.4 * rand(2, pages, page, H, 1))
    st = dict(case=case, table=table, lens=n, slots=slots, rows=slots.clamp_min(0), scales=None,
              q=rand(B, H * case["group"], D).to(TYPES[case["x"]]), new=rand(2, B, H, D).to(TYPES[case["x"]]))
    if case["cache"] == "s8":
        codes, scale = _quant(kv)
        st["kv"], st["scales"] = codes.to(torch.int8), scale[..., 0].contiguous()
    else:
        st["kv"] = kv.to(TYPES[case["cache"]])
    return st


def _act(name, v):
    if name == "silu":
        return v / (1 + torch.exp(-v))
    return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))


def _norm(form, v, w, b, eps):
    if form == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * w
    return v if b is None else v + b


EPS = 1e-6


def _plain_linear(s, real):
    x = s["x"].to(real)
    x, sx = (x, s["sx"].to(real)[:, None]) if "sx" in s else _quant(x)
    y = (x @ s["w"].to(real).t()) * sx * s["sw"].to(real)
    return y if s["bias"] is None else y + s["bias"].to(real)


def _plain_norm(s, real):
    c, up = s["case"], lambda t: None if t is None else t.to(real)  # noqa: E731
    u = up(s["a"])
    if c["post"]:
        u = _norm(c["post"], u, up(s["post_w"]), up(s["post_b"]), EPS)
    if s["gate"] is not None:
        u = u * up(s["gate"]).repeat_interleave(s["per"], 0)[: u.shape[0]]
    r = u + up(s["res"])
    y = _norm(c["pre"], r, up(s["pre_w"]), up(s["pre_b"]), EPS)
    if c["codes"]:
        codes, scale = _quant(y)
        y = codes * scale
    return r, y


def _plain_quant(s, real):
    v = s["x"].to(real)
    if s["gate"] is not None:
        v = v * _act(s["case"]["act"], s["gate"].to(real))
    codes, scale = _quant(v)
    return codes * scale, scale[:, 0]


def _plain_attend(s, real):
    """Attention over the cache as it stands."""
    c = s["case"]
    t = torch.arange(s["table"].shape[1] * c["page"], device="cuda")
    row = s["table"].long()[:, t // c["page"]] * c["page"] + t % c["page"]
    k, v = (s["kv"][i].reshape(-1, c["heads"], c["D"])[row].to(real) for i in range(2))
    if s["scales"] is not None:
        k, v = (a * s["scales"][i].reshape(-1, c["heads"])[row].to(real)[..., None] for i, a in enumerate((k, v)))
    q = s["q"].to(real).reshape(c["B"], c["heads"], c["group"], c["D"])
    seen = (t[None] < s["lens"][:, None])[:, None, None]
    score = (torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(c["D"])).masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0, top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(seen[:, 0, 0, :, None, None], v, 0)
    return (torch.matmul(p / torch.where(total == 0, 1, total), v.permute(0, 2, 1, 3).contiguous())).reshape(c["B"], -1, c["D"])


def _written(s):
    """What the step wrote into the cache: a 16-bit cache whole, of an 8-bit one the new rows as the values they stand for."""
    if s["scales"] is None:
        return s["kv"]
    H, D = s["new"].shape[2:]
    codes, scale = s["kv"].view(2, -1, H, D)[:, s["rows"]], s["scales"].view(2, -1, H, 1)[:, s["rows"]]
    return torch.mul(codes, scale, out=torch.empty(codes.shape, dtype=s["q"].dtype, device="cuda"))


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        from paper_2202_05239_amd import binding as f8
        if kind == "linear":
            if "sx" in s:
                return f8.f8_linear_scaled(s["x"], s["sx"], s["w"], s["sw"], bias=s["bias"], y_dtype=s["y"])
            return f8.f8_linear_tokens(s["x"], s["w"], s["sw"], bias=s["bias"], y_dtype=s["y"])
        if kind == "norm":
            got = f8.f8_norm_tokens(s["a"], res=s["res"], post=c["post"] or None, post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"],
                                    gate_rows=s["per"], pre=c["pre"], pre_w=s["pre_w"], pre_b=s["pre_b"], eps=EPS, codes=c["codes"])
            if not c["codes"]:
                return got
            res, codes, scale = got
            return res, torch.mul(codes, scale[:, None], out=torch.empty_like(res))
        if kind == "quant":
            return f8.f8_quant_tokens(s["x"], gate=s["gate"], act=c["act"] or None, values=True)
        cache = dict(k_scale=s["scales"][0], v_scale=s["scales"][1]) if s["scales"] is not None else {}
        f8.f8_kv_append(s["new"][0], s["new"][1], s["slots"], s["kv"][0], s["kv"][1], **cache)
        out = f8.f8_attend_paged(s["q"], s["kv"][0], s["kv"][1], s["table"], s["lens"], max_len=c["longest"], **cache)
        return {"out": out, "cache": _written(s)}
    if kind == "linear":
        return _plain_linear(s, torch.float32).to(s["y"])
    if kind == "norm":
        r, y = _plain_norm(s, torch.float32)
        return r.to(s["a"].dtype), y.to(s["a"].dtype)
    if kind == "quant":
        v, scale = _plain_quant(s, torch.float32)
        return v.to(s["x"].dtype), scale
    H, D = s["new"].shape[2:]
    there = (s["slots"] >= 0)[None, :, None, None]
    kv = s["kv"].view(2, -1, H, D)
    if s["scales"] is None:
        kv[:, s["rows"]] = torch.where(there, s["new"], kv[:, s["rows"]])
    else:
        codes, scale = _quant(s["new"].float())
        scales = s["scales"].view(2, -1, H)
        kv[:, s["rows"]] = torch.where(there, codes.to(torch.int8), kv[:, s["rows"]])
        scales[:, s["rows"]] = torch.where(there[..., 0], scale[..., 0], scales[:, s["rows"]])
    return {"out": _plain_attend(s, torch.float32).to(s["q"].dtype), "cache": _written(s)}


def work(case):
    kind = case["kind"]
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K * BYTES[case["x"]] + (4 * M if case["x"] == "s8" else 0) + N * K + 4 * N * (1 + case["bias"]) + M * N * BYTES[case["y"]],
                "flops": 2 * M * K * N}
    if kind == "norm":
        n = case["rows"] * case["C"]
        return {"bytes": 4 * n * BYTES[case["type"]] + 4 * case["C"] * BYTES[case["type"]], "flops": n * (20 if case["post"] else 12)}
    if kind == "quant":
        n = case["rows"] * case["C"]
        return {"bytes": n * BYTES[case["type"]] * (3 if case["act"] else 2) + 4 * case["rows"], "flops": n * (12 if case["act"] else 6)}
    total, H, D, new = sum(_lens(case)), case["heads"], case["D"], 2 * case["B"] * case["heads"]
    row = D * BYTES[case["cache"]] + (4 if case["cache"] == "s8" else 0)
    tables = case["B"] * 12 + 4 * -(-total // case["page"])
    return {"bytes": 2 * total * H * row + new * (D * 2 + row) + 2 * case["B"] * H * case["group"] * D * 2 + tables,
            "flops": 4 * total * H * case["group"] * D}


def _exact_linear(s):
    x = s["x"].double()
    if "sx" in s:
        sx = s["sx"].double()
    else:
        sx = torch.clamp(x.abs().max(dim=1).values / 127, min=TINY)
        x = (x / sx[:, None]).round()
    y = torch.mm(x, s["w"].double().t()) * torch.outer(sx, s["sw"].double())
    return y + s["bias"].double() if s["bias"] is not None else y


def _exact_stat(form, v, w, b):
    mean = v.sum(1, keepdim=True) / v.shape[1] if form == "layer" else torch.zeros_like(v[:, :1])
    var = ((v - mean) ** 2).sum(1, keepdim=True) / v.shape[1]
    y = (v - mean) * (var + EPS).rsqrt() * w.double()
    return y if b is None else y + b.double()


def _exact_values(v):
    scale = torch.clamp(v.abs().max(dim=-1, keepdim=True).values / 127, min=TINY)
    return (v / scale).round() * scale, scale


def _exact_norm(s):
    c = s["case"]
    u = s["a"].double()
    if c["post"]:
        u = _exact_stat(c["post"], u, s["post_w"], s["post_b"])
    if s["gate"] is not None:
        of = torch.arange(u.shape[0], device="cuda") // s["per"]
        u = s["gate"].double()[of] * u
    r = s["res"].double() + u
    y = _exact_stat(c["pre"], r, s["pre_w"], s["pre_b"])
    return r, _exact_values(y)[0] if c["codes"] else y


def _exact_quant(s):
    v = s["x"].double()
    if s["gate"] is not None:
        g = s["gate"].double()
        g = g * torch.sigmoid(g) if s["case"]["act"] == "silu" else g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))
        v = v * g
    values, scale = _exact_values(v)
    return values, scale[:, 0]


def _exact_attend(s):
    """Request by request: its pages one behind the other, the new token at the end."""
    c = s["case"]
    H, G, D, page = c["heads"], c["group"], c["D"], c["page"]
    rounded = s["new"].double()
    if s["scales"] is not None:
        rounded = _exact_values(rounded)[0]
    out = torch.zeros(c["B"], H, G, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(c)):
        if n == 0:
            continue
        ids = s["table"][b, : -(-n // page)].long()
        k, v = (s["kv"][i, ids].double().reshape(-1, H, D)[:n] for i in range(2))
        if s["scales"] is not None:
            k, v = (a * s["scales"][i, ids].double().reshape(-1, H, 1)[:n] for i, a in enumerate((k, v)))
        k[n - 1], v[n - 1] = rounded[0, b], rounded[1, b]
        q = s["q"][b].double().reshape(H, G, D)
        for h in range(H):
            w = (q[h] @ k[:, h].t() / math.sqrt(D)).softmax(-1)
            out[b, h] = w @ v[:, h]
    if s["scales"] is None:
        return {"out": out.reshape(c["B"], H * G, D), "cache": None}
    kept = s["kv"].view(2, -1, H, D)[:, s["rows"]].double() * s["scales"].view(2, -1, H, 1)[:, s["rows"]].double()
    return {"out": out.reshape(c["B"], H * G, D), "cache": torch.where((s["slots"] >= 0)[None, :, None, None], rounded, kept)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "norm": _exact_norm, "quant": _exact_quant, "attend": _exact_attend}[case["kind"]](s)
