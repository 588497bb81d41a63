"""The calls on tokens with scales from the data (quantiser, norms, products) against the definition in 64 bits.

Tolerances follow from the stated arithmetic: 32-bit steps, one rounding of the result to its type (half a unit: 2^-24, 2^-11 or
2^-8 relative for 32-bit, f16 and bf16 results, f16 also 2^-25 below its normal range).  Codes of a plain row are compared for
equality: maximum, division and rounding are single correctly rounded operations.
"""
import math

import pytest
import torch

from paper_2202_05239_amd import binding as f8

pytestmark = pytest.mark.gpu

DEV = "cuda"
TINY = 2.0 ** -126
U32 = 2.0 ** -24
HALF = {torch.float32: U32, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
REAL = [torch.float32, torch.float16, torch.bfloat16]


def rnd(y, dtype):
    """How far a correctly rounded `dtype` value may be from y."""
    return HALF[dtype] * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def tokens(g, rows, cols, dtype):
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    return x.to(dtype)


def strided(t, pad, shift):
    """The matrix `t` on the GPU with rows `pad` elements further apart, `shift` elements into its memory; NaN lies between."""
    rows, cols = t.shape
    fill = float("nan") if t.dtype.is_floating_point else 77
    big = torch.full((rows * (cols + pad) + shift,), fill, dtype=t.dtype, device=DEV)
    v = big[shift:].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def quant_ref(v):
    """Codes and scale of float32 rows, each step rounded to float32."""
    s = torch.clamp(v.abs().amax(1, keepdim=True) / torch.tensor(127.0), min=TINY)
    return torch.round(v / s), s


# ---- the quantiser --------------------------------------------------------------------------------

# one column, below and above a piece of 8, every kernel shape's edge, the widest row
WIDTHS = [1, 7, 8, 9, 511, 512, 513, 1024, 1111, 2048, 2049, 4096, 5001, 8192, 8200, 16384, 16390, 32768, 65535, 65536]


@pytest.mark.parametrize("dtype", REAL)
def test_codes_of_plain_rows_are_exact(dtype):
    for n, cols in enumerate(WIDTHS):
        x = tokens(gen(n), 5, cols, dtype)
        x[1] = 0
        for pad, shift in ((0, 0), (3, 1), (8, 8)):
            xt = strided(x, pad, shift)
            codes, scale = f8.f8_quant_tokens(xt)
            values, scale2 = f8.f8_quant_tokens(xt, values=True)
            want, s = quant_ref(x.float())
            assert torch.equal(codes.cpu().float(), want), (cols, pad)
            assert torch.equal(scale.cpu(), s[:, 0]) and torch.equal(scale2, scale)
            assert torch.equal(values.cpu(), (want * s).to(dtype)), (cols, pad)


@pytest.mark.parametrize("cols", [4097, 4100, 6143, 6144, 6145])
def test_many_rows_of_middling_width(cols):
    x = torch.randn(600, cols, generator=gen(cols)).half()
    codes, scale = f8.f8_quant_tokens(x.to(DEV))
    want, s = quant_ref(x.float())
    assert torch.equal(codes.cpu().float(), want) and torch.equal(scale.cpu(), s[:, 0])


def test_ties_and_extreme_scales():
    ties = torch.cat([torch.tensor([127.0]), torch.arange(-126, 126) + 0.5])
    rows = torch.stack([ties * f for f in (1.0, 0.37, 2.0 ** -100, 2.0 ** 100, 1e-3)])
    codes, scale = f8.f8_quant_tokens(rows.to(DEV))
    want, s = quant_ref(rows)
    assert torch.equal(codes.cpu().float(), want) and torch.equal(scale.cpu(), s[:, 0])
    small = torch.tensor([[1e-40, -3e-41, 0.0, 1e-45]])          # below 127 * 2^-126: the scale stops there
    codes, scale = f8.f8_quant_tokens(small.to(DEV))
    assert scale.item() == TINY and torch.equal(codes.cpu().float(), torch.round(small.double() / TINY).float())


def test_ties_of_the_smallest_rows():
    # quotients whose remainder lies below the normal range: ties and their neighbours, scales from 2^-126 to 2^-90
    g = gen(21)
    amax = (127 * torch.exp2(-126 + 36 * torch.rand(300, 1, generator=g)) * (1 + torch.rand(300, 1, generator=g))).float()
    s = torch.clamp(amax / torch.tensor(127.0), min=TINY)
    ties = (torch.arange(126) + 0.5) * s
    rows = torch.cat([amax, ties, torch.nextafter(ties, torch.tensor(math.inf)), -torch.nextafter(ties, torch.tensor(0.0))], 1)
    want, s = quant_ref(rows)
    codes, scale = f8.f8_quant_tokens(rows.to(DEV))
    assert torch.equal(codes.cpu().float(), want) and torch.equal(scale.cpu(), s[:, 0])
    values, _ = f8.f8_quant_tokens(rows.to(DEV), values=True)
    assert torch.equal(values.cpu(), want * s)
    # the same rows through the product, the norm without a norm, and the cache
    w, sw = torch.eye(379, dtype=torch.int8, device=DEV), torch.ones(379, device=DEV)
    for n in (1, 16, 300):
        y = f8.f8_linear_tokens(rows[:n].to(DEV), w, sw)
        assert torch.equal(y.cpu(), (want * s)[:n])
    _, codes, scale = f8.f8_norm_tokens(rows.to(DEV), pre=None, codes=True)
    assert torch.equal(codes.cpu().float(), want) and torch.equal(scale.cpu(), s[:, 0])
    heads = torch.cat([rows[:, :1], rows[:, 127:254], rows[:, 254:]], 1)[:, :240].reshape(300, 1, 240).contiguous()
    want, s = quant_ref(heads[:, 0])
    cache, scales = torch.zeros(2, 300, 1, 1, 240, dtype=torch.int8, device=DEV), torch.zeros(2, 300, 1, 1, device=DEV)
    f8.f8_kv_append(heads.to(DEV), -heads.to(DEV), torch.arange(300, device=DEV), cache[0], cache[1], scales[0], scales[1])
    for i, sign in ((0, 1), (1, -1)):
        assert torch.equal(cache[i, :, 0, 0].cpu().float(), sign * want) and torch.equal(scales[i, :, 0, 0].cpu(), s[:, 0])


def test_rows_that_are_not_finite_show_it():
    x = torch.randn(4, 300, generator=gen(1))
    x[0, 17], x[1, 299], x[2, 0] = float("nan"), float("inf"), -float("inf")
    for dtype in REAL:
        codes, scale = f8.f8_quant_tokens(x.to(dtype).to(DEV))
        values, _ = f8.f8_quant_tokens(x.to(dtype).to(DEV), values=True)
        assert not torch.isfinite(scale[:3]).any() and torch.isfinite(scale[3]).item()
        assert values[:3].isnan().all() and torch.isfinite(values[3]).all() and (codes[:3] == 0).all()
        y = f8.f8_linear_scaled(codes, scale, torch.ones(5, 300, dtype=torch.int8, device=DEV), torch.ones(5, device=DEV))
        assert y[:3].isnan().all() and torch.isfinite(y[3]).all()


@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("dtype", REAL)
def test_gated_rows(act, dtype):
    for n, (rows, cols) in enumerate([(1, 1), (3, 517), (9, 4096), (2, 11000), (700, 96)]):
        x, g = tokens(gen(n), rows, cols, dtype), (3 * torch.randn(rows, cols, generator=gen(50 + n))).to(dtype)
        codes, scale = f8.f8_quant_tokens(strided(x, 5, 2), gate=strided(g, 1, 0), act=act)
        gd, xd = g.double(), x.double()
        if act == "silu":
            gd = gd * torch.sigmoid(gd)
        elif act == "gelu":
            gd = 0.5 * gd * (1 + torch.tanh(math.sqrt(2 / math.pi) * (gd + 0.044715 * gd ** 3)))
        v = gd * xd
        s = torch.clamp(v.abs().amax(1) / 127, min=TINY)
        # v: the exponential to 2 units of its result and of its argument (u <= 40 where it matters: 40 units), sum, quotient, product
        rel = 50 * U32
        assert ((scale.cpu().double() - s).abs() <= 2 * rel * s).all()
        assert ((codes.cpu().double() - v / s[:, None]).abs() <= 0.5 + 127 * 4 * rel).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gates_in_32_bits(act):
    """Rows of one column, whose scale is |act(g)| / 127.  silu: exponential to 2 units in the last place, sum, quotient, division by
    127: 4 + 3 half units, 8 allowed.  gelu: its argument u is off by 5 half units relative, which are |u| times as many of the result."""
    low = -84.0 if act == "silu" else -9.0
    g = torch.cat([torch.linspace(low, 30, 4096), torch.linspace(-1, 1, 1001), torch.tensor([-20.5, -40.25, -60.125, -80.0625]).clamp_min(low)])[:, None]
    codes, scale = f8.f8_quant_tokens(torch.ones_like(g).to(DEV), gate=g.to(DEV), act=act)
    gd = g.double()[:, 0]
    u = gd if act == "silu" else 2 * math.sqrt(2 / math.pi) * (gd + 0.044715 * gd ** 3)
    want = gd / (1 + torch.exp(-u)) / 127
    tol = (8 + (5 * u.abs() if act == "gelu" else 0)) * U32
    assert ((scale.cpu().double() - want.abs()).abs() <= tol * want.abs() + TINY).all()
    assert torch.equal(codes.cpu()[:, 0].sign().int(), want.sign().int())


def test_extreme_gates():
    g = torch.tensor([[-1e4, -88.0, -100.0, 0.0, 1e4, 30.0, -30.0, 3e38]])
    for act in ("silu", "gelu"):
        values, scale = f8.f8_quant_tokens(torch.ones_like(g).to(DEV), gate=g.to(DEV), act=act, values=True)
        assert torch.isfinite(scale).all() and values[0, 7].item() == pytest.approx(3e38, rel=1e-6) and (values[0, :4] == 0).all()


def test_quantiser_in_place_and_empty():
    x = tokens(gen(3), 40, 640, torch.bfloat16).to(DEV)
    want, s = f8.f8_quant_tokens(x, values=True)
    got, s2 = f8.f8_quant_tokens(x, values=True, out=x)
    assert got.data_ptr() == x.data_ptr() and torch.equal(got, want) and torch.equal(s, s2)
    codes, scale = f8.f8_quant_tokens(torch.empty(0, 64, device=DEV))
    assert codes.shape == (0, 64) and scale.shape == (0,)


# ---- the norms ------------------------------------------------------------------------------------

def norm_ref(form, v, w, b, eps):
    if form is None:
        return v
    if form == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    return v * (1 if w is None else w.double()) + (0 if b is None else b.double())


@pytest.mark.parametrize("dtype", REAL)
@pytest.mark.parametrize("post,pre", [(None, "rms"), ("rms", "rms"), ("layer", "layer"), ("rms", None), (None, "layer"), (None, None)])
def test_norms(dtype, post, pre):
    for n, (rows, cols) in enumerate([(1, 1), (1, 4096), (6, 9), (5, 512), (9, 1001), (3, 2050), (17, 4096), (2, 8200), (2, 40000)]):
        g = gen(n)
        a, res = tokens(g, rows, cols, dtype), tokens(g, rows, cols, dtype)
        wt = dtype if n % 2 else torch.float32
        vec = lambda: (1 + 0.2 * torch.randn(cols, generator=g)).to(wt)  # noqa: E731
        pw, pb, qw, qb = (vec() if k & n else None for k in (1, 2, 1, 4))
        per = 4
        gate = (0.5 + torch.randn(-(-rows // per), cols, generator=g)).to(dtype) if n % 3 else None
        alpha, eps = (0.7, 1e-5) if n % 2 else (1.0, 1e-6)
        pad, shift = ((0, 0), (8, 8), (3, 1))[n % 3]
        up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        r, y = f8.f8_norm_tokens(strided(a, pad, shift), res=strided(res, pad, shift) if n % 4 != 3 else None, post=post, post_w=up(pw), post_b=up(pb),
                                 gate=up(gate), gate_rows=per if gate is not None else None, res_scale=alpha, pre=pre, pre_w=up(qw), pre_b=up(qb), eps=eps)
        u = norm_ref(post, a.double(), pw, pb, eps)
        if gate is not None:
            u = u * gate.double().repeat_interleave(per, 0)[:rows]
        want_r = u + (alpha * res.double() if n % 4 != 3 else 0)
        want_y = norm_ref(pre, want_r, qw, qb, eps)
        # elementwise steps: a few units of the largest magnitude that enters; the statistics of a row: log2(threads) + 64 sums in
        # 32 bits, relative (64 + 16) U32 of the root; the centring of a layer norm loses units of the mean's size
        row = lambda t: t.abs().amax(1, keepdim=True)  # noqa: E731
        slack_u = 100 * U32 * (row(u) + 1)
        err_r = slack_u + 4 * U32 * (row(res.double()) + row(want_r))
        assert ((r.cpu().double() - want_r).abs() <= rnd(want_r, dtype) + err_r).all(), (rows, cols)
        if pre is None:
            err_y = err_r
        else:
            c = want_r - (want_r.mean(1, keepdim=True) if pre == "layer" else 0)
            size = torch.sqrt((c * c).mean(1, keepdim=True) + eps)
            err_y = 100 * U32 * row(want_y) + 2 * (err_r + 8 * U32 * row(want_r)) / size * 2 * (1 + row(want_y))
        assert ((y.cpu().double() - want_y).abs() <= rnd(want_y, dtype) + err_y).all(), (rows, cols)


def test_norm_into_codes_is_the_quantised_norm():
    for n, (rows, cols) in enumerate([(1, 64), (3, 1111), (64, 4096), (5, 6000)]):
        for dtype in REAL:
            a, res = tokens(gen(n), rows, cols, dtype).to(DEV), tokens(gen(9 + n), rows, cols, dtype).to(DEV)
            w = (1 + 0.1 * torch.randn(cols, generator=gen(n))).to(DEV)
            r, codes, scale = f8.f8_norm_tokens(a, res=res, pre="rms", pre_w=w, codes=True)
            r2, y = f8.f8_norm_tokens(a.float(), res=res.float(), pre="rms", pre_w=w)
            want, s = f8.f8_quant_tokens(y)
            assert torch.equal(codes, want) and torch.equal(scale, s) and torch.equal(r, r2.to(dtype))


def test_norm_in_place_and_partial_results():
    a, res = tokens(gen(1), 30, 768, torch.bfloat16).to(DEV), tokens(gen(2), 30, 768, torch.bfloat16).to(DEV)
    r, y = f8.f8_norm_tokens(a, res=res, pre="rms")
    none, y2 = f8.f8_norm_tokens(a, res=res, pre="rms", keep_res=False)
    assert none is None and torch.equal(y, y2)
    r3, y3 = f8.f8_norm_tokens(a, res=res, pre="rms", res_out=res, out=a)
    assert r3.data_ptr() == res.data_ptr() and torch.equal(r3, r) and torch.equal(y3, y)


def test_norm_keeps_nan_in_its_row():
    a = torch.randn(3, 700, generator=gen(1)).to(DEV)
    a[1, 5] = float("nan")
    r, y = f8.f8_norm_tokens(a, pre="layer")
    assert y[1].isnan().all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()
    z = torch.zeros(2, 96, device=DEV)
    assert (f8.f8_norm_tokens(z, pre="rms")[1] == 0).all() and (f8.f8_norm_tokens(z + 5, pre="layer")[1] == 0).all()


def test_norm_of_no_rows():
    a = torch.empty(0, 64, dtype=torch.float16, device=DEV)
    for gate in (None, torch.ones(1, 64, dtype=torch.float16, device=DEV), torch.ones(0, 64, dtype=torch.float16, device=DEV)):
        r, y = f8.f8_norm_tokens(a, gate=gate)
        assert r.shape == (0, 64) and y.shape == (0, 64)
        r, codes, scale = f8.f8_norm_tokens(a, res=a, gate=gate, codes=True)
        assert codes.shape == (0, 64) and scale.shape == (0,)


# ---- the products ---------------------------------------------------------------------------------

def codes_of(g, rows, cols):
    t = torch.randint(-128, 128, (rows, cols), generator=g, dtype=torch.int32).to(torch.int8)
    t[0, 0] = -128
    return t


def linear_ref(x, sx, w, sw, b):
    acc = (x.double() @ w.double().t())
    y = acc * sx.double()[:, None] * sw.double()
    return y + (0 if b is None else b.double())


# one and few tokens, every tile's edge, long sums, sizes that divide by nothing
SHAPES = [(1, 1, 1), (1, 4096, 64), (1, 100, 7), (2, 4096, 1000), (3, 65, 129), (4, 4097, 33), (7, 512, 300), (16, 2048, 1000), (17, 2050, 96),
          (31, 8192, 257), (48, 4096, 640), (64, 1024, 1024), (65, 300, 500), (100, 16384, 130), (128, 128, 128), (129, 640, 257), (200, 4100, 513),
          (256, 2048, 1000), (300, 129, 1031), (513, 1536, 520), (520, 4096, 2056), (1031, 777, 333), (2048, 512, 2304)]


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_products_of_codes(M, K, N):
    g = gen(M + K + N)
    x, w = codes_of(g, M, K), codes_of(g, N, K)
    sx, sw = torch.rand(M, generator=g) * 0.02 + 1e-4, torch.rand(N, generator=g) * 0.01 + 1e-4
    b = torch.randn(N, generator=g) if M % 2 else None
    want = linear_ref(x, sx, w, sw, b)
    for n, dtype in enumerate(REAL):
        for pad, shift in ((0, 0), (16, 16), (5, 3))[: 3 if M * N * K < 1 << 27 else 1 + n]:
            y = f8.f8_linear_scaled(strided(x, pad, shift), sx.to(DEV), strided(w, pad, shift), sw.to(DEV), bias=None if b is None else b.to(DEV),
                                    y=strided(torch.zeros(M, N, dtype=dtype), pad, shift)).cpu()
            # the sum into 32-bit floating point, two products, one sum
            err = 4 * U32 * (want.abs() + (0 if b is None else b.double().abs()))
            assert ((y.double() - want).abs() <= rnd(want, dtype) + err).all(), (dtype, pad)


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_products_of_real_tokens_are_those_of_their_codes(M, K, N):
    g = gen(M * 3 + K + N)
    w, sw = codes_of(g, N, K), torch.rand(N, generator=g) * 0.01 + 1e-4
    for dtype in REAL:
        x = tokens(g, M, K, dtype)
        if M > 2:
            x[M // 2] = 0
        for pad, shift in ((0, 0), (3, 1)):
            xt, wt = strided(x, pad, shift), strided(w, pad, shift)
            y = f8.f8_linear_tokens(xt, wt, sw.to(DEV), y_dtype=torch.float32)
            codes, scale = f8.f8_quant_tokens(xt)
            assert torch.equal(y, f8.f8_linear_scaled(codes, scale, wt, sw.to(DEV), y_dtype=torch.float32)), (dtype, pad)


@pytest.mark.parametrize("M,K,N", [(4096, 1024, 5000), (5231, 1024, 6386), (5000, 2048, 4096), (7275, 512, 5251), (2570, 528, 8450)])
def test_products_in_two_parts(M, K, N):
    # sizes that leave a thin last round of tiles: whole rounds of one tile and a second launch over the rest, with bias and pads
    g = torch.Generator(device=DEV).manual_seed(M)
    x, w = (torch.randint(-128, 128, s, generator=g, device=DEV, dtype=torch.int32).to(torch.int8) for s in ((M, K), (N, K)))
    sx, sw, b = (torch.rand(n, generator=g, device=DEV) for n in (M, N, N))
    want = linear_ref(x, sx, w, sw, b)
    big = torch.full((M, N + 3), 7.0, device=DEV)
    y = f8.f8_linear_scaled(x, sx, w, sw, bias=b, y=big[:, :N])
    assert ((y.double() - want).abs() <= 5 * U32 * (want.abs() + b.double())).all() and (big[:, N:] == 7).all()


def test_largest_sums_are_exact():
    K = 131071
    x, w = torch.full((3, K), -128, dtype=torch.int8), torch.full((40, K), -128, dtype=torch.int8)
    w[1] = 127
    w[2, ::2] = 0
    want = (x.double() @ w.double().t())
    y = f8.f8_linear_scaled(x.to(DEV), torch.ones(3, device=DEV), w.to(DEV), torch.ones(40, device=DEV), y_dtype=torch.float32).cpu()
    assert ((y.double() - want).abs() <= U32 * want.abs()).all()


def test_products_repeat_and_replay():
    g = gen(5)
    x, w, sw = tokens(g, 70, 2048, torch.bfloat16).to(DEV), codes_of(g, 1536, 2048).to(DEV), torch.rand(1536, generator=g).to(DEV)
    ws = torch.empty(f8.lib().f8_linear_workspace_bytes(70, 2048), dtype=torch.uint8, device=DEV)
    y = torch.empty(70, 1536, dtype=torch.bfloat16, device=DEV)
    want = f8.f8_linear_tokens(x, w, sw).clone()
    graph = torch.cuda.CUDAGraph()
    f8.f8_linear_tokens(x, w, sw, y=y, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        f8.f8_linear_tokens(x, w, sw, y=y, workspace=ws)
    for _ in range(3):
        y.zero_()
        ws.fill_(0x55)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_few_short_tokens_need_no_workspace():
    g = gen(8)
    for M, K in ((1, 4096), (8, 512), (2, 2048), (3, 1000)):
        assert f8.lib().f8_linear_workspace_bytes(M, K) == 0
        x, w, sw = tokens(g, M, K, torch.bfloat16).to(DEV), codes_of(g, 9000, K).to(DEV), torch.rand(9000, generator=g).to(DEV)
        codes, scale = f8.f8_quant_tokens(x)
        for n in (100, 9000):
            y = f8.f8_linear_tokens(x, w[:n], sw[:n], y_dtype=torch.float32)
            assert torch.equal(y, f8.f8_linear_scaled(codes, scale, w[:n], sw[:n], y_dtype=torch.float32))


def test_another_stream():
    g = gen(6)
    x, w, sw = tokens(g, 9, 1024, torch.float16).to(DEV), codes_of(g, 512, 1024).to(DEV), torch.rand(512, generator=g).to(DEV)
    want = f8.f8_linear_tokens(x, w, sw)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = f8.f8_linear_tokens(x, w, sw)
        torch.cuda.current_stream().synchronize()
    assert torch.equal(got, want)


def test_empty_products():
    w, sw = torch.zeros(8, 32, dtype=torch.int8, device=DEV), torch.ones(8, device=DEV)
    assert f8.f8_linear_tokens(torch.empty(0, 32, device=DEV), w, sw).shape == (0, 8)
