"""Paged attention of one new token and the cache it reads, against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2202_05239_amd import binding as f8

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"s8": torch.int8, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


class Cache:
    """A cache filled at random, and the table of requests of the given lengths; everything a request does not own is NaN (codes:
    127 with NaN scales)."""

    def __init__(self, seed, lens, heads, D, page, kind, heads_first=False, spare=3, wide=0):
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in lens]
        self.pages, self.page, self.kind, self.lens = sum(need) + spare, page, kind, lens
        perm = torch.randperm(self.pages, generator=g).int()
        cols = max(1, max(need)) + wide
        self.table = torch.full((len(lens), cols), -1, dtype=torch.int32)
        at = 0
        real = torch.zeros(self.pages, page, dtype=torch.bool)
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            for i in range(n):
                real[perm[at + i], : min(page, lens[b] - i * page)] = True
            at += n
        kv = torch.randn(2, self.pages, page, heads, D, generator=g) * torch.exp(0.7 * torch.randn(2, self.pages, page, heads, 1, generator=g))
        self.scales = None
        dead = ~real[None, :, :, None]
        if kind == "s8":
            s = torch.clamp(kv.abs().amax(-1) / 127, min=2.0 ** -126)
            kv = torch.round(kv / s[..., None])
            kv[dead.expand(2, -1, -1, heads)] = 127
            self.scales = s.masked_fill(dead.expand_as(s), float("nan"))
        else:
            kv = kv.masked_fill(dead[..., None].expand_as(kv), float("nan"))
        self.kv = kv.to(TYPES[kind])
        dev = self.kv.to(DEV)
        sc = None if self.scales is None else self.scales.to(DEV)
        if heads_first:                                   # the same cache with places behind heads in memory
            dev = dev.transpose(2, 3).contiguous().transpose(2, 3)
            sc = None if sc is None else sc.transpose(2, 3).contiguous().transpose(2, 3)
        self.dev, self.dev_scales = dev, sc

    def args(self):
        return dict(k_cache=self.dev[0], v_cache=self.dev[1], **({} if self.dev_scales is None else
                    dict(k_scale=self.dev_scales[0], v_scale=self.dev_scales[1])))

    def rows(self, b):
        n = self.lens[b]
        ids = self.table[b, : -(-n // self.page)].long()
        kv = self.kv[:, ids].double()
        if self.scales is not None:
            kv = kv * self.scales[:, ids].double()[..., None]
        return kv.flatten(1, 2)[:, :n]                     # [2][n][heads][D]


def check(c, q, out, scale, skip=None):
    """out against softmax(scale q k) v.  Errors: a score's sum of D products and its scaling in 32 bits, q in f16 under 8-bit keys
    (2^-25 of its largest element), twice that relative in each weight; a weight's rounding to 16 bits (f16 also 2^-25 of the
    largest weight below its normal range); the result's own."""
    B, Hq, D = q.shape
    heads = c.kv.shape[3]
    kind = torch.float16 if c.kind == "s8" else c.kv.dtype
    for b in range(B):
        if c.lens[b] == 0:
            assert (out[b] == 0).all()
            continue
        k, v = c.rows(b)
        if skip is not None:
            k, v = k[skip], v[skip]
        k, v = (t.repeat_interleave(Hq // heads, 1) for t in (k, v))
        qd = q[b].double()
        s = torch.einsum("hd,nhd->hn", qd, k) * scale
        p = s.softmax(-1)
        want = torch.einsum("hn,nhd->hd", p, v)
        size = torch.einsum("hd,nhd->hn", qd.abs(), k.abs()).amax(-1) * abs(scale)
        delta = (D + 8) * 2.0 ** -24 * (size + s.abs().amax(-1) + 1)
        if c.kind == "s8":
            delta = delta + D * 2.0 ** -25 * qd.abs().amax(-1) * k.abs().amax((0, 2)) * abs(scale)
        mass = torch.einsum("hn,nhd->hd", p, v.abs())
        tiny = len(v) * 2.0 ** -25 * (p[..., None] * v.permute(1, 0, 2).abs().amax(-1, keepdim=True)).amax((1, 2))
        err = mass * (HALF[kind] + 4 * delta[:, None]) + (tiny[:, None] if kind == torch.float16 else 0) + HALF[q.dtype] * want.abs() + 2.0 ** -25
        far = ((out[b].double() - want).abs() - err).max().item()
        assert far <= 0, (b, c.lens[b], far)


def run(c, B, Hq, D, dtype, seed=0, scale=None, **kw):
    q = (torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype)
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=torch.tensor(c.lens, dtype=torch.int32, device=DEV), scale=scale, **c.args(), **kw)
    return q, out.cpu()


KINDS = [("s8", torch.bfloat16), ("s8", torch.float16), ("f16", torch.float16), ("bf16", torch.bfloat16)]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 144, 192, 256])
def test_lengths_pages_and_groups(kind, dtype, D):
    # no token, one, around a tile of 32, around a workgroup's round of 128, and longer; pages that end inside a tile
    lens = [0, 1, 2, 31, 32, 33, 63, 127, 128, 129, 300, 517]
    for n, (heads, group, page) in enumerate([(1, 1, 16), (2, 3, 1), (3, 8, 24), (1, 16, 7), (2, 17, 64), (1, 40, 128)]):
        c = Cache(n + D, lens, heads, D, page, kind, heads_first=n % 2 == 1)
        q, out = run(c, len(lens), heads * group, D, dtype)
        check(c, q, out, D ** -0.5)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_long_contexts_are_split_and_joined(kind, dtype):
    for lens, heads, group in (([20000], 1, 4), ([9001, 0, 1, 4097], 2, 8), ([3000, 129], 1, 20)):
        c = Cache(7, lens, heads, 128, 32, kind)
        q, out = run(c, len(lens), heads * group, 128, dtype)
        check(c, q, out, 128 ** -0.5)
        # a bound above the longest only changes how the length is shared out
        c2 = Cache(7, lens, heads, 128, 32, kind, wide=200)
        q2, out2 = run(c2, len(lens), heads * group, 128, dtype)
        check(c2, q2, out2, 128 ** -0.5)


@pytest.mark.parametrize("B,heads,group,kind", [(257, 1, 2, "s8"), (700, 2, 1, "bf16"), (1100, 1, 17, "s8")])
def test_many_requests(B, heads, group, kind):
    # more requests than are looked through at a time, stretches of empty ones among them, some far longer than the others
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 90, (B,), generator=g)
    lens[torch.rand(B, generator=g) < 0.3] = 0
    lens[B // 3:B // 3 + 100] = 0
    for i, n in ((0, 700), (B // 2, 1500), (B - 1, 640), (B - 2, 0)):
        lens[i] = n
    c = Cache(B, lens.tolist(), heads, 32, 16, kind)
    dtype = torch.bfloat16 if kind == "bf16" else torch.float16
    q, out = run(c, B, heads * group, 32, dtype)
    check(c, q, out, 32 ** -0.5)
    c.lens = [0] * B                                             # nobody has a token
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=torch.zeros(B, dtype=torch.int32, device=DEV), **c.args())
    assert (out == 0).all()


@pytest.mark.parametrize("heads,group,D,dtype", [(2, 3, 64, torch.float16), (4, 16, 80, torch.bfloat16), (2, 17, 128, torch.bfloat16), (6, 1, 16, torch.float16)])
def test_two_heads_side_by_side(heads, group, D, dtype):
    # enough requests and tokens that a workgroup takes two heads of an 8-bit cache at a time, in either order of the cache
    lens = [4500, 0, 1, 63, 64, 65, 128, 129, 700, 31, 2, 1000, 96, 0, 33, 640, 5, 3200]
    for first in (False, True):
        c = Cache(heads + D, lens, heads, D, 24, "s8", heads_first=first, wide=200)
        q, out = run(c, len(lens), heads * group, D, dtype)
        check(c, q, out, D ** -0.5)


def test_scores_far_apart_and_scales_far_apart():
    c = Cache(3, [700, 40], 2, 64, 16, "s8")
    q, out = run(c, 2, 4, 64, torch.float16, scale=4.0)           # one token takes all the weight
    check(c, q, out, 4.0)
    q, out = run(c, 2, 4, 64, torch.float16, scale=0.0)           # every token the same
    check(c, q, out, 0.0)
    c.scales[1] *= 1e-6                                           # values far below what 16 bits hold
    c.dev_scales.copy_(c.scales)
    q, out = run(c, 2, 4, 64, torch.bfloat16)
    k, v = c.rows(0)
    p = (torch.einsum("hd,nhd->hn", q[0].double(), k.repeat_interleave(2, 1)) / 8).softmax(-1)
    want = torch.einsum("hn,nhd->hd", p, v.repeat_interleave(2, 1))
    assert ((out[0].double() - want).norm() <= 2.0 ** -8 * want.norm())


def test_rows_of_zeros():
    c = Cache(4, [50], 1, 64, 16, "s8")
    c.scales[:] = torch.where(c.scales.isnan(), c.scales, torch.tensor(2.0 ** -126))
    c.kv.zero_()
    c.dev.zero_()
    c.dev_scales.copy_(c.scales)
    _, out = run(c, 1, 2, 64, torch.float16)
    assert (out == 0).all()


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_table_entries_outside_the_cache_are_left_out(kind, dtype):
    c = Cache(5, [100, 64], 2, 64, 16, kind)
    for bad in (-1, -2 ** 31, c.pages, 2 ** 31 - 1):
        c2 = Cache(5, [100, 64], 2, 64, 16, kind)
        c2.table[0, 2] = bad
        c2.table[1] = bad                                        # nothing left of this one
        q, out = run(c2, 2, 4, 64, dtype)
        keep = torch.ones(100, dtype=torch.bool)
        keep[32:48] = False
        assert (out[1] == 0).all()
        c2.table, c2.lens = c.table, [100, 0]
        check(c2, q, out, 0.125, skip=keep)


def test_nan_stays_where_it_belongs():
    c = Cache(6, [70, 33], 1, 64, 16, "bf16")
    page = c.table[0, 1].item()
    c.dev[1, page, 3, 0, 5] = float("nan")                       # a value of request 0, dimension 5
    q, out = run(c, 2, 2, 64, torch.bfloat16)
    assert out[0, :, 5].isnan().all() and out[0].isnan().sum() == 2 and torch.isfinite(out[1]).all()
    c.dev[0, page, 3, 0, 5] = float("nan")                       # a key: its score, and everything of that request
    q, out = run(c, 2, 2, 64, torch.bfloat16)
    assert out[0].isnan().all() and torch.isfinite(out[1]).all()


def test_lens_beyond_the_bound_are_clamped():
    c = Cache(8, [90, 33], 1, 64, 16, "f16")
    lens = torch.tensor([90, -5], dtype=torch.int32, device=DEV)
    q = torch.randn(2, 2, 64).half()
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=lens, max_len=48, **c.args()).cpu()
    c.lens = [48, 0]
    check(c, q, out, 0.125)


def test_a_batch_without_pages():
    c = Cache(12, [20], 2, 64, 16, "s8")
    out = f8.f8_attend_paged(torch.randn(3, 4, 64).half().to(DEV), table=torch.zeros(3, 0, dtype=torch.int32, device=DEV),
                             lens=torch.tensor([0, 5, 0], dtype=torch.int32, device=DEV), **c.args())
    assert out.shape == (3, 4, 64) and (out == 0).all()
    none = f8.f8_attend_paged(torch.empty(0, 4, 64, dtype=torch.float16, device=DEV), table=torch.zeros(0, 2, dtype=torch.int32, device=DEV),
                              lens=torch.zeros(0, dtype=torch.int32, device=DEV), **c.args())
    assert none.shape == (0, 4, 64)


def test_strided_queries_and_results():
    c = Cache(9, [200, 17], 2, 64, 16, "s8")
    big = torch.randn(2, 3, 4, 80, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    q, out = big[:, 1, :, 8:72], torch.full((4, 2, 70), 9.0, dtype=torch.float16, device=DEV)
    view = out.transpose(0, 1)[..., 3:67]
    f8.f8_attend_paged(q, table=c.table.to(DEV), lens=torch.tensor(c.lens, dtype=torch.int32, device=DEV), out=view, **c.args())
    check(c, q.cpu(), view.cpu(), 0.125)
    assert (out[..., :3] == 9).all() and (out[..., 67:] == 9).all()


def test_offsets_beyond_32_bits():
    # one page far behind 4 GiB of others, which are never touched
    pages, page, heads, D = 40000, 64, 8, 128                    # 2.6 GB of codes an array, strides of 5.2 GB
    flat = torch.empty(pages * page * heads * D * 2, dtype=torch.int8, device=DEV)
    kv = flat.view(pages, 2, page, heads, D).transpose(0, 1)
    scales = torch.empty(2, pages, page, heads, device=DEV)
    c = Cache(10, [64 * 3 - 5], heads, D, page, "s8", spare=0)
    ids = torch.tensor([pages - 1, 7, pages - 2])
    old = c.table[0].long()
    kv[:, ids] = c.dev[:, old.to(DEV)]
    scales[:, ids] = c.dev_scales[:, old.to(DEV)]
    q = torch.randn(1, heads * 2, D).bfloat16()
    out = f8.f8_attend_paged(q.to(DEV), kv[0], kv[1], ids[None].int().to(DEV), torch.tensor(c.lens, dtype=torch.int32, device=DEV),
                             k_scale=scales[0], v_scale=scales[1]).cpu()
    check(c, q, out, D ** -0.5)
    # and the writer puts rows there
    new = torch.randn(2, 1, heads, D).to(DEV)
    slot = torch.tensor([(pages - 1) * page + 63], device=DEV)
    f8.f8_kv_append(new[0], new[1], slot, kv[0], kv[1], scales[0], scales[1])
    codes, s = f8.f8_quant_tokens(new.view(-1, D))
    assert torch.equal(kv[:, pages - 1, 63], codes.view(2, heads, D)) and torch.equal(scales[:, pages - 1, 63], s.view(2, heads))


@pytest.mark.parametrize("kind", ["s8", "f16", "bf16"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_append(kind, dtype):
    g = torch.Generator().manual_seed(2)
    for n, (tokens, heads, D, page) in enumerate([(1, 1, 16, 1), (5, 3, 64, 16), (40, 2, 128, 24), (3, 5, 144, 7), (9, 2, 256, 32)]):
        pages = tokens + 3
        first = torch.zeros(2, pages, page, heads, D, dtype=TYPES[kind])
        kv, scales = first.to(DEV), torch.full((2, pages, page, heads), 5.0, device=DEV)
        if n % 2:
            kv = kv.transpose(2, 3).contiguous().transpose(2, 3)
        src = torch.randn(tokens, 2, heads, D + (1 if n == 3 else 0), generator=g).to(dtype)[..., :D]
        slots = torch.randperm(pages * page, generator=g)[:tokens]
        if tokens > 2:
            slots[1], slots[2] = -1, pages * page                # nowhere
        x = src.to(DEV)
        f8.f8_kv_append(x[:, 0], x[:, 1], slots.to(DEV), kv[0], kv[1], *((scales[0], scales[1]) if kind == "s8" else ()))
        want, ws = first.clone(), torch.full((2, pages, page, heads), 5.0)
        for t, s in enumerate(slots.tolist()):
            if not 0 <= s < pages * page:
                continue
            for i in range(2):
                if kind == "s8":
                    v = src[t, i].float()
                    sc = torch.clamp(v.abs().amax(-1) / torch.tensor(127.0), min=2.0 ** -126)
                    want[i, s // page, s % page], ws[i, s // page, s % page] = torch.round(v / sc[:, None]).to(torch.int8), sc
                else:
                    want[i, s // page, s % page] = src[t, i].float().to(TYPES[kind])
        assert torch.equal(kv.cpu(), want), n
        assert torch.equal(scales.cpu(), ws)


def test_repeats_and_replays():
    c = Cache(11, [5000, 77], 2, 128, 16, "s8")
    q = torch.randn(2, 8, 128).bfloat16().to(DEV)
    table, lens = c.table.to(DEV), torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(16, f8.lib().f8_attend_workspace_bytes(2, 8, 2, 128, 5000)), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    want = f8.f8_attend_paged(q, table=table, lens=lens, max_len=5000, **c.args()).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f8.f8_attend_paged(q, table=table, lens=lens, max_len=5000, out=out, workspace=ws, **c.args())
    for _ in range(3):
        out.zero_()
        ws.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    # another length under the same graph: the lengths are read on the device
    lens.copy_(torch.tensor([1000, 5], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, f8.f8_attend_paged(q, table=table, lens=lens, max_len=5000, **c.args()))


def blank_values(c, b, first, last, scale):
    """Tokens first .. last - 1 of request b have value rows of zeros with the given scale (their keys stay)."""
    for t in range(first, last):
        at = (1, c.table[b, t // c.page].long(), t % c.page)
        c.kv[at], c.scales[at] = 0, scale
    c.dev[1].copy_(c.kv[1])
    c.dev_scales[1].copy_(c.scales[1])


# a wave's first tile, a tile in the middle, a workgroup's round, several runs of a long context, all but the last token, everything
BLANK = [(0, 32), (64, 96), (0, 128), (37, 300), (0, 4000), (1024, 3000), (0, -1), (0, None)]


@pytest.mark.parametrize("scale", [2.0 ** -126, 0.0])
@pytest.mark.parametrize("lens,heads,group", [([300, 40], 2, 4), ([513, 1, 129], 1, 1), ([6000, 0, 4097], 2, 8), ([4500, 700] + [300] * 16, 4, 2)])
def test_stretches_of_zero_values(lens, heads, group, scale):
    # in one launch, in two, and two heads side by side; scores that are all alike (scale 0) and scores that differ
    for first, last in BLANK:
        c = Cache(13 + heads, lens, heads, 64, 16, "s8", wide=200 if len(lens) > 8 else 0)
        for b, n in enumerate(lens[:3]):
            end = n if last is None else n + last if last < 0 else min(last, n)
            blank_values(c, b, min(first, n), max(end, 0), scale)
        for s in (0.0, 0.125, 1.0):
            q, out = run(c, len(lens), heads * group, 64, torch.bfloat16, scale=s)
            assert torch.isfinite(out).all()
            check(c, q, out, s)


def test_values_of_every_size():
    # scales of values from 2^-80 to 2^100 in one request, each token's weight such that all of them count alike (or, for the second
    # head, the large ones), and rows of zeros with the largest weights of all
    n, D = 640, 64
    c = Cache(14, [n], 1, D, 16, "s8")
    g = torch.Generator().manual_seed(2)
    t = torch.arange(n)
    at = (c.table[0, t // 16].long(), t % 16)
    size = torch.linspace(-80, 100, n)[torch.randperm(n, generator=g)]
    none = torch.rand(n, generator=g) < 0.1
    score = torch.where(none, 200.0, 120 - size)
    kv, scales = c.kv[:, at[0], at[1], 0], c.scales[:, at[0], at[1], 0]
    kv[0] = 0
    kv[0, :, 0] = 127                                             # keys: one element
    kv[1, none] = 0
    scales[0] = score / 127
    scales[1] = torch.where(none, torch.tensor(2.0 ** -126), torch.exp2(size))
    c.kv[:, at[0], at[1], 0], c.scales[:, at[0], at[1], 0] = kv, scales
    c.dev.copy_(c.kv)
    c.dev_scales.copy_(c.scales)
    q = torch.zeros(1, 2, D)
    q[0, 0, 0], q[0, 1, 0] = 1, 0.5
    q = q.bfloat16()
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=torch.tensor([n], dtype=torch.int32, device=DEV), scale=math.log(2), **c.args()).cpu()
    k, v = (x[:, 0] for x in c.rows(0))
    for h in range(2):
        want = (k @ q[0, h].double() * math.log(2)).softmax(0) @ v
        assert (out[0, h].double() - want).norm() <= 2.0 ** -7 * want.norm()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_of_an_8_bit_cache_that_are_not_finite(bad):
    # their scale is not finite: everything of that request is NaN, beside rows of zeros too
    for n in (40, 3000):
        c = Cache(17, [n, 33], 1, 64, 16, "s8")
        blank_values(c, 0, 0, n - 1, 2.0 ** -126)
        c.dev_scales[1, c.table[0, (n - 1) // 16].item(), (n - 1) % 16] = bad
        c.dev[1, c.table[0, (n - 1) // 16].item(), (n - 1) % 16] = 0
        q, out = run(c, 2, 2, 64, torch.bfloat16)
        assert out[0].isnan().all() and torch.isfinite(out[1]).all()


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("nats", [6, 10, 14, 17, 20, 24])
def test_many_small_weights_beside_a_large_one(kind, dtype, nats):
    """One token with nearly all the weight and a value in dimension 0 only: the other dimensions are the sum of the others' small
    weights.  Errors: those of check(), but a weight's rounding stays relative down to 2^-29 of the largest weight (its type's
    normal range, with the largest one brought to 2^15), and what lies below is off by 2^-40 of the largest.  So many requests that a
    workgroup has one whole request, and a wave of it a quarter of the tokens, the large one among its first; all read the same pages."""
    n, D, B, one = 2000, 64, 512, 5
    g = torch.Generator().manual_seed(nats)
    c = Cache(15, [n], 1, D, 16, kind)
    t = torch.arange(n)
    pg, pl = c.table[0, t // 16].long(), t % 16
    k, v = torch.zeros(n, D), 1 + torch.rand(n, D, generator=g)
    k[one, 0] = 1
    v[one] = 0
    v[one, 0] = 1.5
    for i, x in enumerate((k, v)):
        if kind == "s8":
            s = torch.clamp(x.abs().amax(1) / 127, min=2.0 ** -126)
            c.scales[i, pg, pl, 0] = s
            x = torch.round(x / s[:, None])
        c.kv[i, pg, pl, 0] = x.to(c.kv.dtype)
    c.dev.copy_(c.kv)
    if kind == "s8":
        c.dev_scales.copy_(c.scales)
    q = torch.zeros(B, 2, D, dtype=dtype)
    q[:, :, 0] = 1
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV).repeat(B, 1), lens=torch.full((B,), n, dtype=torch.int32, device=DEV),
                             scale=float(nats), **c.args()).cpu()
    k, v = (x[:, 0] for x in c.rows(0))
    p = (k[:, 0] * nats).softmax(0)
    want = p @ v
    delta = (D + 8) * 2.0 ** -24 * (2 * nats + 1) + (D * 2.0 ** -25 * nats if kind == "s8" else 0)
    half = HALF[torch.bfloat16 if kind == "bf16" else torch.float16]
    err = (p @ v.abs()) * (half + 4 * delta) + n * 2.0 ** -40 * 2 + HALF[dtype] * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0)
    assert ((out.double() - want).abs() <= err).all(), ((out.double() - want).abs() / want).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_small_elements_of_a_query_beside_a_large_one(dtype):
    """8-bit keys that are zero where the query is largest: the scores are those of its small elements, which lose nothing down to
    2^-28 of the largest.  Error of a score: its sum in 32 bits."""
    n, D = 100, 64
    g = torch.Generator().manual_seed(5)
    for small in (2.0 ** -8, 2.0 ** -14, 2.0 ** -17, 2.0 ** -19):
        c = Cache(16, [n], 1, D, 16, "s8")
        t = torch.arange(n)
        c.kv[0, c.table[0, t // 16].long(), t % 16, :, 7] = 0
        c.dev.copy_(c.kv)
        q = torch.randn(1, 2, D, generator=g) * small
        q[0, :, 7] = 1.9
        q = q.to(dtype)
        s = 1 / small                                            # scores of some units
        out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=torch.tensor([n], dtype=torch.int32, device=DEV), scale=s, **c.args()).cpu()
        k, v = (x[:, 0] for x in c.rows(0))
        for h in range(2):
            qd = q[0, h].double()
            score = k @ qd * s
            p = score.softmax(0)
            size = ((k.abs() @ qd.abs()) * s).max()
            delta = (D + 8) * 2.0 ** -24 * (size + score.abs().max() + 1)
            want, mass = p @ v, p @ v.abs()
            err = mass * (2.0 ** -11 + 4 * delta) + n * 2.0 ** -40 * v.abs().max() + HALF[dtype] * want.abs() + 2.0 ** -25
            assert ((out[0, h].double() - want).abs() <= err).all(), small


@pytest.mark.parametrize("top", [2.0 ** -130, 2.0 ** -100, 1.0, 2.0 ** 100, 3e38])
def test_queries_of_every_size(top):
    # bf16 queries as small and as large as there are, and a scale that brings the scores back to some units
    n, D = 70, 64
    c = Cache(18, [n], 1, D, 16, "s8")
    q = torch.randn(1, 2, D, generator=torch.Generator().manual_seed(6)).clamp(-3, 3) / 4
    q[0, 0, 0], q[0, 1, 5] = 1, -1
    q = (q.double() * top).bfloat16()
    s = min(1 / top, 2.0 ** 125)                                  # (2^-130: as far as a scale can, scores of 2^-5 and below)
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=torch.tensor([n], dtype=torch.int32, device=DEV), scale=s, **c.args()).cpu()
    check(c, q, out, s)
    q[0, 1, 5] = float("inf")
    out = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=torch.tensor([n], dtype=torch.int32, device=DEV), scale=s, **c.args()).cpu()
    check(c, q[:, :1], out[:, :1], s)
    assert out[0, 1].isnan().all()


@pytest.mark.parametrize("kind,dtype", KINDS[2:])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_weights_of_16_bit_caches(kind, dtype, D):
    """Weights in two parts of the cache's type: off by the square of its half unit, 2^-16 at most (f16 also by 2^-40 of the largest).
    Otherwise as in check(): scores in 32 bits, the result's own rounding."""
    lens = [2, 9, 64, 300, 1500]
    c = Cache(19 + D, lens, 2, D, 16, kind)
    q, out = run(c, len(lens), 6, D, dtype, scale=0.03)
    for b, n in enumerate(lens):
        k, v = (t.repeat_interleave(3, 1) for t in c.rows(b))
        qd = q[b].double()
        s = torch.einsum("hd,nhd->hn", qd, k) * 0.03
        p = s.softmax(-1)
        want, mass = torch.einsum("hn,nhd->hd", p, v), torch.einsum("hn,nhd->hd", p, v.abs())
        size = torch.einsum("hd,nhd->hn", qd.abs(), k.abs()).amax(-1) * 0.03
        delta = (D + 8) * 2.0 ** -24 * (size + s.abs().amax(-1) + 1)
        err = mass * (2.0 ** -16 + 4 * delta[:, None]) + n * 2.0 ** -40 * v.abs().max() + HALF[dtype] * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0)
        assert ((out[b].double() - want).abs() <= err).all(), n


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 40, 3000])
def test_infinite_values_of_16_bit_caches(dtype, n):
    # an infinity that has some weight gives an infinity of its sign, two that differ give NaN
    c = Cache(20, [n, 33], 2, 64, 16, "f16" if dtype == torch.float16 else "bf16")
    at = (1, c.table[0, (n - 1) // 16].item(), (n - 1) % 16)
    c.dev[at][0, 5], c.dev[at][0, 6], c.dev[at][1, 63] = float("inf"), -float("inf"), float("inf")
    if n > 1:
        c.dev[1, c.table[0, 0].item(), 0, 1, 63] = -float("inf")
    for scale in (0.0, 0.01):                                     # weights that are all the same, with nothing left of them, and others
        q, out = run(c, 2, 4, 64, dtype, scale=scale)
        want = torch.zeros(4, 64)
        want[:2, 5], want[:2, 6], want[2:, 63] = float("inf"), -float("inf"), float("nan") if n > 1 else float("inf")
        odd = ~torch.isfinite(want)
        assert torch.equal(torch.nan_to_num(out[0].float()[odd], 1e9, 2e9, -2e9), torch.nan_to_num(want[odd], 1e9, 2e9, -2e9))
        assert torch.isfinite(out[0][~odd]).all() and torch.isfinite(out[1]).all()
