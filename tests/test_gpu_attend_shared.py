"""Attention of requests that begin alike, against the definition in 64 bits: every request by itself over the tokens that its row lists."""
import pytest
import torch

from paper_2202_05239_amd import binding as f8
from test_gpu_attend import DEV, KINDS, Cache, check

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def share(c, sizes, prefixes, before=0):
    """Makes the requests of a cache begin alike: groups of the given sizes behind the first `before` requests, whose members hold the pages of
    their longest one as far as its prefix fills them, and copies of its page after that.  What nobody holds any more is NaN.  Returns
    first and shared."""
    first, dead, kept = [before], [], set()
    for n, prefix in zip(sizes, prefixes):
        b0 = first[-1]
        first.append(b0 + n)
        if n == 0:
            continue
        lead = max(range(b0, b0 + n), key=lambda b: c.lens[b])
        full, rest = prefix // c.page, prefix % c.page
        for b in range(b0, b0 + n):
            have = -(-c.lens[b] // c.page)
            if b != lead:
                dead += c.table[b, :min(full, have)].tolist()
                c.table[b, :min(full, have)] = c.table[lead, :min(full, have)]
                if rest and have > full and -(-c.lens[lead] // c.page) > full:
                    src, dst = c.table[lead, full], c.table[b, full]
                    m = min(rest, c.lens[b] - full * c.page)
                    c.kv[:, dst, :m] = c.kv[:, src, :m]
                    if c.scales is not None:
                        c.scales[:, dst, :m] = c.scales[:, src, :m]
    kept = {e for b, n in enumerate(c.lens) for e in c.table[b, : -(-n // c.page)].tolist()}
    dead = [e for e in dead if e not in kept]
    c.kv[:, dead] = 127 if c.scales is not None else float("nan")
    c.dev.copy_(c.kv)
    if c.scales is not None:
        c.scales[:, dead] = float("nan")
        c.dev_scales.copy_(c.scales)
    return ints(first), ints(prefixes)


def run(c, Hq, D, dtype, groups, seed=0, scale=None, **kw):
    q = (torch.randn(len(c.lens), Hq, D, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype)
    out = f8.f8_attend_shared(q.to(DEV), table=c.table.to(DEV), lens=ints(c.lens), first=groups[0], shared=groups[1], scale=scale, **c.args(), **kw)
    return q, out.cpu()


# groups of all sizes: prefixes of no token and of one, around a tile and a round, longer; members that are empty, end inside the prefix
# or with it, or go on; requests in front of all groups and behind them
SIZES, PREFIXES = [1, 5, 0, 3, 4, 9], [40, 600, 7, 0, 1, 130]
LENS = [70, 600, 0, 601, 128, 650, 620, 5, 0, 33, 1, 2, 65, 700, 131, 130, 129, 0, 260, 300, 137, 128, 258, 1, 513]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 144, 192, 256])
def test_groups_pages_and_heads(kind, dtype, D):
    for n, (heads, group, page) in enumerate([(1, 1, 16), (2, 3, 1), (3, 8, 24), (1, 16, 7), (2, 17, 64), (1, 40, 128), (1, 70, 32)]):
        c = Cache(n + D, LENS, heads, D, page, kind, heads_first=n % 2 == 1)
        groups = share(c, SIZES, PREFIXES, before=1)
        q, out = run(c, heads * group, D, dtype, groups)
        check(c, q, out, D ** -0.5)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("n,heads,group,D", [(64, 2, 4, 128), (33, 1, 5, 80), (20, 1, 16, 64), (70, 1, 1, 256), (3, 8, 8, 128)])
def test_many_rows_behind_a_long_prefix(kind, dtype, n, heads, group, D):
    g = torch.Generator().manual_seed(n)
    prefix = 5003
    lens = [prefix + int(t) for t in torch.randint(1, 300, (n,), generator=g)]
    lens[n // 2], lens[0], lens[1] = 0, 0, prefix                # the first place is empty
    c = Cache(n, lens, heads, D, 32, kind)
    groups = share(c, [n], [prefix])
    q, out = run(c, heads * group, D, dtype, groups)
    check(c, q, out, D ** -0.5)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_a_long_prefix_of_few_rows(kind, dtype):
    c = Cache(3, [20001, 20040, 20007, 19999], 1, 128, 64, kind)
    groups = share(c, [4], [20000])
    q, out = run(c, 2, 128, dtype, groups)
    check(c, q, out, 128 ** -0.5)


@pytest.mark.parametrize("kind,dtype", [KINDS[0], KINDS[3]])
def test_many_groups_and_requests(kind, dtype):
    # more items than are looked through at a time, more groups than bounds fit a workgroup's memory
    g = torch.Generator().manual_seed(9)
    for groups_n in (300, 1300):
        sizes = torch.randint(0, 4, (groups_n,), generator=g).tolist()
        lens = torch.randint(0, 60, (sum(sizes),), generator=g).tolist()
        for i in (0, len(lens) // 2, len(lens) - 1):
            lens[i] = 600 + i % 100
        prefixes = torch.randint(0, 50, (groups_n,), generator=g).tolist()
        prefixes[groups_n // 2] = 500
        c = Cache(groups_n, lens, 1, 32, 16, kind)
        groups = share(c, sizes, prefixes)
        q, out = run(c, 2, 32, dtype, groups)
        check(c, q, out, 32 ** -0.5)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("scale", [0.0, 4.0, -0.125, -3.0])
def test_scales_of_scores(kind, dtype, scale):
    lens = [900, 0, 1000, 1300]
    c = Cache(4, lens, 2, 64, 16, kind)
    groups = share(c, [4], [900])
    q, out = run(c, 6, 64, dtype, groups, scale=scale)
    check(c, q, out, scale)


def test_nobody_has_a_token_or_shares_one():
    c = Cache(5, [700, 800, 640], 2, 64, 16, "s8")
    for first, shared in (([0, 3], [0]), ([1, 2], [500]), ([3, 3], [500]), ([0, 1, 2, 3], [600, 600, 600]), ([0, 0], [5])):
        q, out = run(c, 4, 64, torch.float16, (ints(first), ints(shared)))
        check(c, q, out, 0.125)
    c.lens = [0, 0, 0]
    _, out = run(c, 4, 64, torch.float16, (ints([0, 3]), ints([600])))
    assert (out == 0).all()
    c.lens = [700, 0, 0]
    _, out = run(c, 4, 64, torch.float16, (ints([0, 3]), ints([800])))             # (longer than anybody)
    q, out = run(c, 4, 64, torch.float16, (ints([0, 3]), ints([2 ** 31 - 1])))
    check(c, q, out, 0.125)
    q, out = run(c, 4, 64, torch.float16, (ints([0, 3]), ints([-4])))
    check(c, q, out, 0.125)


def test_bounds_of_groups_outside_the_batch():
    # values that describe no groups: the call ends, and a request that no group claims is right
    c = Cache(6, [700, 800, 640], 2, 64, 16, "bf16")
    for first in ([-5, 1], [2, 900], [2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 0], [3, 1]):
        q, out = run(c, 4, 64, torch.bfloat16, (ints(first), ints([0])))
        check(c, q, out, 0.125)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_short_requests_go_the_way_of_single_ones(kind, dtype):
    lens = [300, 310, 0, 512, 5]
    c = Cache(7, lens, 2, 64, 16, kind)
    groups = share(c, [4], [299])
    q, out = run(c, 4, 64, dtype, groups, max_len=512)
    check(c, q, out, 0.125)
    alone = f8.f8_attend_paged(q.to(DEV), table=c.table.to(DEV), lens=ints(lens), max_len=512, **c.args()).cpu()
    assert torch.equal(out, alone)
    none = f8.f8_attend_shared(q.to(DEV), table=c.table.to(DEV), lens=ints(lens), first=ints([0]), shared=ints([]), **c.args()).cpu()
    check(c, q, none, 0.125)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_table_entries_outside_the_cache_are_left_out(kind, dtype):
    for bad in (-1, -2 ** 31, 2 ** 31 - 1):
        c = Cache(8, [800, 830, 810], 2, 64, 16, kind)
        groups = share(c, [3], [790])
        kept = c.table.clone()
        c.table[:, 2] = bad                                       # in the prefix
        c.table[1, 50] = bad                                      # behind it: tokens 800 .. 815 of request 1
        q, out = run(c, 4, 64, dtype, groups)
        c.table = kept
        for b in range(3):
            keep = torch.ones(c.lens[b], dtype=torch.bool)
            keep[32:48] = False
            if b == 1:
                keep[800:816] = False
            lens = c.lens
            c.lens = [n if i == b else 0 for i, n in enumerate(lens)]
            alone = torch.zeros_like(out)
            alone[b] = out[b]
            check(c, q, alone, 0.125, skip=keep)
            c.lens = lens


def test_nan_stays_where_it_belongs():
    c = Cache(9, [700, 690, 650, 0], 1, 64, 16, "bf16")
    groups = share(c, [4], [680])
    page = c.table[0, 41].item()                                  # tokens 656 .. 671: of requests 0 and 1, behind the end of request 2
    c.dev[1, page, 3, 0, 5] = float("nan")
    q, out = run(c, 2, 64, torch.bfloat16, groups)
    assert out[:2, :, 5].isnan().all() and out.isnan().sum() == 4
    c.dev[0, page, 3, 0, 5] = float("nan")
    q, out = run(c, 2, 64, torch.bfloat16, groups)
    assert out[:2].isnan().all() and torch.isfinite(out[2:]).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_infinite_values_of_16_bit_caches(dtype):
    c = Cache(10, [3000, 3100], 2, 64, 16, "f16" if dtype == torch.float16 else "bf16")
    groups = share(c, [2], [2999])
    at = (1, c.table[0, 1500 // 16].item(), 1500 % 16)
    c.dev[at][0, 5], c.dev[at][0, 6] = float("inf"), -float("inf")
    for scale in (0.0, 0.01):
        _, out = run(c, 4, 64, dtype, groups, scale=scale)
        assert (out[:, :2, 5] == float("inf")).all() and (out[:, :2, 6] == -float("inf")).all()
        assert torch.isfinite(out).sum() == out.numel() - 8


@pytest.mark.parametrize("scale", [2.0 ** -126, 0.0])
def test_stretches_of_zero_values(scale):
    for first, last in ((0, 32), (64, 96), (37, 300), (0, 900), (0, 1200)):
        c = Cache(11, [1200, 1000], 2, 64, 16, "s8")
        groups = share(c, [2], [900])
        for t in range(first, last):
            at = (1, c.table[0, t // 16].long(), t % 16)
            c.kv[at], c.scales[at] = 0, scale
            if t < 1000 and t >= 896:
                at = (1, c.table[1, t // 16].long(), t % 16)
                c.kv[at], c.scales[at] = 0, scale
        c.dev.copy_(c.kv)
        c.dev_scales.copy_(c.scales)
        for s in (0.0, 0.125, 1.0):
            q, out = run(c, 8, 64, torch.bfloat16, groups, scale=s)
            assert torch.isfinite(out).all()
            check(c, q, out, s)


def test_strided_queries_and_results():
    c = Cache(12, [900, 917], 2, 64, 16, "s8")
    groups = share(c, [2], [890])
    big = torch.randn(2, 3, 4, 80, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    q, out = big[:, 1, :, 8:72], torch.full((4, 2, 70), 9.0, dtype=torch.float16, device=DEV)
    view = out.transpose(0, 1)[..., 3:67]
    f8.f8_attend_shared(q, table=c.table.to(DEV), lens=ints(c.lens), first=groups[0], shared=groups[1], out=view, **c.args())
    check(c, q.cpu(), view.cpu(), 0.125)
    assert (out[..., :3] == 9).all() and (out[..., 67:] == 9).all()


def test_offsets_beyond_32_bits():
    pages, page, heads, D = 40000, 64, 8, 128                    # 2.6 GB of codes an array, strides of 5.2 GB
    kv = torch.empty(pages * page * heads * D * 2, dtype=torch.int8, device=DEV).view(pages, 2, page, heads, D).transpose(0, 1)
    scales = torch.empty(2, pages, page, heads, device=DEV)
    c = Cache(13, [64 * 9 - 5, 64 * 9], heads, D, page, "s8", spare=0)
    groups = share(c, [2], [500])
    ids = torch.arange(pages - c.pages, pages)
    kv[:, ids], scales[:, ids] = c.dev, c.dev_scales
    q = torch.randn(2, heads * 2, D).bfloat16()
    out = f8.f8_attend_shared(q.to(DEV), kv[0], kv[1], torch.where(c.table >= 0, c.table + pages - c.pages, -1).int().to(DEV), ints(c.lens), *groups,
                              k_scale=scales[0], v_scale=scales[1]).cpu()
    check(c, q, out, D ** -0.5)


def test_repeats_and_replays():
    c = Cache(14, [5000, 4970, 5100], 2, 128, 16, "s8")
    first, shared = share(c, [3], [4960])
    q = torch.randn(3, 8, 128).bfloat16().to(DEV)
    table, lens = c.table.to(DEV), ints(c.lens)
    ws = torch.empty(f8.lib().f8_attend_shared_workspace_bytes(3, 1, 8, 2, 128, 5100), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    call = lambda **kw: f8.f8_attend_shared(q, table=table, lens=lens, first=first, shared=shared, max_len=5100, **c.args(), **kw)  # noqa: E731
    want = call().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    # another batch under the same graph: lengths and groups are read on the device
    lens.copy_(ints([1000, 5, 900]))
    first.copy_(ints([0, 2]))
    shared.copy_(ints([4]))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, call())
    c.lens = [1000, 5, 900]
    check(c, q.cpu(), out.cpu(), 128 ** -0.5)


def test_rounding_of_weights():
    """The scores are formed in 32 bits and so are the sums; weights are rounded once (f16 under 8 and f16 bits, bf16 under bf16): relative 2^-11 or 2^-8
    each, random, so the result is off by little more than its own rounding in the mean of many."""
    for kind, dtype in KINDS:
        c = Cache(15, [2000] * 8, 2, 128, 16, kind)
        groups = share(c, [8], [1900])
        q, out = run(c, 8, 128, dtype, groups, scale=0.03)
        far = base = 0.0
        for b in range(8):
            k, v = (t.repeat_interleave(4, 1) for t in c.rows(b))
            p = (torch.einsum("hd,nhd->hn", q[b].double(), k) * 0.03).softmax(-1)
            want = torch.einsum("hn,nhd->hd", p, v)
            far += (out[b].double() - want).square().sum().item()
            base += (want.to(dtype).double() - want).square().sum().item()
        # a rounding to the same type, relative to the summed terms, which no cancellation makes smaller: sqrt(1 + 1) of the result's at most, 1.5 allowed
        assert far <= 1.5 ** 2 * base, (kind, far, base)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,group,D", [(10, 4, 128), (12, 4, 64), (5, 8, 80), (3, 16, 128), (11, 4, 64)])
def test_results_depend_on_the_inputs_alone(dtype, n, group, D):
    # 33 to 48 rows in a block of 64, several tiles to a wave: the columns that nobody fills are the same whatever ran before
    page, heads, whole = 64, 8, 250
    g = torch.Generator(device=DEV).manual_seed(n)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731

    def batch(n, D):
        """n requests behind 16000 tokens, with up to 50 of their own."""
        kv = rand(2, whole + n, page, heads, D).to(dtype)
        table = torch.cat([torch.arange(whole, device=DEV).expand(n, -1), whole + torch.arange(n, device=DEV)[:, None]], 1).int()
        lens = ints([whole * page + 1 + 5 * b % 50 for b in range(n)])
        return lambda q: f8.f8_attend_shared(q, kv[0], kv[1], table, lens, ints([0, n]), ints([whole * page]))
    call, q = batch(n, D), rand(n, heads * group, D).to(dtype)
    want = call(q)
    other = batch(16, 128)                                        # fills all 64 columns; its scores rise late and far
    for size in (1.0, 30.0, 900.0):
        x = (size * rand(16, heads * 4, 128)).to(dtype)
        for _ in range(3):
            other(x)
            assert torch.equal(call(q), want), size


@pytest.mark.parametrize("at", [0, 1777, 4095, 4200])
@pytest.mark.parametrize("score", [-34.0, -100.0])
def test_tokens_that_weigh_nothing(at, score):
    # one token of score 0 and value 0 among tokens of a score far below it and large values, in f16: weights below 2^-48 of the largest one
    # are taken as 0, so the result is off by n 2^-48 of the largest value at most (6e-6), which is then rounded (2^-25 at least)
    n, D = 4300, 64
    c = Cache(18, [n, n - 40], 1, D, 16, "f16")
    groups = share(c, [2], [4096])
    c.kv[0] = 0
    c.kv[0, ..., 0], c.kv[1] = score, 60000.0
    for b in range(2):
        page = c.table[b, at // 16].long()
        c.kv[:, page, at % 16] = 0
    c.dev.copy_(c.kv)
    q = torch.zeros(2, 2, D, dtype=torch.float16)
    q[..., 0] = 1
    out = f8.f8_attend_shared(q.to(DEV), table=c.table.to(DEV), lens=ints(c.lens), first=groups[0], shared=groups[1], scale=1.0, **c.args()).cpu()
    assert out.abs().max().item() <= n * 60000 * 2.0 ** -48 + 2.0 ** -25


@pytest.mark.parametrize("kind,score", [("f16", -27.0), ("bf16", -58.0)])
def test_infinite_values_of_small_weights(kind, score):
    # an infinite value shows under any weight from 2^-40 (f16; e^-27 is 2^-38.95) or 2^-86 (bf16; e^-58 is 2^-83.7) of the largest one up
    n, D, dtype = 3000, 64, {"f16": torch.float16, "bf16": torch.bfloat16}[kind]
    c = Cache(19, [n, n - 40], 1, D, 16, kind)
    groups = share(c, [2], [2900])
    c.kv[0], c.kv[1] = 0, 1
    for t in (5, 1500, 2899, 2950):
        c.kv[0] = 0
        c.kv[0, c.table[0, t // 16].long(), t % 16, 0, 0] = score
        c.kv[0, c.table[1, t // 16].long(), t % 16, 0, 0] = score
        c.dev.copy_(c.kv)
        for b in range(2):
            c.dev[1, c.table[b, t // 16].long(), t % 16, 0, 5] = float("inf")
            c.dev[1, c.table[b, t // 16].long(), t % 16, 0, 9] = -float("inf")
        q = torch.zeros(2, 2, D, dtype=dtype)
        q[..., 0] = 1
        out = f8.f8_attend_shared(q.to(DEV), table=c.table.to(DEV), lens=ints(c.lens), first=groups[0], shared=groups[1], scale=1.0, **c.args()).cpu()
        assert (out[..., 5] == float("inf")).all() and (out[..., 9] == -float("inf")).all()
        assert torch.isfinite(out).sum() == out.numel() - 8


def test_a_prefix_that_is_longer_than_every_member():
    # units are dealt out, no member can lead: every request reads its own tokens
    for kind, dtype in KINDS:
        c = Cache(20, [700, 0, 690, 3], 2, 64, 16, kind)
        for shared in (701, 800, 2 ** 31 - 1):
            q, out = run(c, 8, 64, dtype, (ints([0, 4]), ints([shared])), max_len=704)
            check(c, q, out, 0.125)
