"""Pages of a cache: forks, compaction and copies, against the same steps one by one on the CPU."""
import pytest
import torch

from paper_2202_05239_amd import binding as f8

pytestmark = pytest.mark.gpu

DEV = "cuda"


def forked(parent, table, lens, refs, page, grow):
    """f8_kv_fork by its definition."""
    B, cols = len(table), len(table[0])
    pages, refs = len(refs), list(refs)
    used = [-(-min(max(n, 0), cols * page) // page) for n in lens]
    real = lambda e: 0 <= e < pages  # noqa: E731
    for b in range(B):
        for e in table[b][:used[b]]:
            if real(e):
                refs[e] += sum(p == b for p in parent) - 1
    free = [i for i in range(pages) if refs[i] <= 0]
    new, out_lens, slots, moves, missing = [], [], [], [], 0
    tails = {}
    for b, p in enumerate(parent):
        if 0 <= p < B:
            n = min(max(lens[p], 0), cols * page)
            if grow and n % page and real(table[p][n // page]):
                tails.setdefault(table[p][n // page], []).append(b)
    keeps = {e: w[0] if refs[e] == len(w) else -1 for e, w in tails.items()}

    def take():
        nonlocal missing
        if free:
            refs[free[0]] = 1
            return free.pop(0)
        missing += 1
        return -1
    for b, p in enumerate(parent):
        if not 0 <= p < B:
            new.append([-1] * cols), out_lens.append(0), slots.append([-1] * grow)
            continue
        n = min(max(lens[p], 0), cols * page)
        row = table[p][:used[p]]
        if grow and n % page and real(row[-1]) and keeps[row[-1]] != b:
            e = take()
            refs[row[-1]] -= 1
            if e >= 0:
                moves.append((row[-1], e, n % page))
            row = row[:-1] + [e]
        need = -(-(n + grow) // page)
        while len(row) < min(need, cols):
            row.append(take())
        missing += max(0, need - cols)
        slots.append([row[t // page] * page + t % page if t < cols * page and real(row[t // page]) else -1 for t in range(n, n + grow)])
        new.append(row + [-1] * (cols - len(row))), out_lens.append(min(n + grow, cols * page))
    info = [len(moves), missing]
    return new, out_lens, refs, slots, moves + [(-1, -1, 0)] * (B - len(moves)), info


def state(seed, B, cols, page, spare=5, shares=True, full=False):
    """Tables whose rows share pages at random, tails among them, and the counts; some pages are held from outside."""
    g = torch.Generator().manual_seed(seed)
    ri = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))  # noqa: E731
    lens = [ri(0, cols * page) if not full else cols * page for _ in range(B)]
    need = sum(-(-n // page) for n in lens)
    order = torch.randperm(need + spare, generator=g).tolist()
    table, refs = [], [0] * (need + spare)
    for b, n in enumerate(lens):
        row = [order.pop() for _ in range(-(-n // page))]
        if shares and b and ri(0, 2):                       # begins like an earlier one, or is its copy
            other = ri(0, b - 1)
            if ri(0, 1):
                lens[b] = n = lens[other]
                row = list(table[other][: -(-n // page)])
            else:
                k = ri(0, min(len(row), -(-lens[other] // page)))
                row = table[other][:k] + row[k:]
        table.append(row + [-7] * (cols - len(row)))
        for e in row:
            refs[e] += 1
    for i in range(len(refs)):
        if ri(0, 9) == 0:
            refs[i] += 1
    return table, lens, refs, g, ri


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def check_fork(parent, table, lens, refs, page, grow, **kw):
    got = f8.f8_kv_fork(ints(parent).to(DEV), ints(table).to(DEV), ints(lens).to(DEV), ints(refs).to(DEV), page, grow, **kw)
    want = forked(parent, table, lens, refs, page, grow)
    for name, a, b in zip(("table", "lens", "refs", "slots", "moves", "info"), got, want):
        assert torch.equal(a.cpu(), torch.tensor(b, dtype=a.dtype).view(a.shape)), (name, a.cpu(), b)
    return got


@pytest.mark.parametrize("grow", [0, 1, 3, 40])
@pytest.mark.parametrize("B,cols,page,spare", [(1, 1, 1, 2), (1, 3, 16, 0), (4, 5, 4, 3), (7, 9, 24, 100), (33, 12, 16, 40), (64, 20, 1, 2000), (200, 7, 16, 300)])
def test_forks(B, cols, page, spare, grow):
    for seed in range(4):
        table, lens, refs, g, ri = state(seed * 100 + B, B, cols, page, spare)
        check_fork(list(range(B)), table, lens, refs, page, grow)                              # everybody goes on
        check_fork([ri(-1, B - 1) for _ in range(B)], table, lens, refs, page, grow)           # beams, some of which end
        check_fork([B // 2] * B, table, lens, refs, page, grow)                                # all from one
        check_fork([-1] * B, table, lens, refs, page, grow)                                    # all end


@pytest.mark.parametrize("B,cols,page,spare,grow", [(1500, 13, 16, 700, 1), (64, 300, 16, 20000, 1), (300, 80, 4, 1000, 2), (20, 700, 1, 3, 300), (40, 10, 64, 30000, 200)])
def test_large_tables_and_pools(B, cols, page, spare, grow):
    table, lens, refs, g, ri = state(B + cols, B, cols, page, spare)
    check_fork([ri(-1, B - 1) for _ in range(B)], table, lens, refs, page, grow)
    check_fork(list(range(B)), table, lens, refs, page, grow)


@pytest.mark.parametrize("B,cols,extra", [(1024, 16, 0), (1024, 16, 1), (1025, 15, 0), (1023, 17, 0)])
def test_sizes_around_one_workgroup(B, cols, extra):
    # as many requests, entries and pages as one workgroup takes, and one more of each
    table, lens, refs, g, ri = state(B, B, cols, 4, 8192)
    pages = 8192 + extra
    refs = refs[:pages]
    table = [[e if e < pages else e % pages for e in row] for row in table]
    check_fork([ri(-1, B - 1) for _ in range(B)], table, lens, refs, 4, 1)
    check_fork(list(range(B)), table, lens, refs, 4, 4)
    check_fork(list(range(B)), table, lens, refs, 4, 5)


def test_prompts_and_full_tables():
    # empty places take prompts of many tokens; tables without a column left; a pool without a page left
    for grow in (1, 100, 513):
        check_fork([0, 1, 2], [[-1] * 33] * 3, [0, 0, 0], [0] * 120, 16, grow)
        check_fork([0, 1, 2], [[-1] * 33] * 3, [0, 0, 0], [0] * 7, 16, grow)
        check_fork([0, 0], [[5, 6], [2, 3]], [7, 8], [0, 0, 1, 1, 0, 1, 1], 4, grow)
        check_fork([0, 1], [[5, 6], [2, 3]], [8, 8], [1, 1, 1, 1, 1, 1, 1], 4, grow)


def test_entries_and_lengths_outside():
    # entries that are no page are carried along and hold nothing, lengths are clamped, counts below zero are free
    table = [[3, -1, 9], [99, 2 ** 31 - 1, 4], [-2 ** 31, 5, 6]]
    refs = [0, -3, 0, 1, 1, 1, 1, 0, 0, 1]
    for lens in ([10, 9, 8], [12, -5, 2 ** 31 - 1], [5, 6, 1]):
        for parent in ([0, 1, 2], [2, 2, 0], [1, 0, 3], [-1, -2 ** 31, 2 ** 31 - 1]):
            for grow in (0, 1, 6):
                check_fork(parent, table, lens, refs, 4, grow)


def test_tails_held_from_outside_are_copied():
    got = check_fork([0], [[2, 1]], [6], [0, 2, 1], 4, 1)
    assert got[4].tolist() == [[1, 0, 2]] and got[3].tolist() == [[2]] and got[2].tolist() == [1, 1, 1]


def test_strided_tables_and_replays():
    table, lens, refs, g, ri = state(5, 6, 9, 16, 60)
    B, cols = 6, 9
    parent = [1, 1, 0, -1, 5, 5]
    wide = torch.full((B, 14), 77, dtype=torch.int32, device=DEV)
    wide[:, 2:11] = ints(table).to(DEV)
    dst = torch.full((B, 12), 55, dtype=torch.int32, device=DEV)
    new = lambda *s, t=torch.int32: torch.full(s, 3, dtype=t, device=DEV)  # noqa: E731
    out = (dst[:, 1:10], new(B), new(len(refs)), new(B, 1, t=torch.int64), new(B, 3), new(2))
    ws = torch.empty(f8.lib().f8_kv_fork_workspace_bytes(B, len(refs)), dtype=torch.uint8, device=DEV)
    args = (ints(parent).to(DEV), wide[:, 2:11], ints(lens).to(DEV), ints(refs).to(DEV), 16, 1)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        f8.f8_kv_fork(*args, out=out, workspace=ws)
    for p in (parent, [0, 1, 2, 3, 4, 5], [3, 3, 3, 3, -1, 3]):
        args[0].copy_(ints(p))
        for t in out:
            t.fill_(9)
        ws.fill_(0x5a)
        graph.replay()
        torch.cuda.synchronize()
        want = forked(p, table, lens, refs, 16, 1)
        for a, b in zip(out, want):
            assert torch.equal(a.cpu(), torch.tensor(b, dtype=a.dtype).view(a.shape))
        assert (dst[:, 0] == 55).all() and (dst[:, 10:] == 55).all()


def compacted(table, refs, page):
    pages = len(refs)
    used = [i for i in range(pages) if refs[i] > 0]
    U = len(used)
    goes, holes = [i for i in used if i >= U], [i for i in range(U) if refs[i] <= 0]
    to = dict(zip(goes, holes))
    out = [0] * pages
    for i in used:
        out[to.get(i, i)] = refs[i]
    moves = [(a, b, page) for a, b in zip(goes, holes)]
    return [[to.get(e, e) for e in row] for row in table], out, moves + [(-1, -1, 0)] * (pages // 2 - len(moves)), [len(moves), U]


@pytest.mark.parametrize("pages", [1, 2, 3, 17, 1000, 4095, 4096, 4097, 20000, 100003])
def test_compaction(pages):
    g = torch.Generator().manual_seed(pages)
    for used in (0.0, 0.03, 0.5, 0.97, 1.0, -1.0):
        refs = torch.where(torch.rand(pages, generator=g) < used, torch.randint(1, 6, (pages,), generator=g), -(torch.rand(pages, generator=g) < 0.1).int())
        if used < 0:                                         # all in use lie behind all that are free
            refs = (torch.arange(pages) >= pages // 2).int()
        table = torch.randint(-3, pages + 3, (5, 37), generator=g)
        table[0, 0], table[0, 1] = 2 ** 31 - 1, -2 ** 31
        got = f8.f8_kv_compact(table.int().to(DEV), refs.int().to(DEV), 16)
        want = compacted(table.tolist(), refs.tolist(), 16)
        for a, b in zip(got, want):
            assert torch.equal(a.cpu(), torch.tensor(b, dtype=torch.int32).view(a.shape)), (pages, used)
        # the table in place, no table at all
        t = table.int().to(DEV)
        f8.f8_kv_compact(t, refs.int().to(DEV), 16, out=(t, got[1], got[2], got[3]))
        assert torch.equal(t.cpu(), ints(want[0]))
        none = f8.f8_kv_compact(t[:0], refs.int().to(DEV), 16)
        assert torch.equal(none[1].cpu(), ints(want[1]))


@pytest.mark.parametrize("pages,rows,cols", [(8191, 128, 128), (8192, 128, 128), (8193, 128, 128), (8192, 127, 130), (1, 5, 4000), (2, 3, 6000), (70001, 33, 700)])
def test_compaction_around_one_workgroup(pages, rows, cols):
    g = torch.Generator().manual_seed(pages + cols)
    for used in (0.3, 0.9, -1.0):
        refs = torch.where(torch.rand(pages, generator=g) < used, torch.randint(1, 6, (pages,), generator=g), 0)
        if used < 0:
            refs = (torch.arange(pages) >= pages // 2).int()
        table = torch.randint(-3, pages + 3, (rows, cols), generator=g)
        want = compacted(table.tolist(), refs.tolist(), 16)
        wide = torch.full((rows, cols + 5), 77, dtype=torch.int32, device=DEV)
        wide[:, 2:cols + 2] = table.int().to(DEV)
        for src in (table.int().to(DEV), wide[:, 2:cols + 2]):
            got = f8.f8_kv_compact(src, refs.int().to(DEV), 16)
            for a, b in zip(got, want):
                assert torch.equal(a.cpu(), torch.tensor(b, dtype=torch.int32).view(a.shape)), (pages, used)


TYPES = {"s8": torch.int8, "f16": torch.float16, "bf16": torch.bfloat16}


def order_of(kv, form):
    """The same cache with its dimensions in another order in memory, or rows apart."""
    if form == "heads outside":
        return kv.transpose(2, 3).contiguous().transpose(2, 3)
    if form == "token gaps":
        big = torch.zeros(*kv.shape[:3], kv.shape[3] + 1, *kv.shape[4:], dtype=kv.dtype, device=kv.device)
        big[:, :, :, : kv.shape[3]] = kv
        return big[:, :, :, : kv.shape[3]]
    if form == "row gaps" and kv.dim() == 5:
        big = torch.zeros(*kv.shape[:4], kv.shape[4] + 16, dtype=kv.dtype, device=kv.device)
        big[..., : kv.shape[4]] = kv
        return big[..., : kv.shape[4]]
    if form == "keys and values side by side":
        return kv.transpose(0, 1).contiguous().transpose(0, 1)
    return kv.clone()


@pytest.mark.parametrize("kind", ["s8", "f16", "bf16"])
@pytest.mark.parametrize("form", ["plain", "heads outside", "token gaps", "row gaps", "keys and values side by side"])
def test_copies(kind, form):
    g = torch.Generator().manual_seed(len(form))
    for pages, page, heads, D in ((9, 1, 1, 16), (12, 16, 2, 64), (7, 7, 3, 80), (40, 24, 5, 48), (5, 128, 1, 256), (6, 64, 8, 128)):
        kv = torch.randint(-127, 128, (2, pages, page, heads, D), generator=g).to(TYPES[kind])
        scales = torch.rand(2, pages, page, heads, generator=g)
        order = torch.randperm(pages, generator=g).tolist()
        k = pages // 2
        moves = [(order[i], order[k + i], [page, 1, page // 2, 0, page + 9, -3][i % 6]) for i in range(k)]
        moves += [(-1, -1, 0), (pages, 0, page), (0, pages, page), (2 ** 31 - 1, -2 ** 31, 4), (order[0], order[0], page)]
        want, ws = kv.clone(), scales.clone()
        for s, d, n in moves[:k]:
            n = min(max(n, 0), page)
            want[:, d, :n], ws[:, d, :n] = kv[:, s, :n], scales[:, s, :n]
        for info in (None, torch.tensor([k, 5], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV)):
            dev, sc = order_of(kv.to(DEV), form), order_of(scales.to(DEV), form)
            f8.f8_kv_copy(ints(moves).to(DEV), dev[0], dev[1], *((sc[0], sc[1]) if kind == "s8" else ()), info=info)
            if info is not None and info.numel() == 1:
                s, d, n = moves[0]
                assert torch.equal(dev[:, d, :n].cpu(), kv[:, s, :n]) and torch.equal(dev[:, order[2 * k - 1]].cpu(), kv[:, order[2 * k - 1]] if k > 1 else want[:, d])
                continue
            assert torch.equal(dev.cpu(), want), (pages, page)
            assert torch.equal(sc.cpu(), ws if kind == "s8" else scales)


def test_copies_beyond_32_bits():
    pages, page, heads, D = 40000, 64, 8, 128                    # 2.6 GB of codes an array, strides of 5.2 GB
    kv = torch.empty(pages * page * heads * D * 2, dtype=torch.int8, device=DEV).view(pages, 2, page, heads, D).transpose(0, 1)
    scales = torch.empty(2, pages, page, heads, device=DEV)
    for i, p in enumerate((7, pages - 1, pages - 2)):
        kv[:, p], scales[:, p] = i + 1, i + 0.5
    moves = torch.tensor([[pages - 1, 9, 64], [7, pages - 3, 30]], dtype=torch.int32, device=DEV)
    kv[:, pages - 3], scales[:, pages - 3] = 99, 99.0
    f8.f8_kv_copy(moves, kv[0], kv[1], scales[0], scales[1])
    assert (kv[:, 9] == 2).all() and (kv[:, pages - 3, :30] == 1).all() and (kv[:, pages - 3, 30:] == 99).all()
    assert (scales[:, 9] == 1.5).all() and (scales[:, pages - 3, :30] == 0.5).all() and (scales[:, pages - 3, 30:] == 99).all()


def test_many_lines_and_no_lines():
    pages = 30001
    kv = torch.arange(pages, device=DEV).to(torch.float16).view(1, pages, 1, 1, 1).repeat(2, 1, 2, 1, 16)
    moves = torch.stack([torch.arange(1, 15001), torch.arange(15001, pages), torch.full((15000,), 2)], 1).int().to(DEV)
    f8.f8_kv_copy(moves, kv[0], kv[1])
    assert torch.equal(kv[:, 15001:], kv[:, 1:15001])
    f8.f8_kv_copy(moves[:0], kv[0], kv[1])


@pytest.mark.parametrize("pages", [1, 40, 20000])
def test_forks_of_no_request(pages):
    # the counts do not shrink with the batch: they and `info` are written all the same, into given tensors and new ones
    new = lambda *s, t=torch.int32: torch.full(s, -77, dtype=t, device=DEV)  # noqa: E731
    refs = torch.randint(-2, 5, (pages,), generator=torch.Generator().manual_seed(pages)).int().to(DEV)
    kept = refs.clone()
    out = (new(0, 3), new(0), new(pages), new(0, 2, t=torch.int64), new(0, 3), new(2))
    for given in (out, None):
        got = f8.f8_kv_fork(new(0), new(0, 3), new(0), refs, 16, 2, out=given)
        assert torch.equal(got[2], kept) and got[5].tolist() == [0, 0] and torch.equal(refs, kept)
        assert got[0].shape == (0, 3) and got[3].shape == (0, 2) and got[4].shape == (0, 3)
    assert got[2].data_ptr() != refs.data_ptr()
