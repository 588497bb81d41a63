"""Cases of serving several continuations of one prompt: attention over a prefix that requests share, beam search's selection, and the
pages of the cache that follow it (forked, compacted, copied).

A case is a plain dict.  prepare() makes what a serving program holds before the call (queries, a paged cache with its block table, the
holders of its pages, logits), run() is one pass through one operator, exact() the operator's definition in 64 bits.  Where `own` is
false run() computes the same in elementary torch operations, 32 bits for attention, 64 for the scores that beams are chosen by.

The operators, for a cache in pages and a table whose row b lists the pages of request b:
  attend    out[b] = sum_t softmax_t(scale q[b] . k_t) v_t over the tokens t < lens[b] of request b.  Requests first[g] .. first[g + 1] - 1 have
            their first shared[g] tokens in common, which are read once for all of them.
  beam      S[b, i, t] = scores[b, i] + logits[b, i, t] - log sum_u exp logits[b, i, u]; of a finished beam scores[b, i] for t = eos and -inf
            for every other token.  The `keep` largest of S[b], ties to the lowest (i, t), as score, row b beams + i and token.
  fork      Request b goes on from request parent[b] (-1: it ends) by `grow` tokens: it shares the parent's pages; a last page that is not
            full and that others hold too is copied; new pages are the free ones of the lowest index, requests in their order, the copy first.
  compact   Pages in use beyond the number of pages in use move into the free ones below it, both in ascending order.
  copy      The first n tokens of page src into page dst, for each (src, dst, n) of a list whose unused places are (-1, -1, 0).
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
        # a few answers to one short question, 16-bit cache: one step, latency
        dict(name="shared_short", kind="attend", groups=1, n=8, even=True, prefix=256, tail=40, heads=4, group=2, D=64, page=16, cache="bf16", x="bf16"),
        # beam search over a batch of prompts of all lengths, four beams each, 8-bit cache
        dict(name="shared_beams", kind="attend", groups=16, n=4, even=True, prefix=4096, tail=128, heads=8, group=4, D=128, page=32, cache="s8", x="bf16"),
        # a serving batch behind one long common prompt, one slot of it empty: many rows for each key
        dict(name="shared_prompt", kind="attend", groups=1, n=64, even=True, prefix=32768, tail=512, heads=8, group=4, D=128, page=64, cache="bf16", x="bf16"),
        # groups of different sizes, a head's width and pages that fill no tile
        dict(name="shared_odd", kind="attend", groups=3, n=17, even=False, prefix=9001, tail=700, heads=5, group=5, D=80, page=24, cache="f16", x="f16"),
        # one prompt, four beams, an odd vocabulary, logits in 32 bits: latency
        dict(name="beam_one", kind="beam", batch=1, beams=4, vocab=5001, keep=4, type="f32", done=False),
        # a batch of prompts over a large vocabulary, twice as many candidates as beams, some of them finished: the logits are the traffic
        dict(name="beam_batch", kind="beam", batch=64, beams=8, vocab=131072, keep=16, type="bf16", done=True),
        # beam search's step: beams go on from one another, tails that two of them hold are copied
        dict(name="fork_beams", kind="fork", groups=16, n=4, longest=2048, page=16, spare=500, ends=False),
        # a serving batch's step over a large pool: nearly every request goes on from itself, a few end
        dict(name="fork_batch", kind="fork", groups=512, n=1, longest=32768, page=64, spare=4001, ends=True),
        # a small pool after some requests have ended
        dict(name="compact_small", kind="compact", pages=1001, used=0.5, rows=33, cols=31, page=16),
        # a large pool, a fifth of it free, before it gives memory back
        dict(name="compact_pool", kind="compact", pages=262144, used=0.8, rows=512, cols=513, page=64),
        # the tails that a step of beam search has forked
        dict(name="copy_tails", kind="copy", pages=600, moves=48, places=64, full=False, page=16, heads=8, D=128, cache="bf16"),
        # the pages that a compaction has moved
        dict(name="copy_moved", kind="copy", pages=5001, moves=2048, places=2500, full=True, page=64, heads=8, D=128, cache="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    u = rng.random()
    most = {c["name"]: work(c) for c in listed()}
    if u < 0.4:
        while True:
            cache = rng.choice(("s8", "s8", "bf16", "f16"))
            c = dict(kind="attend", groups=_log(rng, 1, 32), n=_log(rng, 1, 64), even=rng.random() < 0.5, prefix=_log(rng, 1, 65536), tail=_log(rng, 1, 2048),
                     heads=rng.choice((1, 2, 4, 5, 8)), group=rng.choice((1, 2, 4, 5, 8, 16)), D=rng.choice((64, 128, 128, 80, 96, 192, 256)),
                     page=rng.choice((1, 16, 16, 24, 32, 64, 128)), cache=cache, x=rng.choice(("bf16", "f16")) if cache == "s8" else cache)
            if c["groups"] * c["n"] <= 256 and all(work(c)[k] <= most["shared_prompt"][k] for k in ("bytes", "flops")):
                return c
    if u < 0.6:
        while True:
            beams = _log(rng, 1, 16)
            c = dict(kind="beam", batch=_log(rng, 1, 64), beams=beams, vocab=_log(rng, 100, 131072), keep=beams * rng.choice((1, 2)),
                     type=rng.choice(("bf16", "f16", "f32")), done=rng.random() < 0.5)
            if work(c)["bytes"] <= most["beam_batch"]["bytes"]:
                return c
    if u < 0.75:
        while True:
            c = dict(kind="fork", groups=_log(rng, 1, 512), n=_log(rng, 1, 16), longest=_log(rng, 1, 32768), page=rng.choice((1, 16, 16, 24, 64, 128)),
                     spare=_log(rng, 600, 60000), ends=rng.random() < 0.5)
            if c["groups"] * c["n"] <= 512 and work(c)["bytes"] <= most["fork_batch"]["bytes"]:
                return c
    if u < 0.87:
        while True:
            c = dict(kind="compact", pages=_log(rng, 2, 262144), used=rng.uniform(0.05, 0.98), rows=_log(rng, 1, 512), cols=_log(rng, 1, 513), page=rng.choice((1, 16, 64)))
            if work(c)["bytes"] <= most["compact_pool"]["bytes"]:
                return c
    while True:
        moves = _log(rng, 1, 2048)
        c = dict(kind="copy", pages=2 * moves + _log(rng, 1, 900), moves=moves, places=moves + rng.randint(0, 400), full=rng.random() < 0.5,
                 page=rng.choice((1, 16, 16, 24, 32, 64, 128)), heads=rng.choice((1, 2, 4, 5, 8)), D=rng.choice((64, 128, 128, 80, 96, 192, 256)),
                 cache=rng.choice(("bf16", "f16", "s8")))
        if work(c)["bytes"] <= most["copy_moved"]["bytes"]:
            return c


def _sizes(case):
    """Members of each group: a property of the case, the largest group first."""
    if case["even"]:
        return [case["n"]] * case["groups"]
    r = random.Random(case["groups"] * 977 + case["n"])
    return [case["n"]] + [r.randint(1, case["n"]) for _ in range(case["groups"] - 1)]


def _prefixes(case):
    r = random.Random(case["prefix"] * 31 + case["groups"])
    return [case["prefix"]] + [r.randint(1, case["prefix"]) for _ in range(case["groups"] - 1)]


def _tails(case):
    """Tokens of each request behind its prefix, at least one.  In a batch of eight and more the last request of the first group is an
    empty slot (a step captured for a fixed batch): 0, and no prefix either."""
    B = sum(_sizes(case))
    r = random.Random(B * 131 + case["tail"])
    tails = [case["tail"]] + [r.randint(1, case["tail"]) for _ in range(B - 1)]
    if B >= 8 and _sizes(case)[0] > 1:
        tails[_sizes(case)[0] - 1] = 0
    return tails


def _fork_lens(case):
    """(pages that a group's members share, tokens of each member behind them)."""
    r = random.Random(case["groups"] * 7 + case["longest"])
    shared, behind = [], []
    for _ in range(case["groups"]):
        n = r.randint(1, case["longest"])
        shared.append((n // 2) // case["page"] if case["n"] > 1 else 0)
        behind += [max(1, n - shared[-1] * case["page"])] * case["n"]
    return shared, behind


def _quant(v):
    scale = (v.abs().amax(-1, keepdim=True) / 127).clamp_min(TINY)
    return torch.round(v / scale), scale


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(g, case, pages):
    kv = torch.randn(2, pages, case["page"], case["heads"], case["D"], generator=g, device="cuda")
    kv *= torch.exp(0.4 * torch.randn(2, pages, case["page"], case["heads"], 1, generator=g, device="cuda"))
    if case["cache"] == "s8":
        codes, scale = _quant(kv)
        return codes.to(torch.int8), scale[..., 0].contiguous()
    return kv.to(TYPES[case["cache"]]), None


def _prepare_attend(g, case):
    page, sizes, prefixes, tails = case["page"], _sizes(case), _prefixes(case), _tails(case)
    member = [i for i, n in enumerate(sizes) for _ in range(n)]
    lens = [prefixes[member[b]] + t if t else 0 for b, t in enumerate(tails)]
    whole = [n // page for n in prefixes]                        # pages that a group's members share; a page of both is each one's own
    need = [-(-n // page) - whole[member[b]] if n else 0 for b, n in enumerate(lens)]
    pages = sum(whole) + sum(need) + 1                           # page 0 belongs to nobody
    width = max(1, max(-(-n // page) for n in lens))
    order = (torch.randperm(pages - 1, generator=g, device="cuda") + 1).to(torch.int32)
    cols = torch.arange(width, device="cuda")[None]
    before = lambda v: torch.tensor([0] + v[:-1], device="cuda").cumsum(0)  # noqa: E731
    of, w = torch.tensor(member, device="cuda"), torch.tensor(whole, device="cuda")
    mine, n = w[of][:, None], _ints(lens)
    at = torch.where(cols < mine, before(whole)[of][:, None] + cols, sum(whole) + before(need)[:, None] + cols - mine)
    used = cols < -(-n // page)[:, None]
    table = torch.where(used, order[at.clamp(0, pages - 2)], 0).to(torch.int32)
    kv, scales = _cache(g, case, pages)
    # the page that holds a prefix's last tokens and a member's first own ones: the same tokens in each member's copy
    first = before(sizes).to(torch.int32)
    col, rest = w[of][:, None], torch.tensor([m % page for m in prefixes], device="cuda")[of]
    real = (rest > 0) & (n > 0) & (w[of] < width)
    col = col.clamp_max(width - 1)
    copies, source = table.gather(1, col)[:, 0].long(), table[first[of].long()].gather(1, col)[:, 0].long()
    copies, source = torch.where(real, copies, 0), torch.where(real, source, 0)
    place = torch.arange(page, device="cuda")[None] < rest[:, None]
    kv[:, copies] = torch.where(place[None, :, :, None, None], kv[:, source], kv[:, copies])
    if scales is not None:
        scales[:, copies] = torch.where(place[None, :, :, None], scales[:, source], scales[:, copies])
    q = torch.randn(len(lens), case["heads"] * case["group"], case["D"], generator=g, device="cuda").to(TYPES[case["x"]])
    index = before(sizes)[:, None] + torch.arange(max(sizes), device="cuda")[None]     # requests of each group, filled up
    return dict(case=case, q=q, kv=kv, scales=scales, table=table, lens=n, first=torch.cat([first, _ints([sum(sizes)])]), shared=_ints(prefixes),
                member=of, index=index.clamp_max(len(lens) - 1), longest=max(lens), prefix=max(prefixes))


def _prepare_fork(g, case):
    page, n, (shared, behind) = case["page"], case["n"], _fork_lens(case)
    B = len(behind)
    of = torch.arange(B, device="cuda") // n
    s, lens = torch.tensor(shared, device="cuda"), torch.tensor(behind, device="cuda")
    need = -(-lens // page)
    pages, width = int(sum(shared)) + int(need.sum()) + case["spare"], -(-case["longest"] // page) + 2
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    cols = torch.arange(width, device="cuda")[None]
    at = torch.where(cols < s[of][:, None], (s.cumsum(0) - s)[of][:, None] + cols, s.sum() + (need.cumsum(0) - need)[:, None] + cols - s[of][:, None])
    used = cols < (s[of] + need)[:, None]
    table = torch.where(used, order[at.clamp(0, pages - 1)], -1).to(torch.int32)
    refs = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    refs.index_add_(0, torch.where(used, table, pages).flatten().long(), torch.ones(B * width, dtype=torch.int32, device="cuda"))
    parent = of * n + torch.randint(n, (B,), generator=g, device="cuda")
    if case["ends"]:
        parent = torch.where(torch.rand(B, generator=g, device="cuda") < 0.05, -1, parent)
    return dict(case=case, table=table, lens=(s[of] * page + lens).to(torch.int32), refs=refs[:pages].contiguous(), parent=parent.to(torch.int32))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    kind = case["kind"]
    if kind == "attend":
        return _prepare_attend(g, case)
    if kind == "beam":
        B, K, V = case["batch"], case["beams"], case["vocab"]
        x = 3 * torch.randn(B, K, V, generator=g, device="cuda")
        x += torch.where(rand(B, K, V) < 20 / V, 8.0, 0.0)       # a few tokens that the model takes seriously
        scores = -(40 * rand(B, 1) + 6 * rand(B, K)).sort(-1).values
        return dict(case=case, logits=x.to(TYPES[case["type"]]), scores=scores, done=rand(B, K) < 0.2 if case["done"] else None, eos=2)
    if kind == "fork":
        return _prepare_fork(g, case)
    if kind == "compact":
        pages, shape = case["pages"], (case["rows"], case["cols"])
        refs = torch.where(rand(pages) < case["used"], torch.randint(1, 5, (pages,), generator=g, device="cuda"), 0).to(torch.int32)
        held = torch.nonzero(torch.cat([refs, refs.new_ones(1)]))[:, 0].to(torch.int32)       # (the last one is no page: where none is held)
        table = held[torch.randint(max(1, held.numel() - 1), shape, generator=g, device="cuda")]
        return dict(case=case, refs=refs, table=torch.where((rand(*shape) < 0.3) | (table >= pages), -1, table).to(torch.int32))
    # page 0 is in no move
    order = torch.randperm(case["pages"] - 1, generator=g, device="cuda")[: 2 * case["moves"]] + 1
    n = torch.full((case["moves"],), case["page"], device="cuda") if case["full"] else torch.randint(1, case["page"] + 1, (case["moves"],), generator=g, device="cuda")
    moves = torch.tensor([[-1, -1, 0]], dtype=torch.int32, device="cuda").repeat(case["places"], 1)
    moves[: case["moves"]] = torch.stack([order[: case["moves"]], order[case["moves"]:], n], 1).to(torch.int32)
    kv, scales = _cache(g, case, case["pages"])
    return dict(case=case, moves=moves, kv=kv, scales=scales)


def _plain_attend(s, real):
    """Scores of a group's members against their prefix, and of each request against its own tokens, in one softmax."""
    c = s["case"]
    H, G, D, page = c["heads"], c["group"], c["D"], c["page"]
    B, of, longest = s["q"].shape[0], s["member"], s["longest"]
    first, shared, n = s["first"][:-1].long(), s["shared"].long(), s["lens"].long()

    def rows(i, table, t):
        at = table.gather(1, (t // page).clamp_max(table.shape[1] - 1)).long() * page + t % page
        x = s["kv"][i].reshape(-1, H, D)[at].to(real)
        return x if s["scales"] is None else x * s["scales"][i].reshape(-1, H)[at].to(real)[..., None]
    q = s["q"].to(real).reshape(B, H, G, D) / math.sqrt(D)
    # [groups][heads][members, query heads][tokens of the prefix], then by request
    t = torch.arange(s["prefix"], device="cuda")[None].expand(len(shared), -1)
    k, v = (rows(i, s["table"][first], t) for i in range(2))
    qg = q[s["index"]].permute(0, 2, 1, 3, 4).reshape(len(shared), H, -1, D)
    score = torch.matmul(qg, k.permute(0, 2, 3, 1).contiguous())
    place = torch.arange(B, device="cuda") - first[of]
    score = score.reshape(len(shared), H, -1, G, s["prefix"]).permute(0, 2, 1, 3, 4)[of, place]
    score = score.masked_fill(~(t[of] < torch.minimum(shared[of], n)[:, None])[:, None, None], -math.inf)
    # [requests][heads][query heads][own tokens]
    u = shared[of][:, None] + torch.arange(c["tail"], device="cuda")[None]
    ko, vo = (rows(i, s["table"], u) for i in range(2))
    seen = u < n[:, None]
    mine = torch.matmul(q, ko.permute(0, 2, 3, 1).contiguous()).masked_fill(~seen[:, None, None], -math.inf)
    top = torch.maximum(score.amax(-1, keepdim=True), mine.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0, top)
    p, po = torch.exp(score - top), torch.exp(mine - top)
    total = p.sum(-1, keepdim=True) + po.sum(-1, keepdim=True)
    pg = p[s["index"]].permute(0, 2, 1, 3, 4).reshape(len(shared), H, -1, s["prefix"])
    out = torch.matmul(pg, v.permute(0, 2, 1, 3).contiguous())
    out = out.reshape(len(shared), H, -1, G, D).permute(0, 2, 1, 3, 4)[of, place]
    out = out + torch.matmul(po, torch.where(seen[:, :, None, None], vo, 0).permute(0, 2, 1, 3).contiguous())
    return (out / torch.where(total == 0, 1, total)).reshape(B, H * G, D)


def _plain_beam(s):
    c = s["case"]
    k = min(c["keep"], c["vocab"])
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    best, token = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True)
    best, token = best[..., :k].double(), token[..., :k]
    score = s["scores"].double()[..., None] + (best - lse)
    if s["done"] is not None:
        i = torch.arange(k, device="cuda")
        others = torch.where(i == 0, s["eos"], torch.where(i - 1 < s["eos"], i - 1, i))
        token = torch.where(s["done"][..., None], others, token)
        score = torch.where(s["done"][..., None], torch.where(i == 0, s["scores"].double()[..., None], -math.inf), score)
    score, at = torch.sort(score.reshape(c["batch"], -1), dim=-1, descending=True, stable=True)
    score, at = score[:, : c["keep"]], at[:, : c["keep"]]
    row = torch.arange(c["batch"], device="cuda")[:, None] * c["beams"] + at // k
    return score.float(), row.to(torch.int32), token.reshape(c["batch"], -1).gather(1, at).to(torch.int32)


def _plain_fork(s):
    """Every request grows by one token."""
    page, table, refs = s["case"]["page"], s["table"].long(), s["refs"]
    (B, width), pages = table.shape, refs.numel()
    rows, cols = torch.arange(B, device="cuda"), torch.arange(width, device="cuda")
    live = s["parent"] >= 0
    parent = s["parent"].long().clamp_min(0)
    children = torch.zeros(B, dtype=torch.int32, device="cuda").index_add_(0, parent, live.to(torch.int32))
    held = (cols[None] < -(-s["lens"].long() // page)[:, None]) & (table >= 0) & (table < pages)
    more = torch.where(held, (children - 1)[:, None], 0)
    refs = torch.cat([refs, refs.new_zeros(1)]).index_add(0, torch.where(held, table, pages).flatten(), more.flatten().to(torch.int32))
    # the children's rows; a tail that is not full is kept by the lowest of its writers if nobody else holds it
    n = torch.where(live, s["lens"][parent].long(), 0)
    used = -(-n // page)
    new = torch.where(live[:, None] & (cols[None] < used[:, None]), table[parent], -1)
    tail = new.gather(1, (n // page).clamp_max(width - 1)[:, None])[:, 0]
    writes = live & (n % page != 0) & (tail >= 0)
    tail = torch.where(writes, tail, pages)
    writers = torch.zeros_like(refs).index_add_(0, tail, writes.to(torch.int32))
    lowest = torch.full((pages + 1,), B, device="cuda").scatter_reduce_(0, tail, rows, "amin")
    copies = writes & ~((refs[tail] == writers[tail]) & (lowest[tail] == rows))
    # pages for the copies and for the next token, the free ones of the lowest index
    grows = live & (n % page == 0)
    free = torch.nonzero(torch.cat([refs[:pages] <= 0, refs.new_ones(1) > 0]))[:, 0]
    wants = (copies | grows).long()
    at = wants.cumsum(0) - wants
    there = (copies | grows) & (at < free.numel() - 1)
    page_of = torch.where(there, free[at.clamp_max(free.numel() - 1)], -1)
    refs = refs.index_add(0, torch.where(copies, tail, pages), -copies.to(torch.int32))
    refs[torch.where(there, page_of, pages)] = 1
    col = (n // page)[:, None]
    entry = torch.where(copies | grows, page_of, new.gather(1, col)[:, 0])
    new = new.scatter(1, col, torch.where(live, entry, -1)[:, None])
    slots = torch.where(live & (entry >= 0), entry * page + n % page, -1)
    moved = copies & there
    place = torch.where(moved, moved.long().cumsum(0) - 1, B)
    moves = torch.tensor([[-1, -1, 0]], device="cuda").repeat(B + 1, 1)
    moves[place] = torch.stack([tail, page_of, n % page], 1)
    info = torch.stack([moved.sum(), wants.sum() - there.sum()])
    to = lambda t: t.to(torch.int32)  # noqa: E731
    return to(new), to(torch.where(live, n + 1, 0)), to(refs[:pages]), slots[:, None], to(moves[:B]), to(info)


def _plain_compact(s):
    table, refs = s["table"].long(), s["refs"]
    pages = refs.numel()
    most, held, at = pages // 2, refs > 0, torch.arange(pages, device="cuda")
    used = held.sum()
    goes, hole = held & (at >= used), ~held & (at < used)
    order = lambda m: torch.where(m, m.long().cumsum(0) - 1, most)  # noqa: E731
    moves = torch.full((most + 1, 3), s["case"]["page"], device="cuda")
    moves[order(goes), 0] = at
    moves[order(hole), 1] = at
    to = torch.where(goes, moves[order(goes), 1], at)
    valid = (table >= 0) & (table < pages)
    moved = torch.where(valid, to[torch.where(valid, table, 0)], table)
    new = torch.zeros_like(refs).scatter_add_(0, to, torch.where(held, refs, 0))
    real = torch.arange(most, device="cuda")[:, None] < goes.sum()
    moves = torch.where(real, moves[:most], torch.tensor([-1, -1, 0], device="cuda"))
    return moved.to(torch.int32), new, moves.to(torch.int32), torch.stack([goes.sum(), used]).to(torch.int32)


def _copied(s):
    """What the moves wrote: a 16-bit cache whole, of an 8-bit one the written pages as the values they stand for."""
    if s["scales"] is None:
        return s["kv"]
    dst = s["moves"][: s["case"]["moves"], 1].long()
    return s["kv"][:, dst] * s["scales"][:, dst][..., None]


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        from paper_2202_05239_amd import binding as f8
        if kind == "beam":
            return f8.f8_beam_step(s["logits"], s["scores"], keep=c["keep"], done=s["done"], eos=s["eos"])
        if kind == "fork":
            return f8.f8_kv_fork(s["parent"], s["table"], s["lens"], s["refs"], c["page"])
        if kind == "compact":
            return f8.f8_kv_compact(s["table"], s["refs"], c["page"])
        cache = dict(k_scale=s["scales"][0], v_scale=s["scales"][1]) if s["scales"] is not None else {}
        if kind == "copy":
            f8.f8_kv_copy(s["moves"], s["kv"][0], s["kv"][1], **cache)
            return _copied(s)
        return f8.f8_attend_shared(s["q"], s["kv"][0], s["kv"][1], s["table"], s["lens"], s["first"], s["shared"], max_len=s["longest"], **cache)
    if kind == "attend":
        return _plain_attend(s, torch.float32).to(s["q"].dtype)
    if kind == "beam":
        return _plain_beam(s)
    if kind == "fork":
        return _plain_fork(s)
    if kind == "compact":
        return _plain_compact(s)
    src, dst, n = s["moves"].long().clamp_min(0).unbind(1)
    there = torch.arange(c["page"], device="cuda")[None] < n[:, None]
    s["kv"][:, dst] = torch.where(there[None, :, :, None, None], s["kv"][:, src], s["kv"][:, dst])
    if s["scales"] is not None:
        s["scales"][:, dst] = torch.where(there[None, :, :, None], s["scales"][:, src], s["scales"][:, dst])
    return _copied(s)


def work(case):
    kind = case["kind"]
    if kind == "attend":
        H, G, D, sizes, prefixes, tails = case["heads"], case["group"], case["D"], _sizes(case), _prefixes(case), _tails(case)
        member = [i for i, n in enumerate(sizes) for _ in range(n)]
        read = sum(prefixes) + sum(tails)
        seen = sum(prefixes[member[b]] + t for b, t in enumerate(tails) if t)
        row = D * BYTES[case["cache"]] + (4 if case["cache"] == "s8" else 0)
        return {"bytes": 2 * read * H * row + 2 * len(tails) * H * G * D * 2 + 4 * (read // case["page"] + 2 * len(tails) + 2 * len(sizes)),
                "flops": 4 * seen * H * G * D}
    if kind == "beam":
        rows = case["batch"] * case["beams"]
        return {"bytes": rows * (case["vocab"] * BYTES[case["type"]] + 5) + 12 * case["batch"] * case["keep"], "flops": 4 * rows * case["vocab"]}
    if kind == "fork":
        shared, behind = _fork_lens(case)
        used = sum(s * case["n"] for s in shared) + sum(-(-t // case["page"]) for t in behind)
        pages = sum(shared) + sum(-(-t // case["page"]) for t in behind) + case["spare"]
        B, width = len(behind), -(-case["longest"] // case["page"]) + 2
        return {"bytes": 4 * used + 4 * B * width + 8 * pages + 32 * B, "flops": used + pages}
    if kind == "compact":
        n = case["rows"] * case["cols"]
        return {"bytes": 8 * n + 8 * case["pages"] + 12 * (case["pages"] // 2), "flops": n + case["pages"]}
    tokens = case["moves"] * (case["page"] if case["full"] else (case["page"] + 1) / 2)
    row = case["D"] * BYTES[case["cache"]] + (4 if case["cache"] == "s8" else 0)
    return {"bytes": int(4 * tokens * case["heads"] * row + 12 * case["places"]), "flops": 0}


def _exact_attend(s):
    """Request by request: its pages one behind the other."""
    c = s["case"]
    H, G, D, page = c["heads"], c["group"], c["D"], c["page"]
    lens = s["lens"].tolist()
    out = torch.zeros(len(lens), H, G, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n == 0:
            continue
        ids = s["table"][b, : -(-n // page)].long()
        k, v = (s["kv"][i, ids].double().reshape(-1, H, D)[:n] for i in range(2))
        if s["scales"] is not None:
            k, v = (a * s["scales"][i, ids].double().reshape(-1, H, 1)[:n] for i, a in enumerate((k, v)))
        q = s["q"][b].double().reshape(H, G, D)
        for h in range(H):
            out[b, h] = (q[h] @ k[:, h].t() / math.sqrt(D)).softmax(-1) @ v[:, h]
    return out.reshape(len(lens), H * G, D)


def _exact_beam(s):
    """All scores of a prompt in one row, the largest taken off one by one."""
    c = s["case"]
    total = torch.empty(c["batch"], c["keep"], dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        full = s["logits"][b].double().log_softmax(-1) + s["scores"][b].double()[:, None]
        if s["done"] is not None:
            ended = torch.full_like(full, -math.inf)
            ended[:, s["eos"]] = s["scores"][b].double()
            full = torch.where(s["done"][b][:, None], ended, full)
        total[b] = full.flatten().topk(c["keep"]).values
    return total, None, None


def _exact_copy(s):
    """Move by move."""
    kv, scales = s["kv"], s["scales"]
    for src, dst, n in s["moves"][: s["case"]["moves"]].tolist():
        kv[:, dst, :n] = kv[:, src, :n]
        if scales is not None:
            scales[:, dst, :n] = scales[:, src, :n]
    if scales is None:
        return kv.double()
    dst = s["moves"][: s["case"]["moves"], 1].long()
    return kv[:, dst].double() * scales[:, dst].double()[..., None]


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None                                              # whole numbers
    return {"attend": _exact_attend, "beam": _exact_beam, "copy": _exact_copy}[case["kind"]](prepare(case, seed))
