"""A beam search over a paged cache, step by step: attention over the shared prompts, selection, forks, copies, appends and compactions together."""
import pytest
import torch

from paper_2202_05239_amd import binding as f8
from test_gpu_attend import DEV, HALF
from test_gpu_beam_step import check as check_beams

pytestmark = pytest.mark.gpu

PAGE, HEADS, GROUP, D, EOS = 16, 2, 2, 64, 7
VOCAB = HEADS * GROUP * D                                  # logits: the attention's output and a row of the last token


class Search:
    """A model whose keys, values, queries and logits are functions of a token; its cache and the state of its requests."""

    def __init__(self, prompts, beams, dtype, steps):
        g = torch.Generator().manual_seed(len(prompts) * 10 + beams)
        rand = lambda *s: torch.randn(*s, generator=g)     # noqa: E731
        self.k, self.v = rand(VOCAB, HEADS, D).to(dtype), rand(VOCAB, HEADS, D).to(dtype)
        self.q, self.bias = rand(VOCAB, HEADS * GROUP, D).to(dtype), rand(VOCAB, VOCAB)
        self.bias[:, EOS] += 2.5
        self.n, self.rows, self.dtype = beams, len(prompts) * beams, dtype
        self.prompts = [torch.randint(8, VOCAB, (n,), generator=g).tolist() for n in prompts]
        need = [-(-n // PAGE) for n in prompts]
        pages, cols = sum(need) + 3 * self.rows + 40, max(need) + -(-steps // PAGE) + 1
        order = torch.randperm(pages, generator=g).tolist()
        cache = torch.full((2, pages, PAGE, HEADS, D), float("nan")).to(dtype)
        table, refs = torch.full((self.rows, cols), -1, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32)
        for p, tokens in enumerate(self.prompts):
            for c in range(need[p]):
                page, part = order.pop(), tokens[c * PAGE:(c + 1) * PAGE]
                cache[0, page, :len(part)], cache[1, page, :len(part)] = self.k[part], self.v[part]
                table[p * beams:(p + 1) * beams, c] = page
                refs[page] = beams
        lens = torch.tensor(prompts, dtype=torch.int32).repeat_interleave(beams)
        score = torch.full((len(prompts), beams), float("-inf"))
        score[:, 0] = 0.0                                  # the beams are alike to begin with
        last = torch.tensor([t[-1] for t in self.prompts], dtype=torch.int32).repeat_interleave(beams).view(-1, beams)
        self.state = tuple(t.to(DEV) for t in (table, lens, refs, score, last, torch.zeros(len(prompts), beams, dtype=torch.bool)))
        self.cache = cache.to(DEV)
        self.first = torch.arange(0, self.rows + 1, beams, dtype=torch.int32, device=DEV)
        self.shared = torch.tensor(prompts, dtype=torch.int32, device=DEV)
        self.q, self.bias = self.q.to(DEV), self.bias.to(DEV)
        self.k_dev, self.v_dev = self.k.to(DEV), self.v.to(DEV)

    def step(self, state):
        """The state after one more token, and what came out on the way."""
        table, lens, refs, score, last, done = state
        k, v = self.cache[0], self.cache[1]
        o = f8.f8_attend_shared(self.q[last.flatten().long()], k, v, table, lens, self.first, self.shared)
        logits = (o.float().view(-1, self.n, VOCAB) + self.bias[last.long()])
        score2, parent, token = f8.f8_beam_step(logits, score, done=done, eos=EOS)
        table, lens, refs, slots, moves, info = f8.f8_kv_fork(parent.flatten(), table, lens, refs, PAGE)
        f8.f8_kv_copy(moves, k, v, info=info)
        t = token.flatten().long()
        f8.f8_kv_append(self.k_dev[t], self.v_dev[t], slots.flatten(), k, v)
        done = done.flatten()[parent.flatten().long()].view_as(done) | (token == EOS)
        return (table, lens, refs, score2, token, done), (o, logits, parent, info)

    def compact(self, state):
        table, refs, moves, info = f8.f8_kv_compact(state[0], state[2], PAGE)
        f8.f8_kv_copy(moves, self.cache[0], self.cache[1], info=info)
        return (table, state[1], refs) + state[3:], info


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("prompts,beams", [((600, 17, 1023), 4), ((777,), 9), ((530, 640, 512, 1, 900), 2)])
def test_a_search(prompts, beams, dtype):
    steps = 40
    s = Search(prompts, beams, dtype, steps)
    state, rows = s.state, s.rows
    history = [list(t) for t in s.prompts for _ in range(beams)]
    for i in range(steps):
        before = state
        state, (o, logits, parent, info) = s.step(state)
        # the attention over what the beams have said: the bounds of a 16-bit cache
        q = s.q[before[4].flatten().long()].cpu().double()
        for b in range(0, rows, 1 if i % 8 == 0 else 3):
            k, v = (e[history[b]].double().repeat_interleave(GROUP, 1) for e in (s.k, s.v))
            x = (q[b] * k).sum(-1) * D ** -0.5                                   # [tokens][heads]
            p = x.softmax(0)
            want = (p[..., None] * v).sum(0)
            size = (q[b].abs() * k.abs()).sum(-1).amax(0) * D ** -0.5
            delta = (D + 8) * 2.0 ** -24 * (size + x.abs().amax(0) + 1)
            mass = (p[..., None] * v.abs()).sum(0)
            tiny = len(v) * 2.0 ** -25 * (p[..., None] * v.abs().amax(-1, keepdim=True)).amax() if dtype == torch.float16 else 0.0
            err = mass * (HALF[dtype] + 4 * delta[:, None]) + tiny + HALF[dtype] * want.abs() + 2.0 ** -25
            assert ((o[b].cpu().double() - want).abs() <= err).all(), (i, b)
        check_beams(logits.cpu(), before[3].cpu(), beams, before[5].cpu(), EOS, got=(state[3], parent, state[4]))
        # the beams' tokens, and that their pages hold just these
        history = [history[p] + [t] for p, t in zip(parent.flatten().tolist(), state[4].flatten().tolist())]
        assert info.tolist()[1] == 0 and state[1].tolist() == [len(h) for h in history]
        if i % 7 == 6:
            state, moved = s.compact(state)
            used = moved.tolist()[1]
            assert (state[2][:used] > 0).all() and (state[2][used:] == 0).all()
        if i % 4 == 2 or i % 7 == 6:
            table, refs, cache = state[0].cpu(), state[2].cpu(), s.cache.cpu()
            held = torch.zeros_like(refs)
            for b, h in enumerate(history):
                pages = table[b, : -(-len(h) // PAGE)].long()
                held.scatter_add_(0, pages, torch.ones_like(pages, dtype=torch.int32))
                for e, c in ((s.k, cache[0]), (s.v, cache[1])):
                    assert torch.equal(c[pages].flatten(0, 1)[: len(h)], e[h]), (i, b)
            assert torch.equal(held, refs)


def test_a_captured_search():
    # two steps and a compaction under one graph; every replay against the same steps without it
    s = Search((700, 33, 512), 4, torch.bfloat16, 64)
    start, cache = s.state, s.cache.clone()

    def round_of(state):
        return s.compact(s.step(s.step(state)[0])[0])[0]
    want, state = [], start
    for _ in range(5):
        state = round_of(state)
        want.append((state, s.cache.clone()))
    held = tuple(t.clone() for t in start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = round_of(held)
        for a, b in zip(held, out):
            a.copy_(b)
    for _ in range(2):
        s.cache.copy_(cache)
        for a, b in zip(held, start):
            a.copy_(b)
        for state, kv in want:
            graph.replay()
            torch.cuda.synchronize()
            assert same(held, state)
            assert torch.equal(s.cache.view(torch.int16), kv.view(torch.int16))
