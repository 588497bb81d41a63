"""Beam search's selection against its definition in 64 bits: every score of a prompt in one row, sorted."""
import pytest
import torch

from paper_2202_05239_amd import binding as f8

pytestmark = pytest.mark.gpu

DEV = "cuda"
INF = float("inf")


def definition(logits, scores, done=None, eos=0):
    """S [batch][beams * vocab] in 64 bits."""
    x, score = logits.double(), scores.double()[..., None]
    lse = x.logsumexp(-1, keepdim=True)
    s = torch.where(lse == -INF, -INF, score + (x - torch.where(lse == -INF, 0, lse)))
    if done is not None:
        ended = torch.full_like(s, -INF)
        ended[..., eos] = scores.double()
        s = torch.where(done.bool()[..., None], ended, s)
    bad = lse.isnan() | (lse == INF)
    if done is not None:
        bad &= ~done.bool()[..., None]
    s = torch.where(bad | score.isnan() | (score == INF), float("nan"), s)
    return s.flatten(1)


def check(logits, scores, keep, done=None, eos=0, got=None):
    """Errors of S: an exponential is off by its argument's and its own last place (2^-22), 64 of them are added in 32 bits (2^-18) at
    most, sums of them in 64, so the logarithm is off by 2^-17 and the order may differ where S does by less; a score is rounded to 32 bits."""
    B, K, V = logits.shape
    if got is None:
        got = f8.f8_beam_step(logits.to(DEV), scores.to(DEV), keep=keep, done=None if done is None else done.to(DEV), eos=eos)
    score, parent, token = (t.cpu() for t in got)
    s = definition(logits, scores, done, eos)
    # (64 bits may give two logits of a beam the same S where its score is very large; as real numbers their S are as the logits are)
    s3 = torch.where(s.isnan(), INF, s).view(B, K, V)
    inside = torch.sort(torch.where(s3.isfinite(), logits.double(), s3), dim=-1, descending=True, stable=True).indices
    want, order = torch.sort(s3.gather(-1, inside).flatten(1), dim=-1, descending=True, stable=True)
    order = (inside + torch.arange(K)[:, None] * V).flatten(1).gather(1, order)
    want, order = want[:, :keep], order[:, :keep]
    at = (parent.long() - torch.arange(B)[:, None] * K) * V + token
    assert ((at >= 0) & (at < K * V)).all()
    mine = s.gather(1, at)
    tol = 2.0 ** -17 + 2.0 ** -24 * torch.where(want.isfinite(), want.abs(), 0)
    assert torch.equal(score.isnan(), mine.isnan()) and torch.equal(score.isnan(), want == INF)
    real = want.isfinite()
    assert torch.equal(score == -INF, want == -INF)
    assert ((score.double() - want).abs()[real] <= tol[real]).all()
    assert ((mine - want).abs()[real] <= tol[real]).all()
    assert all(len(set(r.tolist())) == keep for r in at)                # nothing twice
    # the same choice wherever S tells the candidates apart, or they are exactly alike
    clear = torch.ones_like(real)
    gap = (want[:, 1:] - want[:, :-1]).abs()
    near = (gap <= 2 * tol[:, 1:]) & (gap > 0) & gap.isfinite()
    clear[:, 1:] &= ~near
    clear[:, :-1] &= ~near
    clear[:, -1] = clear[:, -1] & (keep == K * V)
    assert torch.equal(torch.where(clear, at, -1), torch.where(clear, order, -1))
    return at, order


def draw(seed, B, K, V, dtype, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(B, K, V, generator=g)).to(dtype), -20 * torch.rand(B, K, generator=g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,K,V,keep", [(1, 1, 1, 1), (2, 1, 5, 5), (1, 4, 7, 28), (3, 2, 100, 4), (1, 4, 2047, 4), (2, 5, 2049, 10), (1, 3, 8193, 64), (5, 16, 5001, 32),
                                        (1, 1, 16385, 1), (2, 2, 50001, 7), (1, 8, 131072, 16), (70, 4, 1000, 8), (1, 100, 33, 64), (300, 5, 4097, 5)])
def test_sizes(dtype, B, K, V, keep):
    logits, scores = draw(B * 7 + V, B, K, V, dtype)
    check(logits, scores, keep)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lowest_beam_and_token(dtype):
    # all alike, alike in blocks, beams that are copies of one another
    for V in (3, 70, 5000, 40000):
        flat = torch.zeros(2, 3, V, dtype=dtype)
        at, order = check(flat, torch.zeros(2, 3), min(3 * V, 20))
        assert torch.equal(at, order)
        steps = (torch.arange(V) % 7).to(dtype).expand(2, 3, V).contiguous()
        at, order = check(steps, torch.zeros(2, 3), min(3 * V, 20))
        assert torch.equal(at, order)
        logits, _ = draw(V, 2, 1, V, dtype)
        at, order = check(logits.expand(2, 3, V).contiguous(), torch.full((2, 3), -1.5), min(3 * V, 13))
        assert torch.equal(at, order)
    signed = torch.zeros(1, 1, 50, dtype=dtype)
    signed[..., ::2] = -0.0
    at, _ = check(signed, torch.zeros(1, 1), 6)
    assert at.tolist() == [[0, 1, 2, 3, 4, 5]]


def test_logits_in_any_order():
    # sorted either way, the largest all in one place: far more pass the first bound than are kept
    for V in (5000, 16384, 60000):
        up = torch.linspace(-5, 5, V).view(1, 1, V)
        for x in (up, up.flip(-1), torch.where(torch.arange(V) // 8 % 256 < 17, up + 30, up), torch.cat([up[..., : V // 2], up[..., : V - V // 2] + 9], -1)):
            for keep in (1, 16, 64):
                check(x.contiguous(), torch.zeros(1, 1), keep)


def test_masked_vocabularies():
    logits, scores = draw(3, 4, 3, 30000, torch.float32)
    g = torch.Generator().manual_seed(4)
    logits[0] = torch.where(torch.rand(3, 30000, generator=g) < 0.999, -INF, logits[0])       # few tokens are allowed
    logits[1, 0] = -INF                                                                        # a beam without any
    logits[2] = -INF                                                                           # a prompt without any
    logits[3, :, 5:] = -INF
    at, order = check(logits, scores, 40)
    assert torch.equal(at[2], torch.arange(40))
    lowest = torch.finfo(torch.float32).min                                                    # a mask of the type's lowest value
    logits = torch.full((1, 2, 9000), lowest)
    logits[0, 1, 77] = 1.0
    check(logits, torch.tensor([[-1.0, -30.0]]), 6)
    for dtype in (torch.float16, torch.bfloat16):
        x = torch.full((1, 2, 9000), torch.finfo(dtype).min, dtype=dtype)
        check(x, torch.tensor([[-1.0, -3.0]]), 6)
        x[0, 0, 8000], x[0, 1, 3] = torch.finfo(dtype).max, 2.0
        check(x, torch.tensor([[-1.0, -3.0]]), 6)


def test_scores_that_start_or_end_a_search():
    logits, scores = draw(5, 3, 4, 700, torch.bfloat16)
    scores[0, 1:] = -INF                                                                       # the first step: one beam
    scores[1] = -INF
    scores[2] = -1e30
    check(logits, scores, 8)


@pytest.mark.parametrize("eos", [0, 2, 699])
def test_finished_beams(eos):
    logits, scores = draw(6, 6, 4, 700, torch.float16)
    done = torch.rand(6, 4, generator=torch.Generator().manual_seed(7)) < 0.5
    done[0], done[1] = True, False
    logits[2] = float("nan")                                                                   # not read where all are done
    done[2] = True
    for d in (done, done.to(torch.uint8) * 255):
        check(logits, scores, 4, d, eos)
        check(logits, scores, 40, d, eos)
    check(logits[:, :, :3], scores, 12, done, min(eos, 2))                                     # more than a beam has tokens


def test_what_is_no_number_shows():
    for V in (50, 20000):
        for bad in (float("nan"), INF):
            logits, scores = draw(8, 3, 3, V, torch.float32)
            logits[0, 1, V - 1] = bad
            scores[1, 2] = bad
            at, order = check(logits, scores, 5)
            assert torch.equal(at[0], V + torch.arange(5)) and torch.equal(at[1], 2 * V + torch.arange(5))
            logits[2] = bad
            check(logits, scores, 5)


def test_strided_rows_and_given_results():
    big = torch.randn(3, 4, 1009, generator=torch.Generator().manual_seed(9)).bfloat16()
    scores = -torch.rand(3, 4)
    view = big.to(DEV)[:, :, 3:900]
    out = (torch.empty(3, 8, device=DEV), torch.empty(3, 8, dtype=torch.int32, device=DEV), torch.empty(3, 8, dtype=torch.int32, device=DEV))
    got = f8.f8_beam_step(view, scores.to(DEV), keep=8, out=out)
    assert got is out
    check(big[:, :, 3:900], scores, 8, got=got)
    one = big.to(DEV)[1:2, 2:3, 5:]                                                             # a single row of any distance
    check(big[1:2, 2:3, 5:], scores[:1, :1], 3, got=f8.f8_beam_step(one, scores[:1, :1].to(DEV), keep=3))
    none = f8.f8_beam_step(big.to(DEV)[:0], scores.to(DEV)[:0])
    assert none[0].shape == (0, 4)


def test_repeats_and_replays():
    logits, scores = draw(10, 4, 4, 30000, torch.bfloat16)
    x, s = logits.to(DEV), scores.to(DEV)
    ws = torch.empty(f8.lib().f8_beam_workspace_bytes(4, 4, 30000, 8), dtype=torch.uint8, device=DEV)
    want = [t.clone() for t in f8.f8_beam_step(x, s, keep=8, workspace=ws)]
    out = tuple(torch.empty_like(t) for t in want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f8.f8_beam_step(x, s, keep=8, out=out, workspace=ws)
    for _ in range(3):
        for t in out:
            t.zero_()
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    other, _ = draw(11, 4, 4, 30000, torch.bfloat16)
    x.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    check(other, scores, 8, got=out)


def test_another_stream():
    logits, scores = draw(12, 2, 4, 9000, torch.float32)
    x, s = logits.to(DEV), scores.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = f8.f8_beam_step(x, s)
    side.synchronize()
    check(logits, scores, 4, got=got)


def test_what_is_no_number_shows_under_a_score_of_minus_infinity():
    # -infinity plus NaN is NaN; of a beam that is done no logit is read
    for V in (50, 20000):
        for bad in (float("nan"), INF):
            logits, scores = draw(13, 4, 3, V, torch.float32)
            scores[:, 1] = -INF
            logits[0, 1, 7] = bad
            logits[1] = bad
            logits[2, 1] = -INF
            logits[3, 1, V - 1] = bad
            done = torch.zeros(4, 3, dtype=torch.bool)
            done[3, 1] = True
            at, order = check(logits, scores, 5, done)
            assert torch.equal(at[0], V + torch.arange(5))


def test_more_prompts_than_a_grid_dimension_holds():
    # 2^24 workgroups of 256 threads do not fit one dimension of a launch
    B = 2 ** 24 + 3
    x = torch.randn(B, 1, 2, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).half()
    scores = torch.zeros(B, 1, device=DEV)
    score, parent, token = f8.f8_beam_step(x, scores, keep=1)
    d = x.float()[:, 0]
    want = -torch.log1p(torch.exp(-(d[:, 0] - d[:, 1]).abs()))
    assert torch.equal(parent[:, 0], torch.arange(B, device=DEV, dtype=torch.int32))
    assert torch.equal(token[:, 0], (d[:, 1] > d[:, 0]).int())
    assert (score[:, 0] - want).abs().max().item() <= 2.0 ** -16


@pytest.mark.parametrize("B,K,V,keep", [(1, 16, 131072, 64), (1, 128, 100, 64), (2, 1024, 50, 8), (1, 32, 60000, 64), (1, 1, 2000000, 64)])
def test_as_many_candidates_as_a_prompt_may_have(B, K, V, keep):
    logits, scores = draw(V + K, B, K, V, torch.bfloat16)
    check(logits, scores, keep)
