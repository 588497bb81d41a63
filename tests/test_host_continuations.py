"""What the calls for several continuations of one prompt refuse, before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2202_05239_amd import binding as f8
from test_host_tokens import BAD_LAYOUTS, ODD, P, a_desc, layout


def beam(d, logits=P, scores=P, done=None, score=P, parent=P, token=P, ws=P, n=1 << 40):
    return f8.lib().f8_beam_step(logits, scores, done, score, parent, token, d, ws, n, None)


def b_desc(**kw):
    d = dict(batch=2, beams=3, vocab=100, keep=4, type=f8.F8_BF16, eos=0, ld=100)
    d.update(kw)
    return f8.f8_beam_desc(**d)


def test_beam_step():
    L = f8.lib()
    assert beam(None) == 1
    for k in ("logits", "scores", "score", "parent", "token", "ws"):
        assert beam(b_desc(), **{k: None}) == 1, k
    for bad in (dict(batch=-1), dict(beams=0), dict(vocab=0), dict(keep=0), dict(keep=301), dict(ld=99), dict(batch=1 << 30, beams=512)):
        assert beam(b_desc(**bad)) == 2, bad
    assert beam(b_desc(eos=-1), done=P) == 2 and beam(b_desc(eos=100), done=P) == 2
    assert beam(b_desc(type=f8.F8_S8)) == 5
    for k in ("scores", "score", "parent", "token", "ws"):
        assert beam(b_desc(), **{k: ODD}) == 7, k
    assert beam(b_desc(), logits=ODD) == 7
    for bad in (dict(keep=65), dict(beams=1025, keep=1), dict(vocab=16385, ld=16385, beams=128, keep=64), dict(vocab=1 << 30, ld=1 << 30, beams=1, keep=1)):
        assert beam(b_desc(**bad)) == 8, bad
    need = L.f8_beam_workspace_bytes(2, 3, 100, 4)
    assert need == 2 * 3 * (16 + 4 * 8) and beam(b_desc(), n=need - 1) == 2
    assert beam(b_desc(), scores=at(1), score=at(1)) == 2                   # scores that are read while they are written
    assert L.f8_beam_workspace_bytes(0, 3, 100, 4) == 0 and L.f8_beam_workspace_bytes(2, 3, 100, 65) == 0
    assert beam(b_desc(batch=0), logits=None) == 0


def at(i):
    return ctypes.c_void_p(0x1000 * (i + 1))


def fork(d, ws=P, n=1 << 40, **kw):
    names = ("parent", "table", "lens", "refs", "table_out", "lens_out", "refs_out", "slots", "moves", "info")
    return f8.lib().f8_kv_fork(*(kw.get(k, at(i)) for i, k in enumerate(names)), d, ws, n, None)


def k_desc(**kw):
    d = dict(batch=3, cols=5, pages=40, page_size=16, grow=1, table_ld=5, out_ld=5)
    d.update(kw)
    return f8.f8_kv_fork_desc(**d)


def test_fork():
    L = f8.lib()
    assert fork(None) == 1 and fork(k_desc(), ws=None) == 1
    for k in ("parent", "table", "lens", "refs", "table_out", "lens_out", "refs_out", "slots", "moves", "info"):
        assert fork(k_desc(), **{k: None}) == 1, k
        assert fork(k_desc(), **{k: ODD}) == 7, k
    assert fork(k_desc(), slots=ctypes.c_void_p(0x1004)) == 7 and fork(k_desc(), ws=ctypes.c_void_p(0x1008)) == 7
    for bad in (dict(batch=-1), dict(batch=65536), dict(cols=0), dict(pages=0), dict(page_size=0), dict(grow=-1), dict(table_ld=4), dict(out_ld=4),
                dict(cols=1 << 20, page_size=1 << 12, table_ld=1 << 20, out_ld=1 << 20)):
        assert fork(k_desc(**bad)) == 2, bad
    for bad in (dict(batch=60000, cols=10000, table_ld=10000, out_ld=10000), dict(pages=1 << 30), dict(batch=60000, grow=1 << 20)):
        assert fork(k_desc(**bad)) == 8, bad
    for out, of in (("table_out", 1), ("lens_out", 2), ("lens_out", 0), ("refs_out", 3)):
        assert fork(k_desc(), **{out: at(of)}) == 2, out                # an output that is an input
    need = L.f8_kv_fork_workspace_bytes(3, 40)
    assert need > 0 and fork(k_desc(), n=need - 1) == 2 and L.f8_kv_fork_workspace_bytes(0, 40) == 0 and L.f8_kv_fork_workspace_bytes(3, 0) == 0
    assert fork(k_desc(batch=0), parent=None) == 0


def test_compaction():
    L = f8.lib()

    def compact(d, ws=P, n=1 << 40, **kw):
        return L.f8_kv_compact(*(kw.get(k, at(i)) for i, k in enumerate(("table", "refs", "table_out", "refs_out", "moves", "info"))), d, ws, n, None)
    desc = lambda **kw: f8.f8_kv_compact_desc(**{**dict(rows=3, cols=5, pages=40, page_size=16, table_ld=5, out_ld=5), **kw})  # noqa: E731
    assert compact(None) == 1 and compact(desc(), ws=None) == 1
    for k in ("table", "refs", "table_out", "refs_out", "moves", "info"):
        assert compact(desc(), **{k: None}) == 1, k
        assert compact(desc(), **{k: ODD}) == 7, k
    for bad in (dict(rows=-1), dict(cols=-1), dict(pages=0), dict(page_size=0), dict(table_ld=4), dict(out_ld=4)):
        assert compact(desc(**bad)) == 2, bad
    assert compact(desc(pages=1 << 30)) == 8 and compact(desc(), refs_out=at(1)) == 2
    need = L.f8_kv_compact_workspace_bytes(40)
    assert need > 0 and compact(desc(), n=need - 1) == 2 and compact(desc(), ws=ctypes.c_void_p(0x1008)) == 7
    assert compact(desc(out_ld=6), table_out=at(0)) == 2                     # in place, with rows at another distance
    assert L.f8_kv_compact_workspace_bytes(0) == 0


def test_copies():
    L = f8.lib()
    copy = lambda c=layout(), n=2, moves=P, count=None, k=P, v=P, ks=P: L.f8_kv_copy(moves, count, k, v, ks, P, c, n, None)  # noqa: E731
    for bad, code in BAD_LAYOUTS:
        assert copy(layout(**bad)) == code, bad
    assert copy(None) == 1 and copy(n=-1) == 2 and copy(n=0, moves=None) == 0
    assert copy(moves=None) == 1 and copy(k=None) == 1 and copy(v=None) == 1 and copy(ks=None) == 1
    assert copy(moves=ODD) == 7 and copy(count=ODD) == 7 and copy(ks=ODD) == 7 and copy(layout(type=f8.F8_F16), k=ODD) == 7
    assert copy(layout(page_size=1 << 30)) == 8 and copy(layout(page_size=1 << 20), n=1 << 30) == 8


def test_attention():
    L = f8.lib()

    def att(c=layout(), d=a_desc(max_len=4096, table_cols=256, table_ld=256), q=P, k=P, ks=P, table=P, lens=P, first=P, shared=P, out=P, groups=1, ws=P, n=1 << 40):
        return L.f8_attend_shared(q, k, P, ks, P, table, lens, first, shared, out, c, d, groups, ws, n, None)
    for bad, code in BAD_LAYOUTS:
        assert att(layout(**bad)) == code, bad
    for k in ("c", "d", "q", "k", "ks", "table", "lens", "first", "shared", "out", "ws"):
        assert att(**{k: None}) == 1, k
    assert att(groups=-1) == 2 and att(groups=65536) == 2
    for bad in (dict(batch=-1), dict(batch=65536), dict(q_heads=3), dict(max_len=33), dict(table_ld=1), dict(scale=float("nan"))):
        assert att(d=a_desc(**bad)) == 2, bad
    assert att(d=a_desc(type=f8.F8_F32)) == 5 and att(layout(type=f8.F8_BF16)) == 5
    assert att(first=ODD) == 7 and att(shared=ODD) == 7 and att(q=ODD) == 7 and att(ws=ctypes.c_void_p(0x1008)) == 7 and att(layout(head_stride=60)) == 7
    need = L.f8_attend_shared_workspace_bytes(2, 1, 4, 2, 64, 4096)
    assert need > 0 and att(n=need - 1) == 2
    assert att(layout(heads=512), d=a_desc(batch=65535, q_heads=512, max_len=4096, table_cols=256, table_ld=256)) == 8
    assert att(d=a_desc(batch=0), q=None, first=None) == 0
    # without groups, and where requests are short, the call is f8_attend_paged with its workspace
    assert L.f8_attend_shared_workspace_bytes(2, 0, 4, 2, 64, 4096) == L.f8_attend_workspace_bytes(2, 4, 2, 64, 4096) > 0
    assert L.f8_attend_shared_workspace_bytes(2, 3, 4, 2, 64, 30) == 0 and L.f8_attend_shared_workspace_bytes(2, 1, 5, 2, 64, 4096) == 0


def test_binding_refuses_what_the_library_cannot_see():
    i32 = torch.int32
    x, s = torch.zeros(2, 3, 50), torch.zeros(2, 3)
    with pytest.raises(ValueError):
        f8.f8_beam_step(x[0], s)
    with pytest.raises(ValueError):
        f8.f8_beam_step(x.transpose(0, 1), s.t())
    with pytest.raises(ValueError):
        f8.f8_beam_step(x.transpose(1, 2), s)
    with pytest.raises(ValueError):
        f8.f8_beam_step(torch.zeros(2, 1, 50).expand(2, 3, 50), s)
    with pytest.raises(ValueError):
        f8.f8_beam_step(x, s[:1])
    with pytest.raises(ValueError):
        f8.f8_beam_step(x, s.double())
    with pytest.raises(TypeError):
        f8.f8_beam_step(x.to(i32), s)
    with pytest.raises(TypeError):
        f8.f8_beam_step(x, s, done=s)
    with pytest.raises(ValueError):
        f8.f8_beam_step(x, s, out=(torch.zeros(2, 3), torch.zeros(2, 3), torch.zeros(2, 3)))
    with pytest.raises(RuntimeError, match="gradient"):
        f8.f8_beam_step(x.requires_grad_(), s)
    table, lens, refs, parent = torch.zeros(2, 4, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(9, dtype=i32), torch.zeros(2, dtype=i32)
    with pytest.raises(TypeError):
        f8.f8_kv_fork(parent, table.long(), lens, refs, 16)
    with pytest.raises(ValueError):
        f8.f8_kv_fork(parent, table.t(), lens, refs, 16)
    with pytest.raises(ValueError):
        f8.f8_kv_fork(parent[:1], table, lens, refs, 16)
    with pytest.raises(ValueError):
        f8.f8_kv_fork(parent, table, lens.long(), refs, 16)
    with pytest.raises(ValueError):
        f8.f8_kv_fork(parent, table[:1].expand(2, 4), lens, refs, 16)
    with pytest.raises(TypeError):
        f8.f8_kv_compact(table.long(), refs, 16)
    with pytest.raises(ValueError):
        f8.f8_kv_compact(table, refs.long(), 16)
    kv = torch.zeros(2, 3, 16, 2, 64).half()
    with pytest.raises(ValueError):
        f8.f8_kv_copy(torch.zeros(4, 2, dtype=i32), kv[0], kv[1])
    with pytest.raises(ValueError):
        f8.f8_kv_copy(torch.zeros(4, 3), kv[0], kv[1])
    with pytest.raises(TypeError):
        f8.f8_kv_copy(torch.zeros(4, 3, dtype=i32), kv[0].to(torch.int8), kv[1].to(torch.int8))
    with pytest.raises(TypeError):
        f8.f8_kv_copy(torch.zeros(4, 3, dtype=i32), kv[0], kv[1], info=torch.zeros(2))
    q, lens, table = torch.zeros(2, 4, 64).half(), torch.ones(2, dtype=i32), torch.zeros(2, 3, dtype=i32)
    with pytest.raises(ValueError):
        f8.f8_attend_shared(q, kv[0], kv[1], table, lens, torch.zeros(1, dtype=i32), torch.zeros(1, dtype=i32))
    with pytest.raises(ValueError):
        f8.f8_attend_shared(q, kv[0], kv[1], table, lens, torch.zeros(2), torch.zeros(1, dtype=i32))
    with pytest.raises(RuntimeError, match="gradient"):
        f8.f8_attend_shared(q.requires_grad_(), kv[0], kv[1], table, lens, torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32))


def test_forks_by_more_tokens_than_a_cache_has():
    # the largest step that 32-bit counters pass over; more is refused before anything is launched
    for grow in (0x7fff0001, 0x7fffffff):
        assert fork(k_desc(batch=1, grow=grow, page_size=1 << 20)) == 2
    assert fork(k_desc(batch=1, grow=0x7fff0000, page_size=1 << 20), ws=None) == 1
