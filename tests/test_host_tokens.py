"""What the calls on tokens refuse, before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2202_05239_amd import binding as f8

P = ctypes.c_void_p(0x1000)          # never dereferenced: every call below fails validation, or has nothing to do
ODD = ctypes.c_void_p(0x1001)


def q_desc(**kw):
    d = dict(rows=4, cols=64, x_type=f8.F8_BF16, y_type=f8.F8_S8, act=0, ldx=64, ldg=64, ldy=64)
    d.update(kw)
    return f8.f8_quant_tokens_desc(**d)


def quant(d, x=P, gate=None, y=P, scale=P):
    return f8.lib().f8_quant_tokens(x, gate, y, scale, d, None)


def test_quantiser():
    assert quant(None) == 1 and quant(q_desc(), x=None) == 1 and quant(q_desc(), y=None) == 1 and quant(q_desc(), scale=None) == 1
    assert quant(q_desc(act=1)) == 1                                       # an activation without a gate
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=65537, ldx=65537, ldy=65537), dict(ldx=63), dict(ldy=63)):
        assert quant(q_desc(**bad)) == 2, bad
    assert quant(q_desc(ldg=63), gate=P) == 2
    assert quant(q_desc(x_type=f8.F8_S8)) == 5 and quant(q_desc(y_type=f8.F8_F16)) == 5 and quant(q_desc(y_type=f8.F8_U8)) == 5
    assert quant(q_desc(), x=ODD) == 7 and quant(q_desc(), scale=ODD) == 7 and quant(q_desc(), gate=ODD) == 7
    assert quant(q_desc(act=3), gate=P) == 8
    assert quant(q_desc(rows=0), x=None, y=None, scale=None) == 0


def n_desc(**kw):
    d = dict(rows=4, cols=64, type=f8.F8_F16, y_type=f8.F8_F16, w_type=f8.F8_F32, post=0, pre=1, gate_rows=4, post_eps=1e-6, pre_eps=1e-6,
             res_scale=1.0, lda=64, ldr=64, ldg=64, ldo=64, ldy=64)
    d.update(kw)
    return f8.f8_norm_tokens_desc(**d)


def norm(d, a=P, res=P, gate=None, w=P, res_out=P, y=P, scale=None):
    return f8.lib().f8_norm_tokens(a, res, None, None, gate, w, None, res_out, y, scale, d, None)


def test_norms():
    assert norm(None) == 1 and norm(n_desc(), a=None) == 1 and norm(n_desc(), res_out=None, y=None) == 1
    assert norm(n_desc(y_type=f8.F8_S8)) == 1                              # codes without their scale
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=1 << 20), dict(lda=1), dict(ldr=63), dict(ldo=63), dict(ldy=63), dict(pre_eps=-1.0),
                dict(post_eps=float("nan"))):
        assert norm(n_desc(**bad)) == 2, bad
    assert norm(n_desc(gate_rows=0), gate=P) == 2 and norm(n_desc(ldg=3), gate=P) == 2
    assert norm(n_desc(type=f8.F8_S32)) == 5 and norm(n_desc(y_type=f8.F8_F32)) == 5 and norm(n_desc(w_type=f8.F8_BF16)) == 5
    assert norm(n_desc(pre=3)) == 8 and norm(n_desc(post=-1)) == 8
    assert norm(n_desc(), a=ODD) == 7 and norm(n_desc(), w=ctypes.c_void_p(0x1002)) == 7
    assert norm(n_desc(rows=0)) == 0


def l_desc(**kw):
    d = dict(M=4, N=8, K=32, x_type=f8.F8_S8, y_type=f8.F8_F32, ldx=32, ldw=32, ldy=8)
    d.update(kw)
    return f8.f8_linear_desc(**d)


def test_products():
    L = f8.lib()
    scaled = lambda d, x=P, sx=P, w=P, sw=P, b=None, y=P: L.f8_linear_scaled(x, sx, w, sw, b, y, d, None)  # noqa: E731
    assert scaled(None) == 1
    for k in ("x", "sx", "w", "sw", "y"):
        assert scaled(l_desc(), **{k: None}) == 1, k
    for bad in (dict(M=-1), dict(N=-1), dict(M=(1 << 26) + 1), dict(N=(1 << 26) + 1, ldy=1 << 27), dict(K=0), dict(K=131072, ldx=131072, ldw=131072), dict(ldx=31), dict(ldw=31), dict(ldy=7)):
        assert scaled(l_desc(**bad)) == 2, bad
    assert scaled(l_desc(x_type=f8.F8_F32)) == 5 and scaled(l_desc(y_type=f8.F8_S8)) == 5
    assert scaled(l_desc(), y=ODD) == 7 and scaled(l_desc(), sx=ODD) == 7 and scaled(l_desc(), b=ODD) == 7
    assert scaled(l_desc(M=0), x=None) == 0 and scaled(l_desc(N=0)) == 0
    tokens = lambda d, x=P, ws=P, n=1 << 20: L.f8_linear_tokens(x, P, P, None, P, d, ws, n, None)  # noqa: E731
    real = dict(x_type=f8.F8_BF16)
    assert tokens(l_desc()) == 5 and tokens(l_desc(K=65537, ldx=65537, ldw=65537, **real)) == 2
    real["M"] = 40
    assert tokens(l_desc(**real), ws=None) == 1 and tokens(l_desc(**real), ws=ODD) == 7 and tokens(l_desc(**real), x=ODD) == 7
    need = L.f8_linear_workspace_bytes(40, 32)
    assert need == 40 * 128 + 160 and tokens(l_desc(**real), n=need - 1) == 2
    assert L.f8_linear_workspace_bytes(1, 4096) == 0 and L.f8_linear_workspace_bytes(1, 4097) > 0      # the product quantises them itself
    assert L.f8_linear_workspace_bytes(0, 32) == 0


def layout(**kw):
    d = dict(type=f8.F8_S8, pages=4, page_size=16, heads=2, dim=64, page_stride=2048, token_stride=128, head_stride=64, scale_page=32, scale_token=2,
             scale_head=1)
    d.update(kw)
    return f8.f8_kv_layout(**d)


BAD_LAYOUTS = [(dict(type=f8.F8_F32), 5), (dict(pages=0), 2), (dict(page_size=0), 2), (dict(heads=0), 2), (dict(dim=8), 2), (dict(dim=72), 2),
               (dict(dim=272), 2), (dict(token_stride=-128), 2), (dict(scale_token=-1), 2)]


def test_append():
    L = f8.lib()
    d = f8.f8_kv_append_desc(3, f8.F8_F16, 128, 64, 128, 64)
    app = lambda c=layout(), d=d, k=P, slots=P, ks=P: L.f8_kv_append(k, P, slots, P, P, ks, P, c, d, None)  # noqa: E731
    for bad, code in BAD_LAYOUTS:
        assert app(layout(**bad)) == code, bad
    assert app(None) == 1 and app(d=None) == 1 and app(k=None) == 1 and app(slots=None) == 1 and app(ks=None) == 1
    assert app(k=ODD) == 7 and app(slots=ctypes.c_void_p(0x1004)) == 7
    assert app(d=f8.f8_kv_append_desc(-1, f8.F8_F16, 0, 0, 0, 0)) == 2 and app(d=f8.f8_kv_append_desc(3, f8.F8_S8, 0, 0, 0, 0)) == 5
    assert app(d=f8.f8_kv_append_desc(0, f8.F8_F16, 0, 0, 0, 0)) == 0


def a_desc(**kw):
    d = dict(batch=2, q_heads=4, type=f8.F8_F16, max_len=30, table_cols=2, scale=0.125, table_ld=2, q_token=256, q_head=64, o_token=256, o_head=64)
    d.update(kw)
    return f8.f8_attend_desc(**d)


def test_attention():
    L = f8.lib()

    def att(c=layout(), d=a_desc(), q=P, k=P, ks=P, table=P, lens=P, out=P, ws=P, n=1 << 30):
        return L.f8_attend_paged(q, k, P, ks, P, table, lens, out, c, d, ws, n, None)
    for bad, code in BAD_LAYOUTS:
        assert att(layout(**bad)) == code, bad
    for k in ("c", "d", "q", "k", "ks", "table", "lens", "out"):
        assert att(**{k: None}) == 1, k
    for bad in (dict(batch=-1), dict(batch=65536), dict(q_heads=3), dict(q_heads=0), dict(max_len=33), dict(max_len=-1), dict(table_cols=-1),
                dict(table_ld=1), dict(scale=float("nan"))):
        assert att(d=a_desc(**bad)) == 2, bad
    assert att(d=a_desc(type=f8.F8_F32)) == 5 and att(layout(type=f8.F8_BF16)) == 5      # a bf16 cache under f16 queries
    for bad in (dict(page_stride=2049), dict(token_stride=120), dict(head_stride=60)):
        assert att(layout(**bad)) == 7, bad
    assert att(k=ctypes.c_void_p(0x1008)) == 7 and att(q=ODD) == 7
    long = a_desc(max_len=4096, table_cols=256, table_ld=256)
    need = L.f8_attend_workspace_bytes(2, 4, 2, 64, 4096)
    assert need > 0 and att(d=long, ws=None) == 1 and att(d=long, n=need - 1) == 2 and att(d=long, ws=ctypes.c_void_p(0x1008)) == 7
    assert att(layout(heads=512), d=a_desc(batch=65535, q_heads=512)) == 8            # more pairs than a launch has workgroups
    assert att(d=a_desc(batch=0), q=None) == 0
    assert L.f8_attend_workspace_bytes(2, 5, 2, 64, 4096) == 0 and L.f8_attend_workspace_bytes(0, 4, 2, 64, 4096) == 0


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        f8.f8_quant_tokens(x.to(torch.int8))
    with pytest.raises(ValueError):
        f8.f8_quant_tokens(torch.zeros(64, 4).t())
    with pytest.raises(ValueError):
        f8.f8_quant_tokens(x, gate=torch.zeros(4, 32))
    with pytest.raises(TypeError):
        f8.f8_quant_tokens(x, gate=x.half())
    with pytest.raises(ValueError):
        f8.f8_norm_tokens(x, gate=torch.zeros(1, 64), gate_rows=3)
    with pytest.raises(ValueError):
        f8.f8_norm_tokens(x, pre_w=torch.zeros(63))
    w = torch.zeros(8, 64, dtype=torch.int8)
    with pytest.raises(TypeError):
        f8.f8_linear_scaled(x, torch.ones(4), w, torch.ones(8))
    with pytest.raises(TypeError):
        f8.f8_linear_tokens(x, w.float(), torch.ones(8))
    with pytest.raises(ValueError):
        f8.f8_linear_tokens(x, w[:, :32], torch.ones(8))
    with pytest.raises(ValueError):
        f8.f8_linear_tokens(x, w, torch.ones(7))
    kv = torch.zeros(2, 3, 16, 2, 64)
    with pytest.raises(TypeError):
        f8.f8_kv_append(torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), torch.zeros(1, dtype=torch.int64), *kv.to(torch.int8))
    with pytest.raises(ValueError):
        f8.f8_attend_paged(torch.zeros(1, 4, 32).half(), kv[0].half(), kv[1].half(), torch.zeros(1, 3, dtype=torch.int32), torch.ones(1, dtype=torch.int32))


def overlapping(rows, cols, dtype):
    """Matrices whose rows share elements: one row for all of them, rows one and four elements apart."""
    return [torch.zeros(1, cols, dtype=dtype).expand(rows, cols)] + [torch.zeros(cols + rows * s, dtype=dtype).unfold(0, cols, s)[:rows] for s in (1, 4)]


def test_binding_refuses_matrices_whose_rows_overlap():
    # the library takes rows that lie apart: with the width for their distance it would read behind the tensor
    x, w, s8 = torch.zeros(4, 64), torch.zeros(8, 64, dtype=torch.int8), torch.int8
    for bad in overlapping(4, 64, torch.float32):
        for call in (lambda: f8.f8_quant_tokens(bad), lambda: f8.f8_quant_tokens(x, gate=bad), lambda: f8.f8_quant_tokens(x, values=True, out=bad),
                     lambda: f8.f8_norm_tokens(bad), lambda: f8.f8_norm_tokens(x, res=bad), lambda: f8.f8_norm_tokens(x, gate=bad, gate_rows=1),
                     lambda: f8.f8_norm_tokens(x, res_out=bad), lambda: f8.f8_norm_tokens(x, out=bad),
                     lambda: f8.f8_linear_tokens(bad, w, torch.ones(8))):
            with pytest.raises(ValueError):
                call()
    for bad in overlapping(4, 64, s8):
        with pytest.raises(ValueError):
            f8.f8_linear_scaled(bad, torch.ones(4), w, torch.ones(8))
        with pytest.raises(ValueError):
            f8.f8_linear_scaled(torch.zeros(4, 64, dtype=s8), torch.ones(4), bad, torch.ones(4))
        with pytest.raises(ValueError):
            f8.f8_quant_tokens(x, out=bad)
    for bad in overlapping(4, 8, torch.float32):
        with pytest.raises(ValueError):
            f8.f8_linear_tokens(x, w, torch.ones(8), y=bad)
    kv, q, lens, table = torch.zeros(2, 3, 16, 2, 64).half(), torch.zeros(4, 4, 64).half(), torch.ones(4, dtype=torch.int32), torch.zeros(4, 3, dtype=torch.int32)
    for bad in overlapping(4, 8, torch.int32):
        with pytest.raises(ValueError):
            f8.f8_attend_paged(q, kv[0], kv[1], bad, lens)
    for bad in (torch.zeros(1, 4, 64).half().expand(4, 4, 64), torch.zeros(4, 1, 64).half().expand(4, 4, 64), torch.zeros(4, 200).half().as_strided((4, 4, 64), (200, 32, 1)),
                torch.zeros(4, 256).half().as_strided((4, 4, 64), (192, 64, 1))):
        with pytest.raises(ValueError):
            f8.f8_attend_paged(q, kv[0], kv[1], table, lens, out=bad)


def test_binding_takes_single_rows_of_any_stride():
    assert f8._matrix(torch.zeros(1, 64).expand(1, 64)) == 64 and f8._matrix(torch.zeros(64, 1).t()) == 64 and f8._matrix(torch.zeros(0, 64)) == 64
    assert f8._matrix(torch.zeros(4, 80)[:, :64]) == 80 and f8._matrix(torch.zeros(4, 1)) == 1 and f8._matrix(torch.zeros(4, 2)[:, :1]) == 2


def test_binding_refuses_what_autograd_follows():
    # (a result without its gradient would go unnoticed; under no_grad the same calls go on, here as far as a GPU is needed)
    x, w, one = torch.zeros(4, 64), torch.zeros(8, 64, dtype=torch.int8), torch.ones(8)
    live = lambda t: t.clone().requires_grad_()  # noqa: E731
    kv, q = torch.zeros(2, 3, 16, 2, 64).half(), torch.zeros(1, 4, 64).half()
    new, slot, table, lens = torch.zeros(1, 2, 64).half(), torch.zeros(1, dtype=torch.int64), torch.zeros(1, 3, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    calls = [lambda: f8.f8_quant_tokens(live(x)), lambda: f8.f8_quant_tokens(x, gate=live(x)),
             lambda: f8.f8_norm_tokens(live(x)), lambda: f8.f8_norm_tokens(x, res=live(x)), lambda: f8.f8_norm_tokens(x, pre_w=live(torch.ones(64))),
             lambda: f8.f8_linear_tokens(live(x), w, one), lambda: f8.f8_linear_tokens(x, w, live(one)), lambda: f8.f8_linear_tokens(x, w, one, bias=live(one)),
             lambda: f8.f8_linear_scaled(w, live(one), w, one), lambda: f8.f8_kv_append(live(new), new, slot, kv[0], kv[1]),
             lambda: f8.f8_attend_paged(live(q), kv[0], kv[1], table, lens)]
    for call in calls:
        with pytest.raises(RuntimeError, match="gradient"):
            call()
    with torch.no_grad():
        f8._no_gradient(live(x), None)
    f8._no_gradient(x, None)


def test_products_that_no_launch_holds_are_refused_before_anything_runs():
    # (without a GPU a launch is error 9: the quantiser in front must not have been tried)
    L = f8.lib()
    most = 1 << 26
    ws = L.f8_linear_workspace_bytes(most, 32)
    for y_type, w in ((f8.F8_F32, P), (f8.F8_BF16, P), (f8.F8_F16, ODD)):
        d = l_desc(M=most, N=most, y_type=y_type, ldy=most)
        assert L.f8_linear_scaled(P, P, w, P, None, P, d, None) == 8
        d.x_type = f8.F8_BF16
        assert L.f8_linear_tokens(P, w, P, None, P, d, P, ws, None) == 8
