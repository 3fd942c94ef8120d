"""Refused calls of packed attention, the RMS norm and the balance loss: each argument error returns its code before
anything is launched, so these run without a GPU (the addresses are never read)."""
import ctypes as C
import math

import pytest

A = 1 << 20           # a 16-byte aligned address


def xs():
    from paper_2607_23264_amd import xstage
    return xstage


def test_rmsnorm():
    X = xs()

    def f(x=A, ldx=256, r=A, ldr=256, w=A, wt=X.XS_TYPE_F32, eps=1e-6, rows=4, cols=256, h=2 * A, ldh=256, y=3 * A, ldy=256, c=A, ldc=256, s=A, lds=4):
        return X.xs_rmsnorm(x, ldx, r, ldr, w, wt, eps, rows, cols, h, ldh, y, ldy, c, ldc, s, lds, None)

    for bad in (dict(x=None), dict(x=A + 8), dict(ldx=248), dict(ldx=260), dict(r=A + 2), dict(ldr=200), dict(w=None), dict(w=A + 8), dict(wt=2),
                dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(rows=-1), dict(cols=0), dict(h=A + 4), dict(ldh=252), dict(y=A + 8),
                dict(ldy=128), dict(y=None, c=None, s=None), dict(c=None), dict(s=None), dict(c=A + 8), dict(ldc=128), dict(ldc=264), dict(s=A + 4),
                dict(lds=1), dict(lds=6), dict(h=A, ldh=264), dict(y=A, ldy=264), dict(h=A, ldx=264, ldr=264)):
        assert f(**bad) == X.XS_EINVAL, bad
    for bad in (dict(cols=252), dict(cols=32776, ldx=40000, ldr=40000, ldh=40000, ldy=40000), dict(rows=1 << 31)):
        assert f(**bad) == X.XS_EUNSUPPORTED, bad
    assert f(rows=0) == f(rows=0, x=None, r=None, h=None, y=None, c=None, s=None) == X.XS_OK


def test_rmsnorm_h_and_y_are_not_one_matrix():
    # y in the place of h would take the residual stream away
    X = xs()
    f = lambda h, y, ld=256, x=A, rows=4: X.xs_rmsnorm(x, 256, A, 256, A, X.XS_TYPE_F32, 1e-6, rows, 256, h, 256, y, ld, None, 0, None, 0, None)
    for bad in (dict(h=2 * A, y=2 * A), dict(h=2 * A, y=2 * A, ld=264), dict(h=A, y=A), dict(h=2 * A, y=2 * A, rows=0)):
        assert f(**bad) == X.XS_EINVAL, bad
    assert f(h=None, y=None, rows=0) == f(h=None, y=A, rows=0) == X.XS_OK


def test_rmsnorm_backward():
    X = xs()

    def f(dy=A, l1=256, dh=A, l2=256, h=2 * A, l3=256, w=A, wt=X.XS_TYPE_BF16, eps=1e-6, rows=4, cols=256, dx=3 * A, l4=256, dw=None):
        return X.xs_rmsnorm_backward(dy, l1, dh, l2, h, l3, w, wt, eps, rows, cols, dx, l4, dw, None, 0, None)

    for bad in (dict(dy=None), dict(dy=A + 8), dict(l1=248), dict(dh=A + 8), dict(l2=100), dict(h=None), dict(l3=252), dict(w=None), dict(wt=5), dict(eps=-1.0),
                dict(rows=-1), dict(cols=0), dict(dx=None), dict(l4=128), dict(dx=A + 8), dict(dw=A + 4), dict(dx=A, l4=264), dict(dx=2 * A, l4=264)):
        assert f(**bad) == X.XS_EINVAL, bad
    for bad in (dict(cols=12), dict(rows=1 << 31)):
        assert f(**bad) == X.XS_EUNSUPPORTED, bad
    assert f(rows=0) == f(rows=0, dy=None, dh=None, h=None, dx=None) == X.XS_OK
    n = C.c_int64()
    q = lambda r, c, p=C.byref(n): X.xs_rmsnorm_backward_workspace_bytes(r, c, p)
    assert q(-1, 8) == q(1, 0) == q(1, 8, None) == X.XS_EINVAL
    assert q(1, 12) == q(1 << 31, 8) == q(1, 32776) == X.XS_EUNSUPPORTED
    assert q(0, 8) == X.XS_OK and n.value == 0


def test_balance_loss():
    X = xs()
    g = lambda **kw: X.gate(**{**dict(E=64, k=4), **kw})
    res = X.gate(64, 4)
    res.reserved = 1

    def f(gate=g(), l=A, ld=64, T=8, idx=A, st=A, n=2, alpha=0.1, c=A, m=A, o=A, ws=A, nb=1 << 20):
        return X.xs_balance_loss(gate, l, ld, T, idx, st, n, alpha, c, m, o, ws, nb, None, None)

    def b(gate=g(), l=A, ld=64, T=8, st=A, n=2, alpha=0.1, c=A, dl=A, add=2 * A, lda=64, d=3 * A, ldd=64):
        return X.xs_balance_loss_backward(gate, l, ld, T, st, n, alpha, c, dl, add, lda, d, ldd, None, None)

    for bad in (dict(gate=None), dict(gate=g(E=0)), dict(gate=g(E=1025)), dict(gate=g(k=0)), dict(gate=g(k=33)), dict(gate=g(E=3)), dict(gate=g(score=2)),
                dict(gate=g(logits_type=3)), dict(gate=res), dict(l=None), dict(l=A + 2), dict(ld=63), dict(T=-1), dict(n=0), dict(n=65537),
                dict(st=None), dict(alpha=math.nan), dict(alpha=math.inf), dict(c=None)):
        assert f(**bad) == X.XS_EINVAL, bad
        assert b(**bad) == X.XS_EINVAL, bad
    for bad in (dict(idx=None), dict(m=None), dict(o=None)):
        assert f(**bad) == X.XS_EINVAL, bad
    for bad in (dict(ws=None), dict(ws=A + 8), dict(nb=64 * 8 - 1)):
        assert f(**bad) == X.XS_EWORKSPACE, bad
    for bad in (dict(dl=None), dict(add=A + 2), dict(lda=63), dict(d=None), dict(d=A + 2), dict(ldd=63), dict(d=2 * A, ldd=72), dict(d=A, ldd=72)):
        assert b(**bad) == X.XS_EINVAL, bad
    assert b(T=0) == b(T=0, st=None, n=1) == b(T=0, l=None, add=None, d=None) == X.XS_OK
    assert f(T=2 ** 31 - 10) == X.XS_EUNSUPPORTED
    n = C.c_int64()
    q = lambda T, E, s, p=C.byref(n): X.xs_balance_loss_workspace_bytes(T, E, s, p)
    assert q(-1, 8, 1) == q(1, 0, 1) == q(1, 1025, 1) == q(1, 8, 0) == q(1, 8, 65537) == q(1, 8, 1, None) == X.XS_EINVAL
    assert q(0, 8, 1) == X.XS_OK and n.value > 0


def _attn(**kw):
    X = xs()
    a = X.xs_attn_packed(n_seq=2, heads=8, kv_heads=2, head_dim=128, Tq=64, Tk=128, causal=1, max_k=0, scale=0.0, reserved=0, q_start=A, k_start=A,
                         k_rows=None, q=A, k=A, v=A, o=A, lse=A, q_row=1024, q_head=128, k_row=256, k_head=128, v_row=256, v_head=128, o_row=1024,
                         o_head=128)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


BAD = [dict(n_seq=0), dict(n_seq=65537), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0), dict(Tq=-1), dict(Tk=-1), dict(max_k=-1),
       dict(max_k=129), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(reserved=1), dict(q_start=None), dict(k_start=None), dict(q=None),
       dict(k=None), dict(v=None), dict(o=None), dict(q=A + 8), dict(k=A + 2), dict(v=A + 8), dict(o=A + 4), dict(q_row=120), dict(q_row=1028), dict(q_head=64),
       dict(k_row=100), dict(k_head=0), dict(k_head=132), dict(v_row=0), dict(v_head=120), dict(o_row=-1024), dict(o_head=1 << 40)]
UNSUPPORTED = [dict(head_dim=96, q_head=128), dict(head_dim=32), dict(q_row=(1 << 23) + 8), dict(k_row=1 << 24), dict(Tq=1 << 28), dict(Tk=(1 << 30) + 1),
               dict(heads=1 << 17, kv_heads=1 << 17), dict(heads=1 << 16, kv_heads=1 << 16, Tq=1 << 18), dict(heads=1 << 16, kv_heads=1 << 16, Tk=1 << 22)]


@pytest.mark.parametrize("kw,code", [(b, "XS_EINVAL") for b in BAD] + [(u, "XS_EUNSUPPORTED") for u in UNSUPPORTED])
def test_attention(kw, code):
    X = xs()
    a, n = _attn(**kw), C.c_int64()
    g = X.xs_attn_grads(A, A, A, A, 1024, 128, 1024, 128, 256, 128, 256, 128)
    code = getattr(X, code)
    assert X.xs_attention_packed_workspace_bytes(a, C.byref(n)) == code
    assert X.xs_attention_packed(a, A, 1 << 40, None, None) == code
    assert X.xs_attention_packed_backward_workspace_bytes(a, C.byref(n)) == code
    assert X.xs_attention_packed_backward(a, g, A, 1 << 40, None, None) == code


def test_attention_gradients():
    X = xs()
    grads = lambda **kw: X.xs_attn_grads(**{**dict(d_o=A, dq=A, dk=A, dv=A, do_row=1024, do_head=128, dq_row=1024, dq_head=128, dk_row=256, dk_head=128,
                                                   dv_row=256, dv_head=128), **kw})
    f = lambda a=_attn(), g=grads(), ws=A, nb=1 << 30: X.xs_attention_packed_backward(a, g, ws, nb, None, None)
    for bad in (dict(d_o=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(d_o=A + 8), dict(do_row=100), dict(do_head=0), dict(dq_row=1028),
                dict(dk_head=64), dict(dv_row=128 - 8), dict(dv=A + 8)):
        assert f(g=grads(**bad)) == X.XS_EINVAL, bad
    assert f(g=None) == X.XS_EINVAL
    assert f(a=None) == X.XS_EINVAL
    assert f(a=_attn(lse=None)) == X.XS_EINVAL
    assert f(a=_attn(k_rows=A)) == X.XS_EUNSUPPORTED
    assert f(g=grads(dk_row=1 << 24)) == X.XS_EUNSUPPORTED
    for bad in (dict(ws=None), dict(ws=A + 8), dict(nb=8 * 64 * 4 - 1)):
        assert f(**bad) == X.XS_EWORKSPACE, bad
    n = C.c_int64()
    assert X.xs_attention_packed_backward_workspace_bytes(_attn(), C.byref(n)) == X.XS_OK and n.value >= 8 * 64 * 4
    assert X.xs_attention_packed_workspace_bytes(_attn(), None) == X.XS_EINVAL
    # a single head has no head stride
    assert X.xs_attention_packed_workspace_bytes(_attn(heads=1, kv_heads=1, q_head=0, k_head=0, v_head=0, o_head=0), C.byref(n)) == X.XS_OK
    assert X.xs_attention_packed(_attn(Tq=0), None, 0, None, None) == X.XS_OK
    assert X.xs_attention_packed(_attn(Tq=0, q=None, o=None, lse=None), None, 0, None, None) == X.XS_OK


def test_binding_refuses_other_layouts():
    import torch
    X = xs()
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    i32 = lambda n: t(n, dtype=torch.int32)
    ok = dict(q=t(4, 2, 128), k=t(6, 1, 128), v=t(6, 1, 128), o=t(4, 2, 128), q_start=i32(3), k_start=i32(3))
    a = X.attn_packed(**ok)
    assert (a.n_seq, a.heads, a.kv_heads, a.Tq, a.Tk) == (2, 2, 1, 4, 6)
    assert X.attn_packed(**{**ok, "k_start": i32(2)}, k_rows=i32(2)).n_seq == 2
    for bad in (dict(q=t(4, 128, 2).transpose(1, 2)), dict(q=t(4, 2, 128, dtype=torch.float16)), dict(o=t(4, 2, 64)), dict(o=t(3, 2, 128)), dict(v=t(5, 1, 128)),
                dict(v=t(6, 2, 128)), dict(k=t(6, 1, 64), v=t(6, 1, 64)), dict(q=t(4, 256)), dict(q_start=t(3, dtype=torch.int64)), dict(k_start=i32(2)),
                dict(k_rows=i32(1)), dict(k_rows=i32(2), k_start=i32(1)), dict(q_start=i32(6)[::2]), dict(lse=t(4, 2, dtype=torch.float32)), dict(lse=t(2, 4)),
                dict(v=torch.zeros((6, 1, 128), dtype=torch.bfloat16, device="meta"))):
        with pytest.raises(ValueError):
            X.attn_packed(**{**ok, **bad})
    q, k = ok["q"], ok["k"]
    X.attn_packed_grads(q, q, k, k)
    for bad in ((q[0], q, k, k), (q, q[:3], k, k), (q, q, k, k[:5]), (q, q, k[..., :64], k[..., :64]), (q.float(), q, k, k)):
        with pytest.raises(ValueError):
            X.attn_packed_grads(*bad)


def test_gradients_of_another_shape_than_the_forward_call_s():
    # the C call has pointers and strides alone: its binding compares the tensors' shapes with the descriptor before
    import torch
    X = xs()
    t = lambda *shape, **kw: torch.zeros(shape, dtype=torch.bfloat16, **kw)
    i32 = torch.zeros(3, dtype=torch.int32)
    a = X.attn_packed(t(40, 4, 128), t(60, 2, 128), t(60, 2, 128), t(40, 4, 128), i32, i32, lse=torch.zeros(4, 40))
    q, k, meta = (40, 4, 128), (60, 2, 128), dict(device="meta")
    call = lambda g, a=a: X.xs_attention_packed_backward(a, g, None, 0, None, None)
    grads = lambda q, k, **kw: X.attn_packed_grads(t(*q, **kw), t(*q, **kw), t(*k, **kw), t(*k, **kw))
    assert call(grads(q, k)) == X.XS_EWORKSPACE
    assert call(C.byref(grads(q, k)), C.byref(a)) == X.XS_EWORKSPACE
    for bad in (((39, 4, 128), k), ((40, 3, 128), k), (q, (59, 2, 128)), (q, (60, 1, 128)), ((40, 4, 64), (60, 2, 64)), ((41, 4, 128), k)):
        g = grads(*bad)
        for args in ((g, a), (C.byref(g), a), (g, C.byref(a))):
            with pytest.raises(ValueError):
                call(*args)
    with pytest.raises(ValueError):
        call(grads(q, k, **meta))
    # descriptors that were filled in by hand have no tensors to compare
    assert X.xs_attention_packed_backward(_attn(), X.xs_attn_grads(A, A, A, A, 1024, 128, 1024, 128, 256, 128, 256, 128), None, 0, None, None) == X.XS_EWORKSPACE
    assert X.xs_attention_packed_backward(None, None, None, 0, None, None) == X.XS_EINVAL
