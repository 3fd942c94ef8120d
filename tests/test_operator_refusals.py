"""Refused calls of the gates, the block-scaled E4M3 operators and the SwiGLU checkpoints: each argument
error returns its code before anything is launched, so these run without a GPU (the addresses are
never read)."""
import math

import pytest

A = 1 << 20           # a 16-byte aligned address


def xs():
    from paper_2607_23264_amd import xstage
    return xstage


def _gate(**kw):
    X = xs()
    args = dict(E=64, k=4, score=X.XS_SCORE_SIGMOID, n_group=4, topk_group=2, group_score=X.XS_GROUP_TOP2)
    extra = {k: kw.pop(k) for k in ("reserved",) if k in kw}
    g = X.gate(**{**args, **kw})
    for name, v in extra.items():
        setattr(g, name, v)
    return g


@pytest.mark.parametrize("kw", [dict(E=0), dict(E=1025), dict(k=0), dict(k=33), dict(E=8, n_group=1, topk_group=1, k=9),
                                dict(score=2), dict(n_group=0), dict(n_group=5), dict(n_group=65, E=65, k=1), dict(topk_group=0),
                                dict(topk_group=5), dict(group_score=2), dict(logits_type=7), dict(scale=math.inf),
                                dict(scale=math.nan), dict(reserved=1), dict(k=17, topk_group=1)])
def test_gates(kw):
    X = xs()
    g = _gate(**kw)
    assert X.xs_route_gate(g, A, 1100, 4, A, A, None) == X.XS_EINVAL
    assert X.xs_route_gate_backward(g, A, 1100, 4, A, A, A, 1100, None, None) == X.XS_EINVAL


def test_route_gate_arguments():
    X = xs()
    g = _gate()
    f = lambda gate=g, logits=A, ld=64, T=4, idx=A, w=A: X.xs_route_gate(gate, logits, ld, T, idx, w, None)
    for bad in (dict(gate=None), dict(logits=None), dict(ld=63), dict(T=-1), dict(idx=None), dict(w=None), dict(logits=A + 2)):
        assert f(**bad) == X.XS_EINVAL, bad
    assert f(T=0) == X.XS_OK
    b = lambda gate=g, logits=A, ld=64, T=4, idx=A, dw=A, d=A, ldd=64: X.xs_route_gate_backward(gate, logits, ld, T, idx, dw, d, ldd, None, None)
    for bad in (dict(gate=None), dict(idx=None), dict(dw=None), dict(d=None), dict(ldd=63), dict(d=A + 2), dict(T=-1)):
        assert b(**bad) == X.XS_EINVAL, bad
    assert b(T=0) == X.XS_OK


@pytest.mark.parametrize("name", ["xs_quantize_fp8", "xs_quantize_fp8_tile"])
def test_quantizers(name):
    X = xs()

    def f(x=A, rows=200, cols=256, ldx=256, c=A, ldc=256, s=A, lds=4, ct=A, ldt=256, st=A, ldst=4):
        return getattr(X, name)(x, rows, cols, ldx, c, ldc, s, lds, ct, ldt, st, ldst, None)

    for bad in (dict(x=None), dict(rows=-1), dict(cols=0), dict(ldx=248), dict(ldx=260), dict(x=A + 8), dict(c=None), dict(s=None),
                dict(ct=None), dict(st=None), dict(c=None, s=None, ct=None, st=None), dict(ldc=240), dict(ldc=264), dict(lds=0),
                dict(lds=6), dict(s=A + 4), dict(c=A + 8), dict(ldt=128), dict(ldst=0), dict(ldst=5), dict(ct=A + 8), dict(st=A + 4)):
        assert f(**bad) == X.XS_EINVAL, bad
    assert f(cols=252) == X.XS_EUNSUPPORTED
    assert f(rows=0) == X.XS_OK


def test_gemms():
    X = xs()

    def f(a=A, lda=512, sa=A, lsa=4, b=A, ldb=512, sb=A, lsb=4, blk=X.XS_BLOCK_TILE, c=A, ldc=256, ct=X.XS_TYPE_BF16, M=100, N=256, K=512):
        return X.xs_gemm_fp8(a, lda, sa, lsa, b, ldb, sb, lsb, blk, c, ldc, ct, M, N, K, None)

    for bad in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None), dict(M=-1), dict(N=0), dict(K=0), dict(blk=2),
                dict(ct=2), dict(lda=496), dict(lda=520), dict(lsa=3), dict(lsa=0), dict(ldb=496), dict(lsb=2), dict(ldc=248),
                dict(ldc=260), dict(a=A + 8), dict(sa=A + 4), dict(b=A + 8), dict(sb=A + 8), dict(c=A + 8)):
        assert f(**bad) == X.XS_EINVAL, bad
    for bad in (dict(K=448), dict(N=252), dict(lda=(1 << 22) + 16), dict(lsb=(1 << 20) + 4)):
        assert f(**bad) == X.XS_EUNSUPPORTED, bad
    assert f(M=0) == X.XS_OK

    def g(a=A, lda=512, sa=A, lsa=4, M=100, o=A, r=A, n=3, b=A, sb=A, lsb=4, N=256, K=512, c=A, ldc=256, epi=X.XS_EPI_STORE):
        return X.xs_grouped_gemm_fp8(a, lda, sa, lsa, M, o, r, n, b, sb, lsb, N, K, c, ldc, epi, None, None)

    for bad in (dict(a=None), dict(sa=None), dict(o=None), dict(r=None), dict(n=-1), dict(n=1025), dict(b=None), dict(sb=None),
                dict(lsb=2), dict(c=None), dict(ldc=248), dict(ldc=260), dict(epi=2), dict(M=-1), dict(c=A + 8), dict(lda=500)):
        assert g(**bad) == X.XS_EINVAL, bad
    for bad in (dict(K=500), dict(N=252), dict(N=384, epi=X.XS_EPI_SWIGLU),
                dict(N=1 << 23, ldc=1 << 22, epi=X.XS_EPI_SWIGLU)):
        assert g(**bad) == X.XS_EUNSUPPORTED, bad
    assert g(M=0) == X.XS_OK and g(n=0) == X.XS_OK


def test_swiglu_checkpoints():
    X = xs()

    def f(gu=A, ld=512, rows=10, I=256, h=A, ldh=256, hs=A, lhs=4, ck=A, ldk=512, cs=A, lcs=4):
        return X.xs_swiglu_fp8(gu, ld, rows, I, h, ldh, hs, lhs, ck, ldk, cs, lcs, None)

    for bad in (dict(gu=None), dict(ld=504), dict(ld=516), dict(rows=-1), dict(I=0), dict(h=None), dict(ldh=128), dict(hs=None),
                dict(lhs=1), dict(ck=None), dict(cs=None), dict(ldk=256), dict(lcs=3), dict(gu=A + 2), dict(cs=A + 4)):
        assert f(**bad) == X.XS_EINVAL, bad
    assert f(I=192) == X.XS_EUNSUPPORTED
    assert f(rows=0) == X.XS_OK and f(rows=0, ck=None, cs=None) == X.XS_OK

    def b(ck=A, ldk=512, cs=A, lcs=4, dh=A, ldh=256, rows=10, I=256, d=A, ldd=512, h=A, lh=256):
        return X.xs_swiglu_fp8_backward(ck, ldk, cs, lcs, dh, ldh, rows, I, d, ldd, h, lh, None)

    for bad in (dict(ck=None), dict(cs=None), dict(ldk=256), dict(lcs=2), dict(dh=None), dict(ldh=248), dict(ldh=260), dict(rows=-1),
                dict(I=0), dict(d=None), dict(ldd=504), dict(lh=248), dict(h=A + 8), dict(dh=A + 8), dict(d=A + 8)):
        assert b(**bad) == X.XS_EINVAL, bad
    assert b(I=192) == X.XS_EUNSUPPORTED
    assert b(rows=0) == X.XS_OK


def test_gradient_over_its_logits():
    """In place, rows of the gradient lie where the logits' rows do."""
    X = xs()
    g = _gate()
    assert X.xs_route_gate_backward(g, A, 64, 4, A, A, A, 72, None, None) == X.XS_EINVAL
    assert X.xs_route_gate_backward(g, A, 72, 4, A, A, A, 64, None, None) == X.XS_EINVAL


def test_sizes_past_a_grid():
    """Row and column counts whose product passes 64 bits or a grid are refused, not wrapped."""
    X = xs()
    r, i = 1 << 37, 1 << 29
    assert X.xs_swiglu_fp8_backward(A, 2 * i, A, i, A, i, r, i, A, 2 * i, None, 0, None) == X.XS_EUNSUPPORTED
    assert X.xs_swiglu_fp8(A, 2 * i, r, i, A, i, A, i, None, 0, None, 0, None) == X.XS_EUNSUPPORTED
    assert X.xs_quantize_fp8(A, r, 1 << 30, 1 << 30, A, 1 << 30, A, 1 << 23, None, 0, None, 0, None) == X.XS_EUNSUPPORTED


def test_layers_of_bf16_logits_go_to_their_gate_only():
    """A layer marked as having bf16 logits is refused by every call that would read them as fp32."""
    X = xs()
    import ctypes as C
    win = X.windows([X.xs_window()])
    L = X.xs_ep_layer(n_src=1, T=4, H=256, E=8, k=2, I=128, W=1, e_begin=0, n_experts=8, src=0, cap=8, h_rows=64)
    for f in ("logits", "x", "w1", "w2", "topk_idx", "topk_w", "expert_counts", "src_base", "expert_offsets", "dest_counts", "slot_row",
              "row_src", "h_ws", "out"):
        setattr(L, f, A)
    L.dispatch_win = L.combine_win = C.cast(win, C.POINTER(X.xs_window))
    bf16, f32 = X.gate(8, 2, logits_type=X.XS_TYPE_BF16), X.gate(8, 2)
    nothing = (None, None, None, 0, None, None)                    # no workspace: past the checks, nothing is launched
    plain = lambda: X.xs_fused_ep_layer(C.byref(L), *nothing)
    gated = lambda g: X.xs_fused_ep_layer_gated(C.byref(L), g, *nothing)
    assert plain() == gated(bf16) == gated(f32) == X.XS_EWORKSPACE
    L.reserved = X.XS_LAYER_BF16_LOGITS
    assert gated(bf16) == X.XS_EWORKSPACE
    assert plain() == gated(f32) == X.XS_EINVAL
    L.reserved = 1
    assert gated(bf16) == X.XS_EINVAL
