"""The gates, the E4M3 products and the SwiGLU checkpoints as a program runs them together: layers routed by a
gate, fused and phase by phase, and one rank's training step of an expert layer in E4M3, forward and
backward, every stage against the fp64 oracle of that stage on the stage's own inputs and the whole
against the layer in fp64 without any rounding."""
import ctypes as C

import numpy as np
import pytest
import torch

import synth
from gpu_helpers import assert_close, bits_f64, dev_bits, host_bits, require_gpu, xs
from oracle import ep as oep
from oracle import fp8, gate

pytestmark = pytest.mark.gpu

B = fp8.BLOCK


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _st():
    return torch.cuda.current_stream().cuda_stream


def _ref_layer(inp, l64, g, s):
    """Layer output of source `src` in fp64 for the oracle's routing by the gate."""
    idx, w = gate.route(l64[s.src], s.k, **g)
    out = np.zeros((s.T, s.H))
    x = inp["x"][s.src]
    for e in range(s.E):
        t, j = np.nonzero(idx == e)
        if len(t):
            y = bits_f64(oep.expert_ffn(x[t], inp["w1"][e], inp["w2"][e])[2])
            np.add.at(out, t, w[t, j][:, None] * y)
    return idx, w, out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,groups,renorm,scale", [("sigmoid", (4, 2, True), True, 2.5), ("softmax", (1, 1, False), False, 1.0)])
def test_layers_routed_by_a_gate(dtype, kind, groups, renorm, scale):
    X = xs()
    from paper_2607_23264_amd.layer import EPLayer, Shape, pacing
    cfg = synth.EP_TINY
    inp = synth.ep_inputs(cfg, 5)
    bias = torch.randn(cfg.E, generator=torch.Generator().manual_seed(1)) * 0.1
    gt = X.gate(cfg.E, cfg.k, score=X.XS_SCORE_SIGMOID if kind == "sigmoid" else X.XS_SCORE_SOFTMAX, n_group=groups[0],
                topk_group=groups[1], group_score=X.XS_GROUP_TOP2 if groups[2] else X.XS_GROUP_MAX, renormalize=renorm,
                scale=scale, bias=bias.cuda(), logits_type=X.XS_TYPE_BF16 if dtype == "bf16" else X.XS_TYPE_F32)
    s = Shape(cfg.n_src, cfg.T, cfg.H, cfg.E, cfg.k, cfg.I, cfg.W, 0, cfg.E)
    lay = EPLayer(s, gate=gt)
    lay.upload(inp["logits"], inp["x"], inp["w1"], inp["w2"])
    l64 = lay.logits.cpu().double().numpy()
    idx, w, want = _ref_layer(inp, l64, dict(kind=kind, n_group=groups[0], topk_group=groups[1], top2=groups[2],
                                             bias=bias.double().numpy(), renorm=renorm, scale=scale), s)
    lay.fused(pacing(X.XS_POLICY_INTERLEAVE, lead=1))
    torch.cuda.synchronize()
    assert int(lay.status.item()) == 0
    assert np.array_equal(lay.topk_idx.cpu().numpy()[0], idx)
    assert_close(host_bits(lay.out), want, "fused layer routed by a gate")
    fused = host_bits(lay.out)
    lay.out.zero_()
    lay.unfused()
    torch.cuda.synchronize()
    assert_close(host_bits(lay.out), want, "phase by phase")
    # the quantized layers take the same gate: the same routing, and the same weights bit for bit
    w_bits = lay.topk_w.cpu().numpy()
    mx_lay = EPLayer(s, gate=gt, precision=X.XS_PREC_MXFP8)
    mx_lay.upload(inp["logits"], inp["x"], inp["w1"], inp["w2"])
    mx_lay.fused()
    torch.cuda.synchronize()
    assert np.array_equal(mx_lay.topk_w.cpu().numpy(), w_bits) and np.array_equal(mx_lay.topk_idx.cpu().numpy()[0], idx)
    assert fused.shape == host_bits(mx_lay.out).shape


def test_a_gate_must_fit_its_layer():
    X = xs()
    from paper_2607_23264_amd.layer import EPLayer, Shape
    cfg = synth.EP_TINY
    s = Shape(cfg.n_src, cfg.T, cfg.H, cfg.E, cfg.k, cfg.I, cfg.W, 0, cfg.E)
    with pytest.raises(ValueError):
        EPLayer(s, gate=X.gate(cfg.E * 2, cfg.k))
    lay = EPLayer(s)
    args = (None, None, lay.workspace.data_ptr(), lay.workspace.numel(), lay.status.data_ptr(), _st())
    L = C.byref(lay.L)
    assert X.xs_fused_ep_layer_gated(L, X.gate(cfg.E, cfg.k + 1), *args) == X.XS_EINVAL
    assert X.xs_fused_ep_layer_gated(L, None, *args) == X.XS_EINVAL
    lay.topk_idx.fill_(-5)
    bad = X.gate(cfg.E, cfg.k, score=9)
    assert X.xs_fused_ep_layer_gated(L, bad, *args) == X.XS_EINVAL
    torch.cuda.synchronize()
    assert (lay.topk_idx == -5).all()                             # nothing was launched


def _codes(rows, cols, down=1):
    K = -(-cols // B) * B
    return (torch.zeros((rows, K), dtype=torch.uint8, device="cuda"),
            torch.zeros((-(-rows // down), -(-(K // B) // 4) * 4), device="cuda"))


def _args(c):
    return c[0].data_ptr(), c[0].stride(0), c[1].data_ptr(), c[1].stride(0)


NONE = (None, 0, None, 0)


def _host(c, down=1):
    """fp64 values of device codes and scales."""
    return fp8.values(c[0].cpu().numpy(), c[1].cpu().numpy(), down)


def _within(got, want, bound, half, what):
    err = np.abs(got - want) - half * (np.abs(want) + bound) - bound
    assert np.isfinite(got).all() and err.max() <= 0, f"{what}: {np.abs(got - want).max():.3e}"


def _rel(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def test_a_training_step_of_an_expert_layer():
    X = xs()
    from paper_2607_23264_amd.layer import EPLayer, Shape
    T, H, E, k, I = 200, 512, 8, 2, 256
    cap = T * k
    x = synth.normal_bf16(3, 0, (T, H))
    w1, w2 = synth.normal_bf16(3, 1, (E, 2 * I, H), std=0.05), synth.normal_bf16(3, 2, (E, H, I), std=0.05)
    logits = torch.randn((T, E), generator=torch.Generator().manual_seed(4))
    d_out = synth.normal_bf16(3, 5, (T, H))
    gt = X.gate(E, k, score=X.XS_SCORE_SIGMOID, n_group=4, topk_group=3, group_score=X.XS_GROUP_MAX, renormalize=1, scale=1.5)
    # the layer's buffers and its dispatch, combine and layout calls; this rank has every expert, one window
    lay = EPLayer(Shape(1, T, H, E, k, I, 1, 0, E), gate=gt)
    lay.logits[0].copy_(logits)
    dx, dd = dev_bits(x), dev_bits(d_out)

    # weights, once: 128 x 128 blocks, and transposed for the inputs' gradients
    def weights(w):
        n, r, c = w.shape
        codes, scales = torch.zeros((n, r, c), dtype=torch.uint8, device="cuda"), torch.zeros((n, -(-r // B), -(-(c // B) // 4) * 4), device="cuda")
        codes_t, scales_t = torch.zeros((n, c, r), dtype=torch.uint8, device="cuda"), torch.zeros((n, -(-c // B), -(-(r // B) // 4) * 4), device="cuda")
        for e in range(n):
            b = dev_bits(w[e])
            X.check(X.xs_quantize_fp8_tile(b.data_ptr(), r, c, c, codes[e].data_ptr(), c, scales[e].data_ptr(), scales.shape[2],
                                           codes_t[e].data_ptr(), r, scales_t[e].data_ptr(), scales_t.shape[2], _st()))
        torch.cuda.synchronize()
        return (codes, scales), (codes_t, scales_t)

    (c1, s1), (c1t, s1t) = weights(w1)
    (c2, s2), (c2t, s2t) = weights(w2)
    W1 = [fp8.values(c1[e].cpu().numpy(), s1[e].cpu().numpy(), B) for e in range(E)]
    W2 = [fp8.values(c2[e].cpu().numpy(), s2[e].cpu().numpy(), B) for e in range(E)]

    # ---- forward: route, lay out, quantize the tokens into rows of codes then scales, dispatch those
    lay.route()
    lay.layout()
    pitch = H + 4 * (H // B)
    staged = torch.zeros((T, pitch), dtype=torch.uint8, device="cuda")
    X.check(X.xs_quantize_fp8(dx.data_ptr(), T, H, H, staged.data_ptr(), pitch, staged.data_ptr() + H, pitch // 4, *NONE, _st()))
    window = torch.full((cap, pitch), 0x7F, dtype=torch.uint8, device="cuda")
    wins = X.windows([X.window(window)])
    X.check(X.xs_dispatch_rows(staged.data_ptr(), pitch, pitch, T, lay.topk_idx.data_ptr(), lay.slot_row.data_ptr(), k, E, wins, 1,
                               lay.status.data_ptr(), _st()))
    offs, counts = lay.expert_offsets, lay.expert_counts[0]

    def grouped(a, lda, a_s, lds, w, s, N, K, out, epi=X.XS_EPI_STORE):
        X.check(X.xs_grouped_gemm_fp8(a, lda, a_s, lds, cap, offs.data_ptr(), counts.data_ptr(), E, w.data_ptr(), s.data_ptr(), s.shape[2],
                                      N, K, out.data_ptr(), out.shape[1], epi, lay.status.data_ptr(), _st()))

    bf = lambda r, c: torch.zeros((r, c), dtype=torch.int16, device="cuda")
    gu, h, ck, y = bf(cap, 2 * I), _codes(cap, I), _codes(cap, 2 * I), lay.y_ws
    grouped(window.data_ptr(), pitch, window.data_ptr() + H, pitch // 4, c1, s1, 2 * I, H, gu)
    X.check(X.xs_swiglu_fp8(gu.data_ptr(), 2 * I, cap, I, *_args(h), *_args(ck), _st()))
    grouped(*_args(h), c2, s2, H, I, y)
    lay.combine_send()
    lay.combine_reduce()
    torch.cuda.synchronize()
    assert int(lay.status.item()) == 0
    idx, w = gate.route(logits.double().numpy(), k, "sigmoid", 4, 3, False, None, True, 1.5)
    assert np.array_equal(lay.topk_idx.cpu().numpy()[0], idx)
    o, n = offs.cpu().numpy(), counts.cpu().numpy()
    assert n.sum() == cap and np.array_equal(n, np.bincount(idx.ravel(), minlength=E))
    slots = lay.row_src.cpu().numpy()[0] & ((1 << 24) - 1)
    token = slots // k
    xv = fp8.values(*fp8.quantize(bits_f64(x)))
    rows = window.cpu().numpy()
    assert np.array_equal(rows[:, :H], staged.cpu().numpy()[token][:, :H])
    A = xv[token]
    guv = bits_f64(host_bits(gu))
    _close_quantized(h, fp8.swiglu(guv), "h")
    assert np.array_equal(ck[0].cpu().numpy(), fp8.quantize(guv)[0])
    hv, ckv, yv = _host(h), _host(ck), bits_f64(host_bits(y[:cap]))
    for e in range(E):
        r = slice(o[e], o[e] + n[e])
        _within(guv[r], A[r] @ W1[e].T, fp8.product_bound(A[r], W1[e], False), 2.0 ** -8, f"gate and up of expert {e}")
        _within(yv[r], hv[r] @ W2[e].T, fp8.product_bound(hv[r], W2[e], False), 2.0 ** -8, f"y of expert {e}")
    cw = lay.topk_w.cpu().double().numpy()[0]
    y_slot = np.zeros((T * k, H))
    y_slot[slots] = yv
    assert_close(host_bits(lay.out), (cw[:, :, None] * y_slot.reshape(T, k, H)).sum(1), "combined output")

    # ---- backward: the combine's gradients (plain), then the library's calls
    dv = bits_f64(d_out)
    dy = dev_bits(synth.to_bf16_bits((cw.reshape(-1)[slots][:, None] * dv[token]).astype(np.float32)))
    d_w = torch.from_numpy((y_slot.reshape(T, k, H) * dv[:, None, :]).sum(2).astype(np.float32)).cuda()
    dyq, dh, dgu, h_again, dguq, dxr = _codes(cap, H), bf(cap, I), bf(cap, 2 * I), bf(cap, I), _codes(cap, 2 * I), bf(cap, H)
    X.check(X.xs_quantize_fp8(dy.data_ptr(), cap, H, H, *_args(dyq), *NONE, _st()))
    grouped(*_args(dyq), c2t, s2t, I, H, dh)
    X.check(X.xs_swiglu_fp8_backward(*_args(ck), dh.data_ptr(), I, cap, I, dgu.data_ptr(), 2 * I, h_again.data_ptr(), I, _st()))
    X.check(X.xs_quantize_fp8(dgu.data_ptr(), cap, 2 * I, 2 * I, *_args(dguq), *NONE, _st()))
    grouped(*_args(dguq), c1t, s1t, H, 2 * I, dxr)
    d_logits = torch.zeros((T, E), device="cuda")
    X.check(X.xs_route_gate_backward(gt, lay.logits.data_ptr(), E, T, lay.topk_idx.data_ptr(), d_w.data_ptr(), d_logits.data_ptr(), E,
                                     lay.status.data_ptr(), _st()))
    # a weight's gradient sums over its expert's rows: both operands quantized along them, transposed
    x_rows = dev_bits(np.ascontiguousarray(x[token]))
    dW1, dW2 = torch.zeros((E, 2 * I, H), device="cuda"), torch.zeros((E, H, I), device="cuda")
    pairs = []
    for e in np.flatnonzero(n):
        for a, b, N, M, out in ((dgu, x_rows, H, 2 * I, dW1[e]), (dy, h_again, I, H, dW2[e])):
            at, bt = _codes(M, int(n[e])), _codes(N, int(n[e]))
            X.check(X.xs_quantize_fp8(a.data_ptr() + 2 * M * int(o[e]), int(n[e]), M, M, *NONE, *_args(at), _st()))
            X.check(X.xs_quantize_fp8(b.data_ptr() + 2 * N * int(o[e]), int(n[e]), N, N, *NONE, *_args(bt), _st()))
            X.check(X.xs_gemm_fp8(*_args(at), *_args(bt), X.XS_BLOCK_ROW, out.data_ptr(), N, X.XS_TYPE_F32, M, N, at[0].shape[1], _st()))
            pairs.append((at, bt, out))
    torch.cuda.synchronize()
    assert int(lay.status.item()) == 0
    dhv, dguv = bits_f64(host_bits(dh)), bits_f64(host_bits(dgu))
    want, hw, mag = fp8.swiglu_backward(ckv, dhv)
    loose = 2.0 ** -20 * (1 + np.abs(ckv[:, :I]))
    assert np.all(np.abs(dguv - want) <= 2.0 ** -8 * np.abs(want) + np.concatenate([loose, loose], 1) * mag + 2.0 ** -126)
    assert np.all(np.abs(bits_f64(host_bits(h_again)) - hw) <= (2.0 ** -8 + loose) * np.abs(hw) + 2.0 ** -126)
    dyv, dgq, dxv = _host(dyq), _host(dguq), bits_f64(host_bits(dxr))
    for e in range(E):
        r = slice(o[e], o[e] + n[e])
        _within(dhv[r], dyv[r] @ W2[e], fp8.product_bound(dyv[r], W2[e].T, False), 2.0 ** -8, f"dh of expert {e}")
        _within(dxv[r], dgq[r] @ W1[e], fp8.product_bound(dgq[r], W1[e].T, False), 2.0 ** -8, f"dx of expert {e}")
    for at, bt, out in pairs:
        P, Q = _host(at), _host(bt)
        _within(out.cpu().double().numpy(), P @ Q.T, fp8.product_bound(P, Q, True), 2.0 ** -24, "a weight's gradient")
    grad, gm = gate.backward(logits.double().numpy(), idx, d_w.cpu().numpy(), "sigmoid", True, 1.5)
    assert np.all(np.abs(d_logits.cpu().double().numpy() - grad) <= 2.0 ** -15 * gm)

    # ---- the whole against fp64 without rounding. E4M3 rounds a value by at most 2^-4, 3.6 % r.m.s. at worst.
    # y passes four such roundings (x, W1, h, W2), the first two twice through gate and up (times at most
    # 1.1 sqrt 2): below sqrt(2 (1.56^2 + 1)) 3.6 % = 9.5 %. dx and dW1 add dy, W2^T, the checkpoint's gate and up (silu''s
    # slope at most 0.5 beside silu' of 1.1: 1.5 each), dgu, W1 or x: sqrt(2 + 2 1.5^2 + 2) 3.6 % = 10.5 % on h's 9.5 %.
    f = lambda b: bits_f64(b)
    tx, ty, tdx = f(x), np.zeros((T, H)), np.zeros((T, H))
    tdw1, tdw2 = np.zeros((E, 2 * I, H)), np.zeros((E, H, I))
    tw = np.zeros((T, k))
    for e in range(E):
        t, j = np.nonzero(idx == e)
        g_, h_ = tx[t] @ f(w1[e]).T, None
        h_ = fp8.swiglu(g_)
        ye = h_ @ f(w2[e]).T
        np.add.at(ty, t, w[t, j][:, None] * ye)
        tw[t, j] = (ye * dv[t]).sum(1)
        dye = w[t, j][:, None] * dv[t]
        tdw2[e] = dye.T @ h_
        dg, _, _ = fp8.swiglu_backward(g_, dye @ f(w2[e]))
        tdw1[e] = dg.T @ tx[t]
        np.add.at(tdx, t, dg @ f(w1[e]))
    assert _rel(bits_f64(host_bits(lay.out)), ty) < 0.095
    dx_tok = np.zeros((T, H))
    np.add.at(dx_tok, token, dxv)
    assert _rel(dx_tok, tdx) < 0.15
    assert _rel(dW1.cpu().double().numpy(), tdw1) < 0.15 and _rel(dW2.cpu().double().numpy(), tdw2) < 0.15


def _close_quantized(c, want, what):
    """Codes and scales of values that fp32 computes within 2^-20 (1 + |gate|) <= 2^-16 here."""
    s64 = np.maximum(np.abs(want).reshape(want.shape[0], -1, B).max(-1), 2.0 ** -60) / 448
    scales = c[1].cpu().double().numpy()[:, :s64.shape[1]]
    assert np.all(np.abs(scales - s64) <= 2.0 ** -16 * s64), what
    step = np.maximum(2.0 ** -4 * np.abs(want), np.repeat(s64, B, 1) * 2.0 ** -10)
    assert np.all(np.abs(_host(c) - want) <= step * (1 + 2.0 ** -15) + 2.0 ** -15 * np.abs(want)), what


def test_a_layer_of_bf16_logits_is_refused_by_calls_without_its_gate():
    X = xs()
    from paper_2607_23264_amd.layer import EPLayer, Shape
    cfg = synth.EP_TINY
    s = Shape(cfg.n_src, cfg.T, cfg.H, cfg.E, cfg.k, cfg.I, cfg.W, 0, cfg.E)
    lay = EPLayer(s, gate=X.gate(cfg.E, cfg.k, logits_type=X.XS_TYPE_BF16))
    L, st = C.byref(lay.L), (lay.status.data_ptr(), _st())
    lay.topk_idx.fill_(-5)
    assert X.xs_fused_ep_layer(L, None, None, lay.workspace.data_ptr(), lay.workspace.numel(), *st) == X.XS_EINVAL
    assert X.xs_fused_ep_layer_noalloc(L, None, None, *st) == X.XS_EINVAL
    assert X.xs_fused_ep_layer_gated(L, X.gate(cfg.E, cfg.k), None, None, lay.workspace.data_ptr(), lay.workspace.numel(), *st) == X.XS_EINVAL
    torch.cuda.synchronize()
    assert (lay.topk_idx == -5).all()                             # nothing was launched
    assert EPLayer(s).L.reserved == EPLayer(s, gate=X.gate(cfg.E, cfg.k)).L.reserved == 0
