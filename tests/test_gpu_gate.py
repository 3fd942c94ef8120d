"""GPU parity of the routing gates and their gradient against the fp64 oracle: the selection exactly, the
weights and gradients within their fp32 roundings.

Weights: a score is an exponential of relative error below 2^-21 (argument rounding, weighted by
d e^-d, and the exponential's own), a sum of at most 1024 such terms in fp32 (a lane adds at most 64,
then six levels) and a division: below 2^-17 in all; renormalizing divides two of them: 2^-16.
Gradients: ds multiplies two or three such scores; bounded by 2^-15 of the terms' magnitudes."""
import numpy as np
import pytest
import torch

from gpu_helpers import require_gpu, xs
from oracle import gate

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _logits(T, E, dtype, seed, ld=None):
    """Logits on the GPU (rows ld apart) and as fp64."""
    g = torch.Generator().manual_seed(seed)
    l = (torch.randn((T, E), generator=g) * 1.5).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return l, l.double().numpy()


def _device(l, ld):
    full = torch.full((l.shape[0], ld), float("nan"), dtype=l.dtype, device="cuda")
    full[:, :l.shape[1]] = l.cuda()
    return full


def _gate(E, k, kind, n_group=1, topk_group=1, top2=False, renorm=False, scale=1.0, bias=None, dtype="f32"):
    X = xs()
    return X.gate(E, k, score=X.XS_SCORE_SIGMOID if kind == "sigmoid" else X.XS_SCORE_SOFTMAX, n_group=n_group,
                  topk_group=topk_group, group_score=X.XS_GROUP_TOP2 if top2 else X.XS_GROUP_MAX, renormalize=renorm,
                  scale=scale, bias=bias, logits_type=X.XS_TYPE_BF16 if dtype == "bf16" else X.XS_TYPE_F32)


def _route(g, dev, T):
    X = xs()
    idx = torch.full((T + 1, g.k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T + 1, g.k), -7.0, device="cuda")
    X.check(X.xs_route_gate(g, dev.data_ptr(), dev.stride(0), T, idx.data_ptr(), w.data_ptr(), _stream()))
    torch.cuda.synchronize()
    assert (idx[T] == -7).all() and (w[T] == -7.0).all()          # nothing past the last token
    return idx[:T].cpu().numpy(), w[:T].cpu().double().numpy()


CASES = [  # E, k, groups, kept, top2
    (256, 8, 8, 4, True), (256, 8, 1, 1, False), (8, 2, 1, 1, False), (8, 3, 4, 2, True), (64, 6, 8, 3, False), (60, 4, 4, 2, True),
    (160, 6, 8, 3, False), (384, 8, 8, 4, True), (512, 10, 1, 1, False), (1024, 32, 16, 8, True), (1, 1, 1, 1, False),
    (17, 17, 1, 1, False), (128, 16, 16, 16, True), (64, 1, 64, 1, False), (100, 9, 1, 1, False), (256, 4, 1, 1, False),
    (32, 8, 16, 4, True), (256, 16, 2, 1, True), (72, 5, 1, 1, False), (250, 7, 1, 1, False)]


@pytest.mark.parametrize("E,k,n_group,topk_group,top2", CASES)
@pytest.mark.parametrize("kind,dtype,biased,renorm,scale", [("sigmoid", "f32", True, True, 2.5), ("sigmoid", "bf16", False, False, 1.0),
                                                            ("softmax", "f32", True, False, 16.0), ("softmax", "bf16", False, True, 1.0),
                                                            ("sigmoid", "bf16", True, False, 1.0), ("softmax", "f32", False, False, 1.0)])
def test_selection_and_weights(E, k, n_group, topk_group, top2, kind, dtype, biased, renorm, scale):
    for T, pad in ((1, 0), (37, 3)):
        l, l64 = _logits(T, E, dtype, E + k + T)
        b = torch.randn(E, generator=torch.Generator().manual_seed(5)) * 0.1 if biased else None
        g = _gate(E, k, kind, n_group, topk_group, top2, renorm, scale, b.cuda() if biased else None, dtype)
        idx, w = _route(g, _device(l, E + pad), T)
        want, ww = gate.route(l64, k, kind, n_group, topk_group, top2, b.double().numpy() if biased else None, renorm, scale)
        assert np.array_equal(idx, want)
        assert np.all(np.abs(w - ww) <= 2.0 ** -16 * ww)


@pytest.mark.parametrize("E,n_group,topk_group,top2", [(256, 8, 4, True), (256, 8, 4, False), (64, 1, 1, False), (60, 4, 2, True), (512, 8, 3, True)])
@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("biased", [False, True])
def test_ties_masks_and_scores_an_ulp_apart(E, n_group, topk_group, top2, kind, biased):
    # rows of equal logits, of few distinct ones, masked in part, to one expert and whole, scores that differ
    # by less than an fp32 unit (logits 1e-7 apart, and saturated sigmoids), huge and tiny logits
    k = 6
    g = np.random.default_rng(E)
    rows = [np.zeros(E), g.integers(0, 3, E) / 2.0, np.full(E, -np.inf), np.where(np.arange(E) == 13, 0.5, -np.inf)]
    for frac in (0.5, 0.9, 0.97):
        rows.append(np.where(g.random(E) < frac, -np.inf, g.standard_normal(E)))
    rows.append(1.0 + 1.2e-7 * g.integers(0, 40, E))
    rows.append(14.0 + g.random(E))
    rows.append(g.standard_normal(E) * 30)
    rows.append(-90.0 - g.random(E) * 10)
    half = np.where(np.arange(E) < E // 2, -np.inf, 1.0)           # whole groups masked
    rows += [half, half[::-1]]
    l = torch.from_numpy(np.stack(rows)).float()
    if kind == "softmax":
        l = l[[i for i in range(len(l)) if i != 2]]
    b = torch.zeros(E)
    if biased:
        b[::3] = 0.25
    gt = _gate(E, k, kind, n_group, topk_group, top2, True, 2.0, b.cuda() if biased else None)
    idx, w = _route(gt, _device(l, E), len(l))
    want, ww = gate.route(l.double().numpy(), k, kind, n_group, topk_group, top2, b.double().numpy() if biased else None, True, 2.0)
    assert np.array_equal(idx, want)
    # weights near fp32's smallest normal lose bits: below 2^-120 of the scale they count as 0
    assert np.all(np.abs(w - ww) <= 2.0 ** -16 * ww + 2.0 ** -120)


def test_rows_masked_whole_and_nan_stay_in_range():
    E, k = 256, 8
    l = torch.zeros((4, E))
    l[0] = -float("inf")
    l[1, ::2] = float("nan")
    l[2] = float("nan")
    l[3, 7] = float("inf")
    for kind in ("sigmoid", "softmax"):
        for groups in ((1, 1, False), (8, 4, True), (8, 2, False)):
            for bias in (None, torch.full((E,), float("nan"), device="cuda"), torch.full((E,), -float("inf"), device="cuda")):
                idx, w = _route(_gate(E, k, kind, *groups, bias=bias), _device(l, E), 4)
                assert idx.min() >= 0 and idx.max() < E
                assert all(len(set(r)) == k for r in idx)
                assert idx[0].tolist() == list(range(8)) and not w[0].any()


def test_every_token_of_a_long_batch():
    # bf16 logits tie often; far more tokens than the chip holds waves
    T, E, k = 20011, 256, 8
    l, l64 = _logits(T, E, "bf16", 1)
    b = torch.randn(E, generator=torch.Generator().manual_seed(2)) * 0.02
    idx, w = _route(_gate(E, k, "sigmoid", 8, 4, True, True, 2.5, b.cuda(), "bf16"), _device(l, E), T)
    key = gate.scores(l64, "sigmoid") + b.double().numpy()
    grp = np.sort(key.reshape(T, 8, 32), -1)[..., -2:].sum(-1)
    kept = np.zeros((T, 8), bool)
    np.put_along_axis(kept, np.argsort(-grp, 1, kind="stable")[:, :4], True, 1)
    want = np.argsort(-np.where(np.repeat(kept, 32, 1), key, -np.inf), 1, kind="stable")[:, :k]
    assert np.array_equal(idx, want)
    ww = gate.weights(l64, want, "sigmoid", True, 2.5)
    assert np.all(np.abs(w - ww) <= 2.0 ** -16 * ww)


def _backward(g, dev, T, idx, d_w, out_ld=None, in_place=False):
    X = xs()
    E = g.E
    out = dev if in_place else torch.full((T + 1, out_ld or E), 7.0, dtype=dev.dtype, device="cuda")
    di, dd = torch.from_numpy(np.ascontiguousarray(idx, dtype=np.int32)).cuda(), torch.from_numpy(np.asarray(d_w, dtype=np.float32)).cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    X.check(X.xs_route_gate_backward(g, dev.data_ptr(), dev.stride(0), T, di.data_ptr(), dd.data_ptr(), out.data_ptr(), out.stride(0),
                                     st.data_ptr(), _stream()))
    torch.cuda.synchronize()
    if not in_place:
        assert (out[T] == 7.0).all() and (out[:T, E:] == 7.0).all()
    return out[:T, :E].cpu().double().numpy(), int(st.item())


@pytest.mark.parametrize("E,k", [(256, 8), (8, 2), (64, 6), (60, 4), (160, 6), (512, 10), (1024, 32), (1, 1), (17, 17), (250, 16), (130, 20)])
@pytest.mark.parametrize("kind,dtype,renorm,scale", [("sigmoid", "f32", True, 2.5), ("sigmoid", "bf16", False, 1.0),
                                                     ("softmax", "f32", False, 2.5), ("softmax", "bf16", True, 1.0),
                                                     ("softmax", "bf16", False, 1.0)])
def test_gradient(E, k, kind, dtype, renorm, scale):
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for T, pad in ((1, 0), (37, 4), (21, 1)):
        l, l64 = _logits(T, E, dtype, E * 3 + k + T)
        l64 = l64.copy()
        if T > 1 and E > 8:
            l[3, ::2] = -float("inf")
            l[4] = -float("inf")
            l64 = l.double().numpy()
        g = _gate(E, k, kind, renorm=renorm, scale=scale, dtype=dtype)
        idx = gate.select(l64, k, kind)
        d_w = np.random.default_rng(T).standard_normal((T, k)).astype(np.float32)
        got, status = _backward(g, _device(l, E + pad), T, idx, d_w, E + 2 * pad)
        want, mag = gate.backward(l64, idx, d_w, kind, renorm, scale)
        assert status == 0
        assert np.all(np.abs(got - want) <= half * np.abs(want) + 2.0 ** -15 * mag)


def test_gradient_of_repeated_and_bad_indices_and_in_place():
    T, E, k = 9, 64, 4
    l, l64 = _logits(T, E, "f32", 4)
    idx = gate.select(l64, k, "softmax")
    idx[2] = [5, 5, 9, 5]
    d_w = np.random.default_rng(0).standard_normal((T, k)).astype(np.float32)
    for kind in ("sigmoid", "softmax"):
        for renorm in (False, True):
            g = _gate(E, k, kind, renorm=renorm)
            want, mag = gate.backward(l64, idx, d_w, kind, renorm)
            got, status = _backward(g, _device(l, E), T, idx, d_w)
            assert status == 0 and np.all(np.abs(got - want) <= 2.0 ** -15 * mag)
            again, _ = _backward(g, _device(l, E), T, idx, d_w, in_place=True)
            assert np.array_equal(again, got)
            bad = idx.copy()
            bad[5, 1], bad[6, 0] = E, -3
            want, mag = gate.backward(l64, bad, d_w, kind, renorm)
            got, status = _backward(g, _device(l, E), T, bad, d_w)
            assert status == xs().XS_EBADINPUT and np.all(np.abs(got - want) <= 2.0 ** -15 * mag)


def test_gradient_is_the_differences_of_the_forward_call():
    # central differences of the library's own weights: w is off by 2^-16 w at each end, the step's
    # third-order term is below h^2 / 6 times 6
    T, E, k, h = 5, 64, 4, 2.0 ** -5
    l, _ = _logits(T, E, "f32", 11)
    for kind in ("sigmoid", "softmax"):
        for renorm in (False, True):
            g = _gate(E, k, kind, renorm=renorm)
            idx, _ = _route(g, _device(l, E), T)
            d_w = np.random.default_rng(1).standard_normal((T, k)).astype(np.float32)
            got, _ = _backward(g, _device(l, E), T, idx, d_w)
            for t in range(T):
                for j, e in enumerate(idx[t]):
                    step = torch.zeros((T, E))
                    step[t, e] = h
                    w = []
                    for s in (step, -step):
                        i2, ww = _route(g, _device(l + s, E), T)
                        order = [list(i2[t]).index(x) if x in i2[t] else None for x in idx[t]]
                        w.append(None if None in order else ww[t][order])
                    if w[0] is None or w[1] is None:
                        continue                       # the step changed the selection
                    want = ((w[0] - w[1]) * d_w[t]).sum() / (2 * h)
                    assert abs(got[t, e] - want) <= np.abs(d_w[t]).sum() * (2.0 ** -16 / h + h * h)


def test_gates_in_a_graph_and_on_another_stream():
    X = xs()
    T, E, k = 300, 256, 8
    l, l64 = _logits(T, E, "f32", 8)
    g = _gate(E, k, "sigmoid", 8, 4, True, True, 2.5)
    dev = _device(l, E)
    idx, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
    d = torch.zeros((T, E), device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(s):
        X.check(X.xs_route_gate(g, dev.data_ptr(), E, T, idx.data_ptr(), w.data_ptr(), s))
        X.check(X.xs_route_gate_backward(g, dev.data_ptr(), E, T, idx.data_ptr(), w.data_ptr(), d.data_ptr(), E, st.data_ptr(), s))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(side.cuda_stream)
    torch.cuda.synchronize()
    want = [t.clone() for t in (idx, w, d)]
    assert np.array_equal(idx.cpu().numpy(), gate.select(l64, k, "sigmoid", 8, 4, True))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream().cuda_stream)
    for seed in (8, 9, 8):
        dev.copy_(_logits(T, E, "f32", seed)[0])
        for t in (idx, w, d):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        if seed == 8:
            assert all(torch.equal(a, b) for a, b in zip((idx, w, d), want))
        else:
            assert np.array_equal(idx.cpu().numpy(), gate.select(_logits(T, E, "f32", 9)[1], k, "sigmoid", 8, 4, True))


@pytest.mark.parametrize("E,k", [(8, 1), (8, 3), (64, 8), (256, 5), (512, 16), (700, 20)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_signed_zeros_are_equal(E, k, dtype):
    """Logits of 0 and -0 tie, whichever comes first."""
    l = torch.full((4, E), -1.0)
    l[0, ::2] = 0.0
    l[0, 1::2] = -0.0
    l[1, ::2] = -0.0
    l[1, 1::2] = 0.0
    l[2, :] = -0.0
    l[2, E - 1] = 0.0
    l[3, 1] = -0.0
    l[3, E - 1] = 0.0
    l = l.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    for kind in ("softmax", "sigmoid"):
        idx, _ = _route(_gate(E, k, kind, dtype=dtype), l.cuda(), 4)
        assert np.array_equal(idx, gate.route(l.double().numpy(), k, kind)[0])


@pytest.mark.parametrize("E,k", [(16, 4), (64, 8), (256, 8), (512, 16), (640, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lowest_keys_come_before_masked_ones(E, k, dtype):
    """Finite logits just above -2^127 at the highest indices, behind masked ones."""
    l = torch.full((3, E), float("-inf"))
    low = -(2.0 ** 127) * (1 - 2.0 ** (-7 if dtype == "bf16" else -20))
    l[0, E - k - 1:] = low
    l[1, E - k // 2:] = low
    l[2, E - k // 2:] = low
    l[2, E // 2] = 3.0
    l = l.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    idx, _ = _route(_gate(E, k, "softmax", renorm=True, dtype=dtype), l.cuda(), 3)
    assert np.array_equal(idx, gate.route(l.double().numpy(), k, "softmax", renorm=True)[0])


@pytest.mark.parametrize("E,k,n_group,topk_group,top2", [(30, 4, 2, 1, True), (36, 5, 4, 2, False), (40, 6, 8, 3, True), (48, 4, 16, 5, True),
                                                         (500, 9, 4, 3, True), (502, 16, 2, 1, False), (504, 8, 8, 4, True), (12, 2, 4, 2, True),
                                                         (8, 2, 8, 3, False), (264, 7, 8, 5, True), (2, 1, 2, 1, True)])
@pytest.mark.parametrize("kind,dtype,biased", [("sigmoid", "f32", True), ("softmax", "bf16", False), ("softmax", "f32", True), ("sigmoid", "bf16", True)])
def test_groups_that_do_not_fill_their_lanes(E, k, n_group, topk_group, top2, kind, dtype, biased):
    test_selection_and_weights(E, k, n_group, topk_group, top2, kind, dtype, biased, True, 1.5)
    if E >= 14 and topk_group * (E // n_group) >= 6:               # that test's one unmasked expert, and its k
        test_ties_masks_and_scores_an_ulp_apart(E, n_group, topk_group, top2, kind, biased)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_saturated_sigmoids(dtype, renorm):
    """Scores near 1 keep their slope, about e^-l, to a relative error: logits of 8 to 30 and of -30 to -8. Two
    exponentials, two quotients and three products are below 2^-20 of a slope's terms; renormalized, the difference
    g - sum g r adds 2^-19 of them (r as the weights: three roundings of an exponential, a quotient, a sum of four)."""
    T, E, k = 24, 64, 4
    g = torch.Generator().manual_seed(7)
    l = torch.rand((T, E), generator=g) * 22 + 8
    l[T // 2:] *= -1
    l = l.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    l64 = l.double().numpy()
    idx = gate.select(l64, k, "sigmoid")
    idx[3] = [9, 9, 9, 10]
    d_w = np.random.default_rng(3).standard_normal((T, k)).astype(np.float32)
    got, status = _backward(_gate(E, k, "sigmoid", renorm=renorm, scale=2.5, dtype=dtype), _device(l, E), T, idx, d_w)
    assert status == 0
    want, mag = gate.backward(l64, idx, d_w, "sigmoid", renorm, 2.5)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert np.all(np.abs(got - want) <= half * np.abs(want) + 2.0 ** -18 * mag)


@pytest.mark.parametrize("E,n_group", [(64, 4), (256, 8), (60, 4), (96, 6), (640, 8)])
@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
def test_groups_without_a_live_expert_come_last(E, n_group, kind):
    """Sums of two biased scores may pass -2^127, where no single score counts: they still come before a group whose
    experts are all masked."""
    size, k = E // n_group, 4
    l = torch.zeros((3, E))
    l[0, :size] = -float("inf")                                    # the first group is masked
    l[1, :size * (n_group - 1)] = -float("inf")                    # all but the last are
    l[2, size:] = -float("inf")
    b = torch.full((E,), -1.5e38)
    b[1::2] = -1.2e38
    for topk_group in (1, 2, n_group):
        g = _gate(E, k, kind, n_group, topk_group, True, bias=b.cuda())
        idx, _ = _route(g, _device(l, E), 3)
        want = gate.route(l.double().numpy(), k, kind, n_group, topk_group, True, b.double().numpy())[0]
        assert np.array_equal(idx, want), topk_group


@pytest.mark.parametrize("E,k,n_group,topk_group", [(16, 4, 1, 1), (256, 8, 1, 1), (256, 8, 8, 3), (60, 5, 4, 2), (700, 9, 1, 1), (96, 6, 6, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_order_of_scores_that_64_bits_cannot_tell_apart(E, k, n_group, topk_group, dtype):
    """Saturated sigmoids and softmax scores that underflow: by the logits without a bias, with a bias of zeros as
    computed in 64 bits, where they are equal and go to the lower index."""
    g = np.random.default_rng(E)
    for kind, low in (("sigmoid", 38.0), ("softmax", -900.0)):
        l = low + g.integers(0, 16, (4, E)).astype(np.float64) * (1 if kind == "sigmoid" else 4)
        if kind == "softmax":
            l[:, 3] = 0.0                                          # scores of the others: below 2^-1074
        l[1, ::3] = -float("inf")
        dev = _device(torch.from_numpy(l).to(torch.bfloat16 if dtype == "bf16" else torch.float32), E)
        l = dev.cpu().double().numpy()
        for top2, bias in ((False, None), (False, torch.zeros(E)), (True, torch.zeros(E))):
            idx, _ = _route(_gate(E, k, kind, n_group, topk_group, top2, bias=None if bias is None else bias.cuda(), dtype=dtype), dev, 4)
            want = gate.select(l, k, kind, n_group, topk_group, top2, None if bias is None else bias.numpy())
            assert np.array_equal(idx, want), (kind, top2, bias is None)


def test_renormalized_weights_are_as_exact_as_the_formula_in_fp32():
    """The mean square error against 64 bits is that of sigmoid, sum, division and scale each rounded to fp32 (a product
    with a rounded reciprocal in place of each division has 1.18 times it): within 5 %, thirty times the
    sampling error of 262,144 weights."""
    T, E, k = 32768, 256, 8
    l, l64 = _logits(T, E, "f32", 21)
    idx, w = _route(_gate(E, k, "sigmoid", renorm=True, scale=2.5), _device(l, E), T)
    s = torch.sigmoid(l.cuda()).gather(1, torch.from_numpy(idx).long().cuda())
    plain = (s / s.sum(1, keepdim=True) * 2.5).cpu().double().numpy()
    exact = gate.weights(l64, idx, "sigmoid", True, 2.5)
    rms = lambda v: np.sqrt(np.mean(((v - exact) / exact) ** 2))
    assert rms(w) <= 1.05 * rms(plain)
