"""GPU parity of the balance loss and its gradient against the fp64 oracle.

A share is a quotient of exponentials: below 2^-17 (an exponential 2^-21, a sum of at most 1024 of them in fp32, a
quotient). A sequence's mean share adds them in fp32 (a lane its tokens of a workgroup, the workgroup's groups, the tiles in
turn): at most tokens + 64 additions of positive terms. The loss adds at most 1024 products. Gradient: p (c - sum c p), each
share within 2^-17, the sum within (64 + 6) 2^-24 of its terms: 2^-15 of the terms' magnitudes, one rounding to
the logits' type, and the addition of d_add one more in fp32."""
import numpy as np
import pytest
import torch

from gpu_helpers import require_gpu, xs
from oracle import balance, gate

pytestmark = pytest.mark.gpu

S = -7.0
ALPHA = 0.01


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _gate(E, k, kind, dtype):
    X = xs()
    return X.gate(E, k, score=X.XS_SCORE_SIGMOID if kind == "sigmoid" else X.XS_SCORE_SOFTMAX,
                  logits_type=X.XS_TYPE_BF16 if dtype == "bf16" else X.XS_TYPE_F32)


def _logits(T, E, dtype, seed, pad):
    g = torch.Generator().manual_seed(seed)
    l = (torch.randn((T, E), generator=g) * 2).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    l[torch.rand((T, E), generator=g) < 0.05] = -float("inf")
    if T > 3:
        l[2] = -float("inf")
    full = torch.full((T, E + pad), float("nan"), dtype=l.dtype)
    full[:, :E] = l
    return l.double().numpy(), full.cuda()


def _forward(g, dev, idx, starts, T, alpha=ALPHA):
    X = xs()
    n = len(starts) - 1
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    counts = torch.full((n + 1, g.E), -7, dtype=torch.int32, device="cuda")
    mean, loss = torch.full((n + 1, g.E), S, device="cuda"), torch.full((n + 1,), S, device="cuda")
    ws = X.workspace(X.xs_balance_loss_workspace_bytes, T, g.E, n)
    ws.fill_(255)
    X.check(X.xs_balance_loss(g, dev.data_ptr(), dev.stride(0), T, X.ptr(idx), st.data_ptr(), n, alpha, counts.data_ptr(), mean.data_ptr(),
                              loss.data_ptr(), ws.data_ptr(), ws.numel(), status.data_ptr(), _stream()))
    torch.cuda.synchronize()
    assert (counts[n] == -7).all() and (mean[n] == S).all() and loss[n] == S
    return counts[:n], mean[:n], loss[:n], st, int(status.item())


CASES = [(1, 8, 2, [0, 1]), (37, 256, 8, [0, 37]), (100, 60, 4, [0, 20, 20, 70, 95]), (65, 1, 1, [0, 65]), (300, 512, 10, [3, 4, 200, 300]),
         (40, 1024, 32, [0, 16, 33, 40]), (1000, 64, 6, [0] + list(range(0, 1001, 10))), (129, 130, 3, [0, 129]), (5, 17, 17, [0, 5]),
         (3000, 384, 8, [0, 2999, 3000])]


@pytest.mark.parametrize("T,E,k,starts", CASES)
@pytest.mark.parametrize("kind,dtype,pad", [("softmax", "f32", 0), ("sigmoid", "bf16", 0), ("softmax", "bf16", 3), ("sigmoid", "f32", 4)])
def test_loss_and_gradient(T, E, k, starts, kind, dtype, pad):
    X = xs()
    l64, dev = _logits(T, E, dtype, T + E, pad)
    g = _gate(E, k, kind, dtype)
    idx = gate.select(l64, k, kind) if T <= 300 else np.argsort(-l64, 1, kind="stable")[:, :k].astype(np.int32)
    di = torch.from_numpy(np.ascontiguousarray(idx)).cuda()
    counts, mean, loss, st, status = _forward(g, dev, di, starts, T)
    wc, wm, wl = balance.loss(l64, idx, starts, kind, ALPHA)
    longest = max(b - a for a, b in zip(starts, starts[1:]))
    rel = 2.0 ** -17 + (longest + 64) * 2.0 ** -24
    assert status == 0 and np.array_equal(counts.cpu().numpy(), wc)
    assert np.all(np.abs(mean.cpu().double().numpy() - wm) <= rel * wm + 1e-38)
    assert np.all(np.abs(loss.cpu().double().numpy() - wl) <= (rel + 2.0 ** -13) * wl)
    n = len(starts) - 1
    d_loss = torch.randn(n, generator=torch.Generator().manual_seed(1))
    add64, add = _logits(T, E, dtype, 5, pad)
    add64 = np.where(np.isinf(add64), 0.0, add64) * 1e-4
    add[:, :E] = torch.from_numpy(add64).to(add.dtype).cuda()
    add64 = add[:, :E].cpu().double().numpy()
    want, mag = balance.backward(l64, wc, k, starts, kind, ALPHA, d_loss.double().numpy())
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    used = ~np.isnan(want[:, 0])
    for d_add in (None, add):
        out = torch.full((T + 1, E + 2 * pad), S, dtype=dev.dtype, device="cuda")
        dl = d_loss.cuda()
        X.check(X.xs_balance_loss_backward(g, dev.data_ptr(), dev.stride(0), T, st.data_ptr(), n, ALPHA, counts.data_ptr(), dl.data_ptr(), X.ptr(d_add),
                                           add.stride(0), out.data_ptr(), out.stride(0), None, _stream()))
        torch.cuda.synchronize()
        got = out[:T, :E].cpu().double().numpy()
        assert (out[T] == S).all() and (out[:, E:] == S).all() and (got[~used] == S).all()
        w = want + (add64 if d_add is not None else 0.0)
        tol = half * np.abs(w) + 2.0 ** -15 * mag + 2.0 ** -24 * (np.abs(w) + np.abs(add64)) + 1e-38
        assert np.all((np.abs(got - w) <= tol)[used])
    # in the place of d_add
    X.check(X.xs_balance_loss_backward(g, dev.data_ptr(), dev.stride(0), T, st.data_ptr(), n, ALPHA, counts.data_ptr(), dl.data_ptr(), add.data_ptr(),
                                       add.stride(0), add.data_ptr(), add.stride(0), None, _stream()))
    torch.cuda.synchronize()
    assert torch.equal(add[:, :E][torch.from_numpy(used).cuda()], out[:T, :E][torch.from_numpy(used).cuda()])


@pytest.mark.parametrize("E,pad", [(16, 0), (60, 3), (256, 0), (700, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sigmoid_shares_of_tokens_whose_scores_are_all_small(E, pad, dtype):
    """Scores far below the smallest normal number still have shares; a token a sequence, so that the mean is its shares. A score's
    exponential takes x log2 e, off by 2^-23 |x| relative (the product's rounding and the constant's), |x| at most 64 + 16 where a token's scores are
    large enough to be added as they are, and 2^-21 of its own; a share has two of them and the sum's 64 + 10 roundings."""
    X = xs()
    g = torch.Generator().manual_seed(E)
    shift = torch.tensor([0.0, -30.0, -44.0, -45.0, -60.0, -80.0, -86.9, -87.4, -88.0, -88.8, -95.0, -104.0, -200.0, -600.0])
    l = (torch.randn((len(shift), E), generator=g) * 2 + shift[:, None]).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    l[:, 1] = -float("inf")
    l[8, 2:] = -float("inf")
    T, k = len(shift), 3
    full = torch.full((T, E + pad), float("nan"), dtype=l.dtype)
    full[:, :E] = l
    l64, dev, gt = l.double().numpy(), full.cuda(), _gate(E, k, "sigmoid", dtype)
    idx = np.tile(np.array([[0, 2, 5]], dtype=np.int32), (T, 1))
    starts = list(range(T + 1))
    counts, mean, loss, st, status = _forward(gt, dev, torch.from_numpy(idx).cuda(), starts, T)
    _, wm, wl = balance.loss(l64, idx, starts, "sigmoid", ALPHA)
    rel = 2 * (80 * 2.0 ** -23 + 2.0 ** -21) + 74 * 2.0 ** -24
    assert status == 0 and np.allclose(wm.sum(1), 1.0)
    assert np.all(np.abs(mean.cpu().double().numpy() - wm) <= rel * wm + 1e-38)
    assert np.all(np.abs(loss.cpu().double().numpy() - wl) <= (rel + 2.0 ** -13) * wl)
    d_loss = torch.randn(T, generator=g)
    want, mag = balance.backward(l64, counts.cpu().numpy(), k, starts, "sigmoid", ALPHA, d_loss.double().numpy())
    out, dl = torch.full((T, E + pad), S, dtype=dev.dtype, device="cuda"), d_loss.cuda()
    X.check(X.xs_balance_loss_backward(gt, dev.data_ptr(), dev.stride(0), T, st.data_ptr(), T, ALPHA, counts.data_ptr(), dl.data_ptr(), None, 0, out.data_ptr(),
                                       out.stride(0), None, _stream()))
    torch.cuda.synchronize()
    got = out[:, :E].cpu().double().numpy()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert np.all(np.abs(got - want) <= half * np.abs(want) + (4 * rel + 2.0 ** -15) * mag + 1e-38)


@pytest.mark.parametrize("E", [16, 60, 256, 700])
def test_small_and_ordinary_sigmoid_scores_side_by_side(E):
    # tokens of one wave whose scores are all small, and others; shares within the bound of the test above
    X = xs()
    T, k = 203, 2
    g = torch.Generator().manual_seed(E)
    shift = torch.tensor([0.0, -95.0, -40.0, -600.0, 5.0, -87.4, -50.0])[torch.randint(0, 7, (T,), generator=g)]
    l = torch.randn((T, E), generator=g) * 2 + shift[:, None]
    l64, dev, gt = l.double().numpy(), l.cuda(), _gate(E, k, "sigmoid", "f32")
    idx = np.argsort(-l64, 1, kind="stable")[:, :k].astype(np.int32)
    counts, mean, loss, st, status = _forward(gt, dev, torch.from_numpy(idx).cuda(), [0, T], T)
    wc, wm, wl = balance.loss(l64, idx, [0, T], "sigmoid", ALPHA)
    rel = 2 * (80 * 2.0 ** -23 + 2.0 ** -21) + 74 * 2.0 ** -24
    assert status == 0 and np.array_equal(counts.cpu().numpy(), wc)
    assert np.all(np.abs(mean.cpu().double().numpy() - wm) <= (rel + (T + 64) * 2.0 ** -24) * wm)
    want, mag = balance.backward(l64, wc, k, [0, T], "sigmoid", ALPHA, np.ones(1))
    out, one = torch.zeros_like(dev), torch.ones(1, device="cuda")
    X.check(X.xs_balance_loss_backward(gt, dev.data_ptr(), E, T, st.data_ptr(), 1, ALPHA, counts.data_ptr(), one.data_ptr(), None, 0, out.data_ptr(), E, None,
                                       _stream()))
    torch.cuda.synchronize()
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= 2.0 ** -24 * np.abs(want) + (4 * rel + 2.0 ** -15) * mag + 1e-38)


def test_one_sequence_without_starts_equals_it_with_them():
    X = xs()
    T, E, k = 777, 160, 6
    l64, dev = _logits(T, E, "f32", 0, 0)
    g = _gate(E, k, "sigmoid", "f32")
    di = torch.from_numpy(np.argsort(-l64, 1, kind="stable")[:, :k].astype(np.int32)).cuda()
    counts, mean, loss, st, _ = _forward(g, dev, di, [0, T], T)
    c2, m2, l2 = torch.zeros_like(counts), torch.zeros_like(mean), torch.zeros_like(loss)
    ws = X.workspace(X.xs_balance_loss_workspace_bytes, T, E, 1)
    X.check(X.xs_balance_loss(g, dev.data_ptr(), E, T, di.data_ptr(), None, 1, ALPHA, c2.data_ptr(), m2.data_ptr(), l2.data_ptr(), ws.data_ptr(),
                              ws.numel(), None, _stream()))
    assert torch.equal(counts, c2) and torch.equal(mean, m2) and torch.equal(loss, l2)
    one = torch.ones(1, device="cuda")
    out = [torch.zeros_like(dev) for _ in range(2)]
    for o, s in zip(out, (st.data_ptr(), None)):
        X.check(X.xs_balance_loss_backward(g, dev.data_ptr(), E, T, s, 1, ALPHA, counts.data_ptr(), one.data_ptr(), None, 0, o.data_ptr(), E, None, _stream()))
    assert torch.equal(*out)


def test_bad_indices_and_sequences():
    X = xs()
    T, E, k = 64, 32, 4
    l64, dev = _logits(T, E, "f32", 0, 0)
    g = _gate(E, k, "softmax", "f32")
    idx = gate.select(l64, k, "softmax")
    idx[5, 1], idx[6, 0], idx[7] = E, -3, 1
    counts, mean, loss, _, status = _forward(g, dev, torch.from_numpy(idx).cuda(), [0, 30, 64], T)
    wc, _, wl = balance.loss(l64, idx, [0, 30, 64], "softmax", ALPHA)
    assert status == X.XS_EBADINPUT and np.array_equal(counts.cpu().numpy(), wc)
    assert np.all(np.abs(loss.cpu().double().numpy() - wl) <= 2.0 ** -12 * wl)
    idx = gate.select(l64, k, "softmax")
    for starts, bad in (([0, 30, 65], 1), ([-1, 30, 64], 0), ([0, 50, 40], 1)):
        counts, mean, loss, st, status = _forward(g, dev, torch.from_numpy(idx).cuda(), starts, T)
        assert status == X.XS_EBADINPUT and not counts[bad].any() and not mean[bad].any() and loss[bad] == 0 and counts[1 - bad].any()
    # starts that go up and down: sequences overlap, the call only has to stay in its buffers
    _, _, _, st, status = _forward(g, dev, torch.from_numpy(idx).cuda(), [0, 64] * 40, T)
    assert status == X.XS_EBADINPUT
    d = torch.zeros_like(dev)
    st8 = torch.zeros(1, dtype=torch.int32, device="cuda")
    counts = torch.zeros((79, E), dtype=torch.int32, device="cuda")
    X.check(X.xs_balance_loss_backward(g, dev.data_ptr(), E, T, st.data_ptr(), 79, ALPHA, counts.data_ptr(), torch.ones(79, device="cuda").data_ptr(), None, 0,
                                       d.data_ptr(), E, st8.data_ptr(), _stream()))
    assert int(st8.item()) == X.XS_EBADINPUT


def test_nan_logits_give_nan_shares_and_no_tokens_give_zeros():
    X = xs()
    T, E, k = 20, 16, 2
    l64, dev = _logits(T, E, "f32", 0, 0)
    dev[3, 4] = float("nan")
    g = _gate(E, k, "softmax", "f32")
    idx = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    _, mean, loss, _, _ = _forward(g, dev, idx, [0, 10, 20], T)
    assert torch.isnan(mean[0]).all() and torch.isnan(loss[0]) and torch.isfinite(mean[1]).all()
    counts, mean, loss, _, status = _forward(g, dev, idx, [0, 0, 0], 0)
    assert status == 0 and not counts.any() and not mean.any() and not loss.any()


def test_equal_bits_in_a_replayed_graph():
    X = xs()
    T, E, k, n = 5000, 256, 8, 3
    l64, dev = _logits(T, E, "bf16", 0, 0)
    g = _gate(E, k, "sigmoid", "bf16")
    di = torch.from_numpy(np.argsort(-l64, 1, kind="stable")[:, :k].astype(np.int32)).cuda()
    counts, mean, loss, st, _ = _forward(g, dev, di, [0, 1234, 1240, 5000], T)
    ws = X.workspace(X.xs_balance_loss_workspace_bytes, T, E, n)
    c, m, lo = torch.zeros_like(counts), torch.zeros_like(mean), torch.zeros_like(loss)
    d, one = torch.zeros_like(dev), torch.ones(n, device="cuda")

    def step():
        X.check(X.xs_balance_loss(g, dev.data_ptr(), E, T, di.data_ptr(), st.data_ptr(), n, ALPHA, c.data_ptr(), m.data_ptr(), lo.data_ptr(), ws.data_ptr(),
                                  ws.numel(), None, _stream()))
        X.check(X.xs_balance_loss_backward(g, dev.data_ptr(), E, T, st.data_ptr(), n, ALPHA, c.data_ptr(), one.data_ptr(), None, 0, d.data_ptr(), E, None,
                                           _stream()))

    step()
    torch.cuda.synchronize()
    first = d.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (c, m, lo, d):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, counts) and torch.equal(m, mean) and torch.equal(lo, loss) and torch.equal(d, first)


def test_no_tokens():
    X = xs()
    g = _gate(64, 4, "sigmoid", "f32")
    counts, mean, loss = torch.full((2, 64), 7, dtype=torch.int32, device="cuda"), torch.full((2, 64), S, device="cuda"), torch.full((2,), S, device="cuda")
    starts = torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = X.workspace(X.xs_balance_loss_workspace_bytes, 0, 64, 2)
    X.check(X.xs_balance_loss(g, None, 64, 0, None, starts.data_ptr(), 2, ALPHA, counts.data_ptr(), mean.data_ptr(), loss.data_ptr(), ws.data_ptr(), ws.numel(), None,
                              _stream()))
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in (counts, mean, loss))


def test_thousands_of_short_sequences():
    X = xs()
    lens = np.random.default_rng(0).integers(0, 5, 5000)
    lens[77] = 1200
    starts = [0] + [int(x) for x in np.cumsum(lens)]
    T, E, k = starts[-1], 70, 3
    l64, dev = _logits(T, E, "f32", 0, 0)
    idx = np.argsort(-l64, 1, kind="stable")[:, :k].astype(np.int32)
    counts, mean, loss, st, status = _forward(_gate(E, k, "softmax", "f32"), dev, torch.from_numpy(idx).cuda(), starts, T)
    wc, wm, wl = balance.loss(l64, idx, starts, "softmax", ALPHA)
    rel = 2.0 ** -17 + 1264 * 2.0 ** -24
    assert status == 0 and np.array_equal(counts.cpu().numpy(), wc)
    assert np.all(np.abs(mean.cpu().double().numpy() - wm) <= rel * wm + 1e-38)
    assert np.all(np.abs(loss.cpu().double().numpy() - wl) <= (rel + 2.0 ** -13) * wl)
