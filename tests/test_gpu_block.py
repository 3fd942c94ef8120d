"""The operators around a MoE layer as a program runs them together: a decoder block's training step from the residual stream to the router
and back, in one stream and in a graph, and a prompt whose tokens come again one by one over a cache.

Every result is held against the fp64 oracles on the inputs it was computed from, within their bounds; the products between the operators are
plain torch ones."""
import numpy as np
import pytest
import torch

from gpu_helpers import require_gpu, xs
from oracle import balance, gate, norm, packed

pytestmark = pytest.mark.gpu

EPS, ALPHA = 1e-6, 1e-2
S = -7.0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _f64(t):
    return t.detach().cpu().double().numpy()


class Block:
    """norm, attention of packed documents, norm, router; its weights, activations, gradients and workspaces."""

    def __init__(self, lens, hidden=256, H=4, K=2, D=64, E=32, k=4):
        X = xs()
        self.T, self.hidden, self.H, self.K, self.D, self.E, self.k, self.n = sum(lens), hidden, H, K, D, E, k, len(lens)
        self.starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
        g = torch.Generator().manual_seed(3)
        rnd = lambda *shape, std=1.0: (torch.randn(shape, generator=g) * std).bfloat16().cuda()
        bf = lambda *shape: torch.full(shape, S, dtype=torch.bfloat16, device="cuda")
        f32 = lambda *shape: torch.full(shape, S, device="cuda")
        T = self.T
        self.x, self.up = rnd(T, hidden), rnd(T, hidden, std=1e-2)
        self.w1, self.w2 = 1 + 0.1 * torch.randn(hidden, generator=g).cuda(), (1 + 0.1 * torch.randn(hidden, generator=g)).bfloat16().cuda()
        self.wqkv, self.wo, self.wg = (rnd(n, m, std=m ** -0.5) for n, m in (((H + 2 * K) * D, hidden), (hidden, H * D), (E, hidden)))
        self.st = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.y1, self.h2, self.y2, self.dh2, self.dx = (bf(T, hidden) for _ in range(5))
        self.qkv, self.dqkv, self.o = bf(T, (H + 2 * K) * D), bf(T, (H + 2 * K) * D), bf(T, H * D)
        self.codes, self.scales = torch.zeros((T, hidden), dtype=torch.uint8, device="cuda"), f32(T, 4)
        self.lse, self.idx, self.topw, self.dtopw = f32(H, T), torch.zeros((T, k), dtype=torch.int32, device="cuda"), f32(T, k), torch.randn((T, k), generator=g).cuda()
        self.logits, self.dlogits, self.sum = bf(T, E), bf(T, E), bf(T, E)
        self.counts, self.mean, self.loss = torch.zeros((self.n, E), dtype=torch.int32, device="cuda"), f32(self.n, E), f32(self.n)
        self.dloss = torch.ones(self.n, device="cuda")
        self.dw1, self.dw2 = f32(hidden), f32(hidden)
        self.do, self.a = bf(T, H * D), bf(T, hidden)
        self.gate = X.gate(E, k, score=X.XS_SCORE_SIGMOID, renormalize=True, logits_type=X.XS_TYPE_BF16)
        # q, k and v are slices of one product's rows, their gradients of another's
        heads = lambda t: (t[:, :H * D].unflatten(1, (H, D)), t[:, H * D:(H + K) * D].unflatten(1, (K, D)), t[:, (H + K) * D:].unflatten(1, (K, D)))
        self.q, self.kk, self.v = heads(self.qkv)
        self.dq, self.dk, self.dv = heads(self.dqkv)
        self.attn = X.attn_packed(self.q, self.kk, self.v, self.o.unflatten(1, (H, D)), self.st, self.st, lse=self.lse)
        self.grads = X.attn_packed_grads(self.do.unflatten(1, (H, D)), self.dq, self.dk, self.dv)
        # one workspace for all, as a program keeps that runs them one behind another
        sizes = [X.workspace(X.xs_attention_packed_workspace_bytes, self.attn), X.workspace(X.xs_attention_packed_backward_workspace_bytes, self.attn),
                 X.workspace(X.xs_balance_loss_workspace_bytes, T, E, self.n), X.workspace(X.xs_rmsnorm_backward_workspace_bytes, T, hidden)]
        self.ws = torch.full((max(w.numel() for w in sizes),), 255, dtype=torch.uint8, device="cuda")

    def step(self):
        X, T, hid, E, st, p = xs(), self.T, self.hidden, self.E, _stream(), xs().ptr
        ws, nb, status = p(self.ws), self.ws.numel(), p(self.status)
        X.check(X.xs_rmsnorm(p(self.x), hid, None, 0, p(self.w1), X.XS_TYPE_F32, EPS, T, hid, None, 0, p(self.y1), hid, None, 0, None, 0, st))
        torch.mm(self.y1, self.wqkv.T, out=self.qkv)
        X.check(X.xs_attention_packed(self.attn, ws, nb, status, st))
        torch.mm(self.o, self.wo.T, out=self.a)
        X.check(X.xs_rmsnorm(p(self.a), hid, p(self.x), hid, p(self.w2), X.XS_TYPE_BF16, EPS, T, hid, p(self.h2), hid, p(self.y2), hid, p(self.codes), hid,
                             p(self.scales), 4, st))
        torch.mm(self.y2, self.wg.T, out=self.logits)
        X.check(X.xs_route_gate(self.gate, p(self.logits), E, T, p(self.idx), p(self.topw), st))
        X.check(X.xs_balance_loss(self.gate, p(self.logits), E, T, p(self.idx), p(self.st), self.n, ALPHA, p(self.counts), p(self.mean), p(self.loss), ws, nb,
                                  status, st))
        X.check(X.xs_route_gate_backward(self.gate, p(self.logits), E, T, p(self.idx), p(self.dtopw), p(self.dlogits), E, status, st))
        X.check(X.xs_balance_loss_backward(self.gate, p(self.logits), E, T, p(self.st), self.n, ALPHA, p(self.counts), p(self.dloss), p(self.dlogits), E,
                                           p(self.sum), E, status, st))
        self.dy2 = torch.mm(self.sum, self.wg)
        X.check(X.xs_rmsnorm_backward(p(self.dy2), hid, p(self.up), hid, p(self.h2), hid, p(self.w2), X.XS_TYPE_BF16, EPS, T, hid, p(self.dh2), hid, p(self.dw2),
                                      ws, nb, st))
        torch.mm(self.dh2, self.wo, out=self.do)
        X.check(X.xs_attention_packed_backward(self.attn, self.grads, ws, nb, status, st))
        self.dy1 = torch.mm(self.dqkv, self.wqkv)
        X.check(X.xs_rmsnorm_backward(p(self.dy1), hid, p(self.dh2), hid, p(self.x), hid, p(self.w1), X.XS_TYPE_F32, EPS, T, hid, p(self.dx), hid, p(self.dw1), ws,
                                      nb, st))

    def results(self):
        return [self.y1, self.qkv, self.o, self.lse, self.h2, self.y2, self.codes, self.scales[:, :2], self.logits, self.idx, self.topw, self.counts, self.mean, self.loss,
                self.dlogits, self.sum, self.dh2, self.dw2, self.dqkv, self.dx, self.dw1]


def _close(got, want, bound):
    assert np.all(np.abs(_f64(got) - want) <= bound)


def _check(b):
    spans = [(a, e - a, a, e - a) for a, e in zip(b.starts, b.starts[1:])]
    U, fine = 2.0 ** -8, 2.0 ** -15           # half a step of bf16; the norm's fp32 sums and quotients
    for h, w, y in ((_f64(b.x), b.w1, b.y1), (_f64(b.h2), b.w2, b.y2)):
        want = norm.norm(h, _f64(w), EPS)
        _close(y, want, (U + fine) * np.abs(want))
    assert np.array_equal(_f64(b.h2), norm.stream(_f64(b.a), _f64(b.x)))
    q, k, v, do = (_f64(t) for t in (b.q, b.kk, b.v, b.do.unflatten(1, (b.H, b.D))))
    o, bo, lse, bl = packed.attention(q, k, v, spans)
    _close(b.o.unflatten(1, (b.H, b.D)), o, bo)
    _close(b.lse, lse, bl)
    grads, bounds = packed.gradients(q, k, v, do, spans)
    for name in ("dq", "dk", "dv"):
        _close(getattr(b, name), grads[name], bounds[name])
    l = _f64(b.logits)
    assert np.array_equal(b.idx.cpu().numpy(), gate.select(l, b.k, "sigmoid"))
    counts, mean, loss = balance.loss(l, b.idx.cpu().numpy(), b.starts, "sigmoid", ALPHA)
    assert np.array_equal(b.counts.cpu().numpy(), counts)
    rel = 2.0 ** -17 + (b.T + 64) * 2.0 ** -24
    _close(b.mean, mean, rel * mean)
    _close(b.loss, loss, (rel + 2.0 ** -13) * loss)
    d, mag = balance.backward(l, counts, b.k, b.starts, "sigmoid", ALPHA, _f64(b.dloss))
    _close(b.sum, d + _f64(b.dlogits), U * np.abs(d + _f64(b.dlogits)) + fine * mag)
    for h, w, dy, dh, dx, dw in ((b.h2, b.w2, b.dy2, b.up, b.dh2, b.dw2), (b.x, b.w1, b.dy1, b.dh2, b.dx, b.dw1)):
        want, wd, mag, dmag = norm.backward(_f64(h), _f64(w), _f64(dy), EPS, _f64(dh))
        _close(dx, want, U * np.abs(want) + fine * mag)
        _close(dw, wd, (fine + (b.T + 64) * 2.0 ** -24) * dmag)


@pytest.mark.parametrize("lens", [[70, 1, 129], [600, 33]])
def test_a_training_step_of_a_block(lens):
    b = Block(lens)
    b.step()
    torch.cuda.synchronize()
    assert int(b.status.item()) == 0
    _check(b)
    first = [t.clone() for t in b.results()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(3):
        for t in b.results():
            t.zero_()
        b.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert [i for i, (t, f) in enumerate(zip(b.results(), first)) if not torch.equal(t, f)] == []


@pytest.mark.parametrize("n,cap", [(90, 1024), (90, 1500), (1300, 1500)])
def test_a_prompt_and_its_tokens_one_by_one(n, cap):
    """A prompt in one call, then its last tokens again one by one over the cache, and all of them as one chunk: the same rows within the
    bounds of both."""
    X = xs()
    H, K, D, last = 8, 2, 128, 5
    g = torch.Generator().manual_seed(n)
    q, k, v = (torch.randn((n, h, D), generator=g).bfloat16().cuda() for h in (H, K, K))
    cache = torch.full((2, 2, cap, K, D), float("nan"), dtype=torch.bfloat16, device="cuda")       # two requests, the second's rows stay NaN
    cache[0, 0, :n], cache[1, 0, :n] = k, v
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    status = i32(0)

    def call(q, k, v, q_start, k_start, k_rows=None, max_k=0):
        o = torch.full_like(q, S)
        a = X.attn_packed(q, k, v, o, q_start, k_start, k_rows, max_k=max_k)
        ws = X.workspace(X.xs_attention_packed_workspace_bytes, a)
        X.check(X.xs_attention_packed(a, X.ptr(ws), ws.numel(), status.data_ptr(), _stream()))
        return o

    whole = call(q, k, v, i32(0, n), i32(0, n))
    one = [call(q[i:i + 1], *(c.flatten(0, 1) for c in cache), i32(0, 1), i32(0), i32(i + 1), cap) for i in range(n - last, n)]
    chunk = call(q[n - last:], *(c.flatten(0, 1) for c in cache), i32(0, last), i32(0), i32(n), cap)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    o, bo, _, _ = packed.attention(_f64(q), _f64(k), _f64(v), [(0, n, 0, n)])
    _close(whole, o, bo)
    _close(torch.cat(one), o[n - last:], bo[n - last:])
    _close(chunk, o[n - last:], bo[n - last:])
