"""GPU parity of packed attention and its gradients against the fp64 oracle, within the bounds the oracle
derives (oracle/packed.py): a probability and a result each rounded to bf16, everything else in fp32."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_helpers import require_gpu, xs
from oracle import packed

pytestmark = pytest.mark.gpu

SENTINEL = -7.0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _laid(x, layout):
    """[rows][heads][D] on the GPU: heads side by side, head by head, or rows and heads with room between."""
    x = x.cuda()
    if layout == "token":
        return x.contiguous()
    if layout == "head":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    full = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + 8), float("nan"), dtype=x.dtype, device="cuda")
    full[:, :-1, :-8] = x
    return full[:, :-1, :-8]


class Case:
    """spans: (first query, queries, first key, keys). Rows outside every span are NaN in k, v and q."""

    def __init__(self, spans, Tq, Tk, H, Hkv, D, layout="token", causal=True, seed=0, scale=0.0, cache=False, max_k=0, std=1.0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda rows, h: (torch.randn((rows, h, D), generator=g) * std).bfloat16()
        q, k, v, d_o = rnd(Tq, H), rnd(Tk, Hkv), rnd(Tk, Hkv), rnd(Tq, H)
        self.in_q, self.in_k = np.zeros(Tq, bool), np.zeros(Tk, bool)
        for q0, n, k0, m in spans:
            self.in_q[q0:q0 + n] = True
            self.in_k[k0:k0 + m] = True
        for t, used in ((q, self.in_q), (d_o, self.in_q), (k, self.in_k), (v, self.in_k)):
            t[torch.from_numpy(~used)] = float("nan")
        self.spans, self.causal, self.scale, self.layout = spans, causal, scale, layout
        self.host = {n: t.double().numpy() for n, t in (("q", q), ("k", k), ("v", v), ("d_o", d_o))}
        self.q, self.k, self.v, self.d_o = (_laid(t, layout) for t in (q, k, v, d_o))
        i32 = dict(dtype=torch.int32, device="cuda")
        self.q_start = torch.tensor([s[0] for s in spans] + [spans[-1][0] + spans[-1][1]], **i32)
        if cache:
            self.k_start, self.k_rows = torch.tensor([s[2] for s in spans], **i32), torch.tensor([s[3] for s in spans], **i32)
        else:
            self.k_start, self.k_rows = torch.tensor([s[2] for s in spans] + [spans[-1][2] + spans[-1][3]], **i32), None
        self.max_k = max_k
        self.status = torch.zeros(1, **i32)
        like = lambda t: _laid(torch.full(t.shape, SENTINEL, dtype=t.dtype), layout)
        self.o, self.dq, self.dk, self.dv = like(q), like(q), like(k), like(k)
        self.lse = torch.full((H, Tq), SENTINEL, device="cuda")
        X = xs()
        self.a = X.attn_packed(self.q, self.k, self.v, self.o, self.q_start, self.k_start, self.k_rows, self.lse, causal, max_k, scale)
        self.ws = X.workspace(X.xs_attention_packed_workspace_bytes, self.a)
        self.ws.fill_(255)

    def forward(self):
        X = xs()
        X.check(X.xs_attention_packed(self.a, X.ptr(self.ws), self.ws.numel(), self.status.data_ptr(), _stream()))

    def backward(self):
        X = xs()
        g = X.attn_packed_grads(self.d_o, self.dq, self.dk, self.dv)
        self.bws = X.workspace(X.xs_attention_packed_backward_workspace_bytes, self.a)
        self.bws.fill_(255)
        X.check(X.xs_attention_packed_backward(self.a, g, X.ptr(self.bws), self.bws.numel(), self.status.data_ptr(), _stream()))

    def check_forward(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        h = self.host
        o, bo, lse, bl = packed.attention(h["q"], h["k"], h["v"], self.spans, self.scale or None, self.causal)
        _near(self.o, o, bo, self.in_q, "o")
        got = self.lse.cpu().double().numpy()
        assert (got[:, ~self.in_q] == SENTINEL).all()
        got, lse, bl = got[:, self.in_q], lse[:, self.in_q], bl[:, self.in_q]
        empty = np.isinf(lse)
        assert (got[empty] == -np.inf).all()
        assert np.all(np.abs(got[~empty] - lse[~empty]) <= bl[~empty]), np.max(np.abs(got - lse)[~empty] / bl[~empty])

    def check_backward(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        h = self.host
        out, bound = packed.gradients(h["q"], h["k"], h["v"], h["d_o"], self.spans, self.scale or None, self.causal)
        for name, used in (("dq", self.in_q), ("dk", self.in_k), ("dv", self.in_k)):
            _near(getattr(self, name), out[name], bound[name], used, name)


def _near(got, want, bound, used, what):
    g = got.cpu().double().numpy()
    assert (g[~used] == SENTINEL).all(), f"{what}: rows outside every sequence were written"
    g, want, bound = g[used], want[used], bound[used]
    assert np.isfinite(g).all(), f"{what}: not finite"
    worst = np.max(np.abs(g - want) / np.maximum(bound, 1e-30)) if g.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


def _packed(lens, gap=0):
    at, out = gap, []
    for n in lens:
        out.append((at, n, at, n))
        at += n
    return out, at + gap


FEW = [([1], 2, 1), ([1, 1, 1], 8, 2), ([31, 0, 1], 4, 4), ([33, 64, 5], 6, 2), ([97], 3, 1), ([130, 127], 2, 2), ([257], 16, 1), ([500, 3], 1, 1),
       ([0, 0, 7], 5, 1)]


@pytest.mark.parametrize("lens,H,Hkv", FEW)
@pytest.mark.parametrize("D,layout", [(128, "token"), (64, "head"), (128, "room"), (64, "token")])
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows(lens, H, Hkv, D, layout, causal):
    spans, T = _packed(lens, gap=3)
    c = Case(spans, T, T, H, Hkv, D, layout, causal, seed=len(lens) + H)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


# 64 and 48 query heads make enough tiles of 128 rows for the kernel of many rows
MANY = [([40, 70, 33, 1, 100, 34], 64, 32), ([129, 0, 255], 96, 96), ([64, 65, 63], 128, 64), ([130, 61], 90, 90)]


@pytest.mark.parametrize("lens,H,Hkv", MANY)
@pytest.mark.parametrize("D,layout", [(128, "token"), (64, "token"), (128, "head"), (64, "room")])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows(lens, H, Hkv, D, layout, causal):
    spans, T = _packed(lens, gap=2)
    c = Case(spans, T, T, H, Hkv, D, layout, causal, seed=len(lens))
    assert c.ws.numel() == 0
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,H,Hkv", [(1, 8, 2), (1, 1, 1), (1, 32, 1), (2, 6, 2), (5, 8, 1), (17, 4, 2), (40, 3, 3), (50, 96, 32), (8, 48, 16)])
@pytest.mark.parametrize("cap", [1024, 4200])
def test_new_tokens_over_a_cache(new, H, Hkv, D, cap):
    # keys behind each sequence's rows are NaN; lengths around the tiles' ends, fewer keys than queries, none. Caches of 1024 keys take one
    # launch, in longer ones the keys are dealt out.
    lens = [new, 0, 1, 31, 32, 33, 64, 95, 127, 129, 300, cap - 24]
    spans = [(1 + i * new, new, i * cap, m) for i, m in enumerate(lens)]
    c = Case(spans, 2 + new * len(lens), cap * len(lens), H, Hkv, D, cache=True, max_k=cap, seed=new)
    many = (new * (H // Hkv) * len(lens) // 128 + len(lens)) * Hkv * 4000 > 256 * cap      # tiles of rows that fill the chip
    assert (c.ws.numel() > 0) == (cap > 1024 and not many)
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("Tk", [800, 1600])
def test_a_shared_prefix_and_sequences_in_any_order(Tk):
    spans = [(0, 1, 500, 300), (1, 1, 0, 700), (2, 1, 500, 299), (3, 1, 10, 1)]
    c = Case(spans, 4, Tk, 8, 2, 128, cache=True)
    c.forward()
    c.check_forward()


def test_many_sequences():
    n = 200
    lens = [int(x) for x in np.random.default_rng(0).integers(0, 70, n)]
    spans, at, ks = [], 0, 0
    for i, m in enumerate(lens):
        q = i % 3
        spans.append((at, q, ks, m))
        at += q
        ks += m + 5
    for max_k in (70, 0):              # in one launch, and dealt out
        c = Case(spans, at, ks, 4, 2, 128, cache=True, max_k=max_k)
        assert (c.ws.numel() > 0) == (max_k == 0)
        c.forward()
        c.check_forward()


def test_many_sequences_of_many_rows():
    # more than 64 sequences over units of 128 rows, some without queries or keys, one long
    n = 90
    rng = np.random.default_rng(1)
    spans, at, ks = [], 0, 0
    for i in range(n):
        q, m = (0 if i % 7 == 0 else int(rng.integers(1, 40))), (1500 if i == 70 else int(rng.integers(0, 90)))
        spans.append((at, q, ks, m))
        at += q
        ks += m
    for causal in (True, False):
        c = Case(spans, at, ks, 2, 1, 64, cache=True, causal=causal)
        assert c.ws.numel() > 0
        c.forward()
        c.check_forward()


@pytest.mark.parametrize("G", [3, 8, 48, 128, 130])
def test_groups_of_any_size_over_long_sequences(G):
    # units of as many queries as fit 128 rows; groups of more than 128 heads have none
    spans = [(0, 130, 0, 1300), (130, 1, 1300, 64), (131, 70, 1364, 65)]
    c = Case(spans, 201, 4200, G, 1, 64, cache=True)
    assert (c.ws.numel() > 0) == (G <= 128)
    c.forward()
    c.check_forward()


# 32 query heads a key head have more rows than the kernels of few or short prompts take
@pytest.mark.parametrize("H", [4, 64])
def test_gradients_of_more_keys_than_queries_and_fewer(H):
    # a prompt behind a prefix that has gradients too, queries that see nothing, no queries, no keys
    spans = [(0, 20, 0, 90), (20, 70, 90, 30), (90, 0, 120, 40), (90, 10, 160, 0), (100, 130, 160, 200)]
    for causal in (True, False):
        for D in (64, 128):
            c = Case(spans, 230, 360, H, 2, D, causal=causal)
            c.forward()
            c.check_forward()
            c.backward()
            c.check_backward()


# 512 keys and more a sequence take key tiles of 256; 70, 3 and 1 heads leave tiles inside one workgroup's share and over several
@pytest.mark.parametrize("lens,H,Hkv", [([1025], 4, 1), ([511, 1, 1030], 6, 2), ([700, 900], 70, 35), ([513], 1, 1), ([900], 6, 2), ([521, 503], 20, 20)])
@pytest.mark.parametrize("D,layout", [(128, "token"), (64, "room")])
@pytest.mark.parametrize("causal", [True, False])
def test_long_sequences(lens, H, Hkv, D, layout, causal):
    spans, T = _packed(lens)
    assert T // len(lens) >= 512
    c = Case(spans, T, T, H, Hkv, D, layout, causal, seed=H)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


# each form of the gradients' kernels: key tiles dealt out over ranges with parts of several, and in one launch; rows by 128 and by 32
@pytest.mark.parametrize("lens,H,Hkv,D", [([1025], 4, 1, 128), ([1025], 4, 1, 64), ([511, 1, 1030], 6, 2, 128), ([700, 900], 70, 35, 128), ([521, 503], 20, 20, 64),
                                          ([300, 200, 0, 450], 32, 2, 128), ([300, 200, 0, 450], 32, 2, 64), ([500, 3, 97], 1, 1, 128), ([2100], 2, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_gradients_in_the_2_norm(lens, H, Hkv, D, causal):
    # 256 rows of a head at a time (and the whole tensor): independent roundings, so that a block of rows left out, which a bound of each
    # element's worst case hides, stands out
    spans, T = _packed(lens)
    c = Case(spans, T, T, H, Hkv, D, causal=causal, seed=H + 1)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    h = c.host
    want, _ = packed.gradients(h["q"], h["k"], h["v"], h["d_o"], spans, causal=causal)
    mean = packed.deviations(h["q"], h["k"], h["v"], h["d_o"], spans, causal=causal)
    for x in want:
        off = (getattr(c, x).cpu().double().numpy() - want[x]) ** 2
        assert off.sum() <= mean[x].sum(), f"{x}: {np.sqrt(off.sum() / mean[x].sum()):.3f} of the 2-norm"
        for at, n, _, _ in spans:
            for r in range(at, at + n - 63, 256):
                rows = slice(r, min(r + 256, at + n))
                worst = np.max(np.sqrt(off[rows].sum((0, 2)) / mean[x][rows].sum((0, 2))))
                assert worst <= 1.0, f"{x}, rows {rows}: {worst:.3f} of the 2-norm"


@pytest.mark.parametrize("lens", [[4200], [4100, 1, 4200]])
@pytest.mark.parametrize("D,layout", [(128, "token"), (64, "head")])
@pytest.mark.parametrize("causal", [True, False])
def test_long_prompts_whose_keys_are_dealt_out(lens, D, layout, causal):
    spans, T = _packed(lens, gap=1)
    c = Case(spans, T, T, 2, 1, D, layout, causal)
    assert c.ws.numel() > 0
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("H,Hkv", [(4, 2), (16, 1)])
def test_gradients_of_a_long_prefix_and_of_queries_that_see_nothing(H, Hkv):
    spans = [(0, 33, 0, 1500), (33, 600, 1500, 90), (633, 0, 1590, 257), (633, 700, 1847, 513)]
    for causal in (True, False):
        c = Case(spans, 1333, 2360, H, Hkv, 128, causal=causal)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


@pytest.mark.parametrize("D,layout", [(128, "token"), (64, "head")])
@pytest.mark.parametrize("causal", [True, False])
def test_large_groups_over_short_sequences(D, layout, causal):
    # key tiles of 128 whose blocks are dealt out over ranges, with parts of several
    spans, T = _packed([300, 200, 0, 450], gap=1)
    c = Case(spans, T, T, 32, 2, D, layout, causal)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


def test_no_queries_or_no_keys_at_all():
    X = xs()
    for D in (64, 128):
        k = torch.randn(300, 2, D, device="cuda").bfloat16()
        q = torch.randn(70, 4, D, device="cuda").bfloat16()
        none = torch.empty(0, 4, D, device="cuda", dtype=torch.bfloat16), torch.empty(0, 2, D, device="cuda", dtype=torch.bfloat16)
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
        status = i32(0)
        for qq, kk in ((none[0], k), (q, none[1]), (none[0], none[1])):
            o, lse = torch.full_like(qq, SENTINEL), torch.full((4, qq.shape[0]), SENTINEL, device="cuda")
            a = X.attn_packed(qq, kk, kk.clone(), o, i32(0, 0, qq.shape[0]), i32(0, kk.shape[0], kk.shape[0]), lse=lse)
            ws = X.workspace(X.xs_attention_packed_workspace_bytes, a)
            X.check(X.xs_attention_packed(a, X.ptr(ws), ws.numel(), status.data_ptr(), _stream()))
            dq, dk, dv = torch.full_like(qq, SENTINEL), torch.full_like(kk, SENTINEL), torch.full_like(kk, SENTINEL)
            ws = X.workspace(X.xs_attention_packed_backward_workspace_bytes, a)
            X.check(X.xs_attention_packed_backward(a, X.attn_packed_grads(qq.clone(), dq, dk, dv), X.ptr(ws), ws.numel(), status.data_ptr(), _stream()))
            torch.cuda.synchronize()
            assert int(status.item()) == 0
            assert all((t == 0).all() for t in (o, dq, dk, dv)) and (lse == -np.inf).all()


@pytest.mark.parametrize("causal", [True, False])
def test_thousands_of_short_sequences(causal):
    # queries and keys of 3000 sequences of 0 to 3 tokens, one of 900 among them
    lens = [int(x) for x in np.random.default_rng(2).integers(0, 4, 3000)]
    lens[1717] = 900
    spans, T = _packed(lens)
    for H, Hkv in ((1, 1), (40, 1)):
        c = Case(spans, T, T, H, Hkv, 64, causal=causal)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


def test_large_scores_and_a_given_scale():
    spans, T = _packed([150, 40])
    for std, scale in ((3.0, 0.0), (1.0, 0.5), (2.0, 1e-3)):
        c = Case(spans, T, T, 4, 2, 128, std=std, scale=scale)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


def test_gradients_are_the_differences_of_the_forward_call():
    # central differences of the call's own o (rounded to bf16) along random directions: each end is off by 2^-8 |o| + 2^-8
    # sum P |v| (below 2^-7 max |v| together per element), the inputs' steps are exact in bf16
    spans, T = _packed([48, 17])
    c = Case(spans, T, T, 2, 1, 64, seed=5)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    d_o = c.d_o.double()
    for x, grad in (("q", c.dq), ("k", c.dk), ("v", c.dv)):
        t = getattr(c, x)
        base = t.clone()
        step = 0.25 * torch.sign(torch.randn(t.shape, generator=torch.Generator().manual_seed(1))).cuda().bfloat16()
        ends = []
        for s in (1, -1):
            t.copy_(base + s * step)
            moved = (t.double() - base.double())
            c.forward()
            torch.cuda.synchronize()
            ends.append(((c.o.double() * d_o).sum().item(), moved))
        t.copy_(base)
        # moved differs from +-step where the sum rounded: the secant is taken between the points reached
        along = (grad.double() * (ends[0][1] - ends[1][1])).sum().item()
        size = (grad.double().abs() * step.double().abs()).sum().item()
        # rounding of o: independent signs, so its sum is of the order of the 2-norm, 6 of them allowed; the
        # function's third derivative along a step of 0.25 (softmax: scores move by up to 2) is not small for q and k
        noise = 6 * 2.0 ** -7 * float((c.o.double().abs() * d_o.abs()).norm()) * 2
        assert abs((ends[0][0] - ends[1][0]) - along) <= noise + (0.0 if x == "v" else 0.25 * size), x


@pytest.mark.parametrize("lens,H,Hkv,D", [([48, 17], 2, 1, 64), ([300, 1, 40], 4, 2, 128), ([130, 61], 24, 24, 64)])
def test_gradients_are_the_slope_of_the_forward_call(lens, H, Hkv, D):
    """The call's own o along +-1/8 of the sign of the (fp64) gradient, so that the change is the sum of all its magnitudes and
    every element's counts. Values of one key lie close together and d_o is positive: the change is large beside the roundings of o, all taken
    at their worst, as are the gradients'; the differences' curvature is the fp64 function's at the same points."""
    spans, T = _packed(lens)
    c = Case(spans, T, T, H, Hkv, D)
    g = torch.Generator().manual_seed(5)
    c.v.copy_((torch.randn((T, Hkv, 1), generator=g) + 0.25 * torch.randn((T, Hkv, D), generator=g)).bfloat16())
    c.d_o.copy_((0.5 + torch.rand((T, H, D), generator=g)).bfloat16())
    at = {n: getattr(c, n).cpu().double().numpy() for n in ("q", "k", "v", "d_o")}
    want, bound = packed.gradients(at["q"], at["k"], at["v"], at["d_o"], spans)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    for x in "qkv":
        t, base = getattr(c, x), getattr(c, x).clone()
        got = getattr(c, "d" + x).cpu().double().numpy()
        ends, exact, points, noise = [], [], [], 0.0
        for s in (1, -1):
            t.copy_(base + s * 0.125 * torch.sign(torch.from_numpy(want["d" + x])).cuda().bfloat16())
            c.forward()
            torch.cuda.synchronize()
            points.append(t.cpu().double().numpy())
            o, bo, _, _ = packed.attention(*({**at, x: points[-1]}[n] for n in "qkv"), spans)
            ends.append((c.o.cpu().double().numpy() * at["d_o"]).sum())
            exact.append((o * at["d_o"]).sum())
            noise += (bo * np.abs(at["d_o"])).sum()
        t.copy_(base)
        moved = points[0] - points[1]               # between the points reached: some sums were rounded
        slope = (want["d" + x] * moved).sum()
        tolerance = noise + (bound["d" + x] * np.abs(moved)).sum() + abs(exact[0] - exact[1] - slope)
        assert 4 * tolerance < slope, x              # so that a gradient negated, halved, doubled or of zeros is told from it
        off = lambda grad: abs(ends[0] - ends[1] - (grad * moved).sum())
        assert off(got) <= tolerance, x
        assert all(off(w * got) > tolerance for w in (-1.0, 0.0, 0.5, 2.0)), x


@pytest.mark.parametrize("what", ["q descends", "q past the end", "keys before the start", "keys past the end", "more than max_k", "negative rows"])
def test_bad_sequences_are_skipped(what):
    X = xs()
    spans = [(0, 4, 0, 100), (4, 4, 100, 100), (8, 4, 200, 100)]
    c = Case(spans, 12, 300, 4, 2, 128, cache=True, max_k=100)
    bad = 1
    if what == "q descends":
        c.q_start[2] = 2
        bad = (1, 2)
    elif what == "q past the end":
        c.q_start[3] = 13
        bad = 2
    elif what == "keys before the start":
        c.k_start[1] = -1
    elif what == "keys past the end":
        c.k_start[1] = 201
    elif what == "more than max_k":
        c.k_rows[1] = 101
    else:
        c.k_rows[1] = -1
    c.forward()
    torch.cuda.synchronize()
    assert int(c.status.item()) == X.XS_EBADINPUT
    if what != "q descends":
        assert (c.o[4 * bad:4 * bad + 4] == SENTINEL).all()
        good = [i for i in range(3) if i != bad]
        o, bo, _, _ = packed.attention(c.host["q"], c.host["k"], c.host["v"], [spans[i] for i in good])
        rows = np.concatenate([np.arange(4 * i, 4 * i + 4) for i in good])
        assert np.all(np.abs(c.o.cpu().double().numpy()[rows] - o[rows]) <= bo[rows])


@pytest.mark.parametrize("H", [2, 128])
def test_bad_sequences_have_no_gradients(H):
    X = xs()
    spans, T = _packed([40, 50, 60])
    c = Case(spans, T, T, H, 2, 64)
    c.forward()
    c.backward()
    c.check_backward()
    for t in (c.dq, c.dk, c.dv):
        t.fill_(SENTINEL)
    c.k_start[3] = T + 1
    c.backward()
    torch.cuda.synchronize()
    assert int(c.status.item()) == X.XS_EBADINPUT
    for t in (c.dq, c.dk, c.dv):
        assert (t[90:] == SENTINEL).all() and torch.isfinite(t[:90]).all() and (t[:90] != SENTINEL).any()


def test_two_streams_and_replayed_graphs_with_workspaces_of_their_own():
    spans = [(i, 1, i * 700, 650 - 50 * i) for i in range(5)]
    cases = [Case(spans, 5, 3500, 8, 2, 128, cache=True, seed=s) for s in range(2)]
    assert cases[0].ws.numel() > 0
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, st in zip(cases, streams):
        with torch.cuda.stream(st):
            c.forward()
    for c in cases:
        c.check_forward()
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.forward()
        graphs.append(g)
    for _ in range(3):
        for c, g in zip(cases, graphs):
            c.o.fill_(SENTINEL)
            c.lse.fill_(SENTINEL)
            c.ws.fill_(255)
        for g, st in zip(graphs, streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                g.replay()
        for c in cases:
            c.check_forward()


@pytest.mark.parametrize("H", [8, 64])
def test_a_training_step_in_a_graph_and_equal_bits(H):
    spans, T = _packed([200, 57, 300])
    c = Case(spans, T, T, H, 2, 128)
    c.forward()
    c.backward()
    c.check_forward()
    c.check_backward()
    first = [t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv)]
    X = xs()
    g = X.attn_packed_grads(c.d_o, c.dq, c.dk, c.dv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        X.check(X.xs_attention_packed_backward(c.a, g, X.ptr(c.bws), c.bws.numel(), c.status.data_ptr(), _stream()))
    for _ in range(3):
        for t in (c.o, c.lse, c.dq, c.dk, c.dv):
            t.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((c.o, c.lse, c.dq, c.dk, c.dv), first):
            assert torch.equal(t, w)


@pytest.mark.parametrize("new,H,max_k", [(3, 4, 0), (3, 4, 1100), (60, 192, 0), (60, 4, 4200)])
def test_keys_past_2_gib_and_32_bit_offsets(new, H, max_k):
    # one key head of a cache with rows 2^22 elements apart: 700 rows are 5.5 GiB; all four forms
    m, D, row = 700, 128, 1 << 22
    big = torch.empty((m, row), dtype=torch.bfloat16, device="cuda")
    k, v = big[:, :D].unflatten(1, (1, D)), big[:, D:2 * D].unflatten(1, (1, D))
    c = Case([(0, new, 0, m)], new, m, H, 1, D, cache=True)
    k.copy_(c.k)
    v.copy_(c.v)
    X = xs()
    c.a = X.attn_packed(c.q, k, v, c.o, c.q_start, c.k_start, c.k_rows, c.lse)
    if max_k:                              # Tk and max_k only choose the form: no row behind the 700 is read
        c.a.Tk = c.a.max_k = max_k
    c.ws = X.workspace(X.xs_attention_packed_workspace_bytes, c.a)
    assert (c.ws.numel() > 0) == (max_k > 0)
    c.forward()
    c.check_forward()


def test_a_workspace_that_is_missing_or_small_is_refused():
    X = xs()
    c = Case([(0, 1, 0, 2000)], 1, 2000, 4, 1, 128)
    assert c.ws.numel() > 0
    f = lambda p, n: X.xs_attention_packed(c.a, p, n, c.status.data_ptr(), _stream())
    assert f(None, c.ws.numel()) == f(c.ws.data_ptr(), c.ws.numel() - 1) == f(c.ws.data_ptr() + 8, c.ws.numel()) == X.XS_EWORKSPACE
    g = X.attn_packed_grads(c.d_o, c.dq, c.dk, c.dv)
    n = C.c_int64()
    X.check(X.xs_attention_packed_backward_workspace_bytes(c.a, C.byref(n)))
    b = lambda p, n: X.xs_attention_packed_backward(c.a, g, p, n, c.status.data_ptr(), _stream())
    assert b(None, n.value) == b(c.ws.data_ptr(), n.value - 1) == X.XS_EWORKSPACE
    torch.cuda.synchronize()
    assert (c.o == SENTINEL).all() and (c.dq == SENTINEL).all()
