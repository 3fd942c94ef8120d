"""GPU parity of the block-of-128 E4M3 operators against the fp64 oracle: quantizers bit for bit, products
within the fp32 sums' bound and one rounding, SwiGLU and its checkpoint's gradient within theirs."""
import numpy as np
import pytest
import torch

import synth
from gpu_helpers import bits_f64, dev_bits, host_bits, require_gpu, xs
from oracle import fp8, mx

pytestmark = pytest.mark.gpu

B = fp8.BLOCK


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _up(n, m):
    return -(-n // m) * m


class Codes:
    """Device codes and scales of a [rows][cols] matrix, with guard columns and a guard row."""

    def __init__(self, rows, cols, down=1, pad=0, spad=0):
        self.rows, self.K, self.nb = rows, _up(cols, B), _up(cols, B) // B
        self.srows = -(-rows // down)
        self.ld, self.lds = self.K + pad, _up(self.nb, 4) + spad
        self.codes = torch.full((rows + 1, self.ld), 0x5A, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((self.srows + 1, self.lds), -3.0, device="cuda")

    def args(self):
        return self.codes.data_ptr(), self.ld, self.scales.data_ptr(), self.lds

    def get(self):
        c, s = self.codes.cpu().numpy(), self.scales.cpu().numpy()
        assert (c[self.rows] == 0x5A).all() and (c[:, self.K:] == 0x5A).all()            # guards untouched
        assert (s[self.srows] == -3.0).all() and (s[:, self.nb:] == -3.0).all()
        return c[:self.rows, :self.K], s[:self.srows, :self.nb]


NONE = (None, 0, None, 0)


def _same(got, want):
    assert np.array_equal(got[0], want[0])
    assert np.array_equal(got[1].view(np.uint32), want[1].view(np.uint32)) or np.array_equal(got[1], want[1], equal_nan=True)


def _x(rows, cols, seed, special=True):
    g = np.random.default_rng(seed)
    x = (g.standard_normal((rows, cols)) * np.exp(g.uniform(-9, 9, (rows, 1)))).astype(np.float32)
    if special and rows >= 6:
        t = mx.fmt_values(mx.E4M3)
        mid = np.resize((t[1:] + t[:-1]) / 2, cols)
        mid[::B] = 448.0                                        # scale 1: exact ties between codes
        x[0], x[1], x[2] = 0.0, mid, -mid
        x[3] = 3e38 * np.sign(g.standard_normal(cols))
        x[4] = 1e-38 * g.standard_normal(cols)
        x[5] = 2.0 ** -60 * g.uniform(-2, 2, cols)
    return synth.to_bf16_bits(x)


SHAPES = [(1, 8), (1, 128), (7, 136), (130, 264), (128, 128), (257, 1000), (24, 7168), (1, 2048), (300, 640)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad", [0, 16])
def test_quantize_bitexact(rows, cols, pad):
    X = xs()
    x = _x(rows, cols + pad, rows + cols)
    dx = dev_bits(x)
    v = bits_f64(x[:, :cols])
    want, want_t = fp8.quantize(v), fp8.quantize(v.T)
    for rows_too, cols_too in ((True, False), (False, True), (True, True)):
        r, c = Codes(rows, cols, pad=pad, spad=pad // 4), Codes(cols, rows, pad=pad, spad=pad // 4)
        X.check(X.xs_quantize_fp8(dx.data_ptr(), rows, cols, cols + pad, *(r.args() if rows_too else NONE),
                                  *(c.args() if cols_too else NONE), _stream()))
        torch.cuda.synchronize()
        if rows_too:
            _same(r.get(), want)
        if cols_too:
            _same(c.get(), want_t)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad", [0, 16])
def test_quantize_tile_bitexact(rows, cols, pad):
    X = xs()
    x = _x(rows, cols + pad, rows * 3 + cols)
    dx = dev_bits(x)
    want = fp8.quantize(bits_f64(x[:, :cols]), B)
    want_t = fp8.quantize(bits_f64(x[:, :cols]).T, B)
    for rows_too, cols_too in ((True, False), (False, True), (True, True)):
        r, c = Codes(rows, cols, B, pad, pad // 4), Codes(cols, rows, B, pad, pad // 4)
        X.check(X.xs_quantize_fp8_tile(dx.data_ptr(), rows, cols, cols + pad, *(r.args() if rows_too else NONE),
                                       *(c.args() if cols_too else NONE), _stream()))
        torch.cuda.synchronize()
        if rows_too:
            _same(r.get(), want)
        if cols_too:
            _same(c.get(), want_t)


def test_quotients_are_the_rounded_divisions():
    # every positive bf16 value from 1 to 448 against the scales of 384 maxima: the quotient of two fp32
    # numbers rounds as a division does at every mantissa
    X = xs()
    vals = np.arange(0x3F80, 0x4400, dtype=np.uint16)
    vals = np.resize(vals, _up(len(vals), 127))
    rows = []
    for m in range(384):
        amax = np.uint16(0x4380 + m)                            # 256 and up: every mantissa, three exponents
        for part in vals.reshape(-1, 127)[m % 9::9]:
            rows.append(np.concatenate([[amax], part]))
    x = np.stack(rows).astype(np.uint16)
    dx, r = dev_bits(x), Codes(x.shape[0], 128)
    X.check(X.xs_quantize_fp8(dx.data_ptr(), x.shape[0], 128, 128, *r.args(), *NONE, _stream()))
    torch.cuda.synchronize()
    _same(r.get(), fp8.quantize(bits_f64(x)))


def test_blocks_without_a_finite_maximum_poison_their_products_only():
    X = xs()
    x = _x(200, 256, 5, special=False)
    x[3, 7], x[9, 130], x[150, 200] = 0x7F80, 0x7FC1, 0xFF80     # inf, NaN, -inf
    dx = dev_bits(x)
    with np.errstate(invalid="ignore"):
        v = bits_f64(x)
    for fn, down in ((X.xs_quantize_fp8, 1), (X.xs_quantize_fp8_tile, B)):
        r, c = Codes(200, 256, down), Codes(256, 200, down)
        X.check(fn(dx.data_ptr(), 200, 256, 256, *r.args(), *c.args(), _stream()))
        torch.cuda.synchronize()
        _same(r.get(), fp8.quantize(v, down))
        _same(c.get(), fp8.quantize(v.T, down))
    r, w = Codes(200, 256), Codes(16, 256, B)
    X.check(X.xs_quantize_fp8(dx.data_ptr(), 200, 256, 256, *r.args(), *NONE, _stream()))
    dw = dev_bits(_x(16, 256, 6, special=False))
    X.check(X.xs_quantize_fp8_tile(dw.data_ptr(), 16, 256, 256, *w.args(), *NONE, _stream()))
    out = torch.zeros((200, 16), dtype=torch.int16, device="cuda")
    _gemm(r, w, X.XS_BLOCK_TILE, out, 200, 16, 256)
    nan = np.isnan(bits_f64(host_bits(out)))
    assert nan[[3, 9, 150]].all() and nan.sum() == 3 * 16


def _gemm(a, b, block, out, M, N, K, ldc=None):
    X = xs()
    ct = X.XS_TYPE_F32 if out.dtype == torch.float32 else X.XS_TYPE_BF16
    X.check(X.xs_gemm_fp8(*a.args(), *b.args(), block, out.data_ptr(), out.stride(0), ct, M, N, K, _stream()))
    torch.cuda.synchronize()


def _operand(rows, K, seed, down, pad=0, std=1.0, spad=0):
    """Random codes over the whole range and scales over several binades, on the device and as values."""
    g = np.random.default_rng(seed)
    c = Codes(rows, K, down, pad, spad)
    v = (g.standard_normal((rows, K)) * 60).clip(-448, 448)
    codes = mx.encode(v, mx.E4M3)
    scales = (std * np.exp(g.uniform(-3, 3, (c.srows, K // B)))).astype(np.float32)
    c.codes[:rows, :K] = torch.from_numpy(codes).cuda()
    c.codes[:, K:] = 0x7F                                        # NaN codes between rows are not read
    c.codes[rows] = 0x7F
    c.scales[:] = float("nan")
    c.scales[:c.srows, :K // B] = torch.from_numpy(scales).cuda()
    return c, fp8.values(codes, scales, down)


def _check_product(got, A, W, half, what):
    want = A @ W.T
    bound = fp8.product_bound(A, W, half < 2.0 ** -20)
    err = np.abs(got - want) - half * (np.abs(want) + bound) - bound
    assert np.isfinite(got).all() and err.max() <= 0, f"{what}: off by {np.abs(got - want).max():.3e} at {np.unravel_index(err.argmax(), err.shape)}"


GEMMS = [(1, 8, 128), (1, 256, 512), (7, 1000, 896), (24, 4096, 7168), (16, 136, 1280), (17, 264, 640), (33, 2048, 1024), (64, 256, 128),
         (65, 520, 2176), (100, 64, 3968), (128, 128, 384), (129, 136, 256), (200, 1536, 1152), (256, 256, 128), (257, 264, 1408),
         (300, 4096, 512), (513, 1024, 640), (1000, 1288, 256), (2, 7168, 2048), (48, 7168, 256), (700, 7168, 128)]


@pytest.mark.parametrize("M,N,K", GEMMS)
@pytest.mark.parametrize("block", ["tile", "row"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gemm(M, N, K, block, out):
    X = xs()
    a, A = _operand(M, K, M + N, 1, pad=16 * (M % 3), std=0.01)
    b, W = _operand(N, K, N + K, 1 if block == "row" else B, pad=32 * (N % 2), spad=4 * (M % 2), std=0.02)
    ldc = N + 8 * (M % 2)
    c = torch.full((M + 1, ldc), -1.0, dtype=torch.float32, device="cuda") if out == "f32" else \
        torch.full((M + 1, ldc), -1, dtype=torch.int16, device="cuda")
    _gemm(a, b, X.XS_BLOCK_ROW if block == "row" else X.XS_BLOCK_TILE, c, M, N, K)
    assert (c[M] == -1).all() and (c[:, N:] == -1).all()
    got = c[:M, :N].cpu().double().numpy() if out == "f32" else bits_f64(host_bits(c[:M, :N].contiguous()))
    _check_product(got, A, W, 2.0 ** -24 if out == "f32" else 2.0 ** -8, f"{M}x{N}x{K} {block} {out}")
    first = c.clone()
    _gemm(a, b, X.XS_BLOCK_ROW if block == "row" else X.XS_BLOCK_TILE, c, M, N, K)
    assert torch.equal(first, c)                                 # a fixed order of sums


@pytest.mark.parametrize("block", ["tile", "row"])
@pytest.mark.parametrize("M,N,K", [(5, 264, 768), (40, 512, 1024), (300, 520, 640), (600, 1032, 512)])
def test_gemm_of_integers_is_exact(M, N, K, block):
    # small integers and powers of two as scales: every sum below 2^24 units, so each order of additions
    # gives the same fp32 number
    X = xs()
    g = np.random.default_rng(M)
    down = 1 if block == "row" else B
    a, b = Codes(M, K), Codes(N, K, down)
    vals, mats = [], []
    for c, d in ((a, 1), (b, down)):
        codes = mx.encode(g.integers(-8, 9, (c.rows, K)).astype(np.float64), mx.E4M3)
        scales = (2.0 ** g.integers(-2, 3, (c.srows, K // B))).astype(np.float32)
        c.codes[:c.rows, :K] = torch.from_numpy(codes).cuda()
        c.scales[:c.srows, :K // B] = torch.from_numpy(scales).cuda()
        mats.append(fp8.values(codes, scales, d))
    c = torch.zeros((M, N), device="cuda")
    _gemm(a, b, X.XS_BLOCK_ROW if block == "row" else X.XS_BLOCK_TILE, c, M, N, K)
    assert np.array_equal(c.cpu().double().numpy(), mats[0] @ mats[1].T)


SEGMENTS = [
    [5], [0, 3, 0, 1], [16, 17, 0, 31, 1], [128, 1, 300, 0, 127], [1] * 40, [0, 0, 0], [257, 513], [40] * 9 + [0] * 60 + [3],
    [64, 65, 63, 0, 2], [100, 0, 200, 150], [700, 1]]


@pytest.mark.parametrize("rows", SEGMENTS, ids=lambda r: f"{len(r)}x{sum(r)}")
@pytest.mark.parametrize("N,K,epi", [(256, 128, "store"), (264, 384, "store"), (512, 640, "swiglu"), (768, 256, "swiglu"), (1024, 1152, "store")])
def test_grouped_gemm(rows, N, K, epi):
    X = xs()
    n = len(rows)
    g = np.random.default_rng(sum(rows) + N)
    gaps = g.integers(0, 4, n + 1)                               # rows between and behind the segments
    offs = np.cumsum(gaps[:-1]) + np.concatenate([[0], np.cumsum(rows)[:-1]])
    M = int(offs[-1] + rows[-1] + gaps[-1]) + 1
    order = g.permutation(n)                                     # segments in any order
    offs, lens = offs[order], np.array(rows)[order]
    a, A = _operand(M, K, 3, 1, pad=16, std=0.01)
    tiles = -(-N // B)
    codes, scales, W = [], [], []
    for s in range(n):
        b, w = _operand(N, K, 100 + s, B, std=0.02)
        codes.append(b.codes[:N, :K].contiguous())
        scales.append(b.scales[:tiles])
        W.append(w)
    bc, bs = torch.stack(codes), torch.stack(scales)
    n_out = N // 2 if epi == "swiglu" else N
    c = torch.full((M, n_out + 8), -1, dtype=torch.int16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    do, dr = torch.from_numpy(offs.astype(np.int32)).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda()
    X.check(X.xs_grouped_gemm_fp8(*a.args(), M, do.data_ptr(), dr.data_ptr(), n, bc.data_ptr(), bs.data_ptr(), bs.shape[2], N, K,
                                  c.data_ptr(), c.stride(0), X.XS_EPI_SWIGLU if epi == "swiglu" else X.XS_EPI_STORE, st.data_ptr(),
                                  _stream()))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    bits = host_bits(c)
    outside = np.ones(M, bool)
    for s in range(n):
        o, r = offs[s], lens[s]
        outside[o:o + r] = False
        if r == 0:
            continue
        got = bits_f64(np.ascontiguousarray(bits[o:o + r, :n_out]))
        if epi == "store":
            _check_product(got, A[o:o + r], W[s], 2.0 ** -8, f"segment {s}")
        else:
            gu, bound = A[o:o + r] @ W[s].T, fp8.product_bound(A[o:o + r], W[s], False)
            want = fp8.swiglu(gu)
            gate, up = np.split(gu, 2, 1)
            bg, bu = np.split(bound, 2, 1)
            # silu' is at most 1.1; the activation's own roundings, exponential and reciprocal: 2^-20 (1 + |gate|)
            tol = 1.1 * bg * np.abs(up) + np.abs(fp8.silu(gate)) * bu + 1.1 * bg * bu + 2.0 ** -20 * (1 + np.abs(gate)) * np.abs(want)
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + tol) + tol), s
    assert (bits[outside] == 0xFFFF).all() and (bits[:, n_out:] == 0xFFFF).all()


def test_grouped_gemm_skips_bad_segments():
    X = xs()
    M, N, K = 50, 256, 256
    a, A = _operand(M, K, 3, 1)
    b, W = _operand(N, K, 4, B)
    bc, bs = b.codes[:N].contiguous().repeat(4, 1), b.scales[:2].repeat(4, 1).contiguous()
    for offs, lens in (([0, 10, 45, 20], [5, -1, 6, 9]), ([0, -1, 60, 20], [5, 3, 1, 9])):
        c = torch.full((M, N), -1, dtype=torch.int16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        do, dr = torch.tensor(offs, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
        X.check(X.xs_grouped_gemm_fp8(*a.args(), M, do.data_ptr(), dr.data_ptr(), 4, bc.data_ptr(), bs.data_ptr(), bs.shape[1], N, K,
                                      c.data_ptr(), N, X.XS_EPI_STORE, st.data_ptr(), _stream()))
        torch.cuda.synchronize()
        assert int(st.item()) == X.XS_EBADINPUT
        bits = host_bits(c)
        for o, r in ((0, 5), (20, 9)):
            _check_product(bits_f64(bits[o:o + r]), A[o:o + r], W, 2.0 ** -8, "segment")
        assert (np.delete(bits, np.r_[0:5, 20:29], 0) == 0xFFFF).all()


def _swiglu_inputs(rows, I, pad, seed):
    g = np.random.default_rng(seed)
    gu = (g.standard_normal((rows, 2 * I + pad)) * np.exp(g.uniform(-2, 2, (rows, 1)))).astype(np.float32)
    if rows > 4:
        gu[1] = 0.0
        gu[2, :I] = 100.0 * np.sign(g.standard_normal(I))
        gu[3] = 1e-20
    return synth.to_bf16_bits(gu)


@pytest.mark.parametrize("rows,I,pad", [(1, 128, 0), (5, 384, 8), (37, 2048, 0), (130, 512, 16)])
def test_swiglu_and_its_checkpoint(rows, I, pad):
    X = xs()
    gu = _swiglu_inputs(rows, I, pad, rows)
    dgu = dev_bits(gu)
    v = bits_f64(np.ascontiguousarray(gu[:, :2 * I]))
    want = fp8.swiglu(v)
    for keep in (True, False):
        h, ck = Codes(rows, I, pad=16), Codes(rows, 2 * I, spad=4)
        X.check(X.xs_swiglu_fp8(dgu.data_ptr(), 2 * I + pad, rows, I, *h.args(), *(ck.args() if keep else NONE), _stream()))
        torch.cuda.synchronize()
        codes, scales = h.get()
        # h in fp32 is off by 2^-20 (1 + |gate|) (exponential, reciprocal, three products), so is a scale;
        # a code by half a step: 2^-4 of the value, or of the smallest normal's binade
        rel = 2.0 ** -20 * (1 + np.abs(v[:, :I]))
        amax = np.abs(want).reshape(rows, -1, B).max(-1)
        loose = rel.reshape(rows, -1, B).max(-1)
        s64 = np.maximum(amax, 2.0 ** -60) / 448
        assert np.all(np.abs(scales - s64) <= (loose + 2.0 ** -23) * s64)
        got = fp8.values(codes, scales)
        step = np.maximum(2.0 ** -4 * np.abs(want), np.repeat(scales.astype(np.float64), B, 1) * 2.0 ** -10)
        assert np.all(np.abs(got - want) <= step * (1 + rel) + (rel + np.repeat(loose, B, 1)) * np.abs(want))
        if keep:
            _same(ck.get(), fp8.quantize(v))


@pytest.mark.parametrize("rows,I,pad", [(1, 128, 0), (5, 384, 8), (37, 2048, 0), (130, 512, 16)])
def test_swiglu_gradient_from_the_checkpoint(rows, I, pad):
    X = xs()
    ck_bits = _swiglu_inputs(rows, I, 0, rows + 1)
    codes, scales = fp8.quantize(bits_f64(ck_bits))
    ck = Codes(rows, 2 * I, pad=16, spad=4)
    ck.codes[:rows, :2 * I] = torch.from_numpy(codes).cuda()
    ck.scales[:rows, :2 * I // B] = torch.from_numpy(scales).cuda()
    dh = synth.normal_bf16(0, rows, (rows, I + pad), std=1e-3)
    d, hv, mag = fp8.swiglu_backward(fp8.values(codes, scales), bits_f64(np.ascontiguousarray(dh[:, :I])))
    ddh = dev_bits(dh)
    for keep in (True, False):
        out = torch.full((rows + 1, 2 * I + pad), -1, dtype=torch.int16, device="cuda")
        h = torch.full((rows + 1, I + pad), -1, dtype=torch.int16, device="cuda")
        X.check(X.xs_swiglu_fp8_backward(*ck.args(), ddh.data_ptr(), I + pad, rows, I, out.data_ptr(), 2 * I + pad,
                                         h.data_ptr() if keep else None, I + pad if keep else 0, _stream()))
        torch.cuda.synchronize()
        ob, hb = host_bits(out), host_bits(h)
        assert (ob[rows] == 0xFFFF).all() and (ob[:, 2 * I:] == 0xFFFF).all() and (hb[rows] == 0xFFFF).all()
        gate = np.abs(fp8.values(codes, scales)[:, :I])
        loose = 2.0 ** -20 * (1 + gate)                          # the sigmoid's argument and reciprocal, the products
        err = np.abs(bits_f64(ob[:rows, :2 * I]) - d)
        # bf16 halves its step at 2^-133: results below its normal range count as absolute 2^-133
        assert np.all(err <= 2.0 ** -8 * np.abs(d) + np.concatenate([loose, loose], 1) * mag + 2.0 ** -126)
        if keep:
            assert np.all(np.abs(bits_f64(hb[:rows, :I]) - hv) <= (2.0 ** -8 + loose) * np.abs(hv) + 2.0 ** -126)
        else:
            assert (hb == 0xFFFF).all()


def test_swiglu_gradient_is_the_differences():
    # SwiGLU of checkpoint values g +- h in fp64 against the kernel's gradient: bf16 halves (2^-8 of the
    # value), the difference's own h^2 term
    X = xs()
    rows, I, h = 3, 128, 1e-4
    codes, scales = fp8.quantize(bits_f64(synth.normal_bf16(1, 2, (rows, 2 * I))))
    v = fp8.values(codes, scales)
    ck = Codes(rows, 2 * I)
    ck.codes[:rows] = torch.from_numpy(codes).cuda()
    ck.scales[:rows, :2] = torch.from_numpy(scales).cuda()
    dh = synth.normal_bf16(1, 3, (rows, I))
    out, ddh = torch.zeros((rows, 2 * I), dtype=torch.int16, device="cuda"), dev_bits(dh)
    X.check(X.xs_swiglu_fp8_backward(*ck.args(), ddh.data_ptr(), I, rows, I, out.data_ptr(), 2 * I, None, 0, _stream()))
    torch.cuda.synchronize()
    got = bits_f64(host_bits(out))
    for part in (0, 1):
        step = np.zeros_like(v)
        step[:, part * I:(part + 1) * I] = h
        want = (fp8.swiglu(v + step) - fp8.swiglu(v - step)) * bits_f64(dh) / (2 * h)
        g = got[:, part * I:(part + 1) * I]
        assert np.all(np.abs(g - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * (1 + np.abs(v).max()) ** 2 + 10 * h * h)


def test_a_weights_gradient_in_a_graph_and_on_another_stream():
    # dW = dY^T X over 300 tokens: both operands quantized along the tokens (transposed), an fp32 product
    X = xs()
    T, K, N = 300, 256, 136
    x, dy = synth.normal_bf16(2, 0, (T, K)), synth.normal_bf16(2, 1, (T, N), std=1e-3)
    dx, ddy = dev_bits(x), dev_bits(dy)
    xt, yt = Codes(K, T), Codes(N, T)
    dw = torch.zeros((N, K), device="cuda")

    def step(s):
        X.check(X.xs_quantize_fp8(dx.data_ptr(), T, K, K, *NONE, *xt.args(), s))
        X.check(X.xs_quantize_fp8(ddy.data_ptr(), T, N, N, *NONE, *yt.args(), s))
        X.check(X.xs_gemm_fp8(*yt.args(), *xt.args(), X.XS_BLOCK_ROW, dw.data_ptr(), K, X.XS_TYPE_F32, N, K, xt.K, s))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(side.cuda_stream)
    torch.cuda.synchronize()
    first = dw.clone()
    A, W = (fp8.values(*fp8.quantize(bits_f64(v).T)) for v in (dy, x))
    _check_product(first.cpu().double().numpy(), A, W, 2.0 ** -24, "dW")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        dw.zero_()
        xt.codes.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, first)


def test_more_columns_than_a_grid_of_the_split_form_has():
    """2^28 + 8 columns: sixteen of them to a workgroup of 256 threads would be more threads than a grid's
    dimension has. Repeating rows of b give repeating columns of c."""
    N, K, n = (1 << 28) + 8, 128, 1 << 20
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    X = xs()
    g = torch.Generator(device="cuda").manual_seed(3)
    base = (torch.randint(0, 2, (n, K), device="cuda", generator=g) * 0x38).to(torch.uint8)        # 0 or 1
    b = torch.empty((N, K), dtype=torch.uint8, device="cuda")
    b[:1 << 28].view(-1, n, K).copy_(base)
    b[1 << 28:] = base[:8]
    sb = torch.ones((N // 128 + 1, 4), device="cuda")
    a, sa = torch.full((1, K), 0x38, dtype=torch.uint8, device="cuda"), torch.full((1, 4), 0.5, device="cuda")
    c = torch.full((1, N), -7.0, dtype=torch.bfloat16, device="cuda")
    X.check(X.xs_gemm_fp8(a.data_ptr(), K, sa.data_ptr(), 4, b.data_ptr(), K, sb.data_ptr(), 4, X.XS_BLOCK_TILE, c.data_ptr(), N,
                          X.XS_TYPE_BF16, 1, N, K, _stream()))
    want = ((base != 0).sum(1).float() * 0.5).to(torch.bfloat16)                                 # at most 64: exact
    assert torch.equal(c[0, :1 << 28].view(-1, n), want.expand(1 << 8, n)) and torch.equal(c[0, 1 << 28:], want[:8])
    del a, b, c, sb, base
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,N,blocks", [(384, 4096, 1), (391, 4088, 2), (450, 4096, 3), (333, 4104, 5), (401, 4096, 8), (500, 2048, 18),
                                        (700, 4096, 2), (769, 4088, 3), (900, 4096, 4), (1000, 3976, 5), (1024, 4096, 9), (257, 7168, 11)])
@pytest.mark.parametrize("block", ["tile", "row"])
def test_gemm_of_about_a_tile_to_a_cu(M, N, blocks, block):
    """Fewer blocks of K than stages, as many, more; whole and ragged last tiles."""
    test_gemm(M, N, blocks * B, block, "bf16")


@pytest.mark.parametrize("spans,N,K", [
    ([(0, 100), (0, 100), (100, 100)], 256, 256),                            # more row blocks than M and n_seg alone ask for
    ([(0, 700)] * 5 + [(700, 100)], 256, 384),
    ([(0, 50)] * 70 + [(50, 33), (10, 60), (0, 83)], 512, 256),              # past the 64 segments of one scan, tiles
    ([(0, 3000), (0, 3000), (3000, 500)], 1024, 128),                        # tiles
    ([(5, 1)] * 40 + [(6, 300)], 512, 1152),
    ([(0, 20)] * 100 + [(20, 30)], 256, 128)])                               # past one scan in a split form, two tiles a workgroup
@pytest.mark.parametrize("epi", ["store", "swiglu"])
def test_overlapping_segments_compute_all_their_rows(spans, N, K, epi):
    """Segments race on their common rows only: an element there is that of one of them, and every other row is its
    segment's. Small integers and power-of-two scales: the 8-bit products are exact (test_gemm_of_integers_is_exact)."""
    X = xs()
    M, n = max(o + r for o, r in spans) + 3, len(spans)
    g = np.random.default_rng(M + n)
    a = Codes(M, K)
    vals = g.integers(-4, 5, (M, K)).astype(np.float64)
    a.codes[:M, :K] = torch.from_numpy(mx.encode(vals, mx.E4M3)).cuda()
    a.scales[:M, :K // B] = 0.125
    w = g.integers(-2, 3, (n, N, K)).astype(np.float64)
    bc = torch.from_numpy(mx.encode(w, mx.E4M3)).cuda()
    bs = torch.full((n, -(-N // B), _up(K // B, 4)), 0.25, device="cuda")
    n_out = N // 2 if epi == "swiglu" else N
    c = torch.full((M, n_out), -1, dtype=torch.int16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    do, dr = (torch.tensor([s[i] for s in spans], dtype=torch.int32, device="cuda") for i in (0, 1))
    X.check(X.xs_grouped_gemm_fp8(*a.args(), M, do.data_ptr(), dr.data_ptr(), n, bc.data_ptr(), bs.data_ptr(), bs.shape[2], N, K,
                                  c.data_ptr(), n_out, X.XS_EPI_SWIGLU if epi == "swiglu" else X.XS_EPI_STORE, st.data_ptr(), _stream()))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    bits = host_bits(c)
    got, fits, covered = bits_f64(bits), np.zeros((M, n_out), bool), np.zeros(M, bool)
    for s, (o, r) in enumerate(spans):
        p = vals[o:o + r] @ w[s].T / 32
        want = fp8.swiglu(p) if epi == "swiglu" else p
        tol = 2.0 ** -8 * np.abs(want)
        if epi == "swiglu":                                        # exponential, reciprocal, products: as in test_grouped_gemm
            tol = tol + 2.0 ** -19 * (1 + np.abs(p[:, :n_out])) * np.abs(want)
        fits[o:o + r] |= np.abs(got[o:o + r] - want) <= tol
        covered[o:o + r] = True
    assert fits[covered].all() and (bits[~covered] == 0xFFFF).all()


# Sizes for the forms that the tables above do not reach; which form takes each is checked in test_fp8_forms.py.
FORM_GEMMS = [(96, 1360, 384), (88, 1352, 1280), (33, 4096, 256), (60, 4088, 640), (100, 4096, 256), (190, 4096, 512), (120, 4104, 896)]
LARGE_GEMMS = [(4093, 4096, 128), (4093, 4096, 256), (4093, 4096, 384), (2300, 4104, 640), (8200, 4096, 256), (8300, 1032, 1152)]
LARGE_GROUPS = [([3000, 0, 1, 257, 2500, 700, 129, 5], 4096, 128), ([3000, 0, 1, 257, 2500, 700, 129, 5], 4096, 384),
                ([2600, 1, 255, 256, 3100], 4096, 640), ([0, 3000, 0], 4096, 1152), ([900, 30, 512, 1], 2048, 512),
                ([700, 300, 0, 129, 400], 2048, 640), ([1200, 7, 300], 2048, 1152), ([0, 2100, 1100], 1280, 256),
                ([350, 1, 260, 90], 2048, 1408), ([30, 32, 28], 256, 1024), ([60, 40, 30], 1280, 768), ([35, 20, 14], 3584, 512)]


@pytest.mark.parametrize("M,N,K", FORM_GEMMS)
@pytest.mark.parametrize("block", ["tile", "row"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gemm_of_every_split_form(M, N, K, block, out):
    test_gemm(M, N, K, block, out)


def _integers(rows, K, seed, down, top, low):
    """Integer codes up to `top` under scales 2^low .. 2^(low + 2): every sum of products with its like below 2^24 units, so
    exact in fp32 in any order; products of at most 2^5 lose nothing in the 8-bit unit. Returns device operand, fp32 values."""
    g = np.random.default_rng(seed)
    c = Codes(rows, K, down)
    codes = mx.encode(g.integers(-top, top + 1, (rows, K)).astype(np.float64), mx.E4M3)
    scales = (2.0 ** g.integers(low, low + 3, (c.srows, K // B))).astype(np.float32)
    c.codes[:rows, :K] = torch.from_numpy(codes).cuda()
    c.scales[:c.srows, :K // B] = torch.from_numpy(scales).cuda()
    return c, fp8.values(codes, scales, down).astype(np.float32)


@pytest.mark.parametrize("M,N,K", LARGE_GEMMS)
@pytest.mark.parametrize("block", ["tile", "row"])
def test_gemm_in_large_tiles(M, N, K, block):
    """Every element of exact products, and rows at tiles' edges and elsewhere of random ones, where a persistent
    workgroup takes one tile or several."""
    X = xs()
    down, kind = (1, X.XS_BLOCK_ROW) if block == "row" else (B, X.XS_BLOCK_TILE)
    a, A = _integers(M, K, M, 1, 8, -4)
    b, W = _integers(N, K, N + 1, down, 4, -2)
    c = torch.full((M + 1, N + 8), -1, dtype=torch.int16, device="cuda")
    _gemm(a, b, kind, c, M, N, K)
    bits = host_bits(c)
    assert (bits[M] == 0xFFFF).all() and (bits[:, N:] == 0xFFFF).all()
    got = (bits[:M, :N].astype(np.uint32) << 16).view(np.float32)
    assert np.array_equal(got, (synth.to_bf16_bits(A @ W.T).astype(np.uint32) << 16).view(np.float32))
    del a, b, A, W
    a, A = _operand(M, K, M + N, 1, pad=16, std=0.01)
    b, W = _operand(N, K, N + K, down, pad=32, spad=4, std=0.02)
    _gemm(a, b, kind, c, M, N, K)
    rows = np.unique(np.r_[0:2, 126:130, 254:258, 2046:2050, M - 258:M - 254, M - 2:M, np.random.default_rng(1).integers(0, M, 48)])
    _check_product(bits_f64(host_bits(c)[rows, :N]), A[rows], W, 2.0 ** -8, f"{M}x{N}x{K} {block}")


def large_layout(rows):
    """Segments with a row between and behind each: offsets and the rows in all."""
    return np.cumsum([0] + [r + 1 for r in rows[:-1]]), sum(rows) + len(rows)


@pytest.mark.parametrize("rows,N,K", LARGE_GROUPS, ids=lambda v: f"{len(v)}x{sum(v)}" if isinstance(v, list) else str(v))
@pytest.mark.parametrize("epi", ["store", "swiglu"])
def test_grouped_gemm_of_thousands_of_rows(rows, N, K, epi):
    """Every element: exact products (SwiGLU: of exact gate and up values), empty segments, more tiles than workgroups."""
    X = xs()
    offs, M = large_layout(rows)
    n = len(rows)
    a, A = _integers(M, K, M, 1, 4, -4)
    bs_, W = zip(*(_integers(N, K, 50 + s, B, 2, -2) for s in range(n)))
    bc, bs = torch.stack([b.codes[:N] for b in bs_]), torch.stack([b.scales[:-(-N // B)] for b in bs_])
    n_out = N // 2 if epi == "swiglu" else N
    c = torch.full((M, n_out + 8), -1, dtype=torch.int16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    do, dr = (torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda") for v in (offs, rows))
    X.check(X.xs_grouped_gemm_fp8(*a.args(), M, do.data_ptr(), dr.data_ptr(), n, bc.data_ptr(), bs.data_ptr(), bs.shape[2], N, K,
                                  c.data_ptr(), n_out + 8, X.XS_EPI_SWIGLU if epi == "swiglu" else X.XS_EPI_STORE, st.data_ptr(), _stream()))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    bits, outside = host_bits(c), np.ones(M, bool)
    for s, (o, r) in enumerate(zip(offs, rows)):
        outside[o:o + r] = False
        got, gu = (np.ascontiguousarray(bits[o:o + r, :n_out]).astype(np.uint32) << 16).view(np.float32), A[o:o + r] @ W[s].T
        if epi == "store":
            assert np.array_equal(got, (synth.to_bf16_bits(gu).astype(np.uint32) << 16).view(np.float32)), s
        else:
            # the activation's exponential, reciprocal and products, 2^-20 (1 + |gate|), and one rounding. A sigmoid below
            # 2^-126 (gates below -87.3, -126 log 2, and here they go to -125) is no normal fp32 number: the reciprocal of
            # more than 2^126, or of an exponential past fp32's range, is 0, off by at most 2^-126 times |gate up|
            want, (gate, up) = fp8.swiglu(gu), np.abs(gu.astype(np.float64)).reshape(r, 2, n_out).transpose(1, 0, 2)
            tol = 2.0 ** -20 * (1 + gate) * np.abs(want) + 2.0 ** -126 * gate * up
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + tol) + tol + 2.0 ** -126), s
    assert (bits[outside] == 0xFFFF).all() and (bits[:, n_out:] == 0xFFFF).all()
