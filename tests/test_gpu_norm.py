"""GPU parity of the RMS norm and its gradients against the fp64 oracle.

h is exact (one fp32 sum of two bf16 values, one rounding). y: the row's sum of squares passes at most 128 + 17
fp32 additions of positive terms (a lane's 32 values at 1024 threads, then the wave's and the workgroup's) and half that
error reaches the root, with a division, a root, a quotient and two products: below (80 + 5) 2^-24 < 2^-17; one rounding to bf16
(2^-8). E4M3: the scale is off by as much relative to the largest value, a code by half a step of the format
(2^-4 relative, 2^-10 absolute below the normal range) around a quotient off by 2^-16.
Gradient: dx = i (g - u c): the two row sums are off by (128 + 17) 2^-24 of their terms' magnitudes, i by 2^-17: below
2^-15 of the terms in all, one rounding. dw: a column's fp32 sum over the rows."""
import numpy as np
import pytest
import torch

from gpu_helpers import require_gpu, xs
from oracle import fp8, mx, norm

pytestmark = pytest.mark.gpu

S = -7.0
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _rand(rows, cols, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, cols), generator=g) * std * torch.exp(torch.randn((rows, 1), generator=g))).bfloat16()


def _wide(x, pad):
    """On the GPU with rows cols + pad apart, NaN between."""
    full = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device="cuda")
    full[:, :x.shape[1]] = x
    return full


def _weight(cols, kind, seed=9):
    w = 1 + 0.2 * torch.randn(cols, generator=torch.Generator().manual_seed(seed))
    return w.bfloat16() if kind == "bf16" else w


SHAPES = [(1, 8), (5, 8), (3, 120), (4, 136), (7, 512), (6, 520), (5, 1024), (9, 1032), (3, 2048), (3, 2056), (2, 4096), (5, 4104), (3, 6144), (2, 6152),
          (4, 7168), (3, 8192), (2, 8200), (2, 16384), (2, 16392), (1, 32768), (515, 256), (300, 3080)] + [
          # more rows than CUs: the forms of many rows, each width of theirs
          (257, 1000), (263, 2040), (258, 6000), (257, 8192), (259, 16384), (258, 20000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("residual,kind,pad", [(True, "bf16", 0), (False, "f32", 8), (True, "f32", 24)])
def test_norm(rows, cols, residual, kind, pad):
    X = xs()
    x, r, w = _rand(rows, cols, cols), _rand(rows, cols, cols + 1) if residual else None, _weight(cols, kind)
    h64 = norm.stream(x.double().numpy(), r.double().numpy() if residual else None)
    y64 = norm.norm(h64, w.double().numpy(), EPS)
    dx, dr, dw = _wide(x, pad), _wide(r, pad) if residual else None, w.cuda()
    blocks = -(-cols // 128)
    new = lambda shape, dt: torch.full(shape, 1, dtype=dt, device="cuda")
    for want_h, want_y, want_c in ((True, True, True), (False, True, False), (False, False, True)):
        h, y = _wide(torch.full((rows + 1, cols), S, dtype=torch.bfloat16), pad), _wide(torch.full((rows + 1, cols), S, dtype=torch.bfloat16), 2 * pad)
        codes, scales = new((rows + 1, blocks * 128 + 16), torch.uint8), torch.full((rows + 1, -(-blocks // 4) * 4 + 4), S, device="cuda")
        X.check(X.xs_rmsnorm(dx.data_ptr(), dx.stride(0), X.ptr(dr), dx.stride(0), dw.data_ptr(), X.XS_TYPE_BF16 if kind == "bf16" else X.XS_TYPE_F32,
                             EPS, rows, cols, h.data_ptr() if want_h else None, h.stride(0), y.data_ptr() if want_y else None, y.stride(0),
                             codes.data_ptr() if want_c else None, codes.stride(0), scales.data_ptr() if want_c else None, scales.stride(0), _stream()))
        torch.cuda.synchronize()
        if want_h:
            assert np.array_equal(h[:rows, :cols].cpu().double().numpy(), h64) and (h[rows, :cols] == S).all()
        if want_y:
            got = y[:rows, :cols].cpu().double().numpy()
            assert np.all(np.abs(got - y64) <= (2.0 ** -8 + 2.0 ** -17) * np.abs(y64)) and (y[rows, :cols] == S).all()
            if pad:
                assert torch.isnan(y[:, cols:]).all()
        if want_c:
            c, s = codes[:rows, :blocks * 128].cpu().numpy(), scales[:rows, :blocks].cpu().double().numpy()
            assert (codes[rows] == 1).all() and (codes[:, blocks * 128:] == 1).all() and (scales[rows] == S).all() and (scales[:, blocks:] == S).all()
            full = np.zeros((rows, blocks * 128))
            full[:, :cols] = y64
            amax = np.maximum(np.abs(full.reshape(rows, blocks, 128)).max(2), 2.0 ** -60) / 448
            assert np.all(np.abs(s - amax) <= 2.0 ** -16 * amax)
            got, step = mx.decode(c, mx.E4M3), np.repeat(s, 128, 1)
            q = full / step
            assert np.all(np.abs(got - q) <= np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + 2.0 ** -15 * np.abs(q))
            assert (c[:, cols:] == 0).all()


def test_codes_are_the_quantizer_s_of_values_that_bf16_holds():
    # rows of +-1 and weights of powers of two: y is a power of two, i is off by less than bf16 sees
    X = xs()
    rows, cols = 6, 384
    x = torch.sign(torch.randn((rows, cols), generator=torch.Generator().manual_seed(0))).bfloat16().cuda()
    w = torch.pow(2.0, torch.randint(-6, 6, (cols,), generator=torch.Generator().manual_seed(1)).float()).cuda()
    codes, scales = torch.zeros((rows, cols), dtype=torch.uint8, device="cuda"), torch.zeros((rows, 4), device="cuda")
    X.check(X.xs_rmsnorm(x.data_ptr(), cols, None, 0, w.data_ptr(), X.XS_TYPE_F32, 0.0, rows, cols, None, 0, None, 0, codes.data_ptr(), cols,
                         scales.data_ptr(), 4, _stream()))
    want, ws = fp8.quantize((x.cpu().double() * w.cpu().double()).numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy()[:, :3], ws)


@pytest.mark.parametrize("rows,cols", SHAPES + [(2000, 128)])
@pytest.mark.parametrize("extra,kind,pad", [(True, "bf16", 0), (False, "f32", 8)])
def test_gradient(rows, cols, extra, kind, pad):
    X = xs()
    h, dy, w = _rand(rows, cols, 1), _rand(rows, cols, 2, 1e-2), _weight(cols, kind)
    dh = _rand(rows, cols, 3, 1e-2) if extra else None
    want, want_w, mag, mag_w = norm.backward(h.double().numpy(), w.double().numpy(), dy.double().numpy(), EPS, dh.double().numpy() if extra else None)
    a, b, c, wd = _wide(h, pad), _wide(dy, pad), _wide(dh, pad) if extra else None, w.cuda()
    ws = X.workspace(X.xs_rmsnorm_backward_workspace_bytes, rows, cols)
    ws.fill_(255)
    dx, dw = _wide(torch.full((rows + 1, cols), S, dtype=torch.bfloat16), pad), torch.full((cols + 4,), S, device="cuda")

    def call(out, weight_grad, work, n):
        X.check(X.xs_rmsnorm_backward(b.data_ptr(), b.stride(0), X.ptr(c), b.stride(0), a.data_ptr(), a.stride(0), wd.data_ptr(),
                                      X.XS_TYPE_BF16 if kind == "bf16" else X.XS_TYPE_F32, EPS, rows, cols, out.data_ptr(), out.stride(0),
                                      X.ptr(weight_grad), work, n, _stream()))
        torch.cuda.synchronize()

    call(dx, dw, ws.data_ptr(), ws.numel())
    got = dx[:rows, :cols].cpu().double().numpy()
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * mag)
    assert (dx[rows, :cols] == S).all() and (dw[cols:] == S).all()
    assert np.all(np.abs(dw[:cols].cpu().double().numpy() - want_w) <= ((rows + 64) * 2.0 ** -24 + 2.0 ** -16) * mag_w)
    # without the weight's gradient and its workspace, and in the place of dy
    only = torch.zeros_like(dx)
    call(only, None, None, 0)
    assert torch.equal(only[:rows, :cols], dx[:rows, :cols])
    call(b, dw, ws.data_ptr(), ws.numel())
    assert torch.equal(b[:, :cols], dx[:rows, :cols])


# each width of the forms of few rows and of many
@pytest.mark.parametrize("rows,cols", [(33, 512), (33, 1024), (33, 7168), (33, 16384), (33, 20000), (300, 520), (300, 2048), (300, 3080), (300, 8192), (300, 9000),
                                       (257, 32768)])
@pytest.mark.parametrize("eps", [0.0, EPS])
def test_rows_whose_squares_leave_the_range_of_fp32(rows, cols, eps):
    """Rows of values around 2^-110 to 2^110, one large value among small ones, and rows beside them as ever: a row's mean square and its
    product with the gradient come from values times a power of two, which is exact. Tolerances as above."""
    X = xs()
    e = torch.tensor([0, 110, -110, 0, 56, 60, 63, 64, 90, -40, -50, -60, -64, -75, -100, 10])[torch.arange(rows) % 16]
    h = (_rand(rows, cols, 1).float() * torch.exp2(e.float())[:, None]).bfloat16()
    h[3], h[3, 5] = 2.0 ** -20, 2.0 ** 100
    dy, w = _rand(rows, cols, 2, 1e-2), _weight(cols, "f32")
    y64 = norm.norm(h.double().numpy(), w.double().numpy(), eps)
    hd, wd, gd = h.cuda(), w.cuda(), dy.cuda()
    blocks = -(-cols // 128)
    y = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.zeros((rows, blocks * 128), dtype=torch.uint8, device="cuda"), torch.zeros((rows, -(-blocks // 4) * 4), device="cuda")
    X.check(X.xs_rmsnorm(hd.data_ptr(), cols, None, 0, wd.data_ptr(), X.XS_TYPE_F32, eps, rows, cols, None, 0, y.data_ptr(), cols, codes.data_ptr(),
                         codes.stride(0), scales.data_ptr(), scales.stride(0), _stream()))
    torch.cuda.synchronize()
    # below the normal numbers of bf16 half a step is 2^-134
    assert np.all(np.abs(y.cpu().double().numpy() - y64) <= (2.0 ** -8 + 2.0 ** -17) * np.abs(y64) + 2.0 ** -133)
    full = np.zeros((rows, blocks * 128))
    full[:, :cols] = y64
    amax = np.maximum(np.abs(full.reshape(rows, blocks, 128)).max(2), 2.0 ** -60) / 448
    assert np.all(np.abs(scales[:, :blocks].cpu().double().numpy() - amax) <= 2.0 ** -16 * amax)
    want, want_w, mag, mag_w = norm.backward(h.double().numpy(), w.double().numpy(), dy.double().numpy(), eps)
    ws = X.workspace(X.xs_rmsnorm_backward_workspace_bytes, rows, cols)
    dx, dw = torch.zeros_like(y), torch.zeros(cols, device="cuda")
    X.check(X.xs_rmsnorm_backward(gd.data_ptr(), cols, None, 0, hd.data_ptr(), cols, wd.data_ptr(), X.XS_TYPE_F32, eps, rows, cols, dx.data_ptr(), cols,
                                  dw.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
    torch.cuda.synchronize()
    assert np.all(np.abs(dx.cpu().double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * mag + 2.0 ** -133)
    assert np.all(np.abs(dw.cpu().double().numpy() - want_w) <= ((rows + 64) * 2.0 ** -24 + 2.0 ** -16) * mag_w)


def test_in_place_and_no_rows():
    X = xs()
    rows, cols = 33, 1024
    x, r, w = _rand(rows, cols, 1), _rand(rows, cols, 2), _weight(cols, "f32").cuda()
    h64 = norm.stream(x.double().numpy(), r.double().numpy())
    for over in ("x", "r"):
        dx, dr, y = x.cuda(), r.cuda(), torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
        h = dx if over == "x" else dr
        X.check(X.xs_rmsnorm(dx.data_ptr(), cols, dr.data_ptr(), cols, w.data_ptr(), X.XS_TYPE_F32, EPS, rows, cols, h.data_ptr(), cols, y.data_ptr(),
                             cols, None, 0, None, 0, _stream()))
        assert np.array_equal(h.cpu().double().numpy(), h64)
    dw = torch.full((cols,), S, device="cuda")
    X.check(X.xs_rmsnorm_backward(dx.data_ptr(), cols, None, 0, dx.data_ptr(), cols, w.data_ptr(), X.XS_TYPE_F32, EPS, 0, cols, y.data_ptr(), cols,
                                  dw.data_ptr(), None, 0, _stream()))
    assert not dw.any()


def test_infinities_stay_in_their_row_and_block():
    X = xs()
    rows, cols = 4, 512
    x = _rand(rows, cols, 1)
    x[1, 200], x[2, 3] = float("inf"), float("nan")
    d, w = x.cuda(), torch.ones(cols, device="cuda")
    codes, scales = torch.zeros((rows, cols), dtype=torch.uint8, device="cuda"), torch.zeros((rows, 4), device="cuda")
    X.check(X.xs_rmsnorm(d.data_ptr(), cols, None, 0, w.data_ptr(), X.XS_TYPE_F32, EPS, rows, cols, None, 0, None, 0, codes.data_ptr(), cols,
                         scales.data_ptr(), 4, _stream()))
    s = scales.cpu()
    assert torch.isfinite(s[[0, 3]]).all() and torch.isnan(s[2]).all() and torch.isnan(s[1, 1])
    assert not codes[2].any()


def test_a_long_batch_and_equal_bits_in_a_replayed_graph():
    X = xs()
    rows, cols = 9001, 896
    g = torch.Generator(device="cuda").manual_seed(0)
    h, dy = (torch.randn((rows, cols), generator=g, device="cuda").bfloat16() for _ in range(2))
    w = _weight(cols, "bf16").cuda()
    ws = X.workspace(X.xs_rmsnorm_backward_workspace_bytes, rows, cols)
    dx, dw, y = torch.zeros_like(h), torch.zeros(cols, device="cuda"), torch.zeros_like(h)

    def step():
        X.check(X.xs_rmsnorm(h.data_ptr(), cols, None, 0, w.data_ptr(), X.XS_TYPE_BF16, EPS, rows, cols, None, 0, y.data_ptr(), cols, None, 0, None, 0, _stream()))
        X.check(X.xs_rmsnorm_backward(dy.data_ptr(), cols, None, 0, h.data_ptr(), cols, w.data_ptr(), X.XS_TYPE_BF16, EPS, rows, cols, dx.data_ptr(), cols,
                                      dw.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))

    step()
    hd, wd, yd = h.double(), w.double(), dy.double()
    i = 1 / torch.sqrt((hd * hd).mean(1, keepdim=True) + EPS)
    assert ((y.double() - hd * i * wd).abs() <= (2.0 ** -8 + 2.0 ** -17) * (hd * i * wd).abs()).all()
    want, mag = (yd * hd * i).sum(0), (yd * hd * i).abs().sum(0)
    assert ((dw.double() - want).abs() <= ((rows + 64) * 2.0 ** -24 + 2.0 ** -16) * mag).all()
    first = [t.clone() for t in (y, dx, dw)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (y, dx, dw):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), first))
