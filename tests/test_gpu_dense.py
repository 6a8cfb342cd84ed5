"""Products with bias, activation and residual, and their gradients, against their definitions in 64 bits.

Most cases hold small whole numbers: every product and sum of them is below 2^24, so whatever order they are added in gives the same
float, and the result is that number rounded once to the storage type: equal, bit for bit.  Elsewhere U = 2^-24 is half a step of fp32
and E half a step of the storage type relative to the value; a sum of n terms in any order is off by at most n U of their magnitudes."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_branch as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": (D.DSP_FP32, torch.float32, U), "bf16": (D.DSP_BF16, torch.bfloat16, 2.0 ** -8)}


def rounded(a, td):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(td).float().numpy().astype(np.float64)


class Rows:
    """A matrix on the device with `pad` elements between its rows and guards around; host copy in 64 bits."""

    def __init__(self, a, td, pad=0, off=0):
        self.shape, self.td, self.pad, self.off = a.shape, td, pad, off
        m, c = a.shape
        self.buf = torch.full((off + m * (c + pad) + 16,), 77.0, dtype=td, device="cuda")
        self.view = self.buf[off:off + m * (c + pad)].view(m, c + pad)[:, :c]
        self.view.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(td))

    def get(self):
        torch.cuda.synchronize()
        m, c = self.shape
        whole = self.buf.float().cpu().numpy()
        assert (whole[:self.off] == 77).all() and (whole[self.off + m * (c + self.pad):] == 77).all(), "written outside the rows"
        whole = whole[self.off:self.off + m * (c + self.pad)].reshape(m, c + self.pad)
        assert (whole[:, c:] == 77).all(), "written between the rows"
        return whole[:, :c].astype(np.float64)


def workspace(desc, back):
    n = D.dsp_dense_workspace_bytes(desc, back)
    return torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda"), n  # (NaN in every type: nothing of it may count)


def forward(dtype, x, w, bias, res, act, keep, pad=0, off=0, stream=None, in_place=False):
    code, td, _ = TYPES[dtype]
    (M, K), N = x.shape, w.shape[0]
    desc = D.make_dense_desc(M, K, N, code, act, K + pad, N + pad)
    dx, dw, y = Rows(x, td, pad, off), Rows(w, td, 0, off), Rows(np.full((M, N), 77.0), td, pad, off)
    db = None if bias is None else torch.from_numpy(bias.astype(np.float32)).cuda()
    dr = None if res is None else Rows(res, td, pad, off)
    pre = Rows(np.full((M, N), 77.0), td, pad, off) if keep else None
    ws, n = workspace(desc, False)
    if in_place:
        y = dr
    torch.cuda.synchronize()
    D.dsp_dense_forward(desc, dx.view, dw.view, db, dr.view if dr else None, y.view, pre.view if keep else None, ws, n, stream=stream)
    return y.get(), pre.get() if keep else None


def backward(dtype, dy, x, w, pre, act, want="xwb", pad=0, off=0, stream=None):
    code, td, _ = TYPES[dtype]
    (M, K), N = x.shape, w.shape[0]
    desc = D.make_dense_desc(M, K, N, code, act, K + pad, N + pad)
    ddy, dx, dw = Rows(dy, td, pad, off), Rows(x, td, pad, off), Rows(w, td, 0, off)
    dp = Rows(pre, td, pad, off) if act else None
    gx = Rows(np.full((M, K), 77.0), td, pad, off) if "x" in want else None
    gw = Rows(np.full((N, K), 77.0), td, 0, off) if "w" in want else None
    gb = torch.full((N + 8,), 77.0, device="cuda") if "b" in want else None
    ws, n = workspace(desc, True)
    torch.cuda.synchronize()
    D.dsp_dense_backward(desc, ddy.view, dx.view, dw.view, dp.view if act else None, gx.view if gx else None, gw.view if gw else None, gb, ws, n,
                         stream=stream)
    torch.cuda.synchronize()
    if gb is not None:
        gb = gb.cpu().numpy().astype(np.float64)
        assert (gb[N:] == 77).all()
        gb = gb[:N]
    return gx.get() if gx else None, gw.get() if gw else None, gb


def whole(rng, shape, most=3):
    return rng.integers(-most, most + 1, shape).astype(np.float64)


# one row, a few, tiles that end early in every direction, tiles of every size, long sums
SHAPES = [(1, 1, 1), (1, 64, 64), (2, 7, 3), (1, 520, 136), (5, 40, 24), (16, 256, 128), (17, 100, 33), (33, 31, 65), (64, 64, 64), (65, 129, 127),
          (100, 8, 264), (128, 128, 128), (130, 192, 136), (257, 65, 130), (300, 264, 520), (9, 2048, 72), (3, 4097, 40), (640, 72, 16),
          (1100, 136, 264), (513, 1000, 257), (48, 2056, 40), (33, 520, 264), (64, 1001, 33), (70, 2600, 72), (66, 5000, 8), (1100, 1032, 1000), (4100, 136, 1936),
          (2050, 2008, 1032), (1500, 77, 4099), (2050, 1000, 1003), (4100, 1000, 4104), (6000, 72, 2048)]


@pytest.mark.parametrize("M,K,N", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_whole_numbers_are_exact(dtype, M, K, N):
    td = TYPES[dtype][1]
    rng = np.random.default_rng(M * 7 + K * 3 + N)
    x, w, bias, res = whole(rng, (M, K)), whole(rng, (N, K)), whole(rng, N, 50), whole(rng, (M, N), 100)
    p = x @ w.T
    for act, b, r, keep, pad, off in ((0, None, None, False, 0, 0), (1, bias, res, True, 0, 0), (0, bias, None, True, 8, 8), (1, None, res, False, 3, 1)):
        q = p if b is None else p + b
        y, pre = forward(dtype, x, w, b, r, act, keep, pad, off)
        assert np.array_equal(y, rounded(P.act(act, q) + (0 if r is None else r), td)), (act, pad, off)
        assert not keep or np.array_equal(pre, rounded(q, td)), (act, pad, off)
    dy, pre = whole(rng, (M, N)), whole(rng, (M, N), 2)
    for act, pad, off in ((0, 0, 0), (1, 0, 0), (0, 8, 8), (1, 3, 1)):
        g = dy * P.slope(act, pre)
        gx, gw, gb = backward(dtype, dy, x, w, pre, act, pad=pad, off=off)
        assert np.array_equal(gx, rounded(g @ w, td)), (act, pad, off)
        assert np.array_equal(gw, rounded(g.T @ x, td)), (act, pad, off)
        assert np.array_equal(gb, g.sum(0)), (act, pad, off)


@pytest.mark.parametrize("want", ["x", "w", "b", "xb", "wb"])
def test_gradients_that_are_not_asked_for(want):
    rng = np.random.default_rng(5)
    M, K, N = 70, 90, 50
    x, w, dy, pre = whole(rng, (M, K)), whole(rng, (N, K)), whole(rng, (M, N)), whole(rng, (M, N))
    for act in (0, 1):
        g = dy * P.slope(act, pre)
        for name, got, ref in zip("xwb", backward("bf16", dy, x, w, pre, act, want), (g @ w, g.T @ x, g.sum(0))):
            assert (got is None) == (name not in want)
            assert got is None or np.array_equal(got, rounded(ref, torch.bfloat16 if name != "b" else torch.float32))


@pytest.mark.parametrize("act", [P.GELU, P.SILU], ids=["gelu", "silu"])
def test_activations_relative_to_themselves(act):
    """One product by 1, so that p is the input.  Phi: the fitted polynomial 2.2 U, t and its nine steps 8 U, exp(-x^2/2) 4 U and the
    product's roundings: 20 U of Phi.  x > 0: 1 - q. gelu' = Phi + x phi, below 0 a difference: 24 U of the sum of both magnitudes.
    silu: exp 3 U, its quotient 1 + 2 + 1 U, x: 8 U; its derivative 12 U of the sum of magnitudes.  Below 2^-126 the exponential is 0."""
    rng = np.random.default_rng(act)
    v = np.exp(rng.uniform(np.log(1e-5), np.log(20.0), 4000)) * rng.choice([-1.0, 1.0], 4000)
    v[:14] = [np.inf, -np.inf, np.nan, 0.0, -0.0, 1e30, -1e30, 3e38, -3e38, 15.99, -13.0, -100.0, -127.5, 88.0]
    v = rounded(v, torch.float32)[:, None]
    one = np.ones((1, 1))
    y, pre = forward("fp32", v, one, None, None, act, True)
    assert np.array_equal(pre, v, equal_nan=True)
    ref = P.act(act, v)
    assert np.array_equal(np.isnan(y), np.isnan(ref))
    with np.errstate(all="ignore"):
        tiny = 2.0 ** -126 * np.maximum(1.0, np.where(np.isfinite(v), np.abs(v), 1.0))
        assert not (np.abs(y - ref) > 24 * U * np.abs(ref) + tiny)[np.isfinite(ref)].any()
        assert np.array_equal(y[np.isinf(ref)], ref[np.isinf(ref)])
    n = len(v)
    _, _, gb = backward("fp32", np.ones((1, n)), np.ones((1, 1)), np.ones((n, 1)), v.T, act, "b")
    ref = P.slope(act, v[:, 0])
    with np.errstate(all="ignore"):
        x = np.where(np.isfinite(v[:, 0]), v[:, 0], 0.0)
        parts = P.ndtr(x) + np.abs(x) * np.exp(-x * x / 2) if act == P.GELU else P.expit(x) * (1 + np.abs(x) * P.expit(-x))
    assert np.array_equal(np.isnan(gb), np.isnan(ref))
    assert not (np.abs(gb - ref) > 30 * U * parts + 2.0 ** -120)[~np.isnan(ref)].any()


@pytest.mark.parametrize("M,K,N", [(1, 300, 200), (200, 333, 150), (1024, 512, 384), (333, 777, 1040)])
@pytest.mark.parametrize("act", [0, 1, 2, 3], ids=["identity", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", TYPES)
def test_random_numbers(dtype, act, M, K, N):
    """Sums of n terms within n U of their magnitudes, in one order or another, and 40 U for the activation; the products of the backward
    pass read g rounded once to the storage type."""
    _, td, E = TYPES[dtype]
    rng = np.random.default_rng(M + K + N + act)
    x, w, res = (rounded(rng.standard_normal(s), td) for s in ((M, K), (N, K), (M, N)))
    w = rounded(w / np.sqrt(K), td)
    bias = rounded(0.2 * rng.standard_normal(N), torch.float32)
    p, mag = x @ w.T + bias, np.abs(x) @ np.abs(w).T + np.abs(bias)
    y, pre = forward(dtype, x, w, bias, res, act, True)
    off = (K + 2) * U * mag
    assert (np.abs(pre - p) <= E * np.abs(p) + 1.01 * off).all()
    ref = P.act(act, p) + res
    assert (np.abs(y - ref) <= E * np.abs(ref) + 1.13 * 1.01 * off + 40 * U * (np.abs(p) + np.abs(res))).all()  # (|gelu'| <= 1.129)
    dy = rounded(rng.standard_normal((M, N)), td)
    s = P.slope(act, pre)
    g, og = dy * s, np.abs(dy) * ((E * np.abs(s) if act else 0) + 40 * U * (1 + np.abs(pre) * (act > 1)))
    gx, gw, gb = backward(dtype, dy, x, w, pre, act)
    rx, rw, rb = g @ w, g.T @ x, g.sum(0)
    assert (np.abs(gx - rx) <= E * np.abs(rx) + 1.01 * (og @ np.abs(w) + (N + 2) * U * (np.abs(g) @ np.abs(w)))).all()
    assert (np.abs(gw - rw) <= E * np.abs(rw) + 1.01 * (og.T @ np.abs(x) + (M + 2) * U * (np.abs(g).T @ np.abs(x)))).all()
    assert (np.abs(gb - rb) <= 1.01 * (np.abs(dy) * 40 * U * (1 + np.abs(pre))).sum(0) + (M + 2) * U * np.abs(g).sum(0)).all()


def test_gradients_against_differences():
    """The loss sum c y of the definition in 64 bits, moved by 1e-5 along a direction: the difference is off by its third derivative, below 1e-8
    of the magnitudes, the gradients in fp32 by (n + 40) U of theirs."""
    rng = np.random.default_rng(3)
    M, K, N = 21, 35, 19
    for act in (2, 3):
        x, w = rounded(rng.standard_normal((M, K)), torch.float32), rounded(rng.standard_normal((N, K)) / 6, torch.float32)
        bias, c = rounded(rng.standard_normal(N), torch.float32), rounded(rng.standard_normal((M, N)), torch.float32)
        pre = x @ w.T + bias
        g = backward("fp32", c, x, w, pre, act)
        mags = (np.abs(c) @ np.abs(w), np.abs(c).T @ np.abs(x), np.abs(c).sum(0))
        for i, t in enumerate((rng.standard_normal((M, K)), rng.standard_normal((N, K)), rng.standard_normal(N))):
            def value(h):
                a = [x, w, bias]
                a[i] = a[i] + h * t
                return (c * P.act(act, a[0] @ a[1].T + a[2])).sum()
            diff = (value(1e-5) - value(-1e-5)) / 2e-5
            # (pre is handed over as floats: its rounding moves the slope by U |pre| times the second derivative, below 1)
            assert abs((g[i] * t).sum() - diff) <= (120 * U + 1e-8) * (np.abs(t) * mags[i] * (1 + np.abs(pre).max())).sum(), (act, i)


def test_the_residual_may_be_the_output():
    rng = np.random.default_rng(8)
    for dtype, M, K, N, pad in (("bf16", 300, 64, 136, 0), ("fp32", 70, 33, 41, 3), ("bf16", 1, 64, 64, 0)):
        x, w, res = whole(rng, (M, K)), whole(rng, (N, K)), whole(rng, (M, N), 20)
        y, _ = forward(dtype, x, w, None, res, 0, False, pad, in_place=True)
        assert np.array_equal(y, rounded(x @ w.T + res, TYPES[dtype][1]))


def test_nan_and_infinity_stay_in_their_rows():
    """What a row, a filter or what lies between rows holds reaches no other row's results."""
    rng = np.random.default_rng(9)
    for dtype, M, K, N, pad in (("bf16", 140, 72, 130, 8), ("fp32", 140, 72, 130, 4), ("bf16", 140, 71, 130, 3), ("bf16", 3, 72, 130, 8)):
        code, td, _ = TYPES[dtype]
        x, w = whole(rng, (M, K)), whole(rng, (N, K))
        bad_x, bad_w = x.copy(), w.copy()
        bad_x[1], bad_w[4, 5] = np.nan, np.inf
        buf = torch.full((M, K + pad), float("nan"), dtype=td, device="cuda")
        buf[:, :K] = torch.from_numpy(bad_x).cuda().to(td)
        y = torch.zeros(M, N, dtype=td, device="cuda")
        desc = D.make_dense_desc(M, K, N, code, 0, K + pad)
        ws, n = workspace(desc, False)
        D.dsp_dense_forward(desc, buf, Rows(bad_w, td).view, None, None, y, None, ws, n)
        got, ref = y.float().cpu().numpy(), rounded(x @ w.T, td)
        rows, cols = np.arange(M) != 1, np.arange(N) != 4
        assert np.array_equal(got[rows][:, cols], ref[rows][:, cols]) and np.isnan(got[1]).all() and not np.isfinite(got[:, 4]).all()
        # dy with NaN between its rows, and x likewise
        dy = whole(rng, (M, N))
        dbuf = torch.full((M, N + pad), float("nan"), dtype=td, device="cuda")
        dbuf[:, :N] = torch.from_numpy(dy).cuda().to(td)
        buf[1, :K] = torch.from_numpy(x[1]).cuda().to(td)
        desc = D.make_dense_desc(M, K, N, code, 0, K + pad, N + pad)
        ws, n = workspace(desc, True)
        gx, gw = torch.empty_like(buf), torch.empty(N, K, dtype=td, device="cuda")
        D.dsp_dense_backward(desc, dbuf, buf, Rows(w, td).view, None, gx, gw, None, ws, n)
        assert np.array_equal(gx[:, :K].float().cpu().numpy(), rounded(dy @ w, td))
        assert np.array_equal(gw.float().cpu().numpy(), rounded(dy.T @ x, td))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_far_apart(dtype):
    """Rows whose distances in bytes pass 2^32; nothing between them is touched (that is memory never written)."""
    code, td, _ = TYPES[dtype]
    M, K, N = 5, 48, 40
    stride = (1 << 30) // (1 if dtype == "bf16" else 2) + 8
    rng = np.random.default_rng(2)
    x, w, dy = whole(rng, (M, K)), whole(rng, (N, K)), whole(rng, (M, N))
    big = torch.empty((M - 1) * stride + 64, dtype=td, device="cuda")
    rows = big.as_strided((M, K), (stride, 1))
    outs = big.as_strided((M, N), (stride, 1))
    dw = torch.from_numpy(w).cuda().to(td)
    rows.copy_(torch.from_numpy(x).cuda().to(td))
    y = torch.empty(M, N, dtype=td, device="cuda")
    desc = D.make_dense_desc(M, K, N, code, 0, stride, N)
    ws, n = workspace(desc, True)
    D.dsp_dense_forward(desc, rows, dw, None, None, y, None, ws, n)
    assert np.array_equal(y.float().cpu().numpy(), rounded(x @ w.T, td))
    gw = torch.empty(N, K, dtype=td, device="cuda")
    D.dsp_dense_backward(desc, torch.from_numpy(dy).cuda().to(td), rows, dw, None, None, gw, None, ws, n)
    assert np.array_equal(gw.float().cpu().numpy(), rounded(dy.T @ x, td))
    small = torch.from_numpy(x).cuda().to(td)
    desc = D.make_dense_desc(M, K, N, code, 0, K, stride)
    D.dsp_dense_forward(desc, small, dw, None, None, outs, None, ws, n)
    assert np.array_equal(outs.float().cpu().numpy(), rounded(x @ w.T, td))
    outs.copy_(torch.from_numpy(dy).cuda().to(td))
    gx = torch.empty(M, K, dtype=td, device="cuda")
    ws, n = workspace(desc, True)
    D.dsp_dense_backward(desc, outs, small, dw, None, gx, gw, None, ws, n)
    assert np.array_equal(gx.float().cpu().numpy(), rounded(dy @ w, td))
    assert np.array_equal(gw.float().cpu().numpy(), rounded(dy.T @ x, td))


def test_tiles_beyond_32_bits():
    """Tiles of bf16 rows of which the last lie more than 2^32 bytes behind the first, in every operand and output."""
    code, td, _ = TYPES["bf16"]
    M, K, N, stride = 1100, 1032, 1040, 2000000
    rng = np.random.default_rng(6)
    x, w, dy = whole(rng, (M, K)), whole(rng, (N, K)), whole(rng, (M, N))
    big = [torch.empty((M - 1) * stride + 1048, dtype=td, device="cuda") for _ in range(2)]
    xs, ys = big[0].as_strided((M, K), (stride, 1)), big[1].as_strided((M, N), (stride, 1))
    dw = torch.from_numpy(w).cuda().to(td)
    xs.copy_(torch.from_numpy(x).cuda().to(td))
    desc = D.make_dense_desc(M, K, N, code, 0, stride, stride)
    ws, n = workspace(desc, False)
    D.dsp_dense_forward(desc, xs, dw, None, None, ys, None, ws, n)
    assert np.array_equal(ys.float().cpu().numpy(), rounded(x @ w.T, td))
    ys.copy_(torch.from_numpy(dy).cuda().to(td))
    ws, n = workspace(desc, True)
    gw, gx = torch.empty(N, K, dtype=td, device="cuda"), torch.empty((M - 1) * stride + 1048, dtype=td, device="cuda").as_strided((M, K), (stride, 1))
    D.dsp_dense_backward(desc, ys, xs, dw, None, gx, gw, None, ws, n)
    assert np.array_equal(gx.float().cpu().numpy(), rounded(dy @ w, td))
    assert np.array_equal(gw.float().cpu().numpy(), rounded(dy.T @ x, td))


@pytest.mark.parametrize("M,K,N", [(1, 2048, 520), (300, 264, 520), (1100, 512, 256), (600, 100, 77), (300, 2600, 72), (1100, 1032, 1000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_streams_graphs_and_repetition(dtype, M, K, N):
    """The same bits on another stream, twice, and from a captured graph replayed with eager calls in between."""
    code, td, _ = TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(M)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(td)  # noqa: E731
    x, w, res, dy, bias = r(M, K), r(N, K), r(M, N), r(M, N), torch.randn(N, generator=gen, device="cuda")
    desc = D.make_dense_desc(M, K, N, code, P.GELU)
    new = lambda: [torch.empty(M, N, dtype=td, device="cuda"), torch.empty(M, N, dtype=td, device="cuda"), torch.empty_like(x), torch.empty_like(w),  # noqa: E731
                   torch.empty_like(bias)]
    nf, nb = D.dsp_dense_workspace_bytes(desc), D.dsp_dense_workspace_bytes(desc, True)

    def go(o, ws, stream=None):
        D.dsp_dense_forward(desc, x, w, bias, res, o[0], o[1], ws, nf, stream=stream)
        D.dsp_dense_backward(desc, dy, x, w, o[1], o[2], o[3], o[4], ws, nb, stream=stream)
    ws = [torch.full((max(nf, nb) + 16,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2)]
    first, other, captured = new(), new(), new()
    go(first, ws[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    go(other, ws[1], side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(captured, ws[1])
    for k in range(3):
        for t in captured:
            t.fill_(float(k))
        x.add_(1.0)
        go(first, ws[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, captured)), k
