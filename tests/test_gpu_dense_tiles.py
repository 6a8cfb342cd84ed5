"""The products on every tile, with the ends that each has: sizes next to the ones at which the rules change over.  Whole numbers are equal bit
for bit (test_gpu_dense has the reason); with gelu and silu the bounds are those of its random numbers: sums of n terms within n U of their
magnitudes, 40 U for the activation, one rounding to the storage type."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_branch as P
from tests.test_gpu_dense import U, Rows, backward, forward, rounded, whole, workspace

pytestmark = pytest.mark.gpu

# rows, cin, cout of a bf16 product with rows of whole 16-byte runs
FORWARD = {"256": (3600, 136, 3592), "192": (4100, 72, 1936), "128": (2000, 72, 1032), "256 in parts": (2050, 4104, 2000), "128 in parts": (1100, 1032, 1000),
           "64 in parts": (600, 1032, 520)}
INPUT = {"256": (3600, 3592, 136), "192": (4100, 1936, 72), "128": (2000, 1032, 72), "256 in parts": (2050, 2000, 4104), "128 in parts": (1100, 1000, 1032)}
FILTERS = {"256": (136, 3592, 3600), "192": (136, 2048, 6000), "128": (72, 1032, 2000), "256 in parts": (4104, 2000, 2056), "128 in parts": (1032, 1000, 1104)}


@pytest.mark.parametrize("tile", FORWARD)
def test_forward_ends(tile):
    """Every activation, with and without bias, residual and the stored p."""
    M, K, N = FORWARD[tile]
    rng = np.random.default_rng(M)
    td, E = torch.bfloat16, 2.0 ** -8
    x, res = rounded(rng.standard_normal((M, K)), td), rounded(rng.standard_normal((M, N)), td)
    w = rounded(rng.standard_normal((N, K)) * (1.5 / np.sqrt(K)), td)
    bias = rounded(0.2 * rng.standard_normal(N), torch.float32)
    q, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    for act in range(4):
        for b, r, keep in ((bias, res, True), (None, None, act == 2), (bias, None, act == 3), (None, res, act != 2)):
            y, pre = forward("bf16", x, w, b, r, act, keep, pad=8 * (act % 2))
            p = q if b is None else q + b
            off = (K + 2) * U * (mag + (0 if b is None else np.abs(b)))
            if keep:
                assert (np.abs(pre - p) <= E * np.abs(p) + 1.01 * off).all(), act
            rr = 0.0 if r is None else r
            ref = P.act(act, p) + rr
            assert (np.abs(y - ref) <= E * np.abs(ref) + 1.13 * 1.01 * off + 40 * U * (np.abs(p) + np.abs(rr))).all(), (act, b is None, r is None, keep)


@pytest.mark.parametrize("which,tile", [(k, t) for k in ("x", "w") for t in (INPUT if k == "x" else FILTERS)])
def test_gradients(which, tile):
    """Whole numbers, with relu's g (rows filled up to whole runs in the workspace) and with dy itself."""
    M, K, N = (INPUT if which == "x" else FILTERS)[tile]
    rng = np.random.default_rng(M + K)
    x, w, dy, pre = whole(rng, (M, K)), whole(rng, (N, K)), whole(rng, (M, N)), whole(rng, (M, N), 2)
    for act, pad, off in ((P.RELU, 0, 0), (P.IDENTITY, 8, 8)):
        g = dy * P.slope(act, pre)
        gx, gw, _ = backward("bf16", dy, x, w, pre, act, which, pad, off)
        assert gx is None or np.array_equal(gx, rounded(g @ w, torch.bfloat16)), act
        assert gw is None or np.array_equal(gw, rounded(g.T @ x, torch.bfloat16)), act


@pytest.mark.parametrize("M,K,N", [(3600, 136, 3592), (4100, 72, 1936), (2050, 4104, 2000)])
def test_what_lies_behind_edges_does_not_count(M, K, N):
    """NaN between the rows, behind the last row's end and in one row and one filter."""
    td = torch.bfloat16
    rng = np.random.default_rng(N)
    x, w = whole(rng, (M, K)), whole(rng, (N, K))
    buf = torch.full((M + 300, K + 8), float("nan"), dtype=td, device="cuda")
    buf[:M, :K] = torch.from_numpy(x.astype(np.float32)).cuda().to(td)
    wide = torch.full(((N + 300) * K,), float("nan"), dtype=td, device="cuda")
    wide[:N * K] = torch.from_numpy(w.astype(np.float32)).cuda().to(td).view(-1)
    buf[M - 1, 3], wide[(N - 1) * K + 1] = float("nan"), float("nan")
    y = Rows(np.full((M, N), 77.0), td, 8)
    desc = D.make_dense_desc(M, K, N, D.DSP_BF16, 0, K + 8, N + 8)
    ws, n = workspace(desc, False)
    D.dsp_dense_forward(desc, buf, wide, None, None, y.view, None, ws, n)
    got = y.get()
    assert np.array_equal(got[:-1, :-1], rounded(x @ w.T, td)[:-1, :-1]) and np.isnan(got[-1]).all() and np.isnan(got[:, -1]).all()
