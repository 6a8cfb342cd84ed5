"""States of the recurrence that are infinite: what a row makes of them by the definition, whichever kernel goes through the rows."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_branch as P
from tests.test_gpu_dense import Rows, rounded
from tests.test_gpu_recurrence import TYPES, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [4, 16, 17, 40, 64, 129, 700, 9000])
@pytest.mark.parametrize("dtype", TYPES)
def test_infinite_states(dtype, n):
    """An infinity in x, in the state that goes in and in a gradient goes through decays that are not 0, and comes out of the last row as it is;
    what is NaN by the definition is NaN."""
    code, td, _ = TYPES[dtype]
    C, m = 40, n // 2
    rng = np.random.default_rng(n)
    for decay, coupled in ((P.SIGMOID, True), (P.SIGMOID, False), (P.EXP, True), (P.EXP, False)):
        f = rng.standard_normal((n, C)) + (2.0 if decay == P.SIGMOID else 0.0)
        f = rounded(f if decay == P.SIGMOID else -np.exp(f - 2), td)
        x, dh = rounded(rng.standard_normal((n, C)), td), rounded(rng.standard_normal((n, C)), td)
        state, dlast = (rounded(rng.standard_normal((1, C)), torch.float32) for _ in range(2))
        x[n - 1, 0], x[m, 1], x[0, 2], state[0, 3], x[m, 4] = np.inf, np.inf, -np.inf, np.inf, np.inf
        f[m, 5], state[0, 5] = -np.inf, np.inf      # 0 times infinity
        f[:, 6], state[0, 6] = (np.inf if decay == P.SIGMOID else 0.0), -np.inf
        x[m, 7], x[n - 1, 7] = np.inf, -np.inf
        dh[0, 10], dh[m, 11], dh[n - 1, 12], dlast[0, 13] = np.inf, -np.inf, np.inf, np.inf
        f[:, 14], dlast[0, 14] = (np.inf if decay == P.SIGMOID else 0.0), -np.inf
        desc = D.make_recurrence_desc(1, n, n, C, code, decay, coupled)
        nb = D.dsp_recurrence_workspace_bytes(desc)
        ws = torch.full((nb + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        dx, df, h, ddh = Rows(x, td), Rows(f, td), Rows(np.zeros((n, C)), td), Rows(dh, td)
        gx, gf = Rows(np.zeros((n, C)), td), Rows(np.zeros((n, C)), td)
        st, dl = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (state, dlast))
        last, front = torch.zeros_like(st), torch.zeros_like(st)
        D.dsp_recurrence_forward(desc, dx.view, df.view, None, st, h.view, last, ws, nb)
        got = h.get()
        D.dsp_recurrence_backward(desc, ddh.view, dl, dx.view, df.view, h.view, None, st, gx.view, gf.view, front, ws, nb)
        with np.errstate(all="ignore"):
            rh, rl, oh, ol = P.scan(decay, coupled, x, f, state[0])
            rx, rf, rs, ox, of, os = P.scan_back(decay, coupled, x, f, got, state[0], dh, dlast[0])
        E = TYPES[dtype][2]
        for name, g, r, o, e in (("h", got, rh, oh, E), ("last", last.cpu().numpy()[0], rl, ol, 0), ("dx", gx.get(), rx, ox, E), ("df", gf.get(), rf, of, E),
                                 ("front", front.cpu().numpy()[0], rs, os, 0)):
            g = np.asarray(g, np.float64)
            assert np.array_equal(np.isnan(g), np.isnan(r)), (name, decay, coupled, np.argwhere(np.isnan(g) != np.isnan(r))[:4])
            assert np.array_equal(g[np.isinf(r)], r[np.isinf(r)]), (name, decay, coupled)
            ok = np.isfinite(r)
            assert (np.abs(g[ok] - r[ok]) <= e * np.abs(r[ok]) + 1.01 * U * o[ok] + 1e-38).all(), (name, decay, coupled)
