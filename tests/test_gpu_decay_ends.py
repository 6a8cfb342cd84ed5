"""The decays of the recurrence at the ends of the floats: exp(f) up to 3.4e38 and down to the smallest one."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_branch as P
from tests.test_gpu_dense import rounded
from tests.test_gpu_recurrence import U

pytestmark = pytest.mark.gpu


def test_decays_next_to_the_largest_float():
    """exp(f) up to 3.4e38: 10 U of itself, from a small state and back to front."""
    f = rounded(np.linspace(86.0, 88.7, 271), torch.float32)
    C = len(f)
    for n in (1, 20):
        rows = np.full((n, C), 0.0)
        rows[0] = f
        desc = D.make_recurrence_desc(1, n, n, C, D.DSP_FP32, P.EXP, False)
        nb = D.dsp_recurrence_workspace_bytes(desc)
        ws = torch.empty(nb + 16, dtype=torch.uint8, device="cuda")
        h, gx, gs = torch.empty(n, C, device="cuda"), torch.empty(n, C, device="cuda"), torch.empty(1, C, device="cuda")
        gate, zero, small = torch.from_numpy(rows.astype(np.float32)).cuda(), torch.zeros(n, C, device="cuda"), torch.full((1, C), 2.0 ** -40, device="cuda")
        D.dsp_recurrence_forward(desc, zero, gate, None, small, h, None, ws, nb)
        D.dsp_recurrence_backward(desc, zero, small, zero, gate, h, None, small, gx, None, gs, ws, nb)
        ref = np.exp(f) * 2.0 ** -40
        for got in (h[n - 1], gs[0]):
            got = got.cpu().numpy().astype(np.float64)
            assert (np.abs(got - ref) <= 10 * U * ref).all(), n


def test_decays_below_the_normal_floats():
    """A state of 2^60 shows them: 10 U of themselves and a step and a half of the floats below 2^-126, which are 2^-149 apart."""
    f = rounded(np.linspace(-102.0, -86.0, 331), torch.float32)
    C = len(f)
    for n in (1, 20):
        rows = np.full((n, C), 0.0)
        rows[0] = f
        desc = D.make_recurrence_desc(1, n, n, C, D.DSP_FP32, P.EXP, False)
        nb = D.dsp_recurrence_workspace_bytes(desc)
        ws = torch.empty(nb + 16, dtype=torch.uint8, device="cuda")
        h, df, gs = torch.empty(n, C, device="cuda"), torch.empty(n, C, device="cuda"), torch.empty(1, C, device="cuda")
        gate, zero, large = torch.from_numpy(rows.astype(np.float32)).cuda(), torch.zeros(n, C, device="cuda"), torch.full((1, C), 2.0 ** 60, device="cuda")
        D.dsp_recurrence_forward(desc, zero, gate, None, large, h, None, ws, nb)
        D.dsp_recurrence_backward(desc, zero, torch.ones(1, C, device="cuda"), zero, gate, h, None, large, None, df, gs, ws, nb)
        ref = np.exp(f) * 2.0 ** 60
        for got, r in ((h[n - 1], ref), (df[0], ref)):
            got = got.cpu().numpy().astype(np.float64)
            assert (np.abs(got - r) <= 10 * U * r + 1.5 * 2.0 ** -149 * 2.0 ** 60).all(), n
        assert (np.abs(gs[0].cpu().numpy().astype(np.float64) * 2.0 ** 60 - ref) <= 10 * U * ref + 1.5 * 2.0 ** -149 * 2.0 ** 60).all(), n
