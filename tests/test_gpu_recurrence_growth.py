"""The recurrence with decays above 1 and with large states: h is what the definition gives row by row, whatever the products of decays do that a
scan forms on the way.

The decays are exp(L_t - L_(t-1)) of a path L between -60 and 80: every state and gradient stays within the floats (below e^80 some hundred
times, above e^-80), but over the rows of a slot, a tile or a part the product of the decays goes up to e^140 and down to e^-140.  The bounds are those
of plain_branch.scan, which holds for any decay; what is below 2^-126 may be lost, and is lost before a path that rises again only where it is
e^-60 of the state, far above that."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_branch as P
from tests.test_gpu_dense import rounded
from tests.test_gpu_recurrence import TYPES, U, call

pytestmark = pytest.mark.gpu


def steep(n):
    """Four rows up and four down."""
    t = np.arange(n + 1) % 8
    return -60.0 + 35.0 * np.where(t <= 4, t, 8 - t)


def long_ramps(n):
    """500 rows up and 500 down."""
    t = np.arange(n + 1) % 1000
    return -60.0 + 0.28 * np.where(t <= 500, t, 1000 - t)


def wide_steps(n):
    """Up at once, down at once, after 37 rows each."""
    return np.where(np.arange(n + 1) // 37 % 2, 24.0, -60.0)


def problem(path, lengths, C, dtype, coupled, seed=0):
    rng = np.random.default_rng(seed + C + sum(lengths))
    td = TYPES[dtype][1]
    xs, fs, ds, states, lasts = [], [], [], [], []
    for n in lengths:
        want = path(n)
        f, at = np.zeros((n, C)), np.full(C, want[0])
        level = [at]
        for t in range(n):
            f[t] = rounded(want[t + 1] - at + 0.1 * rng.standard_normal(C), td)
            at = at + f[t]
            level.append(at)
        level = np.array(level)
        size = np.exp(level[1:])
        # (what goes in is 1 - a times x where they are coupled)
        xs.append(rounded(rng.standard_normal((n, C)) * size / (np.maximum(1.0, np.abs(np.expm1(f))) if coupled else 1.0), td))
        ds.append(rounded(rng.standard_normal((n, C)) / size, td))
        fs.append(f)
        states.append(rounded(rng.standard_normal(C) * np.exp(level[0]), torch.float32))
        lasts.append(rounded(rng.standard_normal(C) * np.exp(-level[-1]), torch.float32))
    return {"lengths": list(lengths), "rows": sum(lengths), "C": C, "decay": P.EXP, "coupled": coupled, "x": np.concatenate(xs), "f": np.concatenate(fs),
            "dh": np.concatenate(ds), "state": np.array(states), "dlast": np.array(lasts)}


@pytest.mark.parametrize("lengths,C", [([12], 33), ([40], 33), ([700], 72), ([2600, 9, 1100], 40), ([9000], 8), ([100] * 40, 520)])
@pytest.mark.parametrize("path", [steep, long_ramps, wide_steps])
@pytest.mark.parametrize("dtype", TYPES)
def test_decays_above_one(dtype, path, lengths, C):
    """By a lane (12 rows), uncut, in parts, with sixteen waves and with eight."""
    for coupled in (False, True):
        call(problem(path, lengths, C, dtype, coupled), dtype, len(set(lengths)) > 1)


def by_turns(size):
    """One row up, one row down."""
    return lambda n: -20.0 + size * (np.arange(n + 1) % 2)


def wandering(n):
    """Steps of any size, back from the ends."""
    rng = np.random.default_rng(n)
    level = [0.0]
    for _ in range(n):
        to = level[-1] + 6.0 * rng.standard_normal()
        level.append(-120.0 - to if to < -60.0 else 160.0 - to if to > 80.0 else to)
    return np.array(level)


@pytest.mark.parametrize("lengths,C", [([12], 33), ([700], 72), ([9000], 8)])
@pytest.mark.parametrize("path", [by_turns(1.0), by_turns(4.0), by_turns(9.0), by_turns(14.0), by_turns(17.0), wandering],
                         ids=["1", "4", "9", "14", "17", "wandering"])
def test_growth_and_decay_by_turns(path, lengths, C):
    """Products of decays next to 1 whose factors are not: what they lack of 1 is no sum of what the factors lack."""
    for dtype in TYPES:
        for coupled in (False, True):
            call(problem(path, lengths, C, dtype, coupled), dtype, False)


def test_nothing_goes_in_and_nothing_comes_out():
    """Zeros stay zeros under decays whose product no float holds."""
    for n, f in ((12, 23.0), (40, 23.0), (700, 80.0), (9000, 0.3)):
        C = 40
        desc = D.make_recurrence_desc(1, n, n, C, D.DSP_FP32, P.EXP, False)
        nb = D.dsp_recurrence_workspace_bytes(desc)
        ws = torch.full((nb + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        zero, gate, last = torch.zeros(n, C, device="cuda"), torch.full((n, C), f, device="cuda"), torch.full((1, C), 5.0, device="cuda")
        h, dx, df, ds = (torch.full_like(t, 5.0) for t in (zero, zero, zero, last))
        D.dsp_recurrence_forward(desc, zero, gate, None, None, h, last, ws, nb)
        D.dsp_recurrence_backward(desc, zero, None, zero, gate, h, None, None, dx, df, ds, ws, nb)
        assert not any(bool(t.ne(0).any()) for t in (h, last, dx, df, ds)), n


def test_gradients_in_the_place_of_inputs_under_growth():
    """Parts whose products leave the floats, and outputs that take the place of what the products are formed of."""
    for path, n in ((steep, 2600), (long_ramps, 9000)):
        p = problem(path, [n], 40, "fp32", False)
        gh, gx, gf = call(p, "fp32", False)
        desc = D.make_recurrence_desc(1, n, n, 40, D.DSP_FP32, P.EXP, False)
        nb = D.dsp_recurrence_workspace_bytes(desc)
        assert nb
        ws = torch.empty(nb + 16, dtype=torch.uint8, device="cuda")
        dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
        h, st, dl = dev(gh), dev(p["state"]), dev(p["dlast"])
        for place in ("x", "dh"):
            x, f, dh = dev(p["x"]), dev(p["f"]), dev(p["dh"])
            to = x if place == "x" else dh
            D.dsp_recurrence_backward(desc, dh, dl, x, f, h, None, st, to, f, dl.clone(), ws, nb)
            assert np.array_equal(to.cpu().numpy(), gx.astype(np.float32)) and np.array_equal(f.cpu().numpy(), gf.astype(np.float32)), place


def test_large_states_are_forgotten_by_their_rows():
    """States of 1e30 under decays whose product over some rows is below the floats: what is left of them counts."""
    C = 8
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
    for decay in (P.SIGMOID, P.EXP):
        for n in (12, 40, 700, 9000):
            for f0 in (-28.0, -20.0, -0.1):
                f = rounded(np.full((n, C), f0) + 0.01 * np.arange(C), torch.float32)
                zero, state = np.zeros((n, C)), rounded(np.full((1, C), 1e30), torch.float32)
                desc = D.make_recurrence_desc(1, n, n, C, D.DSP_FP32, decay, False)
                nb = D.dsp_recurrence_workspace_bytes(desc)
                ws = torch.empty(nb + 16, dtype=torch.uint8, device="cuda")
                h = torch.empty(n, C, device="cuda")
                D.dsp_recurrence_forward(desc, dev(zero), dev(f), None, dev(state), h, None, ws, nb)
                rh, _, oh, _ = P.scan(decay, False, zero, f, state[0])
                got = h.cpu().numpy().astype(np.float64)
                assert (np.abs(got - rh) <= 1.01 * U * oh + 2.0 ** -126).all(), (decay, n, f0)


@pytest.mark.parametrize("decay", [P.SIGMOID, P.EXP], ids=["sigmoid", "exp"])
@pytest.mark.parametrize("n", [40, 700, 9000])
def test_what_is_left_of_a_large_input_goes_on(decay, n):
    """e^80 comes in with one row, four rows together forget e^-140 of it and the others next to nothing; the same on the way back."""
    C = 40
    rng = np.random.default_rng(n)
    keep = -1e-3 if decay == P.EXP else 7.0
    for at in range(8, 16, 2):
        f, x, dh = np.full((n, C), keep), np.zeros((n, C)), np.zeros((n, C))
        for first in (at, n - 1 - at - 3):
            f[first:first + 4] = -35.0
        x[at - 4] = rng.standard_normal(C) * np.exp(80.0)
        dh[n - 1 - at + 4] = rng.standard_normal(C) * np.exp(80.0)
        p = {"lengths": [n], "rows": n, "C": C, "decay": decay, "coupled": False, "x": rounded(x, torch.float32), "f": rounded(f, torch.float32),
             "dh": rounded(dh, torch.float32), "state": np.zeros((1, C)), "dlast": np.zeros((1, C))}
        call(p, "fp32", False)
