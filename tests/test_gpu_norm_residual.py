"""Norms around a residual block, its gate and residual scale, forward and backward, against their definitions in 64 bits.

U = 2^-24 is half a step of fp32, E half a step of the storage type relative to the value.  A row's sums run over at most 64
elements a lane, 6 levels of a wave and 16 waves: 86 additions, so a sum is off by at most 90 U of its terms' magnitudes, a
statistic by half of that and its own roundings; what an element takes from two statistics, a product of up to 8 factors and a
rational activation (tanh, exp: 4 U each) is off by at most 256 U of the magnitudes of its terms.  Sums over rows add n rows a lane
(n at most 4, the rows over 512 workgroups or those of a row of the gate), up to 64 rows side by side, then 512 / 16 parts a wave and 16
waves: n + 116 additions."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_operators as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5
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


def within(got, ref, bound, what):
    assert np.array_equal(np.isfinite(got), np.isfinite(ref)), what
    off = np.abs(got - ref) - bound
    assert (off <= 0).all(), (what, float(np.max(np.abs(got - ref) / (bound + 1e-300))))


def problem(M, C, dtype, post, pre, gate, act, bias, seed=0, shift=0.0):
    """Inputs of one call; gate: None or (rows that share one of its rows, its type)."""
    rng = np.random.default_rng(seed + 131 * M + C)
    td = TYPES[dtype][1]
    p = {"post": post, "pre": pre, "alpha": 0.875, "beta": -1.25, "eps": EPS, "gate_act": act, "gate_rows": 0, "gate": None,
         "x": rounded(rng.standard_normal((M, C)) * np.exp(rng.standard_normal((M, 1))) + shift, td),
         "z": rounded(rng.standard_normal((M, C)) * np.exp(rng.standard_normal((M, 1))) - shift, td)}
    for name in ("post", "pre"):
        p[name + "_gain"] = (1 + 0.3 * rng.standard_normal(C)).astype(np.float32).astype(np.float64) if bias != "none" else None
        p[name + "_bias"] = (0.3 * rng.standard_normal(C)).astype(np.float32).astype(np.float64) if bias == "both" else None
    if gate:
        p["gate_rows"], p["gate_type"] = gate
        p["gate"] = rounded(rng.standard_normal((-(-M // gate[0]), C)), TYPES[gate[1]][1])
    p["dy"], p["dh"] = rounded(rng.standard_normal((M, C)), td), rounded(rng.standard_normal((M, C)), td)
    return p


def vec(a):
    return None if a is None else torch.from_numpy(a.astype(np.float32)).cuda()


def run(p, dtype, pad=0, off=0, stream=None):
    """Forward and backward of p on the device, each checked."""
    code, td, E = TYPES[dtype]
    M, C = p["x"].shape
    gt = TYPES[p["gate_type"]] if p["gate"] is not None else None
    desc = D.make_norm_residual_desc(M, C, code, p["post"], p["pre"], p["alpha"], p["beta"], EPS, p["gate_rows"], p["gate_act"],
                                     gt[0] if gt else None, *([C + pad] * 5))
    new = lambda like=None: Rows(np.full((M, C) if like is None else like, 77.0), td, pad, off)  # noqa: E731
    x, z, y, h = Rows(p["x"], td, pad, off), Rows(p["z"], td, pad, off), new(), new()
    gate = Rows(p["gate"], gt[1], pad, off) if gt else None
    vs = [vec(p[n]) for n in ("post_gain", "post_bias", "pre_gain", "pre_bias")]
    stats = [torch.full((2 * M,), float("nan"), device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    D.dsp_norm_residual_forward(desc, x.view, z.view, gate.view if gate else None, *vs, y.view, h.view if p["pre"] else None, *stats,
                                stream=stream)
    ry, rh = P.forward(p)
    a = np.ones((M, C)) if not gt else P.act(p["act"] if "act" in p else p["gate_act"], p["gate"])[np.arange(M) // p["gate_rows"]]
    n = P.norm(p["post"], p["z"], p["post_gain"], p["post_bias"], EPS)
    na = np.abs(n) if not p["post"] else \
        (np.abs(p["z"]) + np.abs(p["z"].mean(1, keepdims=True))) * P.stats(p["post"], p["z"], EPS)[1] * (1 if p["post_gain"] is None else np.abs(p["post_gain"])) + (0 if p["post_bias"] is None else np.abs(p["post_bias"]))
    ya = np.abs(p["alpha"] * p["x"]) + np.abs(p["beta"] * a) * na
    gy = y.get()
    within(gy, ry, E * np.abs(ry) + 256 * U * ya + 1e-40, "y")
    if p["pre"]:
        mean, inv = P.stats(p["pre"], ry, EPS)
        gain = 1 if p["pre_gain"] is None else np.abs(p["pre_gain"])
        # what y is off by, and what the statistics are off by because of it
        ha = (ya + ya.mean(1, keepdims=True) + np.abs(ry - mean) * inv * inv * (ya * (np.abs(ry) + np.abs(mean))).mean(1, keepdims=True) / inv) * inv * gain
        within(h.get(), rh, E * np.abs(rh) + 600 * U * (ha + np.abs(rh)) + 1e-40, "h")
    for kind, u, s in ((p["post"], p["z"], stats[0]), (p["pre"], ry, stats[1])):
        if kind:
            mean, inv = P.stats(kind, u, EPS)
            got = s.cpu().numpy().astype(np.float64)
            mag = np.abs(u).mean(1) if kind == P.LAYER else np.zeros(M)
            ua = ya if u is ry else np.abs(u)
            within(got[:M], mean[:, 0], 400 * U * (mag + ua.mean(1)), "mean")
            spread = (ua * (np.abs(u) + np.abs(mean))).mean(1, keepdims=True) * inv ** 2
            within(got[M:], inv[:, 0], (400 * U * inv * (1 + spread))[:, 0], "deviation")

    # ---- backward, on y as stored and the statistics as kept
    st = [tuple(s.cpu().numpy().astype(np.float64)[i * M:(i + 1) * M, None] for i in range(2)) for s in stats]
    dy, dh, dx, dz = Rows(p["dy"], td, pad, off), Rows(p["dh"], td, pad, off), new(), new()
    dgate = Rows(np.full(p["gate"].shape, 77.0), gt[1], pad, off) if gt else None
    dv = [torch.full((C + 8,), 77.0, device="cuda") for _ in range(4)]
    nbytes = D.dsp_norm_residual_workspace_bytes(desc)
    ws = torch.full((nbytes + 64,), 77, dtype=torch.uint8, device="cuda")
    wanted = [bool(p["post"]), bool(p["post"]), bool(p["pre"]), bool(p["pre"])]
    torch.cuda.synchronize()

    def back(dx, dz, dgate, dv):
        D.dsp_norm_residual_backward(desc, dh.view if p["pre"] else None, dy.view, y.view, z.view, gate.view if gate else None, vs[0], vs[1], vs[2],
                                     *stats, dx.view, dz.view, dgate.view if dgate else None,
                                     *[v if w else None for v, w in zip(dv, wanted)], ws, nbytes, stream=stream)
    back(dx, dz, dgate, dv)
    ref = P.backward(p, gy, p["dy"], p["dh"], st[1], st[0])
    for name, got in (("x", dx), ("z", dz)):
        within(got.get(), ref[name], E * np.abs(ref[name]) + 400 * U * ref[name + "~"] + 1e-40, "d" + name)
    rows = 4 + -(-M // 512) + (p["gate_rows"] if p["gate"] is not None and p["gate_rows"] < M else 0)
    chain = (min(rows, M) + 116 + 400) * U
    if gt:
        within(dgate.get(), ref["gate"], gt[2] * np.abs(ref["gate"]) + chain * ref["gate~"] + 1e-40, "dgate")
    assert (ws[nbytes:] == 77).all(), "written behind the workspace"
    for name, v, w in zip(("post_gain", "post_bias", "pre_gain", "pre_bias"), dv, wanted):
        g = v.cpu().numpy().astype(np.float64)
        assert (g[C if w else 0:] == 77).all()
        if w:
            within(g[:C], ref[name], U * np.abs(ref[name]) + chain * ref[name + "~"] + 1e-40, "d" + name)
    return {"y": y, "h": h, "dx": dx, "dz": dz, "dgate": dgate, "dv": dv, "ref": ref, "desc": desc, "stats": stats, "back": back}


# (rows, elements): a row of 1, 2, 4 lanes .. several waves, ragged ones, more rows than workgroups
SHAPES = [(1, 1), (3, 2), (1, 4096), (37, 63), (300, 64), (2100, 65), (129, 128), (50, 255), (70, 257), (33, 512), (18, 1000), (5, 1431),
          (3, 4097), (2, 8192), (2, 8200), (1, 16384), (1500, 640)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%d" % s)
def test_shapes(shape, dtype):
    M, C = shape
    for k, (post, pre) in enumerate(((1, 1), (2, 2), (0, 1), (1, 0))):
        gate = [None, (M, "fp32"), (1, dtype), (max(2, M // 3), dtype)][(k + M) % 4]
        run(problem(M, C, dtype, post, pre, gate, k % 3, ("both", "gain", "none")[(k + C) % 3]), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post,pre", [(a, b) for a in range(3) for b in range(3)])
def test_norms_gates_and_strides(post, pre, dtype):
    M, C = 83, 200
    for gate in (None, (83, "fp32"), (1000, dtype), (1, dtype), (1, "fp32"), (7, dtype), (40, "fp32")):
        for act in (0, 1, 2) if gate and gate[0] in (1, 83) else (1,):
            for bias in ("both", "none"):
                run(problem(M, C, dtype, post, pre, gate, act, bias), dtype, pad=0 if act else 5, off=0 if act == 1 else 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C,rows", [(5000, 48, 2), (5000, 48, 17), (3000, 900, 1), (3000, 900, 3), (4096, 320, 64), (4100, 320, 1000)])
def test_more_rows_of_the_gate_than_workgroups(M, C, rows, dtype):
    run(problem(M, C, dtype, 1, 2, (rows, dtype), 1, "both"), dtype)


@pytest.mark.parametrize("C", [64, 1024])
def test_rows_whose_offsets_pass_32_bits(C):
    """Rows 20000 elements apart in tensors of 4.4e9: the first and the last ones against a call on those alone."""
    M, stride, td = 220000, 20000, torch.bfloat16
    wide = [torch.empty(M, stride, dtype=td, device="cuda")[:, :C] for _ in range(6)]   # x, z, y, h, then dx, dz
    gen = torch.Generator(device="cuda").manual_seed(1)
    for w in wide[:2]:
        w.copy_(torch.randn(M, C, generator=gen, device="cuda"))
    gate = torch.randn(M, C, generator=gen, device="cuda").to(td)
    gain = torch.ones(C, device="cuda")
    desc = lambda m, s: D.make_norm_residual_desc(m, C, D.DSP_BF16, 1, 2, 1.0, 0.5, EPS, 1, 1, None, s, s, s, s, C)  # noqa: E731
    stats = [torch.empty(2, M, device="cuda") for _ in range(2)]
    x, z, y, h, dx, dz = wide
    D.dsp_norm_residual_forward(desc(M, stride), x, z, gate, gain, None, gain, None, y, h, *stats)
    dgate = torch.empty_like(gate)
    ws = torch.empty(D.dsp_norm_residual_workspace_bytes(desc(M, stride)), dtype=torch.uint8, device="cuda")
    D.dsp_norm_residual_backward(desc(M, stride), h, x, y, z, gate, gain, None, gain, *stats, dx, dz, dgate, d_workspace=ws,
                                 workspace_bytes=ws.numel())
    torch.cuda.synchronize()
    for rows in (slice(0, 50), slice(M - 50, M)):
        small = [w[rows].contiguous() for w in (x, z, gate)]
        out = [torch.empty(50, C, dtype=td, device="cuda") for _ in range(5)]
        st = [torch.empty(2, 50, device="cuda") for _ in range(2)]
        D.dsp_norm_residual_forward(desc(50, 0), *small, gain, None, gain, None, out[0], out[1], *st)
        D.dsp_norm_residual_backward(desc(50, 0), out[1], small[0], out[0], small[1], small[2], gain, None, gain, *st, out[2], out[3], out[4],
                                     d_workspace=ws, workspace_bytes=ws.numel())
        torch.cuda.synchronize()
        for big, alone in zip((y, h, dx, dz, dgate), out):
            a, b = big[rows].float(), alone.float()
            # another row shape adds a row's elements up in another order: 200 U of a sum, and then the other bf16 neighbour
            assert (a - b).abs().max() <= 2.0 ** -7 * b.abs().max() and (a != b).float().mean() < 0.05
    for w in wide[2:]:
        assert torch.isfinite(w[::997]).all()


@pytest.mark.parametrize("dtype,C", [("bf16", c) for c in (300, 1024, 1499, 2048, 2500, 2904, 3500, 4096)] +
                         [("fp32", c) for c in (200, 500, 700, 1024, 1100, 1301, 1700, 2048)])
def test_every_number_of_runs_a_lane(dtype, C):
    """From 1024 rows on the forward pass takes a row a wave, one to eight runs a lane; the backward pass many rows a workgroup."""
    M = 1030 + C % 7
    run(problem(M, C, dtype, 2, 1, (1, dtype), 2, "both"), dtype)
    run(problem(M, C, dtype, 1, 2, (M, "fp32"), 1, "gain"), dtype, pad=8)
    run(problem(M, C, dtype, 0, 1, (300, dtype), 0, "none"), dtype, pad=1 if C % 2 else 0)


def test_rows_far_from_zero_keep_their_variance():
    run(problem(64, 1000, "fp32", 2, 2, None, 0, "both", shift=100.0), "fp32")


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_rows_and_rows_that_are_no_numbers(dtype):
    """A constant row (variance 0), a row of zeros, rows with an infinity or a NaN: the others do not notice."""
    code, td, E = TYPES[dtype]
    M, C = 9, 96
    p = problem(M, C, dtype, 2, 1, None, 0, "both")
    x = Rows(p["x"], td)
    bad = {1: np.inf, 4: np.nan}
    z = p["z"].copy()
    z[2], z[3] = 3.0, 0.0
    for r, v in bad.items():
        z[r, 7] = v
    outs = []
    for zz in (z, np.where(np.isin(np.arange(M), list(bad))[:, None], p["z"], z)):
        d = D.make_norm_residual_desc(M, C, code, 2, 1, p["alpha"], p["beta"], EPS)
        y, h, dz, dx = (Rows(np.zeros((M, C)), td) for _ in range(4))
        zd, dy, dh = Rows(zz, td), Rows(p["dy"], td), Rows(p["dh"], td)
        st = [torch.zeros(2 * M, device="cuda") for _ in range(2)]
        D.dsp_norm_residual_forward(d, x.view, zd.view, None, None, None, None, None, y.view, h.view, *st)
        D.dsp_norm_residual_backward(d, dh.view, dy.view, y.view, zd.view, None, None, None, None, *st, dx.view, dz.view)
        outs.append([t.get() for t in (y, h, dx, dz)])
    keep = ~np.isin(np.arange(M), list(bad))
    for a, b in zip(*outs):
        np.testing.assert_array_equal(a[keep], b[keep])
        assert np.isfinite(a[keep]).all() and np.isfinite(b).all()
    assert not np.isfinite(outs[0][0][list(bad)]).any()
    y = outs[0][0]  # N(constant) = 0 exactly for zeros; the mean of 96 threes is off by 90 U, over sqrt(eps)
    np.testing.assert_allclose(y[3], rounded(p["alpha"] * p["x"][3], td), rtol=2 * E)
    within(y[2], p["alpha"] * p["x"][2], 2 * E * np.abs(p["x"][2]) + 1.25 * 90 * U * 3 / np.sqrt(EPS), "constant row")


@pytest.mark.parametrize("dtype", TYPES)
def test_first_norm_of_a_stack(dtype):
    code, td, E = TYPES[dtype]
    M, C = 65, 300
    p = problem(M, C, dtype, 0, 2, None, 0, "both")
    p["z"] = None
    d = D.make_norm_residual_desc(M, C, code, pre=D.DSP_NORM_LAYER, eps=EPS)
    x, h, dh, dx = Rows(p["x"], td), Rows(np.zeros((M, C)), td), Rows(p["dh"], td), Rows(np.zeros((M, C)), td)
    gain, bias, stats = vec(p["pre_gain"]), vec(p["pre_bias"]), torch.zeros(2 * M, device="cuda")
    D.dsp_norm_residual_forward(d, x.view, d_pre_gain=gain, d_pre_bias=bias, d_h=h.view, d_pre_stats=stats)
    _, rh = P.forward(p)
    mean, inv = P.stats(2, p["x"], EPS)
    within(h.get(), rh, E * np.abs(rh) + 400 * U * ((np.abs(p["x"]) + np.abs(p["x"]).mean(1, keepdims=True)) * inv * np.abs(p["pre_gain"]) + np.abs(rh) + np.abs(p["pre_bias"])), "h")
    st = tuple(stats.cpu().numpy().astype(np.float64)[i * M:(i + 1) * M, None] for i in range(2))
    nbytes = D.dsp_norm_residual_workspace_bytes(d)
    ws, dg, db = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    p["alpha"] = 1.0
    for dy in (None, Rows(p["dy"], td)):
        D.dsp_norm_residual_backward(d, dh.view, None if dy is None else dy.view, x.view, None, None, None, None, gain, None, stats, dx.view,
                                     None, None, None, None, dg, db, ws, nbytes)
        ref = P.backward(p, p["x"], None if dy is None else p["dy"], p["dh"], st, None)
        within(dx.get(), ref["x"], E * np.abs(ref["x"]) + 400 * U * ref["x~"], "dx")
        within(dg.cpu().numpy(), ref["pre_gain"], 500 * U * ref["pre_gain~"] + 1e-40, "dgain")
        within(db.cpu().numpy(), ref["pre_bias"], 500 * U * ref["pre_bias~"] + 1e-40, "dbias")


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_without_what_is_not_asked_for(dtype):
    """y over x, dx over dy, dz over z; statistics not kept; outputs left out: the same bits in those that remain."""
    code, td, E = TYPES[dtype]
    M, C = 77, 264
    p = problem(M, C, dtype, 1, 2, (5, dtype), 2, "both")
    r = run(p, dtype)
    x, z, h = Rows(p["x"], td), Rows(p["z"], td), Rows(np.zeros((M, C)), td)
    gate = Rows(p["gate"], td)
    vs = [vec(p[n]) for n in ("post_gain", "post_bias", "pre_gain", "pre_bias")]
    d = D.make_norm_residual_desc(M, C, code, 1, 2, p["alpha"], p["beta"], EPS, 5, 2)
    D.dsp_norm_residual_forward(d, x.view, z.view, gate.view, *vs, x.view, h.view)
    np.testing.assert_array_equal(x.get(), r["y"].get())
    np.testing.assert_array_equal(h.get(), r["h"].get())
    dy, dh = Rows(p["dy"], td), Rows(p["dh"], td)
    D.dsp_norm_residual_backward(d, dh.view, dy.view, x.view, z.view, gate.view, vs[0], vs[1], vs[2], *r["stats"], dy.view, z.view)
    np.testing.assert_array_equal(dy.get(), r["dx"].get())
    np.testing.assert_array_equal(z.get(), r["dz"].get())
    ws = torch.empty(D.dsp_norm_residual_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    z, dy, dgate = Rows(p["z"], td), Rows(p["dy"], td), Rows(np.zeros(p["gate"].shape), td)
    D.dsp_norm_residual_backward(d, dh.view, dy.view, x.view, z.view, gate.view, vs[0], vs[1], vs[2], *r["stats"], None, None, dgate.view,
                                 d_workspace=ws, workspace_bytes=ws.numel())
    np.testing.assert_array_equal(dgate.get(), r["dgate"].get())
    one = torch.empty(C, device="cuda")
    D.dsp_norm_residual_backward(d, dh.view, dy.view, x.view, z.view, gate.view, vs[0], vs[1], vs[2], *r["stats"], None, None, None,
                                 None, one, None, None, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(one, r["dv"][1][:C])


def test_streams_and_replays():
    p = problem(700, 520, "bf16", 1, 1, (700, "fp32"), 0, "gain")
    a = run(p, "bf16")
    side = torch.cuda.Stream()
    b = run(p, "bf16", stream=side)
    for k in ("y", "h", "dx", "dz", "dgate"):
        np.testing.assert_array_equal(a[k].get(), b[k].get())
    # a captured backward pass, replayed on changing inputs
    graph = torch.cuda.CUDAGraph()
    dx, dz, dgate = (Rows(np.zeros(t.shape), t.td) for t in (b["dx"], b["dz"], b["dgate"]))
    dv = [torch.zeros_like(v) for v in b["dv"]]
    torch.cuda.synchronize()

    def whole(stream):
        desc = b["desc"]
        D.dsp_norm_residual_backward(desc, ins[0], ins[1], b["y"].view, ins[2], gate, gain, None, gain, *b["stats"], dx.view, dz.view, dgate.view,
                                     dv[0], None, dv[2], None, ws, ws.numel(), stream=stream)
    td = torch.bfloat16
    ins = [torch.from_numpy(p[n].astype(np.float32)).cuda().to(td) for n in ("dh", "dy", "z")]
    gate, gain = vec(p["gate"]), vec(p["post_gain"])
    ws = torch.empty(D.dsp_norm_residual_workspace_bytes(b["desc"]), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        whole(side)
    for i in range(4):
        ins[i % 2].mul_(1.5)
        torch.cuda.synchronize()
        whole(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want = [t.clone() for t in (dx.view, dz.view, dgate.view, dv[0], dv[2])]
        for t in (dx.view, dz.view, dgate.view, dv[0], dv[2]):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((dx.view, dz.view, dgate.view, dv[0], dv[2]), want):
            assert torch.equal(t, w), i


@pytest.mark.parametrize("post,pre", [(1, 1), (2, 2), (0, 2), (1, 0)])
def test_gradients_against_differences(post, pre):
    """The device's gradients along random directions against central differences of the definition in 64 bits.

    L = sum(cy y) + sum(ch h); the difference over +-1e-4 is off by 1e-8 / 6 of the third derivative (below 1e3 of L's scale
    here: rows of deviation near 1), the device's gradients by 600 U of their terms' magnitudes."""
    M, C = 40, 72
    p = problem(M, C, "fp32", post, pre, (7, "fp32"), 1, "both")
    p["x"], p["z"] = (np.float64(np.float32(a / a.std(1, keepdims=True))) for a in (p["x"], p["z"]))
    r = run(p, "fp32")
    rng = np.random.default_rng(5)
    got = {"x": r["dx"].get(), "z": r["dz"].get(), "gate": r["dgate"].get()}
    for name, v, has in zip(("post_gain", "post_bias", "pre_gain", "pre_bias"), r["dv"], (post, post, pre, pre)):
        if has:
            got[name] = v.cpu().numpy()[:C].astype(np.float64)
    for name, g in got.items():
        for _ in range(3):
            t = rng.standard_normal(p[name].shape)

            def value(s):
                y, h = P.forward({**p, name: p[name] + s * t})
                return (p["dy"] * y).sum() + ((p["dh"] * h).sum() if pre else 0.0)
            diff = (value(1e-4) - value(-1e-4)) / 2e-4
            mags = np.abs(t * r["ref"][name + "~"]).sum()
            assert abs((g * t).sum() - diff) <= (1000 * U + 1e-7) * mags + 1e-5 * abs(diff), name


def test_a_residual_stack_trains():
    """Norm, linear branch, gate and residual sum, cross-entropy and AdamW as a program strings them together: three steps against
    the same in 64 bits (autograd of the definitions).  In fp32 the rounding of a step is below 1e-5 of each gradient's size."""
    L, M, C, K = 3, 96, 40, 10
    rng = np.random.default_rng(11)
    P0 = {}
    for l in range(L):
        P0["w%d" % l], P0["b%d" % l] = rng.standard_normal((C, C)) / np.sqrt(C), np.zeros(C)
        P0["post%d" % l], P0["pre%d" % l], P0["gate%d" % l] = np.ones(C), np.ones(C), np.full((1, C), 0.5)
    P0["pre%d" % L], P0["head"], P0["hb"] = np.ones(C), rng.standard_normal((K, C)) / np.sqrt(C), np.zeros(K)
    P0 = {k: v.astype(np.float32) for k, v in P0.items()}
    x0, labels = rng.standard_normal((M, C)).astype(np.float32), rng.integers(0, K, M).astype(np.int32)
    dev = {k: torch.from_numpy(v).cuda() for k, v in P0.items()}
    grad = {k: torch.zeros_like(v) for k, v in dev.items()}
    mv = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in dev.items()}
    opt = D.dsp_adamw_init([{"param": dev[k], "grad": grad[k], "m": mv[k][0], "v": mv[k][1], "decay": dev[k].dim() == 2 and k[:4] != "gate"}
                            for k in dev])
    ref = {k: torch.from_numpy(v).double().requires_grad_() for k, v in P0.items()}
    rm = {k: [np.zeros(v.shape), np.zeros(v.shape)] for k, v in P0.items()}
    new = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    first = D.make_norm_residual_desc(M, C, D.DSP_FP32, pre=1)
    mid = D.make_norm_residual_desc(M, C, D.DSP_FP32, 1, 1, 1.0, 1.0, 1e-5, M)
    nbytes = D.dsp_norm_residual_workspace_bytes(mid)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    x, lab = torch.from_numpy(x0).cuda(), torch.from_numpy(labels).cuda()
    try:
        for t in (1, 2, 3):
            ys, hs, zs, posts, pres = [x], [new(M, C)], [], [], [new(2, M)]
            D.dsp_norm_residual_forward(first, x, d_pre_gain=dev["pre0"], d_h=hs[0], d_pre_stats=pres[0])
            for l in range(L):
                z, y, h, ps, qs = new(M, C), new(M, C), new(M, C), new(2, M), new(2, M)
                D.dsp_linear_forward(hs[l], dev["w%d" % l], dev["b%d" % l], z, M, C, C)
                D.dsp_norm_residual_forward(mid, ys[l], z, dev["gate%d" % l], dev["post%d" % l], None, dev["pre%d" % (l + 1)], None, y, h, ps, qs)
                for lst, v in ((ys, y), (hs, h), (zs, z), (posts, ps), (pres, qs)):
                    lst.append(v)
            logits, loss, dl, row = new(M, K), new(1), new(M, K), new(M)
            D.dsp_linear_forward(hs[L], dev["head"], dev["hb"], logits, M, C, K)
            D.dsp_softmax_ce(logits, lab, loss, dl, row, M, K)
            dh, dy = new(M, C), None
            D.dsp_linear_backward(hs[L], dev["head"], dl, dh, grad["head"], grad["hb"], M, C, K)
            for l in reversed(range(L)):
                dx, dz = new(M, C), new(M, C)
                D.dsp_norm_residual_backward(mid, dh, dy, ys[l + 1], zs[l], dev["gate%d" % l], dev["post%d" % l], None, dev["pre%d" % (l + 1)],
                                             posts[l], pres[l + 1], dx, dz, grad["gate%d" % l], grad["post%d" % l], None,
                                             grad["pre%d" % (l + 1)], None, ws, nbytes)
                dh, dy = new(M, C), dx
                D.dsp_linear_backward(hs[l], dev["w%d" % l], dz, dh, grad["w%d" % l], grad["b%d" % l], M, C, C)
            D.dsp_norm_residual_backward(first, dh, dy, x, None, None, None, None, dev["pre0"], None, pres[0], None, None, None, None, None,
                                         grad["pre0"], None, ws, nbytes)
            norm = new(1)
            D.dsp_adamw_step(opt, 1e-3, weight_decay=0.1, max_norm=0.5, d_norm=norm)
            torch.cuda.synchronize()

            rms = lambda u, g: u * torch.rsqrt(u.square().mean(1, keepdim=True) + 1e-5) * g  # noqa: E731
            u = torch.from_numpy(x0).double()
            for l in range(L):
                b = rms(u, ref["pre%d" % l]) @ ref["w%d" % l].t() + ref["b%d" % l]
                u = u + ref["gate%d" % l] * rms(b, ref["post%d" % l])
            o = rms(u, ref["pre%d" % L]) @ ref["head"].t() + ref["hb"]
            want = -torch.log_softmax(o, 1)[torch.arange(M), torch.from_numpy(labels).long()].mean()
            gs = dict(zip(ref, torch.autograd.grad(want, list(ref.values()))))
            assert abs(float(loss) - float(want)) < 1e-5 * abs(float(want))
            total = float(torch.sqrt(sum(g.square().sum() for g in gs.values())))
            assert abs(float(norm) - total) < 1e-5 * total
            c = min(1.0, 0.5 / total)
            for k in ref:
                g = gs[k].numpy()
                err = np.abs(grad[k].cpu().numpy() - g).max()
                assert err < 1e-5 * max(np.abs(g).max(), 1e-3 * total), (t, k, err)
                decay = 0.1 if ref[k].dim() == 2 and k[:4] != "gate" else 0.0
                # the device's own gradient: where it is close to zero its sign decides the first step
                nx, rm[k][0], rm[k][1] = P.adamw(ref[k].detach().numpy(), c * grad[k].cpu().numpy().astype(np.float64), *rm[k], t, 1e-3, 0.9, 0.999, 1e-8, decay)
                assert np.abs(dev[k].cpu().numpy() - nx).max() < 1e-4 * 1e-3 + 4 * U * np.abs(nx).max(), (t, k)
                ref[k] = torch.from_numpy(dev[k].cpu().numpy()).double().requires_grad_()
    finally:
        D.dsp_adamw_destroy(opt)


@pytest.mark.parametrize("dtype,M,C", [("bf16", 1100, c) for c in (4104, 5001, 8192, 8200)] + [("bf16", 600, 12288)] +
                         [("fp32", 1100, c) for c in (2049, 3000, 4104, 5001)] + [("fp32", 600, c) for c in (8192, 8200, 12288)])
def test_many_rows_of_several_waves(dtype, M, C):
    """Rows longer than a wave's, more of them than workgroups: a workgroup goes on to its second and third row, and the column sums
    have many parts."""
    wide = {"fp32": 12288, "bf16": 12288}[dtype] == C
    gates = [None, (M, "fp32"), (1, dtype), (300, dtype), (3, dtype)]
    for i, (post, pre) in enumerate(((2, 2), (1, 1)) if not wide else ((2, 2),)):
        run(problem(M, C, dtype, post, pre, gates[(C + 3 * i + (dtype == "fp32")) % 5], (C + i) % 3, ("both", "gain")[i]), dtype, pad=8 * i, off=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", [(5, 32), (5, 256), (300, 256), (5, 1024), (1100, 1024), (1100, 2048), (5, 4096), (3, 8192), (3, 16384)])
def test_constant_rows_are_exactly_zero_once_centred(M, C, dtype):
    """Row sums of whole numbers below 2^24 and the quotient by a power of two are exact, so is the mean, and u - mean is 0: N(u) is the
    bias, and nothing of the row reaches the gradients of gain and gate."""
    code, td, E = TYPES[dtype]
    rows = np.broadcast_to((8.0 * (125 - 5 * (np.arange(M) % 7)))[:, None], (M, C))
    rng = np.random.default_rng(C)
    bias, g = vec(rng.standard_normal(C)), Rows(rng.standard_normal((M, C)), td)
    u, h, dx, zero = Rows(rows, td), Rows(np.ones((M, C)), td), Rows(np.ones((M, C)), td), Rows(np.zeros((M, C)), td)
    gain, stats = vec(1 + rng.standard_normal(C)), torch.zeros(2 * M, device="cuda")
    ws = torch.empty(1024 * 16 * C, dtype=torch.uint8, device="cuda")
    dg = torch.ones(C, device="cuda")
    d = D.make_norm_residual_desc(M, C, code, pre=D.DSP_NORM_LAYER, eps=EPS)  # in front of the next block
    D.dsp_norm_residual_forward(d, u.view, d_pre_gain=gain, d_pre_bias=bias, d_h=h.view, d_pre_stats=stats)
    assert np.array_equal(h.get(), np.broadcast_to(rounded(bias.cpu().numpy(), td), (M, C)))
    assert np.array_equal(stats[:M].cpu().numpy(), rows[:, 0])
    D.dsp_norm_residual_backward(d, g.view, None, u.view, None, None, None, None, gain, None, stats, dx.view, None, d_dpre_gain=dg, d_workspace=ws,
                                 workspace_bytes=ws.numel())
    assert not dg.any()
    for gate_rows in (0, 1, M):  # behind the branch
        gate = Rows(np.ones((-(-M // max(gate_rows, 1)), C)), td) if gate_rows else None
        dgate = Rows(np.ones(gate.shape), td) if gate else None
        d = D.make_norm_residual_desc(M, C, code, post=D.DSP_NORM_LAYER, beta=-1.25, eps=EPS, gate_rows=gate_rows, gate_act=1)
        y = Rows(np.ones((M, C)), td)
        D.dsp_norm_residual_forward(d, zero.view, u.view, gate.view if gate else None, gain, d_y=y.view, d_post_stats=stats)
        assert not y.get().any()
        D.dsp_norm_residual_backward(d, None, g.view, None, u.view, gate.view if gate else None, gain, None, None, stats, None, None, dx.view,
                                     dgate.view if gate else None, dg.fill_(1.0), d_workspace=ws, workspace_bytes=ws.numel())
        assert not dg.any() and not (gate and dgate.get().any())


@pytest.mark.parametrize("M,C", [(7, 40), (7, 700), (1100, 700), (3, 5000)])
@pytest.mark.parametrize("act", [1, 2], ids=["sigmoid", "tanh"])
def test_gates_far_from_zero(act, M, C):
    """The activation and its derivative relative to themselves, down to where they leave the floats, at infinities and at NaN.

    exp(-a): the product with log2(e) is held in two parts, the hardware's power of two is off by 2 U and the correction rounds once: 3 U.
    Its quotients with 1 + e (U, the reciprocal 2 U): sigmoid at most 3 + 1 + 2 + 1 U; tanh (1 - e) / (1 + e) from 1/4 on, where
    2 e / (1 - e^2) < 2: 6 + 1 + 1 + 2 + 1 U; both derivatives 3 + 2 (1 + 2) + 2 U.  An exp(-a) below 2^-126 may
    be 0 (the hardware's results are normal numbers or 0), and tanh' = 4 exp(-2 |g|) q^2 loses up to 4 times that."""
    rng = np.random.default_rng(act * 1000 + C)
    g = np.exp(rng.uniform(np.log(1e-4), np.log(100.0), (M, C))) * rng.choice([-1.0, 1.0], (M, C))
    special = [np.inf, -np.inf, np.nan, 0.0, -0.0, 1e30, -1e30, 3e38, 0.25, -0.25, 43.5, -87.0, 87.4, -88.0, 1e-30]
    g[0, :15], g[M - 1, C - 15:] = special, special
    g = rounded(g, torch.float32)
    with np.errstate(all="ignore"):
        a, s = P.act(act, g), P.slope(act, g)
        s = np.where(np.isinf(g), 0.0, s)
    tiny = 2.0 ** -126 * (4 if act == 2 else 1)
    one, out = Rows(np.ones((M, C)), torch.float32), [Rows(np.zeros((M, C)), torch.float32) for _ in range(3)]
    x, (y, dz, dgate) = Rows(np.zeros((M, C)), torch.float32), out

    def check(got, ref, n, what):
        assert np.array_equal(np.isnan(got), np.isnan(ref)), what
        off = np.abs(got - ref) / (n * U * np.abs(ref) + tiny)
        assert not (off > 1).any(), (what, float(np.nanmax(off)), g.flat[np.nanargmax(off)])
    d = D.make_norm_residual_desc(M, C, D.DSP_FP32, gate_rows=1, gate_act=act)
    gate = Rows(g, torch.float32)
    D.dsp_norm_residual_forward(d, x.view, one.view, gate.view, d_y=y.view)
    check(y.get(), a, 12, "activation")
    D.dsp_norm_residual_backward(d, None, one.view, None, one.view, gate.view, None, None, None, None, None, None, dz.view, dgate.view)
    check(dz.get(), a, 12, "dz")
    check(dgate.get(), s, 12, "derivative")
    # one row of the gate for all: its derivative from the column sums
    d = D.make_norm_residual_desc(1, C, D.DSP_FP32, gate_rows=1, gate_act=act)
    ws = torch.empty(D.dsp_norm_residual_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    line = [Rows(v, torch.float32) for v in (np.zeros((1, C)), np.ones((1, C)), g[:1], np.zeros((1, C)), np.zeros((1, C)))]
    D.dsp_norm_residual_forward(d, line[0].view, line[1].view, line[2].view, d_y=line[3].view)
    D.dsp_norm_residual_backward(d, None, line[1].view, None, line[1].view, line[2].view, None, None, None, None, None, None, None, line[4].view,
                                 d_workspace=ws, workspace_bytes=ws.numel())
    check(line[3].get(), a[:1], 12, "activation of a vector")
    check(line[4].get(), s[:1], 12, "derivative of a vector")
