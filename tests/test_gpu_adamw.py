"""AdamW over many tensors against its definition in 64 bits, states of 32 and of 8 bits, alone and as the update of blocks.

U = 2^-24 is half a step of fp32.  A moment is a sum of two products of rounded constants: each term carries at most 4 roundings
(the constant, a clipped gradient's factor, one or two products) and the sum one more, so 6 U of the terms' magnitudes; the clip
factor itself (norm rounded, quotient rounded) adds 2 U, 4 U in v.  The step m c1 / (sqrt(v) c2 + eps) multiplies relative
errors: those of m and half of v's, and at most 10 more roundings; lr, the decay term and the difference add 4.
8-bit codes and exponents are equal: the moments are formed with one fp32 rounding per operation, which numpy repeats."""
import numpy as np
import pytest
import torch

import paper_1909_02625_amd as D
from tests import plain_operators as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


class Model:
    """Tensors of the given sizes, some of them off the 16-byte addresses, with guards behind them."""

    def __init__(self, sizes, bits, grad, seed=0, copy=True, off=0, opt_seed=12345678901):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits, self.opt_seed, self.host, self.dev, self.all = sizes, bits, opt_seed, [], [], []
        for j, n in enumerate(sizes):
            s = 10.0 ** rng.uniform(-5, 0)
            g = (rng.standard_normal(n) * s).astype(np.float32)
            if grad == torch.bfloat16:
                g = torch.from_numpy(g).bfloat16().float().numpy()
            h = {"x": rng.standard_normal(n).astype(np.float32), "g": g, "decay": j % 3 != 1}
            m, v = (0.3 * s * rng.standard_normal(n)).astype(np.float32), (s * s * rng.random(n)).astype(np.float32)
            if bits == 8:
                zero = np.zeros(n)
                h["m"], h["m_exp"] = P.encode(m, zero, 3, 7, 7, False)
                h["v"], h["v_exp"] = P.encode(v, zero, 2, 15, 14, True)
            else:
                h["m"], h["v"] = m, v
            self.host.append(h)

            def put(a, dtype):
                t = torch.full((a.size + off + 8,), 77, dtype=dtype, device="cuda")
                t[off:off + a.size] = torch.from_numpy(a).to("cuda").to(dtype)
                self.all.append((t, a.size))
                return t[off:off + a.size]
            st = torch.uint8 if bits == 8 else torch.float32
            d = {"param": put(h["x"], torch.float32), "grad": put(h["g"], grad), "m": put(h["m"], st), "v": put(h["v"], st), "decay": h["decay"]}
            if copy and j % 2 == 0:
                d["copy"] = put(np.zeros(n, np.float32), torch.bfloat16)
            if bits == 8:
                d["m_exp"], d["v_exp"] = put(h["m_exp"], torch.uint8), put(h["v_exp"], torch.uint8)
            self.dev.append(d)
        self.off = off
        self.opt = D.dsp_adamw_init(self.dev, bits, opt_seed)

    def guards(self):
        torch.cuda.synchronize()
        for t, n in self.all:
            f = t.float()
            assert (f[:self.off] == 77).all() and (f[self.off + n:] == 77).all(), "written outside a tensor"

    def check(self, t, max_norm=0.0):
        """The device's tensors after step t (one step from self.host) against the definition; takes them over as the new start."""
        self.guards()
        norm, c = P.clip_factor([h["g"] for h in self.host], max_norm)
        k = 2 if c != 1.0 else 0
        for j, (h, d) in enumerate(zip(self.host, self.dev)):
            n = h["x"].size
            m0, v0 = h["m"], h["v"]
            if self.bits == 8:
                m0, v0 = P.decode(m0, h["m_exp"], 3, 7), P.decode(v0, h["v_exp"], 2, 15)
            wd = HYPER["weight_decay"] if h["decay"] else 0.0
            x, m, v = P.adamw(h["x"], c * h["g"].astype(np.float64), m0, v0, t, HYPER["lr"], 0.9, 0.999, HYPER["eps"], wd)
            got = {name: d[name].cpu().float().numpy().astype(np.float64) if name in ("param", "copy") else d[name].cpu().numpy()
                   for name in d if name not in ("grad", "decay")}
            mt, vt = 0.9 * np.abs(m0) + 0.1 * c * np.abs(h["g"]), v
            em, ev = (6 + k) * U * mt, (7 + 2 * k) * U * vt
            root = np.sqrt(v / (1 - 0.999 ** t)) + HYPER["eps"]
            step = np.abs(m) / (1 - 0.9 ** t) / root
            ex = HYPER["lr"] * (em / (1 - 0.9 ** t) / root + step * (4 + k + 10) * U + 4 * U * wd * np.abs(h["x"])) + 2 * U * (np.abs(x) + HYPER["lr"] * step)
            assert (np.abs(got["param"] - x) <= ex + 1e-45).all(), (j, n, float(np.max(np.abs(got["param"] - x) / ex)))
            if self.bits == 32:
                assert (np.abs(got["m"] - m) <= em + 1e-45).all() and (np.abs(got["v"] - v) <= ev + 1e-45).all(), (j, n)
            elif c == 1.0:
                m32, v32 = P.moments_fp32(h["g"], m0, v0, 0.9, 0.999)
                low, high = P.random_halves(self.opt_seed, t, j, n)
                for name, a, r, args in (("m", m32, low, (3, 7, 7, False)), ("v", v32, high, (2, 15, 14, True))):
                    code, e = P.encode(a, r, *args)
                    np.testing.assert_array_equal(got[name + "_exp"], e)
                    np.testing.assert_array_equal(got[name], code)
            else:  # half a code's distance is what a clip factor's rounding may decide: neighbouring codes, and few of them
                for name, a, args in (("m", m, (3, 7)), ("v", v, (2, 15))):
                    value, mant = P.decode(got[name], got[name + "_exp"], *args), args[0]
                    gap = np.maximum(np.abs(a) * 2.0 ** -mant, np.ldexp(1.0, np.repeat(got[name + "_exp"].astype(int), 256)[:n] - 127 + 1 - args[1] - mant))
                    assert (np.abs(value - a) <= gap * (1 + 1e-5)).all(), (j, name)
            if "copy" in got:
                assert np.array_equal(got["copy"], torch.from_numpy(got["param"].astype(np.float32)).bfloat16().float().numpy())
            h["x"] = got["param"].astype(np.float32)
            for name in ("m", "v", "m_exp", "v_exp"):
                if name in got:
                    h[name] = got[name]
        return norm

    def __del__(self):
        if getattr(self, "opt", None):
            D.dsp_adamw_destroy(self.opt)


SIZES = [1, 2, 3, 5, 63, 64, 255, 256, 257, 1000, 4095, 4096, 4097, 12345]


@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps(bits, grad, off):
    m = Model(SIZES, bits, grad, seed=bits + off, off=off)
    for t in (1, 2, 3):
        D.dsp_adamw_step(m.opt, **HYPER)
        m.check(t)
    assert D.dsp_adamw_get_steps(m.opt) == 3
    D.dsp_adamw_set_steps(m.opt, 5000)
    D.dsp_adamw_step(m.opt, **HYPER)
    m.check(5001)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [1e-3, 1e6])
def test_clip_by_the_norm_of_all_gradients(bits, max_norm):
    m = Model(SIZES + [300001], bits, torch.bfloat16, seed=7)
    out = torch.zeros(1, device="cuda")
    for t in (1, 2):
        D.dsp_adamw_step(m.opt, **HYPER, max_norm=max_norm, d_norm=out)
        norm = m.check(t, max_norm)
        assert abs(float(out) - norm) <= 2 * U * norm
    out.zero_()
    D.dsp_adamw_step(m.opt, **HYPER, d_norm=out)  # the norm alone
    assert abs(float(out) - m.check(3)) <= 2 * U * norm


@pytest.mark.parametrize("bits", [32, 8])
def test_many_small_tensors_and_a_large_one(bits):
    rng = np.random.default_rng(3)
    m = Model([int(n) for n in rng.integers(1, 700, 400)] + [2000003], bits, torch.float32, seed=5, copy=False)
    D.dsp_adamw_step(m.opt, **HYPER)
    m.check(1)


def test_more_elements_than_32_bits_count():
    """Elements on both sides of 2^32 of one tensor, and its last ones."""
    n = (1 << 32) + 70001
    x, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    me, ve = (torch.zeros(-(-n // 256), dtype=torch.uint8, device="cuda") for _ in range(2))
    rng = np.random.default_rng(8)
    places = [(0, 2560), ((1 << 31) - 512, 1024), ((1 << 32) - 1024, 2048), (n // 256 * 256 - 2048, n - n // 256 * 256 + 2048)]
    host = []
    for at, k in places:
        a = torch.from_numpy(rng.standard_normal(k).astype(np.float32)).bfloat16()
        g[at:at + k] = a.cuda()
        host.append(a.float().numpy())
    o = D.dsp_adamw_init([{"param": x, "grad": g, "m": m, "v": v, "m_exp": me, "v_exp": ve}], 8, 77)
    norm = torch.zeros(1, device="cuda")
    D.dsp_adamw_step(o, 1e-3, d_norm=norm)
    torch.cuda.synchronize()
    D.dsp_adamw_destroy(o)
    total = P.clip_factor(host, 0)[0]
    assert abs(float(norm) - total) <= 2 * U * total
    for (at, k), a in zip(places, host):
        low, high = P.random_halves(77, 1, 0, k, first=at)
        m32, v32 = P.moments_fp32(a, np.zeros(k), np.zeros(k), 0.9, 0.999)
        for code, exp, val, r, args in ((m, me, m32, low, (3, 7, 7, False)), (v, ve, v32, high, (2, 15, 14, True))):
            c, e = P.encode(val, r, *args)
            np.testing.assert_array_equal(code[at:at + k].cpu().numpy(), c)
            np.testing.assert_array_equal(exp[at // 256:at // 256 + e.size].cpu().numpy(), e)
        # the first step of AdamW is lr g / |g| (1 - eps / |g| ...): 20 roundings
        ref = -1e-3 * a / (np.abs(a.astype(np.float64)) + 1e-8)
        assert np.abs(x[at:at + k].cpu().numpy() - ref).max() <= 20 * U * 1e-3
    at, k = places[1]
    assert not x[at + k:at + k + 4096].any() and not m[at + k:at + k + 4096].any()


def test_new_moments_of_8_bits():
    """From zero moments: every code stands for one of the two neighbours of its value, and none is favoured."""
    n = 1 << 20
    rng = np.random.default_rng(1)
    g = (rng.standard_normal(n) * np.exp(rng.standard_normal(n))).astype(np.float32)
    z = lambda k, dt: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    d = {"param": z(n, torch.float32), "grad": torch.from_numpy(g).cuda(), "m": z(n, torch.uint8), "v": z(n, torch.uint8),
         "m_exp": z(n // 256, torch.uint8), "v_exp": z(n // 256, torch.uint8)}
    o = D.dsp_adamw_init([d], 8, 99)
    D.dsp_adamw_step(o, **HYPER)
    D.dsp_adamw_destroy(o)
    m32, v32 = P.moments_fp32(g, np.zeros(n), np.zeros(n), 0.9, 0.999)
    for name, a, args in (("m", m32, (3, 7)), ("v", v32, (2, 15))):
        a = a.astype(np.float64)
        exps = d[name + "_exp"].cpu().numpy()
        got = P.decode(d[name].cpu().numpy(), exps, *args)
        gap = np.maximum(np.abs(a) * 2.0 ** -args[0], np.ldexp(1.0, np.repeat(exps.astype(int), 256) - 127 + 1 - args[1] - args[0]))
        assert (np.abs(got - a) <= gap).all()
        if name == "v":
            assert (got[a > 0] > 0).all()
        # an error of mean 0 and variance at most gap^2 / 4: six standard deviations of the mean, and the 2^-17 of a gap that
        # sixteen random bits leave
        large = np.abs(a) > 2.0 ** -8 * np.abs(a).reshape(-1, 256).max(1).repeat(256)
        rel = ((got - a) / gap)[large]
        assert abs(rel.mean()) < 3.0 / np.sqrt(rel.size) + 2.0 ** -16, (name, rel.mean())


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_no_numbers_stay_where_they_are(bits):
    m = Model([1000], bits, torch.float32, seed=2)
    bad = [5, 300, 301, 999]
    vals = [np.inf, np.nan, -np.inf, 1e30]
    before = [h.copy() for h in (m.host[0]["x"], m.host[0]["m"], m.host[0]["v"])]
    g = m.host[0]["g"]
    g[bad] = vals
    m.dev[0]["grad"].copy_(torch.from_numpy(g).cuda())
    norm = torch.zeros(1, device="cuda")
    D.dsp_adamw_step(m.opt, **HYPER, max_norm=1.0, d_norm=norm)  # no finite norm: nothing happens
    m.guards()
    assert not np.isfinite(float(norm)) and D.dsp_adamw_get_steps(m.opt) == 0
    for name, b in zip(("param", "m", "v"), before):
        assert np.array_equal(m.dev[0][name].cpu().numpy(), b)
    D.dsp_adamw_step(m.opt, **HYPER)
    m.guards()
    assert D.dsp_adamw_get_steps(m.opt) == 1
    x = m.dev[0]["param"].cpu().numpy()
    good = np.ones(1000, bool)
    good[bad] = False
    assert np.isnan(x[bad[:3]]).all() and np.isfinite(x[good]).all()
    if bits == 8:
        c = m.dev[0]["m"].cpu().numpy()
        assert ((c[bad[:3]] & 127) == 127).all() and ((c[good] & 127) < 127).all()
        cv = m.dev[0]["v"].cpu().numpy()
        assert (cv[bad] == 127).all() and (cv[good] < 124).all()   # (1e30 squared leaves the floats)
        D.dsp_adamw_step(m.opt, **HYPER)
        assert np.isfinite(m.dev[0]["param"].cpu().numpy()[good]).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [0.0, 0.5])
def test_replays_of_a_captured_step_count_on(bits, max_norm):
    a, b = (Model(SIZES, bits, torch.float32, seed=4) for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        D.dsp_adamw_step(a.opt, **HYPER, max_norm=max_norm)
    assert D.dsp_adamw_get_steps(a.opt) == 0
    for t in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        D.dsp_adamw_step(b.opt, **HYPER, max_norm=max_norm)
        torch.cuda.synchronize()
        assert D.dsp_adamw_get_steps(a.opt) == D.dsp_adamw_get_steps(b.opt) == t
        for p, q in zip(a.dev, b.dev):
            for name in ("param", "m", "v"):
                assert torch.equal(p[name], q[name]), (t, name)
            p["grad"].mul_(0.5)
            q["grad"].mul_(0.5)


def test_the_same_call_gives_the_same_bits_on_another_stream():
    a, b = (Model(SIZES + [1000003], 8, torch.bfloat16, seed=9) for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        D.dsp_adamw_step(a.opt, **HYPER, max_norm=1.0)
        D.dsp_adamw_step(b.opt, **HYPER, max_norm=1.0, stream=side)
    torch.cuda.synchronize()
    for p, q in zip(a.dev, b.dev):
        for name in ("param", "m", "v", "m_exp", "v_exp"):
            assert torch.equal(p[name], q[name])


def test_hyperparameters_that_are_refused():
    m = Model([10], 32, torch.float32)
    nan, inf = float("nan"), float("inf")
    for bad in ({"lr": -1e-3}, {"lr": nan}, {"lr": inf}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": nan}, {"eps": 0.0}, {"eps": 1e-16},
                {"eps": nan}, {"weight_decay": -1.0}, {"weight_decay": inf}, {"max_norm": -1.0}, {"max_norm": nan}, {"max_norm": 1e-60}):
        with pytest.raises(D.DSPError) as e:
            D.dsp_adamw_step(m.opt, **{**HYPER, **bad})
        assert e.value.status == 1
    for steps, b1 in ((-1, 0.9), (3, 1.0)):
        with pytest.raises(D.DSPError):
            D.dsp_adamw_set_steps(m.opt, steps, b1)
    assert D.dsp_adamw_get_steps(m.opt) == 0
    D.dsp_adamw_step(m.opt, **HYPER)
    m.check(1)


def test_tensors_of_no_elements():
    z = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    o = D.dsp_adamw_init([{"param": z(0), "grad": z(0), "m": z(0), "v": z(0)}])
    norm = torch.ones(1, device="cuda")
    D.dsp_adamw_step(o, 1e-3, d_norm=norm)
    assert float(norm) == 0 and D.dsp_adamw_get_steps(o) == 1
    D.dsp_adamw_destroy(o)


def test_betas_that_change():
    """beta^t is the product over the steps taken."""
    n = 512
    rng = np.random.default_rng(6)
    g = rng.standard_normal(n).astype(np.float32)
    z = lambda: torch.zeros(n, device="cuda")  # noqa: E731
    d = {"param": z(), "grad": torch.from_numpy(g).cuda(), "m": z(), "v": z()}
    o = D.dsp_adamw_init([d])
    betas = [(0.9, 0.999), (0.5, 0.9), (0.0, 0.0), (0.8, 0.99)]
    x = m = v = np.zeros(n)
    p1 = p2 = 1.0
    for b1, b2 in betas:
        D.dsp_adamw_step(o, 1e-2, b1, b2)
        p1, p2 = p1 * b1, p2 * b2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g.astype(np.float64) ** 2
        x = x - 1e-2 * (m / (1 - p1)) / (np.sqrt(v / (1 - p2)) + 1e-8)
    got = d["param"].cpu().numpy()
    D.dsp_adamw_destroy(o)
    # four steps of 1e-2 and at most 30 roundings each
    assert np.abs(got - x).max() <= 4 * 30 * U * 1e-2 * 1.5 + 4 * U * np.abs(x).max()


# ---- as the update of blocks and pipelines
def _cfg():
    from workloads import get_config, make_params
    cfg = get_config("tiny2")
    rng = np.random.default_rng(cfg["seed"])
    return cfg, [make_params(layers, rng) for layers in cfg["blocks"]], rng


@pytest.mark.parametrize("dtype", [D.DSP_FP32, D.DSP_BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_block_update(bits, dtype):
    """The block's own gradient, parameters and decay rule through the definition; its next forward pass uses the new parameters."""
    from workloads import flatten_params
    from workloads.configs import param_shapes
    from tests.gpu_harness import block_shapes, build_gpu_blocks, destroy_blocks, to_dev, torch_dtype
    cfg, params, rng = _cfg()
    shapes = block_shapes(cfg)
    blocks = build_gpu_blocks(cfg, params, dtype, m=[0] * cfg["K"], standalone=True)
    try:
        b, layers = blocks[0], cfg["blocks"][0]
        with pytest.raises(D.DSPError) as e:
            D.dsp_param_update_adamw(b, 1e-2)
        assert e.value.status == 2
        D.dsp_block_set_adamw(b, bits, 17)
        with pytest.raises(D.DSPError) as e:
            D.dsp_block_set_adamw(b, bits, 17)
        assert e.value.status == 2
        x = to_dev(rng.standard_normal(shapes[0]).astype(np.float32), dtype)
        out = torch.empty(int(np.prod(shapes[1])), device="cuda", dtype=torch_dtype(dtype) if len(shapes[1]) == 4 else torch.float32)
        gout = torch.from_numpy(rng.standard_normal(out.numel()).astype(np.float32) * 0.1).cuda().to(out.dtype)
        decay = np.concatenate([np.full(int(np.prod(s)), name == "w") for ps in param_shapes(layers) for name, s in ps])
        p0 = flatten_params(layers, params[0]).astype(np.float32)
        np.testing.assert_array_equal(D.dsp_block_get_params(b), p0)
        m = v = np.zeros(p0.size)
        outs = []
        for t in (1, 2):
            D.dsp_block_forward(b, t - 1, x, out)
            outs.append(out.float().cpu().numpy())
            D.dsp_block_recompute_backward(b, t - 1, gout, None)
            g = D.dsp_block_get_grads(b).astype(np.float64)
            norm, c = P.clip_factor([g], 0.3)
            D.dsp_param_update_adamw(b, 1e-2, weight_decay=0.1, max_norm=0.3)
            if bits == 8 and t == 2:
                break   # (codes are compared above; here the step with fresh moments)
            ref, m, v = P.adamw(p0, c * g, m, v, t, 1e-2, 0.9, 0.999, 1e-8, np.where(decay, 0.1, 0.0))
            got = D.dsp_block_get_params(b)
            # |step| <= 1 / (1 - 0.9) for two steps, 40 roundings
            assert np.abs(got - ref).max() <= 40 * U * 1e-2 * 10 + 2 * U * np.abs(ref).max()
            p0 = got
        assert not np.array_equal(outs[0], outs[1])
        assert D.dsp_block_query(b)["version"] == 2
        # another block goes on from this one's checkpoint
        blob = D.dsp_block_get_adamw_state(b)
        with pytest.raises(D.DSPError) as e:
            D.dsp_block_set_adamw_state(b, blob[:-1])
        assert e.value.status == 1
        other = build_gpu_blocks(cfg, params, dtype, m=[0] * cfg["K"], standalone=True)
        blocks += other
        D.dsp_block_set_adamw(other[0], bits, 17)
        D.dsp_block_set_params(other[0], D.dsp_block_get_params(b))
        D.dsp_block_set_adamw_state(other[0], blob)
        for block, batch in ((b, 2), (other[0], 0)):
            D.dsp_block_forward(block, batch, x, out)
            D.dsp_block_recompute_backward(block, batch, gout, None)
            D.dsp_param_update_adamw(block, 1e-2, weight_decay=0.1, max_norm=0.3)
        np.testing.assert_array_equal(D.dsp_block_get_params(b), D.dsp_block_get_params(other[0]))
        np.testing.assert_array_equal(D.dsp_block_get_adamw_state(b), D.dsp_block_get_adamw_state(other[0]))
    finally:
        destroy_blocks(blocks)


@pytest.mark.parametrize("bits", [32, 8])
def test_pipeline_update_resumes_and_replays(bits):
    """Ticks with AdamW: eager, from recorded graphs, and resumed from a checkpoint give the same bits."""
    from tests.gpu_harness import build_gpu_blocks, destroy_blocks, to_dev
    from workloads import make_batch
    cfg, params, rng = _cfg()
    batches = [make_batch(rng, cfg["input"], cfg["classes"]) for _ in range(12)]
    dev = [(to_dev(x, D.DSP_FP32), torch.from_numpy(y).cuda()) for x, y in batches]

    def train(graphs, other=False):
        blocks = build_gpu_blocks(cfg, params, D.DSP_FP32)
        pl = D.dsp_pipeline_init(blocks, cfg["p"], cfg["m"], cfg["lr"], cfg["beta"], cfg["wd"], 64)
        try:
            with pytest.raises(D.DSPError) as e:
                D.dsp_pipeline_set_adamw(pl, 1e-3)
            assert e.value.status == 2
            for k, b in enumerate(blocks):
                D.dsp_block_set_adamw(b, bits, 100 + k)
            D.dsp_pipeline_set_adamw(pl, 1e-3, weight_decay=0.01, max_norm=1.0)
            D.dsp_pipeline_set_graph_replay(pl, graphs)
            for x, y in dev:
                D.dsp_pipeline_step(pl, x, y)
            if other:   # back to Eq. (3) for a few ticks
                D.dsp_pipeline_set_optimizer(pl, cfg["lr"], cfg["beta"], 0, cfg["wd"])
                for x, y in dev[:3]:
                    D.dsp_pipeline_step(pl, x, y)
            losses = D.dsp_pipeline_losses(pl)
            return [np.array(losses)] + [D.dsp_block_get_params(b) for b in blocks] + [D.dsp_block_get_adamw_state(b) for b in blocks]
        finally:
            D.dsp_pipeline_destroy(pl)
            destroy_blocks(blocks)
    a, b, c = train(False), train(True), train(False, True)
    assert np.isfinite(a[0]).all()
    for p, q in zip(a, b):
        np.testing.assert_array_equal(p, q)
    np.testing.assert_array_equal(a[0], c[0][:len(a[0])])
    K = len(cfg["blocks"])
    for k in range(K):  # the moments of AdamW wait; the parameters have moved on
        np.testing.assert_array_equal(a[1 + K + k], c[1 + K + k])
        assert not np.array_equal(a[1 + k], c[1 + k])


def test_the_first_step_is_exactly_the_step_size():
    """Without memory (betas of 0) m / sqrt(v) = g / |g|.  For gradients of 12 bits the square, its root and the quotient are exact, and
    eps is less than half a step of the root."""
    n = 1 << 16
    rng = np.random.default_rng(0)
    g = (rng.integers(1, 4096, n) * 2.0 ** rng.integers(-20, 10, n) * rng.choice([-1, 1], n)).astype(np.float32)
    z = lambda: torch.zeros(n, device="cuda")  # noqa: E731
    d = {"param": z(), "grad": torch.from_numpy(g).cuda(), "m": z(), "v": z()}
    o = D.dsp_adamw_init([d])
    D.dsp_adamw_step(o, 1.0, 0.0, 0.0, 1e-15)
    x = d["param"].cpu().numpy()
    D.dsp_adamw_destroy(o)
    np.testing.assert_array_equal(x, -np.sign(g))


def test_8_bits_keep_the_largest_floats_finite():
    """Values in the last eighth below 2^128 are not rounded up to it: no float would hold that."""
    n = 4096
    g = np.full(n, 1.8e19, np.float32)  # squared 3.24e38, 1.9 * 2^127
    g[::3] = 1.0
    z = lambda k, dt: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    d = {"param": z(n, torch.float32), "grad": torch.from_numpy(g).cuda(), "m": z(n, torch.uint8), "v": z(n, torch.uint8),
         "m_exp": z(n // 256, torch.uint8), "v_exp": z(n // 256, torch.uint8)}
    o = D.dsp_adamw_init([d], 8, 3)
    for t in range(3):
        D.dsp_adamw_step(o, 1e-3, 0.0, 0.0)
        v = P.decode(d["v"].cpu().numpy(), d["v_exp"].cpu().numpy(), 2, 15)
        assert (v < 2.0 ** 128).all() and (v[g > 1] >= 1.75 * 2.0 ** 127).all(), t
        x = d["param"].cpu().numpy().astype(np.float64)
        assert np.isfinite(x).all()
        # every step is lr g / |g|, off by the hardware's root and reciprocal and a few roundings; x adds U of itself
        assert np.abs(x[g > 1] + (t + 1) * 1e-3).max() <= (t + 1) * 12 * U * 1e-3
    D.dsp_adamw_destroy(o)
