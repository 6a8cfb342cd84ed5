"""What AdamW and the norm-gate-residual entry points refuse, on the host: every refusal comes before the first call of the runtime."""
import numpy as np
import pytest

import paper_1909_02625_amd as D
from paper_1909_02625_amd import binding as B
from tests import plain_operators as P

A = 1 << 20   # an address; nothing is read there


def tensor(**over):
    t = D.dsp_adamw_tensor(A, 2 * A, 0, 3 * A, 4 * A, 5 * A, 6 * A, 1000, D.DSP_FP32, 1)
    for k, v in over.items():
        setattr(t, k, v)
    return t


def init(tensors, bits=32):
    arr = (D.dsp_adamw_tensor * len(tensors))(*tensors)
    out = B.C.c_void_p()
    return D.lib().dsp_adamw_init(len(tensors), arr, bits, 0, B.C.byref(out))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_refuses(bits):
    for over in ({"d_param": 0}, {"d_grad": 0}, {"d_m": 0}, {"d_v": 0}, {"n": -1}, {"n": 1 << 41}, {"grad_dtype": 2}, {"d_param": A + 2},
                 {"d_grad": A + 1}, {"d_copy": A + 1}, {"d_m": A}, {"d_v": A + 3996}, {"d_copy": A + 16}, {"d_grad": A + 64},
                 {"d_m": 3 * A, "d_v": 3 * A + 8}):
        assert init([tensor(**over)], bits) == 1, over
        assert D.dsp_last_error()
    assert init([tensor()], 16) == 1 and init([tensor()], 0) == 1
    assert init([tensor(), tensor()], bits) == 1 and "twice" in D.dsp_last_error()
    if bits == 8:
        assert init([tensor(d_m_exp=0)], 8) == 1 and init([tensor(d_v_exp=5 * A + 3)], 8) == 1
    else:
        assert init([tensor(d_m=3 * A + 2)], 32) == 1
    out = B.C.c_void_p()
    assert D.lib().dsp_adamw_init(0, (D.dsp_adamw_tensor * 1)(), bits, 0, B.C.byref(out)) == 1
    assert D.lib().dsp_adamw_init(1, None, bits, 0, B.C.byref(out)) == 1
    for call in (lambda: D.dsp_adamw_step(None, 1e-3, stream=0), lambda: D.dsp_adamw_get_steps(None), lambda: D.dsp_adamw_set_steps(None, 3),
                 lambda: D.dsp_block_set_adamw(None), lambda: D.dsp_param_update_adamw(None, 1e-3, stream=0),
                 lambda: D.dsp_pipeline_set_adamw(None, 1e-3), lambda: D.dsp_block_adamw_state_bytes(None)):
        with pytest.raises(D.DSPError) as e:
            call()
        assert e.value.status == 1
    D.dsp_adamw_destroy(None)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_refuses_more_chunks_than_a_launch_has_workgroups(bits):
    """2^24 workgroups of 256 threads are more than a grid may hold: 4096 or 6144 elements each, in one tensor or in many."""
    B_ = 1 << 42
    big = lambda n: tensor(d_param=B_, d_grad=2 * B_, d_m=3 * B_, d_v=4 * B_, d_m_exp=5 * B_, d_v_exp=6 * B_, n=n)  # noqa: E731
    per = 4096 if bits == 32 else 6144
    assert init([big((1 << 24) * per)], bits) == 1 and "too many" in D.dsp_last_error()
    third = [big((1 << 24) * per // 3 + per) for _ in range(3)]
    for i, t in enumerate(third):
        for f in ("d_param", "d_grad", "d_m", "d_v", "d_m_exp", "d_v_exp"):
            setattr(t, f, getattr(t, f) + i * (B_ // 4))
    assert init(third, bits) == 1 and "too many" in D.dsp_last_error()


def test_adamw_binding_wants_whole_tensors():
    import torch
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)  # noqa: E731
    good = {"param": z(300), "grad": z(300), "m": z(300), "v": z(300)}
    for over in ({"grad": z(299)}, {"m": z(301)}, {"v": z(300, torch.uint8)}, {"copy": z(300)}, {"param": z(600)[::2]}, {"grad": z(300, torch.float64)}):
        with pytest.raises(ValueError):
            D.dsp_adamw_init([{**good, **over}])
    with pytest.raises(ValueError):
        D.dsp_adamw_init([{"param": z(300), "grad": z(300), "m": z(300, torch.uint8), "v": z(300, torch.uint8), "m_exp": z(1, torch.uint8),
                           "v_exp": z(2, torch.uint8)}], 8)


def test_adamw_binding_wants_the_types_that_the_kernels_read():
    """Elements of the right size and another type: a float16 copy would receive bfloat16 bits, integer parameters those of floats."""
    import torch
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)  # noqa: E731
    good = {"param": z(300), "grad": z(300), "m": z(300), "v": z(300)}
    for over in ({"copy": z(300, torch.float16)}, {"copy": z(300, torch.int16)}, {"param": z(300, torch.int32)}, {"grad": z(300, torch.int32)},
                 {"grad": z(300, torch.float16)}, {"m": z(300, torch.int32)}, {"v": z(300, torch.int32)}):
        with pytest.raises(ValueError):
            D.dsp_adamw_init([{**good, **over}])
    byte = lambda n: z(n, torch.uint8)  # noqa: E731
    good = {"param": z(300), "grad": z(300), "m": byte(300), "v": byte(300), "m_exp": byte(2), "v_exp": byte(2)}
    for over in ({"m": z(300, torch.float8_e5m2)}, {"v": z(300, torch.float8_e4m3fn)}, {"m": z(300, torch.int8)}, {"v": z(300, torch.bool)},
                 {"m": z(300, torch.float8_e4m3fnuz)}, {"m_exp": z(2, torch.int8)}, {"v_exp": z(2, torch.bool)}):
        with pytest.raises(ValueError):
            D.dsp_adamw_init([{**good, **over}], 8)


def desc(**over):
    d = D.make_norm_residual_desc(16, 64, D.DSP_FP32, 1, 2, gate_rows=4)
    for k, v in over.items():
        setattr(d, k, v)
    return d


FWD = dict(x=A, z=2 * A, gate=3 * A, g1=0, b1=0, g2=0, b2=0, y=4 * A, h=5 * A, s1=0, s2=0)
BWD = dict(dh=A, dy=2 * A, y=3 * A, z=4 * A, gate=5 * A, g1=0, b1=0, g2=0, s1=6 * A, s2=7 * A, dx=8 * A, dz=9 * A, dgate=10 * A, dg1=11 * A,
           db1=0, dg2=12 * A, db2=0, ws=13 * A)


def fwd(d, **over):
    a = {**FWD, **over}
    return D.lib().dsp_norm_residual_forward(d, *[v or None for v in a.values()], None)


def bwd(d, bytes_=1 << 20, **over):
    a = {**BWD, **over}
    return D.lib().dsp_norm_residual_backward(d, *[v or None for v in a.values()], bytes_, None)


def test_norm_residual_refuses():
    bad = [dict(M=0), dict(M=-1), dict(M=1 << 31), dict(C=0), dict(C=16385), dict(dtype=2), dict(post=3), dict(pre=-1), dict(eps=0.0),
           dict(eps=float("nan")), dict(eps=float("inf")), dict(gate_rows=-1), dict(gate_act=3), dict(gate_dtype=2), dict(gate_dtype=D.DSP_BF16),
           dict(x_stride=63), dict(z_stride=-64), dict(y_stride=1), dict(h_stride=1 << 31), dict(gate_stride=10)]
    for over in bad:
        assert fwd(desc(**over)) == 1 and bwd(desc(**over)) == 1, over
        out = B.C.c_size_t()
        assert D.lib().dsp_norm_residual_workspace_bytes(desc(**over), B.C.byref(out)) == 1
    for over in (dict(x=0), dict(gate=0), dict(y=0), dict(h=0), dict(x=A + 2), dict(z=A + 1), dict(y=A + 3), dict(h=A + 2), dict(gate=A + 2),
                 dict(z=0)):
        assert fwd(desc(), **over) == 1, over
    plain = desc(post=0, gate_rows=0)
    assert fwd(plain, z=0, gate=0) == 1                                         # y is not formed without a branch
    assert fwd(desc(post=0, gate_rows=0, alpha=0.5), z=0, gate=0, y=0) == 1
    assert fwd(desc(post=0, gate_rows=0, pre=0), z=0, gate=0, y=0) == 1
    for over in (dict(dh=0), dict(y=0), dict(z=0), dict(gate=0), dict(s1=0), dict(s2=0), dict(dh=A + 1), dict(dy=A + 2), dict(dz=A + 2), dict(dx=A + 3),
                 dict(dgate=A + 2), dict(ws=0), dict(ws=A + 8)):
        assert bwd(desc(), **over) == 1, over
    assert bwd(desc(), bytes_=D.dsp_norm_residual_workspace_bytes(desc()) // 2 - 1) == 1 and "workspace" in D.dsp_last_error()
    assert bwd(desc(pre=0), dy=0) == 1
    assert bwd(desc(pre=0)) == 1 and "not there" in D.dsp_last_error()          # a gain's gradient without its norm
    assert bwd(desc(post=0)) == 1
    assert bwd(desc(gate_rows=0)) == 1                                          # a gate's without a gate
    assert bwd(desc(), dx=0, dz=0, dgate=0, dg1=0, dg2=0) == 1                  # nothing asked for
    assert D.lib().dsp_norm_residual_forward(None, *[None] * 12) == 1
    assert D.lib().dsp_norm_residual_workspace_bytes(desc(), None) == 1


def test_norm_residual_wants_aligned_vectors_and_statistics():
    """Floats on addresses of floats, as the header says of every buffer."""
    for name in ("g1", "b1", "g2", "b2", "s1", "s2"):
        assert fwd(desc(), **{name: A + 2}) == 1 and "misaligned" in D.dsp_last_error(), name
    for name in ("g1", "b1", "g2", "s1", "s2", "dg1", "db1", "dg2", "db2"):
        assert bwd(desc(), **{name: 20 * A + 1}) == 1 and "misaligned" in D.dsp_last_error(), name


def test_norm_residual_in_place_wants_the_same_stride():
    """With another stride a row's result would fall on rows that others have still to read."""
    for strides in (dict(x_stride=80), dict(y_stride=80), dict(x_stride=72, y_stride=80)):
        assert fwd(desc(**strides), y=FWD["x"]) == 1 and "stride" in D.dsp_last_error(), strides
        assert bwd(desc(**strides), dx=BWD["dy"]) == 1 and "stride" in D.dsp_last_error(), strides


def test_workspace_stays_small():
    for M, C in ((1, 1), (1 << 20, 16384), (1 << 30, 64), (1024, 4096)):
        for rows in (0, 1, 3, 1000, M):
            n = D.dsp_norm_residual_workspace_bytes(D.make_norm_residual_desc(M, C, D.DSP_BF16, 2, 2, gate_rows=rows))
            assert 16 * C <= n <= 1024 * 16 * C


# ---- the plain implementations of the tests themselves
def test_codes_round_trip():
    codes = np.arange(256, dtype=np.uint8)
    for mant, bias, dtype in ((3, 7, "float8_e4m3fn"), (2, 15, "float8_e5m2")):
        import torch
        want = torch.from_numpy(codes).view(getattr(torch, dtype)).double().numpy()
        got = P.decode(codes, [127], mant, bias)
        fin = np.isfinite(want) & ((codes & 127) != 127)
        np.testing.assert_array_equal(got[fin], want[fin])
    rng = np.random.default_rng(0)
    a = rng.standard_normal(1024) * np.exp(3 * rng.standard_normal(1024))
    for args in ((3, 7, 7, False), (2, 15, 14, True)):
        x = np.abs(a) if args[3] else a
        c, e = P.encode(x, np.zeros(1024), *args)
        v = P.decode(c, e, args[0], args[1])
        c2, e2 = P.encode(v, np.full(1024, 65535.0), *args)
        np.testing.assert_array_equal(P.decode(c2, e2, args[0], args[1]), v)
        hi = P.decode(*P.encode(x, np.full(1024, 65535.0), *args), args[0], args[1])
        assert (np.abs(v) <= np.abs(x)).sum() >= 1000 and (np.abs(hi) >= np.abs(x) * (1 - 1e-9)).all() and (np.abs(hi) >= np.abs(v)).all()


def test_random_bits_are_spread():
    n = 1 << 18
    low, high = P.random_halves(5, 1, 0, n)
    for r in (low, high):
        assert abs(r.mean() - 32767.5) < 6 * 18919 / np.sqrt(n)
        assert abs(np.corrcoef(r[:-1], r[1:])[0, 1]) < 6 / np.sqrt(n)
    for other in (P.random_halves(5, 2, 0, n), P.random_halves(5, 1, 1, n), P.random_halves(6, 1, 0, n), P.random_halves(5, 1, 0, n, first=1 << 32)):
        assert abs(np.corrcoef(low, other[0])[0, 1]) < 6 / np.sqrt(n) and abs(np.corrcoef(high, other[1])[0, 1]) < 6 / np.sqrt(n)


@pytest.mark.parametrize("post,pre", [(a, b) for a in range(3) for b in range(3)])
def test_plain_gradients_against_differences(post, pre):
    rng = np.random.default_rng(post * 3 + pre)
    M, C = 6, 9
    r = lambda *s: rng.standard_normal(s)  # noqa: E731
    for act in range(3):
        p = {"x": r(M, C), "z": r(M, C), "gate": r(3, C), "gate_rows": 2, "gate_act": act, "post": post, "pre": pre, "alpha": 0.7, "beta": -1.3,
             "eps": 1e-5, "post_gain": r(C), "post_bias": r(C), "pre_gain": r(C), "pre_bias": r(C)}
        dy, dh = r(M, C), r(M, C)
        y, _ = P.forward(p)
        g = P.backward(p, y, dy, dh, P.stats(pre, y, 1e-5) if pre else None, P.stats(post, p["z"], 1e-5) if post else None)
        names = ["x", "z", "gate"] + (["post_gain", "post_bias"] if post else []) + (["pre_gain", "pre_bias"] if pre else [])
        for name in names:
            t = r(*p[name].shape)

            def value(s):
                yy, hh = P.forward({**p, name: p[name] + s * t})
                return (dy * yy).sum() + ((dh * hh).sum() if pre else 0.0)
            diff = (value(1e-5) - value(-1e-5)) / 2e-5
            assert abs((g[name] * t).sum() - diff) < 1e-6 * np.abs(t * g[name + "~"]).sum() + 1e-7, (name, act)
