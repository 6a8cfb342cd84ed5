"""What the products, the recurrence and the policy loss refuse, on the host: every refusal comes before the first call of the runtime."""
import pytest

import paper_1909_02625_amd as D

A = 1 << 20   # an address; nothing is read there


def refused(call, word=None):
    with pytest.raises(D.DSPError) as e:
        call()
    assert e.value.status == 1 and D.dsp_last_error()
    assert word is None or word in str(e.value), str(e.value)


@pytest.mark.parametrize("dtype", [D.DSP_FP32, D.DSP_BF16])
def test_dense_refuses(dtype):
    fwd = lambda d, x=A, w=2 * A, b=None, r=None, y=3 * A, p=None: D.dsp_dense_forward(d, x, w, b, r, y, p, 8 * A, 1 << 40, stream=0)  # noqa: E731
    bwd = lambda d, dy=A, x=2 * A, w=3 * A, p=4 * A, dx=5 * A, dw=6 * A, db=7 * A, ws=8 * A, n=1 << 40: D.dsp_dense_backward(  # noqa: E731
        d, dy, x, w, p, dx, dw, db, ws, n, stream=0)
    good = dict(M=100, cin=64, cout=48, dtype=dtype, act=D.DSP_ACT_GELU)
    for over in ({"M": 0}, {"M": -1}, {"M": 1 << 31}, {"cin": 0}, {"cout": -3}, {"cin": 1 << 30}, {"dtype": 2}, {"act": 4}, {"act": -1}, {"x_stride": 63},
                 {"y_stride": 47}, {"x_stride": -64}, {"y_stride": 1 << 31}, {"M": (1 << 31) - 1, "cout": 1 << 24}):
        d = D.make_dense_desc(**{**good, **over})
        refused(lambda: fwd(d)), refused(lambda: bwd(d)), refused(lambda: D.dsp_dense_workspace_bytes(d)), refused(lambda: D.dsp_dense_workspace_bytes(d, True))
    d, e = D.make_dense_desc(**good), 2 if dtype == D.DSP_BF16 else 4
    for over in ({"x": None}, {"w": None}, {"y": None}, {"x": A + 1}, {"w": 2 * A + e - 1}, {"y": 3 * A + 1}, {"b": A + 2}, {"r": A + 1}, {"p": A + 1}, {"y": A},
                 {"p": A}, {"p": 3 * A}, {"r": 4 * A, "p": 4 * A}, {"y": 2 * A}):
        refused(lambda: fwd(d, **over))
    for over in ({"dy": None}, {"x": None}, {"w": None}, {"p": None}, {"dx": None, "dw": None, "db": None}, {"dy": A + 1}, {"dx": 5 * A + 1}, {"db": 7 * A + 2},
                 {"ws": None}, {"ws": 8 * A + 8}, {"n": D.dsp_dense_workspace_bytes(d, True) - 1}, {"dx": A}, {"dx": 2 * A}, {"dx": 3 * A}, {"dw": A}, {"dw": 3 * A},
                 {"dw": 5 * A}, {"dx": 4 * A}):
        refused(lambda: bwd(d, **over))
    cut = D.make_dense_desc(100, 8192, 64, dtype)  # few tiles, a long sum: cut into parts
    assert D.dsp_dense_workspace_bytes(cut) > 0 and D.dsp_dense_workspace_bytes(D.make_dense_desc(1, 8192, 64, dtype)) == 0
    refused(lambda: D.dsp_dense_forward(cut, A, 2 * A, None, None, 3 * A, None, None, 0, stream=0), "workspace")
    refused(lambda: D.dsp_dense_forward(cut, A, 2 * A, None, None, 3 * A, None, 8 * A, D.dsp_dense_workspace_bytes(cut) - 1, stream=0), "workspace")
    refused(lambda: D.check(D.lib().dsp_dense_forward(None, *[None] * 7, 0, None), "null"), "null descriptor")
    refused(lambda: D.check(D.lib().dsp_dense_workspace_bytes(None, 0, None), "null"))


@pytest.mark.parametrize("dtype", [D.DSP_FP32, D.DSP_BF16])
def test_recurrence_refuses(dtype):
    fwd = lambda d, x=A, f=2 * A, o=None, s=None, h=3 * A, t=None, ws=8 * A, n=1 << 40: D.dsp_recurrence_forward(d, x, f, o, s, h, t, ws, n, stream=0)  # noqa: E731
    bwd = lambda d, dh=A, dl=None, x=2 * A, f=3 * A, h=4 * A, o=None, s=None, dx=5 * A, df=6 * A, ds=None, ws=8 * A, n=1 << 40: D.dsp_recurrence_backward(  # noqa: E731
        d, dh, dl, x, f, h, o, s, dx, df, ds, ws, n, stream=0)
    good = dict(sequences=3, steps=5000, rows=15000, C_=64, dtype=dtype)
    for over in ({"sequences": 0}, {"sequences": 1 << 17}, {"steps": 0}, {"steps": (1 << 30) + 1}, {"steps": -1}, {"rows": -1}, {"rows": 1 << 31}, {"C_": 0}, {"C_": 1 << 21}, {"dtype": 3},
                 {"decay": 2}, {"x_stride": 63}, {"f_stride": -1}, {"h_stride": 1 << 31}):
        d = D.make_recurrence_desc(**{**good, **over})
        refused(lambda: fwd(d)), refused(lambda: bwd(d)), refused(lambda: D.dsp_recurrence_workspace_bytes(d))
    d = D.make_recurrence_desc(**good)
    d.coupled = 2
    refused(lambda: fwd(d))
    d = D.make_recurrence_desc(**{**good, "rows": 14999})
    refused(lambda: fwd(d), "fewer rows"), refused(lambda: bwd(d), "fewer rows")
    d = D.make_recurrence_desc(**good)
    want = D.dsp_recurrence_workspace_bytes(d)
    assert want > 0 and D.dsp_recurrence_workspace_bytes(D.make_recurrence_desc(9, 1, 9, 64, dtype)) == 0
    for bad in ({"ws": None}, {"ws": 8 * A + 8}, {"n": want - 1}):
        refused(lambda: fwd(d, **bad), "workspace"), refused(lambda: bwd(d, **bad), "workspace")
    for over in ({"x": None}, {"f": None}, {"h": None}, {"x": A + 1}, {"f": A + 1}, {"h": A + 1}, {"o": A + 2}, {"s": A + 2}, {"t": A + 2}, {"h": A}, {"h": 2 * A}):
        refused(lambda: fwd(d, **over))
    for over in ({"dh": None}, {"x": None}, {"f": None}, {"h": None}, {"dx": None, "df": None}, {"dh": A + 1}, {"dx": A + 1}, {"df": A + 1}, {"ds": A + 2},
                 {"dl": A + 2}, {"dx": 4 * A}, {"df": 4 * A}, {"dx": 3 * A}, {"df": 2 * A}, {"df": A}, {"df": 5 * A},
                 {"s": 9 * A, "ds": 9 * A}):
        refused(lambda: bwd(d, **over))
    d.x_stride = 72  # in another tensor's place, with another stride
    refused(lambda: bwd(d, dx=A))
    d.x_stride, d.f_stride = 0, 72
    refused(lambda: D.check(D.lib().dsp_recurrence_workspace_bytes(None, None), "null"))


@pytest.mark.parametrize("dtype", [D.DSP_FP32, D.DSP_BF16])
def test_policy_loss_refuses(dtype):
    lp = lambda d, z=A, l=2 * A, o=3 * A, h=4 * A: D.dsp_token_logprob(d, z, l, o, h, stream=0)  # noqa: E731
    pl = lambda d, z=A, l=2 * A, old=3 * A, ref=4 * A, adv=5 * A, w=6 * A, loss=7 * A, o=8 * A, t=9 * A, dz=10 * A: D.dsp_policy_loss(  # noqa: E731
        d, z, l, old, ref, adv, w, loss, o, t, dz, stream=0)
    good = dict(rows=10, vocab=100, dtype=dtype, kl_coef=0.1)
    nan, inf = float("nan"), float("inf")
    for over in ({"rows": 0}, {"rows": -1}, {"vocab": 0}, {"vocab": 1 << 29}, {"dtype": 2}, {"temperature": 0.0}, {"temperature": -1.0}, {"temperature": nan},
                 {"temperature": inf}, {"logits_stride": 99}, {"grad_stride": -1}, {"grad_stride": 1 << 31}):
        d = D.make_policy_loss_desc(**{**good, **over})
        refused(lambda: lp(d)), refused(lambda: pl(d))
    for over in ({"clip_low": -0.1}, {"clip_low": 1.5}, {"clip_low": nan}, {"clip_high": -0.1}, {"clip_high": inf}, {"clip_high": nan}, {"kl_coef": -1.0},
                 {"kl_coef": nan}, {"kl_coef": inf}, {"entropy_coef": nan}, {"entropy_coef": inf}):
        refused(lambda: pl(D.make_policy_loss_desc(**{**good, **over})))
    d = D.make_policy_loss_desc(**good)
    for over in ({"z": None}, {"l": None}, {"o": None, "h": None}, {"z": A + 1}, {"l": A + 2}, {"o": A + 2}, {"h": A + 1}):
        refused(lambda: lp(d, **over))
    for over in ({"z": None}, {"l": None}, {"adv": None}, {"loss": None}, {"t": None}, {"ref": None}, {"z": A + 1}, {"dz": A + 1}, {"old": A + 2}, {"adv": A + 2},
                 {"w": A + 1}, {"loss": A + 2}, {"o": 3 * A}, {"o": 4 * A}, {"t": A + 1}):
        refused(lambda: pl(d, **over))
    d.grad_stride = 104
    refused(lambda: pl(d, dz=A), "stride")
