"""Host code of AdamW and of the norm-gate-residual entry points on a runtime of host memory (host_launches.cpp), each test in a process of
its own: nothing is computed, but what the library allocates and hands to its kernels can be seen."""
import ctypes
import os
import subprocess
import sys
import types

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    """The stand-in under the name and symbol versions the library asks for."""
    d = tmp_path_factory.mktemp("runtime")
    lib, ver = str(d / "libamdhip64.so.7"), str(d / "versions")
    with open(ver, "w") as f:
        f.write("hip_4.2 { global: *; };\nhip_4.3 { global: hipGraph*; hipStreamBeginCapture; hipStreamEndCapture; } hip_4.2;\n")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-pthread", "-Wl,-soname,libamdhip64.so.7",
                    "-Wl,--version-script," + ver, os.path.join(ROOT, "tests", "host_launches.cpp"), "-o", lib], check=True)
    return lib


CASES = {}


def case(f):
    """Makes `f(rt, D)` a test that runs in a process whose HIP runtime is the stand-in `rt`."""
    CASES[f.__name__] = f
    return f


A = 1 << 20  # an address; nothing is read there


@case
def norm_forward_ignores_gains_of_a_norm_that_is_none(rt, D):
    """The addresses of what is ignored do not reach a kernel, those of what is used do; rows of every kind of kernel."""
    for dtype in (D.DSP_FP32, D.DSP_BF16):
        for M, C in ((5, 40), (5, 700), (3, 9000), (5000, 1000)):
            for post in (0, 1, 2):
                for pre in (0, 1, 2):
                    d = D.make_norm_residual_desc(M, C, dtype, post, pre)
                    rt.host_launches_keep(128)  # (the pointers and strides that a launch's one argument begins with)
                    D.dsp_norm_residual_forward(d, A, 2 * A, None, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A, 8 * A if pre else None, stream=0)
                    assert rt.host_launches_kept() == 1
                    holds = [bool(rt.host_launches_holds(0, i * A)) for i in range(1, 8)]
                    assert holds == [True, True, post > 0, post > 0, pre > 0, pre > 0, True], (dtype, M, C, post, pre, holds)


@case
def adamw_out_of_memory_leaves_nothing_behind(rt, D):
    """Whichever allocation is refused: an error, no memory kept, and none of it reported by the next launch."""
    buffers = [ctypes.c_void_p() for _ in range(4)]
    for b in buffers:
        rt.hipMalloc(ctypes.byref(b), ctypes.c_size_t(4000))
    t = D.dsp_adamw_tensor(*[b.value for b in buffers[:2]], 0, *[b.value for b in buffers[2:]], 0, 0, 1000, D.DSP_FP32, 1)
    out, held = ctypes.c_void_p(), rt.host_launches_bytes_held()
    for n in range(3):
        rt.host_launches_refuse_malloc(n)
        assert D.lib().dsp_adamw_init(1, ctypes.byref(t), 32, 0, ctypes.byref(out)) == 3 and not out.value, n
        assert rt.host_launches_bytes_held() == held
        D.dsp_norm_residual_forward(D.make_norm_residual_desc(5, 40, D.DSP_FP32, 0, 1), A, None, d_h=A, stream=0)
    assert D.lib().dsp_adamw_init(1, ctypes.byref(t), 32, 0, ctypes.byref(out)) == 0
    D.dsp_adamw_step(out.value, 1e-3, max_norm=1.0, stream=0)
    D.dsp_adamw_destroy(out.value)
    assert rt.host_launches_bytes_held() == held


def _blocks(D, n=1, p=0, m=(0, 0)):
    """The first blocks of a small network, `p` ticks from one to the next, block k recomputing m[k] later."""
    import numpy as np
    from workloads import flatten_params, get_config, make_params
    cfg = get_config("tiny2")
    rng, shape, blocks = np.random.default_rng(0), tuple(cfg["input"]), []
    for k, layers in enumerate(cfg["blocks"][:n]):
        desc, keep = D.make_block_desc(layers, shape, D.DSP_BF16, k, n, m[k], p_prev=p if k else 0, needs_input_grad=k > 0)
        blocks.append(D.dsp_block_init(desc, flatten_params(layers, make_params(layers, rng))))
        shape = D.dsp_block_output_shape(blocks[-1])[0]
    return blocks


def _until_it_has_memory(rt, D, call):
    """`call` with its first, second, .. allocation refused until it needs no more; returns what it gives then."""
    held = rt.host_launches_bytes_held()
    for n in range(1000):
        rt.host_launches_refuse_malloc(n)
        try:
            out = call()
        except D.DSPError as e:
            assert e.status == 3
            assert rt.host_launches_bytes_held() == held, n
            D.dsp_norm_residual_forward(D.make_norm_residual_desc(5, 40, D.DSP_FP32, 0, 1), A, None, d_h=A, stream=0)
            continue
        rt.host_launches_refuse_malloc(-1)
        assert n > 0
        return out


@case
def blocks_and_pipelines_out_of_memory_leave_nothing_behind(rt, D):
    held = rt.host_launches_bytes_held()
    (b,) = _until_it_has_memory(rt, D, lambda: _blocks(D))
    D.dsp_block_destroy(b)
    blocks = _blocks(D, 2)
    pl = _until_it_has_memory(rt, D, lambda: D.dsp_pipeline_init(blocks, (0, 0), (0, 0), 0.1, 0.9, 0.0, 4))
    D.dsp_pipeline_destroy(pl)
    for b in blocks:
        D.dsp_block_destroy(b)
    assert rt.host_launches_bytes_held() == held


@case
def a_block_that_gets_no_moments_is_left_as_it_was(rt, D):
    """dsp_block_set_adamw without memory keeps none and can be repeated."""
    (b,) = _blocks(D)
    held, was = rt.host_launches_bytes_held(), D.dsp_block_query(b)
    _until_it_has_memory(rt, D, lambda: D.dsp_block_set_adamw(b, 8, 1) if D.dsp_block_query(b) == was else pytest.fail("the block has changed"))
    state = D.dsp_block_adamw_state_bytes(b)
    assert rt.host_launches_bytes_held() - held < state + 8192  # (beside the moments: 512 partial sums, the table and the clock)
    fresh = _blocks(D)[0]
    D.dsp_block_set_adamw(fresh, 8, 1)
    assert D.dsp_block_query(b) == D.dsp_block_query(fresh)
    D.dsp_block_destroy(fresh)
    D.dsp_block_destroy(b)


@case
def a_pipeline_is_a_probe_while_it_measures_another(rt, D):
    """Either may go first; a probe of pipelines that are gone takes AdamW as any other."""
    blocks, probes = _blocks(D, 2, 1, (2, 0)), _blocks(D, 2)
    for b in probes:
        D.dsp_block_set_adamw(b)
    for probe_first in (False, True):
        pr = D.dsp_pipeline_init(probes, (0, 0), (0, 0), 0.0, 0.0, 0.0, 4)
        pls = [D.dsp_pipeline_init(blocks, (1, 0), (2, 0), 0.1, 0.9, 0.0, 4) for _ in range(2)]
        for pl in pls:
            D.dsp_pipeline_attach_gradient_probe(pl, pr)
        if probe_first:
            D.dsp_pipeline_destroy(pr)
        for pl in pls:
            if not probe_first:
                with pytest.raises(D.DSPError) as e:
                    D.dsp_pipeline_set_adamw(pr, 1e-3)
                assert e.value.status == 2
            else:
                D.dsp_pipeline_gradient_difference(pl, 2)
            D.dsp_pipeline_destroy(pl)
        if not probe_first:
            D.dsp_pipeline_set_adamw(pr, 1e-3)
            D.dsp_pipeline_destroy(pr)
    for b in blocks + probes:
        D.dsp_block_destroy(b)


@case
def an_optimizer_belongs_to_its_device(rt, D):
    """With another device current its calls are refused, and destroying it waits for its own."""
    rt.hipSetDevice(1)
    (b,) = _blocks(D)
    D.dsp_block_set_adamw(b)
    blob = D.dsp_block_get_adamw_state(b)
    t = D.dsp_adamw_tensor(A, 2 * A, 0, 3 * A, 4 * A, 0, 0, 1000, D.DSP_FP32, 1)
    o = ctypes.c_void_p()
    assert D.lib().dsp_adamw_init(1, ctypes.byref(t), 32, 0, ctypes.byref(o)) == 0
    D.dsp_adamw_set_steps(o.value, 5)
    rt.hipSetDevice(0)
    for call in (lambda: D.dsp_adamw_step(o.value, 1e-3, stream=0), lambda: D.dsp_adamw_get_steps(o.value), lambda: D.dsp_adamw_set_steps(o.value, 7),
                 lambda: D.dsp_block_get_adamw_state(b), lambda: D.dsp_block_set_adamw_state(b, blob)):
        with pytest.raises(D.DSPError) as e:
            call()
        assert e.value.status == 1 and "device 1" in str(e.value)
    before = rt.host_launches_synchronised(1)
    D.dsp_adamw_destroy(o.value)
    assert rt.host_launches_synchronised(1) == before + 1
    device = ctypes.c_int(-1)
    rt.hipGetDevice(ctypes.byref(device))
    assert device.value == 0
    rt.hipSetDevice(1)
    assert (D.dsp_block_get_adamw_state(b) == blob).all()
    D.dsp_block_destroy(b)


@pytest.mark.parametrize("name", CASES)
def test_on_the_host(runtime, name):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), runtime, name], capture_output=True, text=True, timeout=100, cwd=ROOT)
    assert r.returncode == 0, r.stdout + r.stderr


def _main(path, name):
    rt = ctypes.CDLL(path, mode=ctypes.RTLD_GLOBAL)  # before the library, which then takes it for the HIP runtime
    rt.host_launches_holds.argtypes = [ctypes.c_int, ctypes.c_uint64]
    rt.host_launches_keep.argtypes = [ctypes.c_size_t]
    rt.host_launches_bytes_held.restype = rt.host_launches_synchronised.restype = ctypes.c_int64
    sys.path.insert(0, ROOT)
    sys.modules["torch"] = types.ModuleType("torch")  # the binding imports it for the sake of that runtime alone
    import paper_1909_02625_amd as D
    CASES[name](rt, D)


if __name__ == "__main__":
    _main(*sys.argv[1:])
