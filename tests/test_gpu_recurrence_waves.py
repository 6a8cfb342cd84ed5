"""The scan by eight waves a workgroup: bf16 and fp32, in parts and uncut, sequences of several tiles and of unequal length; the bounds and the
checks are those of test_gpu_recurrence."""
import numpy as np
import pytest

from tests import plain_branch as P
from tests.test_gpu_recurrence import KINDS, call, problem

pytestmark = pytest.mark.gpu


# workgroups (strips of 32 or 64 channels times sequences times parts) from 384 on; tiles are 64 rows
@pytest.mark.parametrize("dtype,lengths,C", [("bf16", [3000] * 6, 1000), ("bf16", [200] * 40, 1000), ("fp32", [2500] * 6, 520), ("fp32", [200] * 30, 520)])
def test_eight_waves(dtype, lengths, C):
    for i, (decay, coupled) in enumerate(KINDS[:1] if len(lengths) * max(lengths) > 10000 else KINDS):
        pad, off = ((0, 0), (3, 1), (8, 8), (0, 0))[i]
        call(problem(lengths, C, dtype, decay, coupled, i), dtype, False, pad, off)


@pytest.mark.parametrize("dtype,n,C", [("bf16", 30, 1000), ("fp32", 30, 520)])
def test_eight_waves_of_unequal_sequences(dtype, n, C):
    lengths = [int(v) for v in np.random.default_rng(C).integers(0, 400, n)]
    lengths[3] = 0
    for i, (decay, coupled) in enumerate(((P.EXP, False), (P.SIGMOID, True))):
        call(problem(lengths, C, dtype, decay, coupled, i, extra=3), dtype, True, (5, 0)[i], (1, 0)[i], states=i == 1)


def test_eight_waves_of_unequal_sequences_in_parts():
    lengths = [3000, 17, 1500, 0, 640, 641, 2999]
    call(problem(lengths, 1000, "bf16", P.SIGMOID, True, extra=2), "bf16", True)
