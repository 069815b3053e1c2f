"""The operators on a paged layer where numbers are at the ends of their range."""
import numpy as np
import pytest

from test_operators_gpu import Pool, append_case, check_append, run_append, status_is

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("kind", ["e4m3", "int8", "bf16"])
@pytest.mark.parametrize("x", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_keeps_the_sign_of_zeros(kind, x, interleaved):
    """-0 in rows that are not zero: given, and made by a rotation of (0, 0) with a negative cosine.  D = 100 takes single
    elements, the others vectors."""
    def mutate(qkv):
        qkv[::2, :, ::3] = -0.0
        qkv[::3, :, 1::5] = 0.0
        qkv[1, :, 4:] = 0.0
        qkv[2, :, 8:] = -0.0

    rng = np.random.default_rng([interleaved, x == "bf16"])
    for D, rot in ((128, 128), (128, 0), (80, 32), (100, 50)):
        pool = Pool(kind, D=D)
        s = append_case(pool, 37, 4, x, rot, interleaved, rng, mutate=mutate)
        run_append(pool, s)
        check_append(pool, s)
    status_is(0)
