"""Which kernel takes a decode call's prefix, and the workspace that goes with it."""
import ctypes as C

import pytest

import paper_2608_06007_b200 as tc
from operators_split import prefix_taken_by, split
from test_operators_host import decode_args, layer


@pytest.mark.parametrize("R,Hq,H,D,prefix,quantised,taken", [
    (64, 32, 8, 128, 8192, False, "prefix 256"), (512, 32, 8, 128, 4000, True, "prefix 256"), (128, 64, 8, 128, 32768, False, "prefix 256"), (32, 32, 8, 128, 2000, True, "prefix 128"),
    (4, 32, 8, 128, 48, False, "stream"), (128, 32, 8, 128, 64, False, "stream"), (512, 32, 8, 256, 4000, True, "stream"), (4, 4, 1, 128, 100000, False, "stream"),
])
def test_a_long_prefix_that_many_rows_share_has_its_own_kernel(R, Hq, H, D, prefix, quantised, taken):
    assert prefix_taken_by(R, Hq, H, D, 100, prefix, quantised) == taken


def test_the_parts_of_a_prefix_cover_it_and_the_workspace_is_what_the_library_asks_for():
    lib, out = tc.load_library(), C.c_int64()
    for R in (1, 3, 32, 65, 70, 300):
        for prefix in (0, 1, 1000, 9000, 131072):
            s = split(R, 32, 8, 128, 77, prefix, False)
            if s["prefix_parts"]:
                chunks = s["prefix_parts"] // (2 if s["prefix_rows"] == 128 else 1)
                assert s["prefix_chunk"] % 128 == 0 and (chunks - 1) * s["prefix_chunk"] < prefix <= chunks * s["prefix_chunk"]
            assert lib.tc_attn_workspace(layer().ref, C.byref(decode_args(R=R, max_len=77, max_prefix=prefix)), C.byref(out)) == 0
            assert out.value == s["workspace"]
