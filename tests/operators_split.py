"""How tc_attn_decode cuts a call's work, by the library's own rule compiled for the host: tests name the kernels
that they are for, and fail when the rule gives their case to another."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_06007_b200", "csrc")
FIELDS = ("group", "columns", "prefix_rows", "prefix_blocks", "prefix_parts", "prefix_chunk", "stream_ctas", "tile_keys", "whole_parts", "workspace")
CODE = """
#include "attn_split.h"
extern "C" void split(const int64_t *a, int64_t *out)
{
    tc::AttnSplit s;
    tc::split_attn(a[0], a[1], a[2], a[3], a[4], a[5], a[6], &s);
    int64_t i = 0;
    for (int64_t v : {%s}) out[i++] = v;
}
""" % ", ".join(f"(int64_t)s.{name}" for name in FIELDS)


@functools.cache
def _compiled():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "split.cpp"), os.path.join(d, "split.so")
        with open(src, "w") as f:
            f.write(CODE)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared", "-I", CSRC, src, "-o", lib])
        return C.CDLL(lib).split


def split(R, Hq, H, D, max_len, max_prefix, quantised):
    out = (C.c_int64 * len(FIELDS))()
    _compiled()((C.c_int64 * 7)(R, Hq, H, D, max_len, max_prefix, quantised), out)
    return dict(zip(FIELDS, out))


def prefix_taken_by(R, Hq, H, D, max_len, max_prefix, quantised):
    """"stream", or "prefix 128" / "prefix 256" by the rows that a CTA of the prefix kernel takes."""
    rows = split(R, Hq, H, D, max_len, max_prefix, quantised)["prefix_rows"]
    return "stream" if rows == 16 else f"prefix {rows}"
