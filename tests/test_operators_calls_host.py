"""Calls of the operators that are refused, and first calls of a process, without a GPU."""
import ctypes as C
import threading

import pytest
import torch

import paper_2608_06007_b200 as tc
from paper_2608_06007_b200 import binding as b
from test_operators_host import BASE, INVALID, OVERLAP, call, decode_args, gather_args, layer


def test_two_threads_may_make_the_first_call_of_a_process(monkeypatch):
    """The table of integer types is there as soon as the one that says that both are."""
    class Slow(dict):
        def update(self, *args):
            started.set()
            go_on.wait(5)
            super().update(*args)

    started, go_on = threading.Event(), threading.Event()
    monkeypatch.setattr(b, "_dtypes", {})
    monkeypatch.setattr(b, "_integers", Slow())
    k = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    first = threading.Thread(target=b._dtype, args=(k,))
    first.start()
    assert started.wait(5)
    threading.Timer(0.2, go_on.set).start()
    with pytest.raises(tc.TensorCastError):  # the library's refusal of the made-up addresses, not ValueError
        tc.tc_kv_append(layer(), k, k, torch.zeros(3, dtype=torch.int64))
    first.join()


def test_decode_refuses_a_reserved_field_that_is_not_0():
    args, size = decode_args(reserved=1), C.c_int64()
    rc, why = call("tc_attn_decode", layer(), args)
    assert rc == INVALID and "reserved" in why
    assert tc.load_library().tc_attn_workspace(layer().ref, C.byref(args), C.byref(size)) == INVALID


def test_gather_refuses_one_output_for_both_planes():
    rc, why = call("tc_kv_gather", layer(), gather_args(v_out=5 * BASE))
    assert rc == OVERLAP and "v_out" in why
