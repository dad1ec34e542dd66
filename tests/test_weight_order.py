"""When a linear layer's product may fetch weights early (csrc/wfq_weight_order.h), on the CPU.

A product that does so wrongly reads weights while they are written, which on a GPU shows by chance only."""
import ctypes
import itertools
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_19867_b200", "csrc")
SOURCE = """
#include "wfq_weight_order.h"
extern "C" {
wfq::WeightOrder *make() { return new wfq::WeightOrder(); }
void drop(wfq::WeightOrder *o) { delete o; }
void written(wfq::WeightOrder *o, const void *s, int captured) { o->written(s, captured != 0); }
int settled(const wfq::WeightOrder *o, const void *s) { return o->settled(s); }
int pending(const wfq::WeightOrder *o) { return o->pending(); }
void waited(wfq::WeightOrder *o, const void *s, int captured) { o->waited(s, captured != 0); }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("order")
    (d / "order.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "order.so"),
                    str(d / "order.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "order.so"))
    lib.make.restype = ctypes.c_void_p
    for f in (lib.drop, lib.written, lib.settled, lib.pending, lib.waited):
        f.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int][:{"drop": 1, "pending": 1, "settled": 2}.get(f.__name__, 3)]
    return lib


class Order:
    def __init__(self, lib):
        self.lib, self.at = lib, lib.make()

    def written(self, s, captured=False):
        self.lib.written(self.at, s, captured)

    def settled(self, s):
        return bool(self.lib.settled(self.at, s))

    def waited(self, s, captured=False):
        self.lib.waited(self.at, s, captured)


A, B, C = 0x1000, 0x2000, 0x7000


def test_behind_the_preparation_a_product_waits_on_its_stream(lib):
    o = Order(lib)
    o.written(A)
    assert not o.settled(A)
    o.waited(A)
    assert o.settled(A) and o.settled(B)


def test_a_product_on_another_stream_settles_nothing_for_the_preparations_own(lib):
    o = Order(lib)
    o.written(A)
    assert not o.settled(B)
    o.waited(B)
    assert o.settled(B) and o.settled(C) and not o.settled(A)
    o.waited(A)
    assert o.settled(A)


def test_a_launch_that_failed_settles_nothing(lib):
    o = Order(lib)
    o.written(A)
    assert not o.settled(A) and not o.settled(A)           # asked, not launched: nothing is reported as waited


def test_under_capture_nothing_is_settled(lib):
    o = Order(lib)
    o.written(A)
    o.waited(A, captured=True)
    o.waited(B, captured=True)
    assert not o.settled(A) and not o.settled(B)
    o.waited(A)
    assert o.settled(B)


def test_weights_that_a_graph_writes_are_never_settled(lib):
    o = Order(lib)
    o.written(A, captured=True)
    for s in (A, B):
        o.waited(s)
        assert not o.settled(A) and not o.settled(B)
    o.written(B)
    o.waited(B)
    assert not o.settled(B)


def test_the_two_handles_of_the_default_stream_are_one(lib):
    for first, second in ((None, 1), (1, None)):
        o = Order(lib)
        o.written(first)
        o.waited(B)
        assert o.settled(B) and not o.settled(second) and not o.settled(first)
        o.waited(second)
        assert o.settled(first)


def test_every_short_history(lib):
    """Against the definition: early is wrong on the stream of the last write until a product there has waited, and
    everywhere once a graph writes."""
    steps = [("written", A, False), ("written", B, False), ("written", A, True), ("waited", A, False), ("waited", B, False),
             ("waited", C, False), ("waited", A, True), ("waited", B, True)]
    for history in itertools.product(steps, repeat=5):
        o = Order(lib)
        last, waited, graph = None, set(), False
        for name, s, captured in history:
            getattr(o, name)(s, captured)
            if name == "written":
                last, waited, graph = s, set(), graph or captured
            elif not captured:
                waited.add(s)
        for s in (A, B, C):
            wrong = graph or (last == s and s not in waited)
            if wrong:
                assert not o.settled(s), (history, s)
            elif last is None or last in waited or (s != last and waited):
                assert o.settled(s), (history, s)          # and not given up for longer than that
        o.lib.drop(o.at)
