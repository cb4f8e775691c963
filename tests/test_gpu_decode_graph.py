"""A decode step of the library's own operators, captured on one deterministic arena, its argument buffers rebased for another
and replayed there (tests/toy_graph/decode_graph.hip)."""
import ctypes as C
import os

import pytest

pytestmark = pytest.mark.gpu
LIB = os.path.join(os.path.dirname(os.path.abspath(__file__)), "toy_graph", "libtoy_graph.so")


def test_decode_step_captured_rebased_and_replayed():
    import torch

    assert torch.cuda.is_available()
    assert os.path.exists(LIB), "build it first: python -c 'import __graft_entry__ as g; g.build()'"
    import paper_2604_06664_amd as fdy

    fdy.lib()
    C.CDLL(fdy.LIB_PATH, mode=C.RTLD_GLOBAL)
    toy = C.CDLL(LIB)
    toy.decode_graph_check.restype = C.c_int
    toy.decode_graph_check.argtypes = [C.c_char_p, C.c_int]
    msg = C.create_string_buffer(1024)
    print("[decode] captured step, rebased, replayed", flush=True)
    rc = toy.decode_graph_check(msg, 1024)
    print("[decode]", msg.value.decode(), flush=True)
    assert rc == 0, msg.value.decode()
