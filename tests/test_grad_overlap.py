"""Clipping refuses lists in which an output overlaps anything but the gradient that it is, before anything is launched (no GPU needed)."""
import ctypes
import random

import pytest

import paper_2502_02581_amd as moe
from paper_2502_02581_amd.binding import _CGrad

BASE = 1 << 20   # addresses that are never dereferenced: every call below fails before a launch


def clip(*spans, dtype=1):
    """spans: (first byte of the gradient, of its output, values)"""
    lib = moe.load_library()
    grads = (_CGrad * len(spans))(*[_CGrad(g=BASE + g, out=BASE + o, n=n, n_active=None, slot=0, dtype=dtype) for g, o, n in spans])
    return lib.moe_grad_clip(grads, len(spans), ctypes.c_void_p(4096), 1.0, None), lib.moe_last_error().decode()


@pytest.mark.parametrize("spans,what", [
    ([(0, 0, 16), (16, 16, 16)], "outputs 0 and 1 overlap"),                           # the second half of the first one, both in place
    ([(0, 0, 1000), (512, 4096, 8)], "output 0 is another gradient"),                  # a slice of what is written in place is read
    ([(0, 4096, 100), (1024, 4112, 8)], "outputs 0 and 1 overlap"),                    # one output inside another
    ([(0, 4096, 100), (4288, 8192, 8)], "output 0 is another gradient"),               # an output that ends inside another gradient
    ([(0, 16, 100)], "overlaps its gradient"),
    ([(16, 0, 100)], "overlaps its gradient"),
    ([(0, 0, 8), (64, 64, 8), (32, 32, 9), (32 + 16, 4096, 8)], "output 2 is another gradient"),
    ([(0, 0, 0), (0, 0, 8), (4096, 0, 8)], "outputs 1 and 2 overlap"),                 # (an empty tensor overlaps nothing)
    ([(1 << 16, 0, 1 << 15), (1 << 15, 1 << 17, 8)], "output 0 is another gradient"),  # a long span far ahead of the one that it covers
    ([(1 << 20, 0, 1 << 15), (1 << 21, 1024, 8), (1 << 22, 1 << 15, 8)], "overlap"),
])
def test_overlapping_tensors(spans, what):
    rc, text = clip(*spans)
    assert rc == -1 and what in text
    assert clip(*reversed(spans))[0] == -1   # whatever their order


def test_random_lists_against_every_pair():
    """Lists of which some pair overlaps, found pair by pair; lists without one are not called: they would be launched."""
    r = random.Random(4)
    refused = 0
    for _ in range(3000):
        spans = []
        for _ in range(r.randint(1, 6)):
            g = 16 * r.randint(0, 60)
            spans.append((g, g if r.random() < 0.5 else 16 * r.randint(0, 60), r.randint(0, 40)))
        cover = lambda a, b, n, m: n and m and a < b + 2 * m and b < a + 2 * n
        bad = any(cover(spans[i][1], spans[j][x], spans[i][2], spans[j][2]) and not (i == j and (x == 1 or spans[i][0] == spans[i][1]))
                  for i in range(len(spans)) for j in range(len(spans)) for x in (0, 1))
        if bad:
            rc, text = clip(*spans)
            assert rc == -1 and "overlap" in text, spans
            refused += 1
    assert refused > 1000
