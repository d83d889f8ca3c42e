"""Which operands of the layer operators may lie in one buffer: the library's answer
before any launch, against the elements that they are made of."""
import itertools
import random

import pytest

import paper_2606_06510_amd as oz
from paper_2606_06510_amd import _lib

AT = 1 << 40      # addresses that are never read
FAR = 1 << 30


def elements(at, count, stride, rows, ld, cols):
    return {at + k * stride + r * ld + c for k in range(count) for r in range(rows) for c in range(cols)}


def backward(G, N, K, dw, sdw, lddw, db, sdb, w=None, sw=None, ldw=None):
    """The status of the gradients of G layers' products, with dw and db at the given
    elements (fp32) of one buffer, everything else elsewhere.  Valid arguments without
    the workspace are OZ2_E_WORKSPACE."""
    S = 9
    far = itertools.count(1)

    def other():
        return AT + FAR * next(far)
    return oz.load().ozaki2_grouped_linear_backward(
        oz.OZ2_F32, 0, 0, S, G, N, K, other(), other(), N, other(), K,
        other() if w is None else AT + 4 * w, ldw or K, N * K if sw is None else sw, None, 0, other(), K,
        AT + 4 * dw, lddw, sdw, AT + 4 * db, sdb, None, 0, None)


@pytest.mark.parametrize("G", [1, 2, 5])
def test_parameters_of_a_layer_one_after_the_other(G):
    """[layer][W, bias]: a stride of N K + N for both"""
    N, K = 6, 8
    step = N * K + N
    assert backward(G, N, K, 0, step, K, N * K, step) == _lib.OZ2_E_WORKSPACE
    assert backward(G, N, K, N, step, K, 0, step) == _lib.OZ2_E_WORKSPACE      # bias first
    assert backward(G, N, K, 0, step, K, N * K - 1, step) == _lib.OZ2_E_INVALID
    assert backward(G, N, K, N - 1, step, K, 0, step) == _lib.OZ2_E_INVALID


def test_weights_and_gradients_side_by_side():
    """[layer][row][W, dW], and [layer][W, dW]"""
    G, N, K = 4, 6, 8
    kw = dict(db=1 << 24, sdb=N)
    assert backward(G, N, K, K, 2 * N * K, 2 * K, w=0, sw=2 * N * K, ldw=2 * K, **kw) == _lib.OZ2_E_WORKSPACE
    assert backward(G, N, K, N * K, 2 * N * K, K, w=0, sw=2 * N * K, ldw=K, **kw) == _lib.OZ2_E_WORKSPACE
    assert backward(G, N, K, K - 1, 2 * N * K, 2 * K, w=0, sw=2 * N * K, ldw=2 * K, **kw) == _lib.OZ2_E_INVALID
    # one W for every layer, in between
    assert backward(G, N, K, N * K, 2 * N * K, K, w=2 * N * K, sw=0, ldw=K, **kw) == _lib.OZ2_E_INVALID
    assert backward(1, N, K, N * K, 2 * N * K, K, w=0, sw=0, ldw=K, **kw) == _lib.OZ2_E_WORKSPACE


@pytest.mark.parametrize("G", [2, 5])
def test_gradients_row_by_row(G):
    """[row][layer][dW]: no element is in two layers, though every layer's rows lie in
    between the others'"""
    N, K = 6, 8
    assert backward(G, N, K, 0, K, G * K, 1 << 24, N) == _lib.OZ2_E_WORKSPACE
    assert backward(G, N, K, 0, K, G * K - 1, 1 << 24, N) == _lib.OZ2_E_INVALID
    assert backward(G, N, K, 0, K - 1, G * K, 1 << 24, N) == _lib.OZ2_E_INVALID
    assert backward(G, N, K, 0, K, G * K, (N - 1) * G * K, N) == _lib.OZ2_E_INVALID    # dbias in a row


def test_nothing_that_overlaps_is_taken():
    """random stacks: never taken where an element is in both; and the layouts that do not
    overlap by a common period are"""
    rng = random.Random(5)
    taken = 0
    for _ in range(20000):
        G, N, K = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 4)
        lddw = K + rng.randint(0, 6)
        sdw = (N - 1) * lddw + K + rng.randint(0, 30)
        sdb = rng.choice([sdw, sdw, N + rng.randint(0, 60)])
        dw, db = rng.randint(0, 40), rng.randint(0, 60)
        st = backward(G, N, K, dw, sdw, lddw, db, max(sdb, N))
        both = elements(dw, G, sdw, N, lddw, K) & elements(db, G, max(sdb, N), 1, N, N)
        assert st == _lib.OZ2_E_INVALID if both else st in (_lib.OZ2_E_INVALID, _lib.OZ2_E_WORKSPACE)
        taken += st == _lib.OZ2_E_WORKSPACE
    assert taken > 2000
