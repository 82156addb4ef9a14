"""A gradient that shares memory with the logits at another place is refused, one beside them is not.  No GPU: an argument that is
refused later on tells what was let through."""
import ctypes
import itertools
import random

from paper_1811_00206_amd import binding as b


def status(T, V, ld, ldg, first, dtype=0):
    """That of logits at 1 << 20 and a gradient `first` elements behind them; 4 (alignment): it got past the question."""
    size = 4 if dtype == 0 else 2
    p, null = ctypes.c_void_p(4096), ctypes.c_void_p(0)
    return b.load_library().bs_logprobs_backward(ctypes.c_void_p(1 << 20), dtype, T, V, ld, p, ctypes.c_void_p(4098), p, p, p,
                                                 ctypes.c_void_p((1 << 20) + first * size), ldg, null)


def shares(T, V, ld, ldg, first):
    mine = {i * ld + v for i in range(T) for v in range(V)}
    return any(first + i * ldg + v in mine for i in range(T) for v in range(V))


def test_every_place_of_small_tensors():
    for T, V, dtype in itertools.product((1, 2, 4), (1, 3), (0, 2)):
        for ld, ldg in itertools.product(range(V, 2 * V + 3), repeat=2):
            for first in range(-T * ldg - 3, T * ld + 4):
                want = 4 if first == 0 and ld == ldg or not shares(T, V, ld, ldg, first) else 3
                assert status(T, V, ld, ldg, first, dtype) == want, (T, V, ld, ldg, first)


def test_some_places_of_larger_ones():
    rng = random.Random(1)
    for _ in range(300):
        T, V = rng.randint(1, 40), rng.randint(1, 50)
        ld = V + rng.choice((0, rng.randint(0, 80)))
        ldg = rng.choice((ld, V + rng.randint(0, 120)))
        first = rng.choice((1, V, ld, rng.randint(-T * ldg, T * ld)))
        assert status(T, V, ld, ldg, first) == (3 if shares(T, V, ld, ldg, first) else 4) or first == 0, (T, V, ld, ldg, first)


def test_tensors_side_by_side():
    """The two halves of the rows of one tensor; a gradient behind the logits, or in front of them."""
    T, V = 1 << 20, 50000
    assert status(T, V, 2 * V, 2 * V, V) == status(T, V, 2 * V, 2 * V, -V) == 4
    assert status(T, V, V, V, T * V) == 4 and status(T, V, V, V, T * V - 1) == 3
    assert status(T, V, 2 * V, V + 8, 2 * V * T) == 4 and status(T, V, 2 * V, 2 * V, 0) == 4
    assert status(T, V, V, V, V) == 3 and status(T, V, 2 * V, 2 * V, V - 1) == 3
