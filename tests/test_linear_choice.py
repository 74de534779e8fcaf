"""The batches of tests/linear_rings.py reach every kernel that the library's rules choose, with rings that turn (no GPU)."""
import math
import random

import linear_rings as R

BITS = list(R.FORWARD)
# what these have is too short a sum or too few of them for their rings to turn: the rules choose them nowhere else
SHORT = {("gradient", 2, 0, R.Kernel(0, 0, 0, 0, 4, 0)), ("gradient", 3, 0, R.Kernel(1, 2, 1, 1, -1, 0)), ("forward", 4, 8, R.Kernel(1, 1, 4, 1, -1, 0))}


def _forward(T, N, K, E, xbits, wbits):
    c = R.forward_choice(T, N, K, E, xbits, wbits)
    return ("forward", xbits, wbits, c.kernel), c, K


def _gradient(T, N, K, E, wbits, terms, aligned=True):
    c = R.gradient_choice(T, N, K, E, wbits, terms, aligned)
    return ("gradient", terms, wbits if c.kernel.across else 0, c.kernel), c, N


def _covered():
    """kernel -> the deepest that its ring turns beyond its depth, and the parities of stages that turn"""
    got = {}
    for key, c, summed in [_forward(*c) for c in R.FORWARD_CASES] + [_gradient(*c) for c in R.GRADIENT_CASES]:
        n, least = R.steps(c, summed)
        deep, parities = got.setdefault(key, [-99, set()])
        got[key][0] = max(deep, least - c.depth)
        if least - c.depth >= 2:
            parities.add(n % 2)
    return got


def test_every_batch_turns_its_ring():
    for key, (deep, parities) in _covered().items():
        if key in SHORT:
            continue
        assert deep >= 2, f"{key}: no batch loads a place twice again"
        assert key[3].few or parities == {0, 1}, f"{key}: stages of one parity only"


def test_no_kernel_is_left_out():
    rng = random.Random(5)

    def size(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    covered = set(_covered())
    for _ in range(40000):
        T, E = size(1, 20000), rng.choice([0, 0, 0, 2, 3, 4, 8, 16, 32, 64])
        xbits, wbits = rng.choice(BITS)
        key, *_ = _forward(T, size(1, 20000), 64 * size(1, 256), E, xbits, wbits)
        assert key in covered, key
        key, *_ = _gradient(T, size(1, 20000), rng.choice([64 * size(1, 128), size(1, 11008)]), E, rng.choice([8, 4, 2]), rng.choice([2, 3]),
                           rng.random() < 0.7)
        assert key in covered, key
