"""Whether the GPU tests' shapes reach every kernel that calls of ordinary sizes do: the library's rules, asked on the CPU."""
import math
import random

import step_plans as plans


def spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def missing(kinds, tested):
    return set().union(*kinds) - set().union(*tested)


def test_every_kernel_of_orthogonalising_is_tested():
    rng = random.Random(7)
    shapes = [(rng.choice((1, 1, 2, 3, 5)), spread(rng, 8, 9000), spread(rng, 8, 9000), rng.choice(list(plans.TYPES))) for _ in range(30000)]
    assert not missing(plans.orth_kinds(shapes), plans.orth_kinds(plans.ORTH_SHAPES))


def test_every_kernel_of_the_loss_is_tested():
    rng = random.Random(7)
    calls = []
    while len(calls) < 40000:
        rows, classes, cols = spread(rng, 1, 200000), spread(rng, 1, 150000), spread(rng, 1, 9000)
        if rows * classes <= 1 << 31 and max(rows, classes) * cols <= 1 << 28:
            cols = cols if rng.random() < 0.5 else (cols + 63) // 64 * 64
            calls.append((rows, classes, cols, rng.choice(list(plans.TYPES)), rng.random() < 0.6, rng.random() < 0.5, rng.random() < 0.5))
    assert not missing(plans.loss_kinds(calls), plans.loss_kinds(plans.LOSS_CALLS))
