"""Every cut that the linear layers' rules choose has a kernel, and every kernel that is built is chosen for some size."""
import math
import random

import pytest

import linear_plan_util as plan

FORMS = {
    "forward": lambda m, n, t, k, aligned, sms: plan.forward(m, n, t, k % 3, aligned, sms),
    "gated": lambda m, n, t, k, aligned, sms: plan.gated(m, n, t, k % 2 * 2, aligned, sms),
    "gradient_of_x": lambda m, n, t, k, aligned, sms: plan.gradient_of_x(m, n, t, 1 + k % 2, aligned, sms),
}


@pytest.mark.parametrize("form", FORMS)
def test_chosen_and_built(form):
    rng, chosen = random.Random(form), set()
    size = lambda most: int(math.exp(rng.uniform(0, math.log(most + 1))))
    for _ in range(60000):
        chosen.add(FORMS[form](size(12288), size(12288), size(4096), rng.randrange(6), rng.random() < 0.5, 148))
    assert chosen == {(2, 256, 1)} | {(1, nt, c) for nt, c in plan.tiles()}


def test_gradient_of_weights():
    rng, chosen = random.Random(1), set()
    size = lambda most: int(math.exp(rng.uniform(0, math.log(most + 1))))
    for _ in range(20000):
        chosen.add(plan.gradient_of_weights(size(12288), size(12288), size(4096), 1 + rng.randrange(2)))
    assert chosen == {(2, 256, 1), (1, 256, 1), (1, 256, 2), (1, 256, 4), (1, 256, 8)}


@pytest.mark.parametrize("form", FORMS)
def test_other_gpus(form):
    """fewer multiprocessors (a part of a GPU): still nothing that is not built"""
    rng = random.Random(2)
    size = lambda most: int(math.exp(rng.uniform(0, math.log(most + 1))))
    built = {(2, 256, 1)} | {(1, nt, c) for nt, c in plan.tiles()}
    for _ in range(20000):
        assert FORMS[form](size(12288), size(12288), size(4096), rng.randrange(6), rng.random() < 0.5, rng.choice([2, 16, 74, 132])) in built


@pytest.mark.parametrize("form", list(FORMS) + ["gradient_of_weights"])
def test_long_sums_are_shared_out(form):
    """No accumulator takes more than 131,072 terms of a sum of a million."""
    f = FORMS.get(form, lambda m, n, t, k, aligned, sms: plan.gradient_of_weights(m, n, t, 1 + k % 2, sms))
    rng = random.Random(form)
    for _ in range(3000):
        size = [rng.randrange(1, 5000) for _ in range(3)]
        at = {"forward": 1, "gated": 1, "gradient_of_x": 0, "gradient_of_weights": 2}[form]
        size[at] = rng.randrange(100000, 1 << 20) // (2 if at == 0 else 1)
        k = rng.randrange(6)
        terms = size[at] * (1 + k % 2 if at == 0 else 1)
        cg, nt, c = f(*size, k, rng.random() < 0.5, 148)
        assert (cg, nt, c) == (2, 256, 1) or (nt, c) in plan.tiles()
        assert -(-plan.blocks(terms) // c) * 64 <= 131072 + 64
