"""The calls of the GPU tests take every form of the orthogonalisation (host copy of its rules)."""
import random

import pytest

from tests.orth_cases import CALLS, kinds
from tests.orth_forms import GRAM_ROWS, form, gain, workspace_bytes

EVERY = {(p, s, "whole") for p in ("gram", "sym", "apply") for s in ("Big", "Mid", "Small")} | {
    ("two", "Mid", "whole"), ("two", "Small", "whole"),
    ("gram", "Big", "in parts"), ("gram", "Mid", "in parts"), ("gram", "Small", "in parts"),
    ("gram", "Big", "the last round in parts"), ("gram", "Mid", "the last round in parts"),
    ("gram", "Small", "the last round in parts"), ("sym", "Mid", "in parts"),
    ("sym", "Big", "the last round in parts"), ("sym", "Small", "the last round in parts")}


def test_no_other_form_is_reached():
    """By 20,000 calls of up to 60 million values."""
    rng, seen = random.Random(0), set()
    for _ in range(20000):
        b, n = rng.randint(1, 64), rng.randint(1, 24) * 128
        m = max(n, rng.randint(1, 60) * 128)
        if b * n * m <= 6e7:
            f = form(b, n, m, rng.choice([5, 8]))
            seen |= kinds(f) if f else set()
    assert not seen - EVERY, seen - EVERY


def test_the_calls_take_every_form():
    taken = set()
    for b, r, c, steps in CALLS:
        f = form(b, r, c, steps)
        if f is not None:
            taken |= kinds(f)
    assert not EVERY - taken, EVERY - taken
    assert any(form(*c) is None for c in CALLS)


@pytest.mark.parametrize("b,r,c,what", [
    (8, 2048, 7168, {("gram", "Big", "the last round in parts"), ("sym", "Big", "the last round in parts"), ("apply", "Big", "whole")}),
    (16, 2048, 768, {("gram", "Mid", "whole"), ("sym", "Mid", "whole"), ("apply", "Mid", "whole")}),
    (1, 256, 7168, {("gram", "Small", "in parts"), ("sym", "Small", "whole"), ("apply", "Small", "whole")}),
    (8, 1408, 2048, {("gram", "Big", "whole"), ("sym", "Big", "whole"), ("apply", "Mid", "whole")})])
def test_forms_of_layers(b, r, c, what):
    assert kinds(form(b, r, c)) == what


def test_the_gram_form_and_the_gain():
    assert form(1, GRAM_ROWS, 2048) is None and form(1, 2048, GRAM_ROWS) is None and form(1, GRAM_ROWS + 1, 2048) is not None
    assert form(1, 64, 200, 5) is None and form(1, 64, 200, 6)["two"] and not form(1, 200, 1000, 5)["two"]
    assert abs(gain(5) - 484.9) < 0.1
    assert gain(3, [(8.0, 0, 0), (0.1, 0, 0), (2.0, 0, 0)]) == 8.0           # noise of a later step: from 1 on


def test_the_copy_is_that_of_the_library():
    """Workspace sizes hold the sums of the parts and the places of the traces, so they tell one plan from another."""
    from paper_2607_05116_amd import capi
    for b, r, c, _ in [*CALLS, (8, 2048, 7168, 5), (1, 256, 7168, 5), (8, 1408, 2048, 5), (3, 333, 517, 5), (7, 700, 3000, 5)]:
        if min(r, c) > GRAM_ROWS:
            got = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=c, inter=r, max_rows=b)
            assert got == workspace_bytes(b, r, c), (b, r, c)
