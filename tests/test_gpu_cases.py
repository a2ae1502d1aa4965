"""The cases of perf/operators.py: norms without an addend run in both forms, and agree with 64 bits."""
import random

import pytest

pytestmark = pytest.mark.gpu


def _without_addend(P, most=4):
    rng, found = random.Random(3), []
    while len(found) < most:
        c = P.draw(rng)
        if c["op"] == "rmsnorm" and not c["add"] and c["rows"] * c["n"] < 1 << 20:
            found.append(c)
    return found


def test_norms_without_addend():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import perf.operators as P
    try:
        for case in _without_addend(P):
            want = P.exact(case, 1)
            for P.own in (False, True):
                got = P.run(P.prepare(case, 1))
                assert torch.equal(got["sum"].double(), want["sum"])                  # no addend: x itself
                # the element rounded to float32 and the quotient and its rounding, each 2^-24
                assert ((got["scale"].double() - want["scale"]).abs() <= 3 * 2.0 ** -24 * want["scale"]).all()
                # at a border between two integers either may be taken: a step; and the value's rounding to bf16
                step = want["scale"][:, None] * 1.001
                assert ((got["values"].double() - want["values"]).abs() <= step + 2.0 ** -8 * want["values"].abs()).all()
    finally:
        P.own = False
