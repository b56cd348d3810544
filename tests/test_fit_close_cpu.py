"""What fit_close allows, without a device: the definition agrees with fit_reference, two fp16 pieces stay well within it and one is far outside."""
import numpy as np
import pytest

import fit_close as close
from test_gpu_fit import definition, problem

CASES = [(150, 16, 64, {}), (150, 32, 128, {"sm": True, "slow": True}), (5003, 16, 64, {"missing": True}), (1500, 100, 128, {"norm": False})]


def pieces(number):
    """Operands as a call takes them: `number` fp16 pieces, scaled by the largest of their kind."""
    def operand(v):
        most = np.abs(v).max()
        by = v.dtype.type(2.0 ** (13 - np.floor(np.log2(most)))) if most > 0 else v.dtype.type(1)
        rest, out = v * by, np.zeros_like(v)
        for _ in range(number):
            piece = (rest - out).astype(np.float16).astype(v.dtype)
            out = out + piece
        return out / by
    return operand


@pytest.mark.parametrize("count, F, H, kinds", CASES)
def test_two_pieces_are_allowed_and_one_is_not(count, F, H, kinds):
    drop = (0.1, 2, 3)
    s = close.away_from_kinks(problem(90, count, F, H, n=300, m=300, **kinds), drop)
    expected = close.room(s, drop, longest=count / 64)
    two, one = (close.evaluate(s, drop, None, np.float32, pieces(k))[0] for k in (2, 1))
    for name, (value, _, most) in expected.items():
        assert close.distance(two[name], value) < most / 4, name
        assert close.distance(one[name], value) > most or name == "loss", name


@pytest.mark.parametrize("count, F, H, kinds", CASES)
def test_the_definition_is_fit_references(count, F, H, kinds):
    s = problem(91, count, F, H, **kinds)
    got = close.evaluate(s, (0.1, 2, 3))[0]
    for name, (value, _) in definition(s, (0.1, 2, 3)).items():
        assert close.distance(got[name], value) < 1e-10, name
