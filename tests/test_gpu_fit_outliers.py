"""GPU: samples and workloads that stand out do not change what is said of the others."""
import numpy as np
import pytest

import fit_close as close
from test_gpu_fit import call, problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2303_13803_amd as mm
    c = mm.Context(64, 64)
    yield c
    c.close()


def same_bits(a, b, names):
    for name in names:
        assert (a[name].view(np.int32) == b[name].view(np.int32)).all(), name


# ---- targets of samples that name no pair

@pytest.mark.parametrize("H", [64, 128])
@pytest.mark.parametrize("F", [16, 70])
@pytest.mark.parametrize("count", [30, 20000])
@pytest.mark.parametrize("fill", [1e9, -1e20, 3e38, np.inf])
def test_targets_of_samples_that_name_no_pair(ctx, fill, count, F, H):
    """In the same 32 samples as real ones, and in others: every bit is what it is with targets like all others there."""
    s = problem(70, count, F, H, slow=True, missing=True)
    none = (s["on"] < 0) | (s["off"] >= 40)
    assert none.any() and not none.all()
    s["target"][none], s["target_slow"][none] = 0.5, 0.5
    plain = call(ctx, s, (0.1, 2, 3))
    s["target"][none], s["target_slow"][none] = fill, fill
    filled = call(ctx, s, (0.1, 2, 3))
    same_bits(plain, filled, plain)
    s = close.away_from_kinks(s, (0.1, 2, 3))
    close.check(call(ctx, s, (0.1, 2, 3)), close.room(s, (0.1, 2, 3), longest=count / 64))
