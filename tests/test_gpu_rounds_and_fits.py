"""GPU: one context matches in one compute unit, with most of its LDS, and fits predictors of many features, in either order, in a process that has
launched nothing before."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = """
import sys
sys.path[:0] = [%r, %r]
import numpy as np, torch
import fit_close as close, oracle
import paper_2303_13803_amd as mm
from gpu_util import padded_matrix
from test_gpu_fit import call, problem

oracle.build()
ctx = mm.Context(512, 512)


def rounds():
    for n, m in ((60, 60), (80, 120), (80, 256), (70, 500)):       # 1, 2, 4 and 8 columns a lane; 14 to 140 KB
        print("matching of", n, "x", m, flush=True)
        W = np.random.default_rng(n + m).integers(0, 1 << 20, (n, m)).astype(np.int32)
        r2c = torch.empty(n, dtype=torch.int32, device="cuda")
        u, v = torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(m, dtype=torch.int64, device="cuda")
        res = ctx.solve_assignment(padded_matrix(W), n, m, r2c, u, v)
        assert res.cert_ok == 1 and res.primal == oracle.max_weight_matching(W)[0] and res.rounds == 0


def fits():
    for H in (64, 128):
        s = close.away_from_kinks(problem(95, 500, 100, H))
        expected = close.room(s, longest=8)
        for want in (False, True):
            print("loss of", H, "units", want, flush=True)
            got = call(ctx, s, want=want)
            close.check(got, {k: expected[k] for k in got})


for what in sys.argv[1:]:
    {"rounds": rounds, "fits": fits}[what]()
torch.cuda.synchronize()
print("done", flush=True)
"""


@pytest.mark.parametrize("order", [("rounds", "fits"), ("fits", "rounds")])
def test_small_rounds_and_fits_of_many_features(order):
    done = subprocess.run([sys.executable, "-u", "-c", PROGRAM % (HERE, os.path.dirname(HERE)), *order], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and done.stdout.endswith("done\n"), done.stdout[-500:] + done.stderr[-2000:]
