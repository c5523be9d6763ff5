"""How calls of full attention are cut into jobs, on the CPU."""
import pytest

from full_forms import FORMS, PAIRS, case, expected
from full_plans import call, plans

MOST = 2 ** 31 - 4096 - 1   # keys of a call


@pytest.mark.parametrize("nq,nk", [(1, 65537), (25600, 1_900_000_000), (1, 2 ** 31 - 5000), (1, MOST), (33, MOST), (8192, MOST),
                                   (100_000, MOST), (2_000_000, MOST), (8192, 1_880_000_000)])
@pytest.mark.parametrize("bwd", [False, True])
def test_runs_take_every_key(bwd, nq, nk):
    """Up to the most keys that a call takes: the end of a last run is formed without passing 32 bits."""
    row, = plans([call(bwd, 1, 1, 16, 16, False, nq, nk)])
    assert row["status"] == 0 and row["keys"] == nk


@pytest.mark.parametrize("name", list(FORMS))
def test_forms(name):
    """Each form's call reaches the form it is for, at every pair of widths: a change of the plan's lines leaves none untested."""
    H, Hk, qo, ko = case(name)
    rows = plans([call(bwd, H, Hk, d, dv, True, qo[-1], ko[-1], qo, ko) for d, dv in PAIRS for bwd in (False, True)])
    for (d, dv), fwd, bwd in zip(PAIRS, rows[::2], rows[1::2]):
        for plan, (tile, halves, split, jobs, launches) in ((p, {**fwd, **bwd}[p]) for p in ("fwd", "dq", "dkv")):
            assert (tile, halves, split > 0) == expected(name, plan, d, dv), (plan, d, dv)
            assert launches == 1
            if name in ("many", "folded"):
                assert (jobs > 512) == (name == "many"), (plan, d, dv)
