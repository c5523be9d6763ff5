"""How calls of full attention are cut into jobs, on the CPU."""
import pytest

from full_plans import call, plans

MOST = 2 ** 31 - 4096 - 1   # keys of a call


@pytest.mark.parametrize("nq,nk", [(1, 65537), (25600, 1_900_000_000), (1, 2 ** 31 - 5000), (1, MOST), (33, MOST), (8192, MOST),
                                   (100_000, MOST), (2_000_000, MOST), (8192, 1_880_000_000)])
@pytest.mark.parametrize("bwd", [False, True])
def test_runs_take_every_key(bwd, nq, nk):
    """Up to the most keys that a call takes: the end of a last run is formed without passing 32 bits."""
    row, = plans([call(bwd, 1, 1, 16, 16, False, nq, nk)])
    assert row["status"] == 0 and row["keys"] == nk
