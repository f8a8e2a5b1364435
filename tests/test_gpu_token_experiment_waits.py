"""A training run does not return figures from matrix products whose bounded waits have given up."""
import pytest

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200 import token_experiment as te

pytestmark = pytest.mark.gpu

SMALL = dict(n=2, T=32, vocab=16, dim=16, iters=3, every=2, gamma=0.1, hidden=24)


def test_a_run_reports_a_wait_that_gave_up():
    pkg.token_status()
    assert pkg.lib().gpga_selftest_token_wait(None) == pkg.GPGA_OK
    with pytest.raises(pkg.GpgaError) as err:
        te.train("Gossip-PGA, ring", pkg.GPGA_TOPO_RING, 2, **SMALL)
    assert err.value.status == pkg.GPGA_ERR_TIMEOUT
    out = te.train("Gossip-PGA, ring", pkg.GPGA_TOPO_RING, 2, **SMALL)      # reported once
    assert len(out["trajectory"]) == 2
    pkg.token_status()
