"""The losses over a vocabulary on the GPU at widths up to the limit, against float64 on the GPU."""
import pytest
import torch

import vocab_wide_util as VW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,D,V", [(64, 2048, 140000), (32, 4104, 140001)])
def test_ranges_of_few_rows_that_take_turns(M, D, V):
    """Float32 rows and weights whose fragments of dX would take more than 256 MB."""
    print("[case] turns", M, D, V, flush=True)
    c, a = VW.make(M, D, V, "fp32", K=2, tau=2.0, seed=40)
    got = VW.run(c, a)
    ref = VW.reference(c, a, "fp32")
    VW.check(c, a, got, ref)
    VW.check(c, a, VW.run(c, a, want=("dX",)), ref)
    alone = VW.run(c, a, want=("dparams",))
    assert torch.equal(alone["dparams"], got["dparams"])
    again = VW.run(c, a)
    for k in got:
        assert torch.equal(got[k], again[k]), k
