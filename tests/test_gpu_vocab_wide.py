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


# rows, width, vocabulary: 198, 335 and 201 tiles of 256 (of the 256 CUs some have two of the second), the main loop of several stages, a last
# column tile that is not full; the last is as wide as may be
LARGE = [(520, 520, 16700), (1030, 1032, 17001), (600, 2048, 17000), (270, 8192, 16900)]
LOSSES = [(0, 1.0, True), (3, 2.0, True), (5, 1.0, True), (2, 3.0, False)]


def _one_by_one(M, D, V, K, tau, labels, mode, grad="fp32", seed=41):
    print("[case]", M, D, V, K, tau, labels, mode, grad, flush=True)
    c, a = VW.make(M, D, V, mode, bias=M % 4 != 0, K=K, tau=tau, labels=labels, seed=seed)
    got, ref = VW.run(c, a, grad), VW.reference(c, a, grad)
    VW.check(c, a, got, ref, grad)
    # each gradient alone: the same dparams, dX perhaps from other ranges
    alone = VW.run(c, a, grad, want=("dparams",))
    assert torch.equal(alone["dparams"], got["dparams"])
    VW.check(c, a, VW.run(c, a, grad, want=("dX",)), ref, grad)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("K,tau,labels", LOSSES)
@pytest.mark.parametrize("M,D,V", LARGE)
def test_in_tiles_of_256(M, D, V, K, tau, labels, mode):
    _one_by_one(M, D, V, K, tau, labels, mode)


@pytest.mark.parametrize("M,D,V", [(1030, 1032, 17001), (777, 1280, 10007)])
def test_gradients_in_bfloat16(M, D, V):
    _one_by_one(M, D, V, 3, 2.0, True, "bf16", "bf16")


# more than 800 blocks of 64x64 and at most 128 tiles of 256
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("K,tau,labels", LOSSES)
@pytest.mark.parametrize("M,D,V", [(1000, 2048, 3333), (900, 1032, 5001), (520, 8192, 7001)])
def test_in_tiles_of_128(M, D, V, K, tau, labels, mode):
    _one_by_one(M, D, V, K, tau, labels, mode)


# few rows in one pass or both, from one row on
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("K,tau,labels", LOSSES)
@pytest.mark.parametrize("M,D,V", [(1, 8192, 5003), (3, 2056, 12001), (40, 8192, 501), (64, 1032, 2500), (65, 2048, 1001), (100, 8192, 600), (250, 1544, 1300)])
def test_few_rows(M, D, V, K, tau, labels, mode):
    _one_by_one(M, D, V, K, tau, labels, mode)


@pytest.mark.parametrize("mode,V", [("bf16", 40000), ("fp32", 20001)])
@pytest.mark.parametrize("share", [1.0, 0.6, 0.1])
def test_several_pieces(mode, V, share):
    """dz of all rows does not fit one piece; that of the rows which count needs fewer pieces, or one."""
    print("[case] pieces", mode, V, share, flush=True)
    c, a = VW.make(9000, 264, V, mode, K=2, tau=2.0, share=share, seed=42)
    if share < 0.5:
        a["idx"][a["labels"] < 0] = -1
    VW.check(c, a, VW.run(c, a), VW.reference(c, a, "fp32"))
