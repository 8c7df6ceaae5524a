"""Calls on a stream of the caller's, in memory of their own, while work is queued on the current stream that uses what it has just freed."""
import pytest
import torch

import vocab_util as VU

pytestmark = pytest.mark.gpu


def _queue_work_on_freed_memory():
    """Some 20 ms of it, in blocks of every size that a call may ask for."""
    torch.cuda.empty_cache()
    junk = [torch.empty(n, device="cuda") for n in (1 << 28, *[1 << k for k in (8, 10, 12, 14, 16, 18, 20)] * 3)]
    for _ in range(60):
        for t in junk:
            t.fill_(float("nan"))


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [6, 300])
def test_losses_over_a_vocabulary(M, mode):
    c = VU.make(M, 128, 1500, mode, K=2, tau=2.0, seed=26)
    ref = VU.run(c)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        _queue_work_on_freed_memory()
        f = VU.forward(cfg, c, a, stream=side)
        _queue_work_on_freed_memory()
        f.update(VU.backward(cfg, c, a, f["stats"], stream=side))
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(ref[k], f[k]), k
