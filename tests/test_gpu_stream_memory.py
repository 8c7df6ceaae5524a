"""Calls on a stream of the caller's, in memory of their own, while work is queued on the current stream that uses what it has just freed."""
import pytest
import torch

import vocab_util as VU
from paper_2306_09342_amd import binding as B
from paper_2306_09342_amd import synth

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


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_stack(mode):
    cfg = dict(synth.CONFIGS["tiny"], mode=mode)
    c = B.make_cfg(**cfg)
    params = VU.dev(synth.make_params(cfg, seed=0, perturb=True), B.param_dtype(c))
    X, dY1, dY2 = (VU.dev(a) for a in synth.make_inputs(cfg, seed=0))

    def run(side=None, other=None):
        streams = [side, other] if side else [None, torch.cuda.Stream()]
        Y1, Y2 = B.rev_stack_forward(c, params, X, X, stream=side)
        out = [Y1, Y2]
        if side:
            _queue_work_on_freed_memory()
        for r in (B.rev_stack_backward_reprop(c, params, Y1, Y2, dY1, dY2, stream=side),
                  B.rev_stack_backward_pareprop(c, params, Y1, Y2, dY1, dY2, streams[1], stream_grad=streams[0])):
            out += [r[k] for k in ("dX1", "dX2", "dparams")]
        torch.cuda.synchronize()
        return out

    ref = run()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        _queue_work_on_freed_memory()
        for a, b in zip(ref, run(side, other)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_stage_transition(mode):
    c = B.make_merge_cfg(2, 8, 8, 4, 64, mode)
    g = torch.Generator().manual_seed(5)
    params = (0.3 * torch.randn(B.rev_merge_param_count(c), generator=g)).cuda().to(B.param_dtype(c))
    X1, X2, dA, dB = (torch.randn(s, generator=g).cuda() for s in ((128, 64), (128, 64), (32, 128), (32, 128)))

    def run(side=None):
        out = [B.rev_merge_forward(c, params, X1, X2, stream=side)]
        r = B.rev_merge_backward(c, params, X1, X2, dA, dB, stream=side)
        torch.cuda.synchronize()
        return out + [r[k] for k in ("dX1", "dX2", "dparams")]

    ref = run()
    side = torch.cuda.Stream()
    for _ in range(3):
        _queue_work_on_freed_memory()
        for a, b in zip(ref, run(side)):
            assert torch.equal(a, b)


def test_a_stream_that_joins_a_capture():
    """Calls on a stream forked from the captured one, in memory of their own: replays repeat the eager results."""
    c = VU.make(300, 128, 1500, "bf16", K=2, tau=2.0, seed=27)
    ref = VU.run(c)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        f = VU.forward(cfg, c, a, stream=side)
        f.update(VU.backward(cfg, c, a, f["stats"], stream=side))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
        VU.run(c)
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(ref[k], f[k]), k
        for t in f.values():
            t.fill_(3.0)
