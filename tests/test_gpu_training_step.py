"""Training steps in bf16: float32 master weights with a bf16 copy, forward through a stack, a loss over a vocabulary and its gradients, the
reversible backward pass, AdamW."""
import numpy as np
import pytest
import torch

import parity_util as PU
import vocab_util as VU
from oracle import rev_oracle as O
from oracle import vocab_oracle as VO
from paper_2306_09342_amd import binding as B
from paper_2306_09342_amd import synth

pytestmark = pytest.mark.gpu

V, K, TAU = 211, 4, 2.0


def _problem():
    cfg = dict(synth.CONFIGS["tiny"], mode="bf16")
    rng = np.random.default_rng(1)
    rows, D = cfg["batch"] * cfg["seq_len"], cfg["d_model"]
    labels = rng.integers(0, V, rows).astype(np.int32)
    labels[rng.random(rows) < 0.4] = -100
    idx = rng.integers(0, V, (rows, K)).astype(np.int32)
    idx[rng.random(rows) < 0.3] = -1
    head = (rng.standard_normal(V * D + V) * 0.3).astype(np.float32)
    return cfg, synth.make_params(cfg, seed=0, perturb=True), head, synth.make_inputs(cfg, seed=0)[0], labels, idx, rng.standard_normal((rows, K)).astype(np.float32)


class Model:
    """What a program keeps from step to step: masters, their bf16 copies, moments."""

    def __init__(self, cfg, flat, head):
        self.rows, self.D = cfg["batch"] * cfg["seq_len"], cfg["d_model"]
        self.c = B.make_cfg(**cfg)
        self.vc = B.make_vocab_cfg(self.rows, self.D, V, "bf16", top_k=K, temperature=TAU)
        self.master = [VU.dev(flat), VU.dev(head)]
        self.bf16 = [m.bfloat16() for m in self.master]
        self.moments = [(torch.zeros_like(m), torch.zeros_like(m)) for m in self.master]
        self.ws, self.vws = B.alloc_workspace(self.c), torch.empty(B.rev_vocab_workspace_bytes(self.vc), dtype=torch.uint8, device="cuda")

    def gradients(self, X, labels, idx, logits, dce, dkd, side):
        params, head = self.bf16
        Y1, Y2 = B.rev_stack_forward(self.c, params, X, X, workspace=self.ws)
        H = ((Y1 + Y2) / 2).bfloat16().view(self.rows, self.D)
        f = B.rev_distill_forward(self.vc, head, H, idx, logits, labels=labels, workspace=self.vws)
        g = B.rev_distill_backward(self.vc, head, H, idx, logits, f["lse"], dkd, labels=labels, dloss_ce=dce, workspace=self.vws)
        dY = (g["dX"].float() / 2).view(Y1.shape)
        b = B.rev_stack_backward_pareprop(self.c, params, Y1, Y2, dY, dY, side, workspace=self.ws)
        return f, g, b

    def update(self, g, b, step):
        for master, copy, (m, v), grad in zip(self.master, self.bf16, self.moments, (b["dparams"], g["dparams"])):
            B.rev_adamw_step(master, grad, m, v, step, lr=1e-3, params_bf16=copy)


def test_a_step_against_the_oracles():
    cfg, flat, head, x, labels, idx, logits = _problem()
    model = Model(cfg, flat, head)
    rows, D = model.rows, model.D
    count, taught = int((labels >= 0).sum()), int((idx >= 0).any(1).sum())
    dce, dkd = np.full(rows, 0.5 / count, np.float32), np.full(rows, 0.5 / taught, np.float32)
    # the oracles, from the weights on bf16's grid
    flat_b, head_b = (m.float().cpu().numpy() for m in model.bf16)
    blocks = O.unpack_params(flat_b.astype(np.float64), cfg["n_blocks"], D, cfg["d_mlp"])
    y1, y2 = O.stack_forward(x.astype(np.float64), x.astype(np.float64), blocks, cfg["n_heads"])
    ref = VO.vocab_loss(head_b, ((y1 + y2) / 2).reshape(rows, D), V, True, labels, idx, logits, TAU, dce, dkd)
    dy = ref["dX"].reshape(y1.shape) / 2
    rdx1, rdx2, rgrads, _, _ = O.stack_backward_reversible(y1, y2, blocks, cfg["n_heads"], dy, dy)

    before = [m.clone() for m in model.master]
    f, g, b = model.gradients(VU.dev(x), VU.dev(labels), VU.dev(idx), VU.dev(logits), VU.dev(dce), VU.dev(dkd), torch.cuda.Stream())
    model.update(g, b, 1)
    torch.cuda.synchronize()
    # the stack's tolerance holds for the chain: the head adds the rounding of its rows, of dz and of dX, half a step (2^-8) each
    tol = PU.TOL["bf16"]
    for got, want in ((f["loss_ce"], ref["loss_ce"]), (f["loss"], ref["loss_kd"]), (g["dparams"], ref["dparams"]), (b["dX1"], rdx1), (b["dX2"], rdx2),
                      (b["dparams"], O.pack_params(rgrads))):
        assert PU.rel_err(got.cpu().numpy().ravel(), np.asarray(want).ravel()) <= tol
    for old, new, copy in zip(before, model.master, model.bf16):
        assert not torch.equal(old, new) and bool(torch.isfinite(new).all()) and torch.equal(copy, new.bfloat16())


def test_a_captured_step_repeats_the_eager_one():
    """Three steps, each from the weights that the last one left: eager, and as replays of one graph of the gradients, with the eager update between."""
    cfg, flat, head, x, labels, idx, logits = _problem()
    inputs = [VU.dev(a) for a in (x, labels, idx, logits)]
    rows = inputs[1].numel()
    cot = [torch.full((rows,), 1.0 / rows, device="cuda") for _ in range(2)]
    eager, captured, side = Model(cfg, flat, head), Model(cfg, flat, head), torch.cuda.Stream()
    captured.gradients(*inputs, *cot, side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f, g, b = captured.gradients(*inputs, *cot, side)
    for step in (1, 2, 3):
        ef, eg, eb = eager.gradients(*inputs, *cot, side)
        eager.update(eg, eb, step)
        graph.replay()
        captured.update(g, b, step)
        torch.cuda.synchronize()
        for one, two in ((ef, f), (eg, g), (eb, b)):
            for k in one:
                assert one[k] is None or torch.equal(one[k], two[k]), (step, k)
        for one, two in zip(eager.master, captured.master):
            assert torch.equal(one, two), step
