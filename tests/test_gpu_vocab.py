"""The losses over a vocabulary on the GPU against the float64 oracle: every output at every element, within what its roundings add up to."""
import numpy as np
import pytest
import torch

import vocab_util as VU
from paper_2306_09342_amd import binding as B

pytestmark = pytest.mark.gpu

# rows, width, vocabulary
SHAPES = [(1, 8, 1), (1, 64, 2), (2, 8, 3), (3, 16, 7), (1, 768, 1003), (5, 128, 257), (16, 72, 300), (33, 200, 255), (64, 384, 1000),
          (65, 136, 1001), (129, 128, 2049), (200, 256, 513), (257, 64, 770), (300, 384, 1025), (130, 520, 1290), (513, 32, 256)]


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_cross_entropy(shape, mode):
    M, D, V = shape
    print("[case] cross entropy", shape, mode, flush=True)
    VU.check(VU.make(M, D, V, mode, bias=M % 2 == 1, share=1.0 if M < 30 else 0.7, seed=M), "fp32")


# sizes whose logits take tiles of 256: more than 128 of them
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(300, 64, 16641), (513, 128, 11009), (769, 40, 8450)])
def test_cross_entropy_in_large_tiles(shape, mode):
    M, D, V = shape
    print("[case] cross entropy", shape, mode, flush=True)
    VU.check(VU.make(M, D, V, mode, bias=M % 2 == 1, share=0.8, seed=M), "fp32")


# sizes whose logits take tiles of 128 in both passes: more than 800 blocks of 64x64, at most 128 tiles of 256
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("shape,K,tau,labels", [((600, 40, 6001), 0, 1.0, True), ((1100, 72, 3333), 0, 1.0, True), ((1000, 72, 3333), 4, 2.0, True),
                                                ((520, 64, 7001), 5, 2.0, True),
                                                ((700, 136, 5121), 3, 0.5, False)])
def test_in_tiles_of_128(shape, K, tau, labels, mode):
    M, D, V = shape
    print("[case] tiles of 128", shape, K, tau, labels, mode, flush=True)
    VU.check(VU.make(M, D, V, mode, bias=M != 600, K=K, share=0.8, labels=labels, tau=tau, seed=M), "fp32")


@pytest.mark.parametrize("mode,grad", [("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("M,D,V,K,share", [(4097, 40, 130, 0, 1.0), (2600, 264, 301, 3, 0.9), (3000, 8, 1, 0, 0.02), (2049, 520, 257, 0, 0.5), (5000, 128, 900, 0, 0.0)])
def test_many_rows_and_few_weights(M, D, V, K, share, mode, grad):
    """dW in a few tiles, whose rows are cut into ranges."""
    print("[case] ranges of rows", M, D, V, K, share, mode, grad, flush=True)
    VU.check(VU.make(M, D, V, mode, bias=M != 2600, K=K, share=share, seed=M), grad)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("K,tau,labels", [(1, 1.0, False), (5, 1.0, True), (33, 2.0, False), (70, 4.0, True)])
def test_distillation_in_large_tiles(K, tau, labels, mode):
    print("[case] distillation", K, tau, labels, mode, flush=True)
    c = VU.make(290, 64, 16700, mode, bias=labels, K=K, share=0.8, labels=labels, tau=tau, seed=K)
    c["idx"][3] = 16699                        # one entry, K times, the vocabulary's last
    c["idx"][40:140, 0] = np.arange(100) % 64  # many rows name the same 64 entries
    if K > 1:
        c["idx"][200] = np.arange(K)           # more than a tile's wavefront looks at in one go, with those around
        c["idx"][192:224, 1:] = (np.arange(K - 1) * 7) % 61
        if labels:
            c["labels"][195] = c["idx"][195, 1]
    VU.check(c, "fp32")


@pytest.mark.parametrize("mode,M,D,V,K", [("bf16", 20000, 8, 16000, 3), ("fp32", 12000, 8, 10001, 3), ("bf16", 70001, 8, 45000, 2), ("bf16", 70001, 8, 44101, 0)])
def test_several_pieces_of_the_vocabulary(mode, M, D, V, K):
    """Sizes whose dz, and for 70001 rows whose statistics, do not fit one piece, against torch in float64 on the GPU."""
    print("[case] pieces", mode, M, D, V, K, flush=True)
    c = VU.make(M, D, V, mode, K=K, tau=2.0, share=0.9, seed=21)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    f = VU.forward(cfg, c, a)
    b = VU.backward(cfg, c, a, f["stats"])
    W, bias = a["params"][:V * D].view(V, D).double(), a["params"][V * D:].double()
    half, tol = VU.HALF[mode], 2e-5
    dW, dWa, db, dba = torch.zeros_like(W), torch.zeros_like(W), torch.zeros_like(bias), torch.zeros_like(bias)
    dX = torch.zeros(M, D, dtype=torch.float64, device="cuda")
    for r in range(0, M, 4000):
        s = slice(r, min(M, r + 4000))
        x = a["X"][s].double()
        z = x @ W.T + bias
        y = a["labels"][s].long()
        has = y >= 0
        lse = torch.logsumexp(z, 1)
        ce = torch.where(has, lse - z.gather(1, y.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
        assert torch.linalg.norm(f["loss_ce"][s].double() - ce) <= tol * torch.linalg.norm(ce)
        dz = torch.exp(z - lse[:, None])
        dz[torch.arange(len(y), device="cuda"), y.clamp(min=0)] -= 1.0
        dz *= (a["dce"][s].double() * has)[:, None]
        if K:
            idx = a["idx"][s].long()
            on = idx >= 0
            t = torch.where(on, a["logits"][s].double() / 2.0, torch.full_like(idx, -np.inf, dtype=torch.float64))
            taught = on.any(1)
            p = torch.where(on, torch.softmax(t, 1), torch.zeros_like(t))
            logq = torch.log_softmax(z / 2.0, 1)
            kd = 4.0 * torch.where(p > 0, p * (torch.log(p) - logq.gather(1, idx.clamp(min=0))), torch.zeros_like(p)).sum(1)
            kd = torch.where(taught, kd, torch.zeros_like(kd))
            assert torch.linalg.norm(f["loss_kd"][s].double() - kd) <= tol * torch.linalg.norm(kd)
            g = logq.exp()
            g.scatter_add_(1, idx.clamp(min=0), -p)
            dz += g * (a["dkd"][s].double() * taught * 2.0)[:, None]
        dX[s] = dz @ W
        dW += dz.T @ x
        dWa += dz.abs().T @ x.abs()
        db += dz.sum(0)
        dba += dz.abs().sum(0)
    gW, gb = b["dparams"][:V * D].view(V, D).double(), b["dparams"][V * D:].double()
    # dz rounded once, its float32 errors below 2e-5 of it, and sums of M terms in float32
    lim = half * 1.01 + 2e-5 + M * VU.U
    assert ((gW - dW).abs() <= lim * dWa + 1e-9).all() and ((gb - db).abs() <= lim * dba + 1e-9).all()
    norm = 4 * half if mode == "bf16" else 2e-5
    for got, want in ((gW, dW), (gb, db), (b["dX"].double(), dX)):
        assert torch.linalg.norm(got - want) <= norm * torch.linalg.norm(want)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("K,tau", [(1, 1.0), (3, 2.0), (64, 4.0), (65, 0.5), (256, 1.0)])
@pytest.mark.parametrize("labels", [False, True])
def test_distillation(K, tau, labels, mode):
    print("[case] distillation", K, tau, labels, mode, flush=True)
    VU.check(VU.make(70, 136, 515, mode, bias=labels, K=K, share=0.8, labels=labels, tau=tau, seed=K), "fp32")


@pytest.mark.parametrize("shape", [(1, 64, 33), (4, 768, 1001), (300, 320, 1290)])
def test_distillation_shapes(shape):
    M, D, V = shape
    print("[case] distillation", shape, flush=True)
    VU.check(VU.make(M, D, V, "bf16", K=6, tau=2.0, share=0.9, seed=5), "bf16")


def test_bfloat16_gradients_are_the_float32_ones_rounded():
    c = VU.make(150, 256, 777, "bf16", share=0.6, seed=1)
    a, b = VU.run(c, "fp32"), VU.run(c, "bf16")
    assert torch.equal(a["dparams"].bfloat16(), b["dparams"]) and torch.equal(a["dX"], b["dX"])


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("alive", [0, 1, 2])
def test_few_rows_count(alive, mode):
    c = VU.make(300, 128, 600, mode, seed=2)
    keep = c["labels"][:].copy()
    c["labels"][:] = -1
    for r in (299, 17)[:alive]:
        c["labels"][r] = keep[r]
    c["labels"][5], c["labels"][6], c["labels"][7] = 600, 2 ** 31 - 1, -2 ** 31
    got, _ = VU.check(c)
    if alive == 0:
        assert all(not got[k].any() for k in ("loss_ce", "lse", "dX", "dparams"))


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [0, 4])
def test_rows_that_do_not_count_may_hold_anything(K, mode):
    c = VU.make(90, 64, 300, mode, K=K, share=0.5, seed=3)
    ref = VU.run(c)
    on = (c["labels"] >= 0) | ((c["idx"] >= 0).any(1) if K else False)
    assert 0 < on.sum() < 90
    for r in np.nonzero(~on)[0]:
        c["X"][r] = (np.nan, np.inf, -np.inf)[r % 3]
        c["dce"][r] = c["dkd"][r] = np.nan
        if K:
            c["logits"][r] = np.nan
    got = VU.run(c)
    for k in ref:
        assert torch.equal(ref[k], got[k]), k


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
def test_entries_taken_out_by_the_bias(low, mode):
    c = VU.make(80, 64, 1100, mode, seed=4)
    worst = -np.inf if low == "-inf" else float(torch.finfo(torch.bfloat16 if mode == "bf16" else torch.float32).min)
    b = c["params"][1100 * 64:]
    b[0:300] = worst                       # a whole tile of any size, and the first
    b[301:1090:7] = worst
    b[1095:] = worst                       # the last
    keep = np.nonzero(b > -1e30)[0]
    c["labels"] = np.where(c["labels"] >= 0, keep[np.abs(c["labels"]) % len(keep)], -1).astype(np.int32)
    VU.check(c)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("M,V", [(6, 900), (300, 1100), (300, 17000)])
def test_a_row_that_is_not_a_number_keeps_it_to_itself(M, V, mode):
    c = VU.make(M, 64, V, mode, K=3, tau=2.0, seed=20)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    one = VU.forward(cfg, c, a)
    one.update(VU.backward(cfg, c, a, one["stats"], want=("dX",)))
    a["X"][2, 5] = float("nan")
    two = VU.forward(cfg, c, a)
    two.update(VU.backward(cfg, c, a, two["stats"], want=("dX",)))
    for k in ("loss_ce", "loss_kd", "lse", "lse_tau", "dX"):
        assert torch.isnan(two[k][2]).all(), k
        two[k][2] = one[k][2]
        assert torch.equal(one[k], two[k]), k


def test_a_label_that_the_bias_took_out():
    c = VU.make(4, 64, 50, "fp32", seed=6)
    c["params"][50 * 64 + 7] = -np.inf
    c["labels"][:] = [7, 3, 7, 9]
    got = VU.run(c)
    assert torch.isinf(got["loss_ce"]).cpu().tolist() == [True, False, True, False]
    assert torch.isfinite(got["dX"]).all() and torch.isfinite(got["dparams"]).all()


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_large_logits(mode):
    c = VU.make(40, 64, 700, mode, K=3, tau=2.0, seed=7, scale=3000.0)
    VU.check(c)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_teachers_with_repeats_and_gaps(mode):
    c = VU.make(12, 64, 90, mode, K=8, tau=1.5, seed=8)
    c["idx"][0] = 5                                              # one entry, eight times
    c["idx"][1] = [3, 3, 7, 7, 7, -1, 90, 3]
    c["logits"][2, :7] = -np.inf                                 # one left
    c["logits"][3] = -np.inf                                     # none
    c["idx"][4] = c["labels"][4]                                 # the label too
    c["labels"][5] = -1
    c["idx"][6] = -5
    c["logits"][7] = [100.0, -100.0, 0.0, 99.0, -3e38, 1.0, 2.0, 3.0]
    c["idx"][8, 0] = 89
    VU.check(c)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0])
def test_teachers_that_know_lowest_values_alone(tau, mode):
    """They are equally likely, as entries of logit 0 are: the same results, bit for bit."""
    c = VU.make(30, 64, 200, mode, K=70, tau=tau, seed=19)
    c["logits"][::2] = 0.0
    ref, _ = VU.check(c)
    c["logits"][::2] = np.finfo(np.float32).min
    got = VU.run(c)
    for k in ref:
        assert torch.equal(ref[k], got[k]), k


def test_a_student_that_is_its_teacher():
    """The gradient is a difference of two nearly equal probabilities: taken in float32, rounded once."""
    c = VU.make(20, 64, 120, "bf16", bias=False, K=120, tau=2.0, labels=False, seed=9)
    W = c["params"].astype(np.float64).reshape(120, 64)
    c["idx"][:] = np.arange(120)
    c["logits"] = (c["X"].astype(np.float64) @ W.T * 1.01).astype(np.float32)
    VU.check(c)


@pytest.mark.parametrize("want", [("dX",), ("dparams",)])
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_one_gradient_alone(want, mode):
    c = VU.make(100, 96, 500, mode, K=2, seed=10)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    f = VU.forward(cfg, c, a)
    both = VU.backward(cfg, c, a, f["stats"])
    one = VU.backward(cfg, c, a, f["stats"], want=want)
    assert set(one) == set(want) and torch.equal(one[want[0]], both[want[0]])


@pytest.mark.parametrize("mode,grad", [("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("shape", [(37, 136, 515), (300, 128, 259), (3, 64, 1001)])
def test_nothing_is_written_behind_the_outputs_and_the_workspace_may_hold_anything(shape, mode, grad):
    M, D, V = shape
    c = VU.make(M, D, V, mode, K=3, share=0.8, seed=11)
    cfg, a = VU.make_cfg(c, grad), VU.gpu_args(c)
    ref = VU.run(c, grad)
    n = B.rev_vocab_workspace_bytes(cfg)
    outs, pads = {}, []

    def padded(shape, dtype):
        size = int(np.prod(shape))
        t = torch.full((size + 64,), 7.0, dtype=dtype, device="cuda")
        pads.append((t, size))
        return t[:size].view(shape)

    for fill in (0, 255):
        ws = torch.full((n + 4096,), fill, dtype=torch.uint8, device="cuda")
        pads.clear()
        dt = a["X"].dtype
        outs = {"loss": padded((M,), torch.float32), "loss_ce": padded((M,), torch.float32), "lse": padded((2, M), torch.float32),
                "dX": padded((M, D), dt), "dparams": padded((a["params"].numel(),), torch.bfloat16 if grad == "bf16" else torch.float32)}
        f = VU.forward(cfg, c, a, workspace=ws[:n], out=outs)
        b = VU.backward(cfg, c, a, f["stats"], workspace=ws[:n], out=outs)
        torch.cuda.synchronize()
        assert (ws[n:] == fill).all()
        for t, size in pads:
            assert (t[size:] == 7.0).all()
        for k in ("loss_ce", "loss_kd"):
            assert torch.equal(f[k], ref[k])
        for k in ("dX", "dparams"):
            assert torch.equal(b[k], ref[k])


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_many_rows_of_few_columns(mode):
    M, D, V = 70001, 8, 5
    c = VU.make(M, D, V, mode, share=0.5, seed=12)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    f = VU.forward(cfg, c, a)
    b = VU.backward(cfg, c, a, f["stats"])
    z = a["X"].double() @ a["params"][:V * D].view(V, D).double().T + a["params"][V * D:].double()
    y = a["labels"].long()
    on = y >= 0
    logp = torch.log_softmax(z, 1)
    ce = torch.where(on, -logp.gather(1, y.clamp(min=0)[:, None])[:, 0], torch.zeros_like(z[:, 0]))
    assert torch.allclose(f["loss_ce"].double(), ce, atol=2e-5, rtol=2e-5)
    dz = (logp.exp() - torch.nn.functional.one_hot(y.clamp(min=0), V)) * (a["dce"].double() * on)[:, None]
    half = VU.HALF[mode]
    e = (dz.abs() * half + 1e-5 * dz.abs().amax()).T @ a["X"].double().abs() * 1.1
    assert ((b["dparams"][:V * D].view(V, D).double() - dz.T @ a["X"].double()).abs() <= e + M * VU.U * (dz.abs().T @ a["X"].double().abs())).all()
    dX = dz @ a["params"][:V * D].view(V, D).double()
    assert torch.linalg.norm(b["dX"].double() - dX) <= (4 * half if mode == "bf16" else 2e-5) * torch.linalg.norm(dX)


def test_many_pieces_that_no_row_needs():
    """So many rows, of which so few count, that the pieces which all of them would need lie as far as 2^32 entries behind the vocabulary."""
    M, D, V, on = 524800, 8, 1 << 20, 200
    g = torch.Generator(device="cuda").manual_seed(22)
    guarded = torch.full((V * D + 2 * 4096,), 7.0, device="cuda")
    params = torch.randn(V * D, generator=g, device="cuda").bfloat16()
    X = torch.randn(M, D, generator=g, device="cuda").bfloat16()
    rows = torch.arange(on, device="cuda") * 2600
    labels = torch.full((M,), -100, dtype=torch.int32, device="cuda")
    labels[rows] = torch.randint(0, V, (on,), generator=g, device="cuda", dtype=torch.int32)
    dloss = torch.rand(M, generator=g, device="cuda")
    cfg = B.make_vocab_cfg(M, D, V, "bf16", bias=False)
    f = B.rev_xent_forward(cfg, params, X, labels)
    b = B.rev_xent_backward(cfg, params, X, labels, f["lse"], dloss, out={"dparams": guarded[4096:-4096]})
    W, x, y = params.view(V, D).double(), X[rows].double(), labels[rows].long()
    z = x @ W.T
    lse = torch.logsumexp(z, 1)
    ce = lse - z.gather(1, y[:, None])[:, 0]
    assert torch.linalg.norm(f["loss"][rows].double() - ce) <= 2e-5 * torch.linalg.norm(ce)
    dz = torch.exp(z - lse[:, None])
    dz[torch.arange(on, device="cuda"), y] -= 1.0
    dz *= dloss[rows].double()[:, None]
    half = VU.HALF["bf16"]
    for got, want in ((b["dparams"].view(V, D), dz.T @ x), (b["dX"][rows], dz @ W)):
        assert torch.linalg.norm(got.double() - want) <= 4 * half * torch.linalg.norm(want)
    assert (guarded[:4096] == 7.0).all() and (guarded[-4096:] == 7.0).all()
    off = torch.ones(M, dtype=torch.bool, device="cuda")
    off[rows] = False
    assert not f["loss"][off].any() and not b["dX"][off].any()


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_repeats_bit_for_bit_on_any_stream_and_two_at_once(mode):
    c = VU.make(600, 256, 3001, mode, K=4, share=0.7, tau=2.0, seed=13)
    ref = VU.run(c, "fp32")
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            ws = torch.empty(B.rev_vocab_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
            f = VU.forward(cfg, c, a, workspace=ws)
            f.update(VU.backward(cfg, c, a, f["stats"], workspace=ws))
            got.append((f, ws))
    torch.cuda.synchronize()
    for f, _ in got:
        for k in ref:
            assert torch.equal(f[k], ref[k]), k


@pytest.mark.parametrize("M,D,V", [(4, 64, 501), (300, 64, 700), (70001, 8, 45000)])
def test_the_timing_of_kernel_families_counts_the_products_once(M, D, V):
    c = VU.make(M, D, V, "bf16", K=2, seed=23)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    B.rev_profile_begin()
    f = VU.forward(cfg, c, a)
    VU.backward(cfg, c, a, f["stats"])
    _, launches, work, is_flops = B.rev_profile_end()["vocab"]
    assert work == pytest.approx(4 * 2.0 * M * D * V) and launches >= 3 and is_flops


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [4, 300])
def test_captured_and_replayed_with_other_inputs(M, mode):
    c = VU.make(M, 128, 1001, mode, K=3, share=0.9, seed=14)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    ws = torch.empty(B.rev_vocab_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    VU.backward(cfg, c, a, VU.forward(cfg, c, a, workspace=ws)["stats"], workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f = VU.forward(cfg, c, a, workspace=ws)
        f.update(VU.backward(cfg, c, a, f["stats"], workspace=ws))
    for seed in (15, 16, 17):
        d = VU.make(M, 128, 1001, mode, K=3, share=0.3 * (seed - 14), seed=seed)
        for k, v in VU.gpu_args(d).items():
            a[k].copy_(v)
        g.replay()
        torch.cuda.synchronize()
        eager = VU.run(d)
        for k in eager:
            assert torch.equal(f[k], eager[k]), (seed, k)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [7, 300])
def test_two_graphs_that_share_a_workspace(M, mode):
    """Forward and backward captured apart, another problem's call in the same workspace between the replays."""
    c, d = VU.make(M, 64, 901, mode, K=2, tau=2.0, seed=24), VU.make(M, 64, 901, mode, K=2, tau=2.0, share=0.4, seed=25)
    cfg, a, b = VU.make_cfg(c), VU.gpu_args(c), VU.gpu_args(d)
    ws = torch.empty(B.rev_vocab_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    ref = VU.run(c)
    VU.backward(cfg, c, a, VU.forward(cfg, c, a, workspace=ws)["stats"], workspace=ws)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        f = VU.forward(cfg, c, a, workspace=ws)
    with torch.cuda.graph(g2):
        g = VU.backward(cfg, c, a, f["stats"], workspace=ws)
    for _ in range(3):
        g1.replay()
        VU.backward(cfg, d, b, VU.forward(cfg, d, b, workspace=ws)["stats"], workspace=ws)
        g2.replay()
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(ref[k], (f if k in f else g)[k]), k
        for t in (*f.values(), *g.values()):
            t.fill_(3.0)


def test_a_stream_given_by_name_and_memory_of_the_call_itself():
    c = VU.make(300, 128, 1500, "bf16", K=2, seed=26)
    ref = VU.run(c)
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        f = VU.forward(cfg, c, a, stream=side)
        f.update(VU.backward(cfg, c, a, f["stats"], stream=side))
        junk = [torch.full((1 << 22,), float("nan"), device="cuda") for _ in range(4)]      # takes no memory of the calls that run
        torch.cuda.current_stream().wait_stream(side)
        for k in ref:
            assert torch.equal(ref[k], f[k]), k
        del junk


def test_a_row_does_not_depend_on_the_rows_beside_it():
    c = VU.make(400, 128, 2000, "bf16", seed=18)
    one = VU.run(c)
    c["X"][200:] = -c["X"][200:]
    two = VU.run(c)
    assert torch.equal(one["loss_ce"][:200], two["loss_ce"][:200]) and torch.equal(one["dX"][:200], two["dX"][:200])


def test_a_training_step_through_a_stack_and_the_loss():
    """Forward, loss, gradients of the head, reversible backward, AdamW: together against the oracles."""
    from oracle import rev_oracle as O
    from oracle import vocab_oracle as VO
    from paper_2306_09342_amd import synth
    cfg = dict(synth.CONFIGS["tiny"], mode="fp32")
    flat = synth.make_params(cfg, seed=0, perturb=True)
    x, _, _ = synth.make_inputs(cfg, seed=0)
    N, T, D, V = cfg["batch"], cfg["seq_len"], cfg["d_model"], 211
    rng = np.random.default_rng(0)
    head = (rng.standard_normal(V * D + V) * 0.3).astype(np.float32)
    labels = rng.integers(0, V, N * T).astype(np.int32)
    labels[rng.random(N * T) < 0.4] = -100
    count = int((labels >= 0).sum())
    # oracles
    blocks = O.unpack_params(flat.astype(np.float64), cfg["n_blocks"], D, cfg["d_mlp"])
    y1, y2 = O.stack_forward(x.astype(np.float64), x.astype(np.float64), blocks, cfg["n_heads"])
    h = ((y1 + y2) / 2).reshape(N * T, D)
    ref = VO.vocab_loss(head, h, V, True, labels, dce=np.full(N * T, 1.0 / count))
    dy = ref["dX"].reshape(N, T, D) / 2
    rdx1, rdx2, rg, _, _ = O.stack_backward_reversible(y1, y2, blocks, cfg["n_heads"], dy, dy)
    # the framework
    c, dev = B.make_cfg(**cfg), VU.dev
    params, X = dev(flat), dev(x)
    Y1, Y2 = B.rev_stack_forward(c, params, X, X)
    vc = B.make_vocab_cfg(N * T, D, V, "fp32")
    H = ((Y1 + Y2) / 2).view(N * T, D)
    head_gpu = dev(head)
    f = B.rev_xent_forward(vc, head_gpu, H, dev(labels))
    g = B.rev_xent_backward(vc, head_gpu, H, dev(labels), f["lse"], torch.full((N * T,), 1.0 / count, device="cuda"))
    dY = (g["dX"] / 2).view(N, T, D)
    b = B.rev_stack_backward_pareprop(c, params, Y1, Y2, dY, dY, torch.cuda.Stream())
    for master, grad in ((params, b["dparams"]), (head_gpu, g["dparams"])):
        before = master.clone()
        m, v = torch.zeros_like(master), torch.zeros_like(master)
        B.rev_adamw_step(master, grad, m, v, 1, lr=1e-3)
        assert not torch.equal(before, master) and torch.isfinite(master).all()
    torch.cuda.synchronize()

    def near(got, want, tol=1e-4):
        got = got.cpu().numpy().astype(np.float64).ravel()
        want = np.asarray(want).ravel()
        assert np.abs(got - want).max() <= tol * np.abs(want).max()

    near(f["loss"], ref["loss_ce"])
    near(g["dparams"], ref["dparams"])
    near(b["dX1"], rdx1)
    near(b["dX2"], rdx2)
    near(b["dparams"], O.pack_params(rg))


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("M,V", [(6, 900), (300, 1100), (900, 5001), (900, 17000)])
def test_an_entry_that_is_not_a_number(M, V, value, tau, mode):
    """One entry's bias leaves no log-sum-exp: then every dz of a row that counts is no number, whatever of label and teacher the row has."""
    for have in ("label", "teacher", "both"):
        c = VU.make(M, 64, V, mode, K=3, tau=tau, seed=30)
        if have == "label":
            c["idx"][:] = -1
        if have == "teacher":
            c["labels"][:] = -100
        c["labels"][1] = -100
        c["idx"][1] = -1                                       # a row that does not count
        c["params"][V * 64 + V // 2] = value
        got = VU.run(c)
        on = (c["labels"] >= 0) | (c["idx"] >= 0).any(1)
        assert on[2] and not on[1]
        nan = {k: torch.isnan(v).cpu().numpy() for k, v in got.items()}
        assert nan["dX"][on].all() and nan["dparams"].all(), have
        if have != "teacher":
            assert nan["lse"][on].all() and nan["loss_ce"][on].all(), have
        if have != "label":
            assert nan["lse_tau"][on].all() and nan["loss_kd"][on].all(), have
        for k in ("loss_ce", "loss_kd", "lse", "lse_tau", "dX"):
            assert not got[k][1].any(), k


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("M,V", [(6, 900), (300, 1100), (900, 5001), (900, 17000)])
def test_a_cotangent_of_zero_hides_no_nan(M, V, tau, mode):
    c = VU.make(M, 64, V, mode, K=3, tau=tau, seed=31)
    c["labels"][3], c["idx"][4] = -100, -1                     # a teacher alone, a label alone
    for r in (2, 3, 4):
        c["X"][r, 7] = np.nan
        c["dce"][r] = c["dkd"][r] = 0.0
    c["dce"][5] = c["dkd"][5] = 0.0
    got = VU.run(c)
    nan = torch.isnan(got["dX"]).sum(1).cpu().tolist()
    assert nan[:6] == [0, 0, 64, 64, 64, 0] and not any(nan[6:])
    assert not got["dX"][5].any() and int(torch.isnan(got["dparams"]).sum()) == V * 65


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("M,V,K", [(6, 900, 3), (7, 900, 70), (300, 1100, 3), (900, 17000, 5)])
def test_a_teacher_that_is_not_a_number(M, V, K, mode):
    """NaN or +infinity among a row's teacher logits: no number in that row's divergence, and the last row's too, behind which there are no named logits."""
    c = VU.make(M, 64, V, mode, K=K, tau=2.0, seed=32)
    c["idx"][3, 1], c["idx"][M - 1, 0] = 5, 7
    cfg, a = VU.make_cfg(c), VU.gpu_args(c)
    one = VU.forward(cfg, c, a)
    one.update(VU.backward(cfg, c, a, one["stats"], want=("dX",)))
    a["logits"][3, 1], a["logits"][M - 1, 0] = float("nan"), float("inf")
    two = VU.forward(cfg, c, a)
    two.update(VU.backward(cfg, c, a, two["stats"], want=("dX",)))
    for k in ("loss_kd", "dX"):
        assert torch.isnan(two[k][[3, M - 1]]).all(), k
        two[k][[3, M - 1]] = one[k][[3, M - 1]]
    for k in ("loss_ce", "loss_kd", "lse", "lse_tau", "dX"):
        assert torch.equal(one[k], two[k]), k
