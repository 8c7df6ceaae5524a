"""The losses over a vocabulary, as cases that can be timed and compared.

``op``    ``xent``     softmax cross entropy of a linear map to a vocabulary, one label per row
          ``distill``  the divergence from a teacher of which its largest logits are known, alone or (``labels``) with the
                       cross entropy of labels beside it
``pass_`` ``forward``  evaluation: losses and log-sum-exps;  ``train`` the same and then the gradients of the rows and of the map

Rows are what leaves a final LayerNorm: standard normal, moved towards the weights of their label as those of a model
that has learned something are.  Weights are normal and give logits with a standard deviation of 2.5.
"""
import math

import torch

own = False


def _case(name, op, pass_, rows, d_model, vocab, mode="bf16", bias=True, share=1.0, labels=True, top_k=0, temperature=1.0):
    return dict(name=name, op=op, pass_=pass_, rows=rows, d_model=d_model, vocab=vocab, mode=mode, bias=bias, share=share,
                labels=labels, top_k=top_k, temperature=temperature)


def listed():
    return [
        # the log-probability of one next token: everything is the reading of the weights
        _case("xent_score_one", "xent", "forward", 1, 768, 50265),
        # image classification at the benchmark's batch of 64: few rows, few classes, launch latency
        _case("xent_classes", "xent", "train", 64, 768, 1000),
        # the same in float32, a smaller model at its batch of 128
        _case("xent_classes_fp32", "xent", "train", 128, 384, 1000, mode="fp32"),
        # masked language modelling, 32 sequences of 512 tokens: 15 of 100 positions carry a label
        _case("xent_masked", "xent", "train", 16384, 768, 50265, share=0.15),
        # evaluation of a text model, 16 sequences of 512 tokens
        _case("xent_evaluate", "xent", "forward", 8192, 1024, 50265),
        # training on every position over a vocabulary of 2^17
        _case("xent_wide", "xent", "train", 8192, 1024, 131072, bias=False),
        # a float32 run of moderate size
        _case("xent_fp32", "xent", "train", 1000, 768, 32000, mode="fp32", bias=False, share=0.5),
        # a student's divergence on the last tokens of 16 sequences
        _case("distill_few", "distill", "forward", 16, 1024, 50265, labels=False, top_k=8, temperature=2.0),
        # distillation of a text model, 8 sequences of 512 tokens
        _case("distill_text", "distill", "train", 4096, 768, 50265, labels=False, top_k=32, temperature=2.0),
        # the same with labels on half of the positions
        _case("distill_labels", "distill", "train", 8192, 1024, 32000, share=0.5, top_k=64, temperature=4.0),
        # nothing round: a prime vocabulary, an odd number of rows, some of them without teacher
        _case("distill_ragged", "distill", "train", 777, 1280, 10007, share=0.6, labels=False, top_k=5),
        # a small float32 student
        _case("distill_fp32", "distill", "train", 333, 200, 5003, mode="fp32", share=0.7, top_k=3, temperature=1.5),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("xent", "distill"))
    pass_ = rng.choice(("forward", "train", "train"))
    mode = rng.choice(("bf16", "bf16", "bf16", "fp32"))
    while True:
        rows, d, vocab = _spread(rng, 1, 16384), 8 * _spread(rng, 8, 256), _spread(rng, 100, 131072)
        if 2e6 <= rows * d * vocab <= (6e11 if mode == "bf16" else 3e10):
            break
    labels = op == "xent" or rng.random() < 0.5
    return {k: v for k, v in _case("", op, pass_, rows, d, vocab, mode, rng.random() < 0.5, rng.choice((1.0, 1.0, 0.5, 0.15)), labels,
                                   0 if op == "xent" else rng.randint(1, 64), 1.0 if op == "xent" else rng.choice((1.0, 2.0, 4.0))).items()
            if k != "name"}


def _some(case):
    """How many rows carry a label, or, where there are no labels, a teacher's logits."""
    return max(1, round(case["rows"] * case["share"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, D, V, K = case["rows"], case["d_model"], case["vocab"], case["top_k"]
    dtype = torch.bfloat16 if case["mode"] == "bf16" else torch.float32
    params = torch.randn(V * D + (V if case["bias"] else 0), generator=g, device="cuda")
    params[:V * D] *= 2.5 / math.sqrt(D)
    params = params.to(dtype)
    W = params[:V * D].view(V, D)
    label = torch.randint(0, V, (M,), generator=g, device="cuda")
    X = (torch.randn(M, D, generator=g, device="cuda") + 1.3 * W[label].float()).to(dtype)
    keep = torch.randperm(M, generator=g, device="cuda")[:_some(case)]
    st = dict(case=case, params=params, X=X, labels=None)
    if case["labels"]:
        st["labels"] = torch.full((M,), -100, dtype=torch.int32, device="cuda")
        st["labels"][keep] = label[keep].to(torch.int32)
    # the cotangents of a mean over the rows, as a loss scaled for a sum over several steps has them: of order one
    st["dloss"] = torch.rand(M, generator=g, device="cuda") + 0.5
    if K:
        top, idx = [], []
        for r in range(0, M, 2048):     # a teacher that agrees with the student in part
            z = (X[r:r + 2048] @ W.T).float()
            v, i = (z + 1.5 * torch.randn(z.shape, generator=g, device="cuda")).topk(min(K, V), dim=1)
            top.append(v)
            idx.append(i.to(torch.int32))
        st["teacher_logits"], st["teacher_idx"] = torch.cat(top), torch.cat(idx)
        if not case["labels"]:          # rows without a teacher hold no valid entry
            gone = torch.ones(M, dtype=torch.bool, device="cuda")
            gone[keep] = False
            st["teacher_idx"][gone] = -1
        st["dloss_ce"] = 0.5 * torch.rand(M, generator=g, device="cuda") if case["labels"] else None
    return st


def _own(st):
    from paper_2306_09342_amd import binding as B
    c, labels = st["case"], st["labels"]
    cfg = B.make_vocab_cfg(c["rows"], c["d_model"], c["vocab"], c["mode"], grad_mode=c["mode"], bias=c["bias"], top_k=c["top_k"],
                           temperature=c["temperature"])
    if c["op"] == "xent":
        out = B.rev_xent_forward(cfg, st["params"], st["X"], labels)
        if c["pass_"] == "train":
            out.update(B.rev_xent_backward(cfg, st["params"], st["X"], labels, out["lse"], st["dloss"]))
    else:
        out = B.rev_distill_forward(cfg, st["params"], st["X"], st["teacher_idx"], st["teacher_logits"], labels=labels)
        if c["pass_"] == "train":
            out.update(B.rev_distill_backward(cfg, st["params"], st["X"], st["teacher_idx"], st["teacher_logits"], out["lse"], st["dloss"],
                                              labels=labels, dloss_ce=st["dloss_ce"]))
    return out


def run(st):
    if own:
        return _own(st)
    c = st["case"]
    M, D, V, T = c["rows"], c["d_model"], c["vocab"], c["temperature"]
    W = st["params"][:V * D].view(V, D).float()
    X = st["X"].float()
    z = X @ W.T
    if c["bias"]:
        z += st["params"][V * D:].float()
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    lse = m[:, 0] + torch.log(e.sum(1))
    has, y = None, None
    if st["labels"] is not None:
        y = st["labels"].long()
        has = (y >= 0) & (y < V)
        y = torch.where(has, y, torch.zeros_like(y))
        ce = torch.where(has, lse - z.gather(1, y[:, None])[:, 0], torch.zeros_like(lse))
    if c["op"] == "xent":
        out = {"loss": ce, "lse": torch.where(has, lse, torch.zeros_like(lse))}
        if c["pass_"] == "forward":
            return out
        g = torch.where(has, st["dloss"], torch.zeros_like(lse))
        dz = e.mul_((g * torch.exp(m[:, 0] - lse))[:, None])
        dz.scatter_add_(1, y[:, None], -g[:, None])
    else:
        i = st["teacher_idx"].long()
        valid = (i >= 0) & (i < V)
        i = torch.where(valid, i, torch.zeros_like(i))
        taught = valid.any(1)
        t = torch.where(valid, st["teacher_logits"] / T, torch.full_like(st["teacher_logits"], -math.inf))
        tm = t.amax(1, keepdim=True)
        tm = torch.where(taught[:, None], tm, torch.zeros_like(tm))
        p = torch.exp(t - tm)
        total = p.sum(1, keepdim=True)
        total = torch.where(taught[:, None], total, torch.ones_like(total))
        p = p / total
        log_p = t - tm - torch.log(total)
        eT = torch.exp((z - m) / T)
        lse_T = m[:, 0] / T + torch.log(eT.sum(1))
        each = torch.where(p > 0, p * (log_p - (z.gather(1, i) / T - lse_T[:, None])), torch.zeros_like(p))
        zero = torch.zeros_like(lse)
        out = {"loss": T * T * each.sum(1), "lse": torch.stack([torch.where(has, lse, zero) if has is not None else zero, torch.where(taught, lse_T, zero)])}
        if has is not None:
            out["loss_ce"] = ce
        if c["pass_"] == "forward":
            return out
        g = torch.where(taught, st["dloss"] * T, zero)
        dz = eT.mul_((g * torch.exp(m[:, 0] / T - lse_T))[:, None])
        dz.scatter_add_(1, i, -g[:, None] * p)
        if has is not None:
            g = torch.where(has, st["dloss_ce"], zero)
            dz += e.mul_((g * torch.exp(m[:, 0] - lse))[:, None])
            dz.scatter_add_(1, y[:, None], -g[:, None])
    out["dX"] = (dz @ W).to(st["X"].dtype)
    out["dparams"] = torch.cat([(dz.T @ X).flatten()] + ([dz.sum(0)] if c["bias"] else [])).to(st["params"].dtype)
    return out


def work(case):
    M, D, V, K = case["rows"], case["d_model"], case["vocab"], case["top_k"]
    A = M if K and case["labels"] else _some(case)          # rows that count
    e = 2 if case["mode"] == "bf16" else 4
    params = V * D + (V if case["bias"] else 0)
    losses = 1 if case["op"] == "xent" else 4 if case["labels"] else 3
    read = e * (A * D + params) + (4 * M if case["labels"] else 0) + 8 * M * K
    train = case["pass_"] == "train"
    moved = read + 4 * M * (1 + losses) + (e * (M * D + params) + 4 * M if train else 0)
    return {"bytes": moved, "flops": (6.0 if train else 2.0) * A * D * V}


def exact(case, seed):
    """The losses by their definitions in 64 bits, the gradients by reverse-mode differentiation of their sum, some rows at a time."""
    st = prepare(case, seed)
    M, D, V, T = case["rows"], case["d_model"], case["vocab"], case["temperature"]
    train, K = case["pass_"] == "train", case["top_k"]
    f8 = torch.float64
    params = st["params"].to(f8).requires_grad_(train)
    X = st["X"].to(f8).requires_grad_(train)
    loss, loss_ce = torch.zeros(M, dtype=f8, device="cuda"), torch.zeros(M, dtype=f8, device="cuda")
    lse, lse_T = torch.zeros(M, dtype=f8, device="cuda"), torch.zeros(M, dtype=f8, device="cuda")
    step = max(1, min(M, 150_000_000 // V))
    for r in range(0, M, step):
        s = slice(r, min(M, r + step))
        with torch.set_grad_enabled(train):
            z = torch.nn.functional.linear(X[s], params[:V * D].view(V, D), params[V * D:] if case["bias"] else None)
            total = torch.zeros((), dtype=f8, device="cuda")
            if st["labels"] is not None:
                y = st["labels"][s].long()
                rows = ((y >= 0) & (y < V)).nonzero()[:, 0]
                logp = torch.log_softmax(z[rows], 1)
                each = -logp[torch.arange(len(rows), device="cuda"), y[rows]]
                total = total + (each * (st["dloss_ce"] if K else st["dloss"])[s][rows].to(f8)).sum()
                (loss_ce if K else loss)[r + rows] = each.detach()
                lse[r + rows] = torch.logsumexp(z[rows].detach(), 1)
            if K:
                idx = st["teacher_idx"][s].long()
                rows = (idx >= 0).any(1).nonzero()[:, 0]
                p = torch.softmax(st["teacher_logits"][s][rows].to(f8) / T, 1)
                logq = torch.log_softmax(z[rows] / T, 1).gather(1, idx[rows])
                each = T * T * (p * (torch.log(p) - logq)).sum(1)
                total = total + (each * st["dloss"][s][rows].to(f8)).sum()
                loss[r + rows] = each.detach()
                lse_T[r + rows] = torch.logsumexp(z[rows].detach() / T, 1)
        if train and total.requires_grad:
            total.backward()
        del z, total
    out = {"loss": loss, "lse": torch.stack([lse, lse_T]) if K else lse}
    if K and case["labels"]:
        out["loss_ce"] = loss_ce
    if train:
        out["dX"], out["dparams"] = X.grad, params.grad
    return out
