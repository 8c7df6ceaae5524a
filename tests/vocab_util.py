"""Inputs of the losses over a vocabulary, their results in float64 and how far off a kernel's may be (test infrastructure)."""
import numpy as np
import torch

from oracle import vocab_oracle as VO
from paper_2306_09342_amd import binding as B

U = 2.0 ** -24                 # half a step of float32, relative
HALF = {"fp32": U, "bf16": 2.0 ** -8}


def make(M, D, V, mode="bf16", bias=True, K=0, share=1.0, labels=True, tau=1.0, seed=0, scale=2.0):
    """Numpy inputs on the grid of the mode's type."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if mode == "bf16" else torch.float32
    params = torch.randn(V * D + (V if bias else 0), generator=g)
    params[:V * D] *= scale / D ** 0.5
    c = dict(M=M, D=D, V=V, mode=mode, bias=bias, K=K, tau=tau)
    c["params"] = params.to(dt).float().numpy()
    c["X"] = torch.randn(M, D, generator=g).to(dt).float().numpy()
    y = torch.randint(0, V, (M,), generator=g, dtype=torch.int32)
    y[torch.rand(M, generator=g) >= share] = -100
    c["labels"] = y.numpy() if labels else None
    c["idx"] = c["logits"] = None
    if K:
        idx = torch.randint(0, V, (M, K), generator=g, dtype=torch.int32)
        idx[torch.rand(M, generator=g) >= share] = -1
        c["idx"], c["logits"] = idx.numpy(), (3 * torch.randn(M, K, generator=g)).numpy()
    c["dce"] = (torch.rand(M, generator=g) - 0.3).numpy()
    c["dkd"] = (torch.rand(M, generator=g) - 0.3).numpy()
    return c


def reference(c):
    return VO.vocab_loss(c["params"], c["X"], c["V"], c["bias"], c["labels"], c["idx"], c["logits"], c["tau"],
                         c["dce"] if c["labels"] is not None else None, c["dkd"] if c["K"] else None)


def bounds(c, grad_mode):
    """Elementwise bounds of the absolute errors, from the sums and roundings that the header allows: logits, statistics and sums in float32
    (a sum of n products is off by at most n U times the sum of their magnitudes, whatever its order), dz rounded once to the mode's type, results
    rounded once.  exp of x: 4 U + 2 U |x| relative (the argument's own rounding).  Rows that do not count: exactly 0."""
    M, D, V, tau = c["M"], c["D"], c["V"], c["tau"]
    W, b = VO.unpack(c["params"], V, D, c["bias"])
    X = c["X"].astype(np.float64)
    on = np.zeros(M, bool)
    has = np.zeros(M, bool) if c["labels"] is None else (c["labels"] >= 0) & (c["labels"] < V)
    tea = [VO.teacher(c["idx"][r], c["logits"][r], V, tau) if c["K"] else (np.zeros(0, int), np.zeros(0)) for r in range(M)]
    taught = np.array([len(i) > 0 for i, _ in tea])
    on = has | taught
    Xs = np.where(on[:, None], X, 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        z = Xs @ W.T + b
        Ez = (D + 8) * U * (np.abs(Xs) @ np.abs(W).T + np.where(np.isfinite(b), np.abs(b), 0.0))
        Ez = np.where(np.isfinite(b) & (np.abs(z) < 1e30), Ez, 0.0)          # entries taken out of the vocabulary
    dz, Edz = np.zeros((M, V)), np.zeros((M, V))
    out = {k: np.zeros(M) for k in ("loss_ce", "loss_kd", "lse", "lse_tau")}
    for r in np.nonzero(on)[0]:
        live = z[r] > -1e30
        top = np.abs(z[r][live]).max()
        for name, lname, active, t in (("loss_ce", "lse", has[r], 1.0), ("loss_kd", "lse_tau", taught[r], tau)):
            if not active:
                continue
            lse = VO.logsumexp(z[r][live] / t)
            El = Ez[r].max() / t + (V / 8 + 64 + 4 * np.log(V) + 8 * top / t + 4 * abs(lse)) * U
            out[lname][r] = El
            p = np.where(live, np.exp(np.where(live, z[r] / t, 0) - lse), 0.0)
            rel = Ez[r] / t + El + (4 * top / t + 4 * abs(lse) + 16) * U
            if t == 1.0 and name == "loss_ce":
                y = c["labels"][r]
                out[name][r] = El + Ez[r][y] + 4 * U * (abs(z[r][y]) + abs(lse)) if live[y] else 0.0
                f = float(c["dce"][r])
                dz[r] += f * p
                dz[r][y] -= f
                Edz[r] += abs(f) * p * rel
                Edz[r][y] += 4 * U * abs(f)
            else:
                i, q = tea[r]
                keep = (c["idx"][r] >= 0) & (c["idx"][r] < V) & ~(c["logits"][r] == -np.inf)
                big = np.abs(c["logits"][r][keep][q > 0]).max().astype(np.float64) / t      # entries that underflow take no part
                relq = (8 * big + c["K"] + 16) * U
                lq = np.where(q > 0, np.abs(np.log(np.where(q > 0, q, 1))), 0)
                out[name][r] = t * t * np.sum(q * (El + Ez[r][i] / t + (8 * big + 4 * top / t + 4 * abs(lse) + 8 * lq + c["K"] + 32) * U + relq * (lq + np.abs(z[r][i] / t - lse))))
                f = float(c["dkd"][r]) * t
                dz[r] += f * p
                np.add.at(dz[r], i, -f * q)
                Edz[r] += abs(f) * p * rel
                np.add.at(Edz[r], i, abs(f) * q * (relq + 4 * U))
        Edz[r] += 4 * U * np.abs(dz[r])
    half = HALF[c["mode"]]
    Edz = Edz + half * (np.abs(dz) + Edz)
    Wf = np.where(np.isfinite(W), W, 0.0)
    def rounded(v, e, kind):
        return e + HALF[kind] * (np.abs(v) + e)
    dX, EdX = dz @ Wf, Edz @ np.abs(Wf) + (V + 64) * U * (np.abs(dz) + Edz) @ np.abs(Wf)
    n = int(on.sum()) + 64
    dW, EdW = dz.T @ Xs, Edz.T @ np.abs(Xs) + n * U * (np.abs(dz) + Edz).T @ np.abs(Xs)
    db, Edb = dz.sum(0), Edz.sum(0) + n * U * (np.abs(dz) + Edz).sum(0)
    out["dX"] = rounded(dX, EdX, c["mode"])
    flat, e = (np.concatenate([dW.ravel(), db]), np.concatenate([EdW.ravel(), Edb])) if c["bias"] else (dW.ravel(), EdW.ravel())
    out["dparams"] = rounded(flat, e, grad_mode)
    return out


def divergence_terms(c):
    """tau^2 sum_k p_k (|log p_k| + |log q_k|) of every row."""
    W, b = VO.unpack(c["params"], c["V"], c["D"], c["bias"])
    out = np.zeros(c["M"])
    for r in range(c["M"]):
        i, p = VO.teacher(c["idx"][r], c["logits"][r], c["V"], c["tau"])
        if len(i):
            z = (W @ c["X"][r].astype(np.float64) + b) / c["tau"]
            on = p > 0
            out[r] = c["tau"] ** 2 * np.sum(p[on] * (np.abs(np.log(p[on])) + np.abs(z[i[on]] - VO.logsumexp(z))))
    return out


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def gpu_args(c):
    dt = torch.bfloat16 if c["mode"] == "bf16" else torch.float32
    a = dict(params=dev(c["params"], dt), X=dev(c["X"], dt))
    for n in ("labels", "idx", "logits", "dce", "dkd"):
        a[n] = None if c[n] is None else dev(c[n])
    return a


def make_cfg(c, grad_mode="fp32"):
    return B.make_vocab_cfg(c["M"], c["D"], c["V"], c["mode"], grad_mode=grad_mode, bias=c["bias"], top_k=c["K"], temperature=c["tau"])


def forward(cfg, c, a, **more):
    """The forward call that the case means, under the oracle's names."""
    if c["K"] == 0:
        o = B.rev_xent_forward(cfg, a["params"], a["X"], a["labels"], **more)
        return {"loss_ce": o["loss"], "lse": o["lse"], "stats": o["lse"]}
    o = B.rev_distill_forward(cfg, a["params"], a["X"], a["idx"], a["logits"], labels=a["labels"], **more)
    r = {"loss_kd": o["loss"], "lse": o["lse"][0], "lse_tau": o["lse"][1], "stats": o["lse"]}
    if a["labels"] is not None:
        r["loss_ce"] = o["loss_ce"]
    return r


def backward(cfg, c, a, stats, **more):
    if c["K"] == 0:
        return B.rev_xent_backward(cfg, a["params"], a["X"], a["labels"], stats, a["dce"], **more)
    return B.rev_distill_backward(cfg, a["params"], a["X"], a["idx"], a["logits"], stats, a["dkd"], labels=a["labels"],
                                  dloss_ce=a["dce"] if a["labels"] is not None else None, **more)


def run(c, grad_mode="fp32", **more):
    cfg, a = make_cfg(c, grad_mode), gpu_args(c)
    out = forward(cfg, c, a, **more)
    out.update(backward(cfg, c, a, out["stats"], **more))
    torch.cuda.synchronize()
    return out


def check(c, grad_mode="fp32", got=None):
    got = run(c, grad_mode) if got is None else got
    ref, lim = reference(c), bounds(c, grad_mode)
    for k, v in got.items():
        if k == "stats":
            continue
        g, r = v.float().cpu().numpy().astype(np.float64), ref[k]
        assert g.shape == r.shape, k
        assert np.isfinite(g[np.isfinite(r)]).all(), k
        assert (g[~np.isfinite(r)] == r[~np.isfinite(r)]).all(), k
        fin = np.isfinite(r)
        e = np.abs(g - np.where(fin, r, 0))[fin]
        worst = np.max(e / np.maximum(lim[k][fin], 1e-300), initial=0.0)
        assert worst <= 1.0 or (e[e > lim[k][fin]] < 1e-35).all(), f"{k}: {worst:.3g} times what rounding allows"
        norm = np.linalg.norm(r[fin])
        if norm > 0:
            # by norm the roundings at both ends of a product add to a few of their half steps; float32 sums to far less than 2e-5
            # (a divergence is a sum of p log p and -p log q, which may cancel: its float32 errors go with the size of these terms)
            if k == "loss_kd":
                norm = np.linalg.norm(divergence_terms(c))
            tol = 4 * HALF["bf16"] if "bf16" in (c["mode"], grad_mode) and k in ("dX", "dparams") else 2e-5
            assert np.linalg.norm(e) <= tol * norm, f"{k}: relative error {np.linalg.norm(e) / norm:.3g}"
    return got, ref
