"""Inputs, float64 results and bounds of the losses over a vocabulary for sizes that a row at a time on the host would take minutes for: the
same as vocab_util, on the GPU and over all rows at once (test infrastructure)."""
import numpy as np
import torch

import vocab_util as VU

U = VU.U


def make(M, D, V, mode="bf16", bias=True, K=0, share=0.8, labels=True, tau=1.0, seed=0, scale=2.0):
    """(case, GPU tensors), as vocab_util.make and gpu_args give them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if mode == "bf16" else torch.float32
    params = torch.randn(V * D + (V if bias else 0), generator=g, device="cuda")
    params[:V * D] *= scale / D ** 0.5
    a = dict(params=params.to(dt), X=torch.randn(M, D, generator=g, device="cuda").to(dt), labels=None, idx=None, logits=None)
    if labels:
        a["labels"] = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
        a["labels"][torch.rand(M, generator=g, device="cuda") >= share] = -100
    if K:
        a["idx"] = torch.randint(0, V, (M, K), generator=g, device="cuda", dtype=torch.int32)
        a["idx"][torch.rand(M, generator=g, device="cuda") >= share] = -1
        a["logits"] = 3 * torch.randn(M, K, generator=g, device="cuda")
    for n in ("dce", "dkd"):
        a[n] = torch.rand(M, generator=g, device="cuda") - 0.3
    return dict(M=M, D=D, V=V, mode=mode, bias=bias, K=K, tau=tau), a


def reference(c, a, grad_mode):
    """{name: (result, bound of the absolute error)}; the bounds are those of vocab_util.bounds."""
    M, D, V, K, tau = (c[k] for k in ("M", "D", "V", "K", "tau"))
    W = a["params"][:V * D].view(V, D).double()
    b = a["params"][V * D:].double() if c["bias"] else torch.zeros(V, dtype=torch.float64, device="cuda")
    has = torch.zeros(M, dtype=torch.bool, device="cuda") if a["labels"] is None else (a["labels"] >= 0) & (a["labels"] < V)
    taught = (a["idx"] >= 0).any(1) if K else torch.zeros_like(has)
    on = has | taught
    X = torch.where(on[:, None], a["X"].double(), 0.0)
    z = X @ W.T + b
    Ez = (D + 8) * U * (X.abs() @ W.abs().T + b.abs())
    top = z.abs().amax(1)
    dz, Edz, out = torch.zeros_like(z), torch.zeros_like(z), {}
    for name, lname, active, t in (("loss_ce", "lse", has, 1.0), ("loss_kd", "lse_tau", taught, tau)):
        zero = torch.zeros(M, dtype=torch.float64, device="cuda")
        if (a["labels"] if name == "loss_ce" else a["idx"]) is None:
            out[lname] = zero, zero
            continue
        lse = torch.logsumexp(z / t, 1)
        El = Ez.amax(1) / t + (V / 8 + 64 + 4 * np.log(V) + 8 * top / t + 4 * lse.abs()) * U
        out[lname] = torch.where(active, lse, zero), torch.where(active, El, zero)
        p = torch.exp(z / t - lse[:, None])
        rel = Ez / t + (El + (4 * top / t + 4 * lse.abs() + 16) * U)[:, None]
        if name == "loss_ce":
            y = a["labels"].long().clamp(min=0)[:, None]
            zy = z.gather(1, y)[:, 0]
            f = torch.where(has, a["dce"].double(), zero)
            loss, E = lse - zy, El + Ez.gather(1, y)[:, 0] + 4 * U * (zy.abs() + lse.abs())
            dz.scatter_add_(1, y, -f[:, None])
            Edz.scatter_add_(1, y, 4 * U * f.abs()[:, None])
        else:
            keep = a["idx"] >= 0
            i = a["idx"].long().clamp(min=0)
            logits = a["logits"].double() / t
            q = torch.softmax(torch.where(keep, logits, -np.inf), 1).nan_to_num(0.0)
            big = torch.where(keep, logits.abs(), 0.0).amax(1)[:, None]
            relq = (8 * big + K + 16) * U
            lq = torch.where(q > 0, torch.log(torch.where(q > 0, q, 1.0)), 0.0)
            zi = z.gather(1, i)
            f = torch.where(taught, a["dkd"].double() * t, zero)
            loss = t * t * (q * (lq - (zi / t - lse[:, None]))).sum(1)
            E = t * t * (q * (El[:, None] + Ez.gather(1, i) / t + (8 * big + (4 * top / t + 4 * lse.abs())[:, None] + 8 * lq.abs() + K + 32) * U + relq * (
                lq.abs() + (zi / t - lse[:, None]).abs()))).sum(1)
            dz.scatter_add_(1, i, -f[:, None] * q)
            Edz.scatter_add_(1, i, f.abs()[:, None] * q * (relq + 4 * U))
            out["terms"] = t * t * (q * (lq.abs() + (zi / t - lse[:, None]).abs())).sum(1)
        out[name] = torch.where(active, loss, zero), torch.where(active, E, zero)
        dz += f[:, None] * p
        Edz += f.abs()[:, None] * p * rel
    Edz += 4 * U * dz.abs()
    Edz += VU.HALF[c["mode"]] * (dz.abs() + Edz)
    size, n = dz.abs() + Edz, int(on.sum()) + 64

    def rounded(v, e, kind):
        return v, e + VU.HALF[kind] * (v.abs() + e)

    out["dX"] = rounded(dz @ W, Edz @ W.abs() + (V + 64) * U * (size @ W.abs()), c["mode"])
    v, e = (dz.T @ X).flatten(), (Edz.T @ X.abs() + n * U * (size.T @ X.abs())).flatten()
    if c["bias"]:
        v, e = torch.cat([v, dz.sum(0)]), torch.cat([e, Edz.sum(0) + n * U * size.sum(0)])
    out["dparams"] = rounded(v, e, grad_mode)
    return out


def run(c, a, grad_mode="fp32", **more):
    cfg = VU.make_cfg(c, grad_mode)
    got = VU.forward(cfg, c, a)
    got.update(VU.backward(cfg, c, a, got["stats"], **more))
    return got


def check(c, a, got, ref, grad_mode="fp32"):
    """As vocab_util.check."""
    terms = ref.get("terms")
    for k, v in got.items():
        if k == "stats":
            continue
        want, lim = ref[k]
        e = (v.double() - want).abs()
        assert bool(torch.isfinite(e).all()), k
        assert bool(((e <= lim) | (e < 1e-35)).all()), f"{k}: {float((e / lim.clamp(min=1e-300)).max()):.3g} times what rounding allows"
        norm = float(torch.linalg.norm(terms if k == "loss_kd" else want))
        tol = 4 * VU.HALF["bf16"] if "bf16" in (c["mode"], grad_mode) and k in ("dX", "dparams") else 2e-5
        assert norm == 0 or float(torch.linalg.norm(e)) <= tol * norm, f"{k}: relative error {float(torch.linalg.norm(e)) / norm:.3g}"
