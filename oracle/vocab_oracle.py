"""float64 oracle of the losses over a vocabulary: softmax cross entropy, distillation from a teacher's top logits, gradients.

One row at a time from the definitions (include/rev_stack.h); the whole row of logits is kept.  Test infrastructure only.
"""
import numpy as np


def unpack(params, vocab, d_model, bias):
    p = np.asarray(params, dtype=np.float64)
    W = p[:vocab * d_model].reshape(vocab, d_model)
    return W, (p[vocab * d_model:] if bias else np.zeros(vocab))


def logsumexp(z):
    m = z.max()
    return m + np.log(np.exp(z - m).sum())


def teacher(idx, logits, vocab, tau):
    """(indices, probabilities) of the entries of one row that count."""
    keep = (idx >= 0) & (idx < vocab) & ~(logits == -np.inf)
    if not keep.any():
        return idx[keep], np.zeros(0)
    t = logits[keep].astype(np.float64) / tau
    return idx[keep], np.exp(t - logsumexp(t))


def vocab_loss(params, X, vocab, bias, labels=None, teacher_idx=None, teacher_logits=None, tau=1.0, dce=None, dkd=None):
    """Returns loss_ce, loss_kd, lse, lse_tau [rows], dX and dparams (for the cotangents dce and dkd; zeros where they are not given)."""
    X = np.asarray(X)
    M, D = X.shape
    W, b = unpack(params, vocab, D, bias)
    out = {k: np.zeros(M) for k in ("loss_ce", "loss_kd", "lse", "lse_tau")}
    dX, dW, db = np.zeros((M, D)), np.zeros((vocab, D)), np.zeros(vocab)
    for r in range(M):
        y = -1 if labels is None else int(labels[r])
        has = 0 <= y < vocab
        i, p = teacher(teacher_idx[r], teacher_logits[r], vocab, tau) if teacher_idx is not None else (np.zeros(0, int), np.zeros(0))
        if not has and len(i) == 0:
            continue
        x = X[r].astype(np.float64)
        z = W @ x + b
        dz = np.zeros(vocab)
        if has:
            out["lse"][r] = logsumexp(z)
            out["loss_ce"][r] = out["lse"][r] - z[y]
            if dce is not None:
                one = np.zeros(vocab)
                one[y] = 1.0
                dz += float(dce[r]) * (np.exp(z - out["lse"][r]) - one)
        if len(i):
            lt = out["lse_tau"][r] = logsumexp(z / tau)
            on = p > 0
            out["loss_kd"][r] = tau * tau * np.sum(p[on] * (np.log(p[on]) - (z[i[on]] / tau - lt)))
            if dkd is not None:
                target = np.zeros(vocab)
                np.add.at(target, i, p)
                dz += float(dkd[r]) * tau * (np.exp(z / tau - lt) - target)
        dX[r] = dz @ W
        dW += np.outer(dz, x)
        db += dz
    out["dX"] = dX
    out["dparams"] = np.concatenate([dW.ravel(), db]) if bias else dW.ravel()
    return out
