"""Plain float64 definition of the fine-tuning step's head and of the norm in front of it (numpy, CPU).

    Z = X W / temperature                 logits of every token over the vocabulary
    y                                     target distribution of a token: 1 at its label, or the softmax of the teacher's logits
                                          / temperature over the ids given (ids given twice add up)
    loss = sum_v y_v (log y_v - log softmax(Z)_v)
    dZ = g (softmax(Z) - y) / temperature, dX = dZ W^T, dW = X^T dZ

Tokens without a target (a label below zero; a teacher's list without an id or with all logits -inf) have loss 0 and dZ 0.
``tied``: W is [vocab, d_model].  A whole [tokens, vocab] matrix is formed at every step.
"""
import numpy as np

from .layer import norm_fwd


def norm_bwd(dY, X, gamma, eps, kind):
    """dX, dgamma, dbeta of Y = norm(X): the norm's Jacobian row by row in textbook form."""
    Y, xhat, rstd, mu = norm_fwd(X, gamma, None, eps, kind)
    d = X.shape[-1]
    x2, g2, r2 = xhat.reshape(-1, d), (dY * gamma).reshape(-1, d), rstd.reshape(-1)
    dX = np.zeros_like(x2)
    for i in range(x2.shape[0]):
        jac = np.eye(d) - np.outer(x2[i], x2[i]) / d
        if kind == "layernorm":
            jac = jac - 1.0 / d
        dX[i] = r2[i] * (jac @ g2[i])
    flat = dY.reshape(-1, d)
    return dX.reshape(X.shape), (flat * x2).sum(0), flat.sum(0) if kind == "layernorm" else None


def targets(cfg, inp):
    """[tokens, vocab] target distribution and [tokens] whether a token has one."""
    n = cfg.batch * cfg.seq
    y, has = np.zeros((n, cfg.vocab)), np.zeros(n, dtype=bool)
    if not cfg.top_k:
        for i, t in enumerate(np.asarray(inp["targets"]).reshape(-1)):
            if t >= 0:
                y[i, t], has[i] = 1.0, True
        return y, has
    ids = np.asarray(inp["top_ids"]).reshape(n, cfg.top_k)
    logits = np.asarray(inp["top_logits"], dtype=np.float64).reshape(n, cfg.top_k) / cfg.temperature
    for i in range(n):
        there = [(v, z) for v, z in zip(ids[i], logits[i]) if v >= 0]
        top = max((z for _, z in there), default=-np.inf)
        if top == -np.inf:
            continue
        has[i] = True
        mass = sum(np.exp(z - top) for _, z in there)
        for v, z in there:
            y[i, v] += np.exp(z - top) / mass
    return y, has


def head_fwd_bwd(cfg, inp):
    """Returns a dict: loss [batch, seq], total (sum, count), lse, dZ, dX, dW.  ``inp["dloss"]`` [batch, seq]: the gradient of each
    token's loss, None: of the mean over tokens with a target."""
    n = cfg.batch * cfg.seq
    x = inp["X"].reshape(n, -1)
    w = inp["W"].T if cfg.tied else inp["W"]
    y, has = targets(cfg, inp)
    z = x @ w / cfg.temperature
    top = z.max(1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
    logp = z - lse[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        loss = np.where(y > 0, y * (np.log(y) - logp), 0.0).sum(1)
    loss = np.where(has, loss, 0.0)
    count = float(has.sum())
    g = np.full(n, 1.0 / max(count, 1.0)) if inp.get("dloss") is None else np.asarray(inp["dloss"], dtype=np.float64).reshape(-1)
    dz = np.where(has[:, None], g[:, None] * (np.exp(logp) - y) / cfg.temperature, 0.0)
    dw = x.T @ dz
    return {"loss": loss.reshape(cfg.batch, cfg.seq), "total": np.array([loss.sum(), count]), "lse": lse, "Z": z, "dZ": dz,
            "dX": (dz @ w.T).reshape(inp["X"].shape), "dW": dw.T if cfg.tied else dw, "has": has.reshape(cfg.batch, cfg.seq)}
