"""The head of a fine-tuning step, operator by operator: the final norm, the softmax cross entropy over the
vocabulary and the distillation from a teacher's top logits, each as the forward alone or with its gradients.

Matrices are in the framework's tiled layout on both sides.  With 128-byte tile rows it is, as a torch tensor,
``[column panels, padded rows, elements of a 128-byte row]``: a token matrix ``[batch, seq, d_model]`` has its
sequences padded to eight rows each, and padding holds zeros in inputs and outputs alike.  Vectors, losses and per-token
weights are plain fp32 arrays, token ids int32.

``run`` computes the plain form, or with ``own`` set makes the calls that a user makes of the framework.
"""
from __future__ import annotations

import math

import torch

own = False

# Inputs of a drawn case cost no more flops than this; the largest listed cases take 6.4e12.
DRAW_FLOPS, DRAW_FLOPS_FP32 = 4.0e12, 4.0e11


def _norm(name, batch, seq, d_model, dtype, norm, mode="step"):
    return {"name": name, "op": "norm", "mode": mode, "batch": batch, "seq": seq, "d_model": d_model, "dtype": dtype, "norm": norm}


def _loss(name, batch, seq, d_model, vocab, dtype, tied, mode="step", frozen=False, weighted=False, ignored=0.0, top_k=0,
          temperature=1.0):
    return {"name": name, "op": "distill" if top_k else "xent", "mode": mode, "batch": batch, "seq": seq, "d_model": d_model,
            "vocab": vocab, "dtype": dtype, "tied": tied, "frozen": frozen, "weighted": weighted, "ignored": ignored,
            "top_k": top_k, "temperature": temperature}


def listed():
    return [
        # the final norm of one new token of a small decoder: a launch's latency
        _norm("norm one token forward", 1, 1, 768, "bf16", "layernorm", mode="forward"),
        # the same decoder's final norm in a training step of four sequences
        _norm("norm small decoder step", 4, 512, 768, "bf16", "layernorm"),
        # full-precision training on sequences of odd length
        _norm("norm ragged fp32 step", 5, 333, 1280, "fp32", "layernorm"),
        # one long sequence of a wide decoder, norm without a mean
        _norm("norm long wide step", 1, 8192, 4096, "bf16", "rmsnorm"),
        # scoring one token under a large vocabulary that shares the embedding's weights: the weights are read once
        _loss("loss one token forward", 1, 1, 2048, 128256, "bf16", True, mode="forward"),
        # a short prompt's step: fewer tokens than a compute tile, a vocabulary of odd size
        _loss("loss short prompt step", 1, 50, 768, 50257, "bf16", True),
        # a small decoder's step on four sequences whose prompts (a third) carry no loss
        _loss("loss small decoder step", 4, 512, 768, 50257, "bf16", True, ignored=0.33),
        # adapter fine-tuning: the head is frozen, only the hidden states receive a gradient
        _loss("loss frozen head step", 2, 2048, 2048, 128256, "bf16", False, frozen=True, ignored=0.2),
        # full-precision training with per-token weights, sequences and vocabulary of odd size
        _loss("loss ragged fp32 step", 4, 197, 768, 30011, "fp32", False, weighted=True, ignored=0.1),
        # the largest: one long sequence of a wide decoder, a head of its own
        _loss("loss long wide step", 1, 8192, 4096, 32000, "bf16", False),
        # full-precision distillation of a small model from eight teacher logits a token
        _loss("distill small fp32 step", 3, 77, 512, 32000, "fp32", True, top_k=8, ignored=0.1),
        # distillation from a teacher's 64 top logits a token over a large vocabulary
        _loss("distill large vocabulary step", 2, 2048, 2048, 128256, "bf16", True, top_k=64, temperature=2.0, ignored=0.2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choices(["norm", "xent", "distill"], [3, 5, 4])[0]
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        mode = "forward" if rng.random() < 0.25 else "step"
        batch, seq = _log_int(rng, 1, 16), _log_int(rng, 1, 8192)
        d_model = 64 * _log_int(rng, 1, 64)
        if batch * seq > 16384:
            continue
        if op == "norm":
            case = _norm("", batch, seq, d_model, dtype, rng.choice(["layernorm", "rmsnorm"]), mode)
        else:
            vocab = _log_int(rng, 300, 131072)
            top_k = rng.choice([1, 5, 8, 20, 64, 100, 128]) if op == "distill" else 0
            case = _loss("", batch, seq, d_model, vocab, dtype, rng.random() < 0.5, mode, rng.random() < 0.3, rng.random() < 0.4,
                         rng.choice([0.0, 0.1, 0.5]), top_k, rng.choice([1.0, 1.0, 2.0, 4.0]) if top_k else 1.0)
            if work(case)["flops"] > (DRAW_FLOPS_FP32 if dtype == "fp32" else DRAW_FLOPS) or batch * seq * vocab > 6e8:
                continue
        del case["name"]
        return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _aligned(shape, dtype, fill=None):
    """An uninitialised tensor whose data starts at a multiple of 1024 bytes."""
    n = math.prod(shape) * torch.empty(0, dtype=dtype).element_size()
    raw = torch.empty(n + 1024, dtype=torch.uint8, device="cuda")
    off = -raw.data_ptr() % 1024
    t = raw[off:off + n].view(dtype).view(shape)
    if fill is not None:
        t.fill_(fill)
    return t


def _up(v, to):
    return -(-v // to) * to


def _tokens_to_tiles(x, tw):
    """[batch, seq, d] -> [d / tw, batch * seq padded to eight, tw]"""
    b, t, d = x.shape
    tp = _up(t, 8)
    out = _aligned((d // tw, b * tp, tw), x.dtype, 0)
    out.view(d // tw, b, tp, tw)[:, :, :t].copy_(x.view(b, t, d // tw, tw).permute(2, 0, 1, 3))
    return out


def _weights_to_tiles(w, tw, tied):
    """Rows of the vocabulary [vocab, d] -> tiles of [vocab, d] or, with its own head, of [d, vocab]"""
    v, d = w.shape
    if tied:
        out = _aligned((d // tw, _up(v, 8), tw), w.dtype, 0)
        out[:, :v].copy_(w.view(v, d // tw, tw).permute(1, 0, 2))
        return out
    out = _aligned((_up(v, tw) // tw, d, tw), w.dtype, 0)
    full = v // tw
    out[:full].copy_(w[:full * tw].view(full, tw, d).permute(0, 2, 1))
    if v % tw:
        out[full, :, :v % tw].copy_(w[full * tw:].t())
    return out


def _make(case, seed):
    """Inputs from the seed alone, in the layout a user's program has them in."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b, t, d = case["batch"], case["seq"], case["d_model"]
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    tw = 32 if dt is torch.float32 else 64
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    uniform = lambda *shape: torch.rand(shape, generator=gen, device="cuda")
    if case["op"] == "norm":
        # a residual stream: an offset and a scale of its own in every token
        x = normal(b, t, d) * (0.5 + 2 * uniform(b, t, 1)) + 0.3 * normal(b, t, 1)
        inp = {"X": _tokens_to_tiles(x.to(dt), tw), "gamma": 1 + 0.1 * normal(d)}
        inp["beta"] = 0.1 * normal(d) if case["norm"] == "layernorm" else None
        if case["mode"] == "step":
            inp["dY"] = _tokens_to_tiles(normal(b, t, d).to(dt), tw)
        return inp
    v, n, std = case["vocab"], b * t, 0.02
    w = normal(v, d).mul_(std).to(dt)
    # hidden states that point towards their token's row by as much as a model knows about it (up to 12 nats)
    if case["top_k"]:
        k = min(case["top_k"], v)
        # distinct ids, mostly frequent (small) ones, in no order; some tokens' lists are shorter
        gaps = torch.exp(uniform(n, k) * math.log(max(2.0, 2.0 * v / (k + 1) / 3))).long()
        ids = (torch.cumsum(gaps, 1) - 1) % v
        ids = torch.gather(ids, 1, torch.argsort(uniform(n, k), 1)).to(torch.int32)
        logits = 12.0 - 2.5 * torch.log1p(torch.arange(k, device="cuda").float()) + normal(n, k)
        best = torch.gather(ids, 1, torch.argmax(logits, 1, keepdim=True))[:, 0].long()
        short = uniform(n) < 0.05
        ids[short, (k + 1) // 2:] = -1
        ids[uniform(n) < case["ignored"]] = -1
        if case["top_k"] > k:
            pad = case["top_k"] - k
            ids = torch.cat([ids, ids.new_full((n, pad), -1)], 1)
            logits = torch.cat([logits, logits.new_zeros(n, pad)], 1)
        inp = {"ids": ids.contiguous(), "logits": logits.contiguous()}
    else:
        best = torch.exp(uniform(n) * math.log(v)).long().clamp_(1, v) - 1          # frequent ids are small
        targets = best.to(torch.int32)
        targets[uniform(n) < case["ignored"]] = -100
        inp = {"targets": targets}
    pull = uniform(n, 1) * (12.0 / (d * std * std))
    x = normal(n, d) + pull.clamp_(max=2.0 / std) * w[best].float()
    inp["X"] = _tokens_to_tiles(x.to(dt).view(b, t, d), tw)
    inp["W"] = _weights_to_tiles(w, tw, case["tied"])
    inp["dloss"] = (0.5 + uniform(n)) / n if case["weighted"] else None
    return inp


def prepare(case, seed):
    state = {"case": case, "in": _make(case, seed)}
    if own:
        state["call"], state["out"] = _own(case, state["in"])
    torch.cuda.synchronize()
    return state


# ---- the framework's operators --------------------------------------------------------------------------------------

def _own(case, inp):
    """The plan, the buffers beside the inputs, and one pass as a user's program makes it."""
    from paper_2607_21624_b200 import HeadPlan, NormPlan, head_desc, norm_desc

    ptr = lambda a: None if a is None else a.data_ptr()
    stream = lambda: torch.cuda.current_stream().cuda_stream
    work_area = lambda n: _aligned((n,), torch.uint8)
    step = case["mode"] == "step"
    X = inp["X"]
    if case["op"] == "norm":
        plan = NormPlan(norm_desc(case["batch"], case["seq"], case["d_model"], case["dtype"], case["norm"], 1e-5))
        saved, sf, sb = map(work_area, plan.workspace_bytes())
        out = {"Y": _aligned(X.shape, X.dtype)}
        if step:
            out.update(dX=_aligned(X.shape, X.dtype), dgamma=torch.empty_like(inp["gamma"]))
            if inp["beta"] is not None:
                out["dbeta"] = torch.empty_like(inp["beta"])

        def call():
            plan.fwd(ptr(X), ptr(inp["gamma"]), ptr(inp["beta"]), ptr(out["Y"]), ptr(saved), ptr(sf), stream())
            if step:
                plan.bwd(ptr(inp["dY"]), ptr(X), ptr(inp["gamma"]), ptr(saved), ptr(out["dX"]), ptr(out["dgamma"]),
                         ptr(out.get("dbeta")), ptr(sb), stream())
        return call, out

    n = case["batch"] * case["seq"]
    plan = HeadPlan(head_desc(case["batch"], case["seq"], case["d_model"], case["vocab"], case["dtype"], tied=case["tied"],
                              top_k=case["top_k"], temperature=case["temperature"]))
    saved, sf, sb = map(work_area, plan.workspace_bytes())
    W = inp["W"]
    out = {"loss": torch.empty(n, device="cuda"), "total": torch.empty(2, device="cuda")}
    if step:
        out["dX"] = _aligned(X.shape, X.dtype)
        if not case["frozen"]:
            out["dW"] = _aligned(W.shape, W.dtype)

    def call():
        if case["top_k"]:
            plan.distill_fwd(ptr(X), ptr(W), ptr(inp["ids"]), ptr(inp["logits"]), ptr(out["loss"]), ptr(out["total"]),
                             ptr(saved), ptr(sf), stream())
        else:
            plan.xent_fwd(ptr(X), ptr(W), ptr(inp["targets"]), ptr(out["loss"]), ptr(out["total"]), ptr(saved), ptr(sf), stream())
        if step:
            plan.bwd(ptr(X), ptr(W), ptr(inp["dloss"]), ptr(saved), ptr(out["dX"]), ptr(out.get("dW")), ptr(sb), stream())
    return call, out


# ---- the plain form -------------------------------------------------------------------------------------------------

def _rows(tiles):
    """Tiles -> the padded matrix [rows, columns] in fp32."""
    return tiles.permute(1, 0, 2).reshape(tiles.shape[1], -1).float()


def _tiles(m, like):
    """A padded matrix [rows, columns] -> tiles in the type of `like`."""
    p, r, w = like.shape
    return m.to(like.dtype).view(r, p, w).permute(1, 0, 2).contiguous()


def _token_rows(case, tiles):
    """The tokens' rows [batch * seq, d] of a token matrix, in fp32."""
    b, t = case["batch"], case["seq"]
    return _rows(tiles).view(b, _up(t, 8), -1)[:, :t].reshape(b * t, -1)


def _token_tiles(case, m, like):
    b, t = case["batch"], case["seq"]
    full = m.new_zeros(b, _up(t, 8), m.shape[1])
    full[:, :t] = m.view(b, t, -1)
    return _tiles(full.view(b * _up(t, 8), -1), like)


def _plain_norm(case, inp):
    x = _token_rows(case, inp["X"])
    centred = x - x.mean(1, keepdim=True) if case["norm"] == "layernorm" else x
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + 1e-5)
    xh = centred * rstd
    y = xh * inp["gamma"]
    if inp["beta"] is not None:
        y = y + inp["beta"]
    out = {"Y": _token_tiles(case, y, inp["X"])}
    if case["mode"] == "step":
        dy = _token_rows(case, inp["dY"])
        g = dy * inp["gamma"]
        dx = g - xh * (g * xh).mean(1, keepdim=True)
        if case["norm"] == "layernorm":
            dx = dx - g.mean(1, keepdim=True)
            out["dbeta"] = dy.sum(0, dtype=torch.float64).float()
        out["dX"] = _token_tiles(case, dx * rstd, inp["X"])
        out["dgamma"] = (dy * xh).sum(0, dtype=torch.float64).float()
    return out


def _plain_loss(case, inp):
    x, w = _token_rows(case, inp["X"]), _rows(inp["W"])
    v, tau = case["vocab"], case["temperature"]
    w = w[:v].t() if case["tied"] else w[:, :v]                      # [d, vocab]
    z = x @ w / tau
    # the target distribution: one token, or the teacher's softmax over the logits that it gave
    if case["top_k"]:
        there = inp["ids"] >= 0
        raw = torch.where(there, inp["logits"] / tau, float("-inf"))
        counted = there.any(1)
        top = torch.where(counted, raw.amax(1), 0.0)[:, None]
        p = torch.exp(raw - top)
        p = torch.where(there & counted[:, None], p / p.sum(1, keepdim=True), 0.0)
        y = torch.zeros_like(z).scatter_add_(1, inp["ids"].clamp(min=0).long(), p)
    else:
        counted = inp["targets"] >= 0
        y = torch.zeros_like(z)
        y.scatter_(1, inp["targets"].clamp(min=0).long()[:, None], counted.float()[:, None])
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    s = e.sum(1, keepdim=True)
    # sum of y (log y - log softmax): only where y is not zero
    z -= m
    terms = torch.where(y > 0, y * (torch.log(y) - (z - torch.log(s))), 0.0)
    loss = torch.where(counted, terms.sum(1), 0.0)
    del terms, z
    total = torch.stack([loss.sum(dtype=torch.float64).float(), counted.sum().float()])
    out = {"loss": loss, "total": total}
    if case["mode"] == "step":
        g = inp["dloss"] if inp["dloss"] is not None else 1.0 / total[1]
        g = torch.where(counted, g, 0.0)[:, None] / tau
        dz = (e / s - y) * g
        del e, y
        out["dX"] = _token_tiles(case, dz @ w.t(), inp["X"])
        if not case["frozen"]:
            full = dz.new_zeros(inp["W"].shape[1] if case["tied"] else w.shape[0],
                                w.shape[0] if case["tied"] else _up(v, inp["W"].shape[2]))
            if case["tied"]:
                full[:v] = dz.t() @ x
            else:
                full[:, :v] = x.t() @ dz
            out["dW"] = _tiles(full, inp["W"])
    return out


def run(state):
    if own:
        state["call"]()
        return state["out"]
    return (_plain_norm if state["case"]["op"] == "norm" else _plain_loss)(state["case"], state["in"])


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    n, d, e = case["batch"] * case["seq"], case["d_model"], 4 if case["dtype"] == "fp32" else 2
    step = case["mode"] == "step"
    if case["op"] == "norm":
        vectors = (2 if case["norm"] == "layernorm" else 1) * 4 * d
        return {"bytes": float(n * d * e * (4 if step else 2) + vectors * (2 if step else 1)), "flops": (20.0 if step else 8.0) * n * d}
    weights = d * case["vocab"]
    products = 1 if not step else 2 if case["frozen"] else 3
    targets = n * (8 * case["top_k"] if case["top_k"] else 4)
    moved = n * d * (2 if step else 1) + weights * (2 if products == 3 else 1)
    return {"bytes": float(e * moved + targets + 4 * n + (4 * n if step and case["weighted"] else 0)), "flops": 2.0 * n * weights * products}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _unpack64(tiles, batch, seq):
    """A token matrix's tiles -> float64 [batch * seq, d], panel by panel."""
    per = tiles.shape[1] // batch
    cols = [panel.double().view(batch, per, -1)[:, :seq].reshape(batch * seq, -1) for panel in tiles]
    return torch.cat(cols, 1)


def _repack64(m, batch, seq, panels, width):
    per = _up(seq, 8)
    out = torch.zeros(panels, batch, per, width, dtype=torch.float64, device=m.device)
    for p in range(panels):
        out[p, :, :seq] = m[:, p * width:(p + 1) * width].view(batch, seq, width)
    return out.view(panels, batch * per, width)


def _exact_norm(case, inp):
    b, t = case["batch"], case["seq"]
    X, (panels, _, width) = inp["X"], inp["X"].shape
    x, gamma = _unpack64(X, b, t), inp["gamma"].double()
    rows, d = x.shape
    mu = torch.zeros(rows, 1, dtype=torch.float64, device=x.device)
    if case["norm"] == "layernorm":
        mu = x.sum(1, keepdim=True) / d
    sigma = torch.sqrt(((x - mu) ** 2).sum(1, keepdim=True) / d + 1e-5)
    xh = (x - mu) / sigma
    beta = 0.0 if inp["beta"] is None else inp["beta"].double()
    out = {"Y": _repack64(gamma * xh + beta, b, t, panels, width)}
    if case["mode"] == "step":
        dy = _unpack64(inp["dY"], b, t)
        # d xh_j / d x_i = (delta_ij - 1/d [- only with a mean] - xh_i xh_j / d) / sigma
        u = dy * gamma
        dx = u - xh * ((u * xh).sum(1, keepdim=True) / d)
        if case["norm"] == "layernorm":
            dx -= u.sum(1, keepdim=True) / d
            out["dbeta"] = dy.sum(0)
        out["dX"] = _repack64(dx / sigma, b, t, panels, width)
        out["dgamma"] = (dy * xh).sum(0)
    return out


def _exact_loss(case, inp):
    b, t, v, tau = case["batch"], case["seq"], case["vocab"], case["temperature"]
    X, W = inp["X"], inp["W"]
    x = _unpack64(X, b, t)
    n, d = x.shape

    def columns(lo, hi):
        """Weights of tokens lo .. hi - 1 in 64 bits, [hi - lo, d]."""
        if case["tied"]:
            return torch.cat([panel[lo:hi].double() for panel in W], 1)
        w = W.shape[2]
        pick = W[lo // w:-(-hi // w)].double().transpose(1, 2).reshape(-1, d)
        return pick[lo - lo // w * w:hi - lo // w * w]

    # (token, id, probability) of the targets; ids given twice add up
    if case["top_k"]:
        ids, raw = inp["ids"].long(), inp["logits"].double() / tau
        real = ids >= 0
        weight = torch.where(real, torch.exp(raw - raw.max()), torch.zeros((), dtype=torch.float64, device=x.device))
        mass = weight.sum(1)
        live = mass > 0
        i, k = torch.nonzero(real, as_tuple=True)
        flat, inverse = torch.unique(i * v + ids[i, k], return_inverse=True)
        prob = torch.zeros(flat.numel(), dtype=torch.float64, device=x.device).index_add_(0, inverse, weight[i, k] / mass[i])
    else:
        tgt = inp["targets"].long()
        live = tgt >= 0
        i = torch.nonzero(live)[:, 0]
        flat, prob = i * v + tgt[i], torch.ones(i.numel(), dtype=torch.float64, device=x.device)
    who, what = flat // v, flat % v
    # normalisers, a piece of the vocabulary at a time
    piece = max(4096, min(v, int(2.0e8 // max(n, 1)) // 64 * 64))
    cuts = [(lo, min(lo + piece, v)) for lo in range(0, v, piece)]
    lse = torch.full((n,), -math.inf, dtype=torch.float64, device=x.device)
    z_at = torch.zeros_like(prob)
    for lo, hi in cuts:
        z = x @ columns(lo, hi).t() / tau
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
        here = (what >= lo) & (what < hi)
        z_at[here] = z[who[here], what[here] - lo]
    loss = torch.zeros(n, dtype=torch.float64, device=x.device)
    loss.index_add_(0, who, torch.where(prob > 0, prob * (torch.log(prob) - z_at + lse[who]), torch.zeros_like(prob)))
    count = live.sum().double()
    out = {"loss": loss, "total": torch.stack([loss.sum(), count])}
    if case["mode"] == "step":
        g = inp["dloss"].double() if inp["dloss"] is not None else torch.ones(n, dtype=torch.float64, device=x.device) / count
        g = torch.where(live, g, torch.zeros_like(g)) / tau
        dx = torch.zeros_like(x)
        dw = torch.zeros(0)
        if not case["frozen"]:
            dw = torch.zeros(W.shape, dtype=torch.float64, device=x.device)
        for lo, hi in cuts:
            w = columns(lo, hi)
            q = torch.exp(x @ w.t() / tau - lse[:, None])
            here = (what >= lo) & (what < hi)
            q[who[here], what[here] - lo] -= prob[here]
            q *= g[:, None]
            dx += q @ w
            if not case["frozen"]:
                dwp, width = q.t() @ x, W.shape[2]
                if case["tied"]:
                    dw[:, lo:hi] = dwp.view(hi - lo, d // width, width).permute(1, 0, 2)
                else:
                    grown = torch.zeros(_up(hi - lo, width), d, dtype=torch.float64, device=x.device)
                    grown[:hi - lo] = dwp
                    first = lo // width
                    dw[first:first + grown.shape[0] // width] = grown.view(-1, width, d).transpose(1, 2)
        out["dX"] = _repack64(dx, b, t, X.shape[0], X.shape[2])
        if not case["frozen"]:
            out["dW"] = dw
    return out


def exact(case, seed):
    inp = _make(case, seed)
    return (_exact_norm if case["op"] == "norm" else _exact_loss)(case, inp)
