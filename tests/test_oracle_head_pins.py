"""Pins for the head's oracle (oracle/head.py): numerical derivatives, closed forms and structural properties; and the C boundary's
refusals and sizes, which need no device."""
import ctypes as C
import math

import numpy as np
import pytest

from fbl_inputs import HeadConfig, make_head_inputs
from oracle import head as orc
from paper_2607_21624_b200 import FblError, HeadPlan, NormPlan, head_desc, norm_desc


def tiny(top_k=0, tied=False, tau=1.0, V=7, norm="layernorm", seed=3):
    return HeadConfig("tiny", 2, 3, 5, V, "fp32", tied, top_k, tau, norm, 1e-5, seed, 0.7)


def objective(cfg, inp):
    r = orc.head_fwd_bwd(cfg, inp)
    if inp["dloss"] is not None:
        return float((r["loss"] * inp["dloss"]).sum())
    return float(r["total"][0] / max(r["total"][1], 1.0))


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("top_k,tau", [(0, 1.0), (3, 1.0), (4, 2.5)])
@pytest.mark.parametrize("weighted", [False, True])
def test_finite_differences(tied, top_k, tau, weighted):
    cfg = tiny(top_k, tied, tau)
    inp = make_head_inputs(cfg, ignored=0.3, weighted=weighted)
    g = orc.head_fwd_bwd(cfg, inp)
    h = 1e-6
    for name in ("X", "W"):
        flat, got = inp[name].reshape(-1), g["d" + name].reshape(-1)
        for i in range(flat.size):
            keep = flat[i]
            flat[i] = keep + h
            up = objective(cfg, inp)
            flat[i] = keep - h
            down = objective(cfg, inp)
            flat[i] = keep
            assert abs((up - down) / (2 * h) - got[i]) <= 1e-8, (name, i)


@pytest.mark.parametrize("kind", ["layernorm", "rmsnorm"])
def test_norm_backward_finite_differences(kind):
    rng = np.random.default_rng(0)
    X, gamma, beta, dY = rng.normal(size=(2, 3, 6)), rng.normal(size=6), rng.normal(size=6), rng.normal(size=(2, 3, 6))
    if kind == "rmsnorm":
        beta = None
    dX, dg, db = orc.norm_bwd(dY, X, gamma, 1e-5, kind)
    f = lambda: float((orc.norm_fwd(X, gamma, beta, 1e-5, kind)[0] * dY).sum())
    h = 1e-6
    for arr, got in ((X, dX), (gamma, dg)) + (((beta, db),) if beta is not None else ()):
        flat, want = arr.reshape(-1), got.reshape(-1)
        for i in range(flat.size):
            keep = flat[i]
            flat[i] = keep + h
            up = f()
            flat[i] = keep - h
            down = f()
            flat[i] = keep
            assert abs((up - down) / (2 * h) - want[i]) <= 1e-7


def test_closed_forms():
    cfg = tiny()
    inp = make_head_inputs(cfg)
    inp["W"] = np.zeros_like(inp["W"])
    assert np.allclose(orc.head_fwd_bwd(cfg, inp)["loss"], math.log(cfg.vocab), rtol=1e-14)
    # one teacher logit is a label, whatever its value and the temperature's effect on it
    one = tiny(top_k=1)
    a = make_head_inputs(one)
    lab = {**a, "targets": a["top_ids"][..., 0]}
    r, q = orc.head_fwd_bwd(one, a), orc.head_fwd_bwd(tiny(), lab)
    assert np.allclose(r["loss"], q["loss"]) and np.allclose(r["dX"], q["dX"])
    # a teacher that gives the student's own logits over all ids: no divergence, no gradient
    full = tiny(top_k=7, tau=2.0)
    b = make_head_inputs(full)
    z = orc.head_fwd_bwd(full, b)["Z"] * full.temperature
    b["top_ids"] = np.broadcast_to(np.arange(7, dtype=np.int32), (2, 3, 7)).copy()
    b["top_logits"] = z.reshape(2, 3, 7)
    r = orc.head_fwd_bwd(full, b)
    assert np.abs(r["loss"]).max() < 1e-14 and np.abs(r["dX"]).max() < 1e-15


def test_structure():
    cfg = tiny(top_k=4, tau=1.5)
    inp = make_head_inputs(cfg, ignored=0.4)
    r = orc.head_fwd_bwd(cfg, inp)
    assert (r["loss"] >= -1e-15).all()                              # a divergence
    assert np.abs(r["dZ"].sum(1)).max() < 1e-16                     # softmax and y both sum to one
    gone = ~r["has"]
    assert gone.any() and (r["loss"][gone] == 0).all() and (r["dX"][gone] == 0).all()
    # an id given twice with probabilities p, q is the id once with p + q
    twice = dict(inp, top_ids=inp["top_ids"].copy(), top_logits=inp["top_logits"].copy())
    twice["top_ids"][..., 3] = np.where(twice["top_ids"][..., 3] >= 0, twice["top_ids"][..., 0], -1)
    once = dict(twice, top_ids=twice["top_ids"].copy(), top_logits=twice["top_logits"].copy())
    once["top_ids"][..., 3] = -1
    tau = cfg.temperature
    once["top_logits"][..., 0] = tau * np.logaddexp(twice["top_logits"][..., 0] / tau, twice["top_logits"][..., 3] / tau)
    assert np.allclose(orc.head_fwd_bwd(cfg, twice)["loss"], orc.head_fwd_bwd(cfg, once)["loss"], atol=1e-14)
    # tied weights are the transposed ones
    u = tiny()
    a = make_head_inputs(u)
    t = tiny(tied=True)
    b = dict(a, W=a["W"].T.copy())
    assert np.allclose(orc.head_fwd_bwd(u, a)["dW"].T, orc.head_fwd_bwd(t, b)["dW"])


# ---- the C boundary without a device --------------------------------------------------------------------------------

def refused(code, make):
    with pytest.raises(FblError) as e:
        make()
    assert e.value.code == code


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(seq=0), -1), (dict(seq=-3), -1), (dict(d_model=0), -1), (dict(vocab=0), -1), (dict(vocab=-5), -1),
    (dict(top_k=-1), -1), (dict(temperature=0.0), -1), (dict(temperature=-1.0), -1), (dict(temperature=float("nan")), -1),
    (dict(temperature=float("inf"), top_k=4), -1), (dict(temperature=1e-39, top_k=4), -1), (dict(temperature=2.0), -1),
    (dict(d_model=96), -2), (dict(d_model=16448), -2), (dict(vocab=(1 << 20) + 1), -2), (dict(top_k=129), -2), (dict(batch=1 << 20, seq=8), -2),
])
def test_head_plan_refusals(kw, code):
    base = dict(batch=2, seq=5, d_model=128, vocab=1000, dtype="bf16", tied=False, top_k=0, temperature=1.0)
    refused(code, lambda: HeadPlan(head_desc(**{**base, **kw})))


@pytest.mark.parametrize("kw,code", [(dict(batch=0), -1), (dict(seq=0), -1), (dict(d_model=0), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
                                     (dict(d_model=100), -2), (dict(d_model=16448), -2)])
def test_norm_plan_refusals(kw, code):
    base = dict(batch=2, seq=5, d_model=128, dtype="bf16", norm="layernorm", eps=1e-5)
    refused(code, lambda: NormPlan(norm_desc(**{**base, **kw})))


def test_unknown_enumerations_are_refused():
    for field, value in (("dtype", 7), ("vocab_rows", 2)):
        d = head_desc(2, 5, 128, 1000)
        setattr(d, field, value)
        refused(-1, lambda: HeadPlan(d))
    for field, value in (("dtype", 7), ("norm", 2)):
        d = norm_desc(2, 5, 128)
        setattr(d, field, value)
        refused(-1, lambda: NormPlan(d))


OK = 1 << 20        # looks like an aligned device pointer; no call below gets as far as using it


def test_head_calls_refuse_missing_and_misaligned_pointers():
    labels, teacher = HeadPlan(head_desc(2, 5, 128, 1000)), HeadPlan(head_desc(2, 5, 128, 1000, top_k=4, temperature=2.0))
    names = ["X", "W", "targets", "loss", "total", "saved", "scratch"]
    for i, name in enumerate(names):
        args = [OK] * 7
        args[i] = None
        refused(-1, lambda: labels.xent_fwd(*args, 0))
        if name in ("X", "W", "saved", "scratch"):
            args[i] = OK + 512
            refused(-3, lambda: labels.xent_fwd(*args, 0))
    for i, name in enumerate(["X", "W", "top_ids", "top_logits", "loss", "total", "saved", "scratch"]):
        args = [OK] * 8
        args[i] = None
        refused(-1, lambda: teacher.distill_fwd(*args, 0))
        if name in ("X", "W", "saved", "scratch"):
            args[i] = OK + 16
            refused(-3, lambda: teacher.distill_fwd(*args, 0))
    # a plan for labels has no teacher, and the other way round
    refused(-1, lambda: teacher.xent_fwd(*[OK] * 7, 0))
    refused(-1, lambda: labels.distill_fwd(*[OK] * 8, 0))
    for i, name in enumerate(["X", "W", "dloss", "saved", "dX", "dW", "scratch"]):
        args = [OK] * 7
        if name in ("X", "W", "saved", "scratch"):
            args[i] = None
            refused(-1, lambda: labels.bwd(*args, 0))
        if name != "dloss":
            args[i] = OK + 512
            refused(-3, lambda: labels.bwd(*args, 0))
    refused(-1, lambda: labels.bwd(OK, OK, None, OK, None, None, OK, 0))          # no gradient asked for


def test_norm_calls_refuse_missing_and_misaligned_pointers():
    ln, rms = NormPlan(norm_desc(2, 5, 128)), NormPlan(norm_desc(2, 5, 128, norm="rmsnorm"))
    for i, name in enumerate(["X", "gamma", "beta", "Y", "saved", "scratch"]):
        args = [OK] * 6
        args[i] = None
        refused(-1, lambda: ln.fwd(*args, 0))
        if name in ("X", "Y", "saved", "scratch"):
            args[i] = OK + 512
            refused(-3, lambda: ln.fwd(*args, 0))
    for i, name in enumerate(["dY", "X", "gamma", "saved", "dX", "dgamma", "dbeta", "scratch"]):
        args = [OK] * 8
        args[i] = None
        refused(-1, lambda: ln.bwd(*args, 0))                                      # dgamma without dbeta, too
        if name in ("dY", "X", "saved", "dX", "scratch"):
            args[i] = OK + 512
            refused(-3, lambda: ln.bwd(*args, 0))
    refused(-1, lambda: rms.bwd(*[OK] * 8, 0))                                     # no mean, no dbeta


@pytest.mark.parametrize("dtype,tw", [("bf16", 64), ("fp32", 32)])
@pytest.mark.parametrize("vocab", [1, 7, 64, 1000, 50257])
def test_sizes(dtype, tw, vocab):
    e = 4 if dtype == "fp32" else 2
    up = lambda v, to: -(-v // to) * to
    own, tied = HeadPlan(head_desc(3, 5, 128, vocab, dtype)), HeadPlan(head_desc(3, 5, 128, vocab, dtype, tied=True))
    assert own.tensor_bytes(0) == tied.tensor_bytes(0) == 3 * 8 * 128 * e
    assert own.tensor_bytes(1) == 128 * up(vocab, tw) * e
    assert tied.tensor_bytes(1) == up(vocab, 8) * 128 * e
    for plan in (own, tied):
        assert all(b % 1024 == 0 and b > 0 for b in plan.workspace_bytes())
        with pytest.raises(FblError):
            plan.tensor_bytes(2)
    # no work area grows like tokens x vocabulary once pieces come into it
    big = HeadPlan(head_desc(8, 2048, 1024, 128256, dtype)).workspace_bytes()
    assert max(big) < 16384 * 128256 * e / 4


def test_launch_counts_of_no_plan():
    from paper_2607_21624_b200 import lib
    L = lib()
    L.fbl_head_launch_count.restype = L.fbl_norm_launch_count.restype = C.c_int64
    assert L.fbl_head_launch_count(None) == -1 and L.fbl_norm_launch_count(None) == -1
