"""The head (fbl_head_*) and the norm in front of it on the GPU, through the C ABI, against the float64 oracle.

Tolerances, from the arithmetic.  u = 2^-8 is half a step of bf16 relative to the value, 2^-24 of fp32.
  logits (bf16)  products of bf16 are exact; the tensor core cuts each of its additions (one per 16 columns) by at most 2^-23 of the
                 sum it holds, which is at most |x| |w|:  |dz| <= (D/16 + 2) 2^-23 max(|x| |w|) =: e_z  (the correction for it is smaller)
  loss           2 e_z / temperature, and fp32 steps of values of the size of lse and z (eight of them), and 2^-20 for the exponentials
                 (2^-22 of the sum each) and the sums of 64 and joins
  dz = g (p - y) its rounding u, one per element; and the error of p, which is left in full where p - y cancels: p (2 e_z + 2^-19) for the
                 logits, the exponentials, the sums of them and the division
  dX, dW (bf16)  sums over independent roundings of dz, standard deviation u / sqrt(3) sqrt(sum dz^2 w^2): six of them; additions cut by
                 2^-23 of sum |dz| |w| per 16 columns; the result's own rounding u
                 and in the Frobenius norm two roundings at their rms of u / sqrt(3), added up in full
                 values below 2^-126 are zero in fp32
  fp32           1e-5 of an element or of the tensor's rms: sums in fp32 by parts (2e-7 of the norm), probabilities 3e-6
"""
import numpy as np
import pytest

from fbl_inputs import HeadConfig, make_head_inputs
from oracle import head as orc
from paper_2607_21624_b200 import HeadPlan, HeadRunner, NormHeadRunner, NormRunner, aligned_bytes, head_desc

from util import fp32_err

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
RMS = U / np.sqrt(3.0)


def cfg(batch, seq, d, vocab, dtype="bf16", tied=False, top_k=0, tau=1.0, seed=5, w_std=0.05, norm="layernorm"):
    name = f"{batch}x{seq}x{d}-v{vocab}-{dtype}-{'vd' if tied else 'dv'}-k{top_k}"
    return HeadConfig(name, batch, seq, d, vocab, dtype, tied, top_k, tau, norm, 1e-5, seed, w_std)


def logit_error(c, inp, ref):
    """e_z / temperature of each token"""
    n = c.batch * c.seq
    x = np.abs(inp["X"].reshape(n, -1))
    w = np.abs(inp["W"].T if c.tied else inp["W"])
    e_z = (c.d_model / 16 + 2) * 2.0 ** -23 * (x @ w).max(1) if c.dtype == "bf16" else 1e-6 * np.abs(ref["Z"] * c.temperature).max(1)
    return e_z / c.temperature


def loss_bound(c, inp, ref):
    size = np.abs(ref["lse"]) + np.abs(ref["Z"]).max(1)
    return (2 * logit_error(c, inp, ref) + 8 * 2.0 ** -24 * size + 2.0 ** -20).reshape(c.batch, c.seq)


def dz_slack(c, inp, ref):
    """What the error of p leaves in dz where p - y cancels."""
    n = c.batch * c.seq
    g = np.full(n, 1.0 / max(ref["total"][1], 1.0)) if inp["dloss"] is None else inp["dloss"].reshape(-1)
    p = np.where(ref["has"].reshape(-1)[:, None], np.exp(ref["Z"] - ref["lse"][:, None]), 0.0)
    return p * (g * (2 * logit_error(c, inp, ref) + 2.0 ** -19) / c.temperature)[:, None]


def check_grad(name, c, got, ref, a, b, terms, slack):
    """a, b: the factors of the product |a| |b|, in whose rounded factor the error lies; slack: a product of the same kind."""
    assert np.isfinite(got).all(), name
    if c.dtype == "fp32":
        assert fp32_err(got, ref) <= 1e-5, (name, fp32_err(got, ref))
        return
    bound = 6 * RMS * np.sqrt((a ** 2) @ (b ** 2)) + (terms / 16 * 2.0 ** -23 + 2.0 ** -18) * (np.abs(a) @ np.abs(b)) + U * np.abs(ref) + slack + \
        terms * 2.0 ** -126 * max(1.0, np.abs(a).max(), np.abs(b).max())
    over = np.abs(got - ref) - bound.reshape(ref.shape)
    assert over.max() <= 0, (name, float(over.max()), float(np.abs(ref).max()))
    norm = np.linalg.norm(ref)
    if norm > 0:
        assert np.linalg.norm(got - ref) <= 2 * RMS * norm, (name, np.linalg.norm(got - ref) / norm)


def compare(c, inp, run, ref=None, dw=True):
    ref = ref or orc.head_fwd_bwd(c, inp)
    n = c.batch * c.seq
    loss = run.fetch("loss").reshape(c.batch, c.seq)
    bound = loss_bound(c, inp, ref)
    assert (np.abs(loss - ref["loss"]) <= bound).all(), float((np.abs(loss - ref["loss"]) - bound).max())
    assert (loss[~ref["has"]] == 0).all()
    total = run.fetch("total")
    assert total[1] == ref["total"][1] and abs(total[0] - ref["total"][0]) <= bound.sum() + 2.0 ** -22 * abs(ref["total"][0])
    w = inp["W"].T if c.tied else inp["W"]
    x = inp["X"].reshape(n, -1)
    slack = dz_slack(c, inp, ref)
    dX = run.fetch("dX")
    check_grad("dX", c, dX.reshape(n, -1), ref["dX"].reshape(n, -1), ref["dZ"], w.T, c.vocab, slack @ np.abs(w.T))
    assert (dX[~ref["has"]] == 0).all()
    if dw:
        dW = run.fetch("dW")
        check_grad("dW", c, dW.T if c.tied else dW, ref["dW"].T if c.tied else ref["dW"], x.T, ref["dZ"], n, np.abs(x.T) @ slack)
    assert run.status() == 0
    assert run.guards_intact() == []
    return ref


def run_and_compare(c, ignored=0.0, weighted=False, frozen=False):
    inp = make_head_inputs(c, ignored=ignored, weighted=weighted)
    run = HeadRunner(c, guard_bytes=4096, frozen=frozen)
    for b in (run.saved, run.scratch_fwd, run.scratch):          # work areas hold anything
        b.fill_(0xC3)
    run.load_inputs(inp)
    run.step()
    compare(c, inp, run, dw=not frozen)
    return run, inp


SHAPES = [
    (1, 1, 64, 1), (1, 1, 64, 300), (1, 1, 128, 5), (3, 1, 192, 77), (1, 9, 64, 64), (2, 50, 128, 1000), (3, 41, 256, 257),
    (1, 127, 128, 511), (1, 128, 64, 512), (5, 129, 128, 513), (2, 300, 320, 2049), (1, 700, 128, 3001), (16, 24, 64, 127),
]


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_labels(shape, dtype, tied):
    run_and_compare(cfg(*shape, dtype, tied), ignored=0.3 if shape[1] % 2 else 0.0, weighted=shape[0] > 1)


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape,top_k,tau", [((1, 1, 64, 300), 1, 1.0), ((2, 50, 128, 1000), 8, 2.0), ((3, 41, 256, 257), 20, 1.0),
                                             ((1, 300, 128, 2049), 64, 4.0), ((5, 129, 128, 513), 128, 0.5), ((2, 7, 64, 3), 3, 1.0)],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_teacher(shape, top_k, tau, dtype, tied):
    run_and_compare(cfg(*shape, dtype, tied, top_k, tau), ignored=0.25 if shape[1] > 1 else 0.0, weighted=shape[0] == 2)


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("piece,slices", [("256", "1"), ("512", "3"), ("1024", "40"), ("100000", "5")])
def test_pieces_and_slices(monkeypatch, piece, slices, dtype, tied):
    monkeypatch.setenv("FBL_HEAD_PIECE", piece)
    monkeypatch.setenv("FBL_HEAD_SLICES", slices)
    run_and_compare(cfg(2, 150, 128, 1339, dtype, tied), ignored=0.2)
    run_and_compare(cfg(1, 60, 192, 1290, dtype, tied, 16, 2.0), weighted=True)


@pytest.mark.parametrize("pair", ["0", "1"])
def test_one_block_and_pairs(monkeypatch, pair):
    monkeypatch.setenv("FBL_GEMM_PAIR", pair)
    for tied in (False, True):
        run_and_compare(cfg(2, 333, 256, 1500, tied=tied), ignored=0.3)
        run_and_compare(cfg(1, 40, 128, 700, tied=tied, top_k=32))


@pytest.mark.parametrize("tile", ["0", "1", "2", "3", "4"])
def test_every_tile_of_the_logits(monkeypatch, tile):
    """Pairs and one block, sets of epilogue warps in turn, side by side and one; vocabularies that end in every part of a tile."""
    monkeypatch.setenv("FBL_HEAD_TILE", tile)
    for vocab in (1, 64, 65, 129, 190, 257, 450):
        run_and_compare(cfg(2, 75, 192, vocab, tied=vocab % 2 == 0), ignored=0.3)
    run_and_compare(cfg(3, 130, 64, 3000, tied=True), weighted=True)
    run_and_compare(cfg(2, 140, 320, 2200, top_k=40, tau=2.0), ignored=0.2)


@pytest.mark.parametrize("bn", ["64", "128"])
def test_fp32_tiles(monkeypatch, bn):
    monkeypatch.setenv("FBL_F32_BN", bn)
    for vocab in (1, 33, 64, 65, 97, 129, 450):
        run_and_compare(cfg(2, 75, 96, vocab, "fp32", tied=vocab % 2 == 0), ignored=0.3)
    run_and_compare(cfg(2, 140, 320, 2200, "fp32", top_k=40, tau=2.0), weighted=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_frozen_sides(dtype):
    c = cfg(2, 77, 128, 1000, dtype)
    run, inp = run_and_compare(c, ignored=0.2, frozen=True)
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.buf["dX"].fill_(0x5A)
    run.forward()
    run.backward(dx=False)                                       # a frozen model under a new head
    dW = run.fetch("dW")
    xt = inp["X"].reshape(154, -1).T
    check_grad("dW", c, dW, ref["dW"], xt, ref["dZ"], 154, np.abs(xt) @ dz_slack(c, inp, ref))
    assert bool((run.buf["dX"] == 0x5A).all()) and run.guards_intact() == []


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("piece", [None, "1024"])
@pytest.mark.parametrize("shape", [(1, 50, 128, 9000), (1, 7, 512, 6011), (2, 150, 128, 5003)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_together_and_alone_in_turn(monkeypatch, shape, piece, dtype):
    """dX alone is cut into slices of its own: of one plan and one area, whatever came before it there."""
    if piece:
        monkeypatch.setenv("FBL_HEAD_PIECE", piece)
    c = cfg(*shape, dtype, tied=True)
    inp = make_head_inputs(c, ignored=0.2)
    n = c.batch * c.seq
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.forward()
    ref, first = orc.head_fwd_bwd(c, inp), {}
    slack, x = dz_slack(c, inp, ref) @ np.abs(inp["W"]), inp["X"].reshape(n, -1)
    for fill, dx, dw in ((0xFF, True, True), (0xFF, True, False), (0x7F, True, False), (0x7F, False, True), (0x7F, True, True), (0xFF, True, False)):
        run.scratch.fill_(fill)
        run.buf["dX"].fill_(0x11)
        run.buf["dW"].fill_(0x11)
        run.backward(dx=dx, dw=dw)
        assert run.status() == 0 and run.guards_intact() == []
        for name, on in (("dX", dx), ("dW", dw)):
            if on:
                got = run.fetch(name)
                assert np.array_equal(first.setdefault((name, dx, dw), got), got)
            else:
                assert bool((run.buf[name] == 0x11).all())
        if dx:
            check_grad("dX", c, run.fetch("dX").reshape(n, -1), ref["dX"].reshape(n, -1), ref["dZ"], inp["W"], c.vocab, slack)
        if dw:                                       # (fp32's reductions over the tokens are cut by the launch's problems, too)
            check_grad("dW", c, run.fetch("dW").T, ref["dW"].T, x.T, ref["dZ"], n, np.abs(x.T) @ dz_slack(c, inp, ref))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top_k", [0, 4])
def test_no_token_has_a_loss(dtype, top_k):
    for shape in ((1, 1, 64, 300), (2, 150, 128, 1000)):
        c = cfg(*shape, dtype, top_k=top_k)
        run, _ = run_and_compare(c, ignored=2.0)
        for n in ("loss", "total", "dX", "dW"):
            assert (run.fetch(n) == 0).all(), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top_k", [0, 4])
def test_rows_without_a_loss_are_not_looked_at(dtype, top_k):
    import torch
    c = cfg(3, 45, 128, 700, dtype, top_k=top_k)
    inp = make_head_inputs(c, ignored=0.4)
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c)
    run.load_inputs(inp)
    run.step()
    want = {n: run.fetch(n) for n in ("loss", "total", "dX", "dW")}
    for bad in (np.nan, np.inf, -np.inf, -3e38):
        x = inp["X"].copy()
        x[~ref["has"]] = bad
        run.load_inputs({**inp, "X": x})
        # the padding between sequences, too
        e = 4 if dtype == "fp32" else 2
        pad = run.buf["X"].view(run.tdtype).view(c.d_model * e // 128, 3, 48, 128 // e)[:, :, 45:]
        pad.fill_(bad if dtype == "fp32" or abs(bad) > 3.1e38 or bad != bad else -3e38)
        run.step()
        for n, v in want.items():
            assert np.array_equal(v, run.fetch(n)), (n, bad)
    torch.cuda.synchronize()
    assert run.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_labels_past_the_vocabulary_make_nan_and_nothing_else(dtype):
    c = cfg(2, 30, 64, 300, dtype)
    inp = make_head_inputs(c)
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    bad = dict(inp, targets=inp["targets"].copy())
    bad["targets"][1, 7], bad["targets"][0, 29] = 300, 2 ** 31 - 1
    run.load_inputs(bad)
    run.step()
    loss, dX = run.fetch("loss").reshape(2, 30), run.fetch("dX")
    gone = np.zeros((2, 30), dtype=bool)
    gone[1, 7] = gone[0, 29] = True
    assert np.isnan(loss[gone]).all() and np.isnan(dX[gone]).all() and np.isnan(run.fetch("total")[0])
    assert run.fetch("total")[1] == 60
    assert (np.abs(loss - ref["loss"])[~gone] <= loss_bound(c, inp, ref)[~gone]).all()
    assert np.isfinite(dX[~gone]).all() and np.isnan(run.fetch("dW")).all()
    assert run.guards_intact() == [] and run.status() == 0
    bad["targets"][1, 7], bad["targets"][0, 29] = -1, -(2 ** 31)           # below zero: no loss
    run.load_inputs(bad)
    run.step()
    compare(c, bad, run)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_teachers_lists(dtype):
    """The same id twice, logits of -inf, short lists, lists of nothing, and what makes a row NaN."""
    c = cfg(1, 24, 64, 200, dtype, top_k=6, tau=2.0)
    inp = make_head_inputs(c)
    ids, lg = inp["top_ids"][0], inp["top_logits"][0]
    ids[0] = [5, 5, 5, 5, 5, 5]                     # one id, six times: a label
    ids[1] = [9, 3, 9, 3, 9, 3]
    ids[2, 1:] = -1
    ids[3, ::2] = -7
    lg[4, :5] = -np.inf                             # all on the last
    lg[5] = -np.inf                                 # nothing
    lg[6, 2] = -np.inf
    lg[7] = 1e30                                    # equal, large
    lg[8] = [3e38, -3e38, 0, 0, 0, 0]
    ids[9, 0], lg[9, 0] = -1, np.nan                # not there, whatever it says
    ids[10, 0], lg[10, 0] = -1, np.inf
    ids[11] = [199, 0, 63, 64, 65, 128]
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    clean = dict(inp, top_logits=np.where(inp["top_ids"] < 0, 0.0, inp["top_logits"]))
    ref = compare(c, clean, run)
    assert not ref["has"][0, 5] and ref["has"].sum() == 23
    ids[12, 3] = 200
    lg[13, 0] = np.nan
    lg[14, 5] = np.inf
    run.load_inputs(inp)
    run.step()
    loss, dX = run.fetch("loss").reshape(-1), run.fetch("dX")[0]
    gone = np.isin(np.arange(24), [12, 13, 14])
    assert np.isnan(loss[gone]).all() and np.isnan(dX[gone]).all()
    assert (np.abs(loss - ref["loss"][0])[~gone] <= loss_bound(c, clean, ref)[0][~gone]).all() and np.isfinite(dX[~gone]).all()
    assert run.guards_intact() == [] and run.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tau", [0.5, 1e-30, 3.0, 1e30])
def test_teachers_large_logits_and_temperatures(tau, dtype):
    """Finite logits have a loss at any temperature, also where a logit / temperature leaves fp32, and count by their distances, also where
    those are a step of fp32 beside the logits themselves.  Weights of zero: a loss is log vocab - entropy of the list, whose probabilities
    are off by 2^-24 of a distance of at most 160 (beyond, a probability is below 2^-126 and zero in fp32), and by expf's two steps."""
    c = cfg(1, 24, 64, 200, dtype, top_k=6, tau=tau)
    inp = make_head_inputs(c)
    inp["W"][:] = 0.0
    ids, lg = inp["top_ids"][0], inp["top_logits"][0]
    ids[:] = [3, 17, 64, 128, 199, 0]
    lg[0] = [3e38, -3e38, 3e38, 0, 0, 0]
    lg[1] = -3e38                                   # finite, equal: a loss
    lg[2] = [-3e38, -3e38, -np.inf, -np.inf, -np.inf, -np.inf]
    lg[3] = [3e38, 3e38, 3e38, 3e38, 3e38, 3e38]
    for i in range(4, 24):                          # 1e4 to 1e5, a few apart
        lg[i] = np.float32(1e4 * 1.13 ** (i - 4) * (-1 if i % 3 == 0 else 1)) + np.float32([0, 1, -1, 2, 0.5, -0.25])
    ids[23, 2], lg[23, 2] = -1, 3e38                # not there
    lg[:] = lg.astype(np.float32)
    ref = orc.head_fwd_bwd(c, inp)
    y, has = orc.targets(c, inp)
    assert has.all()
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    with np.errstate(divide="ignore", invalid="ignore"):
        terms = np.where(y > 0, y * (1 + np.abs(np.log(y))), 0.0).sum(1)
    off = np.abs(run.fetch("loss") - ref["loss"][0])
    assert (off <= terms * 160 * 2.0 ** -24 + 8 * 2.0 ** -24 * np.log(200) + 2.0 ** -20).all(), off.max()
    assert run.fetch("total")[1] == 24 and run.guards_intact() == [] and run.status() == 0
    assert (run.fetch("dX") == 0).all()
    x, dz = inp["X"].reshape(24, -1).T, ref["dZ"]
    check_grad("dW", c, run.fetch("dW") * min(tau, 1.0), ref["dW"] * min(tau, 1.0), x, dz * min(tau, 1.0), 24, np.abs(x) @ (np.abs(dz) + y / 24 / tau) * min(tau, 1.0) * 2.0 ** -16)


def test_one_teacher_logit_is_a_label_bit_for_bit():
    a, b = cfg(2, 100, 128, 900, top_k=1), cfg(2, 100, 128, 900)
    inp = make_head_inputs(a, ignored=0.2)
    lab = {**inp, "targets": inp["top_ids"][..., 0]}
    ra, rb = HeadRunner(a), HeadRunner(b)
    ra.load_inputs(inp)
    rb.load_inputs(lab)
    ra.step()
    rb.step()
    for n in ("loss", "total", "dX", "dW"):
        assert np.array_equal(ra.fetch(n), rb.fetch(n)), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
def test_confident_and_large_logits(dtype, tied):
    """Losses far below the size of their logits, logits of thousands, probabilities that vanish: all finite, and exact to fp32 steps of
    the logits' distances.  Hidden states and weights are powers of two, whose products and sums are exact."""
    d, v, n = 64, 130, 48
    c = cfg(1, n, d, v, dtype, tied)
    inp = make_head_inputs(c)
    x, w, t = np.zeros((n, d)), np.zeros((d, v)), np.zeros(n, dtype=np.int32)
    for j in range(64):
        w[j, j] = 1.0
    for i in range(n):
        t[i] = i % 40
        x[i, t[i]] = 2.0 ** (i % 13)                # 1 .. 4096 above the rest, which are 0
        if i >= 39:
            x[i, 50] = 2.0 ** (i % 13)              # and a rival of the same size
    inp.update(X=x[None], W=w.T.copy() if tied else w, targets=t[None])
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    loss = run.fetch("loss")[:]
    want = ref["loss"][0]
    # bf16: logits are scaled up by 2.2e-8 + 1.6e-8 d / 16 against what the tensor core cuts off, which here is nothing
    shift = 1e-7 * np.abs(ref["Z"]).max(1) if dtype == "bf16" else 3e-7 * np.abs(ref["Z"]).max(1)
    assert (np.abs(loss - want) <= 2.0 ** -20 * want + shift * np.minimum(1.0, want) + 2.0 ** -22).all()
    assert np.isfinite(run.fetch("dX")).all() and np.isfinite(run.fetch("dW")).all()
    compare(c, inp, run, ref)


@pytest.mark.parametrize("kind", ["infinite", "overflow"])
@pytest.mark.parametrize("top_k", [0, 4])
@pytest.mark.parametrize("dtype,tile", [("bf16", t) for t in (None, "0", "1", "2", "3", "4")] + [("fp32", t) for t in ("64", "128")],
                         ids=lambda v: str(v))
def test_logits_of_minus_infinity(monkeypatch, dtype, tile, top_k, kind):
    """Columns whose logits are -inf, from weights of -inf or from products past the range of fp32, panels of 64 and tiles of 256 of them
    and single ones, are columns that are not there: everything else is what a vocabulary without them gives."""
    if tile:
        monkeypatch.setenv("FBL_HEAD_TILE" if dtype == "bf16" else "FBL_F32_BN", tile)
    v = 1100
    gone = np.zeros(v, dtype=bool)
    gone[:130] = gone[256:512] = gone[640:704] = True                    # the first panels of a row, too
    gone[[200, 530, 999, 1099]] = True
    kept = np.flatnonzero(~gone)
    for batch, seq in ((1, 20), (2, 150)):
        few = cfg(batch, seq, 128, len(kept), dtype, top_k=top_k)
        inp = make_head_inputs(few, ignored=0.2)
        inp["X"][..., 0], inp["W"][0] = (1.0 if kind == "infinite" else 2.0 ** 64), 0.0
        ref = orc.head_fwd_bwd(few, inp)
        c = cfg(batch, seq, 128, v, dtype, top_k=top_k)
        W = np.zeros((128, v))
        W[:, kept], W[0, gone] = inp["W"], -np.inf if kind == "infinite" else -2.0 ** 70
        names = "top_ids" if top_k else "targets"
        run = HeadRunner(c, guard_bytes=4096)
        run.load_inputs({**inp, "W": W, names: np.where(inp[names] < 0, -1, kept[np.maximum(inp[names], 0)]).astype(np.int32)})
        run.step()
        loss = run.fetch("loss").reshape(batch, seq)
        assert (np.abs(loss - ref["loss"]) <= loss_bound(few, inp, ref)).all() and (loss[~ref["has"]] == 0).all()
        # dX along the first column is 0 times -inf where there are such weights; dW along it has hidden states of 2^64
        n, dz, slack = batch * seq, ref["dZ"], dz_slack(few, inp, ref)
        x, w = inp["X"].reshape(n, -1).T[1:], inp["W"].T[:, 1:]
        dX, dW = run.fetch("dX").reshape(n, -1), run.fetch("dW")
        check_grad("dX", c, dX[:, 1:], ref["dX"].reshape(n, -1)[:, 1:], dz, w, c.vocab, slack @ np.abs(w))
        check_grad("dW", c, dW[1:, kept], ref["dW"][1:], x, dz, n, np.abs(x) @ slack)
        assert (dW[:, gone] == 0).all() and run.status() == 0 and run.guards_intact() == []


@pytest.mark.parametrize("top_k", [0, 5])
@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("tile", [None, "0", "1", "2", "3", "4"])
def test_few_tokens_gradients_are_off_by_their_own_rounding(monkeypatch, tile, tied, top_k):
    """Up to 64 padded rows dz comes in two parts, so that what is left in the norm is the results' rounding, at most half a step each and
    2^-8 / sqrt(3) in the rms, and what the error of p leaves (dz in one part: another rounding of every value, 2.3e-3 to 3.5e-3 in all)."""
    if tile:
        monkeypatch.setenv("FBL_HEAD_TILE", tile)
    for batch, seq, d, vocab in ((1, 1, 256, 700), (1, 64, 128, 515), (3, 13, 192, 2050), (8, 1, 320, 64)):
        c = cfg(batch, seq, d, vocab, "bf16", tied, top_k)
        run, inp = run_and_compare(c, ignored=0.2 if seq > 1 else 0.0, weighted=seq == 13)
        ref = orc.head_fwd_bwd(c, inp)
        s, n = dz_slack(c, inp, ref), batch * seq
        x, w = np.abs(inp["X"].reshape(n, -1)), np.abs(inp["W"].T if tied else inp["W"])
        for name, slack in (("dX", s @ w.T), ("dW", (s.T @ x) if tied else x.T @ s)):
            want = ref[name].reshape(-1)
            off = np.linalg.norm(run.fetch(name).reshape(-1) - want)
            assert off <= RMS * np.linalg.norm(want) + np.linalg.norm(slack), (name, batch, seq, off / np.linalg.norm(want))


@pytest.mark.parametrize("top_k", [0, 3])
@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
def test_few_tokens_targets_in_64_bits(tied, top_k):
    """Losses of few tokens take the products at their targets from sums in 64 bits.  A target's logit of 1024 and 4095 terms of 2^-17,
    which a sum of 24 bits that cuts its additions off loses in part (2^-5 in all, of which 16 columns lose up to 2^-13), beside a rival of
    1024 exactly: the loss, log(1 + 2^(-2^-5 log2 e)), would be off by up to 2^-6.  What is left is what logits are scaled up by against
    such cuts, (2.2e-8 + 1e-9 d) 1024 for the rival, which has none: 4.3e-3 of it at most.  (Gradients take the softmax from the sums that
    are cut off: p may be off by p (1 - p) 2^-6 here, as dz_slack has it, all tokens alike, which their norms' bound does not.)"""
    d, v, n = 4096, 70, 11
    c = cfg(1, n, d, v, "bf16", tied, top_k)
    inp = make_head_inputs(c)
    w, x = np.zeros((d, v)), np.full((1, n, d), 2.0 ** -9)
    w[0, 41] = w[0, 66] = x[..., 0] = 32.0
    w[1:, 66] = 2.0 ** -8
    inp.update(X=x, W=w.T.copy() if tied else w)
    if top_k:
        inp.update(top_ids=np.array([[[-1, 66, -1]] * n], dtype=np.int32), top_logits=np.ones((1, n, 3)))
    else:
        inp["targets"] = np.full((1, n), 66, dtype=np.int32)
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    assert (np.abs(run.fetch("loss") - ref["loss"]) <= 4.4e-3).all()
    assert run.guards_intact() == []


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("n,top_k,exact", [(16, 64, True), (17, 64, False), (8, 128, True), (9, 128, False), (64, 16, True), (61, 17, False)])
def test_several_targets_in_64_bits_and_where_that_ends(n, top_k, exact, tied):
    """As above, a teacher's list of targets that hold half of the probability together, and as many rivals of 1024 exactly: up to 1024 rows
    times entries the loss is off by what the rivals are scaled up by, (2.2e-8 + 1e-9 d) 1024 of half of it, beyond by half of the 2^-5 that
    the targets' sums may lose as well."""
    d, v = 4096, 2 * top_k + 3
    c = cfg(1, n, d, v, "bf16", tied, top_k)
    inp = make_head_inputs(c)
    w, x = np.zeros((d, v)), np.full((1, n, d), 2.0 ** -9)
    w[0, :2 * top_k] = x[..., 0] = 32.0
    w[1:, top_k:2 * top_k] = 2.0 ** -8
    inp.update(X=x, W=w.T.copy() if tied else w, top_ids=(top_k + np.array([np.random.default_rng(i).permutation(top_k) for i in range(n)])[None]).astype(np.int32))
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.forward()
    off = np.abs(run.fetch("loss") - ref["loss"][0])
    assert (off <= 4.4e-3 + (0.0 if exact else 2.0 ** -6)).all(), off.max()
    assert run.guards_intact() == []


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_backward_does_not_read_x(dtype):
    """dX may take X's place, and X may hold anything once the forward is done."""
    c = cfg(2, 150, 128, 900, dtype)
    inp = make_head_inputs(c, ignored=0.3)
    run = HeadRunner(c)
    run.load_inputs(inp)
    run.step()
    want = {k: run.fetch(k) for k in ("dX", "dW")}
    run.buf["X"].fill_(0xFF)
    run.buf["dX"] = run.buf["X"]
    run.backward()
    for k, v in want.items():
        assert np.array_equal(v, run.fetch(k)), k
    assert run.status() == 0


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
def test_fp32_operands_beyond_the_parts_range(monkeypatch, tied):
    """Hidden states of 2^100 and weights of 2^97, whose products and gradients leave the range that operands in parts have: their tiles
    are formed by multiply-adds, and the others are what they are without them."""
    monkeypatch.setenv("FBL_HEAD_PIECE", "512")
    c = cfg(2, 150, 128, 1339, "fp32", tied)
    inp = make_head_inputs(c, ignored=0.2)
    plain = HeadRunner(c)
    plain.load_inputs(inp)
    plain.step()
    big = dict(inp, X=inp["X"].copy(), W=inp["W"].copy())
    ref = orc.head_fwd_bwd(c, inp)
    rows = np.argwhere(ref["has"])[[3, 170]]
    for b, t in rows:
        big["X"][b, t] *= 2.0 ** 100
    ref = orc.head_fwd_bwd(c, big)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(big)
    run.step()
    assert run.status() == 0 and run.guards_intact() == []
    loss, want = run.fetch("loss").reshape(2, 150), ref["loss"]
    assert np.isfinite(loss).all() and (np.abs(loss - want) <= 1e-5 * np.abs(want) + 1e-5).all()
    dX = run.fetch("dX")
    assert np.isfinite(dX).all() and fp32_err(dX, ref["dX"]) <= 1e-5
    # dW is sums of 2^100 dz of those tokens: to fp32 steps of its terms
    x = np.abs(big["X"].reshape(300, -1))
    terms = x.T @ np.abs(ref["dZ"])
    dW = run.fetch("dW")
    assert (np.abs(dW - ref["dW"]) <= 1e-5 * (terms.T if tied else terms) + 1e-30).all()
    # the other tokens' losses and gradients have not moved
    same = np.ones((2, 150), dtype=bool)
    same[rows[:, 0], rows[:, 1]] = False
    assert np.abs(loss - plain.fetch("loss").reshape(2, 150))[same].max() <= 1e-5
    assert fp32_err(dX[same], plain.fetch("dX")[same]) <= 1e-5


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("batch,seq,share", [(4, 197, 1.0), (1, 333, 1.0), (6, 61, 0.5), (3, 20, 1.0)], ids=str)
@pytest.mark.parametrize("top_k,tau", [(0, 1.0), (1, 3.0)], ids=["labels", "teacher"])
def test_equal_weights_leave_no_common_factor(batch, seq, share, top_k, tau, tied):
    """1 / n given as every token's weight, or every other one's and 0 for the rest: dX and dW are those of the mean, no factor larger or
    smaller.  A target's entry of dz is 1 - p of its weight, which comes out as the weight where p is below 2^-9: off by p.  Beside it stand 6000
    entries of some p, rounded independently (RMS p sqrt(6000) < 1e-4 of it) and the results' roundings, RMS / sqrt(n d) < 5e-5.
    (1/788, 1/333, 1/366 and 1/1098 in bf16 are 2.0e-3 to 6e-4 off.)"""
    c = cfg(batch, seq, 64, 6000, "bf16", tied, top_k, tau, w_std=0.02)
    inp = make_head_inputs(c)
    n = batch * seq
    if top_k:
        inp["top_ids"] = np.maximum(inp["top_ids"], 0)
    else:
        inp["targets"] = np.maximum(inp["targets"], 0)
    on = (np.arange(n) % 2 == 0).reshape(batch, seq) if share < 1 else np.ones((batch, seq), dtype=bool)
    inp["dloss"] = np.where(on, 1.0 / n, 0.0).astype(np.float32).astype(np.float64)
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    got = {k: run.fetch(k) for k in ("dX", "dW")}
    y, _ = orc.targets(c, inp)
    p = np.exp(ref["Z"] - ref["lse"][:, None])[y > 0]
    for k, v in got.items():
        factor = (v * ref[k]).sum() / (ref[k] ** 2).sum()
        assert abs(factor - 1) <= p.max() + 1.5e-4, (k, factor - 1)
    if share == 1:
        # against the mean's path: weights a step of fp32 apart change a rounding, one bf16 step of at most 2^-7, in less than one of 2^13
        # elements of dz and of the results (few rows, in two parts: the results')
        run.load_inputs({**inp, "dloss": None})
        run.step()
        for k, v in got.items():
            mean = run.fetch(k)
            assert np.linalg.norm(v - mean) <= 2.5e-4 * np.linalg.norm(mean), (k, np.linalg.norm(v - mean) / np.linalg.norm(mean))
    assert run.status() == 0 and run.guards_intact() == []


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [1e-30, 1e36, 0.0])
def test_weights_of_any_size(size, dtype):
    """Weights at the ends of fp32's range, and what tokens without a loss have for one, which is not looked at; a weight of NaN is its
    token's alone."""
    c = cfg(3, 45, 128, 700, dtype, w_std=0.02)
    inp = make_head_inputs(c, ignored=0.4, weighted=True)
    inp["dloss"] = (inp["dloss"] * size).astype(np.float32).astype(np.float64)
    ref = orc.head_fwd_bwd(c, inp)
    run = HeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    assert np.isfinite(run.fetch("dX")).all() and np.isfinite(run.fetch("dW")).all()
    if size:
        scaled = {**ref, "dX": ref["dX"] / size, "dW": ref["dW"] / size}
        for k in ("dX", "dW"):
            off = np.linalg.norm(run.fetch(k) / size - scaled[k]) / np.linalg.norm(scaled[k])
            assert off <= (2 * RMS if dtype == "bf16" else 1e-5), (k, off)
    else:
        assert (run.fetch("dX") == 0).all() and (run.fetch("dW") == 0).all()
    want = {k: run.fetch(k) for k in ("loss", "dX", "dW")}
    has = ref["has"].reshape(-1)
    for junk in (np.inf, np.nan, -3e38):
        run.load_inputs({**inp, "dloss": np.where(ref["has"], inp["dloss"], junk)})
        run.step()
        for k, v in want.items():
            assert np.array_equal(v, run.fetch(k)), (k, junk)
    bad = inp["dloss"].copy()
    bad.reshape(-1)[np.flatnonzero(has)[5]] = np.nan
    run.load_inputs({**inp, "dloss": bad})
    run.step()
    dX, same = run.fetch("dX").reshape(135, -1), np.arange(135) != np.flatnonzero(has)[5]
    assert np.isnan(dX[~same]).all() and np.isfinite(dX[same]).all() and np.isnan(run.fetch("dW")).all()
    assert run.guards_intact() == [] and run.status() == 0


@pytest.mark.parametrize("top_k", [0, 3])
def test_total_is_the_losses_sum_rounded_once(top_k):
    """Every eight rows are one block's, and here all alike, so that what a block's sum loses every block's loses: the total is the losses
    added up in 64 bits, to half a step of fp32."""
    for batch in (9, 11, 13, 25, 41, 63, 299):
        c = cfg(batch, 8, 64, 500, "bf16", top_k=top_k, seed=batch)
        inp = make_head_inputs(c)
        for k in ("X",) + (("top_ids", "top_logits") if top_k else ("targets",)):
            inp[k] = np.repeat(inp[k][:1], batch, axis=0)
        run = HeadRunner(c, guard_bytes=4096)
        run.load_inputs(inp)
        run.forward()
        loss, total = run.fetch("loss"), run.fetch("total")
        assert total[1] == batch * 8
        assert abs(total[0] - loss.sum()) <= 2.0 ** -24 * (1 + 1e-6) * loss.sum(), (batch, total[0] / loss.sum() - 1)
        assert run.guards_intact() == []


def test_bits_repeat_on_dirty_work_areas():
    for c in (cfg(2, 300, 256, 5003, tied=True), cfg(4, 77, 128, 1500, top_k=32, tau=2.0), cfg(2, 150, 128, 1500, "fp32")):
        inp = make_head_inputs(c, ignored=0.3)
        run = HeadRunner(c)
        run.load_inputs(inp)
        run.step()
        names = ("loss", "total", "dX", "dW")
        first = {n: run.fetch(n) for n in names}
        for fill in (0xFF, 0x7F, 0x00):
            for b in (run.saved, run.scratch_fwd, run.scratch, run.buf["dX"], run.buf["dW"]):
                b.fill_(fill)
            for _ in range(5):
                run.step()
            assert run.status() == 0
            for n in names:
                assert np.array_equal(first[n], run.fetch(n)), (c.name, n, hex(fill))


def test_a_backward_may_follow_again_and_fewer_tokens_after_more():
    c = cfg(2, 140, 128, 900)
    run = HeadRunner(c, guard_bytes=4096)
    for ignored in (0.0, 0.9, 0.5):                 # rows left by a call with more tokens lie behind those of the next
        inp = make_head_inputs(c, ignored=ignored)
        run.load_inputs(inp)
        run.forward()
        run.backward()
        run.buf["dX"].fill_(0x11)
        run.backward()
        compare(c, inp, run)


def test_a_runner_whose_buffers_are_filled_in_place():
    """Without load_inputs, as behind a layer that writes X: the mean's gradient."""
    import torch
    c = cfg(2, 40, 128, 900)
    inp = make_head_inputs(c, ignored=0.3)
    a, b = HeadRunner(c, guard_bytes=4096), HeadRunner(c, guard_bytes=4096)
    a.load_inputs(inp)
    for n in ("X", "W"):
        b.buf[n].copy_(a.buf[n])
    b.vec["targets"].copy_(a.vec["targets"])
    torch.cuda.synchronize()
    b.step()
    compare(c, inp, b)


def test_padding_of_outputs_is_zero():
    import torch
    for dtype in ("bf16", "fp32"):
        for tied in (False, True):
            c = cfg(3, 13, 128, 203, dtype, tied)
            run = HeadRunner(c)
            inp = make_head_inputs(c)
            run.load_inputs(inp)
            run.buf["dX"].fill_(0x33)
            run.buf["dW"].fill_(0x33)
            run.step()
            torch.cuda.synchronize()
            tw = 32 if dtype == "fp32" else 64
            dx = run.buf["dX"].view(run.tdtype).view(128 // tw, 3, 16, tw)
            assert bool((dx[:, :, 13:] == 0).all())
            dw = run.buf["dW"].view(run.tdtype)
            if tied:
                assert bool((dw.view(128 // tw, 208, tw)[:, 203:] == 0).all())
            else:
                assert bool((dw.view(-1, 128, tw)[-1, :, 203 % tw:] == 0).all())


def test_other_streams_and_captured_replays():
    """Two heads on two streams at once, each with its own work areas; and a captured step, replayed on new inputs."""
    import torch
    a, b = cfg(2, 200, 128, 3001, tied=True), cfg(1, 333, 192, 2049, top_k=16, tau=2.0)
    ia, ib = make_head_inputs(a, ignored=0.3), make_head_inputs(b)
    ra, rb = HeadRunner(a, guard_bytes=4096), HeadRunner(b, guard_bytes=4096)
    ra.load_inputs(ia)
    rb.load_inputs(ib)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(sa):
            ra.step()
        with torch.cuda.stream(sb):
            rb.step()
    torch.cuda.synchronize()
    compare(a, ia, ra)
    compare(b, ib, rb)
    graphs = []
    for run, st in ((ra, sa), (rb, sb)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            run.step()
        graphs.append(g)
    ia2, ib2 = make_head_inputs(HeadConfig(**{**a.__dict__, "seed": 11}), ignored=0.7), make_head_inputs(HeadConfig(**{**b.__dict__, "seed": 12}), ignored=0.4)
    ra.load_inputs(ia2)
    rb.load_inputs(ib2)
    for g, st in zip(graphs, (sa, sb)):
        with torch.cuda.stream(st):
            g.replay()
    torch.cuda.synchronize()
    compare(a, ia2, ra)
    compare(b, ib2, rb)


def test_wide_and_long():
    run_and_compare(cfg(1, 2100, 512, 4097, tied=True, w_std=0.04), ignored=0.1)
    run_and_compare(cfg(1, 300, 4096, 1030, w_std=0.02))
    run_and_compare(cfg(40, 3, 16384, 70, w_std=0.01, tied=True))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape,top_k", [((5, 8000, 64, 300), 0), ((11, 3333, 64, 130), 3), ((9, 8001, 64, 70), 0)],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_more_rows_than_a_block_brings_together_at_once(shape, top_k, dtype):
    """From 32768 padded rows on a block has 64 of them and more, 32 at a time, across the ends of sequences."""
    run_and_compare(cfg(*shape, dtype, tied=top_k > 0, top_k=top_k), ignored=0.3)


@pytest.mark.parametrize("tied", [False, True], ids=["dv", "vd"])
@pytest.mark.parametrize("tile", [None, "0", "1"])
def test_pairs_in_bands_of_rows(monkeypatch, tile, tied):
    """More than 4096 rows with a loss: a pair's tiles go in bands of eight row tiles, the last of them shorter; and fewer of them than that
    in a launch made for more."""
    monkeypatch.setenv("FBL_GEMM_PAIR", "1")
    if tile:
        monkeypatch.setenv("FBL_HEAD_TILE", tile)
    for seq, ignored in ((4098, 0.0), (5200, 0.1), (5200, 0.5)):
        run_and_compare(cfg(1, seq, 128, 1030, tied=tied), ignored=ignored)


def test_weights_beyond_32_bit_offsets():
    """A head of 2.4e9 weights, labels at its end; the plain form on the GPU stands in for the oracle's time."""
    import torch
    d, v, n = 16384, 147457, 5
    plan = HeadPlan(head_desc(1, n, d, v, "bf16", tied=True))
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn((v, d), generator=gen, device="cuda", dtype=torch.bfloat16).mul_(0.01)
    x = torch.randn((n, d), generator=gen, device="cuda", dtype=torch.bfloat16)
    t = torch.tensor([v - 1, 0, v - 2, 131072, 5], dtype=torch.int32, device="cuda")
    X, W, dX, dW = [aligned_bytes(torch, plan.tensor_bytes(i), "cuda") for i in (0, 1, 0, 1)]
    sv, sf, sb = [aligned_bytes(torch, k, "cuda") for k in plan.workspace_bytes()]
    st = torch.cuda.current_stream().cuda_stream
    plan.pack(0, x.data_ptr(), X.data_ptr(), st)
    plan.pack(1, w.data_ptr(), W.data_ptr(), st)
    loss, total = torch.empty(n, device="cuda"), torch.empty(2, device="cuda")
    plan.xent_fwd(X.data_ptr(), W.data_ptr(), t.data_ptr(), loss.data_ptr(), total.data_ptr(), sv.data_ptr(), sf.data_ptr(), st)
    plan.bwd(X.data_ptr(), W.data_ptr(), None, sv.data_ptr(), dX.data_ptr(), dW.data_ptr(), sb.data_ptr(), st)
    z = torch.cat([x.double() @ part.double().t() for part in w.split(16384)], 1)
    lse = torch.logsumexp(z, 1)
    want = lse - z.gather(1, t.long()[:, None])[:, 0]
    # logits of some 1.3 x 10, off by up to 2 (d / 16) 2^-23 of sum |x w| = 104 at the very most; a hundredth of it as they come
    assert float((loss.double() - want).abs().max()) <= 2 * (d / 16 + 2) * 2.0 ** -23 * 140 + 1e-5
    dz = torch.exp(z - lse[:, None])
    dz[torch.arange(n), t.long()] -= 1
    dz /= n
    got = torch.empty_like(x)
    plan.unpack(0, dX.data_ptr(), got.data_ptr(), st)
    ref = sum(dz[:, i:i + 16384] @ w[i:i + 16384].double() for i in range(0, v, 16384))
    assert float((got.double() - ref).norm() / ref.norm()) <= 2 * RMS
    rows = dW.view(torch.bfloat16).view(d // 64, (v + 7) // 8 * 8, 64)
    for j in (0, 5, 131072, v - 2, v - 1, 100000):
        ref = (dz[:, j:j + 1].t() @ x.double())[0]
        assert float((rows[:, j].reshape(-1).double() - ref).norm() / ref.norm()) <= 2 * RMS, j
    assert bool((rows[:, v:] == 0).all())


# ---- the norm, and both together ------------------------------------------------------------------------------------

@pytest.mark.parametrize("norm", ["layernorm", "rmsnorm"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1, 64), (1, 1, 768), (3, 5, 128), (2, 197, 320), (7, 13, 1088), (1, 600, 2048), (2, 9, 16384), (3, 399, 448),
                                   (1, 1190, 1280), (2, 595, 960), (1, 1184, 2048), (1, 3561, 4096), (2, 1777, 3584)],
                         ids=lambda s: "x".join(map(str, s)))
def test_norm(shape, dtype, norm):
    c = cfg(*shape, 8, dtype, norm=norm)
    inp = make_head_inputs(c)
    inp["X"] = inp["X"] * 2.0 + 1.0 if dtype == "fp32" else inp["X"]
    inp["X"] = inp["X"].astype(np.float32).astype(np.float64)
    rng = np.random.default_rng(1)
    inp["dY"] = rng.normal(size=inp["X"].shape).astype(np.float32)
    inp["dY"] = (inp["dY"].view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)      # bf16 values
    run = NormRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    d = c.d_model
    Y, xhat, rstd, _ = orc.norm_fwd(inp["X"], inp["gamma"], inp["beta"], c.eps, norm)
    g = inp["dY"] * inp["gamma"]
    dX = g - xhat * (g * xhat).mean(-1, keepdims=True) - (g.mean(-1, keepdims=True) if norm == "layernorm" else 0.0)
    ref = {"Y": Y, "dX": dX * rstd, "dgamma": (inp["dY"] * xhat).reshape(-1, d).sum(0)}
    mags = {"Y": np.abs(Y), "dX": np.abs(g) * rstd, "dgamma": np.abs(inp["dY"] * xhat).reshape(-1, d).sum(0)}
    if norm == "layernorm":
        ref["dbeta"] = inp["dY"].reshape(-1, d).sum(0)
        mags["dbeta"] = np.abs(inp["dY"]).reshape(-1, d).sum(0)
    for name, want in ref.items():
        got = run.fetch(name)
        # fp32 steps of row sums (mean and variance of up to 16384 columns in trees and runs of 64) and of sums over tokens; the result's
        # rounding where it is bf16
        room = 2.0 ** -24 * 64 * (mags[name] + np.sqrt(np.mean(want ** 2)) + 1.0 / np.sqrt(d)) + (U * np.abs(want) if dtype == "bf16" and name in ("Y", "dX") else 0.0)
        assert (np.abs(got - want) <= room).all(), (name, float((np.abs(got - want) - room).max()))
    assert run.guards_intact() == []
    # frozen: the same dX, the vectors left alone
    keep = run.fetch("dX")
    run.vec["dgamma"].fill_(7.0)
    run.backward(frozen=True)
    assert np.array_equal(keep, run.fetch("dX")) and (run.fetch("dgamma") == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1, 64), (3, 5, 1088), (2, 1777, 3584), (1, 1665, 1280)], ids=lambda s: "x".join(map(str, s)))
def test_norms_forward_leaves_its_scratch_alone(shape, dtype):
    """Nobody reads a status there, and a store may land while the launch in front still uses that memory."""
    c = cfg(*shape, 8, dtype)
    inp = make_head_inputs(c)
    run = NormRunner(c)
    run.load_inputs({**inp, "dY": inp["X"]})
    for b in (run.scratch_fwd, run.scratch):
        b.fill_(0xC3)
    run.forward()
    run.torch.cuda.synchronize()
    assert bool((run.scratch_fwd == 0xC3).all()) and bool((run.scratch == 0xC3).all())
    run.backward()
    run.torch.cuda.synchronize()
    assert bool((run.scratch[:1024] == 0xC3).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top_k,tied", [(0, True), (8, False)])
def test_norm_and_head_together(dtype, top_k, tied):
    """The end of a step as it runs: norm, head, back through both.  What the norm's backward is given is the head's own dX, so its
    results are held against the formula on that."""
    c = cfg(3, 77, 192, 1201, dtype, tied, top_k, 2.0 if top_k else 1.0, norm="rmsnorm" if top_k else "layernorm")
    inp = make_head_inputs(c, ignored=0.3)
    run = NormHeadRunner(c, guard_bytes=4096)
    run.load_inputs(inp)
    run.step()
    Y, xhat, _, _ = orc.norm_fwd(inp["X"], inp["gamma"], inp["beta"], c.eps, c.norm)
    got_y = run.fetch("Y")
    # xhat gamma + beta may cancel: fp32 steps of its terms (sixteen: mean, variance, rstd, two products), then the result's rounding
    terms = np.abs(xhat * inp["gamma"]) + (0.0 if inp["beta"] is None else np.abs(inp["beta"])) + 1.0 / np.sqrt(192)
    assert (np.abs(got_y - Y) <= (U if dtype == "bf16" else 0.0) * np.abs(Y) + 16 * 2.0 ** -24 * terms).all()
    mid = dict(inp, X=got_y)
    ref = orc.head_fwd_bwd(c, mid)
    n = c.batch * c.seq
    assert (np.abs(run.fetch("loss").reshape(3, 77) - ref["loss"]) <= loss_bound(c, mid, ref)).all()
    w = inp["W"].T if tied else inp["W"]
    dY = run.fetch("dY")
    slack = dz_slack(c, mid, ref)
    check_grad("dY", c, dY.reshape(n, -1), ref["dX"].reshape(n, -1), ref["dZ"], w.T, c.vocab, slack @ np.abs(w.T))
    dW = run.fetch("dW")
    check_grad("dW", c, dW.T if tied else dW, ref["dW"].T if tied else ref["dW"], got_y.reshape(n, -1).T, ref["dZ"], n, np.abs(got_y.reshape(n, -1).T) @ slack)
    dX, dg, db = orc.norm_bwd(dY, inp["X"], inp["gamma"], c.eps, c.norm)
    scale = np.sqrt(np.mean(dX ** 2))
    assert (np.abs(run.fetch("dX") - dX) <= (U if dtype == "bf16" else 0.0) * np.abs(dX) + 1e-5 * scale).all()
    assert fp32_err(run.fetch("dgamma"), dg) <= 1e-5
    if db is not None:
        assert fp32_err(run.fetch("dbeta"), db) <= 1e-5
    assert run.status() == 0 and run.guards_intact() == []
