"""ctypes binding of the fine-tuning step's head (fbl_head_*): logits over the vocabulary and their cross entropy with labels
or with a teacher's top logits, and runners that own the device buffers."""
from __future__ import annotations

import ctypes as C

from .binding import DTYPES, FblError, _check, aligned_bytes, guard_bands_intact, lib, raw_stream
from .norm import NormRunner

HEAD_TENSOR = {"X": 0, "W": 1}


class FblHeadDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "seq", "d_model", "vocab", "dtype", "vocab_rows", "top_k")] + [("temperature", C.c_float)]


_bound = False


def _bind():
    global _bound
    L = lib()
    if _bound:
        return L
    vp, psz = C.c_void_p, C.POINTER(C.c_size_t)
    L.fbl_head_plan_create.argtypes = [C.POINTER(FblHeadDesc), C.POINTER(vp)]
    L.fbl_head_plan_destroy.argtypes = [vp]
    L.fbl_head_plan_destroy.restype = None
    L.fbl_head_tensor_bytes.argtypes = [vp, C.c_int, psz]
    L.fbl_head_workspace_bytes.argtypes = [vp, psz, psz, psz]
    L.fbl_head_pack.argtypes = [vp, C.c_int, vp, vp, vp]
    L.fbl_head_unpack.argtypes = [vp, C.c_int, vp, vp, vp]
    L.fbl_head_xent_fwd.argtypes = [vp] * 9
    L.fbl_head_distill_fwd.argtypes = [vp] * 10
    L.fbl_head_bwd.argtypes = [vp] * 9
    L.fbl_head_status_poll.argtypes = [vp, vp, C.POINTER(C.c_int32)]
    L.fbl_head_launch_count.argtypes = [vp]
    L.fbl_head_launch_count.restype = C.c_int64
    _bound = True
    return L


def head_desc(batch, seq, d_model, vocab, dtype="bf16", tied=False, top_k=0, temperature=1.0) -> FblHeadDesc:
    """``tied``: W is stored as [vocab, d_model], as an embedding is; else [d_model, vocab].  ``top_k`` 0: labels."""
    return FblHeadDesc(batch, seq, d_model, vocab, DTYPES[dtype], int(tied), top_k, temperature)


class HeadPlan:
    """One fbl_head_plan; methods carry the C entry points' names without the ``fbl_head_`` prefix."""

    def __init__(self, desc: FblHeadDesc):
        self._h = C.c_void_p()
        self.desc = desc
        L = _bind()
        _check(L.fbl_head_plan_create(C.byref(desc), C.byref(self._h)))
        # looked up once: a call of a few tokens is host work
        self._xent_fwd, self._distill_fwd, self._bwd = L.fbl_head_xent_fwd, L.fbl_head_distill_fwd, L.fbl_head_bwd

    def close(self):
        if self._h:
            lib().fbl_head_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def tensor_bytes(self, matrix_id) -> int:
        out = C.c_size_t()
        _check(lib().fbl_head_tensor_bytes(self._h, matrix_id, C.byref(out)))
        return out.value

    def workspace_bytes(self):
        a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
        _check(lib().fbl_head_workspace_bytes(self._h, C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def pack(self, matrix_id, rowmajor_ptr, tiled_ptr, stream):
        _check(lib().fbl_head_pack(self._h, matrix_id, rowmajor_ptr, tiled_ptr, stream))

    def unpack(self, matrix_id, tiled_ptr, rowmajor_ptr, stream):
        _check(lib().fbl_head_unpack(self._h, matrix_id, tiled_ptr, rowmajor_ptr, stream))

    def xent_fwd(self, X, W, targets, loss, total, saved, scratch, stream):
        code = self._xent_fwd(self._h, X, W, targets, loss, total, saved, scratch, stream)
        if code:
            _check(code)

    def distill_fwd(self, X, W, top_ids, top_logits, loss, total, saved, scratch, stream):
        code = self._distill_fwd(self._h, X, W, top_ids, top_logits, loss, total, saved, scratch, stream)
        if code:
            _check(code)

    def bwd(self, X, W, dloss, saved, dX, dW, scratch, stream):
        """dloss None: the gradient of the mean loss.  dX or dW None: not formed."""
        code = self._bwd(self._h, X, W, dloss, saved, dX, dW, scratch, stream)
        if code:
            _check(code)

    def status_poll(self, scratch) -> int:
        out = C.c_int32()
        code = lib().fbl_head_status_poll(self._h, scratch, C.byref(out))
        if code not in (0, -6):
            _check(code)
        return out.value

    def launch_count(self) -> int:
        return lib().fbl_head_launch_count(self._h)


class HeadRunner:
    """Device buffers for one head plus pack / forward / backward / unpack helpers (torch for memory and streams only).
    ``cfg`` has batch, seq, d_model, vocab, dtype, tied, top_k and temperature.  ``X`` and ``dX``: buffers to use in place of
    its own (the norm's output and its gradient).  ``frozen``: no dW."""

    def __init__(self, cfg, device="cuda:0", guard_bytes=0, X=None, dX=None, frozen=False):
        import torch
        if not torch.cuda.is_available():
            raise FblError(-101, "no CUDA device: the head has no CPU path")
        self.torch, self.cfg, self.dev = torch, cfg, torch.device(device)
        self.weighted = False           # load_inputs: whether there are weights of losses
        self.plan = HeadPlan(head_desc(cfg.batch, cfg.seq, cfg.d_model, cfg.vocab, cfg.dtype, cfg.tied, cfg.top_k, cfg.temperature))
        self.tdtype = torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
        al = lambda n: aligned_bytes(torch, n, self.dev, guard=guard_bytes)
        self.saved, self.scratch_fwd, self.scratch = map(al, self.plan.workspace_bytes())
        self._own = {n: al(self.plan.tensor_bytes(HEAD_TENSOR[n[-1]])) for n in ("X", "W", "dX", "dW")
                     if not (n == "X" and X is not None) and not (n == "dX" and dX is not None) and not (n == "dW" and frozen)}
        self.buf = {**self._own, **({} if X is None else {"X": X}), **({} if dX is None else {"dX": dX})}
        n = cfg.batch * cfg.seq
        lens = {"loss": n, "total": 2, "dloss": n}
        lens.update({"top_ids": n * cfg.top_k, "top_logits": n * cfg.top_k} if cfg.top_k else {"targets": n})
        self._vec_raw = {k: al(4 * v) for k, v in lens.items()}
        self.vec = {k: v.view(torch.int32 if k in ("targets", "top_ids") else torch.float32) for k, v in self._vec_raw.items()}

    def load_inputs(self, inp):
        """Row-major float arrays X [batch, seq, d_model] (if present) and W ([vocab, d_model] if tied, else [d_model, vocab]);
        targets [batch, seq], or top_ids and top_logits [batch, seq, top_k]; dloss [batch, seq] (optional)."""
        torch = self.torch
        for n in ("X", "W"):
            if inp.get(n) is not None:
                rm = torch.from_numpy(inp[n].astype("float32")).to(self.dev).to(self.tdtype).contiguous()
                self.plan.pack(HEAD_TENSOR[n], rm.data_ptr(), self.buf[n].data_ptr(), raw_stream(torch, self.dev))
        for n, kind in (("targets", "int32"), ("top_ids", "int32"), ("top_logits", "float32"), ("dloss", "float32")):
            if n in self.vec and inp.get(n) is not None:
                self.vec[n].copy_(torch.from_numpy(inp[n].astype(kind).reshape(-1)))
        self.weighted = inp.get("dloss") is not None
        torch.cuda.synchronize(self.dev)

    def forward(self):
        p = lambda t: t.data_ptr()
        b, v, st = self.buf, self.vec, raw_stream(self.torch, self.dev)
        rest = (p(v["loss"]), p(v["total"]), p(self.saved), p(self.scratch_fwd), st)
        if self.cfg.top_k:
            self.plan.distill_fwd(p(b["X"]), p(b["W"]), p(v["top_ids"]), p(v["top_logits"]), *rest)
        else:
            self.plan.xent_fwd(p(b["X"]), p(b["W"]), p(v["targets"]), *rest)

    def backward(self, dx=True, dw=True):
        b = self.buf
        self.plan.bwd(b["X"].data_ptr(), b["W"].data_ptr(), self.vec["dloss"].data_ptr() if self.weighted else None,
                      self.saved.data_ptr(), b["dX"].data_ptr() if dx else None,
                      b["dW"].data_ptr() if dw and "dW" in b else None, self.scratch.data_ptr(), raw_stream(self.torch, self.dev))

    def step(self):
        self.forward()
        self.backward()

    def fetch(self, name):
        """A matrix (row-major) or a vector as a float64 numpy array."""
        torch, c = self.torch, self.cfg
        if name in self.vec:
            torch.cuda.synchronize(self.dev)
            return self.vec[name].cpu().numpy().astype("float64")
        shape = (c.batch, c.seq, c.d_model) if name[-1] == "X" else (c.vocab, c.d_model) if c.tied else (c.d_model, c.vocab)
        out = torch.empty(shape, dtype=self.tdtype, device=self.dev)
        self.plan.unpack(HEAD_TENSOR[name[-1]], self.buf[name].data_ptr(), out.data_ptr(), raw_stream(torch, self.dev))
        torch.cuda.synchronize(self.dev)
        return out.float().cpu().numpy().astype("float64")

    def guards_intact(self):
        self.torch.cuda.synchronize(self.dev)
        named = {"saved": self.saved, "scratch_fwd": self.scratch_fwd, "scratch_bwd": self.scratch, **self._own, **self._vec_raw}
        return [k for k, v in named.items() if not guard_bands_intact(v)]

    def status(self) -> int:
        """Device status of the last forward and backward (0, or the code of the first bounded wait that expired)."""
        self.torch.cuda.synchronize(self.dev)
        fwd = self.plan.status_poll(self.scratch_fwd.data_ptr())
        return fwd if fwd != 0 else self.plan.status_poll(self.scratch.data_ptr())


class NormHeadRunner:
    """The end of a model as a step runs it: the final norm, the head behind it, and back through both.  ``cfg`` has the
    fields of both runners."""

    def __init__(self, cfg, device="cuda:0", guard_bytes=0, frozen=False):
        self.norm = NormRunner(cfg, device, guard_bytes)
        self.head = HeadRunner(cfg, device, guard_bytes, X=self.norm.buf["Y"], dX=self.norm.buf["dY"], frozen=frozen)

    def load_inputs(self, inp):
        import numpy as np
        c = self.norm.cfg
        self.norm.load_inputs({**inp, "dY": np.zeros((c.batch, c.seq, c.d_model))})
        self.head.load_inputs({k: v for k, v in inp.items() if k != "X"})

    def step(self):
        self.norm.forward()
        self.head.step()
        self.norm.backward()

    def fetch(self, name):
        """X, Y, dX, dgamma, dbeta of the norm; loss, total, W, dW of the head; dY: the gradient between them."""
        return (self.head if name in self.head.vec or name[-1] == "W" else self.norm).fetch(name)

    def guards_intact(self):
        return self.norm.guards_intact() + self.head.guards_intact()

    def status(self) -> int:
        return self.head.status()
