"""ctypes binding of the norm as an operator of its own (fbl_norm_*), and a runner that owns its device buffers."""
from __future__ import annotations

import ctypes as C

from .binding import DTYPES, NORMS, FblError, _check, aligned_bytes, guard_bands_intact, lib, raw_stream


class FblNormDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "seq", "d_model", "dtype", "norm")] + [("eps", C.c_float)]


_bound = False


def _bind():
    global _bound
    L = lib()
    if _bound:
        return L
    vp, psz = C.c_void_p, C.POINTER(C.c_size_t)
    L.fbl_norm_plan_create.argtypes = [C.POINTER(FblNormDesc), C.POINTER(vp)]
    L.fbl_norm_plan_destroy.argtypes = [vp]
    L.fbl_norm_plan_destroy.restype = None
    L.fbl_norm_tensor_bytes.argtypes = [vp, psz]
    L.fbl_norm_workspace_bytes.argtypes = [vp, psz, psz, psz]
    L.fbl_norm_pack.argtypes = [vp, vp, vp, vp]
    L.fbl_norm_unpack.argtypes = [vp, vp, vp, vp]
    L.fbl_norm_fwd.argtypes = [vp] * 8
    L.fbl_norm_bwd.argtypes = [vp] * 10
    L.fbl_norm_launch_count.argtypes = [vp]
    L.fbl_norm_launch_count.restype = C.c_int64
    _bound = True
    return L


def norm_desc(batch, seq, d_model, dtype="bf16", norm="layernorm", eps=1e-5) -> FblNormDesc:
    return FblNormDesc(batch, seq, d_model, DTYPES[dtype], NORMS[norm], eps)


class NormPlan:
    """One fbl_norm_plan; methods carry the C entry points' names without the ``fbl_norm_`` prefix."""

    def __init__(self, desc: FblNormDesc):
        self._h = C.c_void_p()
        self.desc = desc
        L = _bind()
        _check(L.fbl_norm_plan_create(C.byref(desc), C.byref(self._h)))
        # looked up once: a call of a few tokens is host work
        self._fwd, self._bwd = L.fbl_norm_fwd, L.fbl_norm_bwd

    def close(self):
        if self._h:
            lib().fbl_norm_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def tensor_bytes(self) -> int:
        out = C.c_size_t()
        _check(lib().fbl_norm_tensor_bytes(self._h, C.byref(out)))
        return out.value

    def workspace_bytes(self):
        a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
        _check(lib().fbl_norm_workspace_bytes(self._h, C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def pack(self, rowmajor_ptr, tiled_ptr, stream):
        _check(lib().fbl_norm_pack(self._h, rowmajor_ptr, tiled_ptr, stream))

    def unpack(self, tiled_ptr, rowmajor_ptr, stream):
        _check(lib().fbl_norm_unpack(self._h, tiled_ptr, rowmajor_ptr, stream))

    def fwd(self, X, gamma, beta, Y, saved, scratch, stream):
        code = self._fwd(self._h, X, gamma, beta, Y, saved, scratch, stream)
        if code:
            _check(code)

    def bwd(self, dY, X, gamma, saved, dX, dgamma, dbeta, scratch, stream):
        """dgamma and dbeta None: the norm's parameters are frozen."""
        code = self._bwd(self._h, dY, X, gamma, saved, dX, dgamma, dbeta, scratch, stream)
        if code:
            _check(code)

    def launch_count(self) -> int:
        return lib().fbl_norm_launch_count(self._h)


class NormRunner:
    """Device buffers for one norm plus pack / forward / backward / unpack helpers (torch for memory and streams only).
    ``cfg`` has batch, seq, d_model, dtype, norm and eps."""

    def __init__(self, cfg, device="cuda:0", guard_bytes=0):
        import torch
        if not torch.cuda.is_available():
            raise FblError(-101, "no CUDA device: the norm has no CPU path")
        self.torch, self.cfg, self.dev = torch, cfg, torch.device(device)
        self.plan = NormPlan(norm_desc(cfg.batch, cfg.seq, cfg.d_model, cfg.dtype, cfg.norm, cfg.eps))
        self.tdtype = torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
        al = lambda n: aligned_bytes(torch, n, self.dev, guard=guard_bytes)
        self.saved, self.scratch_fwd, self.scratch = map(al, self.plan.workspace_bytes())
        self.buf = {n: al(self.plan.tensor_bytes()) for n in ("X", "Y", "dY", "dX")}
        self._vec_raw = {n: al(4 * cfg.d_model) for n in ("gamma", "beta", "dgamma", "dbeta")}
        self.vec = {n: v.view(torch.float32) for n, v in self._vec_raw.items()}

    def load_inputs(self, inp):
        """Row-major float arrays X, dY [batch, seq, d_model], gamma and (LayerNorm) beta [d_model]."""
        for n in ("X", "dY"):
            rm = self.torch.from_numpy(inp[n].astype("float32")).to(self.dev).to(self.tdtype).contiguous()
            self.plan.pack(rm.data_ptr(), self.buf[n].data_ptr(), raw_stream(self.torch, self.dev))
        for n in ("gamma", "beta"):
            if inp.get(n) is not None:
                self.vec[n].copy_(self.torch.from_numpy(inp[n].astype("float32")))
        self.torch.cuda.synchronize(self.dev)

    def forward(self):
        b, v = self.buf, self.vec
        self.plan.fwd(b["X"].data_ptr(), v["gamma"].data_ptr(), v["beta"].data_ptr() if self.cfg.norm == "layernorm" else None,
                      b["Y"].data_ptr(), self.saved.data_ptr(), self.scratch_fwd.data_ptr(), raw_stream(self.torch, self.dev))

    def backward(self, frozen=False):
        b, v = self.buf, self.vec
        self.plan.bwd(b["dY"].data_ptr(), b["X"].data_ptr(), v["gamma"].data_ptr(), self.saved.data_ptr(), b["dX"].data_ptr(),
                      None if frozen else v["dgamma"].data_ptr(),
                      v["dbeta"].data_ptr() if self.cfg.norm == "layernorm" and not frozen else None,
                      self.scratch.data_ptr(), raw_stream(self.torch, self.dev))

    def step(self):
        self.forward()
        self.backward()

    def fetch(self, name):
        """A matrix (row-major) or a vector as a float64 numpy array."""
        torch, c = self.torch, self.cfg
        if name in self.vec:
            torch.cuda.synchronize(self.dev)
            return self.vec[name].cpu().numpy().astype("float64")
        out = torch.empty((c.batch, c.seq, c.d_model), dtype=self.tdtype, device=self.dev)
        self.plan.unpack(self.buf[name].data_ptr(), out.data_ptr(), raw_stream(torch, self.dev))
        torch.cuda.synchronize(self.dev)
        return out.float().cpu().numpy().astype("float64")

    def guards_intact(self):
        self.torch.cuda.synchronize(self.dev)
        named = {"saved": self.saved, "scratch_fwd": self.scratch_fwd, "scratch_bwd": self.scratch, **self.buf, **self._vec_raw}
        return [k for k, v in named.items() if not guard_bands_intact(v)]
