"""``DesLoc``: owns nothing but a context handle; holds references to the caller's tensors.  ``token_logprobs`` and its gradient
need no context."""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Sequence

import torch

from . import binding as B

try:
    from . import _native
except ImportError as e:
    raise ImportError(f"the native part of this module is missing ({e}): build it with "
                      "`python -m paper_2505_22549_b200.build`") from e
if _native.torch_version != str(torch.__version__):
    raise ImportError(f"the native part of this module was built for torch {_native.torch_version}, this is torch "
                      f"{torch.__version__}: build it again with `python -m paper_2505_22549_b200.build`")

_entry = lambda f: ctypes.cast(f, ctypes.c_void_p).value
_native.bind(*(_entry(getattr(B.raw_lib(), "desloc_" + n))
               for n in ("step", "step_masked", "step_normclip", "step_diag", "rel_change", "get_diag_norms", "step_host", "embed", "embed_grad",
                         "embed_grad_bytes", "clip_grads", "clip_grads_bytes", "token_logprobs", "token_logprobs_grad")))

_GRAD_MISFIT = "gradient tensor of wrong dtype, size or layout"
_SNAP_MISFIT = "snapshot tensor of wrong dtype, size or layout"
_HOST_MISFIT = "host gradient tensor of wrong dtype, size, layout or device"


_TYPES = {torch.float32: B.DESLOC_F32, torch.bfloat16: B.DESLOC_BF16}
_TORCH_TYPES = {code: t for t, code in _TYPES.items()}
_TOKEN_TYPES = {torch.int32: B.DESLOC_I32, torch.int64: B.DESLOC_I64}


def _merged(sizes, strides):
    """The one stride of these dimensions taken as one, or None where they have none."""
    size, stride = 1, 0
    for n, s in zip(reversed(sizes), reversed(strides)):
        if n == 1:
            continue
        if size == 1:
            stride = s
        elif s != size * stride:
            return None
        size *= n
    return stride


def _split(lead, tensors):
    """(outer, inner, [strides of each tensor]): the dimensions `lead`, first ones of every tensor, as two; None where the tensors
    do not lie so."""
    for k in range(len(lead) + 1):
        strides = [(_merged(lead[:k], t.stride()[:k]), _merged(lead[k:], t.stride()[k:len(lead)])) for t in tensors]
        if all(a is not None and b is not None for a, b in strides):
            outer = inner = 1
            for n in lead[:k]:
                outer *= n
            for n in lead[k:]:
                inner *= n
            return outer, inner, strides
    return None


def _on(device, what, *tensors):
    for t in tensors:
        if t.device != device:
            raise ValueError(f"{what} must be on {device}")


class BoundGrads:
    """Gradient tensors already checked and marshalled (see DesLoc.bind_grads): `fits` says for what (workers, sizes, type)."""

    def __init__(self, array, keep, fits=None):
        self.array, self._keep, self.fits = array, keep, fits
        self.address = ctypes.addressof(array)
        self._device = None

    def device(self) -> int:
        """The device of all tensors, looked up once; -1 where there is none."""
        if self._device is None:
            found = {t.get_device() for row in self._keep for t in row}
            self._device = found.pop() if len(found) == 1 else -1
        return self._device


class DesLoc:
    """M worker replicas of a tensor list, stepped by the CUDA library.

    x, u, v: lists (one per worker) of lists of CUDA fp32 tensors (one per model tensor),
    updated in place by :meth:`step`.  v is None for SGDM.
    """

    def __init__(self, x: Sequence[Sequence[torch.Tensor]], u, v, *, opt, grad_dtype,
                 beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, clip_rho=0.0,
                 K=(1, 1, 1), flags=0):
        M = len(x)
        numel = [int(t.numel()) for t in x[0]]
        dev = x[0][0].device
        if dev.type != "cuda":
            raise ValueError("DesLoc needs CUDA tensors (there is no CPU path)")
        for arrs in (x, u) + ((v,) if v is not None else ()):
            if len(arrs) != M:
                raise ValueError("x, u, v need one tensor list per worker")
            for lst in arrs:
                if [int(t.numel()) for t in lst] != numel:
                    raise ValueError("every worker needs the same tensor list")
                for t in lst:
                    if t.dtype != torch.float32 or not t.is_contiguous() or t.device != dev:
                        raise ValueError("state tensors must be contiguous fp32 on one device")
        self._keep = (x, u, v)
        self.M, self.numel, self.device = M, numel, dev
        self.grad_dtype = B.DTYPE_BY_NAME.get(grad_dtype, grad_dtype)
        self.cfg = B.make_config(M, numel, opt, grad_dtype, beta1, beta2, eps, weight_decay,
                                 clip_rho, K[0], K[1], K[2], flags)
        flat = lambda a: [t.data_ptr() for lst in a for t in lst]
        self._index = dev.index if dev.index is not None else torch.cuda.current_device()
        self.ctx: Optional[int] = B.desloc_create(
            self.cfg, flat(x), flat(u), flat(v) if v is not None else None, self._index)
        self._tables()

    def _tables(self) -> None:
        # one buffer of pointers per kind of argument, written anew at every call
        self._table = _native.Table(self.numel, self.M)
        self._table2 = _native.Table(self.numel, self.M)
        self._fits = (self.M, tuple(self.numel), self.grad_dtype)

    def bind_grads(self, grads: Sequence[Sequence[torch.Tensor]]):
        """Check a set of gradient tensors once and return a handle every step method accepts in
        place of the nested lists: a loop that reuses its gradient buffers then pays no
        per-step marshalling.  The handle keeps the tensors alive, and is refused where other workers, sizes or another
        type are wanted than it was checked for."""
        if isinstance(grads, BoundGrads):
            self._handle(grads)
            return grads
        n = self.M * len(self.numel)
        grads = [tuple(row) for row in grads]
        # (a table of its own: another thread may be inside a step, which reads the buffer of self._table with
        # the interpreter's lock released)
        table = _native.Table(self.numel, self.M)
        address = self._fill(table, grads, self.grad_dtype, 0, _GRAD_MISFIT)
        return BoundGrads((ctypes.c_void_p * n).from_buffer_copy((ctypes.c_void_p * n).from_address(address)), grads, self._fits)

    def _handle(self, grads) -> int:
        """Address of a handle's array, if it was made for the workers, sizes and type that these are."""
        if grads.fits is not self._fits:
            if grads.fits != self._fits:
                raise ValueError(_GRAD_MISFIT)
            grads.fits = self._fits     # (the next look is a short one)
        return grads.address

    def _grad_address(self, grads) -> int:
        """Address of the array of gradient pointers, good until the next call of this method."""
        if isinstance(grads, BoundGrads):
            return grads.address if grads.fits is self._fits else self._handle(grads)
        return self._fill(self._table, grads, self.grad_dtype, 0, _GRAD_MISFIT)

    def _fill(self, table, nested, kind: int, where: int, misfit: str) -> int:
        """Checks and marshals nested lists of tensors into the buffer of `table`; its address.  Objects that are no
        torch.Tensor but answer the same questions go one by one."""
        if not isinstance(nested, (list, tuple)):
            nested = [list(row) for row in nested]
        address = table.fill(nested, kind, where, misfit)
        if address is None:
            want = torch.bfloat16 if kind == B.DESLOC_BF16 else torch.float32
            ptrs = []
            for row in nested:
                for t, n in zip(row, self.numel):
                    if t.dtype != want or t.numel() != n or not t.is_contiguous() or (where == 1 and t.is_cuda) or (where >= 2 and t.get_device() != where - 2):
                        raise ValueError(misfit)
                    ptrs.append(t.data_ptr())
            if len(ptrs) != self.M * len(self.numel):
                raise ValueError("need one gradient list per worker")
            address = table.set(ptrs)
        return address

    def _raise(self, status: int, where: str):
        raise B.DeslocError(status, where, B.desloc_last_cuda_error(self.ctx))

    def step(self, t: int, lr: float, grads, clip_bound: float = 0.0) -> int:
        """Step t on torch's current stream; returns the sync mask."""
        r = _native.step(self.ctx, t, lr, clip_bound, 0.0, self._grad_address(grads), self._index, 0)
        if r < 0:
            self._raise(r, "desloc_step")
        return r

    def step_normclip(self, t: int, lr: float, grads, max_norm: float, clip_bound: float = 0.0) -> int:
        """Step t with norm-based gradient clipping (per worker, over the whole tensor list)."""
        r = _native.step(self.ctx, t, lr, clip_bound, max_norm, self._grad_address(grads), self._index, 1)
        if r < 0:
            self._raise(r, "desloc_step_normclip")
        return r

    def step_diag(self, t: int, lr: float, grads, max_norm: float = 0.0, clip_bound: float = 0.0) -> int:
        """Step t that also accumulates the gradient, parameter and update norms (read them with
        diag_norms()); max_norm > 0 adds norm-based clipping in front."""
        r = _native.step(self.ctx, t, lr, clip_bound, max_norm, self._grad_address(grads), self._index, 2)
        if r < 0:
            self._raise(r, "desloc_step_diag")
        return r

    def diag_norms(self):
        """(per_tensor [3][M][num_tensors], total [3][M]) of the latest step_diag; kind 0 =
        gradient as read, 1 = new parameters, 2 = update d_t.  Waits for the results: what was on the current stream is done."""
        r = _native.diag_norms(self.ctx, self.M, len(self.numel), self._index)
        if isinstance(r, int):
            self._raise(r, "desloc_get_diag_norms")
        return r

    def grad_norms(self):
        """(norms, clip factors) of the latest step_normclip; synchronises the current stream."""
        stream = torch.cuda.current_stream(self.device).cuda_stream
        return B.desloc_get_grad_norms(self.ctx, self.M, stream)

    def rel_change(self, array: int, then: Sequence[Sequence[torch.Tensor]]):
        """Per-worker ||s - then|| / ||then|| against a snapshot (lists like x); waits like diag_norms()."""
        r = _native.rel_change(self.ctx, array, self._fill(self._table2, then, B.DESLOC_F32, 0, _SNAP_MISFIT),
                               self._index, self.M)
        if not isinstance(r, list):
            self._raise(r, "desloc_rel_change")
        return r

    def _rows_of(self, tensor: int, width: Optional[int]) -> int:
        """Columns of a state tensor taken as rows: its last dimension, unless the caller says."""
        if not 0 <= tensor < len(self.numel):
            raise ValueError("no such tensor")
        shape = self._keep[0][0][tensor].shape
        if width is None and len(shape) < 2:
            raise ValueError("the tensor has one dimension: say how wide its rows are")
        return int(shape[-1] if width is None else width)

    def _tokens(self, tokens: torch.Tensor):
        if tokens.dtype not in _TOKEN_TYPES or tokens.dim() < 1 or tokens.shape[0] != self.M:
            raise ValueError("tokens are int32 or int64, [workers, ...]")
        _on(self.device, "tokens", tokens)
        flat = tokens.reshape(self.M, tokens.numel() // self.M)
        return B.rows(flat.data_ptr(), _TOKEN_TYPES[flat.dtype], *flat.stride()), flat

    def embed(self, tensor: int, tokens: torch.Tensor, scale: float = 1.0, dtype="bf16", width: Optional[int] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """scale * rows of every worker's x of `tensor` by token, on torch's current stream.  tokens: [M, ...] -> [M, ..., width] of `dtype`
        ("f32", "bf16" or torch's; that of `out` where it is given).  Tokens outside the vocabulary give zeros."""
        width = self._rows_of(tensor, width)
        kind = _TYPES.get(dtype, B.DTYPE_BY_NAME.get(dtype))
        if kind is None:
            raise ValueError("embeddings are fp32 or bf16")
        if out is None:     # the usual layouts, natively
            r = _native.embed(self.ctx, tensor, width, self.M, tokens, scale, kind, self._index)
            if r is not None:
                return r if type(r) is not int else self._raise(r, "desloc_embed")
        rows, flat = self._tokens(tokens)
        shape = tuple(tokens.shape) + (width,)
        if out is None:
            out = torch.empty(shape, dtype=_TORCH_TYPES[kind], device=self.device)
        elif tuple(out.shape) != shape or out.dtype not in _TYPES:
            raise ValueError("out does not fit the tokens")
        _on(self.device, "out", out)
        to = _split(shape[:-1], [out]) if out.stride(-1) == 1 or width == 1 else None
        if to is None or (to[0] != self.M and self.M * flat.shape[1] != to[1]):
            raise ValueError("out has rows that the kernels do not reach: at most one stride behind the workers'")
        stride = to[2][0] if to[0] == self.M else (to[2][0][1] * flat.shape[1], to[2][0][1])
        B.desloc_embed(self.ctx, tensor, width, rows, flat.shape[1], scale, B.rows(out.data_ptr(), _TYPES[out.dtype], *stride),
                       torch.cuda.current_stream(self.device).cuda_stream)
        _native.wrote(out)
        return out

    def embed_grad(self, tensor: int, tokens: torch.Tensor, dout: torch.Tensor, grads, scale: float = 1.0, accumulate: bool = False,
                   width: Optional[int] = None) -> None:
        """The gradient of embed() into the workers' gradients of `tensor` in `grads` (what step() reads: nested lists, of which only that
        tensor is looked at, or bind_grads()' handle).  accumulate: added to what they hold."""
        width = self._rows_of(tensor, width)
        r = _native.embed_grad(self.ctx, tensor, width, self.M, tokens, dout, self._bound(grads) if isinstance(grads, BoundGrads) else grads, len(self.numel),
                               self.numel[tensor], self.grad_dtype, scale, accumulate, self._index)
        if r is not None:
            if r != 0:
                self._raise(r, "desloc_embed_grad")
            if isinstance(grads, BoundGrads):   # (lists: done natively)
                _native.wrote([row[tensor] for row in grads._keep])
            return None
        rows, flat = self._tokens(tokens)
        if tuple(dout.shape) != tuple(tokens.shape) + (width,) or dout.dtype not in _TYPES:
            raise ValueError("dout does not fit the tokens")
        _on(self.device, "dout", dout)
        d = dout.reshape(self.M, flat.shape[1], width)
        if d.stride(-1) != 1 and width > 1:
            d = d.contiguous()
        nt = len(self.numel)
        if isinstance(grads, BoundGrads):
            array = grads.array
        else:
            array = (ctypes.c_void_p * (self.M * nt))()
            if len(grads) != self.M:
                raise ValueError("need one gradient list per worker")
            for m, row in enumerate(grads):
                g = row[tensor]
                if g.dtype != _TORCH_TYPES[self.grad_dtype] or g.numel() != self.numel[tensor] or not g.is_contiguous() or g.device != self.device:
                    raise ValueError(_GRAD_MISFIT)
                array[m * nt + tensor] = g.data_ptr()
        n = flat.shape[1]
        work = torch.empty(B.desloc_embed_grad_bytes(self.ctx, tensor, width, n), dtype=torch.uint8, device=self.device)
        B.desloc_embed_grad(self.ctx, tensor, width, rows, n, B.rows(d.data_ptr(), _TYPES[d.dtype], *d.stride()[:2]), scale, accumulate, array,
                            work.data_ptr(), work.numel(), torch.cuda.current_stream(self.device).cuda_stream)
        _native.wrote([row[tensor] for row in (grads._keep if isinstance(grads, BoundGrads) else grads)])

    def _bound(self, grads) -> int:
        """The same, if its tensors are on this device."""
        address = self._handle(grads)
        if grads.device() != self._index:
            raise ValueError(_GRAD_MISFIT)
        return address

    def _list_of(self, table, grads):
        """(address, type code) of a set of gradient tensors of one type, on this context's device."""
        if isinstance(grads, BoundGrads):
            return self._bound(grads), self.grad_dtype
        kind = _TYPES.get(grads[0][0].dtype) if len(grads) and len(grads[0]) else None
        if kind is None:
            raise ValueError(_GRAD_MISFIT)
        return self._fill(table, grads, kind, 2 + self._index, _GRAD_MISFIT), kind

    def clip_grads(self, grads, max_norm: float, out=None):
        """Norm-based clipping on its own: every worker's gradients (nested lists, fp32 or bf16) times min(1, max_norm / their norm over the
        whole tensor list), into `out` (the same, either type) or in place.  Returns (norms, factors), [M] fp32 on the device; nothing waits."""
        address, kind = self._list_of(self._table, grads)
        to, to_kind = (address, kind) if out is None else self._list_of(self._table2, out)
        written = grads if out is None else out
        r = _native.clip_grads(self.ctx, max_norm, kind, address, to_kind, to, self.M, self._index,
                               written._keep if isinstance(written, BoundGrads) else written)
        return r if type(r) is not int else self._raise(r, "desloc_clip_grads")

    def set_workers(self, x, u, v, first_new: int) -> None:
        """New worker set (lists like the constructor's); workers first_new.. start from the mean
        of the current workers.  Synchronises the current stream."""
        M = len(x)
        for arrs in (x, u) + ((v,) if v is not None else ()):
            if len(arrs) != M or any([int(t.numel()) for t in lst] != self.numel for lst in arrs):
                raise ValueError("every worker needs the same tensor list")
        flat = lambda a: [t.data_ptr() for lst in a for t in lst]
        stream = torch.cuda.current_stream(self.device).cuda_stream
        B.desloc_set_workers(self.ctx, M, first_new, flat(x), flat(u),
                             flat(v) if v is not None else None, stream)
        self._keep = (x, u, v)
        self.M = M
        self._tables()

    def step_host(self, t: int, lr: float, host_grads, dev_grads, clip_bound: float = 0.0) -> int:
        """Step t with gradients in (pinned) host tensors; dev_grads are device staging tensors."""
        hp = self._fill(self._table2, host_grads, self.grad_dtype, 1, _HOST_MISFIT)
        r = _native.step_host(self.ctx, t, lr, clip_bound, hp, self._grad_address(dev_grads), self._index)
        if r < 0:
            self._raise(r, "desloc_step_host")
        return r

    def step_masked(self, mask: int, lr: float, grads, clip_bound: float = 0.0) -> None:
        r = _native.step_masked(self.ctx, mask, lr, clip_bound, self._grad_address(grads), self._index)
        if r < 0:
            self._raise(r, "desloc_step_masked")

    def counters(self):
        return B.desloc_get_counters(self.ctx)

    def launches(self) -> int:
        return B.desloc_get_launch_count(self.ctx)

    def close(self) -> None:
        if self.ctx is not None:
            B.desloc_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class TokenLogprobs(NamedTuple):
    """What token_logprobs() returns; what was not asked for is None."""
    logp: torch.Tensor                    # [...]
    lse: torch.Tensor                     # [...]
    entropy: Optional[torch.Tensor]       # [...]
    top_ids: Optional[torch.Tensor]       # [..., top], int64
    top_logp: Optional[torch.Tensor]      # [..., top]


def _logit_rows(logits, tokens, *more):
    """The two-level rows of logits, tokens and what else has one row each; copies what does not lie so."""
    if logits.device.type != "cuda":
        raise ValueError("logits must be CUDA tensors (there is no CPU path)")
    if logits.dtype not in _TYPES or logits.dim() < 1 or logits.shape[-1] < 1:
        raise ValueError("logits are fp32 or bf16, [..., vocabulary]")
    if tokens.dtype not in _TOKEN_TYPES or tokens.shape != logits.shape[:-1]:
        raise ValueError("tokens are int32 or int64, of the shape of the logits without their last dimension")
    _on(logits.device, "tokens", tokens)
    if logits.stride(-1) != 1 and logits.shape[-1] > 1:
        logits = logits.contiguous()
    lead = tuple(logits.shape[:-1])
    found = _split(lead, [logits, tokens, *more])
    if found is None:
        logits, tokens = logits.contiguous(), tokens.contiguous()
        found = _split(lead, [logits, tokens, *more])
    if found is None:
        raise ValueError("out has rows that the kernels do not reach: more than two strides")
    return logits, tokens, found


def _refuse(status: int, where: str):
    raise B.DeslocError(status, where)


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, entropy: bool = False, top: int = 0) -> TokenLogprobs:
    """Log probabilities of `tokens` [...] under `logits` [..., vocabulary] (fp32 or bf16), on torch's current stream: logp (0 for tokens outside the
    vocabulary), lse, and on request the entropy and the `top` likeliest tokens.  exp(-logp.mean(...)) is the perplexity.  torch records nothing: the
    results require no gradient even where the logits do; token_logprobs_grad() is what goes back."""
    r = _native.token_logprobs(logits, tokens, entropy, top)     # the usual layouts, natively
    if r is not None:
        return TokenLogprobs(*r) if type(r) is not int else _refuse(r, "desloc_token_logprobs")
    if not 0 <= top <= B.DESLOC_MAX_TOP:
        _refuse(B.DESLOC_E_RANGE, "desloc_token_logprobs")
    logits, tokens, (outer, inner, strides) = _logit_rows(logits, tokens)
    lead, dev = logits.shape[:-1], logits.device
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)
    r = TokenLogprobs(new(*lead), new(*lead), new(*lead) if entropy else None, new(*lead, top, dtype=torch.int64) if top else None,
                      new(*lead, top) if top else None)
    at = lambda t: t.data_ptr() if t is not None else 0
    B.desloc_token_logprobs(outer, inner, logits.shape[-1], B.rows(logits.data_ptr(), _TYPES[logits.dtype], *strides[0]),
                            B.rows(tokens.data_ptr(), _TOKEN_TYPES[tokens.dtype], *strides[1]), top, *map(at, r), dev.index,
                            torch.cuda.current_stream(dev).cuda_stream)
    return r


def token_logprobs_grad(logits: torch.Tensor, tokens: torch.Tensor, lse: torch.Tensor, dlogp: torch.Tensor, entropy: Optional[torch.Tensor] = None,
                        dentropy: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of sum(dlogp * logp) + sum(dentropy * entropy) with respect to the logits, in their type; lse and entropy are what
    token_logprobs() gave.  out may be the logits themselves; it counts as changed in place for torch."""
    r = _native.token_logprobs_grad(logits, tokens, lse, dlogp, entropy, dentropy, out)
    if r is not None:
        return r if type(r) is not int else _refuse(r, "desloc_token_logprobs_grad")
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device or (out.stride(-1) != 1 and out.shape[-1] > 1):
        raise ValueError("out does not fit the logits")
    if dentropy is not None and entropy is None:
        raise ValueError("the entropy's gradient needs the entropy")
    logits, tokens, (outer, inner, strides) = _logit_rows(logits, tokens, out)
    dense = []
    for t in (lse, dlogp, entropy, dentropy):
        if t is not None and (t.dtype != torch.float32 or t.shape != tokens.shape or t.device != logits.device):
            raise ValueError("lse, dlogp, entropy and dentropy are fp32, of the tokens' shape, where the logits are")
        dense.append(t if t is None or t.is_contiguous() else t.contiguous())
    at = lambda t: t.data_ptr() if t is not None else 0
    B.desloc_token_logprobs_grad(outer, inner, logits.shape[-1], B.rows(logits.data_ptr(), _TYPES[logits.dtype], *strides[0]),
                                 B.rows(tokens.data_ptr(), _TOKEN_TYPES[tokens.dtype], *strides[1]), *map(at, dense),
                                 B.rows(out.data_ptr(), _TYPES[out.dtype], *strides[2]), logits.device.index,
                                 torch.cuda.current_stream(logits.device).cuda_stream)
    _native.wrote(out)
    return out
