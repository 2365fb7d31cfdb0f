"""Operators for training a language model on from an embedding table, over torch CUDA tensors.

    Embedding   rows of a table looked up for a batch of tokens, times a scale; the gradient of the table by sorted
                tokens (the whole table, added to it, or the touched rows alone); the AdamW step of the touched rows.
    AdamW       an AdamW step over many tensors at once, with moments in 32 or in 8 bits.

Every call enqueues its kernels on the current stream of the tensors' device and returns without waiting; tensors
that another stream is still writing are ordered by the caller, as for torch's own operators.  There is no fallback:
a missing library, a CPU tensor or a refused argument is an error.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B

_FLOATS = {torch.float32: B.FLOAT32, torch.bfloat16: B.BFLOAT16, torch.float16: B.FLOAT16}
_INTS = {torch.int32: B.INT32, torch.int64: B.INT64}
# the current stream's handle without a Stream object around it (2 us of a call that takes 10)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None) or torch.cuda.is_current_stream_capturing
# Every tensor that a call has written into is told to autograd: a backward pass that still needs what was there is an error then, as
# after torch's own in-place operations.
_written = torch.autograd.graph.increment_version
_T = torch.Tensor
_NO_PADDING = -(1 << 63)
BLOCK = 256                      # elements that share a scale of the 8-bit moments


def _current_stream(index: int) -> int:
    """The cudaStream_t of the current stream of device `index`, which has to be the current device."""
    if _current_device() != index:
        raise ValueError(f"the tensors' device {index} is not the current one")
    return _raw_stream(index)


def _settle(device):
    """Waits for the current stream, once, when an object has allocated memory of its own: whatever stream it is used on then, neither
    the memory's earlier users nor the zeros written to it are still to come."""
    if not _capturing():
        torch.cuda.current_stream(device).synchronize()


def _need(cond, what: str):
    if not cond:
        raise ValueError(what)


class Embedding:
    """Lookup and gradient calls for tables of V rows of d elements and batches of up to max_tokens tokens.

    scale multiplies every looked-up row (and so every gradient row).  padding_id names an id that stands for "no token":
    its positions read as zero rows and have no gradient.  The object owns the workspace of the gradient calls and the error
    word that ids outside [0, V) are reported in (`check`), and orders their use where calls come on several streams; it is used
    from one thread at a time, and has to outlive the graphs that its calls were captured into.
    """

    def __init__(self, V: int, d: int, max_tokens: int, scale: float = 1.0, padding_id: Optional[int] = None, device: int = 0):
        _need(torch.cuda.is_available(), "no CUDA device: the operators have no CPU implementation")
        self.V, self.d, self.max_tokens, self.scale = V, d, max_tokens, scale
        self.device, self.index = torch.device("cuda", device), device
        lib = B.lib()
        size = C.c_uint64(0)
        B._check(lib.tensair_embedding_workspace_bytes(max_tokens, V, d, C.byref(size)), "tensair_embedding_workspace_bytes")
        self.workspace_bytes = size.value
        self.workspace = torch.empty(max(1, size.value), dtype=torch.uint8, device=self.device)
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)
        _settle(self.device)
        self._known = {torch.cuda.current_stream(self.device).cuda_stream}
        self._workspace_stream = self._workspace_user = None
        self._lib = lib
        self._tokens = B.Tokens(V=V, padding_id=_NO_PADDING if padding_id is None else padding_id, error=self.error.data_ptr())
        self._rows = [B.Rows(d=d) for _ in range(4)]
        self._adamw = B.Adamw()
        # references made once: a call then converts no argument
        self._at = [C.byref(x) for x in [self._tokens] + self._rows + [self._adamw]]
        self._workspace_at = self.workspace.data_ptr()

    # ---- arguments (checked on every call: the messages are made only when one is refused)
    def _set_tokens(self, ids):
        kind = _INTS.get(ids.dtype)
        n = ids.numel()
        if kind is None or ids.get_device() != self.index or n > self.max_tokens:
            raise ValueError(f"ids: {n} of {ids.dtype} on {ids.device}; up to {self.max_tokens} int32 or int64 on {self.device} go")
        if not ids.is_contiguous():
            ids = ids.contiguous()
        t = self._tokens
        t.ids, t.n, t.type = ids.data_ptr(), n, kind
        return ids, n

    def _set_rows(self, which, x, rows, name):
        kind = _FLOATS.get(x.dtype)
        shape, stride = x.shape, x.stride()
        if (kind is None or x.get_device() != self.index or len(shape) != 2 or shape[0] != rows or shape[1] != self.d
                or (stride[1] != 1 and self.d > 1) or (stride[0] < self.d and rows > 1)):
            raise ValueError(f"{name}: {tuple(shape)} of {x.dtype} with strides {stride} on {x.device}; ({rows}, {self.d}) of float32, "
                             f"bfloat16 or float16 on {self.device} with columns next to each other go")
        r = self._rows[which]
        r.data, r.stride, r.type = x.data_ptr(), stride[0] if rows > 1 else self.d, kind
        return self._at[1 + which]

    def _grad_rows(self, grad, n):
        if grad.dim() != 2:
            if grad.dim() == 0 or grad.shape[-1] != self.d or grad.numel() != n * self.d:
                raise ValueError(f"grad: shape {tuple(grad.shape)} for {n} tokens of width {self.d}")
            grad = grad.reshape(n, self.d)
        row, column = grad.stride()
        if column != 1 or row < self.d:       # broadcast or transposed: the rows are laid out first
            grad = grad.contiguous()
        return grad

    def _stream(self):
        """The current stream, on which the object's memory is in use from now on: the allocator hands it out again only after that."""
        stream = _current_stream(self.index)
        if stream not in self._known and not _capturing():
            now = torch.cuda.current_stream(self.device)
            self.error.record_stream(now)
            self.workspace.record_stream(now)
            self._known.add(stream)
        return stream

    def _workspace_on(self):
        """(workspace, its address, current stream), after the calls of another stream that may still use the workspace.  A call that is
        captured into a graph has one of its own, out of the graph's memory: nobody here knows when the graph runs."""
        stream = self._stream()
        if _capturing():
            own = torch.empty(max(1, self.workspace_bytes), dtype=torch.uint8, device=self.device)
            return own, own.data_ptr(), stream
        if stream != self._workspace_stream:
            now = torch.cuda.current_stream(self.device)
            if self._workspace_user is not None:
                now.wait_stream(self._workspace_user)
            self._workspace_stream, self._workspace_user = stream, now
        return self.workspace, self._workspace_at, stream

    # ---- calls
    def lookup(self, table, ids, out=None, dtype=None):
        """scale * table[ids], zero rows at padding; shape ids.shape + (d,), of `dtype` (default: the table's)."""
        flat, n = self._set_tokens(ids)
        rt = self._set_rows(0, table, self.V, "table")
        given = shaped = out
        if out is None:
            dtype = dtype or table.dtype
            _need(dtype in _FLOATS, "dtype: float32, bfloat16 or float16")
            out = shaped = torch.empty((n, self.d), dtype=dtype, device=self.device)
            r = self._rows[1]
            r.data, r.stride, r.type = out.data_ptr(), self.d, _FLOATS[dtype]
            ro = self._at[2]
            if ids.dim() != 1:
                shaped = out.view(*ids.shape, self.d)
        else:
            ro = self._set_rows(1, out if out.dim() == 2 else out.view(n, self.d), n, "out")
        rc = self._lib.tensair_embedding_lookup(self._at[0], rt, ro, self.scale, self._stream())
        if rc:
            B._check(rc, "tensair_embedding_lookup")
        if given is not None:
            _written(given)
        return shaped

    def gradient(self, grad, ids, out=None, dtype=None, accumulate=False):
        """The gradient of the whole table, (V, d): scale times the sum of the gradient rows of each token's positions.

        accumulate adds it to `out`, of which only the rows of tokens that occur are read and written."""
        flat, n = self._set_tokens(ids)
        grad = self._grad_rows(grad, n)
        _need(out is not None or not accumulate, "accumulate needs out")
        given = out
        if out is None:
            out = torch.empty(self.V, self.d, dtype=dtype or grad.dtype, device=self.device)
        rg = self._set_rows(0, grad, n, "grad")
        ro = self._set_rows(1, out, self.V, "out")
        workspace, at, stream = self._workspace_on()
        rc = self._lib.tensair_embedding_gradient(self._at[0], rg, ro, self.scale, accumulate, at, self.workspace_bytes, stream)
        if rc:
            B._check(rc, "tensair_embedding_gradient")
        if given is not None:
            _written(given)
        return out

    def gradient_rows(self, grad, ids, out=None):
        """The touched rows alone: (row ids int32 [m], rows float32 [m, d], count int32 [1]), m = min(tokens, V).

        The first `count` entries are written, row ids ascending; the rest is left alone."""
        flat, n = self._set_tokens(ids)
        grad = self._grad_rows(grad, n)
        most = min(n, self.V)
        given = out
        if out is None:
            out = (torch.empty(most, dtype=torch.int32, device=self.device),
                   torch.empty(most, self.d, dtype=torch.float32, device=self.device),
                   torch.empty(1, dtype=torch.int32, device=self.device))
        row_ids, rows, count = out
        for x, least in ((row_ids, most), (count, 1)):
            if x.device != self.device or x.dtype != torch.int32 or not x.is_contiguous() or x.numel() < least:
                raise ValueError(f"row ids and count: contiguous int32 tensors on {self.device}, at least {most} and 1 long")
        _need(rows.shape[0] >= most, "rows: fewer than the batch can touch")
        rg = self._set_rows(0, grad, n, "grad")
        ro = self._set_rows(1, rows, rows.shape[0], "rows")
        workspace, at, stream = self._workspace_on()
        rc = self._lib.tensair_embedding_gradient_rows(self._at[0], rg, self.scale, row_ids.data_ptr(), ro, count.data_ptr(), at,
                                                       self.workspace_bytes, stream)
        if rc:
            B._check(rc, "tensair_embedding_gradient_rows")
        if given is not None:
            _written(given)
        return out

    def adamw(self, grad, ids, table, m, v, step: int, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None):
        """The AdamW step, in place, of the rows of table, m and v (float32) whose tokens occur; see AdamW for the formula.

        A graph that captures it repeats the step of this number, lr and constants at every replay."""
        flat, n = self._set_tokens(ids)
        grad = self._grad_rows(grad, n)
        rg = self._set_rows(0, grad, n, "grad")
        rt = self._set_rows(1, table, self.V, "table")
        rm = self._set_rows(2, m, self.V, "m")
        rv = self._set_rows(3, v, self.V, "v")
        h = self._adamw
        _set_adamw(h, lr, betas, eps, weight_decay, step, 0, grad_scale, self.device)
        workspace, at, stream = self._workspace_on()
        rc = self._lib.tensair_embedding_adamw(self._at[0], rg, self.scale, rt, rm, rv, self._at[5], at, self.workspace_bytes, stream)
        if rc:
            B._check(rc, "tensair_embedding_adamw")
        _written((table, m, v))

    def __call__(self, table, ids):
        """lookup(table, ids) with autograd: the table's gradient is `gradient` of the incoming one."""
        return _Lookup.apply(table, ids, self)

    def check(self):
        """Waits for the device, all its streams, and raises TensairError (EBADTOKEN) if a call since the last check met an id outside [0, V)."""
        torch.cuda.synchronize(self.device)
        flags = int(self.error.item())
        if flags:
            self.error.zero_()
            torch.cuda.current_stream(self.device).synchronize()      # whatever stream the next call is on
            raise B.TensairError(B.tensair_error_of_flags(flags), "Embedding")


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, embedding):
        ctx.save_for_backward(ids)
        ctx.embedding, ctx.dtype = embedding, table.dtype
        return embedding.lookup(table, ids)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        ids, = ctx.saved_tensors
        return ctx.embedding.gradient(grad, ids, dtype=ctx.dtype), None, None


def _set_adamw(h, lr, betas, eps, weight_decay, step, seed, grad_scale, device):
    h.lr, h.eps, h.weight_decay, h.step, h.seed = lr, eps, weight_decay, step, seed
    h.beta1, h.beta2 = betas
    if grad_scale is not None:
        _need(grad_scale.device == device and grad_scale.dtype == torch.float32 and grad_scale.numel() == 1,
              "grad_scale: one float32 on the tensors' device")
        h.grad_scale = grad_scale.data_ptr()
    else:
        h.grad_scale = None


_DESCRIPTOR = np.dtype({"names": [f[0] for f in B.AdamwTensor._fields_],
                        "formats": ["u8"] * 8 + ["f8"] * 2 + ["u4"] * 4,
                        "offsets": [getattr(B.AdamwTensor, f[0]).offset for f in B.AdamwTensor._fields_],
                        "itemsize": C.sizeof(B.AdamwTensor)})


class AdamW:
    """AdamW over a list of contiguous parameters, in one launch for each combination of parameter and gradient types (and for every
    336 parameters):

        m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2,
        p <- p (1 - lr decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)

    state_bits 32 keeps m and v as float32; 8 keeps m and sqrt(v) as float8_e4m3fn with a float32 scale for every 256 elements
    (`m_scale`, `v_scale`), rounded stochastically with bits that depend on `seed`, the step and the element's place in the list of
    parameters alone, whichever of them have a gradient.
    copies: tensors (bfloat16 or float16, or None) that receive the updated parameters, rounded.  lr_factors and
    decay_factors: per-parameter factors on lr and weight_decay.  state: dict of lists to start from (m, v and for 8 bits
    m_scale, v_scale; they become the optimizer's own), zeros by default; step: steps already made.

    A parameter may change its place or its type between steps (model.bfloat16()), not its size.  The moments and copies are those of
    the constructor: they can be written into, not replaced.  Moments that the constructor made are there on any stream; steps on
    several streams are ordered by the caller, as everything else that uses the parameters.  The optimizer has to outlive the graphs
    that its steps were captured into.
    """

    def __init__(self, params: Sequence[torch.Tensor], lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32,
                 copies=None, lr_factors=None, decay_factors=None, state=None, step=0, seed=0):
        params = list(params)
        _need(params, "params: empty")
        _need(state_bits in (32, 8), "state_bits: 32 or 8")
        self.params, self.lr, self.betas, self.eps, self.weight_decay = params, lr, betas, eps, weight_decay
        self.state_bits, self.step_count, self.seed = state_bits, step, seed
        self.device = params[0].device
        _need(self.device.type == "cuda", "no CUDA device: the operators have no CPU implementation")
        self.index = self.device.index
        kept = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        names = ["m", "v"] + (["m_scale", "v_scale"] if state_bits == 8 else [])
        self._known = None                 # streams that the moments are known to be used on, where they were made here
        if not state:
            state = {k: [torch.zeros(-(-p.numel() // BLOCK) if k.endswith("scale") else p.numel(),
                                     dtype=torch.float32 if k.endswith("scale") else kept, device=self.device) for p in params]
                     for k in names}
            _settle(self.device)
            self._known = {_raw_stream(self.index)}
        _need(sorted(state) == sorted(names), f"state: needs {names}")
        self._t = (B.AdamwTensor * len(params))()
        self._np = np.frombuffer(self._t, dtype=_DESCRIPTOR)
        self._copies = tuple(copies) if copies is not None else (None,) * len(params)
        self._state = {k: tuple(state[k]) for k in names}
        lists = [self._copies, lr_factors or params, decay_factors or params] + [self._state[k] for k in names]
        _need(all(len(x) == len(params) for x in lists), "copies, factors and state need one entry per parameter")
        for i, p in enumerate(params):
            t = self._t[i]
            self._fits(p, p.numel(), _FLOATS, f"params[{i}]")
            t.n = p.numel()
            for k in names:
                want = -(-p.numel() // BLOCK) if k.endswith("scale") else p.numel()
                self._fits(self._state[k][i], want, (torch.float32,) if k.endswith("scale") else (kept,), f"{k}[{i}]")
                setattr(t, k, self._state[k][i].data_ptr())
            c = self._copies[i]
            if c is not None:
                self._fits(c, p.numel(), (torch.bfloat16, torch.float16), f"copies[{i}]")
                t.copy, t.copy_type = c.data_ptr(), _FLOATS[c.dtype]
            t.lr_factor = lr_factors[i] if lr_factors else 1.0
            t.decay_factor = decay_factors[i] if decay_factors else 1.0
        # what the descriptors point to is held here, whatever becomes of the tensors that the caller has
        self._held = [x.detach() for xs in [self._copies, *self._state.values()] for x in xs if x is not None]
        self._lib = B.lib()
        self._hyper = B.Adamw()
        self._at = C.byref(self._hyper)
        self._said, self._left_out = [None, None, None, None], []
        self._numel, self._shapes = [p.numel() for p in params], [p.shape for p in params]
        self._describe_params([p.data_ptr() for p in params], [p.dtype for p in params])      # as they were checked above

    def _describe_params(self, places, kinds):
        self._np["param_type"] = [_FLOATS[k] for k in kinds]
        self._np["param"] = places
        self._said[1], self._said[3] = places, kinds
        self._written = self._all_written(self._left_out)

    def _all_written(self, left_out):
        """What a step writes that may be part of a graph: parameters and copies, but for those that are left out."""
        return [x for i, pair in enumerate(zip(self.params, self._copies)) if i not in left_out for x in pair if x is not None]

    # The tensors that the descriptors point to, once and for all: tuples, so that an entry cannot be replaced unseen.
    @property
    def m(self):
        return self._state["m"]

    @property
    def v(self):
        return self._state["v"]

    @property
    def m_scale(self):
        return self._state.get("m_scale")

    @property
    def v_scale(self):
        return self._state.get("v_scale")

    @property
    def copies(self):
        return self._copies

    def _fits(self, x, n, dtypes, name):
        _need(x.device == self.device and x.dtype in dtypes and x.numel() == n and x.is_contiguous(),
              f"{name}: a contiguous tensor of {n} elements on {self.device}, of {', '.join(str(d) for d in dtypes)}")

    def step(self, grads=None, grad_scale=None):
        """One step with `grads` (default: the parameters' .grad; a parameter whose gradient is None is left alone), each of its
        parameter's shape, or flat.

        grad_scale: a float32 on the device that multiplies every gradient; if it is not finite the parameters and moments
        stay as they are (the step still counts).

        A captured step (32-bit moments alone) counts when it is captured; every replay is that step again, with the bias
        corrections of its number and the lr and other constants of that moment."""
        if grads is None:
            grads = [p.grad for p in self.params]
        _need(len(grads) == len(self.params), "grads: one for each parameter, or None")
        # one list per property, each made in one go: a fifth of the time of a loop with its checks
        try:
            kinds, left_out = [g.dtype for g in grads], []
        except AttributeError:                     # there is a None
            left_out = [i for i, g in enumerate(grads) if g is None]
            grads = list(grads)
            for i in left_out:
                grads[i] = self.params[i]          # stands in for the checks
            kinds = [g.dtype for g in grads]
        shapes = [g.shape for g in grads]
        index, a, said = self.index, self._np, self._said     # what the descriptors say is written again only where it changed
        if (shapes != self._shapes or (kinds != said[2] and not _FLOATS.keys() >= set(kinds))
                or False in map(_T.is_contiguous, grads) or set(map(_T.get_device, grads)) != {index}):
            for i, (g, p) in enumerate(zip(grads, self.params)):
                self._fits(g, self._numel[i], _FLOATS, f"grads[{i}]")
                _need(g.shape == p.shape or g.dim() == 1, f"grads[{i}]: shape {tuple(g.shape)} for a parameter of shape {tuple(p.shape)}")
            self._shapes = shapes
        ptrs = list(map(_T.data_ptr, grads))
        if ptrs != said[0]:
            a["grad"] = said[0] = ptrs
        # a parameter may have been converted or moved: its place and type are looked at in every step, the rest where one of them changed
        ptrs, param_kinds = list(map(_T.data_ptr, self.params)), [p.dtype for p in self.params]
        if ptrs != said[1] or param_kinds != said[3]:
            for i, p in enumerate(self.params):
                self._fits(p, self._numel[i], _FLOATS, f"params[{i}]")
            self._describe_params(ptrs, param_kinds)
        if kinds != said[2]:
            said[2] = kinds
            a["grad_type"] = [_FLOATS[k] for k in kinds]
        if left_out != self._left_out:
            a["skip"] = 0
            a["skip"][left_out] = 1
            self._left_out = left_out
            self._written = self._all_written(left_out)
        _set_adamw(self._hyper, self.lr, self.betas, self.eps, self.weight_decay, self.step_count + 1, self.seed, grad_scale, self.device)
        stream = _current_stream(index)
        if self._known is not None and stream not in self._known and not _capturing():
            now = torch.cuda.current_stream(self.device)
            for xs in self._state.values():
                for x in xs:
                    x.record_stream(now)
            self._known.add(stream)
        rc = self._lib.tensair_adamw_step(self._t, len(grads), self.state_bits, self._at, stream)
        if rc:
            B._check(rc, "tensair_adamw_step")
        self.step_count += 1
        _written(self._written)

    def moments(self, i: int):
        """(m, v) of parameter i as float32 tensors, whatever they are kept in."""
        if self.state_bits == 32:
            return self.m[i].clone(), self.v[i].clone()
        n = self._numel[i]
        wide = [s[i].repeat_interleave(BLOCK)[:n] for s in (self.m_scale, self.v_scale)]
        return self.m[i].float().view(-1) * wide[0], (self.v[i].float().view(-1) * wide[1]).square()
