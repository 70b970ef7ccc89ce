"""Microscaled 4-bit linear layers and 8-bit activation checkpoints on the GPU: the buffers they
need and the sequences of C-ABI calls of a training step and of serving.  torch only allocates
device memory here; every arithmetic step is a libshiftquant call.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import native as N


def _blocks(rows: int, cols: int, device) -> tuple[torch.Tensor, torch.Tensor]:
    """codes [rows, bytes] and scales of an mx4 tensor [rows, cols]."""
    codes = torch.zeros((rows, max((cols + 31) // 32 * 16, 16)), dtype=torch.uint8, device=device)
    scales = torch.zeros(N.shiftquant_mx4_scale_bytes(rows, cols), dtype=torch.uint8, device=device)
    return codes, scales


def _elsewhere(t: torch.Tensor, device: torch.device) -> ValueError:
    """Kernels take addresses: a tensor of another device than the object's (`_on`) has none of its own."""
    return ValueError(f"a tensor on {device} expected, not on {t.device}")


def _require_alike(new, share, what: tuple[str, ...]) -> None:
    """An object shares buffers with one that was made alike."""
    for name in what:
        if getattr(new, name) != getattr(share, name):
            raise ValueError(f"buffers are shared with an object of the same {name}: "
                             f"{getattr(share, name)}, not {getattr(new, name)}")
    if new.status.device != share.status.device:
        raise ValueError(f"buffers are shared on one device: {share.status.device}, not {new.status.device}")


@dataclass
class Mx4Tensor:
    """A [R, C] tensor in mx4: codes and scales along its rows, and of its transpose."""
    shape: tuple[int, int]
    codes: torch.Tensor | None
    scales: torch.Tensor | None
    codes_t: torch.Tensor | None
    scales_t: torch.Tensor | None
    status: torch.Tensor

    def __post_init__(self):
        self._own = self.arguments()   # the tensor's buffers stay
        self._on = self.status.device

    @staticmethod
    def alloc(R: int, C: int, device, rows: bool = True, cols: bool = True,
              status: torch.Tensor | None = None) -> "Mx4Tensor":
        codes, scales = _blocks(R, C, device) if rows else (None, None)
        codes_t, scales_t = _blocks(C, R, device) if cols else (None, None)
        if status is None:
            status = torch.zeros(1, dtype=torch.int32, device=device)
        return Mx4Tensor((R, C), codes, scales, codes_t, scales_t, status)

    def operand(self) -> tuple[int, int, int]:
        """codes, leading dimension and scales along the rows, as a product's arguments."""
        return (*N._fixed(self.codes), self.scales.data_ptr())

    def operand_t(self) -> tuple[int, int, int]:
        """The same of the transpose."""
        return (*N._fixed(self.codes_t), self.scales_t.data_ptr())

    def arguments(self) -> tuple[int, ...]:
        """What a quantizer call writes, as its arguments."""
        none = (0, 0, 0)
        return (*(self.operand() if self.codes is not None else none),
                *(self.operand_t() if self.codes_t is not None else none), self.status.data_ptr())

    def quantize(self, x: torch.Tensor, stochastic: bool = False, seed: int = 0, row0: int = 0,
                 stream=None) -> "Mx4Tensor":
        """Both orientations this tensor holds from x, in one pass."""
        if x.shape != self.shape:
            raise ValueError(f"a tensor of {self.shape}, not {tuple(x.shape)}")
        if x.device != self._on:
            raise _elsewhere(x, self._on)
        N._check(N.load().shiftquant_mx4_quantize(
            x.data_ptr(), N._dtype(x), *self.shape, N._ld(x),
            N.SQ_ROUND_STOCHASTIC if stochastic else N.SQ_ROUND_NEAREST_EVEN, seed & (2**64 - 1), row0, *self._own,
            N._stream(stream)))
        return self

    def values(self, out: torch.Tensor, stream=None) -> torch.Tensor:
        """The values the codes along the rows stand for, into out [R, C]."""
        if tuple(out.shape) != self.shape:
            raise ValueError(f"an output of {self.shape}, not {tuple(out.shape)}")
        if out.device != self._on:
            raise _elsewhere(out, self._on)
        N.shiftquant_mx4_dequantize(self.codes, self.scales, out, stream)
        return out

    def values_t(self, out: torch.Tensor, stream=None) -> torch.Tensor:
        """The same of the transpose, into out [C, R]."""
        if tuple(out.shape) != self.shape[::-1]:
            raise ValueError(f"an output of {self.shape[::-1]}, not {tuple(out.shape)}")
        if out.device != self._on:
            raise _elsewhere(out, self._on)
        N.shiftquant_mx4_dequantize(self.codes_t, self.scales_t, out, stream)
        return out


class Mx4Linear:
    """Y = X W with X [M, K] and W [K, N] in mx4: nearest-even forward operands, stochastic
    gradients.  The layer owns its outputs y, dx (of `dtype`) and dw (fp32), whose addresses its
    calls pass; with train=False it holds the forward weight alone.  Calls take up to M rows, and
    the codes of x and dy are laid out for the last call's.

    share: a layer made alike, whose buffers of what does not outlast a call's use this one takes
    too (y, dx, the codes of dy and those of x for the forward product); its own are the weight, what
    the backward pass needs of x, and dw.  An output of either then stays until the next call of
    the same kind of any of them, and their calls are in order on one stream."""

    def __init__(self, M: int, K: int, Nout: int, dtype: torch.dtype, device, train: bool = True,
                 share: "Mx4Linear | None" = None):
        self.M, self.K, self.N, self.dtype, self.train = M, K, Nout, dtype, train
        self._rows = None              # of the last forward call whose codes are kept
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.w = Mx4Tensor.alloc(K, Nout, device, train, True, self.status)
        self.dx = self.dw = None
        if share is None:
            self.x = Mx4Tensor.alloc(M, K, device, True, train, self.status)
            self.y = torch.zeros((M, Nout), dtype=dtype, device=device)
        else:
            _require_alike(self, share, ("M", "K", "N", "dtype", "train"))
            codes_t, scales_t = _blocks(K, M, device) if train else (None, None)
            self.x = Mx4Tensor((M, K), share.x.codes, share.x.scales, codes_t, scales_t, self.status)
            self.y = share.y
        if train:
            if share is None:
                self.g = Mx4Tensor.alloc(M, Nout, device, True, True, self.status)
                self.dx = torch.zeros((M, K), dtype=dtype, device=device)
            else:
                g, self.dx = share.g, share.dx
                self.g = Mx4Tensor((M, Nout), g.codes, g.scales, g.codes_t, g.scales_t, self.status)
            self.dw = torch.zeros((K, Nout), dtype=torch.float32, device=device)
        self._lib, self._dtype, self._status = N.load(), N._dtype(self.y), self.status.data_ptr()
        self._on = self.status.device
        x, w = self.x, self.w
        self._quantize_x = x.arguments()
        self._y = N._fixed(self.y)
        # codes, leading dimension and scales of both operands
        self._forward = (*x.operand(), *w.operand_t())
        self._serve = (*w.operand_t(), Nout, *self._y, *x.operand(), self._status)
        if train:
            g = self.g
            self._quantize_g = g.arguments()
            # ... and what follows the number of rows
            self._dx = (*g.operand(), *w.operand()), (K, Nout, self.dx.data_ptr(), self._dtype, K, self._status)
            self._dw = (*x.operand_t(), *g.operand_t(), K, Nout), (self.dw.data_ptr(), N.SQ_F32, Nout, self._status)

    def set_weight(self, w: torch.Tensor, stream=None) -> None:
        self.w.quantize(w, stream=stream)

    def forward(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """y [rows of x, N]; x's codes stay for the backward pass."""
        m, k = x.shape
        if k != self.K or m > self.M:
            raise ValueError(f"x of [{self.M}, {self.K}] expected, not {(m, k)}")
        if x.device != self._on:
            raise _elsewhere(x, self._on)
        lib, s, dtype = self._lib, N._stream(stream), N._dtype(x)
        if not self.train and dtype == self._dtype:
            status = lib.shiftquant_mx4_linear(x.data_ptr(), dtype, m, k, N._ld(x), *self._serve, s)
        else:
            status = lib.shiftquant_mx4_quantize(x.data_ptr(), dtype, m, k, N._ld(x), N.SQ_ROUND_NEAREST_EVEN, 0, 0,
                                                 *self._quantize_x, s)
            if status == N.SQ_OK:
                status = lib.shiftquant_mx4_gemm(*self._forward, m, self.N, k, self._y[0], self._dtype, self._y[1],
                                                 self._status, s)
        N._check(status)
        self._rows = m if self.train else None
        return self.y if m == self.M else self.y[:m]

    def backward(self, dy: torch.Tensor, seed: int, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
        """dx and dw from dy and the codes the last forward left (of as many rows)."""
        m, n = dy.shape
        if n != self.N or m > self.M:
            raise ValueError(f"dy of [{self.M}, {self.N}] expected, not {(m, n)}")
        if dy.device != self._on:
            raise _elsewhere(dy, self._on)
        if m != self._rows:
            raise _not_kept(m, self._rows)
        lib, s = self._lib, N._stream(stream)
        status = lib.shiftquant_mx4_quantize(dy.data_ptr(), N._dtype(dy), m, n, N._ld(dy), N.SQ_ROUND_STOCHASTIC,
                                             seed & (2**64 - 1), 0, *self._quantize_g, s)
        if status == N.SQ_OK:
            operands, rest = self._dx
            status = lib.shiftquant_mx4_gemm(*operands, m, *rest, s)
        if status == N.SQ_OK:
            operands, rest = self._dw
            status = lib.shiftquant_mx4_gemm(*operands, m, *rest, s)
        N._check(status)
        return self.dx if m == self.M else self.dx[:m], self.dw


def _not_kept(rows: int, kept: int | None) -> ValueError:
    """A backward pass takes the rows of the last forward pass, whose codes are what is kept."""
    return ValueError(f"a gradient of {rows} rows, where " +
                      ("no forward pass has kept its input" if kept is None
                       else f"the last forward pass kept {kept}"))


def _kept(rows: int, cols: int, parts: int, device) -> tuple[torch.Tensor, torch.Tensor]:
    """codes and scales of an input kept in 8 bits: `parts` tensors [rows, cols] side by side.  Rows
    of scales are whole words, which the norm's backward pass reads faster."""
    blocks = max((cols + 31) // 32, 1) * parts
    return (torch.zeros((rows, 32 * blocks), dtype=torch.int8, device=device),
            torch.zeros((rows, (blocks + 3) // 4 * 4), dtype=torch.uint8, device=device))


ACTIVATIONS = {"gelu": N.SQ_ACT_GELU, "gelu_tanh": N.SQ_ACT_GELU_TANH, "silu": N.SQ_ACT_SILU}


class Act8:
    """y = f(h) of h [M, F], or gated y = f(a) u of h = [a | u] [M, 2 F]; h is kept in 8 bits
    for the backward pass (33 bytes per 32 elements).  The object owns y and dh, whose addresses
    its calls pass, and which may not be the same call's input; with train=False it keeps nothing.
    Both calls take up to M rows.  share: an object made alike, whose y and dh this one takes too:
    they stay until the next call of either, and calls are in order on one stream."""

    def __init__(self, M: int, F: int, dtype: torch.dtype, act: str, gated: bool, device, train: bool = True,
                 share: "Act8 | None" = None):
        if act not in ACTIVATIONS:
            raise ValueError(f"an activation of {sorted(ACTIVATIONS)}, not {act!r}")
        self.M, self.F, self.dtype, self.parts, self.act = M, F, dtype, 2 if gated else 1, ACTIVATIONS[act]
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.codes = self.scales = self.dh = None
        self.train, self._rows = train, None
        if share is None:
            self.y = torch.zeros((M, F), dtype=dtype, device=device)
            if train:
                self.dh = torch.zeros((M, self.parts * F), dtype=dtype, device=device)
        else:
            _require_alike(self, share, ("M", "F", "dtype", "parts", "train"))
            self.y, self.dh = share.y, share.dh
        if train:
            self.codes, self.scales = _kept(M, F, self.parts, device)
        self._lib, self._dtype, self._on = N.load(), N._dtype(self.y), self.status.device
        kept = (*N._fixed(self.codes), *N._fixed(self.scales))
        self._forward = (self.act, self.parts - 1, *N._fixed(self.y), *kept, self.status.data_ptr())
        self._backward = (*kept, self.act, self.parts - 1, *N._fixed(self.dh))

    def _check(self, t: torch.Tensor, cols: int) -> int:
        m, c = t.shape
        if m > self.M or c != cols:
            raise ValueError(f"a tensor of [{self.M}, {cols}] expected, not {(m, c)}")
        if t.dtype != self.dtype:
            raise TypeError(f"a tensor of {self.dtype} expected, not {t.dtype}")
        if t.device != self._on:
            raise _elsewhere(t, self._on)
        return m

    def forward(self, h: torch.Tensor, stream=None) -> torch.Tensor:
        m = self._check(h, self.parts * self.F)
        N._check(self._lib.shiftquant_act8_forward(h.data_ptr(), self._dtype, m, self.F, N._ld(h), *self._forward,
                                                   N._stream(stream)))
        self._rows = m if self.train else None
        return self.y if m == self.M else self.y[:m]

    def backward(self, dy: torch.Tensor, stream=None) -> torch.Tensor:
        """dh from dy and the input the last forward kept (as many rows)."""
        m = self._check(dy, self.F)
        if m != self._rows:
            raise _not_kept(m, self._rows)
        N._check(self._lib.shiftquant_act8_backward(dy.data_ptr(), self._dtype, m, self.F, N._ld(dy), *self._backward,
                                                    N._stream(stream)))
        return self.dh if m == self.M else self.dh[:m]


class Norm8:
    """Layer norm ("layer") or root-mean-square norm ("rms") of the rows of x [M, C], or of
    x + residual, whose input is kept in 8 bits for the backward pass.  The object owns the
    outputs, whose addresses its calls pass; both calls take up to M rows.  A call's inputs may not
    be its own outputs, but for the residual stream in place: residual = sum, and dsum = dx.
    share: an object made alike, whose y, sum, dx and workspace this one takes too: they stay until
    the next call of either, and calls are in order on one stream."""

    def __init__(self, M: int, C: int, dtype: torch.dtype, norm: str, device, residual: bool = False,
                 eps: float = 1e-5, train: bool = True, share: "Norm8 | None" = None):
        if norm not in ("layer", "rms"):
            raise ValueError(f"a norm of 'layer' and 'rms', not {norm!r}")
        self.M, self.C, self.dtype, self.layer, self.residual, self.eps = M, C, dtype, norm == "layer", residual, eps
        self.train, self._rows = train, None
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        if share is None:
            self.y = torch.zeros((M, C), dtype=dtype, device=device)
            self.sum = torch.zeros((M, C), dtype=dtype, device=device) if residual else None
        else:
            _require_alike(self, share, ("M", "C", "dtype", "residual", "train"))
            self.y, self.sum = share.y, share.sum
        self.codes = self.scales = self.stats = None
        if train:
            self.codes, self.scales = _kept(M, C, 1, device)
            self.stats = torch.zeros((M, 2), dtype=torch.float32, device=device)
            self.dgamma = torch.zeros(C, dtype=torch.float32, device=device)
            self.dbeta = torch.zeros(C, dtype=torch.float32, device=device) if self.layer else None
            if share is None:
                self.dx = torch.zeros((M, C), dtype=dtype, device=device)
                self.workspace = torch.zeros(max(N.shiftquant_norm8_workspace_bytes(M, C), 16), dtype=torch.uint8,
                                             device=device)
            else:
                self.dx, self.workspace = share.dx, share.workspace
        self._lib, self._dtype, self._on = N.load(), N._dtype(self.y), self.status.device
        kept = (*N._fixed(self.codes), *N._fixed(self.scales))
        self._sum = N._fixed(self.sum)
        self._forward = (eps, *N._fixed(self.y), *kept, N._fixed(self.stats)[0], self.status.data_ptr())
        if train:
            self._backward = (*kept, self.stats.data_ptr())
            self._grads = (*N._fixed(self.dx), self.dgamma.data_ptr(), self.dbeta.data_ptr() if self.layer else 0,
                           self.workspace.data_ptr(), self.workspace.numel())

    def _check(self, x: torch.Tensor, other: torch.Tensor | None) -> int:
        m, c = x.shape
        if m > self.M or c != self.C:
            raise ValueError(f"a tensor of [{self.M}, {self.C}] expected, not {(m, c)}")
        if x.dtype != self.dtype:
            raise TypeError(f"a tensor of {self.dtype} expected, not {x.dtype}")
        if x.device != self._on:
            raise _elsewhere(x, self._on)
        if other is not None:
            if other.shape != x.shape or other.dtype != x.dtype:
                raise ValueError(f"tensors of one shape and type expected, not {(m, c)} and {tuple(other.shape)}")
            if other.device != self._on:
                raise _elsewhere(other, self._on)
        return m

    def _param(self, p: torch.Tensor) -> int:
        if p.shape != (self.C,) or p.dtype != torch.float32 or not p.is_contiguous():
            raise ValueError(f"gamma and beta are fp32 vectors of {self.C}")
        if p.device != self._on:
            raise _elsewhere(p, self._on)
        return p.data_ptr()

    def forward(self, x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor | None = None,
                residual: torch.Tensor | None = None, stream=None):
        """y and, where a residual is added, the sum (else None)."""
        m = self._check(x, residual)
        if (beta is not None) != self.layer or (residual is not None) != (self.sum is not None):
            raise ValueError("beta goes with the layer norm, a residual with residual=True")
        res = (0, 0) if residual is None else (residual.data_ptr(), N._ld(residual))
        N._check(self._lib.shiftquant_norm8_forward(
            x.data_ptr(), self._dtype, m, self.C, N._ld(x), *res, *self._sum, self._param(gamma),
            0 if beta is None else self._param(beta), *self._forward, N._stream(stream)))
        self._rows = m if self.train else None
        if m == self.M:
            return self.y, self.sum
        return self.y[:m], None if self.sum is None else self.sum[:m]

    def backward(self, dy: torch.Tensor, gamma: torch.Tensor, dsum: torch.Tensor | None = None, stream=None):
        """dx (with dsum, the gradient that reaches the sum another way, added), dgamma and dbeta
        (None for the root-mean-square norm), of as many rows as the last forward kept."""
        m = self._check(dy, dsum)
        if m != self._rows:
            raise _not_kept(m, self._rows)
        ds = (0, 0) if dsum is None else (dsum.data_ptr(), N._ld(dsum))
        N._check(self._lib.shiftquant_norm8_backward(
            dy.data_ptr(), self._dtype, m, self.C, N._ld(dy), *self._backward, self._param(gamma), *ds, *self._grads,
            N._stream(stream)))
        return self.dx if m == self.M else self.dx[:m], self.dgamma, self.dbeta


class Mx4MlpBlock:
    """A pre-norm MLP block, x + W2 f(W1 norm(x)), in 4-bit products and 8-bit checkpoints: an RMS
    norm, a gated or plain activation between two mx4 linear layers, and the residual sum of the
    previous block's output folded into the norm.

    forward(delta, x): x_new = x + delta (the residual stream), out = W2 f(W1 norm(x_new)), which the
    next block adds.  backward(dout, dx_new, seed) returns d(delta) = d(x) and leaves the weights'
    gradients in dw1, dw2 and dgamma.  It takes the draws of seed for dout and of seed + 1 for the
    gradient between the products: calls whose draws are not to meet have seeds two apart or more.

    share: a block made alike, whose buffers of what only one block at a time needs this one takes
    too.  A chain of blocks that share with its first holds one set of them; x_new and the gradient
    of the stream then pass along the chain in place, and a block's own are its weights, their
    gradients, and the 8-bit and 4-bit codes that its backward pass needs.  Outputs stay until
    the next block's call, and calls are in order on one stream."""

    def __init__(self, M: int, C: int, F: int, dtype: torch.dtype, device, act: str = "silu", gated: bool = True,
                 share: "Mx4MlpBlock | None" = None):
        parts = 2 if gated else 1
        norm, up, mid, down = (None,) * 4 if share is None else (share.norm, share.up, share.act, share.down)
        self.norm = Norm8(M, C, dtype, "rms", device, residual=True, share=norm)
        self.up = Mx4Linear(M, C, parts * F, dtype, device, share=up)
        self.act = Act8(M, F, dtype, act, gated, device, share=mid)
        self.down = Mx4Linear(M, F, C, dtype, device, share=down)

    def set_weights(self, gamma: torch.Tensor, w1: torch.Tensor, w2: torch.Tensor, stream=None) -> None:
        """gamma [C] (fp32, read at each call), w1 [C, F or 2 F], w2 [F, C]."""
        self.gamma = gamma
        self.up.set_weight(w1, stream)
        self.down.set_weight(w2, stream)

    def forward(self, delta: torch.Tensor, x: torch.Tensor, stream=None):
        y, x_new = self.norm.forward(delta, self.gamma, residual=x, stream=stream)
        return self.down.forward(self.act.forward(self.up.forward(y, stream), stream), stream), x_new

    def backward(self, dout: torch.Tensor, dx_new: torch.Tensor, seed: int, stream=None) -> torch.Tensor:
        da, self.dw2 = self.down.backward(dout, seed, stream)
        dy, self.dw1 = self.up.backward(self.act.backward(da, stream), seed + 1, stream)
        dx, self.dgamma, _ = self.norm.backward(dy, self.gamma, dx_new, stream)
        return dx

    def status(self) -> int:
        """The device status bits of all calls so far (synchronises)."""
        s = 0
        for part in (self.norm, self.up, self.act, self.down):
            s |= int(part.status.item())
        return s
