"""Device-memory plumbing around the C ABI: allocates the n x d state with
PyTorch-ROCm, binds it, and keeps the tensors alive.  No arithmetic of the
method happens here - every update goes through libgpga."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


def _current_stream(index: int) -> int:
    """Address of torch's current stream on a device."""
    return torch.cuda.current_stream(index).cuda_stream


# the same without building a Stream object (0.1 us for 2), where this torch has it
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)

_DTYPE = {torch.float32: B.GPGA_F32, torch.bfloat16: B.GPGA_BF16, torch.float16: B.GPGA_F16}

# smallest p that drops anything: the library keeps p as fp32 and then to 16 bits, so what rounds to 2^-17 or more
_LEAST_P = 2.0 ** -17 * (1 - 2.0 ** -25)


class Simulation:
    """n simulated nodes with d parameters each on one GPU.

    Owns four (n, ld) fp32 CUDA tensors (x, x_new, m, g) and a libgpga context
    bound to them on ``stream`` (a torch.cuda.Stream; default: current stream).
    """

    def __init__(self, n: int, d: int, *, topology: str, H: int, lr: float, momentum: float = 0.0,
                 ld: int | None = None, device: str = "cuda:0", stream: torch.cuda.Stream | None = None,
                 x0=None, alloc_m: bool | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("libgpga needs a GPU (torch.cuda.is_available() is False)")
        self.n, self.d = n, d
        self.ld = d if ld is None else ld
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._stream_address = self.stream.cuda_stream
        self.ctx = B.gpga_create(n, d, topology, H, lr, momentum)
        with torch.cuda.stream(self.stream):
            self._bufs = [torch.empty((n, self.ld), dtype=torch.float32, device=self.device) for _ in range(2)]
            need_m = (momentum != 0.0) if alloc_m is None else alloc_m
            self.m = torch.zeros((n, self.ld), dtype=torch.float32, device=self.device) if need_m else None
            self.g = torch.zeros((n, self.ld), dtype=torch.float32, device=self.device)
        self._device_index = self.g.get_device()
        self._addr = {t.data_ptr(): t for t in self._bufs}
        B.gpga_bind(self.ctx, self._bufs[0], self._bufs[1], self.m, self.g, self.ld, self.stream.cuda_stream)
        self._keep = []
        x0_dev = None
        if x0 is not None:
            x0_dev = torch.as_tensor(np.asarray(x0, dtype=np.float32)).to(self.device)
            self._keep.append(x0_dev)
        self.stream.synchronize()
        B.gpga_reset(self.ctx, x0_dev)

    # -- state access -----------------------------------------------------------
    @property
    def X(self) -> torch.Tensor:
        """Live iterates, (n, d) view of the (n, ld) buffer."""
        x = self._addr[B.gpga_current_x(self.ctx)]
        return x[...] if self.ld == self.d else x[:, : self.d]     # the same view; a whole one takes half the time

    @property
    def G(self) -> torch.Tensor:
        return self.g[...] if self.ld == self.d else self.g[:, : self.d]

    @property
    def M(self):
        return None if self.m is None else self.m[:, : self.d]

    @property
    def k(self) -> int:
        return B.gpga_iter(self.ctx)

    def set_state(self, X=None, M=None, G=None, k=None):
        """Overwrite device state from host arrays (lock-step comparisons)."""
        with torch.cuda.stream(self.stream):
            if X is not None:
                self.X.copy_(torch.as_tensor(np.asarray(X, dtype=np.float32)))
            if M is not None and self.m is not None:
                self.M.copy_(torch.as_tensor(np.asarray(M, dtype=np.float32)))
            if G is not None:
                self.G.copy_(torch.as_tensor(np.asarray(G, dtype=np.float32)))
        self.stream.synchronize()
        if k is not None:
            B.gpga_set_iter(self.ctx, k)

    # -- problems ------------------------------------------------------------------
    def _upload(self, a, dtype):
        t = torch.as_tensor(np.ascontiguousarray(a)).to(dtype).to(self.device)
        self._keep.append(t)
        return t

    def problem_lsq(self, A, b):
        A_d, b_d = self._upload(A, torch.float32), self._upload(b, torch.float32)
        B.gpga_problem_lsq(self.ctx, A_d, b_d, A.shape[1])
        return A_d, b_d

    def problem_logreg(self, feat, y):
        f_d, y_d = self._upload(feat, torch.float32), self._upload(y, torch.float32)
        B.gpga_problem_logreg(self.ctx, f_d, y_d, feat.shape[1])
        return f_d, y_d

    def problem_logreg_virtual(self, seed: int, y, mu_var: float):
        y_d = self._upload(y, torch.float32)
        B.gpga_problem_logreg_virtual(self.ctx, seed, y_d, y.shape[1], mu_var)
        return y_d

    def problem_synthetic(self, seed: int, grad_var: float):
        B.gpga_problem_synthetic(self.ctx, seed, grad_var)

    def upload_batches(self, idx):
        """(T, n, B) int32 minibatch table -> device tensor."""
        return self._upload(idx, torch.int32)

    # -- the iteration -------------------------------------------------------------
    def local_grad(self, batch_idx=None):
        if batch_idx is None:
            B.gpga_local_grad(self.ctx, None, 0)
        else:
            B.gpga_local_grad(self.ctx, batch_idx, batch_idx.shape[-1])

    def local_loss(self, batch_idx=None) -> torch.Tensor:
        out = torch.empty(self.n, dtype=torch.float32, device=self.device)
        B.gpga_local_loss(self.ctx, batch_idx, 0 if batch_idx is None else batch_idx.shape[-1], out)
        return out

    def step(self):
        B.gpga_step(self.ctx)

    def set_mixing(self, W):
        """Attach a dense (n, n) doubly stochastic W: its non-zeros are handed over in CSR form."""
        W = np.asarray(W)
        rows, cols = np.nonzero(W)          # row-major order
        ptr = np.concatenate([[0], np.cumsum(np.bincount(rows, minlength=self.n))])
        B.gpga_set_mixing_csr(self.ctx, ptr, cols, W[rows, cols].astype(np.float32))

    @property
    def beta(self) -> float:
        return B.gpga_mixing_beta(self.ctx)

    def set_nesterov(self, on: bool = True):
        B.gpga_set_nesterov(self.ctx, on)

    @property
    def lr(self) -> float:
        """Step size the next step will use."""
        return B.gpga_lr(self.ctx)

    def run(self, T: int, batch_table=None):
        """T iterations (gradient + step) from one call; batch_table: (>= T, n, B) int32 device tensor."""
        if batch_table is None:
            B.gpga_run(self.ctx, T, None, 0)
        else:
            assert batch_table.shape[0] >= T and batch_table.is_contiguous()
            B.gpga_run(self.ctx, T, batch_table, batch_table.shape[-1])

    def aga_enable(self, H_init: int, warmup_iters: int, H_max: int):
        B.gpga_aga_enable(self.ctx, H_init, warmup_iters, H_max)

    def aga_step(self, loss: torch.Tensor):
        B.gpga_aga_step(self.ctx, loss)

    @property
    def period(self) -> int:
        return B.gpga_period(self.ctx)

    def consensus_error(self) -> float:
        return B.gpga_consensus_error(self.ctx)

    def consensus_error_static(self, out: torch.Tensor):
        """Consensus distance into ``out`` (one float64 on the device), asynchronously, no allocation."""
        B.gpga_consensus_error_static(self.ctx, out)

    def attach_trace(self, capacity: int) -> torch.Tensor:
        """Device array that receives the consensus distance after every step (no host sync)."""
        self.trace = torch.full((capacity,), float("nan"), dtype=torch.float64, device=self.device)
        self.stream.synchronize()
        B.gpga_set_trace(self.ctx, self.trace, capacity)
        return self.trace

    def mean(self) -> torch.Tensor:
        out = torch.empty(self.d, dtype=torch.float32, device=self.device)
        B.gpga_mean(self.ctx, out)
        return out

    # -- operators of language models --------------------------------------------------
    # Activations are (n, T, D) tensors whose tokens lie a common number of elements apart (rows of a wider tensor are
    # fine); parameters are named by their column offset in X, their gradients land in the same columns of G.  What the
    # calls return is allocated for, and written on, the simulation's stream.  The gradients are calls of their own: torch's
    # autograd knows nothing of these, so activations that it follows are refused (hand over x.detach(), or call under no_grad).
    def _foreign(self) -> bool:
        """Whether torch's current stream is another one than the simulation's."""
        return _current_stream(self._device_index) != self._stream_address

    def _empty(self, shape, dtype, foreign: bool):
        """Memory of the simulation's stream."""
        if not foreign:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _like(self, x: torch.Tensor, ld: int, foreign: bool):
        """Memory for activations beside ``x``: rows as far apart."""
        if foreign:
            with torch.cuda.stream(self.stream):
                return self._like(x, ld, False)
        if x.is_contiguous():
            return torch.empty_like(x)
        n, T, D = x.shape
        return torch.empty((n, T, ld), dtype=x.dtype, device=self.device)[..., :D]

    def _tokens(self, t: torch.Tensor) -> int:
        """Tokens a node of an (n, T) int32 tensor."""
        if (t.dtype != torch.int32 or t.dim() != 2 or t.shape[0] != self.n or not t.is_contiguous() or
                t.get_device() != self._device_index):
            raise ValueError(f"expected a contiguous (n = {self.n}, T) int32 tensor on the simulation's GPU, "
                             f"got {tuple(t.shape)} {t.dtype} on {t.device}")
        return t.shape[1]

    def _rows(self, first: torch.Tensor, *others):
        """(T, D, ld, dtype) of activations of one call."""
        shape, dtype = first.shape, first.dtype
        if len(shape) != 3 or shape[0] != self.n or dtype not in _DTYPE or first.get_device() != self._device_index:
            raise ValueError(f"expected an (n = {self.n}, T, D) fp32, bf16 or fp16 tensor on the simulation's GPU, "
                             f"got {tuple(shape)} {dtype} on {first.device}")
        n, T, D = shape
        ld = D if first.is_contiguous() else first.stride(1) if T > 1 else first.stride(0) if n > 1 else D
        for t in (first, *others):
            if t is None:
                continue
            if t.requires_grad and torch.is_grad_enabled():
                raise ValueError("an activation requires grad: these calls are not recorded for torch's backward()")
            if t is not first and (t.shape != shape or t.dtype != dtype or t.get_device() != self._device_index):
                raise ValueError("the activations of a call differ in shape, type or device")
            if ld == D and t.is_contiguous():
                continue
            if t.numel() and (ld < D or (D > 1 and t.stride(2) != 1) or (T > 1 and t.stride(1) != ld) or
                              (n > 1 and t.stride(0) != T * ld)):
                raise ValueError("the activations of a call need rows that are dense and a common number of elements apart")
        return T, D, max(ld, D), _DTYPE[dtype]

    def _used(self, *tensors):
        """Memory that another stream allocated is not handed out again before this stream is through with it."""
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)

    def embed(self, tokens: torch.Tensor, table_off: int, V: int, D: int, *, scale: float = 1.0,
              dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """scale * E_i[tokens]: (n, T, D); tokens below 0 give zeros."""
        if dtype not in _DTYPE:
            raise ValueError(f"dtype must be fp32, bf16 or fp16, got {dtype}")
        T, foreign = self._tokens(tokens), self._foreign()
        y = self._empty((self.n, T, D), dtype, foreign)
        B.gpga_embed(self.ctx, tokens, T, table_off, V, D, scale, y, D, _DTYPE[dtype])
        if foreign:
            self._used(tokens)
        return y

    def embed_grad(self, tokens: torch.Tensor, dy: torch.Tensor, table_off: int, V: int, *, scale: float = 1.0,
                   accumulate: bool = False):
        """Gradient of the table into G[:, table_off : table_off + V*D]."""
        T, D, ld, dt = self._rows(dy)
        if self._tokens(tokens) != T:
            raise ValueError("tokens and dy differ in their tokens a node")
        B.gpga_embed_grad(self.ctx, tokens, T, table_off, V, D, scale, dy, ld, dt, accumulate)
        if self._foreign():
            self._used(tokens, dy)

    def dropout(self, x: torch.Tensor, p: float, *, seed: int, layer: int = 0, residual: torch.Tensor | None = None,
                out: torch.Tensor | None = None) -> torch.Tensor:
        """residual + mask * x / (1 - p), the mask that of iteration k; with x = a gradient, its backward pass."""
        T, D, ld, dt = self._rows(x, residual, out)
        foreign = self._foreign()
        y = self._like(x, ld, foreign) if out is None else out
        B.gpga_dropout(self.ctx, x, residual, T, D, ld, dt, p, seed, layer, y)
        if foreign:
            self._used(x, residual, out)
        return y

    def layer_norm(self, x: torch.Tensor, gamma_off: int, beta_off: int, *, eps: float = 1e-5,
                   residual: torch.Tensor | None = None, p: float = 0.0, seed: int = 0, layer: int = 0):
        """(y, u, stats): layer norm y of u = residual + dropout(x); u is x itself where there is neither."""
        T, D, ld, dt = self._rows(x, residual)
        foreign = self._foreign()
        plain = residual is None and p == 0.0
        y = self._like(x, ld, foreign)
        u = None if plain else self._like(x, ld, foreign)
        stats = self._empty((self.n, T, 2), torch.float32, foreign)
        B.gpga_layer_norm(self.ctx, x, residual, T, D, ld, dt, p, seed, layer, gamma_off, beta_off, eps, u, y, stats)
        if foreign:
            self._used(x, residual)
        return y, x if plain else u, stats

    def layer_norm_grad(self, dy: torch.Tensor, u: torch.Tensor, stats: torch.Tensor, gamma_off: int, beta_off: int, *,
                        p: float = 0.0, seed: int = 0, layer: int = 0, more: torch.Tensor | None = None,
                        accumulate: bool = False):
        """(du, dx): gradients of the residual and of x; those of gamma and beta land in G.  dx is du where p is 0."""
        T, D, ld, dt = self._rows(dy, u, more)
        if stats.dtype != torch.float32 or stats.shape != (self.n, T, 2) or not stats.is_contiguous() or stats.get_device() != self._device_index:
            raise ValueError("stats are the (n, T, 2) fp32 pairs that layer_norm returns")
        foreign = self._foreign()
        du = self._like(dy, ld, foreign)
        drops = _LEAST_P <= p < 1.0     # others keep everything, or are the library's to refuse
        dx = self._like(dy, ld, foreign) if drops else None
        B.gpga_layer_norm_grad(self.ctx, dy, u, stats, more, T, D, ld, dt, p, seed, layer, gamma_off, beta_off, du, dx,
                               accumulate)
        if foreign:
            self._used(dy, u, stats, more)
        return du, du if dx is None else dx

    def token_loss(self, logits: torch.Tensor, labels: torch.Tensor, *, grad=True, grad_scale: float = 1.0):
        """(loss, dlogits): n mean losses, and the gradient (None if ``grad`` is False, in the tensor ``grad`` if it
        is one, e.g. ``logits`` itself)."""
        into = grad if isinstance(grad, torch.Tensor) else None
        T, V, ld, dt = self._rows(logits, into)
        if self._tokens(labels) != T:
            raise ValueError("labels and logits differ in their tokens a node")
        foreign = self._foreign()
        loss = self._empty((self.n,), torch.float32, foreign)
        dlogits = into if into is not None else self._like(logits, ld, foreign) if grad else None
        B.gpga_token_loss(self.ctx, logits, labels, T, V, ld, dt, grad_scale, loss, dlogits)
        if foreign:
            self._used(logits, labels, into)
        return loss, dlogits

    def gated_ff(self, x: torch.Tensor, gate_off: int, up_off: int, down_off: int, F: int, *, act: str = "silu",
                 keep: bool = False):
        """(y, hidden): y = Wd_i (act(Wg_i x) * Wu_i x); hidden = [Wg_i x | Wu_i x], (n, T, 2F), for the backward pass if
        ``keep``, else None."""
        T, D, ld, dt = self._rows(x)
        if act not in B.ACTIVATION:
            raise ValueError(f"act must be one of {sorted(B.ACTIVATION)}, got {act!r}")
        if not 1 <= F <= 1 << 21:
            raise ValueError(f"F must be 1..2^21, got {F}")
        foreign = self._foreign()
        y = self._like(x, ld, foreign)
        hidden = self._empty((self.n, T, 2 * F), x.dtype, foreign) if keep else None
        B.gpga_gated_ff(self.ctx, x, T, D, F, ld, dt, B.ACTIVATION[act], gate_off, up_off, down_off, hidden, y)
        if foreign:
            self._used(x)
        return y, hidden

    def gated_ff_grad(self, dy: torch.Tensor, x: torch.Tensor, hidden: torch.Tensor, gate_off: int, up_off: int, down_off: int,
                      *, act: str = "silu", accumulate: bool = False) -> torch.Tensor:
        """dx; the gradients of the three matrices land in G."""
        T, D, ld, dt = self._rows(dy, x)
        if act not in B.ACTIVATION:
            raise ValueError(f"act must be one of {sorted(B.ACTIVATION)}, got {act!r}")
        if (hidden.dtype != x.dtype or hidden.dim() != 3 or hidden.shape[:2] != (self.n, T) or hidden.shape[2] % 2 or
                not hidden.is_contiguous() or hidden.get_device() != self._device_index):
            raise ValueError("hidden is the contiguous (n, T, 2F) tensor of the activations' type that gated_ff keeps, on the simulation's GPU")
        if hidden.requires_grad and torch.is_grad_enabled():
            raise ValueError("an activation requires grad: these calls are not recorded for torch's backward()")
        foreign = self._foreign()
        dx = self._like(dy, ld, foreign)
        B.gpga_gated_ff_grad(self.ctx, dy, x, hidden, T, D, hidden.shape[2] // 2, ld, dt, B.ACTIVATION[act], gate_off, up_off,
                             down_off, dx, accumulate)
        if foreign:
            self._used(dy, x, hidden)
        return dx

    def orthogonalize(self, off: int, rows: int, cols: int, *, count: int = 1, velocity: torch.Tensor | None = None,
                      mu: float = 0.0, nesterov: bool = False, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315),
                      eps: float = 1e-7, scale: float = 1.0):
        """The gradients of ``count`` matrices of rows x cols in G[:, off:] become scale times orthogonalised updates;
        ``velocity``: (n, count * rows * cols) fp32, the running sums, updated in place."""
        if velocity is not None:
            if (velocity.dtype != torch.float32 or tuple(velocity.shape) != (self.n, count * rows * cols) or
                    not velocity.is_contiguous() or velocity.get_device() != self._device_index):
                raise ValueError("velocity is a contiguous (n, count * rows * cols) fp32 tensor on the simulation's GPU")
            if velocity.requires_grad and torch.is_grad_enabled():
                raise ValueError("velocity requires grad: these calls are not recorded for torch's backward()")
        a, b, c = coefficients
        B.gpga_orthogonalize(self.ctx, off, rows, cols, count, velocity, mu, nesterov, steps, a, b, c, eps, scale)
        if velocity is not None and self._foreign():
            self._used(velocity)

    def tune(self, launches: int = 16):
        """Let the pacing controllers settle (state arrays are left with unspecified contents)."""
        B.gpga_tune(self.ctx, launches)

    def query(self, name: str) -> float:
        return B.gpga_query(self.ctx, name)

    def set_option(self, name: str, value: int):
        B.gpga_set_option(self.ctx, name, value)

    def close(self):
        if self.ctx is not None:
            B.gpga_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
