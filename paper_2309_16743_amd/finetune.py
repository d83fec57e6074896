"""One trained surrogate adapted to several ensembles at once.

An ensemble with other solver settings or materials needs a surrogate of its own,
but not a copy of every weight (the output layer of a 1000x1000 field has 10^9):
each layer of the trained surrogate stays frozen and gets a bank of low-rank
adapters, one per ensemble (include/adapters.h).  A batch may mix rows of all
ensembles in any order, as a buffer fed by all of them hands them out; one
backward gives every ensemble's gradients, which are clipped by their global norm
and applied by one Adam over the list (include/gradients.h).

    sur = Surrogate(widths, ...)                    # trained
    tuner = AdapterTrainer(sur, n_ensembles=4, rank=8, batch=256)
    tuner.train_step(x, u, ids)                     # ids: int32 device tensor, one ensemble per row
    tuner.predict(x, ids, y)

python -m paper_2309_16743_amd.finetune runs a small demonstration.
"""
from __future__ import annotations

import contextlib
import math
from typing import Optional

import torch

from . import OT_BF16, OT_FP32, AdamTensors, LowRankAdapters, Surrogate


def _padded(shape, dtype, device) -> torch.Tensor:
    """Zeros whose rows are padded to whole 16-byte pieces: (whole array, view without the padding)."""
    n = shape[-1]
    full = torch.zeros(*shape[:-1], (n + 7) // 8 * 8, dtype=dtype, device=device)
    return full, full[..., :n]


class AdapterTrainer:
    """Low-rank adapters of a trained surrogate for n_ensembles ensembles.

    precision OT_BF16 holds the frozen weights, activations and the products' copies of
    the adapters in bf16 (the first layer, fed by raw temperatures, stays fp32 as in
    the surrogate); master adapters, gradients and Adam are fp32.  alpha: the adapters'
    scale is alpha / rank.  max_norm: bound of the gradients' global norm (0: none).
    up starts at zero, so the adapted surrogate starts as the trained one.

    A call runs on the stream current when it is made, behind the trainer's call before it
    whichever stream that ran on.  With a stream given here every call runs on that one,
    behind what the caller's current stream holds, and the current stream waits for it in
    turn, so inputs and results belong to the current stream in both cases.  A call under
    capture waits for nothing but its own stream, or forks from it and joins it again; the
    order of replays among other calls is the caller's."""

    def __init__(self, surrogate: Surrogate, n_ensembles: int, rank: int = 8, batch: int = 1024,
                 precision: int = OT_FP32, lr: float = 1e-3, alpha: Optional[float] = None, max_norm: float = 1.0,
                 seed: int = 0, device=None, stream: Optional[torch.cuda.Stream] = None):
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self.widths, self.batch, self.rank, self.n_ensembles = surrogate.widths, batch, rank, n_ensembles
        self.max_norm = max_norm
        self.stream = stream
        # where the buffers below are allocated, and where the last call ran
        self._home = self._last = stream if stream is not None else torch.cuda.current_stream()
        op = torch.bfloat16 if precision == OT_BF16 else torch.float32
        layers = len(self.widths) - 1
        with torch.cuda.stream(self._home):
            gen = torch.Generator(device=dev)
            gen.manual_seed(seed)
            self.scale = torch.full((n_ensembles,), (float(rank) if alpha is None else alpha) / rank, device=dev)
            self.banks, self.w, self.bias, self.acts, self.t = [], [], [], [], []
            self.down, self.up, self.ddown, self.dup = [], [], [], []
            params, grads, copies = [], [], []
            for l in range(layers):
                n_in, n_out = self.widths[l], self.widths[l + 1]
                lt = torch.float32 if l == 0 else op
                W, b = surrogate.get_params(l)
                w = _padded((n_out, n_in), lt, dev)[1]
                w.copy_(torch.from_numpy(W).to(dev))
                self.w.append(w)
                self.bias.append(torch.from_numpy(b).to(dev))
                self.banks.append(LowRankAdapters(n_in, n_out, rank, n_ensembles, max_rows=batch,
                                                  precision=OT_BF16 if lt == torch.bfloat16 else OT_FP32))
                for dim, use, grad in ((n_in, self.down, self.ddown), (n_out, self.up, self.dup)):
                    master, view = _padded((n_ensembles, rank, dim), torch.float32, dev)
                    if use is self.down:
                        bound = 1.0 / math.sqrt(n_in)
                        view.uniform_(-bound, bound, generator=gen)
                    params.append(master)
                    g, gview = _padded((n_ensembles, rank, dim), torch.float32, dev)
                    grads.append(g)
                    grad.append(gview)
                    if lt == torch.bfloat16:
                        c = master.to(torch.bfloat16)
                        copies.append(c)
                        use.append(c[..., :dim])
                    else:
                        copies.append(None)
                        use.append(view)
                self.t.append(torch.zeros(batch, rank, device=dev))
                # activations: what the next layer reads, in its type
                self.acts.append(_padded((batch, n_out), torch.float32 if l == layers - 1 else op, dev)[1])
            # gradients of the output, of the activations, and the first layer's in its own type
            self.dy = _padded((batch, self.widths[-1]), lt, dev)[1]
            self.dx = [None] + [_padded((batch, self.widths[l]), op, dev)[1] for l in range(1, layers)]
            self.dy_first = None
            if layers > 1 and op != torch.float32:
                self.dy_first = _padded((batch, self.widths[1]), torch.float32, dev)[1]
            self.params, self.grads = params, grads
            self.m = [torch.zeros_like(p) for p in params]
            self.v = [torch.zeros_like(p) for p in params]
            self.adam = AdamTensors(params, grads, self.m, self.v, copies=copies, lr=lr)
            self.norm = torch.zeros(1, device=dev)
            self.loss = torch.zeros(1, device=dev)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)

    @contextlib.contextmanager
    def _ordered(self):
        """The call's stream as the current one, in order with the caller's stream and the call before."""
        here = torch.cuda.current_stream()
        if self.stream is not None:
            if self.stream == here:
                yield
                return
            self.stream.wait_stream(here)
            with torch.cuda.stream(self.stream):
                yield
            here.wait_stream(self.stream)
            return
        if not torch.cuda.is_current_stream_capturing():
            if self._last != here:
                here.wait_stream(self._last)
            self._last = here
        yield

    @property
    def n_layers(self) -> int:
        return len(self.widths) - 1

    def _forward(self, x, ids, out=None, save: bool = False):
        n = x.shape[0]
        if n > self.batch:
            raise ValueError(f"{n} rows, the trainer holds {self.batch}")
        a = x
        for l, bank in enumerate(self.banks):
            last = l + 1 == self.n_layers
            y = out if last and out is not None else self.acts[l][:n]
            bank.forward(a, self.w[l], self.down[l], self.up[l], ids, y, bias=self.bias[l], scale=self.scale,
                         t=self.t[l][:n] if save else None, relu=not last)
            a = y
        return a

    def predict(self, x, ids, y) -> None:
        """y (fp32 or bf16, rows padded to whole 16-byte pieces) of up to `batch` rows x, each with its
        ensemble's adapters (an id outside the bank: the surrogate as it was)."""
        with self._ordered():
            self._forward(x, ids, out=y)

    def train_step(self, x, u, ids) -> None:
        """One step on 1 to `batch` rows x -> u of ensembles ids: mean squared error, gradients of every adapter,
        clipping, Adam.  self.loss and self.norm receive the loss and the gradients' norm before clipping."""
        n = x.shape[0]
        if n < 1:
            raise ValueError("x: expected at least one row")
        if tuple(u.shape) != (n, self.widths[-1]):
            raise ValueError(f"u: expected a {n} x {self.widths[-1]} tensor")
        with self._ordered():
            y = self._forward(x, ids, save=True)
            r = y - u
            self.loss.copy_((r * r).mean())
            last = self.n_layers - 1
            dy = self.dy[:n]
            dy.copy_(r * (2.0 / r.numel()))
            for l in range(last, -1, -1):
                inp = x if l == 0 else self.acts[l - 1][:n]
                dx = None if l == 0 else self.dx[l][:n]
                self.banks[l].backward(inp, self.w[l], self.down[l], self.up[l], ids, dy, self.t[l][:n],
                                       self.ddown[l], self.dup[l], dx=dx, scale=self.scale, relu_input=l > 0)
                if l > 0:
                    dy = dx
                    if l == 1 and self.dy_first is not None:              # the first layer computes in fp32
                        dy = self.dy_first[:n]
                        dy.copy_(dx)
            self.adam.step(self.max_norm, self.norm)

    def close(self) -> None:
        if self._last != self._home:           # the buffers go back to the allocations of the stream they are from
            self._home.wait_stream(self._last)
            self._last = self._home
        for b in self.banks:
            b.close()
        self.adam.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def main() -> None:
    """A surrogate of 16x16 fields trained on one ensemble, then adapted to three whose fields are damped and shifted."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(0)
    widths, n = (6, 64, 64, 256), 96
    col = torch.arange(256, device=dev) / 256
    mixer = torch.rand(6, 8, generator=gen, device=dev)
    modes = torch.stack([torch.sin((k + 1) * math.pi * col) for k in range(8)])

    def sample(k):
        x = torch.zeros(n, 8, device=dev)[:, :6]
        x.copy_(torch.rand(n, 6, generator=gen, device=dev))
        u = torch.tanh(x @ mixer) @ modes
        return x, (u if k < 0 else (0.6 + 0.3 * k) * u + 0.2 * k).contiguous()

    sur = Surrogate(widths, lr=2e-3, seed=1, max_batch=n)
    for _ in range(400):
        sur.train_step(*sample(-1))
    tuner = AdapterTrainer(sur, n_ensembles=3, rank=4, batch=n, lr=4e-3, max_norm=1.0)

    def mixed():
        ids = torch.randint(0, 3, (n,), generator=gen, device=dev).to(torch.int32)
        x, _ = sample(-1)
        base = torch.tanh(x @ mixer) @ modes
        k = ids.float()[:, None]
        return x, (0.6 + 0.3 * k) * base + 0.2 * k, ids

    for step in range(601):
        tuner.train_step(*mixed())
        if step % 200 == 0:
            torch.cuda.synchronize()
            print(f"step {step}: loss {tuner.loss.item():.5f}, gradient norm {tuner.norm.item():.4f}", flush=True)
    tuner.close()
    sur.close()


if __name__ == "__main__":
    main()
