"""A block of several operators trained by one local Forward-Forward loss.

The paper's layers are single linear or convolution layers, each with its own loss (Sec. III, IV-B).  A `LocalBlock` puts a
pre-norm MLP in the place of such a layer,

    y = x + W2 act(W1 layernorm(x)),      goodness G = ||y||^2 per sample, losses of Eq. 1 / Eq. 2 against theta,

so that the loss stays local to the block and the gradient is propagated inside it only.  Everything the block keeps between
its forward and its backward pass is held in 8 bits (beside one FP32 number a row): one checkpoint of the normalised input (it
serves the layer norm's backward pass and, with gamma and beta folded in, the gradient of W1), one of the activation's input
and one of its output.  What a pass computes on the way is freed when it returns.  The workspace of the library's calls
(2 bytes per value of the wider weight gradient's input and more) belongs to the context; blocks that run one after another
on a stream share one.  The two forward products and the two input gradients are plain matrix products.

Run as a program it trains a small block on seeded synthetic samples and prints the loss:

    python -m paper_2506_22771_b200.local_block [--steps N] [--rows B] [--width D] [--hidden H]
"""
from __future__ import annotations

import argparse

from . import binding as ffb

_ACT = {"relu": ffb.FF_ACT_RELU, "gelu": ffb.FF_ACT_GELU, "silu": ffb.FF_ACT_SILU}


def _descs(width, hidden, dtype):
    """Descriptors whose workspaces a block needs: the layer norm's and the two weight gradients'."""
    import torch
    codes = {torch.float32: ffb.FF_F32, torch.bfloat16: ffb.FF_BF16, torch.float16: ffb.FF_F16}
    if dtype not in codes:
        raise ValueError(f"dtype has to be float32, bfloat16 or float16: {dtype}")
    code = codes[dtype]
    return (ffb.ff_layernorm_desc(cols=width, dtype=code, index=0), ffb.ff_ckpt8_wgrad_desc(N=hidden, K=width, dtype=code),
            ffb.ff_ckpt8_wgrad_desc(N=width, K=hidden, dtype=code))


def _address(name, t, rows, cols, dtype, device):
    """(address, row pitch) of a tensor that the kernels are about to read; they see nothing but these, so its size, type, place and
    strides have to be right."""
    if tuple(t.shape) != (rows, cols):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, the block takes {(rows, cols)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, the block computes in {dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the block on {device}")
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols):
        raise ValueError(f"{name} has strides {t.stride()}; its rows have to be contiguous and apart from each other")
    return t.data_ptr(), max(t.stride(0), cols)


class LocalBlock:
    """Parameters, checkpoints and gradients of one block for batches of `rows` samples (positive and negative ones together).
    context: a binding.Context that blocks share, with at least the `workspace_bytes` of each; by default the block has its own."""

    def __init__(self, rows: int, width: int, hidden: int, act: str = "gelu", dtype=None, eps: float = 1e-5, seed: int = 0,
                 stochastic: bool = True, device_index: int = 0, context=None):
        import torch
        self.rows, self.width, self.hidden = rows, width, hidden
        self.dtype = dtype or torch.bfloat16
        if act not in _ACT:
            raise ValueError(f"act has to be one of {sorted(_ACT)}: {act!r}")
        self.ln, self.g1, self.g2 = _descs(width, hidden, self.dtype)
        need = self.workspace_bytes(rows, width, hidden, self.dtype)
        if context is not None and context.workspace.numel() < need:
            raise ValueError(f"the context's workspace has {context.workspace.numel()} bytes, the block needs {need}")
        dev = self.device = torch.device(f"cuda:{device_index}")
        gen = torch.Generator(device=dev).manual_seed(seed)
        new = lambda *s: torch.zeros(s, device=dev)
        self.gamma, self.beta = torch.ones(width, device=dev), new(width)
        self.W1 = torch.randn((hidden, width), generator=gen, device=dev) * width ** -0.5
        self.W2 = torch.randn((width, hidden), generator=gen, device=dev) * (0.5 * hidden ** -0.5)
        self.dgamma, self.dbeta, self.dW1, self.dW2 = new(width), new(width), new(hidden, width), new(width, hidden)
        self.rstd = new(rows)
        self.c_norm, self.c_in, self.c_out = ffb.Ckpt8(rows, width, dev), ffb.Ckpt8(rows, hidden, dev), ffb.Ckpt8(rows, hidden, dev)
        rounding = ffb.FF_ROUND_STOCHASTIC if stochastic else ffb.FF_ROUND_NEAREST_EVEN
        self.ln.eps, self.ln.round, self.ln.seed = eps, rounding, seed
        keep = ffb.FF_ROUND_KEEP_SIGN if act == "relu" else 0          # the slope of a ReLU is its input's sign
        self.act = ffb.ff_activation_desc(kind=_ACT[act], cols=hidden, dtype=self.ln.dtype, round=rounding | keep, seed=seed, index=1)
        self._own = context is None
        self.ctx = ffb.Context(device_index=device_index, workspace_bytes=need) if self._own else context

    @staticmethod
    def workspace_bytes(rows: int, width: int, hidden: int, dtype=None) -> int:
        """Workspace of a context that a block of these sizes (or smaller batches of it) runs on."""
        import torch
        ln, g1, g2 = _descs(width, hidden, dtype or torch.bfloat16)
        return max(ffb.ff_layernorm_workspace_bytes(ln, rows), ffb.ff_ckpt8_wgrad_workspace_bytes(g1, rows),
                   ffb.ff_ckpt8_wgrad_workspace_bytes(g2, rows))

    def close(self):
        if self._own:
            self.ctx.close()

    def saved_bytes(self) -> int:
        """What the block holds from the forward to the backward pass: its checkpoints and one FP32 number a row."""
        return sum(c._q.numel() + c.e.numel() for c in (self.c_norm, self.c_in, self.c_out)) + 4 * self.rows

    def forward(self, x, step: int):
        """y for x [rows, width]; fills the checkpoints."""
        import torch
        x = x.detach()                                                # the gradient is `backward`'s, not autograd's
        px, ld_x = _address("x", x, self.rows, self.width, self.dtype, self.device)
        n = torch.empty((self.rows, self.width), dtype=self.dtype, device=self.device)
        st = torch.cuda.current_stream(self.device).cuda_stream
        ffb.ff_layernorm_forward(self.ctx.ctx, self.ln, ffb.ff_layernorm_bufs(
            X=px, ld_x=ld_x, gamma=self.gamma.data_ptr(), beta=self.beta.data_ptr(), Y=n.data_ptr(), ld_y=self.width,
            rstd=self.rstd.data_ptr(), C=self.c_norm.struct), self.rows, step, st)
        h = n @ self.W1.to(self.dtype).t()
        ffb.ff_activation_forward(self.ctx.ctx, self.act, ffb.ff_activation_bufs(
            H=h.data_ptr(), ld_h=self.hidden, Z=h.data_ptr(), ld_z=self.hidden, CH=self.c_in.struct, CZ=self.c_out.struct), self.rows, step, st)
        return x + h @ self.W2.to(self.dtype).t()

    def backward(self, dy):
        """dx for dy [rows, width]; leaves the parameters' gradients in dgamma, dbeta, dW1, dW2."""
        import torch
        dy = dy.detach()
        pdy, ld_dy = _address("dy", dy, self.rows, self.width, self.dtype, self.device)
        st = torch.cuda.current_stream(self.device).cuda_stream
        ctx = self.ctx.ctx
        ffb.ff_ckpt8_wgrad(ctx, self.g2, ffb.ff_ckpt8_wgrad_bufs(dY=pdy, ld_dy=ld_dy, C=self.c_out.struct, dW=self.dW2.data_ptr()),
                           self.rows, st)
        dh = dy @ self.W2.to(self.dtype)
        ffb.ff_activation_backward(ctx, self.act, ffb.ff_activation_bufs(dZ=dh.data_ptr(), ld_dz=self.hidden, dH=dh.data_ptr(), ld_dh=self.hidden,
                                                                         CH=self.c_in.struct), self.rows, st)
        ffb.ff_ckpt8_wgrad(ctx, self.g1, ffb.ff_ckpt8_wgrad_bufs(dY=dh.data_ptr(), ld_dy=self.hidden, C=self.c_norm.struct, gamma=self.gamma.data_ptr(),
                                                                 beta=self.beta.data_ptr(), dW=self.dW1.data_ptr()), self.rows, st)
        dx = dh @ self.W1.to(self.dtype)
        ffb.ff_layernorm_backward(ctx, self.ln, ffb.ff_layernorm_bufs(
            dY=dx.data_ptr(), ld_dy=self.width, dAdd=pdy, ld_dadd=ld_dy, dX=dx.data_ptr(), ld_dx=self.width,
            gamma=self.gamma.data_ptr(), rstd=self.rstd.data_ptr(), C=self.c_norm.struct, dgamma=self.dgamma.data_ptr(),
            dbeta=self.dbeta.data_ptr()), self.rows, st)
        return dx

    def train_step(self, x, theta: float, lr: float, step: int):
        """One step on x: the first half of the rows positive, the second negative samples.  Returns the loss (a device scalar)."""
        import torch
        y = self.forward(x, step)
        G = y.float().square().sum(dim=1)
        sign = torch.ones(self.rows, device=self.device)
        sign[: self.rows // 2] = -1.0
        margin = sign * (G - theta)                                   # Eq. 1: theta - G, Eq. 2: G - theta
        loss = torch.nn.functional.softplus(margin).mean()
        coef = 2.0 / self.rows * sign * torch.sigmoid(margin)
        self.backward((coef[:, None] * y.float()).to(self.dtype))
        for p, g in ((self.gamma, self.dgamma), (self.beta, self.dbeta), (self.W1, self.dW1), (self.W2, self.dW2)):
            p.sub_(g, alpha=lr)
        return loss


def synthetic_batch(rows: int, width: int, step: int, device, dtype, seed: int = 7):
    """Positive samples lie along a few fixed directions, negative ones have the same length and no preferred direction."""
    import torch
    fixed = torch.Generator(device=device).manual_seed(seed)
    basis = torch.randn((16, width), generator=fixed, device=device)
    gen = torch.Generator(device=device).manual_seed(seed + 1 + step)
    half = rows // 2
    pos = torch.randn((half, 16), generator=gen, device=device) @ basis * 0.25 + 0.3 * torch.randn((half, width), generator=gen, device=device)
    x = torch.cat([pos, torch.randn((rows - half, width), generator=gen, device=device)])
    return (x * (width ** 0.5 / x.norm(dim=1, keepdim=True))).to(dtype)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--width", type=int, default=500)
    ap.add_argument("--hidden", type=int, default=2000)
    a = ap.parse_args(argv)
    block = LocalBlock(a.rows, a.width, a.hidden)
    first = last = None
    for step in range(a.steps):
        x = synthetic_batch(a.rows, a.width, step, block.device, block.dtype)
        loss = block.train_step(x, theta=float(1.5 * a.width), lr=0.002, step=step)
        if step % 10 == 0 or step == a.steps - 1:
            last = float(loss)
            first = last if first is None else first
            print(f"step {step:4d}  loss {last:.4f}")
    ffb.ff_poll_status(block.ctx.ctx)
    held = block.saved_bytes()
    plain = 2 * a.rows * (a.width + 2 * a.hidden)
    print(f"held between the passes: {held} bytes ({held / plain:.2f} of 16-bit activations); "
          f"workspace, which blocks can share: {block.ctx.workspace.numel()} bytes")
    block.close()
    return first, last


if __name__ == "__main__":
    main()
