"""Training a MambaByte model on the library's kernels.

`Model` is the decoder's stack (decoder.py) over whole spans, for training:

    residual = emb[bytes]                                            mb_embed
    per layer: h = rmsnorm(residual) * w                             torch
        [x; z] = h [W_in_x; W_in_z]^T                                cuBLAS
        xc = silu(conv1d(x))                                         mb_conv1d
        [dt_low | B | C] = xc W_xproj^T, dt = dt_low W_dt^T          cuBLAS
        y = (C.h + D xc) * silu(z)  (B, C in place: bc_stride)       mb_scan_prefill_ckpt
        residual += y W_out^T                                        cuBLAS
    rmsnorm, tied byte head, next-byte cross entropy                 mb_cross_entropy

Each library call is an autograd function whose backward is the library's
(mb_scan_backward, mb_conv1d_backward, mb_embed_backward, mb_cross_entropy), so
torch composes them with the projections and norms. `train_step` ends with mb_grad_norm and mb_grad_clip over all gradients and an
optimizer step. Weights are those of decoder.init_weights: projections in
`dtype`, the rest fp32; the residual stream is fp32.

    python -m paper_2401_13660_gb300.trainer --steps 30     # learns a repeating text from random weights
"""
from __future__ import annotations

import argparse

import torch
from torch.autograd.function import once_differentiable

from . import mbscan as mb
from .decoder import CONFIGS, STORED_KEYS, DecoderConfig, init_weights


class Workspace:
    """One device buffer for the calls of a model, which follow each other on one stream; grows as asked and keeps its
    status block then, with what earlier calls have recorded there."""

    STATUS = 256

    def __init__(self, device):
        self.buffer = torch.zeros(self.STATUS, dtype=torch.uint8, device=device)

    def get(self, nbytes: int) -> torch.Tensor:
        if self.buffer.numel() < nbytes:
            status = self.buffer[:self.STATUS]
            self.buffer = torch.zeros(nbytes, dtype=torch.uint8, device=self.buffer.device)
            self.buffer[:self.STATUS] = status
        return self.buffer


class Tied:
    """What the two uses of a tied table share in one pass: the head's part of its gradient, fp32, until the lookup's is
    added to it."""
    grad = None


class Embed(torch.autograd.Function):
    """scale * table[tokens] in fp32 (the residual stream). With `tied`, its backward pass, which follows the head's, gives
    the table's whole gradient: the lookup's part is added to the head's in fp32 and the sum rounded once."""

    @staticmethod
    def forward(ctx, table, tokens, scale, ws, tied=None):
        ctx.save_for_backward(tokens)
        ctx.scale, ctx.ws, ctx.tied, ctx.table = scale, ws, tied, (table.shape, table.dtype)
        out = torch.empty(*tokens.shape, table.shape[1], device=table.device)
        return mb.mb_embed(tokens, table, out, scale=scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (tokens,) = ctx.saved_tensors
        shape, dtype = ctx.table
        d = None
        if ctx.tied is not None:
            d, ctx.tied.grad = ctx.tied.grad, None
        add = d is not None
        if not add:
            d = torch.empty(shape, device=dout.device)
        ws = ctx.ws.get(mb.mb_embed_backward_workspace_size(tokens.numel(), *shape))
        mb.mb_embed_backward(tokens, dout.contiguous(), d, scale=ctx.scale, accumulate=add, ws=ws)
        return d.to(dtype), None, None, None, None


class Head(torch.autograd.Function):
    """h table^T, through cuBLAS both ways; the table's gradient goes to the lookup's backward pass (Embed)."""

    @staticmethod
    def forward(ctx, h, table, tied):
        ctx.save_for_backward(h, table)
        ctx.tied = tied
        return h @ table.t()

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogits):
        h, table = ctx.saved_tensors
        d, rows = dlogits.flatten(0, -2).t(), h.flatten(0, -2)
        ctx.tied.grad = torch.mm(d, rows) if h.dtype == torch.float32 else torch.mm(d, rows, out_dtype=torch.float32)
        return dlogits @ table, None, None


class Conv1d(torch.autograd.Function):
    """silu(causal depthwise convolution) of a span that starts a sequence."""

    @staticmethod
    def forward(ctx, x, w, bias, ws):
        ctx.save_for_backward(x, w, bias)
        ctx.ws = ws
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        return mb.mb_conv1d(x, w, out, bias=bias)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, w, bias = ctx.saved_tensors
        g = dict(dx=torch.empty(x.shape, dtype=x.dtype, device=x.device), dw=torch.empty_like(w),
                 dbias=torch.empty_like(bias))
        ws = ctx.ws.get(mb.mb_conv1d_backward_workspace_size(*x.shape))
        mb.mb_conv1d_backward(x, w, dout.contiguous(), bias=bias, grads=g, ws=ws)
        return g["dx"], g["dw"], g["dbias"], None


class Scan(torch.autograd.Function):
    """The layer core over a span that starts a sequence."""

    @staticmethod
    def forward(ctx, x, z, dt, B, C, A, D, dt_bias, ws):
        y = torch.empty_like(x)
        ctx.ws = ws
        ctx.nbytes = mb.mb_workspace_size(mb.make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias))
        ckpt = torch.empty(x.shape[0], -(-x.shape[1] // mb.MB_CKPT_STEPS), *A.shape, device=x.device)
        mb.mb_scan_prefill_ckpt(x, dt, B, C, A, y, ckpt, z=z, D=D, dt_bias=dt_bias, ws=ws.get(ctx.nbytes))
        ctx.save_for_backward(x, z, dt, B, C, A, D, dt_bias, ckpt)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, z, dt, B, C, A, D, dt_bias, ckpt = ctx.saved_tensors
        g = mb.mb_scan_backward(x, dt, B, C, A, ckpt, dy.contiguous(), z=z, D=D, dt_bias=dt_bias,
                                ws=ctx.ws.get(ctx.nbytes))
        return (g["dx"], g["dz"], g["ddt"], g["dB"].to(B.dtype), g["dC"].to(C.dtype), g["dA"], g["dD"], g["ddt_bias"],
                None)


class CrossEntropy(torch.autograd.Function):
    """Sum over the targets of scale * -log softmax(logits)[target]; targets outside the vocabulary are ignored."""

    @staticmethod
    def forward(ctx, logits, targets, scale):
        loss = torch.empty(targets.shape, device=logits.device)
        mb.mb_cross_entropy(logits, targets, loss)
        ctx.save_for_backward(logits, targets)
        ctx.scale = scale
        return loss.sum() * scale

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        # the incoming gradient as every row's weight: multiplied in fp32, in the pass that makes dlogits
        logits, targets = ctx.saved_tensors
        weight = dloss.expand(targets.shape).contiguous()
        _, dlogits = mb.mb_cross_entropy(logits, targets, torch.empty_like(weight), torch.empty_like(logits),
                                         weight=weight, scale=ctx.scale)
        return dlogits, None, None


def rmsnorm(residual, w, eps, dtype):
    return (residual * torch.rsqrt(residual.square().mean(-1, keepdim=True) + eps) * w).to(dtype)


class Model:
    """MambaByte over spans of bytes; `parameters` are leaf tensors that collect gradients."""

    def __init__(self, cfg: DecoderConfig, device, dtype=torch.bfloat16, seed: int = 0):
        self.cfg, self.dtype, self.ws = cfg, dtype, Workspace(device)
        layers, emb, norm_f = init_weights(cfg, torch.device(device), seed)

        def leaf(t):
            t = t.to(dtype) if t.dtype == torch.bfloat16 else t
            return t.clone().requires_grad_()
        self.layers = [{k: leaf(L[k]) for k in STORED_KEYS} for L in layers]
        # small, as a tied head wants it (logits of unit variance); the lookup scales it up to the residual stream's
        self.emb, self.norm_f = leaf(emb / cfg.d_model ** 0.5), leaf(norm_f)
        self.parameters = [p for L in self.layers for p in L.values()] + [self.emb, self.norm_f]

    def logits(self, tokens):
        """tokens [batch, L] (uint8, int32 or int64) -> [batch, L, vocab]."""
        cfg, R, N = self.cfg, self.cfg.dt_rank, self.cfg.d_state
        tied = Tied()
        residual = Embed.apply(self.emb, tokens, cfg.d_model ** 0.5, self.ws, tied)
        for L in self.layers:
            h = rmsnorm(residual, L["norm_w"], cfg.eps, self.dtype)
            xc = Conv1d.apply(h @ L["W_in"][0].t(), L["conv_w"], L["conv_b"], self.ws)
            rows = xc @ L["W_xproj"].t()
            y = Scan.apply(xc, h @ L["W_in"][1].t(), rows[..., :R] @ L["W_dt"].t(), rows[..., R:R + N], rows[..., R + N:],
                           L["A"], L["D"], L["dt_bias"], self.ws)
            residual = residual + (y @ L["W_out"].t()).float()
        return Head.apply(rmsnorm(residual, self.norm_f, cfg.eps, self.dtype), self.emb, tied)

    def loss(self, tokens, targets, counted: int | None = None):
        """Mean loss (nats per byte) of predicting targets [batch, L]; `counted`: how many of them are bytes."""
        return CrossEntropy.apply(self.logits(tokens), targets, 1.0 / (counted or targets.numel()))

    def check(self):
        """Raise if a scan recorded a device-side error (blocking)."""
        st, detail = mb.mb_check(self.ws.buffer)
        if st != mb.MB_OK:
            raise mb.MbError(st, f"training step (detail {detail})")


class Trainer:
    """AdamW steps (the paper's betas) with the gradients clipped by their global norm."""

    def __init__(self, model: Model, lr: float = 1e-3, max_norm: float = 1.0):
        self.model, self.max_norm = model, max_norm
        # gradients that stay where they are: the list of them is made once
        for p in model.parameters:
            p.grad = torch.zeros_like(p)
        self.grads = mb.mb_tensor_list([p.grad for p in model.parameters])
        self.norm = torch.empty(1, device=model.emb.device)
        self.norm_ws = torch.zeros(mb.mb_grad_norm_workspace_size(), dtype=torch.uint8, device=model.emb.device)
        self.optimizer = torch.optim.AdamW(model.parameters, lr=lr, betas=(0.9, 0.95), weight_decay=0.0)

    def train_step(self, tokens, targets, counted: int | None = None):
        """One step; returns the loss and the gradient norm before clipping (device tensors). Waits for the gradients
        and leaves the model as it was if their norm is not finite (one overflow would stay in the weights and moments
        for good), or raises if a scan recorded a device-side error."""
        for g in self.grads.tensors:
            g.zero_()
        loss = self.model.loss(tokens, targets, counted)
        loss.backward()
        mb.mb_grad_norm(self.grads, self.norm, ws=self.norm_ws)
        mb.mb_grad_clip(self.grads, self.norm, self.max_norm)
        self.model.check()
        if bool(torch.isfinite(self.norm)):
            self.optimizer.step()
        return loss.detach(), self.norm


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="tiny_2x64", choices=sorted(CONFIGS))
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--length", type=int, default=256)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    model = Model(CONFIGS[a.config], "cuda")
    trainer = Trainer(model, lr=3e-3)
    text = torch.frombuffer(bytearray(b"the quick brown fox jumps over the lazy dog. "), dtype=torch.uint8)
    stream = text.repeat(a.batch * (a.length + 1) // len(text) + 2)[:a.batch * (a.length + 1)]
    rows = stream.view(a.batch, a.length + 1).cuda()
    tokens, targets = rows[:, :-1].contiguous(), rows[:, 1:].contiguous()
    for step in range(a.steps):
        loss, norm = trainer.train_step(tokens, targets)
        if step % 5 == 0 or step + 1 == a.steps:
            print(f"step {step:4d}  bits per byte {float(loss) / 0.6931471805599453:.4f}  gradient norm {float(norm):.4f}")
    model.check()


if __name__ == "__main__":
    main()
