"""Recurrent decoding of a whole MambaByte model on the library's kernels.

One call of `Decoder.step` generates the next byte of every stream: byte
embedding (mb_embed), then per layer the Mamba block of MambaByte (Figure 6; Table 6 rows
"Linear projections", "Pre-SSM 1D convolution", "Delta, B, C from input x",
the scan rows, "Element-wise gating"):

    residual += previous block output;  h = rmsnorm(residual) * w   mb_rmsnorm
    [x; z] = h [W_in_x; W_in_z]^T         (one batched GEMM)         cuBLAS
    xc = silu(conv1d_step(x));  [dt_low | B | C] = xc W_xproj^T      mb_conv_xproj
        (the convolution step fused into a split-K projection)
    dt = dt_low W_dt^T                                               cuBLAS
    y = (C.h + D xc) * silu(z), state updated in place               mb_step
        (B, C read in place from the x-projection rows: bc_stride)
    out = y W_out^T                                                  cuBLAS

and finally rmsnorm and the tied byte head (logits over 256 bytes). The
input, Delta, output and head projections are plain bf16 GEMMs (fp32
accumulation) through cuBLAS (torch.bmm / torch.mm); every other step is a
kernel of libmbscan.so. With `bits=8` the input and output projections, nearly
all of the weights, are held and multiplied in 8 bits with block scales:

    h = rmsnorm(residual) * w in 8 bits                              mb_rmsnorm_q8
    [x; z] = h [W_in_x; W_in_z]^T                                    mb_matmul_q8
    ...
    y in 8 bits;  out = y W_out^T                                    mb_quantize_q8, mb_matmul_q8

The whole step can be captured once in a CUDA graph
(`capture`) and replayed per generated byte. `draw` takes the next bytes from
the logits (mb_sample), `generate` alternates the two.
Weights are random (seeded): the kernels and the memory traffic do not depend
on trained values.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import mbscan as mb


@dataclass(frozen=True)
class DecoderConfig:
    n_layers: int
    d_model: int
    d_inner: int
    dt_rank: int
    d_state: int = 16
    vocab: int = 256
    eps: float = 1e-5


CONFIGS = {
    # 48 layers, d_model 2304, expansion 2 (d_inner 4608), dt_rank = d_model / 16
    "mambabyte_48x2304": DecoderConfig(n_layers=48, d_model=2304, d_inner=4608, dt_rank=144),
    "tiny_2x64": DecoderConfig(n_layers=2, d_model=64, d_inner=128, dt_rank=8),
}

WEIGHT_KEYS = ("norm_w", "W_in_x", "W_in_z", "conv_w", "conv_b", "W_dtlow", "W_B", "W_C", "W_dt", "dt_bias",
               "A", "D", "W_out")
# tensors a layer stores; the keys above that are not listed are views of them
STORED_KEYS = ("norm_w", "W_in", "conv_w", "conv_b", "W_xproj", "W_dt", "dt_bias", "A", "D", "W_out")


def init_weights(cfg: DecoderConfig, device, seed: int = 0):
    """Seeded random weights of the given shapes: projections bf16, the rest
    fp32 (A = -(n+1), D = 1, dt_bias = softplus^-1 of log-uniform [1e-3, 0.1])."""
    g = torch.Generator(device=device).manual_seed(seed)

    def lin(out_f, in_f):
        return (torch.randn(out_f, in_f, device=device, generator=g) / math.sqrt(in_f)).to(torch.bfloat16)

    D, E, R, N = cfg.d_model, cfg.d_inner, cfg.dt_rank, cfg.d_state
    layers = []
    for _ in range(cfg.n_layers):
        u = torch.rand(E, device=device, generator=g, dtype=torch.float64)
        target = torch.exp(math.log(1e-3) + u * (math.log(0.1) - math.log(1e-3)))
        W_in = torch.stack([lin(E, D), lin(E, D)])            # [2, E, D]: x and z rows
        W_xproj = torch.cat([lin(R, E), lin(N, E), lin(N, E)])  # [R + 2N, E]: dt_low, B, C rows
        L = {
            "norm_w": torch.ones(D, device=device),
            "W_in": W_in,
            "conv_w": (torch.rand(E, 4, device=device, generator=g) - 0.5).contiguous(),
            "conv_b": (torch.rand(E, device=device, generator=g) - 0.5) * 0.1,
            "W_xproj": W_xproj, "W_dt": lin(E, R),
            "dt_bias": (target + torch.log(-torch.expm1(-target))).float(),
            "A": -torch.arange(1, N + 1, dtype=torch.float32, device=device).repeat(E, 1).contiguous(),
            "D": torch.ones(E, device=device),
            "W_out": lin(D, E),
        }
        L.update(W_in_x=W_in[0], W_in_z=W_in[1], W_dtlow=W_xproj[:R], W_B=W_xproj[R:R + N],
                 W_C=W_xproj[R + N:])
        layers.append(L)
    emb = (torch.randn(cfg.vocab, D, device=device, generator=g)).to(torch.bfloat16)
    return layers, emb, torch.ones(D, device=device)


class Matrix8:
    """A weight matrix [rows, width] in 8 bits with a scale for each block of 128 x 128."""

    def __init__(self, W):
        rows, width = W.shape
        self.q = torch.empty(rows, width, dtype=torch.float8_e4m3fn, device=W.device)
        self.scales = torch.empty(-(-rows // mb.Q8_BLOCK), mb.mb_q8_scale_stride(width), dtype=torch.uint8, device=W.device)
        mb.mb_quantize_q8(W, self.q, self.scales, block_rows=mb.Q8_BLOCK)

    def values(self):
        return mb.mb_dequantize_q8(self.q, self.scales, torch.empty(self.q.shape, device=self.q.device), block_rows=mb.Q8_BLOCK)

    def nbytes(self):
        return self.q.numel() + self.scales.numel()


class Rows8:
    """Activations [rows, width] in 8 bits with a scale for 128 columns."""

    def __init__(self, rows, width, device):
        self.q = torch.empty(rows, width, dtype=torch.float8_e4m3fn, device=device)
        self.scales = torch.empty(rows, mb.mb_q8_scale_stride(width), dtype=torch.uint8, device=device)

    def values(self):
        return mb.mb_dequantize_q8(self.q, self.scales, torch.empty(self.q.shape, device=self.q.device))


class Decoder:
    """Recurrent byte-level decoder over `batch` streams (bf16 activations,
    fp32 residual stream and SSM states, bf16 convolution windows). bits: 16
    (bf16 projections) or 8 (input and output projections in 8 bits; needs
    d_inner % 128 == 0, and the decoder keeps no bf16 copy of them)."""

    def __init__(self, cfg: DecoderConfig, batch: int, device, seed: int = 0, weights=None, bits: int = 16):
        if bits not in (8, 16):
            raise ValueError(f"bits {bits}, expected 8 or 16")
        if bits == 8 and (cfg.d_inner % mb.Q8_BLOCK or cfg.d_model % 16):
            raise ValueError(f"no 8-bit projections for d_model {cfg.d_model}, d_inner {cfg.d_inner}")
        # fp32 accumulation all the way in the bf16 GEMMs
        torch.backends.cuda.matmul.allow_bf16_reduced_precision_reduction = False
        self.cfg, self.batch, self.device = cfg, batch, torch.device(device)
        self.layers, self.emb, self.norm_f = weights or init_weights(cfg, self.device, seed)
        D, E, R, N, B = cfg.d_model, cfg.d_inner, cfg.dt_rank, cfg.d_state, batch
        dev, bf = self.device, torch.bfloat16
        self.ssm = [torch.zeros(B, E, N, device=dev) for _ in range(cfg.n_layers)]
        self.conv = [torch.zeros(B, 3, E, device=dev, dtype=bf) for _ in range(cfg.n_layers)]
        self.tokens = torch.zeros(B, dtype=torch.int64, device=dev)
        self.residual = torch.empty(B, D, device=dev)
        self.h = torch.empty(B, D, device=dev, dtype=bf)
        self.out = torch.empty(B, D, device=dev, dtype=bf)
        self.xz = torch.empty(2, B, E, device=dev, dtype=bf)   # x = xz[0], z = xz[1]
        self.xc, self.dt, self.y = (torch.empty(B, E, device=dev, dtype=bf) for _ in range(3))
        self.xdbl = torch.empty(B, R + 2 * N, device=dev, dtype=bf)   # [dt_low | B | C]
        self.logits = torch.empty(B, cfg.vocab, device=dev, dtype=bf)
        self.drawn = torch.zeros(B, dtype=torch.int64, device=dev)
        self.bits = bits
        if bits == 8:
            # the layers' own dicts stay as they were given
            self.layers = [dict(L, W_in=Matrix8(L["W_in"].view(2 * E, D)), W_out=Matrix8(L["W_out"])) for L in self.layers]
            for L in self.layers:
                del L["W_in_x"], L["W_in_z"]
            self.h8, self.y8 = Rows8(B, D, dev), Rows8(B, E, dev)
        # status block of the scan steps and of the fused convolution +
        # x-projection (a wait that times out is recorded there), then the
        # projection's fp32 partial sums
        ws_bytes = mb.mb_conv_xproj_workspace_size(B, E, R + 2 * N)
        if ws_bytes == 0:
            raise ValueError(f"no fused convolution + x-projection for d_inner {E}, dt_rank {R}")
        self.ws = torch.zeros(ws_bytes, dtype=torch.uint8, device=dev)
        self.graph = None

    def reset(self):
        for t in self.ssm + self.conv:
            t.zero_()

    def _forward(self, trace=None):
        cfg = self.cfg
        mb.mb_embed(self.tokens, self.emb, self.residual)
        add = None
        R, N = cfg.dt_rank, cfg.d_state
        hb = self.h.unsqueeze(0).expand(2, -1, -1)
        Bv = self.xdbl[:, R:R + N].unsqueeze(1)
        Cv = self.xdbl[:, R + N:].unsqueeze(1)
        for l, L in enumerate(self.layers):
            if trace is not None:   # copies of the block's inputs (host memory)
                trace.append({"residual": self.residual.cpu(), "add": None if add is None else add.cpu(),
                              "ssm": self.ssm[l].cpu(), "conv": self.conv[l].cpu()})
            if self.bits == 8:
                h8, y8, W_in, W_out = self.h8, self.y8, L["W_in"], L["W_out"]
                mb.mb_rmsnorm_q8(self.residual, L["norm_w"], h8.q, h8.scales, add=add, eps=cfg.eps)
                mb.mb_matmul_q8(h8.q, h8.scales, W_in.q, W_in.scales, self.xz, ws=self.ws)
            else:
                mb.mb_rmsnorm(self.residual, L["norm_w"], self.h, add=add, eps=cfg.eps)
                torch.bmm(hb, L["W_in"].transpose(1, 2), out=self.xz)
            mb.mb_conv_xproj(self.xz[0], self.conv[l], L["conv_w"], L["W_xproj"], self.xc, self.xdbl, self.ws,
                             bias=L["conv_b"])
            torch.mm(self.xdbl[:, :R], L["W_dt"].t(), out=self.dt)
            mb.mb_step(self.xc[:, None], self.dt[:, None], Bv, Cv, L["A"], self.y[:, None], self.ssm[l],
                       z=self.xz[1][:, None], D=L["D"], dt_bias=L["dt_bias"], ws=self.ws)
            if self.bits == 8:
                mb.mb_quantize_q8(self.y, y8.q, y8.scales)
                mb.mb_matmul_q8(y8.q, y8.scales, W_out.q, W_out.scales, self.out, ws=self.ws)
            else:
                torch.mm(self.y, L["W_out"].t(), out=self.out)
            add = self.out
            if trace is not None:   # its intermediates and outputs
                trace[-1].update(residual_out=self.residual.cpu(), h=(h8.values() if self.bits == 8 else self.h).cpu(),
                                 x=self.xz[0].cpu(),
                                 z=self.xz[1].cpu(), xc=self.xc.cpu(), xdbl=self.xdbl.cpu(), dt=self.dt.cpu(),
                                 y=self.y.cpu(), out=self.out.cpu(), ssm_out=self.ssm[l].cpu(),
                                 conv_out=self.conv[l].cpu())
                if self.bits == 8:
                    trace[-1].update(y8=y8.values().cpu())
        mb.mb_rmsnorm(self.residual, self.norm_f, self.h, add=add, eps=cfg.eps)
        torch.mm(self.h, self.emb.t(), out=self.logits)

    def capture(self):
        """Record one step into a CUDA graph (after one eager warm-up step on
        a copy of the states, so that the states are left as they were)."""
        saved = [t.clone() for t in self.ssm + self.conv]
        s = torch.cuda.Stream(self.device)
        s.wait_stream(torch.cuda.current_stream(self.device))
        with torch.cuda.stream(s):
            self._forward()
        torch.cuda.current_stream(self.device).wait_stream(s)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._forward()
        for t, v in zip(self.ssm + self.conv, saved):
            t.copy_(v)
        return self.graph

    def step(self, tokens, trace=None):
        """Feed one byte per stream (int64 [batch]); returns the logits of the
        next byte [batch, 256] (bf16). A token outside the vocabulary is no
        error: it is looked up as zeros (mb_embed), as for a stream that has
        nothing to say, and touches no other stream. With a list `trace` (eager
        decoders only), host copies of every block's inputs and outputs are
        appended to it, one dict per layer."""
        self.tokens.copy_(tokens)
        if self.graph is not None:
            if trace is not None:
                raise ValueError("trace needs an eager decoder (no captured graph)")
            self.graph.replay()
        else:
            self._forward(trace)
        return self.logits

    def draw(self, u, *, temperature=None, top_k=None, top_p=None, min_p=None, prob=None):
        """Draw every stream's next byte from the logits of the last step, by the
        random numbers u [batch] (fp32 in [0, 1)). The settings are those of
        mb_sample: a number for all streams, or a tensor [batch]. Returns the
        bytes, int64 [batch] (overwritten by the next draw)."""
        def each(v, dtype):
            return v if v is None or isinstance(v, torch.Tensor) else torch.full((self.batch,), v, dtype=dtype, device=self.device)
        return mb.mb_sample(self.logits, u, self.drawn, temperature=each(temperature, torch.float32),
                            top_k=each(top_k, torch.int32), top_p=each(top_p, torch.float32),
                            min_p=each(min_p, torch.float32), prob=prob)

    def generate(self, tokens, u, **settings):
        """Feed one byte per stream (int64 [batch]), then generate u.shape[0]
        more of each, drawn by u [bytes, batch]: int64 [bytes, batch]."""
        out = torch.empty(u.shape[0], self.batch, dtype=torch.int64, device=self.device)
        for i in range(u.shape[0]):
            self.step(tokens)
            tokens = self.draw(u[i], **settings)
            out[i] = tokens
        return out

    def check(self):
        """Raise if a scan step recorded a device-side error (blocking)."""
        st, detail = mb.mb_check(self.ws)
        if st != mb.MB_OK:
            raise mb.MbError(st, f"decoder step (detail {detail})")

    def bytes_per_step(self) -> int:
        """Bytes one step must move: every weight once, the SSM states and
        convolution windows read and written, the embedding rows and head."""
        w = sum(L[k].nbytes() if isinstance(L[k], Matrix8) else L[k].numel() * L[k].element_size()
                for L in self.layers for k in STORED_KEYS)
        w += self.emb.numel() * self.emb.element_size() + self.norm_f.numel() * 4
        st = sum(t.numel() * t.element_size() for t in self.ssm + self.conv)
        return w + 2 * st
