"""One training step of a small language model in the paper's formats, from
tokens to the log probabilities of the tokens that follow -- on the library's
kernels.

Sequences of any lengths are packed into T tokens.  The residual stream is FP32
(or FP16 codes), GEMM operands are FP8, the last layer's FP16 (Sec. 3).  Per
step, with FP16 master weights E (vocab x width), g1, g2 (width), Wqkv (width x
(Hq + 2 Hkv) D), Wo (Hq D x width), Wl (width x vocab), FP8 copies of Wqkv and
Wo, and FP16 momentum buffers:

  S0 = sqrt(width) E[tokens] (embed_fwd);
  X8 = norm(S0) g1 (rms_norm_fwd);
  QKV = chunk_gemm(X8, Wqkv8) in FP16 and FP8 in one pass; the query and key
    heads turned by their positions (rotary_embed);
  O = attention(Q, K, V) (attn_fwd_fp8);  A = chunk_gemm(O8, Wo8);
  S1 = S0 + A, Y = norm(S1) g2 in FP16 (rms_norm_fwd);
  Z = chunk_gemm_p16(Y, Wl): the logits; log probabilities of the given tokens,
    entropies and, if wanted, the likeliest tokens (token_logprobs);
  dZ from the gradients of the log probabilities and entropies
    (token_logprobs_bwd), dY = chunk_gemm_p16(dZ, Wl^T), dWl = chunk_gemm_p16(Y^T, dZ);
  dS1, dA8 and dg2 (rms_norm_bwd); dWo = chunk_gemm(O8^T, dA8), dO8 =
    Q8(chunk_gemm(dA8, Wo8^T)); dQ, dK, dV (attn_bwd_fp8), turned back;
  dWqkv = chunk_gemm(X8^T, dQKV8), dX = chunk_gemm(dQKV8, Wqkv8^T);
  dS0 = dS1 + the norm's, dg1 (rms_norm_bwd); dE (embed_bwd);
  update: sr_weight_update of the six weights, the loss scale removed through
    the scalars (lr / loss_scale, weight_decay * loss_scale; the norms' weights
    do not decay).

Everything is allocated once, in __init__; calls only launch.
"""
import math

import numpy as np

from . import (EXACT, attn_bwd_fp8, attn_bwd_fp8_workspace_size, attn_fwd_fp8,
               attn_fwd_fp8_workspace_size, chunk_gemm, chunk_gemm_fp8,
               chunk_gemm_fp8_workspace_size, chunk_gemm_p16, chunk_gemm_p16_workspace_size,
               chunk_gemm_workspace_size, embed_bwd, embed_bwd_workspace_size, embed_fwd,
               fp8_quantize, lib, rms_norm_bwd, rms_norm_bwd_workspace_size, rms_norm_fwd,
               rotary_embed, sr_weight_update, token_logprobs, token_logprobs_bwd,
               token_logprobs_workspace_size)
from .lm import rotary_freqs

NAMES = ("E", "g1", "Wqkv", "Wo", "g2", "Wl")


class Fp8TokenLm:
    def __init__(self, lengths, width=256, Hq=4, Hkv=2, D=64, vocab=1024, CL=64, mode=EXACT, eps=1e-5,
                 base=10000.0, top=0, stream="f32", device="cuda:0"):
        """top: alternatives that forward() gives for each token; stream: "f32"
        or "fp16"."""
        import torch
        lib()
        self.torch, self.dev = torch, device
        self.lengths = [int(n) for n in lengths]
        self.T, self.width, self.vocab = sum(self.lengths), width, vocab
        self.Hq, self.Hkv, self.D, self.CL, self.mode, self.eps = Hq, Hkv, D, int(CL), int(mode), eps
        self.scale = math.sqrt(width)
        T, H, k = self.T, Hq + 2 * Hkv, int(top)
        zeros = lambda dtype: lambda *s: torch.zeros(*s, dtype=dtype, device=device)
        u8, u16, f32, i64 = (zeros(t) for t in (torch.uint8, torch.uint16, torch.float32, torch.int64))
        stored = {"f32": f32, "fp16": u16}[stream]
        self.shapes = dict(E=(vocab, width), g1=(width,), Wqkv=(width, H * D), Wo=(Hq * D, width),
                           g2=(width,), Wl=(width, vocab))
        self.W16, self.V16, self.dW16 = ({n: u16(*s) for n, s in self.shapes.items()} for _ in range(3))
        self.W8 = {n: u8(*self.shapes[n]) for n in ("Wqkv", "Wo")}
        self.S0, self.S1, self.dS0, self.dS1 = (stored(T, width) for _ in range(4))
        self.X8, self.rstd1, self.rstd2 = u8(T, width), f32(T), f32(T)
        self.QKV16, self.dQKV16 = u16(T, H, D), u16(T, H, D)
        self.QKV8, self.dQKV8 = u8(T, H, D), u8(T, H, D)
        self.O16, self.O8, self.dO8, self.lse = u16(T, Hq, D), u8(T, Hq, D), u8(T, Hq, D), f32(Hq, T)
        self.A16, self.Y16, self.dY16, self.dX16 = (u16(T, width) for _ in range(4))
        self.dA8, self.Z16, self.dZ16 = u8(T, width), u16(T, vocab), u16(T, vocab)
        self.logp, self.entropy, self.stats = f32(T, 1), f32(T), f32(T, 2)
        self.top_idx, self.top_logp = (i64(T, k), f32(T, k)) if k else (None, None)
        starts = np.concatenate([[0], np.cumsum(self.lengths)])
        self.cu = torch.from_numpy(starts.astype(np.int64)).to(device)
        positions = np.concatenate([np.arange(0)] + [np.arange(n) for n in self.lengths]).astype(np.int64)
        self.positions = torch.from_numpy(positions).to(device)
        freqs, self.mscale = rotary_freqs(D // 2 * 2, base)
        self.freqs = torch.from_numpy(freqs).to(device)
        part = lambda x: (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
        longest = max(self.lengths, default=0)
        self.attn = (*part(self.QKV8), self.cu, self.cu, longest, longest, True, 1.0 / math.sqrt(D))
        self.dqkv = part(self.dQKV16)
        qkv, o = H * D, Hq * D
        need = [attn_fwd_fp8_workspace_size(*self.attn), attn_bwd_fp8_workspace_size(*self.attn),
                embed_bwd_workspace_size(self.positions, self.dS0, self.dW16["E"]),
                rms_norm_bwd_workspace_size(self.S0), token_logprobs_workspace_size(self.Z16, k),
                chunk_gemm_fp8_workspace_size(0, 0, T, qkv, width, CL, mode),
                chunk_gemm_workspace_size(1, 0, width, qkv, T, CL, mode),
                chunk_gemm_workspace_size(0, 1, T, width, qkv, CL, mode),
                chunk_gemm_workspace_size(0, 0, T, width, o, CL, mode),
                chunk_gemm_workspace_size(1, 0, o, width, T, CL, mode),
                chunk_gemm_fp8_workspace_size(0, 1, T, o, width, CL, mode),
                chunk_gemm_p16_workspace_size(0, 0, T, vocab, width, CL),
                chunk_gemm_p16_workspace_size(0, 1, T, width, vocab, CL),
                chunk_gemm_p16_workspace_size(1, 0, width, vocab, T, CL)]
        self.ws_bytes = max(need)
        self.ws = u8(max(1, self.ws_bytes))

    def set_weights(self, W16_codes):
        """FP16 master weights (a dict of numpy uint16 codes by NAMES); the FP8
        copies are their quantization, the momentum buffers start at 0."""
        torch = self.torch
        for n in NAMES:
            t = torch.from_numpy(np.ascontiguousarray(W16_codes[n], np.uint16).view(np.int16))
            self.W16[n].copy_(t.to(self.dev).view(torch.uint16))
            self.V16[n].zero_()
            if n in self.W8:
                fp8_quantize(self.W16[n], self.W8[n])

    def forward(self, tokens, given, tau=1.0):
        """Log probabilities (T x 1) of the tokens `given` (T x 1 int64, -1:
        none) after the tokens `tokens` (T int64) and those before them;
        self.entropy, and self.top_idx and self.top_logp if wanted, too."""
        T, W, CL, mode, ws = self.T, self.width, self.CL, self.mode, (self.ws, self.ws_bytes)
        qkv, o, turned = self.shapes["Wqkv"][1], self.shapes["Wo"][0], self.Hq + self.Hkv
        embed_fwd(tokens, self.W16["E"], self.S0, self.scale)
        rms_norm_fwd(self.S0, None, self.W16["g1"], self.eps, None, self.X8, rstd=self.rstd1)
        chunk_gemm_fp8(0, 0, T, qkv, W, CL, self.X8, W, self.W8["Wqkv"], qkv, self.QKV16, qkv, self.QKV8,
                       qkv, 1.0, mode, *ws)
        rotary_embed(self.QKV16[:, :turned], self.positions, self.freqs, self.QKV8[:, :turned],
                     mscale=self.mscale)
        attn_fwd_fp8(*self.attn, self.O16, self.O8, 1.0, self.lse, *ws)
        chunk_gemm(0, 0, T, W, o, CL, self.O8, o, self.W8["Wo"], W, self.A16, W, mode, *ws)
        rms_norm_fwd(self.A16, self.S0, self.W16["g2"], self.eps, self.S1, self.Y16, rstd=self.rstd2)
        chunk_gemm_p16(0, 0, T, self.vocab, W, CL, self.Y16, W, self.W16["Wl"], self.vocab, self.Z16,
                       self.vocab, *ws)
        token_logprobs(self.Z16, given, tau, self.logp, self.entropy, self.stats, self.top_idx,
                       self.top_logp, *ws)
        return self.logp

    def backward(self, tokens, given, d_logp, d_entropy, loss_scale, tau=1.0):
        """Gradients of all weights, times loss_scale, from those of the log
        probabilities (T x 1; -1/T for the mean of -logp) and of the entropies
        (T, or None), after forward() on the same tokens."""
        T, W, V, CL, mode, ws = self.T, self.width, self.vocab, self.CL, self.mode, (self.ws, self.ws_bytes)
        qkv, o, turned = self.shapes["Wqkv"][1], self.shapes["Wo"][0], self.Hq + self.Hkv
        d = self.dW16
        token_logprobs_bwd(self.Z16, given, tau, self.stats, self.entropy, d_logp, d_entropy, loss_scale,
                           self.dZ16)
        chunk_gemm_p16(0, 1, T, W, V, CL, self.dZ16, V, self.W16["Wl"], V, self.dY16, W, *ws)
        chunk_gemm_p16(1, 0, W, V, T, CL, self.Y16, W, self.dZ16, V, d["Wl"], V, *ws)
        rms_norm_bwd(self.S1, self.W16["g2"], self.rstd2, self.dY16, None, self.dS1, self.dA8, 1.0, d["g2"],
                     *ws)
        chunk_gemm(1, 0, o, W, T, CL, self.O8, o, self.dA8, W, d["Wo"], W, mode, *ws)
        chunk_gemm_fp8(0, 1, T, o, W, CL, self.dA8, W, self.W8["Wo"], W, None, o, self.dO8, o, 1.0, mode, *ws)
        attn_bwd_fp8(*self.attn, self.O16, self.dO8, self.lse, *self.dqkv, 1.0, *ws)
        fp8_quantize(self.dQKV16, self.dQKV8)
        rotary_embed(self.dQKV16[:, :turned], self.positions, self.freqs, self.dQKV8[:, :turned],
                     inverse=True, mscale=self.mscale)
        chunk_gemm(1, 0, W, qkv, T, CL, self.X8, W, self.dQKV8, qkv, d["Wqkv"], qkv, mode, *ws)
        chunk_gemm(0, 1, T, W, qkv, CL, self.dQKV8, qkv, self.W8["Wqkv"], qkv, self.dX16, W, mode, *ws)
        rms_norm_bwd(self.S0, self.W16["g1"], self.rstd1, self.dX16, self.dS1, self.dS0, None, 1.0, d["g1"],
                     *ws)
        embed_bwd(tokens, self.dS0, d["E"], self.scale, *ws)

    def update(self, lr, momentum, weight_decay, loss_scale, seed, t):
        lr_eff = float(np.float32(lr) / np.float32(loss_scale))
        wd_eff = float(np.float32(weight_decay) * np.float32(loss_scale))
        for i, n in enumerate(NAMES):
            sr_weight_update(self.W16[n], self.dW16[n], self.V16[n], self.W8.get(n), self.W16[n].numel(),
                             lr_eff, momentum, 0.0 if n in ("g1", "g2") else wd_eff, seed,
                             t * len(NAMES) + i)

    def step(self, tokens, given, d_logp, d_entropy, lr, momentum, weight_decay, loss_scale, seed, t,
             tau=1.0):
        """forward, backward and update; returns the log probabilities."""
        self.forward(tokens, given, tau)
        self.backward(tokens, given, d_logp, d_entropy, loss_scale, tau)
        self.update(lr, momentum, weight_decay, loss_scale, seed, t)
        return self.logp
