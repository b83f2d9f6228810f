"""One training step of a small language model in the paper's formats: an
attention block between two projections and an FP16 last layer, distilled from
a teacher's top logits -- on the library's kernels.

Sequences of any lengths are packed into T tokens.  Per step, with FP16 master
weights Wqkv (width x (Hq + 2 Hkv) D), Wo (Hq D x hidden), Wl (hidden x vocab),
their FP8 copies (not of Wl, Sec. 3: the last layer stays in FP16) and FP16
momentum buffers:

  QKV = chunk_gemm(X8, Wqkv8) in FP16 and FP8 in one pass; the query and key
    heads are turned by their positions from FP16 into the FP8 result
    (rotary_embed), the value heads are in place;
  O = attention(Q, K, V) (attn_fwd_fp8): FP8 for the next GEMM, FP16 and the
    log-sum-exps for the backward pass;
  H = chunk_gemm(O8, Wo8), A = ReLU(H), Y = chunk_gemm_p16(A, Wl): the logits;
  loss and E = loss_scale dloss/dY (distill_loss), in FP16;
  dA = chunk_gemm_p16(E, Wl^T), dWl = chunk_gemm_p16(A^T, E);
  E8 = Q8(dA [H > 0]), dWo = chunk_gemm(O8^T, E8), dO8 = Q8(chunk_gemm(E8, Wo8^T));
  dQ, dK, dV = attn_bwd_fp8 in FP16, rounded to FP8, the query and key heads
    turned back (rotary_embed, inverse); dWqkv = chunk_gemm(X8^T, dQKV8);
  update: sr_weight_update of the three weights, the loss scale removed through
    the scalars (lr / loss_scale, weight_decay * loss_scale).

Everything is allocated once, in __init__; step() only launches.
"""
import math

import numpy as np

from . import (EXACT, attn_bwd_fp8, attn_bwd_fp8_workspace_size, attn_fwd_fp8,
               attn_fwd_fp8_workspace_size, chunk_gemm, chunk_gemm_fp8,
               chunk_gemm_fp8_workspace_size, chunk_gemm_p16, chunk_gemm_p16_workspace_size,
               chunk_gemm_workspace_size, distill_loss, fp8_quantize, lib, relu_backward_fp8,
               relu_codes, rotary_embed, sr_weight_update)


def rotary_freqs(R, base=10000.0, scaling=None, factor=1.0, original_length=4096, slow_turns=1.0,
                 fast_turns=32.0):
    """(freqs, mscale) for rotary_embed: R/2 float64 angles per position,
    base^(-2 j / R), scaled for contexts `factor` times longer than the
    original_length that the model was trained on:

    * "linear":   every angle divided by factor;
    * "base":     base raised to base factor^(R / (R - 2)), so that the slowest
                  pair turns factor times slower and the fastest as before;
    * "by_parts": pairs that turn more than fast_turns times within
                  original_length are kept, those below slow_turns are divided
                  by factor, the ones between are blended; mscale is
                  0.1 ln(factor) + 1.
    """
    if R % 2 or R < 2:
        raise ValueError("rotary_freqs: R must be even and positive")
    if scaling not in (None, "linear", "base", "by_parts"):
        raise ValueError(f"rotary_freqs: unknown scaling {scaling!r}")
    if scaling is not None and not 1.0 <= factor < math.inf:
        raise ValueError("rotary_freqs: factor must be at least 1 and finite")
    if scaling == "by_parts" and not slow_turns < fast_turns:
        raise ValueError("rotary_freqs: slow_turns must be below fast_turns")
    if scaling == "base" and R > 2:
        base = base * factor ** (R / (R - 2.0))
    freqs = base ** (-np.arange(0, R, 2, dtype=np.float64) / R)
    if scaling == "linear":
        return freqs / factor, 1.0
    if scaling == "by_parts":
        turns = freqs * original_length / (2.0 * math.pi)
        keep = np.clip((turns - slow_turns) / (fast_turns - slow_turns), 0.0, 1.0)
        return freqs - (freqs - freqs / factor) * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return freqs, 1.0


class Fp8AttentionLm:
    def __init__(self, lengths, width=256, Hq=4, Hkv=2, D=64, hidden=256, vocab=1024, CL=64,
                 mode=EXACT, base=10000.0, device="cuda:0"):
        import torch
        lib()
        self.torch, self.dev = torch, device
        self.lengths = [int(n) for n in lengths]
        self.T, self.width, self.hidden, self.vocab = sum(self.lengths), width, hidden, vocab
        self.Hq, self.Hkv, self.D, self.CL, self.mode = Hq, Hkv, D, int(CL), int(mode)
        T, H = self.T, Hq + 2 * Hkv
        self.shapes = [(width, H * D), (Hq * D, hidden), (hidden, vocab)]
        u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=device)
        u16 = lambda *s: torch.zeros(*s, dtype=torch.uint16, device=device)
        f32 = lambda *s: torch.zeros(*s, dtype=torch.float32, device=device)
        self.W16, self.V16, self.dW16 = ([u16(*s) for s in self.shapes] for _ in range(3))
        self.W8 = [u8(*s) for s in self.shapes[:2]]
        self.X8 = u8(T, width)
        self.QKV16, self.QKV8, self.dQKV16, self.dQKV8 = u16(T, H, D), u8(T, H, D), u16(T, H, D), u8(T, H, D)
        self.O16, self.O8, self.dO8, self.lse = u16(T, Hq, D), u8(T, Hq, D), u8(T, Hq, D), f32(Hq, T)
        self.H16, self.H8, self.A16, self.dA16 = u16(T, hidden), u8(T, hidden), u16(T, hidden), u16(T, hidden)
        self.E8, self.Y16, self.E16, self.loss = u8(T, hidden), u16(T, vocab), u16(T, vocab), f32(T)
        starts = np.concatenate([[0], np.cumsum(self.lengths)])
        self.cu = torch.from_numpy(starts.astype(np.int64)).to(device)
        positions = np.concatenate([np.arange(n) for n in self.lengths]).astype(np.int64)
        self.positions = torch.from_numpy(positions).to(device)
        freqs, self.mscale = rotary_freqs(D // 2 * 2, base)
        self.freqs = torch.from_numpy(freqs).to(device)
        part = lambda x: (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
        self.q, self.k, self.v = part(self.QKV8)
        self.dq, self.dk, self.dv = part(self.dQKV16)
        longest = max(self.lengths, default=0)
        self.attn = (self.q, self.k, self.v, self.cu, self.cu, longest, longest, True, 1.0 / math.sqrt(D))
        need = [attn_fwd_fp8_workspace_size(*self.attn), attn_bwd_fp8_workspace_size(*self.attn)]
        for i, (n, m) in enumerate(self.shapes):
            if i == 2:
                need += [chunk_gemm_p16_workspace_size(0, 0, T, m, n, CL),
                         chunk_gemm_p16_workspace_size(0, 1, T, n, m, CL),
                         chunk_gemm_p16_workspace_size(1, 0, n, m, T, CL)]
            else:
                need += [chunk_gemm_fp8_workspace_size(0, 0, T, m, n, CL, mode),
                         chunk_gemm_fp8_workspace_size(0, 1, T, n, m, CL, mode),
                         chunk_gemm_workspace_size(1, 0, n, m, T, CL, mode)]
        self.ws_bytes = max(need)
        self.ws = u8(max(1, self.ws_bytes))

    def set_weights(self, W16_codes):
        """FP16 master weights (numpy uint16 codes: Wqkv, Wo, Wl); their FP8
        copies are their quantization, the momentum buffers start at 0."""
        torch = self.torch
        for i, codes in enumerate(W16_codes):
            t = torch.from_numpy(np.ascontiguousarray(codes, np.uint16).view(np.int16))
            self.W16[i].copy_(t.to(self.dev).view(torch.uint16))
            self.V16[i].zero_()
            if i < 2:
                fp8_quantize(self.W16[i], self.W8[i])

    def step(self, X8, idx, logits, weights, tau, lr, momentum, weight_decay, loss_scale, seed, t):
        """X8: FP8 features of the tokens (T x width); idx, logits: the
        teacher's entries (T x k); weights: per-token weights of the loss (1 /
        tokens for a mean).  Returns the tokens' losses."""
        T, CL, mode, ws = self.T, self.CL, self.mode, (self.ws, self.ws_bytes)
        (w0, w1), (o0, h), (_, V) = self.shapes
        turned = self.Hq + self.Hkv
        self.X8.copy_(X8)
        chunk_gemm_fp8(0, 0, T, w1, w0, CL, self.X8, w0, self.W8[0], w1, self.QKV16, w1, self.QKV8, w1,
                       1.0, mode, *ws)
        rotary_embed(self.QKV16[:, :turned], self.positions, self.freqs, self.QKV8[:, :turned],
                     mscale=self.mscale)
        attn_fwd_fp8(*self.attn, self.O16, self.O8, 1.0, self.lse, *ws)
        chunk_gemm_fp8(0, 0, T, h, o0, CL, self.O8, o0, self.W8[1], h, self.H16, h, self.H8, h, 1.0,
                       mode, *ws)
        relu_codes(self.H16, 16, self.A16, T * h)
        chunk_gemm_p16(0, 0, T, V, h, CL, self.A16, h, self.W16[2], V, self.Y16, V, *ws)
        distill_loss(self.Y16, idx, logits, weights, tau, loss_scale, self.loss, self.E16)
        chunk_gemm_p16(0, 1, T, h, V, CL, self.E16, V, self.W16[2], V, self.dA16, h, *ws)
        chunk_gemm_p16(1, 0, h, V, T, CL, self.A16, h, self.E16, V, self.dW16[2], V, *ws)
        relu_backward_fp8(self.dA16, self.H16, self.E8, T * h, 1.0)
        chunk_gemm(1, 0, o0, h, T, CL, self.O8, o0, self.E8, h, self.dW16[1], h, mode, *ws)
        chunk_gemm_fp8(0, 1, T, o0, h, CL, self.E8, h, self.W8[1], h, None, o0, self.dO8, o0, 1.0, mode,
                       *ws)
        attn_bwd_fp8(*self.attn, self.O16, self.dO8, self.lse, self.dq, self.dk, self.dv, 1.0, *ws)
        fp8_quantize(self.dQKV16, self.dQKV8)
        rotary_embed(self.dQKV16[:, :turned], self.positions, self.freqs, self.dQKV8[:, :turned],
                     inverse=True, mscale=self.mscale)
        chunk_gemm(1, 0, w0, w1, T, CL, self.X8, w0, self.dQKV8, w1, self.dW16[0], w1, mode, *ws)
        lr_eff = float(np.float32(lr) / np.float32(loss_scale))
        wd_eff = float(np.float32(weight_decay) * np.float32(loss_scale))
        for i, (n, m) in enumerate(self.shapes):
            sr_weight_update(self.W16[i], self.dW16[i], self.V16[i], self.W8[i] if i < 2 else None, n * m,
                             lr_eff, momentum, wd_eff, seed, t * 3 + i)
        return self.loss
