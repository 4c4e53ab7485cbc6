"""Attention over a cache held in codes from its definition, in 64 bits, one query row at a time; and how far the kernels may be off.

Bounds, as in attend_ref (u = 2^-24), with a row's two numbers taken apart, since the kernels sum scale times codes and zeros separately: a logit is off by at most
dx = (d + 8) u sum_c |q_c| (|s| c + |z|) / sqrt(d), a weight by a factor of 1 + 2 dx + (n + 16) u.  Beside that
  few rows    fp32 queries enter as two parts of 11 bits (taken as 2^-22 of an element; 2^-23 at most), every element with 2^-25 beside a largest of 2^14 or more (2^-39 of it); weights
              times scale with 2^-11 (bf16) or 2^-22 (fp32) and 2^-25 beside a largest of 2^7 or more (2^-32 of the largest, in which a scale of 0 counts as
              2^-24), times codes up to L; with bf16, sums of V's codes drop what lies 2^-20 below a largest product
  many rows   queries with 2^-39 of the largest element, their sum with 2^-33 of it and 2^-25 beside one of up to 2^8 times 2^14 (2^-24 of the largest element, for
              values up to |zero| + 2^(bits - 1) |scale|); V's values rounded to half precision, 2^-11 of the value and 2^-25, weights with 2^-11 and 2^-32 of the largest
bf16 calls of more than 64 rows take one or the other by their sizes: the larger of both bounds.  The result is then rounded once to its type."""
import math

import torch

from tests.attend_ref import HALF, U, visible

FEW = 64


def quantise(x, bits):
    """[..., d] -> (codes uint8 [..., d], scale, zero float16 [...]), single precision, each operation rounded by itself."""
    L = float((1 << bits) - 1)
    x = x.float()
    lo, hi = x.amin(-1), x.amax(-1)
    zero, scale = lo.half(), ((hi - lo) / L).half()
    q = torch.round((x - zero.float()[..., None]) / scale.float()[..., None]).clamp(0, L)
    return torch.where(scale.float()[..., None] > 0, q, torch.zeros_like(q)).to(torch.uint8), scale, zero


def pack(codes, bits):
    return codes if bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(codes, bits):
    return codes if bits == 8 else torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)


def values(codes, scale, zero):
    return zero.double()[..., None] + scale.double()[..., None] * codes.double()


def attend(Q, K, V, bits, kv_len, causal=True, window=0, sink=0, sink_len=None):
    """Q [S,Hq,T,d]; K, V: (codes [S,H,R,d], one code a byte, scale, zero [S,H,R]), all on the CPU.  Returns O, lse and bounds on their errors."""
    S, Hq, T, d = Q.shape
    H, R = K[0].shape[1], K[0].shape[2]
    g, L, f32 = Hq // H, float((1 << bits) - 1), Q.dtype == torch.float32
    kernels = ["few", "many"] if not f32 and g * T > FEW else ["few"]
    O = torch.zeros((S, Hq, T, d), dtype=torch.float64)
    lse = torch.full((S, Hq, T), -math.inf, dtype=torch.float64)
    tol_O, tol_lse = torch.zeros_like(O), torch.zeros_like(lse)
    for s in range(S):
        for h in range(H):
            n = int(kv_len[s, h])
            n = n if 0 <= n <= R else 0
            sk = max(0, int(sink_len[s, h]) if sink_len is not None else sink)
            for t in range(T):
                at = torch.tensor(visible(n, T, t, causal, window, sk), dtype=torch.long)
                if at.numel() == 0:
                    continue
                k, v = values(*(x[s, h, at] for x in K)), values(*(x[s, h, at] for x in V))
                k_abs, v_abs = (values(x[0][s, h, at], x[1][s, h, at].abs(), x[2][s, h, at].abs()) for x in (K, V))
                q = Q[s, h * g:(h + 1) * g, t].double()
                x = q @ k.t() / math.sqrt(d)
                c = torch.logsumexp(x, dim=1)
                w = torch.exp(x - c[:, None])
                qa = q.abs()
                row = slice(h * g, (h + 1) * g)
                O[s, row, t] = w @ v
                for kernel in kernels:
                    dx = (d + 8) * U * (qa @ k_abs.t())
                    if kernel == "many":
                        middle = values(torch.full_like(K[0][s, h, at][:, :1], 1 << (bits - 1)), K[1][s, h, at].abs(), K[2][s, h, at].abs())[:, 0]
                        dx = dx + (2.0 ** -39 * d + 2.0 ** -24) * qa.amax(dim=1)[:, None] * middle
                        dx = dx + (d + 8) * U * qa.sum(dim=1)[:, None] * middle
                        p_eps, spare = 2.0 ** -11, 2.0 ** -32 * w.amax(dim=1)[:, None] * v.abs().sum(dim=0)
                        off = w @ (2.0 ** -11 * v.abs() + 2.0 ** -25)
                    else:
                        codes = values(K[0][s, h, at], K[1][s, h, at].abs(), torch.zeros_like(K[2][s, h, at]))
                        dx = dx + (2.0 ** -22 if f32 else 0.0) * (qa @ codes.t()) + 2.0 ** -39 * qa.amax(dim=1)[:, None] * codes.sum(dim=1)
                        p_eps = 2.0 ** -22 if f32 else 2.0 ** -11 + 2.0 ** -20
                        vs = V[1][s, h, at].double().abs().clamp(min=2.0 ** -24)
                        spare, off = 2.0 ** -32 * L * at.numel() * (w * vs).amax(dim=1)[:, None], 0.0
                    dx = (dx.amax(dim=1) / math.sqrt(d))[:, None]
                    e = 2 * dx + (at.numel() + 16) * U
                    tol_O[s, row, t] = torch.maximum(tol_O[s, row, t], (w @ v).abs() * HALF[Q.dtype] * 1.01 + (w @ v_abs) * (e + p_eps) + off + spare)
                    tol_lse[s, row, t] = torch.maximum(tol_lse[s, row, t], (dx + (at.numel() + 16) * U).amax(dim=1) + 4 * U * c.abs())
                lse[s, row, t] = c
    return O, lse, tol_O, tol_lse
