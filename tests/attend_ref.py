"""The operators on a relayed cache from their definitions, in 64 bits, one query row at a time; and how far the kernels may be off.

Bounds (u = 2^-24, half a step of single precision): a logit of d products summed in single precision is off by at most
dx = (d + 8) u sum_c |q_c k_c| / sqrt(d) (products of bf16 values are exact, those of fp32 values rounded once; 8 more for the
scale, the reference and the exponential's argument); a weight by a factor of 1 + 2 dx + (n + 16) u, the n for the sum it is divided
by.  The weights enter the product with V with a relative error of p_eps.  The result is then rounded once to its type."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def visible(n, T, t, causal, window, sink):
    """Row numbers that query t of a head of n rows sees."""
    p = n - T + t
    return [j for j in range(n) if not causal or (j <= p and (window == 0 or j > p - window or j < sink))]


def attend(Q, K, V, kv_len, causal=True, window=0, sink=0, sink_len=None, prefix=None, p_eps=2.0 ** -8):
    """Q [S,Hq,T,d], K, V [S,H,R,d] on the CPU; prefix: (K, V, len).  Returns O, lse, the mass added, and bounds on their errors."""
    S, Hq, T, d = Q.shape
    H, R = K.shape[1], K.shape[2]
    g = Hq // H
    half = HALF[Q.dtype]
    O = torch.zeros((S, Hq, T, d), dtype=torch.float64)
    lse = torch.full((S, Hq, T), -math.inf, dtype=torch.float64)
    mass = torch.zeros((S, H, R), dtype=torch.float64)
    tol_O, tol_lse, tol_mass = torch.zeros_like(O), torch.zeros_like(lse), torch.zeros_like(mass)
    Qd = Q.double()
    for s in range(S):
        for h in range(H):
            n = int(kv_len[s, h])
            n = n if 0 <= n <= R else 0
            sk = max(0, int(sink_len[s, h]) if sink_len is not None else sink)
            pk = pv = torch.zeros((0, d), dtype=torch.float64)
            if prefix is not None and 0 <= int(prefix[2][h]) <= prefix[0].shape[1]:
                pk, pv = (x[h, : int(prefix[2][h])].double() for x in prefix[:2])
            P = pk.shape[0]
            for t in range(T):
                at = torch.tensor(visible(n, T, t, causal, window, sk), dtype=torch.long)
                k, v = torch.cat([pk, K[s, h, at].double()]), torch.cat([pv, V[s, h, at].double()])
                if k.shape[0] == 0:
                    continue
                q = Qd[s, h * g:(h + 1) * g, t]
                x = q @ k.t() / math.sqrt(d)
                c = torch.logsumexp(x, dim=1)
                w = torch.exp(x - c[:, None])
                dx = ((d + 8) * U * (q.abs() @ k.abs().t()).amax(dim=1) / math.sqrt(d))[:, None]
                e = 2 * dx + (k.shape[0] + 16) * U
                O[s, h * g:(h + 1) * g, t] = w @ v
                tol_O[s, h * g:(h + 1) * g, t] = (w @ v).abs() * half * 1.01 + (w @ v.abs()) * (e + p_eps)
                lse[s, h * g:(h + 1) * g, t] = c
                tol_lse[s, h * g:(h + 1) * g, t] = (dx + (k.shape[0] + 16) * U).amax(dim=1) + 4 * U * c.abs()
                mass[s, h, at] += w[:, P:].sum(dim=0)
                # a row's sum takes g T terms; lse enters as a rounded number of its own error
                tol_mass[s, h, at] += (w[:, P:] * (2 * e + g * T * U + 8 * U * c.abs()[:, None])).sum(dim=0)
    return O, lse, mass, tol_O, tol_lse, tol_mass


def evict(mass, n, budget, recent, sink):
    """Rows of one head that are kept, ascending: mass [n rows or more]."""
    first = min(sink, n)
    keep = min(budget, n - first)
    if first + keep == n:
        return list(range(n))
    middle = sorted(range(first, n - recent), key=lambda j: (-float(mass[j]), j))[: budget - recent]
    return list(range(first)) + sorted(middle) + list(range(n - recent, n))
