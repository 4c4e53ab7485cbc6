"""Workloads of the operators that read and thin out a relayed cache, for timing and comparing them.

Three operators, each through `paper_2604_13349_amd.binding` as a program calls it (`own`), or in plain torch operations:

  attend   attention of one sample's or a batch's queries over a cache in which every KV head has its own number of rows: causal,
           with or without a sliding window and first rows that stay visible; `mass`: the weights that a row of the cache receives
           are added to its accumulated attention weight
  shared   the same for samples that all read one message (rows shared by the whole batch) before their own rows; `mass`: the
           accumulated weight of their own rows
  evict    a cache cut to its first rows, its newest rows and the rows of the largest accumulated weight

Keys and values are drawn as the benchmark's synthetic caches are: a low-rank part plus noise under a log-normal scale per channel,
a hundredth of a sample's tokens eight times as large; queries are i.i.d. normal.  Rows behind the end of a head hold what an
earlier, longer sequence would have left there.
"""
import math

import numpy as np
import torch

own = False

LOWRANK, OUTLIER_FRAC, OUTLIER_SCALE = 16, 0.01, 8.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _attend(name, dtype, d, samples, heads, group, queries, stride, len_lo, len_hi, **more):
    """Heads hold len_lo to len_hi rows of `stride`; window 0: none; sink_hi > sink: between sink and sink_hi first rows per head."""
    c = {"name": name, "kind": "attend", "dtype": dtype, "d": d, "samples": samples, "heads": heads, "group": group, "queries": queries,
         "stride": stride, "len_lo": len_lo, "len_hi": len_hi, "window": 0, "sink": 0, "sink_hi": 0, "mass": False, "prefix_lo": 0, "prefix_hi": 0}
    c.update(more)
    return c


def _evict(name, dtype, d, layers, heads, stride, len_lo, len_hi, budget, recent, sink):
    return {"name": name, "kind": "evict", "dtype": dtype, "d": d, "layers": layers, "heads": heads, "stride": stride, "len_lo": len_lo,
            "len_hi": len_hi, "budget": budget, "recent": recent, "sink": sink}


def listed():
    return [
        # one sample generates behind a relayed message of the method's own setting (a few hundred rows): latency is all there is
        _attend("decode_one_sample", "bf16", 128, 1, 8, 4, 1, 512, 100, 340),
        # sixteen samples generate over long caches, some four times as long as others
        _attend("decode_long_ragged", "bf16", 128, 16, 8, 4, 1, 32768, 8192, 32768),
        # generation with a sliding window behind a message that stays visible, five query heads per KV head
        _attend("decode_window", "bf16", 128, 48, 8, 5, 1, 8192, 3001, 8100, window=1024, sink=20, sink_hi=36),
        # generation with a cache that will be thinned out: the weights are accumulated
        _attend("decode_mass", "bf16", 128, 32, 8, 4, 1, 4096, 1000, 4096, mass=True),
        # the receiver reads its own prompt of 8192 tokens behind 1229 retained rows
        _attend("prefill_8k", "bf16", 128, 1, 8, 4, 8192, 9500, 9421, 9421),
        # a longer prompt under a sliding window with four first tokens, head_dim 64
        _attend("prefill_window", "bf16", 64, 1, 8, 4, 16384, 16384, 16384, 16384, window=1024, sink=4),
        # two prompts of 2048 tokens whose cache will be thinned out, five query heads per KV head
        _attend("prefill_mass", "bf16", 128, 2, 8, 5, 2048, 2300, 2048, 2253, mass=True),
        # a single-precision model of two KV heads: a short odd prompt behind messages of different lengths
        _attend("prefill_fp32", "f32", 64, 3, 2, 2, 333, 600, 333, 512),
        # sixty-four continuations of one 8192-token message, each with up to 512 rows of its own
        _attend("shared_decode", "bf16", 128, 64, 8, 4, 1, 512, 1, 512, kind="shared", prefix_lo=8192, prefix_hi=8192),
        # eight receivers of one message (a retained count per head) read prompts of 500 tokens
        _attend("shared_prefill", "bf16", 128, 8, 8, 4, 500, 700, 500, 500, kind="shared", prefix_lo=1639, prefix_hi=3277, mass=True),
        # every layer of an 8B-shaped model: grown caches cut back to 15 %, an eighth of it the newest rows
        _evict("evict_all_layers", "bf16", 128, 36, 8, 8192, 7000, 8192, 1229, 154, 4),
        # the smallest cache: two fp32 heads of 512 rows
        _evict("evict_tiny_fp32", "f32", 64, 1, 2, 512, 512, 512, 64, 16, 4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode_mass", "prefill", "prefill", "prefill_mass", "fp32", "shared_decode", "shared_decode",
                       "shared_prefill", "evict", "evict"])
    dtype, d, heads, group = "bf16", rng.choice([64, 128, 128]), rng.choice([2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 5, 8])
    if kind == "evict":
        n = _log_int(rng, 64, 32768)
        layers = max(1, min(rng.randint(1, 40), 36 * 8192 // n))
        budget = max(8, int(n * rng.uniform(0.05, 0.6)))
        c = _evict("", rng.choice(["bf16", "bf16", "f32"]), d, layers, heads, n + rng.randint(0, 9), rng.randint(n // 2, n), n, budget,
                   rng.randint(0, budget // 2), rng.choice([0, 4, 7]))
        if c["dtype"] == "f32":
            c["layers"] = max(1, layers // 2)
    else:
        more = {}
        if kind in ("decode", "decode_mass"):
            queries = rng.choice([1, 1, 1, 2, 5])
            n = max(queries, _log_int(rng, 1, 32768))
            samples = max(1, min(_log_int(rng, 1, 64), 16 * 32768 // n))
            lo = rng.randint(max(queries, n // 4), n)
            more["mass"] = kind == "decode_mass"
        elif kind in ("prefill", "prefill_mass"):
            queries = _log_int(rng, 17, 6000 if kind == "prefill" else 3000)
            n = queries + rng.choice([0, rng.randint(1, 1300)])
            lo = rng.randint(queries, n)
            samples = max(1, min(rng.randint(1, 6), int(6e7 / (queries * n))))
            more["mass"] = kind == "prefill_mass"
        elif kind == "fp32":
            dtype, queries = "f32", rng.choice([1, 1, 3, _log_int(rng, 2, 700)])
            n = queries + _log_int(rng, 1, 2000)
            lo, samples = rng.randint(queries, n), rng.randint(1, 4)
            more["mass"] = rng.random() < 0.3
        else:
            one = kind == "shared_decode"
            queries = rng.choice([1, 1, 3]) if one else _log_int(rng, 17, 700)
            samples = _log_int(rng, 2, 96) if one else rng.randint(2, 8)
            n = queries + _log_int(rng, 1, 900)
            lo = rng.randint(queries, n)
            p = _log_int(rng, 32, 16384 if one else 4000)
            more.update(kind="shared", prefix_lo=rng.randint(max(1, p // 2), p), prefix_hi=p, mass=rng.random() < 0.3)
        if rng.random() < 0.35:
            more.update(window=_log_int(rng, 16, 2048), sink=rng.choice([0, 4, 4]))
            if rng.random() < 0.4:
                more["sink_hi"] = more["sink"] + rng.randint(1, 40)
        c = _attend("", dtype, d, samples, heads, group, queries, n + rng.randint(0, 70), lo, n, **more)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _spread(lo, hi, count):
    """`count` whole numbers between lo and hi, both among them where there are many, in no order."""
    i = np.arange(count)
    return (hi - (i * 37 % 101) * (hi - lo) // 100).astype(np.int64)


def _structured(gen, heads, n, d, outliers):
    """[heads, n, d] float32: (noise + rank-16 part) under a scale per head and channel, outlier tokens larger."""
    x = torch.randn((heads, n, d), generator=gen, device="cuda")
    f = torch.randn((heads, n, LOWRANK), generator=gen, device="cuda")
    g = torch.randn((heads, LOWRANK, d), generator=gen, device="cuda")
    x.mul_(math.sqrt(0.5)).add_(torch.matmul(f, g), alpha=math.sqrt(0.5 / LOWRANK))
    x.mul_(torch.exp(0.5 * torch.randn((heads, 1, d), generator=gen, device="cuda")))
    x[:, outliers] *= OUTLIER_SCALE
    return x


def _cache(gen, groups, heads, n, d, dtype):
    """K, V [groups, heads, n, d]."""
    K = torch.empty((groups, heads, n, d), dtype=dtype, device="cuda")
    V = torch.empty_like(K)
    for i in range(groups):
        out = torch.randperm(n, generator=gen, device="cuda")[: int(round(OUTLIER_FRAC * n))]
        K[i] = _structured(gen, heads, n, d, out)
        V[i] = _structured(gen, heads, n, d, out)
    return K, V


def _lens(case):
    """(rows per head, first rows that stay visible per head) of the samples' own caches, [samples, heads] each."""
    shape = (case["samples"], case["heads"])
    n = _spread(case["len_lo"], case["len_hi"], shape[0] * shape[1]).reshape(shape)
    s = _spread(case["sink"], max(case["sink"], case["sink_hi"]), shape[0] * shape[1]).reshape(shape)
    return n, s


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    d, H, dt = case["d"], case["heads"], DTYPES[case["dtype"]]
    s = {"case": case, "out": None}
    if case["kind"] == "evict":
        L, n = case["layers"], case["stride"]
        s["K"], s["V"] = _cache(gen, L, H, n, d, dt)
        # weights as a long generation leaves them: a few rows hold most, many hold next to none
        s["mass"] = torch.exp(2.5 * torch.randn((L, H, n), generator=gen, device="cuda"))
        s["pos"] = torch.arange(n, dtype=torch.int32, device="cuda").expand(L, H, n).contiguous()
        s["len"] = _dev(_spread(case["len_lo"], case["len_hi"], L * H).reshape(L, H))
        return s
    S, T = case["samples"], case["queries"]
    s["K"], s["V"] = _cache(gen, S, H, case["stride"], d, dt)
    s["Q"] = torch.randn((S, H * case["group"], T, d), generator=gen, device="cuda").to(dt)
    n, sink = _lens(case)
    s["len"] = _dev(n)
    s["sink_len"] = _dev(sink) if case["sink_hi"] > case["sink"] else None
    if case["kind"] == "shared":
        pk, pv = _cache(gen, 1, H, case["prefix_hi"], d, dt)
        s["prefix_K"], s["prefix_V"] = pk[0], pv[0]
        s["prefix_len"] = _dev(_spread(case["prefix_lo"], case["prefix_hi"], H))
    if case["mass"]:
        # what earlier steps left; a prompt begins with none
        s["mass_before"] = torch.zeros((S, H, case["stride"]), device="cuda")
        if T < 16:
            s["mass_before"] += torch.exp(2.5 * torch.randn((S, H, case["stride"]), generator=gen, device="cuda"))
        s["mass"] = torch.empty_like(s["mass_before"])
    return s


# ------------------------------------------------------------------------------------------------ the plain form
def _visible(n, sink, T, t0, t1, G, L, window):
    """Which of L rows the queries t0 .. t1 of every head see: n, sink [..., 1, 1] -> [..., G * (t1 - t0), L]."""
    j = torch.arange(L, device=n.device)
    p = (n - T) + torch.arange(t0, t1, device=n.device).repeat(G)[:, None]
    see = j <= p
    if window:
        see = see & ((j > p - window) | (j < sink))
    return see


def _plain_attend(s):
    case = s["case"]
    S, H, G, T, d = case["samples"], case["heads"], case["group"], case["queries"], case["d"]
    L = case["len_hi"]
    dt = DTYPES[case["dtype"]]
    O = torch.empty((S, H, G, T, d), dtype=dt, device="cuda")
    lse = torch.empty((S, H, G, T), device="cuda")
    shared = case["kind"] == "shared"
    P = case["prefix_hi"] if shared else 0
    sink_len = s["sink_len"] if s["sink_len"] is not None else torch.full_like(s["len"], case["sink"])
    mass = s["mass_before"].clone() if case["mass"] else None
    if shared:
        pk, pv = s["prefix_K"].float(), s["prefix_V"].float()
        behind = torch.arange(P, device="cuda") >= s["prefix_len"][:, None]                          # [H, P]
    # as many samples, or else as many queries of one, as keep the table of scores near a gigabyte
    nb = max(1, (1 << 28) // (H * G * T * (P + L)))
    tb = T if nb > 1 else max(1, (1 << 28) // (H * G * (P + L)))
    for b in range(0, S, nb):
        e = min(S, b + nb)
        k, v = s["K"][b:e, :, :L].float(), s["V"][b:e, :, :L].float()
        n, sk = s["len"][b:e, :, None, None], sink_len[b:e, :, None, None]
        for t0 in range(0, T, tb):
            t1 = min(T, t0 + tb)
            q = s["Q"][b:e].view(e - b, H, G, T, d)[:, :, :, t0:t1].float().reshape(e - b, H, G * (t1 - t0), d)
            x = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d)
            x.masked_fill_(~_visible(n, sk, T, t0, t1, G, L, case["window"]), -math.inf)
            if shared:
                rows = q.transpose(0, 1).reshape(H, -1, d)                                           # all samples against the message at once
                y = torch.matmul(rows, pk.transpose(-1, -2)) / math.sqrt(d)
                y.masked_fill_(behind[:, None], -math.inf)
                x = torch.cat([y.view(H, e - b, G * (t1 - t0), P).transpose(0, 1), x], dim=-1)
            m = x.amax(dim=-1, keepdim=True)
            m = torch.where(m > -math.inf, m, torch.zeros_like(m))
            w = torch.exp(x - m)
            z = w.sum(dim=-1, keepdim=True)
            lse[b:e, :, :, t0:t1] = (m + torch.log(z)).view(e - b, H, G, t1 - t0)
            w /= torch.where(z > 0, z, torch.ones_like(z))
            o = torch.matmul(w[..., P:], v)
            if shared:
                rows = w[..., :P].transpose(0, 1).reshape(H, -1, P)
                o += torch.matmul(rows, pv).view(H, e - b, G * (t1 - t0), d).transpose(0, 1)
            O[b:e, :, :, t0:t1] = o.view(e - b, H, G, t1 - t0, d).to(dt)
            if mass is not None:
                mass[b:e, :, :L] += w[..., P:].sum(dim=-2)
    out = {"O": O.view(S, H * G, T, d), "lse": lse.view(S, H * G, T)}
    if mass is not None:
        out["mass"] = mass
    return out


def _plain_evict(s):
    case = s["case"]
    n, sink, cap = s["len"].long()[..., None], case["sink"], case["sink"] + case["budget"]
    j = torch.arange(case["stride"], device="cuda")
    first = torch.clamp(n, max=sink)
    count = first + torch.clamp(n - first, max=case["budget"])
    worth = s["mass"].masked_fill((j < first) | (j >= n - case["recent"]), math.inf).masked_fill(j >= n, -1.0)
    order = torch.sort(worth, dim=-1, descending=True, stable=True).indices[..., :cap]
    place = torch.arange(order.shape[-1], device="cuda")
    idx = torch.sort(order.masked_fill(place >= count, case["stride"]), dim=-1).values
    there = place < count
    src = torch.where(there, idx, torch.zeros_like(idx))
    rows = src[..., None].expand(*src.shape, case["d"])
    zero = torch.zeros((), dtype=s["K"].dtype, device="cuda")
    return {"K_out": torch.where(there[..., None], torch.gather(s["K"], 2, rows), zero),
            "V_out": torch.where(there[..., None], torch.gather(s["V"], 2, rows), zero),
            "mass_out": torch.gather(s["mass"], 2, src) * there, "pos_out": torch.gather(s["pos"], 2, src) * there,
            "idx": torch.where(there, idx, torch.full_like(idx, -1)).int(), "len_out": count[..., 0].int()}


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if not own:
        return _plain_evict(s) if case["kind"] == "evict" else _plain_attend(s)
    from paper_2604_13349_amd import binding as B

    if case["kind"] == "evict":
        if s["out"] is None:
            # the caches that the program goes on with; rows behind the end of a head stay as they are
            cap = case["sink"] + case["budget"]
            shape = tuple(s["K"].shape[:2]) + (cap,)
            s["out"] = {"K_out": torch.zeros(shape + (case["d"],), dtype=s["K"].dtype, device="cuda"),
                        "V_out": torch.zeros(shape + (case["d"],), dtype=s["K"].dtype, device="cuda"),
                        "mass_out": torch.zeros(shape, device="cuda"), "pos_out": torch.zeros(shape, dtype=torch.int32, device="cuda")}
        s["out"] = B.evict(s["K"], s["V"], s["mass"], case["budget"], kv_len=s["len"], recent=case["recent"], sink=case["sink"], pos=s["pos"],
                           out=s["out"])
        return {k: s["out"][k] for k in ("K_out", "V_out", "mass_out", "pos_out", "idx", "len_out")}
    how = {"kv_len": s["len"], "window": case["window"], "sink": case["sink"], "sink_len": s["sink_len"]}
    if case["mass"]:
        s["mass"].copy_(s["mass_before"])
    if case["kind"] == "shared":
        s["out"] = B.attend_shared(s["Q"], s["prefix_K"], s["prefix_V"], s["K"], s["V"], prefix_len=s["prefix_len"], out=s["out"], **how)
        if case["mass"]:
            B.attend_mass(s["Q"], s["K"], s["out"]["lse"], s["mass"], **how)
    else:
        s["out"] = B.attend(s["Q"], s["K"], s["V"], mass=s["mass"] if case["mass"] else None, out=s["out"], **how)
    out = {"O": s["out"]["O"], "lse": s["out"]["lse"]}
    if case["mass"]:
        out["mass"] = s["mass"]
    return out


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    d, es = case["d"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "evict":
        n = _spread(case["len_lo"], case["len_hi"], case["layers"] * case["heads"])
        first = np.minimum(n, case["sink"])
        kept = int((first + np.minimum(n - first, case["budget"])).sum())
        # the weights once; of every kept row key, value, weight and position, read and written; its number and the new length
        return {"bytes": float(4 * int(n.sum()) + kept * (2 * (2 * d * es + 8) + 4) + 8 * n.size), "flops": float(n.sum())}
    S, H, G, T, W = case["samples"], case["heads"], case["group"], case["queries"], case["window"]
    pairs = rows = 0
    t = np.arange(T)
    for n, sk in zip(*(a.reshape(-1) for a in _lens(case))):
        p = n - T + t
        p = p[p >= 0]
        if W:
            start = np.maximum(0, p + 1 - W)
            pairs += int((p + 1 - start + np.minimum(start, sk)).sum())
            lo = max(0, n - T + 1 - W)
            rows += int(n - lo + min(lo, sk))
        else:
            pairs += int((p + 1).sum())
            rows += int(n)
    own_rows = rows
    if case["kind"] == "shared":
        p = _spread(case["prefix_lo"], case["prefix_hi"], H)
        pairs += int(p.sum()) * S * T
        rows += int(p.sum())
    q = S * H * G * T
    byts = rows * 2 * d * es + q * (2 * d * es + 4) + (own_rows * 8 if case["mass"] else 0)
    return {"bytes": float(byts), "flops": 4.0 * d * G * pairs}


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_evict(s):
    """Kept rows one head at a time, from the list of its rows in falling order of weight; whole numbers have no value of their own here."""
    case = s["case"]
    L, H, d, cap = case["layers"], case["heads"], case["d"], case["sink"] + case["budget"]
    weight, lens = s["mass"].cpu().numpy(), s["len"].cpu().numpy()
    out = {"K_out": torch.zeros((L, H, cap, d), dtype=torch.float64, device="cuda"), "V_out": torch.zeros((L, H, cap, d), dtype=torch.float64, device="cuda"),
           "mass_out": torch.zeros((L, H, cap), dtype=torch.float64, device="cuda"), "pos_out": None, "idx": None, "len_out": None}
    for l in range(L):
        for h in range(H):
            n, a = int(lens[l, h]), weight[l, h]
            if n <= cap:
                kept = list(range(n))
            else:
                middle = range(case["sink"], n - case["recent"])
                best = sorted(middle, key=lambda j: (-a[j], j))[: case["budget"] - case["recent"]]
                kept = list(range(case["sink"])) + sorted(best) + list(range(n - case["recent"], n))
            at = torch.tensor(kept, dtype=torch.long, device="cuda")
            out["K_out"][l, h, : len(kept)] = s["K"][l, h, at].double()
            out["V_out"][l, h, : len(kept)] = s["V"][l, h, at].double()
            out["mass_out"][l, h, : len(kept)] = s["mass"][l, h, at].double()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "evict":
        return _exact_evict(s)
    S, H, G, T, d, W = (case[k] for k in ("samples", "heads", "group", "queries", "d", "window"))
    lens, sinks = _lens(case)
    O = torch.zeros((S, H * G, T, d), dtype=torch.float64, device="cuda")
    lse = torch.full((S, H * G, T), -math.inf, dtype=torch.float64, device="cuda")
    mass = s["mass_before"].double() if case["mass"] else None
    front = _spread(case["prefix_lo"], case["prefix_hi"], H) if case["kind"] == "shared" else np.zeros(H, dtype=np.int64)
    for b in range(S):
        for h in range(H):
            n, sk, P = int(lens[b, h]), int(sinks[b, h]), int(front[h])
            keys, vals = s["K"][b, h, :n].double(), s["V"][b, h, :n].double()
            if P:
                keys = torch.cat([s["prefix_K"][h, :P].double(), keys])
                vals = torch.cat([s["prefix_V"][h, :P].double(), vals])
            row = torch.arange(-P, n, device="cuda")                  # the message's rows are negative
            step = max(1, (1 << 26) // (G * (P + n)))
            for t0 in range(0, T, step):
                t1 = min(T, t0 + step)
                at = torch.arange(n - T + t0, n - T + t1, device="cuda")[:, None]
                hidden = row > at
                if W:
                    hidden |= (row >= sk) & (at - row >= W)
                hidden &= row >= 0
                q = s["Q"][b, h * G:(h + 1) * G, t0:t1].double()
                for g in range(G):
                    z = (q[g] @ keys.t()) * d ** -0.5
                    z[hidden] = -math.inf
                    c = torch.logsumexp(z, dim=1)
                    lse[b, h * G + g, t0:t1] = c
                    a = torch.exp(z - torch.where(torch.isinf(c), torch.zeros_like(c), c)[:, None])
                    O[b, h * G + g, t0:t1] = a @ vals
                    if mass is not None:
                        mass[b, h, :n] += a[:, P:].sum(dim=0)
    out = {"O": O, "lse": lse}
    if mass is not None:
        out["mass"] = mass
    return out
