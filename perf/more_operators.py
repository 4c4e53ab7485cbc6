"""Workloads of the operators of a cache held in codes of 4 or 8 bits, for timing and comparing them.

Three operators, each through `paper_2604_13349_amd.binding` as a program calls it (`own`), or in plain torch operations:

  store    new keys and values quantised into the cache behind what every head holds already, and the written rows read back
  read     rows of such a cache by their numbers, or all rows, as bf16 or fp32 again
  attend   attention of one sample's or a batch's queries over such a cache, in which every KV head has its own number of rows:
           causal, with or without a sliding window and first rows that stay visible

A row x of d values is held as d codes q and two half-precision numbers: with L = 2^bits - 1, zero = fp16(min x), scale =
fp16((max x - min x) / L), q = clamp(rint((x - zero) / scale), 0, L), decided in single precision, each operation rounded by itself;
it stands for zero + scale * q.

Keys and values are drawn as the benchmark's synthetic caches are: a low-rank part plus noise under a log-normal scale per channel,
a hundredth of a sample's tokens eight times as large; queries are i.i.d. normal.
"""
import math

import numpy as np
import torch

own = False

LOWRANK, OUTLIER_FRAC, OUTLIER_SCALE = 16, 0.01, 8.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _attend(name, bits, dtype, d, samples, heads, group, queries, stride, len_lo, len_hi, **more):
    """Heads hold len_lo to len_hi rows of `stride`; window 0: none; sink_hi > sink: between sink and sink_hi first rows per head."""
    c = {"name": name, "kind": "attend", "bits": bits, "dtype": dtype, "d": d, "samples": samples, "heads": heads, "group": group, "queries": queries,
         "stride": stride, "len_lo": len_lo, "len_hi": len_hi, "window": 0, "sink": 0, "sink_hi": 0}
    c.update(more)
    return c


def _store(name, bits, dtype, d, samples, heads, rows, new_lo, new_hi, before_lo, before_hi, token_major):
    """new_lo to new_hi of `rows` rows per head go behind before_lo to before_hi rows; token_major: [samples, rows, heads, d] in memory."""
    return {"name": name, "kind": "store", "bits": bits, "dtype": dtype, "d": d, "samples": samples, "heads": heads, "rows": rows, "new_lo": new_lo,
            "new_hi": new_hi, "before_lo": before_lo, "before_hi": before_hi, "token_major": token_major}


def _read(name, bits, dtype, d, samples, heads, stride, len_lo, len_hi, picked):
    """picked: that many rows of every head by their numbers; 0: all."""
    return {"name": name, "kind": "read", "bits": bits, "dtype": dtype, "d": d, "samples": samples, "heads": heads, "stride": stride, "len_lo": len_lo,
            "len_hi": len_hi, "picked": picked}


def listed():
    return [
        # one sample generates behind a relayed message of the method's own setting (a few hundred rows): latency is all there is
        _attend("attend4_one_sample", 4, "bf16", 128, 1, 8, 4, 1, 512, 100, 340),
        # sixteen samples generate over long caches, some four times as long as others
        _attend("attend4_long_ragged", 4, "bf16", 128, 16, 8, 4, 1, 32768, 8192, 32768),
        # the same with codes of 8 bits and thirty-two shorter caches
        _attend("attend8_decode", 8, "bf16", 128, 32, 8, 4, 1, 4096, 1000, 4096),
        # generation with a sliding window behind a message that stays visible, five query heads per KV head
        _attend("attend4_window", 4, "bf16", 128, 48, 8, 5, 1, 8192, 3001, 8100, window=1024, sink=20, sink_hi=36),
        # a receiver reads its own prompt of 4096 tokens behind a message of 9421 rows
        _attend("attend4_prompt", 4, "bf16", 128, 1, 8, 4, 4096, 14000, 13517, 13517),
        # prompts of 500 tokens behind messages of different lengths, head_dim 64, 8 bits
        _attend("attend8_prompt_ragged", 8, "bf16", 64, 3, 8, 5, 500, 2200, 700, 2139),
        # a single-precision model of two KV heads: a short odd prompt behind messages of different lengths
        _attend("attend4_fp32", 4, "f32", 64, 3, 2, 2, 333, 600, 333, 512),
        # one step of thirty-two samples: a row per head
        _store("store4_step", 4, "bf16", 128, 32, 8, 1, 1, 1, 1000, 4095, True),
        # four prompts of 8192 tokens as the projections leave them
        _store("store4_prompts", 4, "bf16", 128, 4, 8, 8192, 8192, 8192, 0, 0, True),
        # every layer of an 8B-shaped model: the rows that compression kept, behind an inherited message of 20 to 36 rows
        _store("store8_message", 8, "bf16", 128, 36, 8, 1229, 800, 1229, 20, 36, False),
        # every layer of an 8B-shaped model: 1229 rows of each head, by their numbers
        _read("read4_kept", 4, "bf16", 128, 36, 8, 8192, 7000, 8192, 1229),
        # a small single-precision cache of odd lengths, whole
        _read("read8_fp32", 8, "f32", 64, 3, 2, 517, 100, 517, 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "prompt", "prompt", "fp32", "store", "store", "read"])
    bits, dtype, d = rng.choice([4, 4, 8]), "bf16", rng.choice([64, 128, 128])
    heads, group = rng.choice([2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 5, 8])
    if kind == "store":
        rows = rng.choice([1, 1, _log_int(rng, 2, 8192)])
        samples = max(1, min(_log_int(rng, 1, 64), 32 * 8192 // (rows * 8)))
        before = rng.choice([0, _log_int(rng, 1, 4000)])
        dt = rng.choice(["bf16", "bf16", "f32"])
        c = _store("", bits, dt, d, samples, heads, rows, rng.randint(max(1, rows // 2), rows), rows, rng.randint(before // 2, before), before,
                   rng.random() < 0.6)
        if dt == "f32":
            c["samples"] = max(1, samples // 2)
    elif kind == "read":
        n = _log_int(rng, 16, 8192)
        samples = max(1, min(_log_int(rng, 1, 40), 36 * 8192 // n))
        lo = rng.randint(max(1, n // 4), n)
        c = _read("", bits, rng.choice(["bf16", "bf16", "f32"]), d, samples, heads, n + rng.randint(0, 70), lo, n,
                  rng.choice([0, rng.randint(1, max(1, lo // 8))]))
        c["samples"] = max(1, samples // ((8 if c["picked"] == 0 else 1) * (2 if c["dtype"] == "f32" else 1)))
    else:
        more = {}
        if kind == "decode":
            queries = rng.choice([1, 1, 1, 2, 5])
            n = max(queries, _log_int(rng, 1, 32768))
            samples = max(1, min(_log_int(rng, 1, 64), 64 * 32768 // (bits * n)))
            lo = rng.randint(max(queries, n // 4), n)
        elif kind == "prompt":
            queries = _log_int(rng, 17, 4000)
            n = queries + rng.choice([0, _log_int(rng, 1, 9000)])
            lo = rng.randint(queries, n)
            samples = max(1, min(rng.randint(1, 6), int(5e7 / (queries * n))))
            group = min(group, 32 // heads)
        else:
            dtype, queries = "f32", rng.choice([1, 1, 3, _log_int(rng, 2, 700)])
            n = queries + _log_int(rng, 1, 2000)
            lo, samples = rng.randint(queries, n), rng.randint(1, 4)
        if rng.random() < 0.35:
            more.update(window=_log_int(rng, 16, 2048), sink=rng.choice([0, 4, 4]))
            if rng.random() < 0.4:
                more["sink_hi"] = more["sink"] + rng.randint(1, 40)
        c = _attend("", bits, dtype, d, samples, heads, group, queries, n + rng.randint(0, 70), lo, n, **more)
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


def _rows(gen, samples, heads, n, d, dtype):
    """K, V of one sample after the other, [heads, n, d] each."""
    for _ in range(samples):
        out = torch.randperm(n, generator=gen, device="cuda")[: int(round(OUTLIER_FRAC * n))]
        yield tuple(_structured(gen, heads, n, d, out).to(dtype) for _ in range(2))


def _quantise(x, bits):
    """[..., d] -> codes [..., d * bits / 8], scale, zero [...]."""
    L = (1 << bits) - 1
    x = x.float()
    lo, hi = x.amin(dim=-1), x.amax(dim=-1)
    zero, scale = lo.half(), ((hi - lo) / float(L)).half()
    s = scale.float()[..., None]
    q = torch.round((x - zero.float()[..., None]) / s).clamp(0, L)
    q = torch.where(s > 0, q, torch.zeros_like(q)).to(torch.uint8)
    if bits == 4:
        q = q[..., 0::2] | (q[..., 1::2] << 4)
    return q, scale, zero


def _values(codes, scale, zero, bits):
    """What codes stand for, float32 [..., d]."""
    if bits == 4:
        codes = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    return zero.float()[..., None] + scale.float()[..., None] * codes.float()


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _lens(case):
    """(rows per head, first rows that stay visible per head), [samples, heads] each."""
    shape = (case["samples"], case["heads"])
    n = _spread(case["len_lo"], case["len_hi"], shape[0] * shape[1]).reshape(shape)
    sink, sink_hi = case.get("sink", 0), case.get("sink_hi", 0)
    return n, _spread(sink, max(sink, sink_hi), shape[0] * shape[1]).reshape(shape)


def _news(case):
    """(rows before, new rows) per head, [samples, heads] each."""
    shape = (case["samples"], case["heads"])
    count = shape[0] * shape[1]
    return _spread(case["before_lo"], case["before_hi"], count).reshape(shape), _spread(case["new_lo"], case["new_hi"], count)[::-1].reshape(shape)


def _room(case):
    """Rows between the heads of the case's cache."""
    return case["stride"] if case["kind"] != "store" else case["before_hi"] + case["rows"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    d, H, S, bits, dt = case["d"], case["heads"], case["samples"], case["bits"], DTYPES[case["dtype"]]
    room = _room(case)
    # the cache: codes, scale, zero of the keys and of the values
    cache = [torch.zeros((S, H, room, d * bits // 8), dtype=torch.uint8, device="cuda") if i % 3 == 0 else
             torch.zeros((S, H, room), dtype=torch.float16, device="cuda") for i in range(6)]
    s = {"case": case, "cache": cache, "out": None, "own": None}
    if case["kind"] == "store":
        before, new = _news(case)
        s["len"], s["new"] = _dev(before + new), _dev(new)
        n = case["rows"]
        shape = (S, n, H, d) if case["token_major"] else (S, H, n, d)
        s["K"], s["V"] = (torch.empty(shape, dtype=dt, device="cuda") for _ in range(2))
        if case["token_major"]:
            s["K"], s["V"] = s["K"].transpose(1, 2), s["V"].transpose(1, 2)
        for i, (k, v) in enumerate(_rows(gen, S, H, n, d, dt)):
            s["K"][i], s["V"][i] = k, v
        # the numbers of the written rows, -1 behind them
        t = np.arange(n)
        s["idx"] = _dev(np.where(t < new[..., None], before[..., None] + t, -1))
        return s
    for i, (k, v) in enumerate(_rows(gen, S, H, room, d, dt)):
        for j, x in enumerate(_quantise(k, bits) + _quantise(v, bits)):
            cache[j][i] = x
    n, sink = _lens(case)
    s["len"] = _dev(n)
    if case["kind"] == "read":
        s["idx"] = None
        if case["picked"]:
            # rows of falling weight leave an ascending list with gaps of all sizes
            w = torch.rand((S, H, room), generator=gen, device="cuda").masked_fill_(torch.arange(room, device="cuda") >= s["len"][..., None], -1.0)
            s["idx"] = torch.sort(torch.topk(w, case["picked"], dim=-1).indices, dim=-1).values.int()
        return s
    s["Q"] = torch.randn((S, H * case["group"], case["queries"], d), generator=gen, device="cuda").to(dt)
    s["sink_len"] = _dev(sink) if case["sink_hi"] > case["sink"] else None
    return s


# ------------------------------------------------------------------------------------------------ the plain form
def _plain_read(s, idx, rows):
    """The rows idx (None: the first `rows`) of every head, zeros in the place of rows that it does not have."""
    case, cache = s["case"], s["cache"]
    S, H = case["samples"], case["heads"]
    if idx is None:
        idx = torch.arange(rows, device="cuda").expand(S, H, rows)
    idx = idx.long()
    there = (idx >= 0) & (idx < s["len"][..., None])
    src = torch.where(there, idx, torch.zeros_like(idx))
    out = []
    for x in (cache[:3], cache[3:]):
        codes = torch.gather(x[0], 2, src[..., None].expand(*src.shape, x[0].shape[-1]))
        y = _values(codes, torch.gather(x[1], 2, src), torch.gather(x[2], 2, src), case["bits"])
        out.append((y * there[..., None]).to(DTYPES[case["dtype"]]))
    return {"K_out": out[0], "V_out": out[1]}


def _plain_store(s):
    case = s["case"]
    S, H, n, room = case["samples"], case["heads"], case["rows"], _room(case)
    t = torch.arange(n, device="cuda")
    new = s["new"].long()
    head = torch.arange(S * H, device="cuda").view(S, H, 1) * room
    there = t < new[..., None]
    at = (head + (s["len"].long() - new)[..., None] + t)[there]
    for x, first in ((s["K"], 0), (s["V"], 3)):
        for j, y in enumerate(_quantise(x, case["bits"])):
            held = s["cache"][first + j]
            held.view((S * H * room,) + tuple(held.shape[3:]))[at] = y[there]
    return _plain_read(s, s["idx"], n)


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
    S, H, G, T, d, L = case["samples"], case["heads"], case["group"], case["queries"], case["d"], case["len_hi"]
    dt = DTYPES[case["dtype"]]
    O = torch.empty((S, H, G, T, d), dtype=dt, device="cuda")
    lse = torch.empty((S, H, G, T), device="cuda")
    sink_len = s["sink_len"] if s["sink_len"] is not None else torch.full_like(s["len"], case["sink"])
    # as many samples, or else as many queries of one, as keep the table of scores near a gigabyte
    nb = max(1, (1 << 28) // (H * G * T * L))
    tb = T if nb > 1 else max(1, (1 << 28) // (H * G * L))
    for b in range(0, S, nb):
        e = min(S, b + nb)
        k, v = (_values(x[0][b:e, :, :L], x[1][b:e, :, :L], x[2][b:e, :, :L], case["bits"]) for x in (s["cache"][:3], s["cache"][3:]))
        n, sk = s["len"][b:e, :, None, None], sink_len[b:e, :, None, None]
        for t0 in range(0, T, tb):
            t1 = min(T, t0 + tb)
            q = s["Q"][b:e].view(e - b, H, G, T, d)[:, :, :, t0:t1].float().reshape(e - b, H, G * (t1 - t0), d)
            x = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d)
            x.masked_fill_(~_visible(n, sk, T, t0, t1, G, L, case["window"]), -math.inf)
            m = x.amax(dim=-1, keepdim=True)
            m = torch.where(m > -math.inf, m, torch.zeros_like(m))
            w = torch.exp(x - m)
            z = w.sum(dim=-1, keepdim=True)
            lse[b:e, :, :, t0:t1] = (m + torch.log(z)).view(e - b, H, G, t1 - t0)
            w /= torch.where(z > 0, z, torch.ones_like(z))
            O[b:e, :, :, t0:t1] = torch.matmul(w, v).view(e - b, H, G, t1 - t0, d).to(dt)
    return {"O": O.view(S, H * G, T, d), "lse": lse.view(S, H * G, T)}


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if not own:
        if case["kind"] == "attend":
            return _plain_attend(s)
        return _plain_store(s) if case["kind"] == "store" else _plain_read(s, s["idx"], case["picked"] or case["stride"])
    from paper_2604_13349_amd import binding as B

    if s["own"] is None:
        s["own"] = B.CodeCache(*s["cache"], d=case["d"], bits=case["bits"])
    if case["kind"] == "attend":
        s["out"] = B.attend_codes(s["Q"], s["own"], kv_len=s["len"], window=case["window"], sink=case["sink"], sink_len=s["sink_len"], out=s["out"])
        return {"O": s["out"]["O"], "lse": s["out"]["lse"]}
    if s["out"] is None:
        # the rows that the program goes on with; those that a head does not have stay as they are
        n = case["rows"] if case["kind"] == "store" else case["picked"] or case["stride"]
        s["out"] = {k: torch.zeros((case["samples"], case["heads"], n, case["d"]), dtype=DTYPES[case["dtype"]], device="cuda") for k in ("K_out", "V_out")}
    if case["kind"] == "store":
        B.cache_write(s["own"], s["K"], s["V"], kv_len=s["len"], n_new=s["new"])
    s["out"] = B.cache_read(s["own"], DTYPES[case["dtype"]], kv_len=s["len"], idx=s["idx"], out=s["out"])
    return {"K_out": s["out"]["K_out"], "V_out": s["out"]["V_out"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    d, es = case["d"], 2 if case["dtype"] == "bf16" else 4
    held = d * case["bits"] // 8 + 4                     # bytes of a row in the cache
    if case["kind"] == "store":
        # new rows in, their codes and what these stand for out; a subtraction, a division, a rounding, two comparisons, a product and a sum per value
        rows = int(_news(case)[1].sum())
        return {"bytes": float(2 * rows * (held + 2 * d * es) + 4 * rows), "flops": 14.0 * d * rows}
    if case["kind"] == "read":
        n = _lens(case)[0]
        rows = case["picked"] * n.size if case["picked"] else int(n.sum())
        return {"bytes": float(2 * rows * (held + d * es) + (4 * rows if case["picked"] else 0)), "flops": 4.0 * d * rows}
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
    return {"bytes": float(rows * 2 * held + S * H * G * T * (2 * d * es + 4)), "flops": 4.0 * d * G * pairs}


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_codes(x, bits):
    """Rows [n, d] in 64 bits: (codes, scale, zero); every operation of the decision is rounded to single precision by itself."""
    L = 2.0 ** bits - 1.0
    x = x.double()
    low, high = x.min(dim=1).values, x.max(dim=1).values
    zero = low.to(torch.float16).double()
    scale = ((high - low).float().double() / L).float().to(torch.float16).double()
    part = (x - zero[:, None]).float().double() / scale[:, None].clamp(min=2.0 ** -30)
    q = torch.round(part.float().double()).clamp(0.0, L)
    return q * (scale > 0)[:, None], scale, zero


def _exact_held(codes, scale, zero, d, bits):
    """Rows [n, bytes] of a cache in 64 bits."""
    out = torch.empty((codes.shape[0], d), dtype=torch.float64, device=codes.device)
    if bits == 8:
        out[:] = codes
    else:
        out[:, 0::2] = codes.long().remainder(16).double()
        out[:, 1::2] = torch.div(codes.long(), 16, rounding_mode="floor").double()
    return out.mul_(scale.double()[:, None]).add_(zero.double()[:, None])


def exact(case, seed):
    s = prepare(case, seed)
    S, H, d, bits = case["samples"], case["heads"], case["d"], case["bits"]
    if case["kind"] == "store":
        before, new = _news(case)
        out = [torch.zeros((S, H, case["rows"], d), dtype=torch.float64, device="cuda") for _ in range(2)]
        for b in range(S):
            for h in range(H):
                n = int(new[b, h])
                for y, x in zip(out, (s["K"], s["V"])):
                    q, scale, zero = _exact_codes(x[b, h, :n], bits)
                    y[b, h, :n] = zero[:, None] + scale[:, None] * q
        return {"K_out": out[0], "V_out": out[1]}
    lens, sinks = _lens(case)
    if case["kind"] == "read":
        rows = case["picked"] or case["stride"]
        out = [torch.zeros((S, H, rows, d), dtype=torch.float64, device="cuda") for _ in range(2)]
        for b in range(S):
            for h in range(H):
                at = s["idx"][b, h].long() if case["picked"] else torch.arange(int(lens[b, h]), device="cuda")
                for y, x in zip(out, (s["cache"][:3], s["cache"][3:])):
                    y[b, h, : at.numel()] = _exact_held(x[0][b, h, at], x[1][b, h, at], x[2][b, h, at], d, bits)
        return {"K_out": out[0], "V_out": out[1]}
    G, T, W = case["group"], case["queries"], case["window"]
    O = torch.zeros((S, H * G, T, d), dtype=torch.float64, device="cuda")
    lse = torch.full((S, H * G, T), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(S):
        for h in range(H):
            n, sk = int(lens[b, h]), int(sinks[b, h])
            keys, vals = (_exact_held(x[0][b, h, :n], x[1][b, h, :n], x[2][b, h, :n], d, bits) for x in (s["cache"][:3], s["cache"][3:]))
            row = torch.arange(n, device="cuda")
            step = max(1, (1 << 26) // n)
            for t0 in range(0, T, step):
                t1 = min(T, t0 + step)
                at = torch.arange(n - T + t0, n - T + t1, device="cuda")[:, None]
                hidden = row > at
                if W:
                    hidden |= (row >= sk) & (at - row >= W)
                for g in range(G):
                    z = (s["Q"][b, h * G + g, t0:t1].double() @ keys.t()) * d ** -0.5
                    z[hidden] = -math.inf
                    c = torch.logsumexp(z, dim=1)
                    lse[b, h * G + g, t0:t1] = c
                    O[b, h * G + g, t0:t1] = torch.exp(z - torch.where(torch.isinf(c), torch.zeros_like(c), c)[:, None]) @ vals
    return {"O": O, "lse": lse}
