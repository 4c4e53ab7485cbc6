"""Attention over a relayed cache, a shared message, accumulated weights and eviction, against their definitions in 64 bits."""
import math

import pytest
import torch

from tests import attend_ref as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _b():
    from paper_2604_13349_amd import binding as B
    return B


def _make(seed, dtype, d, S, H, g, T, rows, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    K = torch.randn((S, H, rows, d), generator=gen)
    K[:, :, ::17] *= 6.0
    V = torch.randn((S, H, rows, d), generator=gen) * torch.exp(torch.randn((S, H, 1, d), generator=gen))
    Q = torch.randn((S, H * g, T, d), generator=gen) * scale
    return Q.to(dtype), K.to(dtype), V.to(dtype)


def _spoil(x, kv_len, value):
    """What lies behind a head's rows must not matter."""
    x = x.clone()
    for s in range(x.shape[0]):
        for h in range(x.shape[1]):
            n = int(kv_len[s, h])
            x[s, h, n if 0 <= n <= x.shape[2] else 0:] = value
    return x


def _lens(seed, S, H, lo, hi):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(lo, hi + 1, (S, H), generator=gen, dtype=torch.int32)


def _check(name, got, want, tol):
    got = got.double().cpu()
    assert torch.isfinite(got).all() or not torch.isfinite(want).all(), f"{name}: not finite"
    same = got == want                                       # infinities of lse among them
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bad.any(), f"{name}: {int(bad.sum())} values off, worst {((got - want).abs() / tol.clamp(min=1e-300))[bad].max():.3g} times the bound"


def _p_eps(dtype, rows):
    """How the weights enter the product with V: as they are, as two bf16 parts (half a step of half a step), as one."""
    return 0.0 if dtype == F32 else 2.0 ** -16 if rows <= 32 else 2.0 ** -8


def _attend_and_check(Q, K, V, kv_len, mass=True, spoil=math.nan, **kw):
    B = _b()
    O, lse, add, tO, tl, tm = R.attend(Q, K, V, kv_len, p_eps=_p_eps(Q.dtype, Q.shape[1] // K.shape[1] * Q.shape[2]), **kw)
    Kd, Vd = _spoil(K, kv_len, spoil).cuda(), _spoil(V, kv_len, spoil).cuda()
    call = dict(kw)
    if kw.get("sink_len") is not None:
        call["sink_len"] = kw["sink_len"].cuda()
    before = torch.rand(K.shape[:3], generator=torch.Generator().manual_seed(1)) * 3
    m = before.cuda() if mass else None
    o = B.attend(Q.cuda(), Kd, Vd, kv_len=kv_len.cuda(), mass=m, **call)
    torch.cuda.synchronize()
    _check("lse", o["lse"], lse, tl)
    _check("O", o["O"], O, tO)
    if mass:
        _check("mass", m, before.double() + add, tm + 2 * R.U * (before.double() + add))
        assert torch.equal(m.cpu()[add == 0], before[add == 0]), "mass of rows that nothing sees"
    return o


CASES = [
    # dtype, d, S, H, g, T, rows, (shortest, longest), causal, window, sink
    (BF, 128, 1, 1, 1, 1, 1, (1, 1), True, 0, 0),
    (BF, 128, 2, 3, 4, 1, 70, (1, 70), True, 0, 0),
    (BF, 64, 3, 2, 8, 1, 33, (1, 33), True, 0, 0),
    (BF, 128, 1, 2, 5, 1, 1100, (900, 1100), True, 0, 0),
    (BF, 128, 2, 2, 4, 1, 600, (300, 600), True, 100, 4),
    (BF, 64, 2, 2, 16, 1, 600, (40, 600), True, 33, 0),
    (BF, 128, 2, 1, 20, 1, 300, (200, 300), True, 64, 40),
    (BF, 128, 1, 2, 4, 3, 400, (3, 400), True, 0, 0),
    (BF, 128, 1, 2, 4, 5, 400, (5, 400), True, 7, 2),
    (BF, 128, 1, 1, 128, 1, 100, (90, 100), True, 0, 0),
    (BF, 128, 1, 2, 4, 65, 200, (65, 200), True, 0, 0),
    (BF, 128, 2, 1, 5, 130, 300, (130, 300), True, 0, 0),
    (BF, 64, 1, 2, 3, 129, 260, (129, 260), True, 50, 3),
    (BF, 128, 1, 1, 2, 257, 257, (257, 257), True, 64, 0),
    (BF, 128, 1, 1, 2, 200, 331, (331, 331), True, 1, 0),
    (BF, 128, 1, 1, 4, 200, 331, (331, 331), True, 1000, 5),
    (BF, 128, 1, 2, 4, 150, 150, (100, 150), False, 0, 0),
    (BF, 64, 1, 2, 1, 1, 300, (100, 300), False, 0, 0),
    (BF, 128, 1, 1, 1, 300, 300, (300, 300), True, 90, 130),
    (BF, 128, 1, 2, 4, 5, 66000, (100, 300), True, 0, 0),
    (BF, 64, 1, 2, 3, 8, 66000, (100, 300), True, 40, 3),
    (BF, 128, 1, 2, 1, 32, 66000, (20, 300), False, 0, 0),
    (BF, 128, 1, 2, 4, 8, 66000, (200, 400), True, 64, 4),
    (BF, 128, 2, 2, 17, 1, 300, (100, 300), True, 0, 0),
    (BF, 128, 1, 1, 33, 1, 300, (100, 300), True, 0, 0),
    (F32, 64, 1, 1, 1, 1, 1, (1, 1), True, 0, 0),
    (F32, 64, 2, 2, 2, 1, 333, (1, 333), True, 0, 0),
    (F32, 128, 2, 2, 5, 1, 700, (500, 700), True, 128, 4),
    (F32, 64, 1, 2, 2, 77, 150, (77, 150), True, 0, 0),
    (F32, 128, 1, 1, 4, 60, 100, (60, 100), True, 9, 1),
    (F32, 128, 1, 1, 3, 33, 65, (65, 65), False, 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{i}-{'bf16' if c[0] == BF else 'f32'}-d{c[1]}-g{c[4]}-T{c[5]}-R{c[6]}-w{c[9]}-s{c[10]}" for i, c in enumerate(CASES)])
def test_attend(case):
    dtype, d, S, H, g, T, rows, (lo, hi), causal, window, sink = case
    Q, K, V = _make(hash((d, S, H, g, T, rows)) & 0xffff, dtype, d, S, H, g, T, rows)
    _attend_and_check(Q, K, V, _lens(5, S, H, lo, hi), causal=causal, window=window, sink=sink)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_heads_without_rows_short_heads_and_bad_lengths(dtype, d, T):
    """Lengths of 0, 1, fewer than the queries, and numbers that are no length: queries that see nothing get 0 and -inf."""
    Q, K, V = _make(3, dtype, d, 3, 3, 2, T, 50)
    kv_len = torch.tensor([[0, 1, 2], [-1, 51, 50], [39, 1 << 30, -(1 << 31)]], dtype=torch.int32)
    o = _attend_and_check(Q, K, V, kv_len, causal=True)
    assert (o["O"][0, :2] == 0).all() and (o["lse"][0, :2] == -math.inf).all()
    assert (o["O"][1, 2:4] == 0).all() and (o["O"][2, 2:] == 0).all()
    _attend_and_check(Q, K, V, kv_len, causal=True, window=3, sink=1)
    _attend_and_check(Q, K, V, kv_len, causal=False)


@pytest.mark.parametrize("T", [1, 4, 90])
def test_first_rows_per_head_stay_visible(T):
    Q, K, V = _make(4, BF, 128, 2, 3, 4, T, 300)
    sink_len = torch.tensor([[0, 10, 299], [-5, 1000, 37]], dtype=torch.int32)
    _attend_and_check(Q, K, V, _lens(2, 2, 3, 100, 300), causal=True, window=20, sink_len=sink_len)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,window", [(2, 0), (13, 5), (40, 0), (70, 11), (150, 64)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_hidden_rows_of_any_value_do_not_reach_a_query(dtype, T, window, value):
    """Rows that later queries see (or, behind a window, earlier ones saw) hold infinities or no numbers: a query that does not see them is as if they were 0."""
    B = _b()
    n = T + 30
    Q, K, V = _make(9, dtype, 128, 1, 2, 2, T, n)
    kv_len = torch.full((1, 2), n, dtype=torch.int32)
    kw = dict(causal=True, window=window, sink=2)
    seen_by_few = n - 2                                    # the last two queries
    for where in ([seen_by_few], [n - T // 2], [25]):
        Kb, Vb, Kz, Vz = K.clone(), V.clone(), K.clone(), V.clone()
        Vb[:, :, where] = value
        Kb[:, 1, where] = value
        clean = torch.tensor([not set(where) & set(R.visible(n, T, t, True, window, 2)) for t in range(T)])
        if not clean.any():
            continue
        O, lse, _, tO, tl, _ = R.attend(Q, Kz, Vz, kv_len, p_eps=_p_eps(dtype, 2 * T), **kw)
        o = B.attend(Q.cuda(), Kb.cuda(), Vb.cuda(), kv_len=kv_len.cuda(), **kw)
        _check("O", o["O"][:, :, clean], O[:, :, clean], tO[:, :, clean])
        _check("lse", o["lse"][:, :, clean], lse[:, :, clean], tl[:, :, clean])
        assert not torch.isfinite(o["O"][:, :, ~clean].float()).all() if (~clean).any() else True


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,rows", [(1, 90), (1, 9000), (40, 90), (40, 9000)])
def test_visible_logits_that_are_no_numbers_reach_the_result(dtype, T, rows):
    """A query, or all visible keys of a head, without numbers: no number comes out, not the zeros of a query that sees nothing; the other rows are as before."""
    B = _b()
    Q, K, V = _make(24, dtype, 128, 1, 2, 2, T, rows)
    # (the other rows' bits may differ: a wave's rows take over larger references together, and a row without numbers never asks for one)
    O, lse, _, tO, tl, _ = R.attend(Q, K, V, torch.full((1, 2), rows), p_eps=_p_eps(dtype, 2 * T))
    Q, K, V = Q.cuda(), K.cuda(), V.cuda()
    bad = Q.clone()
    bad[0, 1, T - 1] = math.nan
    mass = torch.zeros((1, 2, rows), device="cuda")
    o = B.attend(bad, K, V, mass=mass)
    assert torch.isnan(o["O"][0, 1, T - 1]).all() and torch.isnan(o["lse"][0, 1, T - 1])
    assert torch.isnan(mass[0, 0]).all() and torch.isfinite(mass[0, 1]).all()
    keep = torch.ones((4, T), dtype=torch.bool)
    keep[1, T - 1] = False
    _check("O", o["O"][0].cpu()[keep], O[0][keep], tO[0][keep])
    _check("lse", o["lse"][0].cpu()[keep], lse[0][keep], tl[0][keep])
    K[0, 0] = math.nan
    o = B.attend(Q, K, V)
    assert torch.isnan(o["O"][0, :2]).all() and torch.isnan(o["lse"][0, :2]).all()
    _check("O", o["O"][0, 2:], O[0, 2:], tO[0, 2:])
    o = B.attend_shared(Q, K[0, :, :70].contiguous(), V[0, :, :70].contiguous(), K[:, :, :50].contiguous(), V[:, :, :50].contiguous())
    assert torch.isnan(o["O"][0, :2]).all() and torch.isfinite(o["O"][0, 2:].float()).all()


@pytest.mark.parametrize("T", [1, 60])
def test_strided_queries_outputs_and_the_layers_of_a_batch(T):
    """Q and O as [samples, queries, heads, d], the caches as one layer of [samples, layers, heads, rows, d], lengths as one layer of [samples, layers, heads]."""
    B = _b()
    S, L, H, g, rows, d = 3, 4, 2, 3, 190, 128
    Q, K, V = _make(12, BF, d, S, H, g, T, rows)
    kv_len = _lens(8, S, H, T, rows)
    plain = B.attend(Q.cuda(), K.cuda(), V.cuda(), kv_len=kv_len.cuda(), mass=torch.zeros(S, H, rows, device="cuda"))
    wide = torch.randn((S, T, H * g + 2 * H, d), generator=torch.Generator().manual_seed(0)).to(BF).cuda()
    wide[:, :, : H * g] = Q.cuda().transpose(1, 2)
    caches = [torch.full((S, L, H, rows, d), math.nan, dtype=BF, device="cuda") for _ in range(2)]
    caches[0][:, 2], caches[1][:, 2] = K.cuda(), V.cuda()
    lens = torch.full((S, L, H), -7, dtype=torch.int32, device="cuda")
    lens[:, 2] = kv_len.cuda()
    mass = torch.zeros((S, L, H, rows), device="cuda")
    out = {"O": torch.zeros((S, T, H * g, d), dtype=BF, device="cuda").transpose(1, 2)}
    o = B.attend(wide[:, :, : H * g].transpose(1, 2), caches[0][:, 2], caches[1][:, 2], kv_len=lens[:, 2], mass=mass[:, 2], out=out)
    assert torch.equal(o["O"], plain["O"]) and torch.equal(o["lse"], plain["lse"])
    ref = torch.zeros(S, H, rows, device="cuda")
    B.attend(Q.cuda(), K.cuda(), V.cuda(), kv_len=kv_len.cuda(), mass=ref)
    assert torch.equal(mass[:, 2], ref) and (mass[:, [0, 1, 3]] == 0).all()
    # lengths of one layer and first rows of their own make: strides that differ
    sink_len = torch.full((S, H), 3, dtype=torch.int32, device="cuda")
    a = B.attend(Q.cuda(), K.cuda(), V.cuda(), kv_len=lens[:, 2], window=30, sink_len=sink_len)
    b = B.attend(Q.cuda(), K.cuda(), V.cuda(), kv_len=kv_len.cuda(), window=30, sink=3)
    assert torch.equal(a["O"], b["O"])


SHARED = [
    # dtype, d, S, H, g, T, rows, own lengths, message rows, message lengths, window
    (BF, 128, 2, 2, 4, 1, 40, (1, 40), 100, (60, 100), 0),
    (BF, 128, 9, 2, 4, 1, 70, (0, 70), 700, (650, 700), 0),
    (BF, 64, 40, 1, 8, 1, 20, (1, 20), 300, (300, 300), 0),
    (BF, 128, 3, 2, 4, 2, 90, (2, 90), 333, (1, 333), 16),
    (BF, 128, 2, 1, 5, 70, 100, (70, 100), 270, (200, 270), 0),
    (BF, 64, 3, 1, 2, 64, 100, (64, 100), 129, (129, 129), 33),
    (BF, 128, 3, 2, 8, 3, 50, (3, 50), 700, (600, 700), 9),
    (BF, 64, 2, 2, 4, 6, 50, (6, 50), 64, (0, 64), 0),
    (BF, 128, 2, 2, 3, 40, 600, (500, 600), 1000, (900, 1000), 0),
    (F32, 64, 3, 2, 2, 1, 50, (1, 50), 150, (100, 150), 0),
    (F32, 128, 2, 1, 3, 20, 50, (20, 50), 65, (65, 65), 0),
]


@pytest.mark.parametrize("case", SHARED, ids=[f"{i}-{'bf16' if c[0] == BF else 'f32'}-d{c[1]}-S{c[2]}-g{c[4]}-T{c[5]}-P{c[8]}" for i, c in enumerate(SHARED)])
def test_attend_shared(case):
    B = _b()
    dtype, d, S, H, g, T, rows, (lo, hi), P, (plo, phi), window = case
    Q, K, V = _make(21, dtype, d, S, H, g, T, rows)
    _, PK, PV = _make(22, dtype, d, 1, H, g, T, P)
    kv_len, plen = _lens(3, S, H, lo, hi), _lens(4, 1, H, plo, phi)
    kw = dict(causal=True, window=window, sink=2)
    O, lse, add, tO, tl, tm = R.attend(Q, K, V, kv_len, prefix=(PK[0], PV[0], plen[0]), p_eps=_p_eps(dtype, S * T * g), **kw)
    Kd, Vd = _spoil(K, kv_len, math.nan).cuda(), _spoil(V, kv_len, math.nan).cuda()
    PKd, PVd = _spoil(PK, plen, math.nan).cuda()[0], _spoil(PV, plen, math.nan).cuda()[0]
    o = B.attend_shared(Q.cuda(), PKd, PVd, Kd, Vd, prefix_len=plen[0].cuda(), kv_len=kv_len.cuda(), **kw)
    _check("lse", o["lse"], lse, tl)
    _check("O", o["O"], O, tO)
    mass = torch.zeros((S, H, rows), device="cuda")
    B.attend_mass(Q.cuda(), Kd, o["lse"], mass, kv_len=kv_len.cuda(), **kw)
    _check("mass", mass, add, tm + 2 * R.U * add)


def test_shared_message_without_rows_or_with_a_bad_length_is_plain_attention():
    B = _b()
    Q, K, V = (x.cuda() for x in _make(5, BF, 128, 2, 3, 4, 2, 60))
    _, PK, PV = (x.cuda()[0] for x in _make(6, BF, 128, 1, 3, 4, 1, 90))
    kv_len = _lens(9, 2, 3, 2, 60).cuda()
    plain = B.attend(Q, K, V, kv_len=kv_len)
    plen = torch.tensor([0, -1, 91], dtype=torch.int32, device="cuda")
    o = B.attend_shared(Q, PK, PV, K, V, prefix_len=plen, kv_len=kv_len)
    assert (o["lse"] - plain["lse"]).abs().max() <= 1e-5 and (o["O"].float() - plain["O"].float()).abs().max() <= 2.0 ** -8 * plain["O"].float().abs().max()
    # and own caches without rows: the message alone
    none = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    full = torch.tensor([90, 5, 33], dtype=torch.int32, device="cuda")
    o = B.attend_shared(Q, PK, PV, K, V, prefix_len=full, kv_len=none)
    want = B.attend(Q, PK.expand(2, 3, 90, 128).contiguous(), PV.expand(2, 3, 90, 128).contiguous(), kv_len=full.expand(2, 3).contiguous(), causal=False)
    assert (o["lse"] - want["lse"]).abs().max() <= 1e-5 and (o["O"].float() - want["O"].float()).abs().max() <= 2.0 ** -8 * want["O"].float().abs().max()


EVICT = [
    # dtype, d, heads, rows, lengths, budget, recent, sink, room, ties
    (BF, 128, 5, 300, (200, 300), 64, 10, 4, 80, False),
    (BF, 64, 3, 1500, (1200, 1500), 300, 0, 0, 300, True),
    (F32, 64, 2, 512, (512, 512), 64, 16, 4, 68, False),
    (F32, 128, 4, 90, (0, 90), 30, 30, 4, 40, False),
    (BF, 128, 3, 9000, (8000, 9000), 1229, 154, 4, 1240, False),
    (BF, 128, 2, 40, (1, 40), 60, 8, 4, 40, False),
    (BF, 128, 2, 400, (300, 400), 1, 0, 0, 2, True),
    (BF, 64, 2, 400, (300, 400), 0, 0, 3, 3, False),
    (BF, 64, 2, 33000, (32900, 33000), 5000, 11, 1, 5001, True),
    (BF, 64, 3, 32768, (1, 32768), 3277, 100, 4, 3300, False),
    (BF, 64, 3, 20000, (15000, 20000), 7000, 100, 4, 7004, True),
    (BF, 64, 2, 1024, (1000, 1024), 512, 0, 0, 512, True),
    (F32, 64, 2, 1025, (1025, 1025), 1000, 999, 24, 1024, False),
]


@pytest.mark.parametrize("case", EVICT, ids=[f"{i}-{'bf16' if c[0] == BF else 'f32'}-R{c[3]}-B{c[5]}" for i, c in enumerate(EVICT)])
def test_evict(case):
    B = _b()
    dtype, d, heads, rows, (lo, hi), budget, recent, sink, room, ties = case
    _, K, V = _make(31, dtype, d, 1, heads, 1, 1, rows)
    K, V = K[0], V[0]
    gen = torch.Generator().manual_seed(77)
    mass = torch.exp(2.5 * torch.randn((heads, rows), generator=gen))
    if ties:
        mass = (mass * 2).floor()                              # many equal, many 0
    pos = torch.arange(rows, dtype=torch.int32).expand(heads, rows) * 3 + 1
    kv_len = _lens(6, 1, heads, lo, hi)[0]
    for s in range(heads):
        mass[s, int(kv_len[s]):] = math.inf                    # behind the head: never kept
    out = {"K_out": torch.full((heads, room, d), 7.0, dtype=dtype, device="cuda"), "V_out": torch.full((heads, room, d), 7.0, dtype=dtype, device="cuda"),
           "mass_out": torch.full((heads, room), 7.0, device="cuda"), "pos_out": torch.full((heads, room), 7, dtype=torch.int32, device="cuda")}
    o = B.evict(K.cuda(), V.cuda(), mass.cuda(), budget, kv_len=kv_len.cuda(), recent=recent, sink=sink, pos=pos.contiguous().cuda(), out=out)
    o = {k: v.cpu() for k, v in o.items()}
    for h in range(heads):
        keep = R.evict(mass[h], int(kv_len[h]), budget, recent, sink)
        n = len(keep)
        assert int(o["len_out"][h]) == n
        assert o["idx"][h].tolist() == keep + [-1] * (room - n)
        assert torch.equal(o["K_out"][h, :n], K[h, keep]) and torch.equal(o["V_out"][h, :n], V[h, keep])
        assert torch.equal(o["mass_out"][h, :n], mass[h, keep]) and torch.equal(o["pos_out"][h, :n], pos[h, keep])
        for k in ("K_out", "V_out", "mass_out", "pos_out"):
            assert (o[k][h, n:] == 7).all(), f"{k}: rows behind the head's end"


def test_evict_flags_bad_lengths_and_heads_without_room():
    B = _b()
    _, K, V = _make(1, BF, 128, 1, 5, 1, 1, 50)
    mass = torch.rand((5, 50), generator=torch.Generator().manual_seed(2))
    kv_len = torch.tensor([-1, 51, 50, 50, 0], dtype=torch.int32)
    sink_len = torch.tensor([0, 0, 9, 3, 7], dtype=torch.int32)
    o = B.evict(K[0].cuda(), V[0].cuda(), mass.cuda(), 10, kv_len=kv_len.cuda(), recent=2, sink_len=sink_len.cuda(), out_stride=15)
    assert o["len_out"].tolist() == [-1, -1, -1, 13, 0]
    assert (o["idx"][[0, 1, 2, 4]] == -1).all() and o["idx"][3].tolist() == R.evict(mass[3], 50, 10, 2, 3) + [-1, -1]


def test_evict_takes_the_largest_budgets():
    """budget, recent and sink of 2^31 - 1: their sums pass 32 bits, and every row is kept."""
    B = _b()
    _, K, V = _make(3, BF, 64, 1, 4, 1, 1, 700)
    mass = torch.rand((4, 700), generator=torch.Generator().manual_seed(4))
    kv_len = torch.tensor([700, 0, 1, 333], dtype=torch.int32)
    most = 2**31 - 1
    for budget, recent, sink in ((most, 0, 9), (most, most, 0), (most, 5, most), (0, 0, most)):
        o = B.evict(K[0].cuda(), V[0].cuda(), mass.cuda(), budget, kv_len=kv_len.cuda(), recent=recent, sink=sink, out_stride=700)
        assert o["len_out"].tolist() == kv_len.tolist(), (budget, recent, sink)
        for h, n in enumerate(kv_len.tolist()):
            assert o["idx"][h].tolist() == list(range(n)) + [-1] * (700 - n)
            assert torch.equal(o["K_out"][h, :n].cpu(), K[0, h, :n]) and torch.equal(o["V_out"][h, :n].cpu(), V[0, h, :n])
            assert torch.equal(o["mass_out"][h, :n].cpu(), mass[h, :n])


def test_repeated_calls_and_a_used_workspace_change_no_bit():
    B = _b()
    Q, K, V = (x.cuda() for x in _make(15, BF, 128, 2, 2, 4, 1, 2000))
    kv_len = _lens(1, 2, 2, 1500, 2000).cuda()
    o = B.attend(Q, K, V, kv_len=kv_len, mass=torch.zeros(2, 2, 2000, device="cuda"))
    first = o["O"].clone(), o["lse"].clone()
    o["ws"].view(torch.uint8).fill_(255)
    again = B.attend(Q, K, V, kv_len=kv_len, out=o)
    assert torch.equal(again["O"], first[0]) and torch.equal(again["lse"], first[1])


@pytest.mark.parametrize("T", [1, 100])
def test_captured_calls_replay(T):
    """Two graphs with a workspace each, replayed in turn with eager work between, on inputs that change."""
    B = _b()
    S, H, g, rows, d = 2, 2, 4, 600, 128
    Q, K, V = (x.cuda() for x in _make(16, BF, d, S, H, g, T, rows))
    _, PK, PV = (x.cuda()[0] for x in _make(17, BF, d, 1, H, g, 1, 300))
    kv_len = _lens(2, S, H, 300, 600).cuda()
    mass = torch.zeros((S, H, rows), device="cuda")

    def plain(out):
        mass.zero_()
        return B.attend(Q, K, V, kv_len=kv_len, window=200, sink=4, mass=mass, out=out)

    def shared(out):
        return B.attend_shared(Q, PK, PV, K, V, kv_len=kv_len, out=out)

    def cut(out):
        return B.evict(K, V, mass, 100, kv_len=kv_len, recent=10, sink=4, out=out)

    outs = [plain(None), shared(None), cut(None)]
    torch.cuda.synchronize()
    graphs = []
    for f, out in zip((plain, shared, cut), outs):
        gph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gph):
            f(out)
        graphs.append(gph)
    for step in range(4):
        Q.copy_(torch.randn(Q.shape, generator=torch.Generator().manual_seed(step)).to(BF))
        kv_len.copy_(_lens(step, S, H, 300, 600))
        torch.cuda.synchronize()
        for gph in graphs:
            gph.replay()
        torch.cuda.synchronize()
        got = [{k: v.clone() for k, v in o.items() if k != "ws"} for o in outs]
        got[0]["mass"] = mass.clone()
        fresh = [plain(None), shared(None), cut(None)]
        for a, b in zip(got, fresh):
            for k, v in a.items():
                want = mass if k == "mass" else b[k]
                if k in ("K_out", "V_out", "mass_out"):
                    continue
                assert torch.equal(v, want), f"replay {step}: {k}"
        for s in range(S):
            for h in range(H):
                n = int(got[2]["len_out"][s, h])
                assert torch.equal(got[2]["K_out"][s, h, :n], K[s, h, got[2]["idx"][s, h, :n].long()])


def test_queries_shared_by_samples_or_heads():
    """Broadcast queries (strides of 0) and one KV head per query head."""
    B = _b()
    Q, K, V = _make(23, BF, 64, 3, 2, 3, 5, 90)
    kv_len = _lens(7, 3, 2, 5, 90)
    for q in (Q[:1].expand(3, 6, 5, 64), Q[:, :1].expand(3, 6, 5, 64), Q[:, :, :1].expand(3, 6, 5, 64)):
        O, lse, _, tO, tl, _ = R.attend(q, K, V, kv_len)
        qd = q[[0]].cuda().expand(3, 6, 5, 64) if q.stride(0) == 0 else q[:, [0]].cuda().expand(3, 6, 5, 64) if q.stride(1) == 0 \
            else q[:, :, [0]].cuda().expand(3, 6, 5, 64)
        assert 0 in qd.stride()
        o = B.attend(qd, K.cuda(), V.cuda(), kv_len=kv_len.cuda())
        _check("O", o["O"], O, tO)
        _check("lse", o["lse"], lse, tl)


def test_two_calls_on_two_streams():
    B = _b()
    Q, K, V = (x.cuda() for x in _make(18, BF, 128, 4, 4, 4, 1, 3000))
    kv_len = _lens(3, 4, 4, 2000, 3000).cuda()
    want = B.attend(Q, K, V, kv_len=kv_len)
    want2 = B.attend(Q, V, K, kv_len=kv_len)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for st, (k, v) in zip(streams, ((K, V), (V, K))):
        with torch.cuda.stream(st):
            got.append([B.attend(Q, k, v, kv_len=kv_len) for _ in range(5)])
    torch.cuda.synchronize()
    for o in got[0]:
        assert torch.equal(o["O"], want["O"])
    for o in got[1]:
        assert torch.equal(o["O"], want2["O"])


def test_binding_refuses_tensors_that_do_not_match():
    B = _b()
    Q, K, V = (x.cuda() for x in _make(19, BF, 128, 2, 2, 2, 3, 40))
    n = torch.full((2, 2), 40, dtype=torch.int32, device="cuda")
    mass = torch.zeros((2, 2, 40), device="cuda")
    bad = [lambda: B.attend(Q.float(), K, V), lambda: B.attend(Q[:1], K, V), lambda: B.attend(Q[:, :3], K, V), lambda: B.attend(Q, K, V[:, :, :39]),
           lambda: B.attend(Q, K.transpose(2, 3).contiguous().transpose(2, 3), V), lambda: B.attend(Q, K, V, kv_len=n.long()),
           lambda: B.attend(Q, K, V, kv_len=n[:1]), lambda: B.attend(Q, K, V, mass=mass.double()), lambda: B.attend(Q, K, V, mass=mass[:, :, :39]),
           lambda: B.attend(Q.cpu(), K, V), lambda: B.attend(Q, K, V, kv_len=n.cpu()), lambda: B.attend(Q.half(), K.half(), V.half()),
           lambda: B.attend(Q, K, V, out={"O": torch.empty((2, 4, 3, 64), dtype=BF, device="cuda")}),
           lambda: B.attend(Q, K, V, out={"O": torch.empty((1, 4, 3, 128), dtype=BF, device="cuda").expand(2, 4, 3, 128)}),
           lambda: B.attend(Q[:1, :1, :1].expand(2, 4, 3, 128), K, V), lambda: B.attend(Q, K, V, window=1 << 31), lambda: B.attend(Q, K, V, sink=1 << 32),
           lambda: B.evict(K, V, mass, 1 << 32), lambda: B.attend(Q, K[:1].expand(2, 2, 40, 128), V[:1].expand(2, 2, 40, 128)),
           lambda: B.attend_shared(Q, K, V, K, V), lambda: B.attend_shared(Q, K[0].float(), V[0].float(), K, V),
           lambda: B.attend_shared(Q, K[0], V[0], K, V, prefix_len=n), lambda: B.attend_mass(Q, K, mass, mass),
           lambda: B.evict(K, V, mass[..., :39], 8), lambda: B.evict(K, V, mass, 8, sink_len=n), lambda: B.evict(K, V, mass, 8, pos=mass)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    for f in (lambda: B.attend(Q, K, V, out={"O": Q}), lambda: B.attend(Q[..., 1:65], K[..., :64].contiguous(), V[..., :64].contiguous()),
              lambda: B.attend(Q, K, V, window=-1), lambda: B.attend(Q, K, V, window=3, causal=False), lambda: B.attend(Q, K, V, sink=-1),
              lambda: B.evict(K, V, mass, 8, recent=9), lambda: B.evict(K, V, mass, -1), lambda: B.evict(K, V, mass, 8, sink=3, out_stride=10),
              lambda: B.evict(K, V, mass, 40, out={"K_out": K, "V_out": torch.empty_like(V)}),
              lambda: B.attend(torch.empty((1 << 8, 2), dtype=BF, device="cuda").expand(1, 1, 1 << 8, 2), torch.empty((1, 1, 5, 2), dtype=BF, device="cuda"),
                               torch.empty((1, 1, 5, 2), dtype=BF, device="cuda"))):
        with pytest.raises(B.ObfError):
            f()


def test_a_relay_its_receivers_and_their_caches_cut():
    """Compress a prompt, hand the message on, let three receivers read prompts behind it, cut their caches, generate with a window: every step against 64 bits."""
    B = _b()
    H, g, d, N, S, T, room = 2, 4, 128, 400, 3, 40, 80
    _, K, V = _make(41, BF, d, 1, H, g, 1, N)
    win = torch.randn((1, H * g, 16, d), generator=torch.Generator().manual_seed(6)).to(BF)
    c = B.compress_relay(K.cuda(), V.cuda(), win.cuda(), budgets=[48, 70], rank=2)
    msg_K, msg_V, msg_len = B.append_message(K.cuda(), V.cuda(), None, c["K_out"], c["V_out"], c["n_keep"], None, None, 90, prev_len_all=4)
    assert msg_len.tolist() == [52, 74]
    # the receivers' prompts
    Q, own_K, own_V = _make(42, BF, d, S, H, g, T, room)
    kv_len = torch.full((S, H), T, dtype=torch.int32)
    prefix = (msg_K.cpu(), msg_V.cpu(), msg_len.cpu())
    O, lse, add, tO, tl, tm = R.attend(Q, own_K, own_V, kv_len, prefix=prefix)
    o = B.attend_shared(Q.cuda(), msg_K, msg_V, own_K.cuda(), own_V.cuda(), prefix_len=msg_len, kv_len=kv_len.cuda())
    _check("O", o["O"], O, tO)
    mass = torch.zeros((S, H, room), device="cuda")
    B.attend_mass(Q.cuda(), own_K.cuda(), o["lse"], mass, kv_len=kv_len.cuda())
    _check("mass", mass, add, tm + 2 * R.U * add)
    # their caches, cut to 4 first, 5 newest and 11 heaviest rows
    e = B.evict(own_K.cuda(), own_V.cuda(), mass, 16, kv_len=kv_len.cuda(), recent=5, sink=4, out={
        "K_out": torch.zeros((S, H, 60, d), dtype=BF, device="cuda"), "V_out": torch.zeros((S, H, 60, d), dtype=BF, device="cuda")})
    m = mass.cpu()
    for s in range(S):
        for h in range(H):
            assert e["idx"][s, h, :20].tolist() == R.evict(m[s, h], T, 16, 5, 4)
    # one generated token at a time: its row goes behind each head's own end
    n = e["len_out"]
    for step in range(3):
        q, k, v = _make(50 + step, BF, d, S, H, g, 1, 1)
        at = n.long()[..., None, None].expand(S, H, 1, d)
        e["K_out"].scatter_(2, at, k.cuda())
        e["V_out"].scatter_(2, at, v.cuda())
        n = n + 1
        kw = dict(window=12, sink=4)
        O, lse, add, tO, tl, tm = R.attend(q, e["K_out"].cpu(), e["V_out"].cpu(), n.cpu(), prefix=prefix, **kw)
        o = B.attend_shared(q.cuda(), msg_K, msg_V, e["K_out"], e["V_out"], prefix_len=msg_len, kv_len=n, **kw)
        _check("O", o["O"], O, tO)
        _check("lse", o["lse"], lse, tl)


@pytest.mark.parametrize("T", [1, 60])
def test_caches_whose_offsets_pass_32_bits(T):
    """Two heads of 2^24 rows of storage: the second head, and the last rows of either, lie more than 2^32 bytes behind the start."""
    B = _b()
    H, g, d, rows = 2, 2, 128, 1 << 24
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    K, V = (torch.zeros((1, H, rows, d), dtype=BF, device="cuda") for _ in range(2))
    Q, k, v = (x.cuda() for x in _make(61, BF, d, 1, H, g, T, 700))
    n = torch.tensor([[rows, rows - 5]], dtype=torch.int32, device="cuda")
    for h in range(H):
        at = int(n[0, h])
        K[0, h, :4], V[0, h, :4] = k[0, h, :4], v[0, h, :4]
        K[0, h, at - 696:at], V[0, h, at - 696:at] = k[0, h, 4:], v[0, h, 4:]
    kw = dict(window=500, sink=4)
    o = B.attend(Q, K, V, kv_len=n, **kw)
    small = B.attend(Q, k, v, **kw)
    assert (o["lse"] - small["lse"]).abs().max() <= 1e-5 and (o["O"].float() - small["O"].float()).abs().max() <= 2.0 ** -7 * small["O"].float().abs().max()
    if T > 1:
        return
    # without a window: the other rows' logits are 0, their values too; and the rows of largest weight of such a cache
    K[0, :, 1 << 23], V[0, :, 1 << 23] = Q[0, ::g, 0] * 0.5, 1.0
    o = B.attend(Q, K, V, kv_len=n, mass=(mass := torch.zeros((1, H, rows), device="cuda")))
    for h in range(H):
        at = int(n[0, h])
        seen = torch.cat([torch.arange(4), torch.tensor([1 << 23]), torch.arange(at - 696, at)]).cuda()
        x = (Q[0, h * g:(h + 1) * g, 0].double() @ K[0, h, seen].double().t()) / math.sqrt(d)
        lse = torch.log(torch.exp(x).sum(dim=1) + (at - 701))
        w = torch.exp(x - lse[:, None])
        assert (o["lse"][0, h * g:(h + 1) * g, 0].double() - lse).abs().max() <= 2e-5
        assert (o["O"][0, h * g:(h + 1) * g, 0].double() - w @ V[0, h, seen].double()).abs().max() <= 2.0 ** -7 * (w @ V[0, h, seen].double()).abs().max()
        assert (mass[0, h, seen].double() - w.sum(dim=0)).abs().max() <= 1e-4 * w.sum(dim=0).max()
    e = B.evict(K, V, mass, 300, kv_len=n, recent=50, sink=4)
    for h in range(H):
        at = int(n[0, h])
        worth = mass[0, h, :at].clone()
        worth[:4] = worth[at - 50:] = math.inf
        keep = torch.sort(torch.sort(worth, descending=True, stable=True).indices[:304]).values
        assert torch.equal(e["idx"][0, h].long(), keep) and torch.equal(e["K_out"][0, h], K[0, h, keep])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,rows,where", [(1, 90, [50]), (1, 9000, [5000]), (1, 9000, range(0, 9000, 100)), (3, 9000, [4000]), (40, 300, [100])])
def test_one_visible_key_without_numbers_takes_every_weight_of_its_rows(dtype, T, rows, where):
    """Also where the keys are cut into ranges and only some, or all, of those hold such a key: the weights come from the row's whole normaliser."""
    B = _b()
    Q, K, V = (x.cuda() for x in _make(25, dtype, 128, 1, 2, 2, T, rows))
    want = torch.zeros((1, 2, rows), device="cuda")
    B.attend(Q, K, V, mass=want)
    K[0, 0, list(where)] = math.nan
    mass = torch.zeros((1, 2, rows), device="cuda")
    o = B.attend(Q, K, V, mass=mass)
    assert torch.isnan(o["O"][0, :2]).all() and torch.isnan(o["lse"][0, :2]).all()
    assert torch.isnan(mass[0, 0]).all() and torch.equal(mass[0, 1], want[0, 1])
    again = torch.zeros((1, 2, rows), device="cuda")
    B.attend_mass(Q, K, o["lse"], again)
    assert torch.isnan(again[0, 0]).all() and torch.isfinite(again[0, 1]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [2, 60])
def test_queries_that_do_not_count_may_hold_anything(dtype, T):
    """A query whose lse the caller set to -inf (a padded one) adds nothing, whatever it holds."""
    B = _b()
    n = T + 200
    Q, K, V = _make(26, dtype, 128, 1, 2, 2, T, n)
    kv_len = torch.full((1, 2), n)
    _, lse, add, _, _, tol = R.attend(Q, K, V, kv_len)
    o = B.attend(Q.cuda(), K.cuda(), V.cuda())
    off = [1] if T == 2 else [3, 17, 18, 59]
    for t in off:
        one = torch.full((1, 2), n - T + t + 1)
        add = add - R.attend(Q[:, :, t:t + 1], K, V, one)[2]
    Q[:, :, off] = math.nan
    o["lse"][:, :, off] = -math.inf
    mass = torch.zeros((1, 2, n), device="cuda")
    B.attend_mass(Q.cuda(), K.cuda(), o["lse"], mass)
    _check("mass", mass, add, tol + 2 * R.U * add)


@pytest.mark.parametrize("P", [63, 64, 128, 1024])
@pytest.mark.parametrize("window", [0, 90])
def test_messages_of_whole_tiles_before_a_prompt(P, window):
    """Tiles without masks of the message, then at once those of the own rows."""
    B = _b()
    S, H, g, T, rows, d = 2, 8, 2, 40, 400, 128
    Q, K, V = _make(30, BF, d, S, H, g, T, rows)
    _, PK, PV = _make(31, BF, d, 1, H, g, 1, P)
    kv_len = _lens(12, S, H, 300, rows)
    plen = torch.full((H,), P, dtype=torch.int32)
    kw = dict(window=window, sink=2)
    O, lse, _, tO, tl, _ = R.attend(Q, K, V, kv_len, prefix=(PK[0], PV[0], plen), **kw)
    o = B.attend_shared(Q.cuda(), PK[0].cuda(), PV[0].cuda(), _spoil(K, kv_len, math.nan).cuda(), _spoil(V, kv_len, math.nan).cuda(), kv_len=kv_len.cuda(), **kw)
    _check("lse", o["lse"], lse, tl)
    _check("O", o["O"], O, tO)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 9, 40])
def test_long_and_short_first_rows_per_head(dtype, T):
    """An inherited message of thousands of rows behind a small window, beside heads with few first rows; what `sink` says of them changes no result but by rounding."""
    Q, K, V = _make(32, dtype, 128, 1, 4, 2, T, 4000)
    sink_len = torch.tensor([[3500, 0, 4000, 7]], dtype=torch.int32)
    kv_len = torch.tensor([[4000, 3900, 3000, 60]], dtype=torch.int32)
    for sink in (0, 8, 3500):
        _attend_and_check(Q, K, V, kv_len, causal=True, window=64, sink=sink, sink_len=sink_len)


@pytest.mark.parametrize("S,T,d", [(8, 1, 128), (9, 1, 128), (40, 1, 64), (5, 3, 64), (3, 8, 128)])
def test_precision_of_few_queries_does_not_depend_on_the_batch(S, T, d):
    """Up to 32 query rows per sample and KV head the weights keep 16 bits, however many samples share the message."""
    B = _b()
    Q, K, V = _make(27, BF, d, S, 1, 4, T, 40)
    _, PK, PV = _make(28, BF, d, 1, 1, 4, 1, 700)
    kv_len, plen = _lens(3, S, 1, T, 40), torch.tensor([700], dtype=torch.int32)
    O, lse, _, tO, tl, _ = R.attend(Q, K, V, kv_len, prefix=(PK[0], PV[0], plen), p_eps=2.0 ** -16)
    o = B.attend_shared(Q.cuda(), PK[0].cuda(), PV[0].cuda(), K.cuda(), V.cuda(), prefix_len=plen.cuda(), kv_len=kv_len.cuda())
    _check("lse", o["lse"], lse, tl)
    _check("O", o["O"], O, tO)


def test_an_expanded_workspace_is_replaced():
    B = _b()
    Q, K, V = (x.cuda() for x in _make(33, BF, 128, 1, 2, 2, 1, 3000))
    want = B.attend(Q, K, V)
    byte = torch.zeros(1, dtype=torch.uint8, device="cuda")
    o = B.attend(Q, K, V, out={"ws": byte.expand(want["ws"].nbytes)})
    assert torch.equal(o["O"], want["O"]) and o["ws"].is_contiguous() and byte.item() == 0
    mass = [torch.zeros((1, 2, 3000), device="cuda") for _ in range(2)]
    B.attend_mass(Q, K, want["lse"], mass[0])
    B.attend_mass(Q, K, want["lse"], mass[1], ws=byte.expand(1 << 24))
    assert torch.equal(mass[0], mass[1]) and byte.item() == 0


@pytest.mark.parametrize("T", [1, 100])
def test_a_used_workspace_changes_no_weight(T):
    B = _b()
    Q, K, V = (x.cuda() for x in _make(15, BF, 128, 2, 2, 4, T, 2000))
    kv_len = _lens(1, 2, 2, 1500, 2000).cuda()
    mass = [torch.zeros(2, 2, 2000, device="cuda") for _ in range(3)]
    o = B.attend(Q, K, V, kv_len=kv_len, mass=mass[0])
    first = o["O"].clone(), o["lse"].clone()
    o["ws"].fill_(255)
    again = B.attend(Q, K, V, kv_len=kv_len, mass=mass[1], out=o)
    assert torch.equal(again["O"], first[0]) and torch.equal(again["lse"], first[1]) and torch.equal(mass[0], mass[1])


@pytest.mark.parametrize("d,S,H,g,T,window", [(128, 1, 8, 2, 70, 0), (64, 2, 8, 2, 40, 33), (128, 2, 8, 3, 20, 0), (64, 3, 8, 1, 140, 0), (128, 1, 6, 2, 40, 0)])
def test_heads_in_multiples_of_eight(d, S, H, g, T, window):
    """Samples times KV heads in one, two and three rounds of eight, and in rounds of two: the order in which the sets of keys go round the dies."""
    Q, K, V = _make(29, BF, d, S, H, g, T, 300)
    _attend_and_check(Q, K, V, _lens(11, S, H, T, 300), window=window, sink=3)


@pytest.mark.parametrize("sink", [0, 9, 2500])
def test_evictions_behind_long_and_short_first_rows(sink):
    """An inherited message of thousands of rows beside a small budget; what `sink` says of its length changes nothing."""
    B = _b()
    _, K, V = _make(34, BF, 64, 1, 5, 1, 1, 3000)
    mass = torch.rand((5, 3000), generator=torch.Generator().manual_seed(8))
    kv_len = torch.tensor([3000, 2900, 2600, 100, 0], dtype=torch.int32)
    sink_len = torch.tensor([2500, 0, 2599, 2000, 7], dtype=torch.int32)
    o = B.evict(K[0].cuda(), V[0].cuda(), mass.cuda(), 40, kv_len=kv_len.cuda(), recent=8, sink=sink, sink_len=sink_len.cuda(), out_stride=2700)
    for h in range(5):
        keep = R.evict(mass[h], int(kv_len[h]), 40, 8, int(sink_len[h]))
        n = len(keep)
        assert int(o["len_out"][h]) == n and o["idx"][h].tolist() == keep + [-1] * (2700 - n)
        assert torch.equal(o["K_out"][h, :n].cpu(), K[0, h, keep]) and torch.equal(o["V_out"][h, :n].cpu(), V[0, h, keep])
        assert torch.equal(o["mass_out"][h, :n].cpu(), mass[h, keep])
