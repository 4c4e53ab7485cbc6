"""Host side of the operators on a relayed cache, without a GPU: workspace sizes and refusals before anything is enqueued; the 64-bit definitions on cases with a known answer."""
import ctypes as C
import math
import os

import pytest
import torch

from paper_2604_13349_amd import binding as B
from tests import attend_ref as R


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.lib_path()):
        from paper_2604_13349_amd import build
        build.build(verbose=False)
    return B.load_library()


def _call(**kw):
    c = B._Attend(2, 2, 4, 128, 1, 100, B.OBF_BF16, 1, 0, 0, 100, 0, 0)
    for k, v in kw.items():
        setattr(c, k, (C.c_int64 * 3)(*v) if k.endswith("_stride") and isinstance(v, tuple) else v)
    return c


FAKE, FAKE_O = C.c_void_p(1 << 20), C.c_void_p(1 << 40)      # never dereferenced: every call below fails on the host


def _attend(lib, c, Q=FAKE, K=FAKE, V=FAKE, O=FAKE_O, ws=FAKE, ws_bytes=1 << 40):
    rc = lib.obf_attend(C.byref(c) if c is not None else None, Q, K, V, None, None, O, None, None, ws, ws_bytes, None)
    return rc, lib.obf_last_error().decode()


REFUSED = [
    (dict(n_samples=0), 1, "n_samples"), (dict(n_kv_heads=0), 1, "n_kv_heads"), (dict(group=0), 1, "group"), (dict(n_queries=0), 1, "n_queries"),
    (dict(token_stride=0), 1, "token_stride"), (dict(dtype=2), 1, "dtype"), (dict(window=-1), 1, "window"), (dict(sink=-1), 1, "sink"),
    (dict(window=5, causal=0), 1, "causal"), (dict(kv_len_all=101), 1, "kv_len_all"), (dict(kv_len_all=-1), 1, "kv_len_all"),
    (dict(len_stride=1), 1, "len_stride"), (dict(len_stride=-1), 1, "len_stride"), (dict(sample_stride=199), 1, "sample_stride"),
    (dict(q_stride=(1024, 128, 4)), 1, "16 bytes"), (dict(o_stride=(1024, -8, 128)), 1, "16 bytes"),
    (dict(head_dim=96), 2, "head_dim"), (dict(token_stride=(1 << 24) + 1), 2, "token_stride"), (dict(n_queries=(1 << 20) + 1), 2, "n_queries"),
    (dict(group=129), 2, "group"), (dict(n_samples=32768), 2, "65535"), (dict(n_samples=4096, n_queries=1 << 13), 2, "2^26"),
    (dict(n_samples=16384, token_stride=1 << 16), 2, "2^30"),
]


@pytest.mark.parametrize("change,status,word", REFUSED, ids=[w for _, _, w in REFUSED])
def test_refused_descriptors(lib, change, status, word):
    c = _call(**change)
    rc, msg = _attend(lib, c)
    assert rc == status and word in msg
    assert lib.obf_attend_workspace_bytes(C.byref(c), 0, 1) == 0
    assert lib.obf_attend_shared(C.byref(c), FAKE, FAKE, FAKE, None, 10, 10, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 40, None) == status
    assert lib.obf_attend_mass(C.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, FAKE, 1 << 40, None) == status


def test_refused_pointers_and_workspaces(lib):
    c = _call()
    assert _attend(lib, None)[0] == 1
    for name in ("Q", "K", "V", "O"):
        rc, msg = _attend(lib, c, **{name: None})
        assert rc == 1 and name in msg
        rc, msg = _attend(lib, c, **{name: C.c_void_p((1 << 20) + 8)})
        assert rc == 1 and "aligned" in msg
    assert _attend(lib, c, O=FAKE)[0] == 1
    assert _attend(lib, c, ws=None)[0] == 1
    assert _attend(lib, c, ws=C.c_void_p((1 << 20) + 16))[0] == 1
    less, need = (lib.obf_attend_workspace_bytes(C.byref(c), 0, m) for m in (0, 1))
    assert 0 < less < need and _attend(lib, c, ws_bytes=less - 1)[0] == 3
    assert lib.obf_attend(C.byref(c), FAKE, FAKE, FAKE, None, None, FAKE_O, None, FAKE, FAKE, need - 1, None) == 3
    assert lib.obf_attend_workspace_bytes(C.byref(c), 4000, 0) > less
    assert lib.obf_attend_workspace_bytes(C.byref(c), -1, 0) == 0

    def shared(pk=FAKE, pv=FAKE, n=10, stride=10):
        return lib.obf_attend_shared(C.byref(c), FAKE, pk, pv, None, n, stride, FAKE, FAKE, None, None, FAKE_O, None, FAKE, less, None)

    assert shared(pk=None) == 1 and shared(pv=None) == 1 and shared(n=11) == 1 and shared(n=-1) == 1 and shared(stride=0, n=0) == 1
    assert shared(n=1, stride=(1 << 24) + 1) == 2
    assert shared(n=4000, stride=4000) == 3
    assert lib.obf_attend_mass(C.byref(c), FAKE, FAKE, None, None, None, FAKE, FAKE, need, None) == 1
    assert lib.obf_attend_mass(C.byref(c), FAKE, FAKE, FAKE, None, None, None, FAKE, need, None) == 1
    assert lib.obf_attend_mass(C.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, None, need, None) == 1
    assert lib.obf_attend_mass(C.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, FAKE, need - 1, None) == 3


def test_refused_evictions(lib):
    p = [C.c_void_p((i + 1) << 30) for i in range(12)]

    def evict(heads=4, d=128, dtype=1, K=p[0], V=p[1], mass=p[2], pos=p[3], n=50, rows=50, budget=10, recent=4, sink=2, K_out=p[4], V_out=p[5], mass_out=p[6],
              pos_out=p[7], idx=p[8], len_out=p[9], room=12):
        return lib.obf_evict(heads, d, dtype, K, V, mass, pos, None, n, rows, budget, recent, None, sink, K_out, V_out, mass_out, pos_out, idx, len_out, room, None)

    one = [dict(heads=0), dict(heads=65536), dict(dtype=2), dict(rows=0, n=0), dict(room=0), dict(n=51), dict(n=-1), dict(budget=-1), dict(recent=-1), dict(sink=-1),
           dict(recent=11), dict(room=11), dict(pos=None), dict(pos_out=None), dict(K_out=p[0]), dict(V_out=C.c_void_p((2 << 30) + 256 * 49)), dict(K_out=p[1]),
           dict(V_out=p[4]), dict(mass_out=p[2]), dict(pos_out=p[3]), dict(K=C.c_void_p((1 << 30) + 4))]
    one += [{k: None} for k in ("K", "V", "mass", "K_out", "V_out", "mass_out", "idx", "len_out")]
    for kw in one:
        assert evict(**kw) == 1, kw
    assert evict(d=96) == 2 and evict(rows=(1 << 24) + 1) == 2 and evict(room=(1 << 24) + 1) == 2


def test_tensors_must_be_on_a_gpu():
    x = torch.zeros((1, 1, 1, 64))
    with pytest.raises(ValueError):
        B.attend(x, x, x)
    with pytest.raises(ValueError):
        B.evict(x, x, torch.zeros((1, 1, 1)), 1)


def test_definition_on_known_answers():
    """Equal logits: the mean of the visible values; one visible row: that row; a message in front: one softmax over both."""
    d, n, T = 64, 9, 4
    K, Q = torch.zeros((1, 1, n, d)), torch.randn((1, 2, T, d), generator=torch.Generator().manual_seed(0))
    V = torch.arange(n, dtype=torch.float32)[None, None, :, None].expand(1, 1, n, d).contiguous()
    lens = torch.tensor([[n]])
    O, lse, mass, *_ = R.attend(Q, K, V, lens)
    for t in range(T):
        assert torch.allclose(O[0, :, t], torch.full((2, d), (n - T + t) / 2, dtype=torch.float64)) and lse[0, 0, t] == pytest.approx(math.log(n - T + t + 1))
    assert mass.sum().item() == pytest.approx(2 * T)
    O, *_ = R.attend(Q, K, V, lens, window=1)
    assert torch.allclose(O[0, 0, :, 0], torch.arange(n - T, n, dtype=torch.float64))
    O, *_ = R.attend(Q, K, V, lens, window=2, sink=1)
    assert O[0, 0, T - 1, 0] == pytest.approx((0 + 7 + 8) / 3)
    O, lse, *_ = R.attend(Q, K, V, torch.tensor([[2]]))
    assert (O[0, :, :2] == 0).all() and lse[0, 0, 1] == -math.inf and O[0, 0, 3, 0] == pytest.approx(0.5)
    O, *_ = R.attend(Q, K, V, torch.tensor([[1]]), prefix=(K[0], V[0] + 10, torch.tensor([3])))
    assert O[0, 0, T - 1, 0] == pytest.approx((10 + 11 + 12 + 0) / 4) and O[0, 0, 0, 0] == pytest.approx(11)
    assert R.evict([5., 1., 9., 9., 2., 9., 0.], 7, 4, 1, 1) == [0, 2, 3, 5, 6]
    assert R.evict([5., 1., 9.], 3, 4, 1, 1) == [0, 1, 2]


def test_first_rows_per_head_of_unknown_number_get_ranges(lib):
    """A window beside sink_len: unless `sink` says that they are few, the launch and its workspace are planned for heads that see all their rows."""
    sizes = {}
    for sink in (0, 30, 8000):
        c = _call(n_samples=1, n_kv_heads=8, token_stride=8200, kv_len_all=8200, window=64, sink=sink)
        sizes[sink] = lib.obf_attend_workspace_bytes(C.byref(c), 0, 0)
    assert sizes[30] < sizes[0] and sizes[8000] <= sizes[0]
    c = _call(n_samples=1, n_kv_heads=8, token_stride=8200, kv_len_all=8200, window=64)
    assert lib.obf_attend(C.byref(c), FAKE, FAKE, FAKE, None, FAKE, FAKE_O, None, None, FAKE, sizes[0] - 1, None) == 3
    whole = _call(n_samples=1, n_kv_heads=8, token_stride=8200, kv_len_all=8200)
    assert sizes[0] == lib.obf_attend_workspace_bytes(C.byref(whole), 0, 0)


def test_outputs_that_meet_inputs_are_refused(lib):
    """Every output, and the workspace, against every input and one another: the same start, the other's last byte, an output around an input."""
    S, H, g, T, rows, d, P = 2, 2, 4, 3, 100, 128, 10
    c = _call(n_queries=T)
    size = {"Q": S * H * g * T * d * 2, "K": S * H * rows * d * 2, "V": S * H * rows * d * 2, "O": S * H * g * T * d * 2, "kv_len": S * H * 4, "sink_len": S * H * 4,
            "lse": S * H * g * T * 4, "mass": S * H * rows * 4, "prefix_K": H * P * d * 2, "prefix_V": H * P * d * 2, "prefix_len": H * 4}
    names = {"attend": ("Q", "K", "V", "kv_len", "sink_len", "O", "lse", "mass"), "mass": ("Q", "K", "lse", "kv_len", "sink_len", "mass"),
             "shared": ("Q", "prefix_K", "prefix_V", "prefix_len", "K", "V", "kv_len", "sink_len", "O", "lse")}
    outs = {"attend": ("O", "lse", "mass", "ws"), "mass": ("mass", "ws"), "shared": ("O", "lse", "ws")}

    def call(kind, at):
        p = {k: C.c_void_p(v) for k, v in at.items()}
        a = [p[k] for k in names[kind]]
        if kind == "attend":
            return lib.obf_attend(C.byref(c), *a, p["ws"], size["ws"], None)
        if kind == "mass":
            return lib.obf_attend_mass(C.byref(c), *a, p["ws"], size["ws"], None)
        return lib.obf_attend_shared(C.byref(c), *a[:4], P, P, *a[4:], p["ws"], size["ws"], None)

    for kind in names:
        size["ws"] = lib.obf_attend_workspace_bytes(C.byref(c), P if kind == "shared" else 0, int(kind != "shared"))
        apart = {k: (i + 1) << 30 for i, k in enumerate(names[kind] + ("ws",))}
        for o in outs[kind]:
            for other in apart:
                if other == o:
                    continue
                for at in (apart[other], apart[other] + (size[other] - 1) // 256 * 256, apart[other] - size[o] // 512 * 256):
                    if apart[other] - size[o] < at:
                        assert call(kind, {**apart, o: at}) == 1, (kind, o, other)
                        assert o.replace("ws", "workspace") in lib.obf_last_error().decode()


def test_evictions_whose_outputs_meet_inputs_are_refused(lib):
    heads, d, rows, room = 4, 128, 50, 12
    ins = {"K": heads * rows * d * 2, "V": heads * rows * d * 2, "mass": heads * rows * 4, "pos": heads * rows * 4, "kv_len": heads * 4, "sink_len": heads * 4}
    outs = {"K_out": heads * room * d * 2, "V_out": heads * room * d * 2, "mass_out": heads * room * 4, "pos_out": heads * room * 4, "idx": heads * room * 4, "len_out": heads * 4}
    size = {**ins, **outs}
    apart = {k: (i + 1) << 30 for i, k in enumerate(size)}

    def evict(**moved):
        p = {k: C.c_void_p(v) for k, v in {**apart, **moved}.items()}
        return lib.obf_evict(heads, d, 1, p["K"], p["V"], p["mass"], p["pos"], p["kv_len"], rows, rows, 10, 4, p["sink_len"], 0, p["K_out"], p["V_out"], p["mass_out"],
                             p["pos_out"], p["idx"], p["len_out"], room, None)

    for o in outs:
        for other in size:
            if other == o:
                continue
            for at in (apart[other], apart[other] + (size[other] - 1) // 16 * 16, apart[other] - (size[o] - 1) // 16 * 16):
                assert evict(**{o: at}) == 1, (o, other)
                assert o in lib.obf_last_error().decode() and other in lib.obf_last_error().decode()


def test_rows_of_outputs_that_overlap_are_refused(lib):
    """Samples, query heads and queries (2, 8, 5) at strides that put two rows in one place; and other orders, with gaps, that do not."""
    for o in ((1024, 128, 64), (128, 128, 128), (0, 640, 128), (5112, 640, 128), (5120, 632, 128), (640, 1272, 128)):
        c = _call(n_queries=5, o_stride=o)
        rc, msg = _attend(lib, c)
        assert rc == 1 and "overlap" in msg, o
        assert lib.obf_attend_workspace_bytes(C.byref(c), 0, 0) == 0
    for o in ((0, 0, 0), (5120, 640, 128), (5120, 128, 1024), (1024, 128, 2048), (640, 1280, 128), (8192, 648, 128)):
        c = _call(n_queries=5, o_stride=o)
        assert lib.obf_attend_workspace_bytes(C.byref(c), 0, 0) > 0, o
    one = _call(n_samples=1, n_kv_heads=1, group=1, n_queries=5, o_stride=(0, 0, 128))
    assert lib.obf_attend_workspace_bytes(C.byref(one), 0, 0) > 0


def test_a_workspace_that_is_not_as_large_as_it_looks_is_not_used():
    cpu = torch.device("cpu")
    for ws in (None, torch.zeros(1, dtype=torch.uint8).expand(4096), torch.zeros(8192, dtype=torch.uint8)[::2], torch.zeros(4095, dtype=torch.uint8)):
        got = B._workspace(ws, 4096, cpu)
        assert got is not ws and got.is_contiguous() and got.nbytes == 4096
    for ws in (torch.zeros(4096, dtype=torch.uint8), torch.zeros(1024), torch.zeros((2, 3000), dtype=torch.uint8)):
        assert B._workspace(ws, 4096, cpu) is ws


def test_tensors_that_require_a_gradient_are_refused():
    x, m = torch.zeros((1, 1, 1, 64)), torch.zeros((1, 1, 1))
    g, gm = x.clone().requires_grad_(), m.clone().requires_grad_()
    calls = [lambda: B.attend(g, x, x), lambda: B.attend(x, g, x), lambda: B.attend(x, x, g), lambda: B.attend(x, x, x, mass=gm), lambda: B.attend_shared(g, x[0], x[0], x, x),
             lambda: B.attend_shared(x, g[0], x[0], x, x), lambda: B.attend_shared(x, x[0], g[0], x, x), lambda: B.attend_mass(g, x, m, m), lambda: B.attend_mass(x, g, m, m),
             lambda: B.attend_mass(x, x, gm, m), lambda: B.attend_mass(x, x, m, gm), lambda: B.evict(g, x, m, 1), lambda: B.evict(x, g, m, 1), lambda: B.evict(x, x, gm, 1)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="gradient"):
            call()
            pytest.fail(f"call {i} was taken")
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):       # (as without: the tensors of this test are not on one)
            call()
