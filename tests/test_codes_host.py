"""Host side of the operators of a cache held in codes, without a GPU: refusals before anything is enqueued; the 64-bit definitions on cases with a known answer."""
import ctypes as C
import math
import os
import random

import pytest
import torch

from paper_2604_13349_amd import binding as B
from tests import attend_ref
from tests import codes_ref as R


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.lib_path()):
        from paper_2604_13349_amd import build
        build.build(verbose=False)
    return B.load_library()


SIZE = {"n_samples": 2, "n_kv_heads": 3, "head_dim": 128, "bits": 4, "dtype": B.OBF_BF16, "n_rows": 5, "token_stride": 40, "kv_len_all": 40}
CODES = ("K.codes", "K.scale", "K.zero", "V.codes", "V.scale", "V.zero")
# addresses that are never dereferenced: every call below fails on the host
AT = {name: (i + 1) << 30 for i, name in enumerate(("K", "V", "kv_len", "per_head") + CODES)}


def _rows(**kw):
    c = B._CacheRows(*[SIZE[k] for k in SIZE])
    for k, v in kw.items():
        setattr(c, k, (C.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return c


def _codes(at, which):
    return B._Codes(*[at[f"{which}.{x}"] for x in ("codes", "scale", "zero")])


def _call(lib, kind, c, at=AT):
    k, v = _codes(at, "K"), _codes(at, "V")
    p = {n: C.c_void_p(a) if a else None for n, a in at.items()}
    d = C.byref(c) if c is not None else None
    if kind == "write":
        rc = lib.obf_cache_write(d, p["K"], p["V"], p["kv_len"], p["per_head"], C.byref(k), C.byref(v), None)
    else:
        rc = lib.obf_cache_read(d, C.byref(k), C.byref(v), p["kv_len"], p["per_head"], p["K"], p["V"], None)
    return rc, lib.obf_last_error().decode()


REFUSED = [
    (dict(n_samples=0), 1, "n_samples"), (dict(n_kv_heads=0), 1, "n_kv_heads"), (dict(n_rows=0), 1, "n_rows"), (dict(token_stride=0, kv_len_all=0), 1, "token_stride"),
    (dict(bits=3), 1, "bits"), (dict(dtype=2), 1, "dtype"), (dict(kv_len_all=41), 1, "kv_len_all"), (dict(kv_len_all=-1), 1, "kv_len_all"),
    (dict(len_stride=2), 1, "len_stride"), (dict(len_stride=-1), 1, "len_stride"), (dict(sample_stride=119), 1, "sample_stride"),
    (dict(k_stride=(1920, 640, 4)), 1, "16 bytes"), (dict(v_stride=(1920, -8, 128)), 1, "16 bytes"),
    (dict(head_dim=96), 2, "head_dim"), (dict(token_stride=(1 << 24) + 1), 2, "token_stride"), (dict(n_rows=(1 << 24) + 1), 2, "n_rows"),
    (dict(n_samples=21846), 2, "65535"), (dict(n_samples=1 << 14, token_stride=1 << 15, kv_len_all=0), 2, "2^30"), (dict(n_samples=1 << 14, n_rows=1 << 15), 2, "2^30"),
]


@pytest.mark.parametrize("kind", ["write", "read"])
@pytest.mark.parametrize("change,status,word", REFUSED, ids=[f"{w}{i}" for i, (_, _, w) in enumerate(REFUSED)])
def test_refused_descriptors(lib, kind, change, status, word):
    rc, msg = _call(lib, kind, _rows(**change))
    assert rc == status and word in msg


@pytest.mark.parametrize("kind", ["write", "read"])
def test_refused_pointers(lib, kind):
    assert _call(lib, kind, None)[0] == 1
    for name in ("K", "V") + CODES:
        assert _call(lib, kind, _rows(), {**AT, name: 0})[0] == 1, name
        assert _call(lib, kind, _rows(), {**AT, name: AT[name] + (8 if name in ("K", "V") or "codes" in name else 1)})[0] == 1, name
    f = lib.obf_cache_write
    k = _codes(AT, "K")
    assert f(C.byref(_rows()), AT["K"], AT["V"], None, None, None, C.byref(k), None) == 1
    assert f(C.byref(_rows()), AT["K"], AT["V"], None, None, C.byref(k), None, None) == 1


def test_outputs_that_meet_inputs_or_one_another_are_refused(lib):
    heads = 6
    size = {"K": heads * 5 * 256, "V": heads * 5 * 256, "kv_len": heads * 4, "per_head": heads * 4}
    size.update({x: heads * 40 * (64 if "codes" in x else 2) for x in CODES})
    for kind, outs in (("write", CODES), ("read", ("K", "V"))):
        if kind == "read":
            size["per_head"] = heads * 5 * 4
        for o in outs:
            for other in AT:
                if other == o:
                    continue
                for at in (AT[other], AT[other] + (size[other] - 1) // 16 * 16, AT[other] - (size[o] - 1) // 16 * 16):
                    rc, msg = _call(lib, kind, _rows(), {**AT, o: at})
                    assert rc == 1 and "overlap" in msg, (kind, o, other)


def test_rows_read_into_rows_that_overlap_are_refused(lib):
    for s in ((0, 640, 128), (1920, 632, 128), (1920, 640, 64), (128, 128, 128), (640, 1272, 128)):
        for name in ("k_stride", "v_stride"):
            rc, msg = _call(lib, "read", _rows(**{name: s}))
            assert rc == 1 and "overlap" in msg, s


def test_refused_attention(lib):
    at = {**AT, "Q": 30 << 30, "O": 31 << 30, "lse": 32 << 30, "ws": 33 << 30, "sink_len": 34 << 30}

    def call(bits=4, ws_bytes=1 << 29, c=None, K=True, **moved):
        a = {**at, **moved}
        d = c if c is not None else B._Attend(2, 3, 4, 128, 1, 40, B.OBF_BF16, 1, 0, 0, 40, 0, 0)
        k, v = _codes(a, "K"), _codes(a, "V")
        return lib.obf_attend_codes(C.byref(d), bits, a["Q"], C.byref(k) if K else None, C.byref(v), a["kv_len"], a["sink_len"], a["O"], a["lse"], a["ws"], ws_bytes, None)

    for kw in [dict(bits=2), dict(K=False), dict(Q=0), dict(O=0), dict(ws=0), dict(Q=at["Q"] + 8), dict(O=at["O"] + 8), dict(ws=at["ws"] + 16)] + \
              [{x: 0} for x in CODES] + [{x: at[x] + 1} for x in CODES]:
        assert call(**kw) == 1, kw
    for change, status in ((dict(n_samples=0), 1), (dict(window=5, causal=0), 1), (dict(head_dim=96), 2), (dict(group=129), 2), (dict(n_queries=(1 << 20) + 1), 2)):
        d = B._Attend(2, 3, 4, 128, 1, 40, B.OBF_BF16, 1, 0, 0, 40, 0, 0)
        for k, v in change.items():
            setattr(d, k, v)
        assert call(c=d) == status
        assert lib.obf_attend_codes_workspace_bytes(C.byref(d), 4) == 0
    long = B._Attend(1, 2, 4, 128, 1, 40000, B.OBF_BF16, 1, 0, 0, 40000, 0, 0)
    need = lib.obf_attend_codes_workspace_bytes(C.byref(long), 4)
    assert need > 256 and call(c=long, ws_bytes=need - 1) == 3 and lib.obf_attend_codes_workspace_bytes(C.byref(long), 5) == 0
    for o in ("O", "lse", "ws"):
        for other in at:
            if other not in (o, "V", "per_head") and not (other == "K"):
                assert call(**{o: at[other]}, ws_bytes=256) == 1, (o, other)
                assert "overlap" in lib.obf_last_error().decode()


def test_a_workspace_serves_calls_with_and_without_first_rows_per_head(lib):
    """The launch is planned by the rows that a query may see, which sink_len changes; refused for its O, a call has had its workspace looked at."""
    rng = random.Random(5)
    calls = [(1, 8, 1, 64, 50, 1638, 8, 1501, B.OBF_F32), (7, 2, 4, 128, 1, 5057, 4, 3944, B.OBF_F32), (2, 2, 5, 128, 4, 7974, 4, 7079, B.OBF_BF16),
             (1, 1, 1, 128, 66, 15457, 4, 8136, B.OBF_BF16)]
    for _ in range(3000):
        calls.append((rng.choice([1, 2, 7]), rng.choice([1, 2, 8]), rng.choice([1, 4, 5, 16]), rng.choice([64, 128]), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(5, 17)),
                      rng.choice([4, 8]), rng.choice([0, int(2 ** rng.uniform(3, 16))]), rng.choice([B.OBF_BF16, B.OBF_F32])))
    sizes = set()
    codes = B._Codes(1 << 50, 1 << 51, 1 << 52)
    for S, H, g, d, T, rows, bits, window, dtype in calls:
        c = B._Attend(S, H, g, d, T, rows, dtype, 1, window, rng.choice([0, 0, 4, 3000]), rows, 0, 0)
        need = lib.obf_attend_codes_workspace_bytes(C.byref(c), bits)
        sizes.add(need)
        for sink_len in (None, 1 << 53):
            rc = lib.obf_attend_codes(C.byref(c), bits, 1 << 40, C.byref(codes), C.byref(codes), None, sink_len, 1 << 40, None, 1 << 60, need, None)
            assert rc == 1 and "overlap" in lib.obf_last_error().decode(), (rc, S, H, g, d, T, rows, bits, window)
    assert len(sizes) > 500


def test_the_least_workspace(lib):
    """A call that would like copies of the rows takes a workspace without them, and none that is smaller; one that needs none asks for the same bytes both times."""
    codes = B._Codes(1 << 50, 1 << 51, 1 << 52)
    for S, H, g, d, T, rows, window, copies in ((1, 2, 4, 128, 1, 40000, 0, False), (1, 8, 4, 128, 4096, 13517, 0, True), (3, 8, 5, 64, 500, 2139, 0, True), (1, 2, 2, 128, 3000, 5000, 2048, True),
                                                (1, 2, 2, 128, 3000, 5000, 64, False)):
        for bits in (4, 8):
            c = B._Attend(S, H, g, d, T, rows, B.OBF_BF16, 1, window, 0, rows, 0, 0)
            need, least = lib.obf_attend_codes_workspace_bytes(C.byref(c), bits), lib.obf_attend_codes_workspace_least(C.byref(c), bits)
            assert (need - least >= 4 * S * H * rows * d) if copies else need == least
            for sink_len in (None, 1 << 53):
                for size, status, word in ((need, 1, "overlap"), (least, 1, "overlap"), (need - 1, 1, "overlap") if copies else (need, 1, "overlap")):
                    rc = lib.obf_attend_codes(C.byref(c), bits, 1 << 40, C.byref(codes), C.byref(codes), None, sink_len, 1 << 40, None, 1 << 60, size, None)
                    assert rc == status and word in lib.obf_last_error().decode()
                small = min(255, least - 1)
                assert lib.obf_attend_codes(C.byref(c), bits, 1 << 40, C.byref(codes), C.byref(codes), None, sink_len, 1 << 41, None, 1 << 60, small, None) == 3
    assert lib.obf_attend_codes_workspace_least(C.byref(c), 5) == 0


@pytest.mark.parametrize("kind", ["write", "read"])
@pytest.mark.parametrize("samples, heads, rows", [(65535, 1, 8192), (1 << 14, 2, 1 << 14), (1 << 13, 7, 9362), (32, 1, 1 << 24)])
def test_a_launch_has_fewer_than_2_32_threads(lib, kind, samples, heads, rows):
    """256 threads for 64 rows of a head at most; a call of 2^29 rows gets past the sizes (to arrays that overlap), one of more is refused for them."""
    assert samples * heads * -(-rows // 64) * 256 < 1 << 32 and samples * heads * rows <= 1 << 29 < (samples + 1) * heads * (rows + 1)
    at = {**AT, "K": AT["K.codes"]}
    rc, msg = _call(lib, kind, _rows(n_samples=samples, n_kv_heads=heads, token_stride=32, kv_len_all=0, n_rows=rows), at)
    assert rc == 1 and "overlap" in msg
    rc, msg = _call(lib, kind, _rows(n_samples=min(samples + 1, 65535 // heads), n_kv_heads=heads, token_stride=32, kv_len_all=0, n_rows=min(rows + 1, 1 << 24)), at)
    assert rc == 2 and "2^29" in msg


def test_tensors_must_be_on_a_gpu_and_need_no_gradient():
    u, f = torch.zeros((1, 1, 4, 32), dtype=torch.uint8), torch.zeros((1, 1, 4), dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU"):
        B.CodeCache(u, f, f, u, f, f, d=64, bits=4)
    x = torch.zeros((1, 1, 1, 64))
    g = x.clone().requires_grad_()
    for call in (lambda: B.attend_codes(g, None), lambda: B.cache_write(None, g, x), lambda: B.cache_write(None, x, g)):
        with pytest.raises(ValueError, match="gradient"):
            call()


def test_a_cache_keeps_its_tensors_and_its_layout():
    """Both are checked where the cache is made, and go to the GPU as they were then."""
    cache = object.__new__(B.CodeCache)
    for name in ("K_codes", "K_scale", "K_zero", "V_codes", "V_scale", "V_zero", "d", "bits", "shape", "between", "device"):
        with pytest.raises(AttributeError):
            setattr(cache, name, 8)
            pytest.fail(f"{name} was set")


def test_sizes_and_strides_past_32_bits(lib):
    """The C side takes them as int32: lengths that lie further apart are copied, an expanded tensor of more rows is refused.  By the plans, which go by metadata alone."""
    dev = torch.device("cuda", 0)
    cache, far = ((2, 3, 40), 120, 128, 4, dev), 1 << 32

    def meta(shape, stride, dtype):
        return torch.Size(shape), stride, dtype, dev

    Q, lse = meta((2, 3, 1, 128), (384, 128, 128, 1), torch.bfloat16), meta((2, 3, 1), (3, 1, 1), torch.float32)
    K = meta((2, 3, 40, 128), (15360, 5120, 128, 1), torch.bfloat16)
    for apart, stride, copy in ((3, 3, False), (7, 7, False), ((1 << 31) - 1, (1 << 31) - 1, False), (1 << 31, 0, True), (far + 3, 0, True)):
        n = meta((2, 3), (apart, 1), torch.int32)
        for c, *_, copied in (B._attend_codes_plan(cache, Q, Q, lse, n, n, True, 0, 0), B._rows_plan(cache, K, K, n, n, None),
                              B._attend_plan(Q, K, K, Q, lse, None, n, n, None, None, None, True, 0, 0)):
            assert (c.len_stride, copied) == (stride, copy)
    one = meta((2, 3, far + 5, 128), (384, 128, 0, 1), torch.bfloat16)
    with pytest.raises(ValueError, match="out of range"):
        B._rows_plan(cache, one, one, None, None, None)
    for wide in (((2, 3, far + 40), 3 * (far + 40), 128, 4, dev), ((far + 2, 3, 40), 120, 128, 4, dev)):
        k = meta(wide[0][:2] + (1, 128), (384, 128, 128, 1), torch.bfloat16)
        with pytest.raises(ValueError, match="out of range"):
            B._rows_plan(wide, k, k, None, None, None)
        with pytest.raises(ValueError, match="out of range"):
            B._attend_codes_plan(wide, k, k, meta(wide[0][:2] + (1,), (3, 1, 1), torch.float32), None, None, True, 0, 0)


def test_definition_on_known_answers():
    """The code's values by hand; over exact codes the attention is that of the values."""
    q, s, z = R.quantise(torch.tensor([[1.0, 2.0, 8.5, 16.0]]), 4)
    assert q.tolist() == [[0, 1, 8, 15]] and s.item() == 1.0 and z.item() == 1.0          # (7.5: to even)
    assert R.quantise(torch.full((1, 8), 1.5), 8)[0].eq(0).all()
    codes = torch.arange(64, dtype=torch.uint8).view(1, 1, 1, 64) % 16
    assert torch.equal(R.unpack(R.pack(codes, 4), 4), codes) and R.pack(codes, 4)[0, 0, 0, :2].tolist() == [0x10, 0x32]
    gen = torch.Generator().manual_seed(0)
    K, V = ((torch.randint(0, 16, (1, 2, 30, 64), generator=gen).to(torch.uint8), torch.rand((1, 2, 30), generator=gen).half(), torch.randn((1, 2, 30), generator=gen).half())
            for _ in range(2))
    Q = torch.randn((1, 4, 3, 64), generator=gen)
    n = torch.tensor([[30, 2]])
    O, lse, tO, tl = R.attend(Q, K, V, 4, n, window=9, sink=2)
    O2, lse2, *_ = attend_ref.attend(Q, R.values(*K), R.values(*V), n, window=9, sink=2)
    assert torch.allclose(O, O2) and torch.equal(lse == -math.inf, lse2 == -math.inf) and torch.allclose(lse[lse > -9e9], lse2[lse2 > -9e9])
    assert (lse[0, 2:, 0] == -math.inf).all() and (tO >= 0).all() and (tl >= 0).all()
