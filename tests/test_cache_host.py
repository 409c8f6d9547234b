"""Host-side checks of include/vico_cache.h: exports, plans and refusals, all before any HIP call; and pins of
the oracles that its GPU tests compare with.  None of these tests touches a GPU."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2606_19849_amd as vico
import paper_2606_19849_amd._binding as binding
from oracle import kv4, rope

lib = vico.load_library()
A, B = 0x100000000, 0x4000000000     # fake, aligned device addresses: validation never dereferences them
HEADER = os.path.join(os.path.dirname(binding.HEADER), "vico_cache.h")


def test_header_functions_are_exported_and_bound():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(vico_\w+)\s*\(", src))
    assert names == {"vico_qk_norm_rope", "vico_kv_append_q4", "vico_kv_load_q4", "vico_gather_attn_q4",
                     "vico_gather_plan_q4"}
    for n in names:
        assert hasattr(lib, n) and n in binding._SIGNATURES and n in vico.__all__


# ---------------------------------------------------------------- refusals

def _rope(**kw):
    G = 1 << 32
    a = dict(q=A, qs=36 * 128, k=A + G, ks=36 * 128, v=A + 2 * G, vs=36 * 128, T=16, Hq=28, Hkv=4, D=128, qw=A + 3 * G,
             kw=A + 4 * G, wt=0, eps=1e-6, pos=A + 5 * G, axes=3, freq=A + 6 * G, rot=128, sec=(16, 24, 24), flags=0,
             qo=B, ko=B + G, vo=B + 2 * G)
    a.update(kw)
    sec = None if a["sec"] is None else (ctypes.c_int32 * len(a["sec"]))(*a["sec"])
    return lib.vico_qk_norm_rope(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["T"], a["Hq"], a["Hkv"], a["D"],
                                 a["qw"], a["kw"], a["wt"], a["eps"], a["pos"], a["axes"], a["freq"], a["rot"], sec,
                                 a["flags"], a["qo"], a["ko"], a["vo"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=1025), -1), (dict(D=96), -2), (dict(wt=2), -2),
    (dict(flags=4), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(axes=2), -1), (dict(axes=0), -1), (dict(rot=0), -1), (dict(rot=24), -1), (dict(rot=144), -1),
    (dict(sec=None), -1), (dict(sec=(16, 24, 23)), -1), (dict(sec=(80, -8, -8)), -1), (dict(axes=1, sec=(63,)), -1),
    (dict(flags=2), -1),                                   # 24 strided pairs of an axis do not fit 64
    (dict(flags=2, axes=1, sec=None), -1),
    (dict(qs=28 * 128 - 8), -1), (dict(ks=4 * 128 - 8), -1), (dict(vs=0), -1), (dict(qs=36 * 128 + 4), -1),
    (dict(qs=1 << 31), -1),
    (dict(v=None), -1), (dict(vo=None), -1), (dict(q=None), -1), (dict(pos=None), -1), (dict(freq=None), -1),
    (dict(ko=None), -1),
    (dict(q=A + 8), -4), (dict(kw=A + 8), -4), (dict(vo=B + 8), -4), (dict(pos=A + 2), -4), (dict(freq=A + 1), -4),
    (dict(qo=A), -1),                                      # q is strided: in place is not possible
    (dict(qo=A + 16, qs=28 * 128), -1), (dict(ko=B), -1), (dict(vo=A + (1 << 32)), -1), (dict(qo=A + (5 << 32)), -1),
    (dict(ko=A + (3 << 32)), -1),
    (dict(T=1 << 20), -1),                                 # an output of 2^31 bytes and more
])
def test_rope_rejects_bad_arguments(kw, status):
    assert _rope(**kw) == status


def test_rope_of_no_tokens_is_a_noop():
    assert _rope(T=0, q=None, k=None, v=None, vo=None, qo=None, ko=None, pos=None, freq=None) == 0
    assert _rope(T=0, flags=2, sec=(24, 20, 20)) == 0


def _append(**kw):
    G = 1 << 34
    a = dict(k=A, v=A + G, C=64, sk=B, sv=B + G, ck=B + 2 * G, cv=B + 3 * G, R=256, H=300, Hkv=4, D=128)
    a.update(kw)
    return lib.vico_kv_append_q4(a["k"], a["v"], a["C"], a["sk"], a["sv"], a["ck"], a["cv"], a["R"], a["H"], a["Hkv"],
                                 a["D"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(C=-1), -1), (dict(R=-1), -1), (dict(H=-1), -1), (dict(Hkv=0), -1), (dict(Hkv=1025), -1), (dict(D=32), -2),
    (dict(C=257), -3), (dict(C=1, R=0), -3), (dict(k=None), -1), (dict(cv=None), -1), (dict(sk=B + 4), -4),
    (dict(ck=B + 8), -4), (dict(sk=A), -1), (dict(cv=B), -1), (dict(sv=B + 256 * 4 * 64 - 16), -1),
    (dict(C=1 << 20, R=1 << 20, Hkv=8), -1), (dict(R=(1 << 30) + 1), -1),
])
def test_append_rejects_bad_arguments(kw, status):
    assert _append(**kw) == status


def test_append_of_nothing_is_a_noop():
    assert _append(C=0, k=None, v=None, sk=None) == 0


def _load(**kw):
    G = 1 << 34
    a = dict(sk=A, sv=A + G, ck=A + 2 * G, cv=A + 3 * G, R=256, ss=A + 4 * G, sl=A + 5 * G, n=3, ok=B, ov=B + G, rows=100,
             cnt=B + 2 * G, Hkv=4, D=128)
    a.update(kw)
    return lib.vico_kv_load_q4(a["sk"], a["sv"], a["ck"], a["cv"], a["R"], a["ss"], a["sl"], a["n"], a["ok"], a["ov"],
                               a["rows"], a["cnt"], a["Hkv"], a["D"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(R=-1), -1), (dict(n=-1), -1), (dict(n=2049), -1), (dict(rows=-1), -1), (dict(Hkv=0), -1), (dict(D=256), -2),
    (dict(n=2048, R=1 << 20), -1), (dict(rows=1 << 21), -1), (dict(ok=None), -1), (dict(ss=None), -1), (dict(cv=None), -1),
    (dict(ov=B + 8), -4), (dict(ss=A + 4), -4), (dict(sl=A + 2), -4), (dict(cnt=B + 2), -4), (dict(ok=A), -1),
    (dict(ov=B), -1), (dict(cnt=B), -1), (dict(cnt=A + (4 << 34)), -1),
])
def test_load_rejects_bad_arguments(kw, status):
    assert _load(**kw) == status


def test_load_of_nothing_is_a_noop():
    assert _load(rows=0, cnt=None, ok=None, ov=None) == 0


def _gather(**kw):
    G = 1 << 34
    a = dict(q=A, Lq=1, tk=A + G, tv=A + 2 * G, T=5, xk=A + 3 * G, xv=A + 4 * G, S=16, sk=A + 5 * G, sv=A + 6 * G,
             ck=A + 7 * G, cv=A + 8 * G, R=4096, ss=A + 9 * G, sl=A + 10 * G, n=3, hint=0, Hq=28, Hkv=4, D=128, scale=0.0,
             out=B, dt=0, lse=B + G, splits=0, ws=B + 2 * G, wsb=1 << 30)
    a.update(kw)
    return lib.vico_gather_attn_q4(a["q"], a["Lq"], a["tk"], a["tv"], a["T"], a["xk"], a["xv"], a["S"], a["sk"], a["sv"],
                                   a["ck"], a["cv"], a["R"], a["ss"], a["sl"], a["n"], a["hint"], a["Hq"], a["Hkv"], a["D"],
                                   a["scale"], a["out"], a["dt"], a["lse"], a["splits"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(Lq=-1), -1), (dict(Lq=6), -1), (dict(S=-1), -1), (dict(R=-1), -1), (dict(n=-1), -1), (dict(n=2049), -1),
    (dict(hint=-1), -1), (dict(splits=-1), -1), (dict(Hq=30), -1), (dict(Hkv=0), -1), (dict(D=96), -2), (dict(dt=2), -2),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(wsb=-1), -1), (dict(q=None), -1),
    (dict(tv=None), -1), (dict(out=None), -1), (dict(xk=None), -1), (dict(sl=None), -1), (dict(ck=None), -1),
    (dict(q=A + 8), -4), (dict(cv=A + 4), -4), (dict(ss=A + 4), -4), (dict(lse=B + 2), -4), (dict(ws=B + 8), -4),
    (dict(splits=4, wsb=100), -5), (dict(splits=4, ws=None), -5),
    (dict(out=A), -1), (dict(lse=B), -1), (dict(out=A + (7 << 34)), -1), (dict(lse=A + (9 << 34)), -1),
    (dict(splits=4, ws=B), -1), (dict(splits=4, ws=A + (5 << 34)), -1),
    (dict(T=(1 << 20) + 1), -1), (dict(n=2048, R=1 << 20), -1), (dict(Lq=1 << 18, T=1 << 18), -1),
])
def test_gather_rejects_bad_arguments(kw, status):
    assert _gather(**kw) == status


def test_gather_of_no_rows_is_a_noop():
    assert _gather(Lq=0, q=None, out=None) == 0


def test_plan_reports_the_workspace():
    for heads in ((28, 4, 128), (16, 2, 128), (8, 2, 64), (32, 32, 64), (64, 1, 128)):
        for q_len in (1, 2, 5, 32, 300, 2048):
            for hint in (0, 1, 500, 20000, 300000):
                parts, wb = vico.vico_gather_plan_q4(q_len, q_len + 7, 64, 1 << 18, 32, hint, *heads)
                assert 1 <= parts <= 64 and (wb > 0) == (parts > 1) and wb < 48e6
                p3, w3 = vico.vico_gather_plan_q4(q_len, q_len + 7, 64, 1 << 18, 32, hint, *heads, num_splits=3)
                assert p3 == 3 and w3 >= 3 * 4 * q_len * heads[0] * (heads[2] + 1)
    with pytest.raises(vico.VicoError):
        vico.vico_gather_plan_q4(3, 2, 0, 0, 0, 0, 8, 2, 64)


def route(q_len, tail, S, slots, n_segs, hint, heads, splits=0):
    out = (ctypes.c_int32 * 4)()
    assert lib.vico_gather_q4_route(q_len, tail, S, slots, n_segs, ctypes.c_int64(hint), *heads, splits, out) == 0
    return tuple(out)


def test_which_kernel_runs():
    """Few rows or few keys: the rows kernel; many rows over many keys, or more parts than its row tiles have room for:
    256-row tiles.  The parts of the plan are those of the route."""
    b7, small = (28, 4, 128), (8, 2, 64)
    assert route(1, 64, 64, 200000, 32, 18000, b7) == (2, 64, 256, 16)
    assert route(1, 64, 0, 0, 0, 0, b7)[:2] == (2, 1)
    assert route(32, 32, 64, 200000, 32, 18000, b7) == (2, 9, 252, 32)
    assert route(1024, 1024, 64, 8192, 2, 8192, b7) == (0, 2, 224, 256)
    assert route(2048, 2048, 16, 200, 2, 200, b7)[::3] == (0, 256)
    assert route(130, 130, 16, 300, 2, 300, b7, 16) == (0, 16, 256, 256)
    assert route(257, 300, 16, 300, 2, 300, small, 64) == (0, 64, 640, 256)
    for q_len in (1, 3, 17, 40, 200, 1000, 3000):
        for hint in (0, 100, 5000, 200000):
            parts, _ = vico.vico_gather_plan_q4(q_len, q_len, 64, 1 << 18, 32, hint, *b7)
            assert route(q_len, q_len, 64, 1 << 18, 32, hint, b7)[1] == parts


def test_host_tensors_and_wrong_shapes_are_refused():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)   # noqa: E731
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)      # noqa: E731
    store = u8(8, 2, 32), u8(8, 2, 32), u8(8, 2, 2), u8(8, 2, 2)
    seg = torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="k_chunk"):
        vico.vico_kv_append_q4(bf(4, 2, 64), bf(4, 2, 64), *store, 0)
    with pytest.raises(ValueError, match="out_k"):
        vico.vico_kv_load_q4(*store, *seg, bf(4, 2, 64), bf(4, 2, 64))
    with pytest.raises(ValueError, match="q:"):
        vico.vico_gather_attn_q4(bf(1, 4, 64), bf(1, 2, 64), bf(1, 2, 64), None, None, *store, *seg, bf(1, 4, 64))
    with pytest.raises(ValueError, match="q:"):
        vico.vico_qk_norm_rope(bf(4, 4, 64), bf(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(32),
                               bf(4, 4, 64), bf(4, 2, 64))


# ---------------------------------------------------------------- pins of the oracles

def test_kv4_scale_rule():
    assert kv4.group_exponent(7.0) == 0 and kv4.group_exponent(7.03125) == 1 and kv4.group_exponent(3.5) == -1
    assert kv4.group_exponent(0.0) == -123 and kv4.group_exponent(3.3e38) == 125
    # the bf16 pattern rule: exponent field plus carry from fractions above 1.75, less 2
    for bits in range(1, 0x7F80, 7):
        v = float(np.array(bits << 16, dtype=np.uint32).view(np.float32))
        assert kv4.group_exponent(v) + 127 == min(max(((bits + 0x1F) >> 7) - 2, 4), 252), hex(bits)


def test_kv4_codes_and_round_trip():
    ties = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6, 7.0: 7, 100.0: 7, 0.3: 1, 4.9: 6, 5.1: 7}
    for v, c in ties.items():
        assert kv4.nearest_code(v, 1.0) == c and kv4.nearest_code(-8 * v, 8.0) == c + 8
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 256, (3, 2, 32), dtype=np.uint8)
    codes[..., 0] |= 7                                     # a six in each group fixes its scale
    codes[..., 16] |= 7
    scales = rng.integers(4, 253, (3, 2, 2), dtype=np.uint8)
    c2, s2 = kv4.encode(kv4.decode(codes, scales))
    assert np.array_equal(scales, s2) and np.array_equal(kv4.decode(codes, scales), kv4.decode(c2, s2))
    x = rng.standard_normal((2, 1, 64))
    x[1, 0, 40] = np.inf
    d = kv4.decode(*kv4.encode(x))
    assert np.isnan(d[1, 0, 32:]).all() and np.isfinite(d[1, 0, :32]).all()
    step = np.repeat(2.0 ** np.array([[kv4.group_exponent(np.abs(x[0, 0, g:g + 32]).max()) for g in (0, 32)]]), 32)
    assert np.all(np.abs(d[0, 0] - x[0, 0]) <= step)       # half of the widest step


def test_rope_oracle_pins():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, 2, 64))
    f = 10000.0 ** (-np.arange(32) / 32)
    pos = np.arange(5)[None]
    for adjacent in (False, True):
        y = rope.rotate(x, pos, f, adjacent=adjacent)
        assert np.array_equal(y[0], x[0]) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        # scores depend on the distance alone
        a, b = rope.rotate(x, pos + 11, f, adjacent=adjacent), rope.rotate(x, pos, f, adjacent=adjacent)
        assert np.allclose(np.einsum("hd,hd->h", a[1], a[3]), np.einsum("hd,hd->h", b[1], b[3]))
    assert np.allclose(rope.rotate(x, pos, f)[1, 0, 3], x[1, 0, 3] * np.cos(f[3]) - x[1, 0, 35] * np.sin(f[3]))
    assert np.allclose(rope.rotate(x, pos, f, adjacent=True)[1, 0, 6], x[1, 0, 6] * np.cos(f[3]) - x[1, 0, 7] * np.sin(f[3]))
    assert rope.pair_axes(8, (2, 3, 3)).tolist() == [0, 0, 1, 1, 1, 2, 2, 2]
    assert rope.pair_axes(8, (4, 2, 2), strided=True).tolist() == [0, 1, 2, 0, 1, 2, 0, 0]
    assert rope.pair_axes(32, (12, 10, 10), strided=True)[:6].tolist() == [0, 1, 2, 0, 1, 2]
    n = rope.head_norm(x, np.ones(64), 0.0)
    assert np.allclose((n ** 2).mean(-1), 1) and np.array_equal(rope.head_norm(x, None, 0.0), x)
