"""GPU parity of include/vico_cache.h against the fp64 oracle.

Tolerances, derived:
  * vico_qk_norm_rope: fp32 arithmetic, one rounding to bf16 (2^-8 relative).
    With E = |x0'| + |x1'| of the pair: the norm's sum of 16 FMAs and 3 sums,
    its root and quotient, the weight and the products are 26 roundings of
    2^-24; the angle's turns are a product exact to 2^-53 (up to 2^30 turns: 2^-23)
    and one fp32 rounding of a half turn (2^-24 * pi/2), sine and cosine 2 ulp: below
    2^-22 + 2^-22 + 2^-23; together below 2^-20 E.  2^-19 E is taken.
  * 4-bit codes, scales and their values in bf16: exact.
  * attention: the derived per-element bounds of tests/_bounds.py on the values
    that the store stands for; fp32 and bf16 outputs and the log-sum-exp.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import paper_2606_19849_amd as vico
from oracle import kv4, rope
from tests._bounds import U8, gather_bound
from tests._gpu import check_bf16, check_f32

pytestmark = pytest.mark.gpu
DEV = "cuda"


def f64(t):
    return t.double().cpu().numpy()


def normal(g, *shape, sigma=1.0):
    return (torch.randn(*shape, generator=g) * sigma).to(torch.bfloat16)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------- norms and rotation

def rope_case(seed, T, Hq, Hkv, D, rot=None, axes=1, adjacent=False, strided=False, norm="qk", wt=torch.bfloat16,
              packed=True, with_v=True, far=False, tweak=None, in_place=False, stream=None):
    g = gen(seed)
    rot = D if rot is None else rot
    half = rot // 2
    sec = None if axes == 1 else ((half - 2 * (half // 16 * 5), half // 16 * 5, half // 16 * 5) if strided
                                  else (half // 4, half // 4, half - half // 4 * 2))
    x = normal(g, T, Hq + 2 * Hkv, D, sigma=2.0)
    if tweak:
        tweak(x)
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(wt) if n in norm else None for n in "qk"]
    lo, hi = (-(1 << 31), (1 << 31) - 1) if far else (0, 5000)
    pos = torch.randint(lo, hi, (axes, T), generator=g, dtype=torch.int64).to(torch.int32)
    freq = (1e6 ** (-torch.arange(half, dtype=torch.float64) / half)).float()
    xd = x.to(DEV)
    parts = [p if packed else p.contiguous() for p in xd.split((Hq, Hkv, Hkv), 1)]
    pad = 128                                              # guard elements on both sides of each output
    outs, raw = [], []
    for i, p in enumerate(parts):
        if in_place:
            outs.append(p)
            continue
        r = torch.full((2 * pad + p.numel(),), 7.25, dtype=torch.bfloat16, device=DEV)
        raw.append(r)
        outs.append(r[pad:pad + p.numel()].view(p.shape))
    torch.cuda.synchronize()
    vico.vico_qk_norm_rope(parts[0], parts[1], pos.to(DEV)[0] if axes == 1 else pos.to(DEV), freq.to(DEV), outs[0], outs[1],
                           v=parts[2] if with_v else None, v_out=outs[2] if with_v else None,
                           q_weight=None if w[0] is None else w[0].to(DEV), k_weight=None if w[1] is None else w[1].to(DEV),
                           eps=1e-6, sections=sec, flags=adjacent + 2 * strided, stream=stream)
    torch.cuda.synchronize()
    for r in raw:
        assert torch.all(r[:pad] == 7.25) and torch.all(r[-pad:] == 7.25)
    if with_v:
        assert torch.equal(outs[2].view(torch.int16).cpu(), x[:, Hq + Hkv:].contiguous().view(torch.int16))
    elif not in_place:
        assert torch.all(outs[2] == 7.25)
    res = []
    for y, xs, wi in ((outs[0], x[:, :Hq], w[0]), (outs[1], x[:, Hq:Hq + Hkv], w[1])):
        n = rope.head_norm(f64(xs), None if wi is None else f64(wi), 1e-6)
        ref = rope.rotate(n, pos.numpy(), f64(freq), sec, adjacent, strided)
        E = np.abs(n)
        for i in range(half):
            p, q = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
            E[..., p] = E[..., q] = np.abs(n[..., p]) + np.abs(n[..., q])
        res.append((f64(y), ref, E))
    return res


def check_rope(res):
    for y, ref, E in res:
        fine = 2.0 ** -19 * E
        bound = fine + U8 * (np.abs(ref) + fine) + 1e-38
        assert np.all(np.isfinite(y))
        assert np.all(np.abs(y - ref) <= bound), float(np.max(np.abs(y - ref) - bound))


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 28, 4, 128), (7, 16, 2, 128), (33, 8, 2, 64), (2, 3, 5, 64), (1, 1, 1, 128),
                                        (131, 1, 1, 64), (300, 28, 4, 128)])
@pytest.mark.parametrize("kw", [dict(), dict(adjacent=True, norm="q"), dict(axes=3, norm="", packed=False),
                                dict(axes=3, strided=True, wt=torch.float32), dict(rot=32, with_v=False, norm="k"),
                                dict(rot=32, adjacent=True, far=True), dict(rot=16, far=True)],
                         ids=lambda k: "-".join(k) or "plain")
def test_rope(T, Hq, Hkv, D, kw):
    check_rope(rope_case(T * 7 + D, T, Hq, Hkv, D, **kw))


@pytest.mark.parametrize("axes,strided", [(1, False), (3, False), (3, True)])
def test_rope_far_positions_keep_their_angle(axes, strided):
    check_rope(rope_case(3, 64, 4, 2, 128, axes=axes, strided=strided, far=True))


def test_rope_in_place_and_on_another_stream():
    check_rope(rope_case(4, 50, 6, 2, 128, packed=False, in_place=True))
    s = torch.cuda.Stream()
    check_rope(rope_case(5, 50, 6, 2, 64, stream=s))


def test_rope_nan_stays_in_its_head():
    def tweak(x):
        x[2, 1, 5] = float("nan")
        x[3, 4, 7] = float("inf")
    with np.errstate(all="ignore"):
        for (y, ref, E), bad in zip(rope_case(6, 5, 4, 2, 64, tweak=tweak), ((2, 1), (3, 0))):
            assert not np.isfinite(y[bad]).all()
            y[bad], ref[bad], E[bad] = 0, 0, 0
            check_rope([(y, ref, E)])


# ---------------------------------------------------------------- the store

def empty_store(slots, Hkv, D, fill=0xA5):
    new = lambda w: torch.full((slots, Hkv, w), fill, dtype=torch.uint8, device=DEV)   # noqa: E731
    return new(D // 2), new(D // 2), new(D // 32), new(D // 32)


def filled_store(g, slots, Hkv, D, sigma=1.0):
    st = empty_store(max(slots, 1), Hkv, D)
    k, v = normal(g, slots, Hkv, D, sigma=sigma).to(DEV), normal(g, slots, Hkv, D).to(DEV)
    vico.vico_kv_append_q4(k, v, *st, 0)
    torch.cuda.synchronize()
    return st


def store_values(st):
    c = [t.cpu().numpy() for t in st]
    return kv4.decode(c[0], c[2]), kv4.decode(c[1], c[3])


@pytest.mark.parametrize("C,Hkv,D,R,H", [(1, 4, 128, 1, 0), (3, 1, 64, 7, 5), (5, 2, 128, 5, 12), (70, 2, 64, 100, 1050),
                                         (1, 3, 64, 9, 2 ** 40 + 3)])
def test_append_matches_the_definition_and_leaves_the_rest(C, Hkv, D, R, H):
    g = gen(C)
    k, v = normal(g, C, Hkv, D, sigma=3.0), normal(g, C, Hkv, D, sigma=0.02)
    st = empty_store(R, Hkv, D)
    vico.vico_kv_append_q4(k.to(DEV), v.to(DEV), *st, H)
    torch.cuda.synchronize()
    slots = (H + np.arange(C)) % R
    for x, codes, scales in ((k, st[0], st[2]), (v, st[1], st[3])):
        c, s = kv4.encode(f64(x))
        codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
        assert np.array_equal(codes[slots], c) and np.array_equal(scales[slots], s)
        rest = np.setdiff1d(np.arange(R), slots)
        assert np.all(codes[rest] == 0xA5) and np.all(scales[rest] == 0xA5)


def test_append_every_bf16_pattern():
    """All 65536 bit patterns, sorted (groups of like size), shuffled (groups of unlike ones), and each in a group
    of small values that it alone sets the scale of."""
    bits = np.arange(65536, dtype=np.uint32)
    finite = bits[(bits & 0x7F80) != 0x7F80]
    rng = np.random.default_rng(0)
    order = np.concatenate([bits, finite[np.argsort(finite & 0x7FFF, kind="stable")], rng.permutation(finite)])
    order = np.concatenate([order, np.zeros(-len(order) % 128, dtype=np.uint32)])
    x = torch.from_numpy(order.astype(np.uint16).view(np.int16)).view(torch.bfloat16).reshape(-1, 1, 128)
    alone = torch.zeros(len(finite) // 4, 1, 128, dtype=torch.bfloat16)
    alone.view(-1, 32)[:, 0] = torch.from_numpy(finite[:len(finite) // 4 * 4].astype(np.uint16).view(np.int16)).view(torch.bfloat16)
    for y in (x, alone):
        st = empty_store(y.shape[0], 1, 128)
        vico.vico_kv_append_q4(y.to(DEV), y.to(DEV), *st, 0)
        torch.cuda.synchronize()
        c, s = st[0].cpu().numpy(), st[2].cpu().numpy()
        assert torch.equal(st[0], st[1]) and torch.equal(st[2], st[3])
        xs = f64(y).reshape(-1, 32)
        with np.errstate(invalid="ignore"):
            amax = np.abs(xs).max(1)
        fine = np.isfinite(xs).all(1)
        scales = s.reshape(-1)
        assert np.all(scales[~fine] == 255) and np.all(scales[fine] <= 252) and np.all(scales[fine] >= 4)
        sc = np.ldexp(1.0, scales[fine].astype(np.int64) - 127)
        m = amax[fine]
        assert np.all((m <= 7 * sc) | (scales[fine] == 252)) and np.all((m > 3.5 * sc) | (scales[fine] == 4))
        codes = np.stack([c & 15, c >> 4], -1).reshape(-1, 32)
        assert np.all(codes[~fine] == 0)
        a = np.minimum(np.abs(xs[fine]) / sc[:, None], 6.0)
        grid = np.array(kv4.GRID)
        d = np.abs(a[..., None] - grid)
        best = d.min(-1, keepdims=True)
        want = np.where(d == best, np.arange(8) % 2 * 8 + np.arange(8), 99).argmin(-1)      # the even one of a tie
        assert np.array_equal(codes[fine] & 7, want) and np.array_equal(codes[fine] >> 3, np.signbit(xs[fine]))


@pytest.mark.parametrize("starts,lens,rows", [
    ([], [], 5), ([0], [40], 40), ([3, 3, 10], [5, 5, 0], 10), ([-4, 35, 100, 2], [8, 50, 3, -1], 20),
    (list(range(40)), [1] * 40, 33), ([7] * 300, [2] * 300, 700), ([0, 39] * 1024, [0, 1] * 1024, 1024), ([0], [40], 0)])
def test_load(starts, lens, rows):
    Hkv, D = 2, 64
    st = filled_store(gen(9), 40, Hkv, D)
    want = [np.concatenate([x[max(a, 0):max(a, 0, min(a + n, 40))] for a, n in zip(starts, lens)] or [x[:0]])
            for x in store_values(st)]
    out = [torch.full((rows, Hkv, D), 9.0, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    cnt = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    vico.vico_kv_load_q4(*st, torch.tensor(starts, dtype=torch.int64, device=DEV),
                         torch.tensor(lens, dtype=torch.int32, device=DEV), *out, out_count=cnt)
    torch.cuda.synchronize()
    n = len(want[0])
    assert int(cnt) == n
    for o, w in zip(out, want):
        o = f64(o)
        assert np.array_equal(o[:n], w[:rows]) and np.all(o[n:] == 9.0)


# ---------------------------------------------------------------- attention

class Case:
    def __init__(self, seed, Hq, Hkv, D, q_len, tail, S, slots, starts, lens, sigma=1.4, tweak=None):
        g = gen(seed)
        self.q = normal(g, q_len, Hq, D, sigma=sigma)
        self.tail = normal(g, tail, Hkv, D, sigma=sigma), normal(g, tail, Hkv, D)
        self.sink = (normal(g, S, Hkv, D, sigma=sigma), normal(g, S, Hkv, D)) if S else (None, None)
        self.store = filled_store(g, slots, Hkv, D, sigma)
        if tweak:
            tweak(self)
        self.seg = torch.tensor(starts, dtype=torch.int64), torch.tensor(lens, dtype=torch.int32)
        cut = [(max(a, 0), min(a + n, slots)) for a, n in zip(starts, lens)]
        cut = [(a, b) if b > a else (0, 0) for a, b in cut]      # what is empty or outside, as the oracle takes it
        empty = np.zeros((0, Hkv, D))
        self.sizes = (q_len, tail, S, self.store[0].shape[0], len(starts), 0, Hq, Hkv, D)
        self.args = (f64(self.q), f64(self.tail[0]), f64(self.tail[1]), f64(self.sink[0]) if S else empty,
                     f64(self.sink[1]) if S else empty, *store_values(self.store), [a for a, _ in cut], [b - a for a, b in cut])
        self.keys = sum(b - a for a, b in cut)

    def run(self, splits=0, dtype=torch.float32, hint=None, stream=None, scale=0.0):
        dev = lambda t: None if t is None else t.to(DEV)   # noqa: E731
        hint = self.keys if hint is None else hint
        self.parts, wb = vico.vico_gather_plan_q4(*self.sizes[:5], hint, *self.sizes[6:], num_splits=splits)
        ws = torch.full((wb + 256,), 0xFF, dtype=torch.uint8, device=DEV)      # NaN patterns: nothing is read unwritten
        out = torch.full((self.q.numel() + 64,), 3.0, dtype=dtype, device=DEV)
        lse = torch.full((self.sizes[6], self.sizes[0]), 3.0, device=DEV)
        o = out[:self.q.numel()].view(self.q.shape)
        args = [dev(self.q), *map(dev, self.tail), *map(dev, self.sink), *self.store, *map(dev, self.seg)]
        torch.cuda.synchronize()
        vico.vico_gather_attn_q4(*args, o, lse=lse, workspace=ws, keys_hint=hint, num_splits=splits, stream=stream,
                                 softmax_scale=scale)
        torch.cuda.synchronize()
        assert torch.all(out[self.q.numel():] == 3.0) and torch.all(ws[wb:] == 0xFF)
        return f64(o), f64(lse)

    def check(self, splits=0, dtype=torch.float32, hint=None, stream=None, scale=None):
        o, l = self.run(splits, dtype, hint, stream, scale or 0.0)
        ref, ref_lse = oracle.gather_attention(*self.args, scale=scale)
        b = gather_bound(*self.args, scale=scale, parts=max(self.parts, 2))
        if dtype == torch.float32:
            check_f32(o, ref, b, l, ref_lse)
        else:
            check_bf16(o, ref, b)


HEADS = [(28, 4, 128), (16, 2, 128), (8, 2, 64), (5, 5, 64), (24, 1, 128)]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("q_len,tail,S,starts,lens", [
    (1, 1, 0, [], []), (1, 65, 64, [0], [300]), (1, 40, 7, [5, 100, 260], [31, 33, 40]), (3, 3, 16, [200, 0], [100, 150]),
    (9, 50, 0, [11, 11, 290], [0, 65, 10]), (40, 41, 33, [0, 150], [96, 97])])
def test_attention(heads, q_len, tail, S, starts, lens):
    c = Case(q_len + tail, *heads, q_len, tail, S, 300, starts, lens)
    c.check()
    c.check(splits=3, hint=0)


@pytest.mark.parametrize("splits", [0, 1, 2, 16, 17, 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_attention_parts_and_types(splits, dtype):
    Case(1, 14, 2, 128, 2, 70, 64, 2000, [0, 1000, 500], [400, 999, 3]).check(splits, dtype)
    Case(2, 4, 2, 64, 5, 6, 0, 40, [3], [20]).check(splits, dtype)


@pytest.mark.parametrize("heads", HEADS[1:3], ids=str)
@pytest.mark.parametrize("n,length", [(64, 3), (65, 1), (300, 5), (2048, 1), (2048, 7)])
def test_attention_many_segments(heads, n, length):
    """Tables longer than a wave, segments shorter than a block, empty ones and ones outside of the store among them."""
    rng = np.random.default_rng(n)
    starts = rng.integers(-3, 600, n)
    lens = np.where(rng.random(n) < 0.3, 0, rng.integers(0, length + 1, n))
    c = Case(n, *heads, 2, 9, 5, 590, starts.tolist(), lens.tolist())
    for splits in (0, 1, 5):
        c.check(splits)


def test_attention_one_long_segment_among_empty_ones():
    c = Case(8, 8, 2, 64, 1, 3, 0, 5000, [0] * 1500 + [4, 7], [0] * 1500 + [4900, 2])
    c.check()
    c.check(splits=7)


@pytest.mark.parametrize("heads", HEADS[:3], ids=str)
@pytest.mark.parametrize("C,W", [(65, 128), (130, 300), (257, 64)])
def test_attention_of_a_chunk_over_a_ring_window(heads, C, W):
    first = 3 * W // 8
    c = Case(C, *heads, C, C, 16, W, [first, 0], [W - first, first])
    c.check()
    c.check(dtype=torch.bfloat16)
    c.check(splits=2)


@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 2, 64), (16, 1, 128)], ids=str)
@pytest.mark.parametrize("splits", [16, 64])
@pytest.mark.parametrize("q_len,tail,S,starts,lens", [
    (130, 130, 16, [112, 0], [188, 112]), (257, 300, 0, [5, 100, 260], [31, 33, 40]), (150, 151, 100, [], []),
    (140, 200, 64, list(range(0, 300, 2)), [2, 0, 3] * 50)])
def test_attention_in_256_row_tiles(heads, splits, q_len, tail, S, starts, lens):
    c = Case(q_len + S, *heads, q_len, tail, S, 300, starts, lens)
    c.check(splits)
    c.check(splits, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_large_chunk_without_parts(dtype):
    """224 tiles of 256 rows, one work-group each; a few heads against the oracle."""
    c = Case(20, 28, 4, 128, 2048, 2048, 16, 200, [75, 0], [125, 75])
    o, l = c.run(0, dtype)
    assert c.parts == 1
    heads = [0, 13, 27]
    ref, ref_lse = oracle.gather_attention(*c.args, heads=heads)
    b = gather_bound(*c.args, heads=heads, parts=2)
    if dtype == torch.float32:
        check_f32(o[:, heads], ref, b, l[heads], ref_lse)
    else:
        check_bf16(o[:, heads], ref, b)


@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 2, 64)], ids=str)
@pytest.mark.parametrize("q_len", [1, 3, 11])
def test_a_long_sink_and_tail(heads, q_len):
    """Each wave has several bf16 blocks, before and after those of the store."""
    c = Case(16, *heads, q_len, 1400, 700, 300, [5, 200], [150, 90])
    c.check(splits=1)
    c.check(splits=2)


def test_attention_scales_and_large_logits():
    c = Case(11, 8, 2, 64, 4, 30, 10, 200, [0], [200], sigma=12.0)
    c.check()
    c.check(scale=0.7)
    c.check(scale=1e-4)


def test_attention_streams_and_repeats():
    c = Case(12, 28, 4, 128, 1, 20, 64, 3000, [0, 2000], [1500, 900])
    s = torch.cuda.Stream()
    c.check(stream=s)
    a, b = c.run(dtype=torch.bfloat16), c.run(dtype=torch.bfloat16)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("heads,q_len,splits", [((1024, 1024, 64), 1, 0), ((1024, 4, 64), 1, 2), ((1024, 2, 128), 2, 5),
                                                ((200, 200, 128), 130, 1)], ids=str)
def test_attention_of_very_many_heads(heads, q_len, splits):
    Case(13, *heads, q_len, q_len + 3, 5, 90, [2, 70], [60, 11]).check(splits)


def test_the_other_calls_with_very_many_heads():
    check_rope(rope_case(8, 3, 1024, 1024, 64))
    check_rope(rope_case(9, 2, 1024, 1, 128, axes=3))
    st, x = empty_store(9, 1024, 128), normal(gen(30), 9, 1024, 128).to(DEV)
    vico.vico_kv_append_q4(x, x.flip(0).contiguous(), *st, 4)
    back = torch.empty_like(x), torch.empty_like(x)
    vico.vico_kv_load_q4(*st, torch.tensor([4, 0], device=DEV), torch.tensor([5, 4], dtype=torch.int32, device=DEV), *back)
    torch.cuda.synchronize()
    order = [4, 5, 6, 7, 8, 0, 1, 2, 3]
    assert np.array_equal(f64(back[0]), store_values(st)[0][order]) and torch.equal(back[0], back[1].flip(0))
    # a group's largest magnitude is above 3.5 scales, and no value is further off than one
    groups = lambda t: f64(t).reshape(9, 1024, 4, 32)   # noqa: E731
    assert np.all(np.abs(groups(back[0]) - groups(x)) <= np.abs(groups(x)).max(-1, keepdims=True) / 3.5)


def test_two_calls_at_once():
    """The same table and store read from two streams, each with its own workspace: rows and 256-row kernel."""
    a = Case(14, 28, 4, 128, 2, 70, 64, 20000, [0, 9000], [8000, 9000])
    b = Case(15, 28, 4, 128, 300, 310, 64, 20000, [0, 9000], [8000, 9000])
    sets = []
    for c in (a, b):
        parts, wb = vico.vico_gather_plan_q4(*c.sizes[:5], c.keys, *c.sizes[6:])
        args = [t.to(DEV) for t in (c.q, *c.tail, *c.sink)] + list(a.store) + [t.to(DEV) for t in a.seg]
        sets.append((args, torch.empty(c.q.shape, device=DEV), torch.empty(max(wb, 1), dtype=torch.uint8, device=DEV), c.keys))
    streams = torch.cuda.Stream(), torch.cuda.Stream()

    def call(i, stream):
        args, out, ws, hint = sets[i]
        vico.vico_gather_attn_q4(*args, out, workspace=ws, keys_hint=hint, stream=stream)

    for i in range(2):
        call(i, None)
    torch.cuda.synchronize()
    want = [s[1].clone() for s in sets]
    for s in sets:
        s[1].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            call(i, streams[i])
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        assert torch.equal(s[1], w)


@pytest.mark.parametrize("heads", [(8, 2, 64), (14, 2, 128)], ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("q_len,tail,parts", [(5, 9, (1, 3)), (70, 90, (1, 3)), (140, 170, (1, 16))])
def test_what_is_masked_does_not_reach_a_row(heads, bad, where, q_len, tail, parts):
    """Tail tokens that are not finite change the rows that see them and no others."""
    at = tail - q_len + 2                                  # first seen by row 2
    clean = Case(13, *heads, q_len, tail, 3, 100, [0], [77])
    def tweak(c):                                          # noqa: E306
        c.tail["kv".index(where)][at, 1, 3] = bad
    dirty = Case(13, *heads, q_len, tail, 3, 100, [0], [77], tweak=tweak)
    for splits in parts:
        a, la = clean.run(splits)
        b, lb = dirty.run(splits)
        g = heads[0] // heads[1]
        assert np.array_equal(a[:, :g], b[:, :g]) and np.array_equal(la[:g], lb[:g])
        # rows before it: as exact as ever (a row tile raises its running maxima together, so not bit for bit)
        ref, ref_lse = oracle.gather_attention(*clean.args)
        bound = gather_bound(*clean.args, parts=max(clean.parts, 2))
        assert np.all(np.abs(b[:2] - ref[:2]) <= bound.f32(ref)[:2])
        assert np.all(np.abs(lb[:, :2] - ref_lse[:, :2]) <= bound.lse(ref_lse)[:, :2])
        seen = b[2:, g:]
        if where == "v":
            assert np.array_equal(la, lb)
            assert np.all(np.isnan(seen[..., 3]) if np.isnan(bad) else seen[..., 3] == bad)
            mask = np.arange(heads[2]) != 3
            assert np.array_equal(a[2:, g:][..., mask], seen[..., mask])
        elif np.isnan(bad):
            assert np.isnan(seen).all() and np.isnan(lb[g:, 2:]).all()


def test_nan_of_the_store_reaches_every_row():
    def tweak(c):
        c.store[3][5, 0, 1] = 255                          # V, dims 32 .. 63 of slot 5, KV head 0
        c.store[2][9, 1, 0] = 255                          # K of slot 9, KV head 1
    c = Case(14, 8, 2, 64, 2, 4, 3, 100, [0], [77], tweak=tweak)
    for splits in (1, 4):
        o, l = c.run(splits)
        assert np.isnan(o[:, :4, 32:]).all() and np.isfinite(o[:, :4, :32]).all() and np.isfinite(l[:4]).all()
        assert np.isnan(o[:, 4:]).all() and np.isnan(l[4:]).all()


@pytest.mark.parametrize("q_len,tail,parts", [(2, 4, (1, 3)), (60, 61, (1, 3)), (150, 151, (1, 16))])
@pytest.mark.parametrize("S", [5, 64])
def test_nan_of_the_sink_or_the_old_tail_reaches_every_row(q_len, tail, parts, S):
    def tweak(c):
        c.sink[1][3, 0, 7] = float("nan")                  # KV head 0
        c.tail[1][0, 1, 9] = float("inf")                  # KV head 1: a token before every row
    c = Case(19, 8, 2, 64, q_len, tail, S, 100, [0], [77], tweak=tweak)
    clean = Case(19, 8, 2, 64, q_len, tail, S, 100, [0], [77])
    for splits in parts:
        (o, l), (a, la) = c.run(splits), clean.run(splits)
        assert np.isnan(o[:, :4, 7]).all() and np.all(o[:, 4:, 9] == np.inf) and np.array_equal(l, la)
        o[:, :4, 7], o[:, 4:, 9], a[:, :4, 7], a[:, 4:, 9] = 0, 0, 0, 0
        assert np.array_equal(o, a)


def test_store_beyond_32_bit_offsets():
    """Slots past 4 GiB of codes: append, load and attention there, against the same tokens at the front."""
    Hkv, D, R, C = 64, 128, (1 << 32) // (64 * 64) + 500, 90
    g = gen(15)
    k, v = normal(g, C, Hkv, D).to(DEV), normal(g, C, Hkv, D).to(DEV)
    st = [torch.empty(R, Hkv, w, dtype=torch.uint8, device=DEV) for w in (64, 64, 4, 4)]
    far = R - 200
    vico.vico_kv_append_q4(k, v, *st, far)
    vico.vico_kv_append_q4(k, v, *st, 10)
    q, tail = normal(g, 2, Hkv, D).to(DEV), (normal(g, 2, Hkv, D).to(DEV), normal(g, 2, Hkv, D).to(DEV))
    got = []
    for at in (far, 10):
        seg = torch.tensor([at, at + 40], device=DEV), torch.tensor([40, 50], dtype=torch.int32, device=DEV)
        back = torch.empty(C, Hkv, D, dtype=torch.bfloat16, device=DEV), torch.empty(C, Hkv, D, dtype=torch.bfloat16, device=DEV)
        out = torch.empty(2, Hkv, D, device=DEV)
        vico.vico_kv_load_q4(*st, *seg, *back)
        vico.vico_gather_attn_q4(q, *tail, None, None, *st, *seg, out, keys_hint=90, num_splits=1)
        torch.cuda.synchronize()
        got.append((*back, out))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    want = kv4.decode(*kv4.encode(f64(k[:, :2])))
    assert np.array_equal(f64(got[0][0][:, :2]), want)


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("heads", [(8, 2, 64), (28, 4, 128)], ids=str)
def test_a_stream_through_the_layer(heads):
    """Chunks of a stream as a layer runs them: projection -> norm and rotation -> attention over the 4-bit ring ->
    append; then a decode step over segments of it, and the segments back as bf16.  Every stage against its
    definition on the stage's own inputs."""
    Hq, Hkv, D = heads
    g, W, R, hist = gen(16), 96, 128, 0
    wq, wk = [(1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16) for _ in "qk"]
    freq = (1e6 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float()
    st = empty_store(R, Hkv, D, fill=0)
    sink = normal(g, 5, Hkv, D), normal(g, 5, Hkv, D)
    lin_k, lin_v = np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))
    ws = torch.empty(8 << 20, dtype=torch.uint8, device=DEV)
    new = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)   # noqa: E731
    for C in (40, 33, 64, 7, 1):
        x = normal(g, C, Hq + 2 * Hkv, D)
        pos = torch.stack([torch.full((C,), 1000 + hist), torch.arange(C) // 8, torch.arange(C) % 8]).to(torch.int32)
        sec = (D // 8, D // 8 + D // 16, D // 8 + D // 16)
        q, k, v, out = new(C, Hq, D), new(C, Hkv, D), new(C, Hkv, D), new(C, Hq, D)
        xd = x.to(DEV)
        vis = min(W, hist)
        s0 = (hist - vis) % R
        n0 = min(vis, R - s0)
        seg = torch.tensor([s0, 0], device=DEV), torch.tensor([n0, vis - n0], dtype=torch.int32, device=DEV)
        a, b, c = xd.split((Hq, Hkv, Hkv), 1)
        vico.vico_qk_norm_rope(a, b, pos.to(DEV), freq.to(DEV), q, k, v=c, v_out=v, q_weight=wq.to(DEV),
                               k_weight=wk.to(DEV), sections=sec)
        vico.vico_gather_attn_q4(q, k, v, sink[0].to(DEV), sink[1].to(DEV), *st, *seg, out, workspace=ws, keys_hint=vis)
        vico.vico_kv_append_q4(k, v, *st, hist)
        torch.cuda.synchronize()
        for y, xs, w in ((q, x[:, :Hq], wq), (k, x[:, Hq:Hq + Hkv], wk)):
            ref = rope.rotate(rope.head_norm(f64(xs), f64(w), 1e-6), pos.numpy(), f64(freq), sec)
            assert np.all(np.abs(f64(y) - ref) <= U8 * np.abs(ref) + 2.0 ** -16)
        args = (f64(q), f64(k), f64(v), f64(sink[0]), f64(sink[1]), lin_k, lin_v, [hist - vis], [vis])
        check_bf16(f64(out), oracle.gather_attention(*args)[0], gather_bound(*args, parts=64))
        lin_k = np.concatenate([lin_k, kv4.decode(*kv4.encode(f64(k)))])
        lin_v = np.concatenate([lin_v, kv4.decode(*kv4.encode(f64(v)))])
        hist += C
    newest = hist - min(hist, R)
    segs = [(newest + 3, 20), (newest + 50, 31)]
    pieces = []
    for a, n in segs:                                      # linear history to ring slots, split at the ring's end
        s0, n0 = a % R, min(n, R - a % R)
        pieces += [(s0, n0), (0, n - n0)]
    seg = torch.tensor([p[0] for p in pieces], device=DEV), torch.tensor([p[1] for p in pieces], dtype=torch.int32, device=DEV)
    q, tk, tv, out = normal(g, 1, Hq, D), normal(g, 4, Hkv, D), normal(g, 4, Hkv, D), new(1, Hq, D)
    back, cnt = (new(51, Hkv, D), new(51, Hkv, D)), torch.empty(1, dtype=torch.int32, device=DEV)
    vico.vico_gather_attn_q4(q.to(DEV), tk.to(DEV), tv.to(DEV), None, None, *st, *seg, out, workspace=ws, keys_hint=51)
    vico.vico_kv_load_q4(*st, *seg, *back, out_count=cnt)
    torch.cuda.synchronize()
    empty = np.zeros((0, Hkv, D))
    args = (f64(q), f64(tk), f64(tv), empty, empty, lin_k, lin_v, [a for a, _ in segs], [n for _, n in segs])
    check_bf16(f64(out), oracle.gather_attention(*args)[0], gather_bound(*args, parts=64))
    assert int(cnt) == 51
    assert np.array_equal(f64(back[0]), np.concatenate([lin_k[a:a + n] for a, n in segs]))
    assert np.array_equal(f64(back[1]), np.concatenate([lin_v[a:a + n] for a, n in segs]))


@pytest.mark.parametrize("q_len", [1, 20])
def test_a_layer_replays_as_a_graph(q_len):
    """Norms with rotation, attention, append and load captured into one graph: every replay, with eager work and
    synchronisation between the replays, equals the eager calls."""
    Hq, Hkv, D, g = 28, 4, 128, gen(17)
    st = filled_store(g, 2000, Hkv, D)
    x = normal(g, q_len, Hq + 2 * Hkv, D).to(DEV)
    pos, freq = torch.arange(q_len, dtype=torch.int32, device=DEV), torch.rand(64, generator=g).to(DEV)
    seg = torch.tensor([0, 900], device=DEV), torch.tensor([800, 300], dtype=torch.int32, device=DEV)
    new = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)   # noqa: E731
    bufs = [new(q_len, Hq, D), new(q_len, Hkv, D), new(q_len, Hkv, D), new(q_len, Hq, D), new(40, Hkv, D), new(40, Hkv, D)]
    ws = torch.empty(16 << 20, dtype=torch.uint8, device=DEV)

    def layer():
        q, k, v, out, bk, bv = bufs
        a, b, c = x.split((Hq, Hkv, Hkv), 1)
        vico.vico_qk_norm_rope(a, b, pos, freq, q, k, v=c, v_out=v)
        vico.vico_gather_attn_q4(q, k, v, None, None, *st, *seg, out, workspace=ws, keys_hint=1100)
        vico.vico_kv_append_q4(k, v, *st, 1990)
        vico.vico_kv_load_q4(*st, *seg, bk, bv)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            layer()
    for i in range(4):
        x.copy_(normal(gen(100 + i), q_len, Hq + 2 * Hkv, D))
        store = [t.clone() for t in st]
        torch.cuda.synchronize()
        layer()
        torch.cuda.synchronize()
        want = [b.clone() for b in bufs] + [t.clone() for t in st]
        for t, u in zip(st, store):
            t.copy_(u)
        for b in bufs:
            b.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for b, w in zip(bufs + list(st), want):
            assert torch.equal(b, w)


def test_both_paths_of_the_binding_give_the_same(monkeypatch):
    import paper_2606_19849_amd._binding as binding
    seen = []

    def everything():
        c = Case(18, 8, 2, 64, 3, 20, 4, 120, [0, 60], [50, 40])
        seen.append((c.run(2)[0], c.run(dtype=torch.bfloat16)[0], rope_case(1, 9, 4, 2, 64, axes=3)[0][0],
                     rope_case(1, 1, 4, 2, 64, wt=torch.float32, with_v=False)[0][0], *store_values(c.store)))
        test_load([3, 9], [5, 5], 12)

    class Never:
        def __getattr__(self, name):
            return lambda *a: None

    everything()
    monkeypatch.setattr(binding, "_calls", Never())
    everything()
    for a, b in zip(*seen):
        assert np.array_equal(a, b)


def test_a_stream_handle_takes_the_short_path():
    """Plain calls with a stream are answered by the C++ part of the binding, on that stream."""
    import paper_2606_19849_amd._binding as binding
    calls, s = binding._fast(), torch.cuda.Stream()
    st, k = empty_store(8, 2, 64), normal(gen(19), 4, 2, 64).to(DEV)
    out = [torch.zeros_like(k) for _ in range(4)]
    seg = torch.zeros(1, dtype=torch.int64, device=DEV), torch.full((1,), 4, dtype=torch.int32, device=DEV)
    pos, freq = torch.arange(4, dtype=torch.int32, device=DEV)[None], torch.rand(32, generator=gen(20)).to(DEV)
    torch.cuda.synchronize()
    h = s.cuda_stream
    assert calls.append_q4(k, k, *st, 0, h) == 0
    assert calls.load_q4(*st, *seg, out[0], out[1], None, h) == 0
    assert calls.gather_q4(k[:1], k, k, None, None, *st, *seg, out[2][:1], None, 4, 1, 0.0, h, None) == 0
    assert calls.qk_norm_rope(k, k, pos, freq, out[2], out[3], None, None, None, None, 1e-6, 0, 0, 0, 0, h) == 0
    s.synchronize()
    assert np.array_equal(f64(out[0]), store_values(st)[0][:4]) and torch.equal(out[0], out[1])
    assert torch.equal(out[2], out[3]) and bool(out[2].any())


def test_refusals_of_the_binding():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)   # noqa: E731
    st = empty_store(8, 2, 64)
    k = bf(4, 2, 64)
    seg = torch.zeros(2, dtype=torch.int64, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    pos, freq = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(32, device=DEV)
    for bad in (lambda: vico.vico_kv_append_q4(k, k, st[0], st[1], st[2], st[2][:4], 0),
                lambda: vico.vico_kv_append_q4(k, k[:3], *st, 0),
                lambda: vico.vico_kv_append_q4(k.float(), k, *st, 0),
                lambda: vico.vico_kv_append_q4(k, k.clone(), st[0].to(torch.int8), *st[1:], 0),
                lambda: vico.vico_kv_load_q4(*st, seg[0], seg[1][:1], bf(4, 2, 64), bf(4, 2, 64)),
                lambda: vico.vico_kv_load_q4(*st, *seg, bf(4, 2, 128), bf(4, 2, 128)),
                lambda: vico.vico_gather_attn_q4(bf(1, 4, 64), k, k[:3], None, None, *st, *seg, bf(1, 4, 64)),
                lambda: vico.vico_gather_attn_q4(bf(1, 4, 64), k, k, k, None, *st, *seg, bf(1, 4, 64)),
                lambda: vico.vico_gather_attn_q4(bf(1, 4, 64), k, k, None, None, *st, *seg, bf(2, 4, 64)),
                lambda: vico.vico_qk_norm_rope(k, k, pos[:3], freq, bf(4, 2, 64), bf(4, 2, 64)),
                lambda: vico.vico_qk_norm_rope(k, k, pos, freq, bf(4, 2, 64), bf(4, 1, 64)),
                lambda: vico.vico_qk_norm_rope(k.transpose(1, 2), k, pos, freq, bf(4, 2, 64), bf(4, 2, 64)),
                lambda: vico.vico_qk_norm_rope(k, k, pos, freq, bf(4, 2, 64), bf(4, 2, 64), v=k),
                lambda: vico.vico_qk_norm_rope(k, k, pos, freq, bf(4, 2, 64), bf(4, 2, 64), q_weight=freq),
                lambda: vico.vico_qk_norm_rope(k, k, pos, freq, bf(4, 2, 64), bf(4, 2, 64), sections=(1, 2))):
        with pytest.raises(ValueError):
            bad()
    for status, bad in ((-3, lambda: vico.vico_kv_append_q4(bf(9, 2, 64), bf(9, 2, 64), *st, 0)),
                        (-1, lambda: vico.vico_kv_append_q4(k, k, st[0], st[0], st[2], st[3], 0)),
                        (-5, lambda: vico.vico_gather_attn_q4(bf(1, 4, 64), k, k, None, None, *st, *seg, bf(1, 4, 64),
                                                              num_splits=2)),
                        (-1, lambda: vico.vico_qk_norm_rope(k, k, pos, freq, k, k)),
                        (-1, lambda: vico.vico_qk_norm_rope(k, k, pos, freq[:20], bf(4, 2, 64), bf(4, 2, 64)))):
        with pytest.raises(vico.VicoError) as e:
            bad()
        assert e.value.status == status
    torch.cuda.synchronize()
