"""GPU tests of include/vico_cache.h at the edges of its arguments' values."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import paper_2606_19849_amd as vico
from oracle import rope
from tests._bounds import gather_bound
from tests._gpu import check_f32
from tests.test_gpu_cache import DEV, Case, check_rope, empty_store, f64, gen, normal, rope_case, store_values

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- values that are not finite

@pytest.mark.parametrize("heads", [(8, 2, 64), (14, 2, 128)], ids=str)
@pytest.mark.parametrize("where,bad", [("tail", float("nan")), ("tail", float("inf")), ("store", None)])
def test_a_value_of_vanishing_weight_that_is_not_finite(heads, where, bad):
    """A row's weights outside of one part are 0 in fp32 (that part's key is e^400 ahead): a NaN or an infinity there
    reaches the row all the same, however many parts there are."""
    def tweak(c):
        c.q[:] = 8.0
        c.sink[0][0] = 8.0                                 # logit 8 * 8 * sqrt(D), against a spread of about 90
        if where == "tail":
            c.tail[1][0, 1, 9] = bad
        else:
            c.store[3][777, 1, 0] = 255                    # V, dims 0 .. 31 of slot 777, KV head 1
    c = Case(3, *heads, 2, 9, 1, 1000, [0], [1000], tweak=tweak)
    clean = Case(3, *heads, 2, 9, 1, 1000, [0], [1000], tweak=lambda c: (c.q.fill_(8.0), c.sink[0][0].fill_(8.0)))
    g = heads[0] // heads[1]
    for splits in (1, 3, 16, 17, 64):
        (o, l), (a, la) = c.run(splits), clean.run(splits)
        assert c.parts == splits
        assert not np.isfinite(o[:, g:, 9]).any()
        hit = np.zeros(heads[2], bool)
        hit[9 if where == "tail" else slice(0, 32)] = True
        assert np.array_equal(o[:, :g], a[:, :g]) and np.array_equal(o[:, g:, ~hit], a[:, g:, ~hit])
        assert np.array_equal(l, la)


# ---------------------------------------------------------------- norms over the whole range of bf16

def normed(x, Hq, w, eps, adjacent=False):
    """(result, definition, E) of test_gpu_cache.check_rope for q and k of x [T, heads, D] with weights w."""
    T, heads, D = x.shape
    pos, freq = torch.arange(T, dtype=torch.int32) * 37, (1e4 ** (-torch.arange(D // 2, dtype=torch.float64) / D)).float()
    q, k = x.to(DEV).split((Hq, heads - Hq), 1)
    out = [torch.empty(T, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hq, heads - Hq)]
    vico.vico_qk_norm_rope(q, k, pos.to(DEV), freq.to(DEV), *out, q_weight=w.to(DEV), k_weight=w.to(DEV), eps=eps,
                           flags=vico.VICO_ROPE_ADJACENT * adjacent)
    torch.cuda.synchronize()
    res = []
    for y, xs in ((out[0], x[:, :Hq]), (out[1], x[:, Hq:])):
        n = rope.head_norm(f64(xs), f64(w), eps)
        pair = (lambda a: a.reshape(*a.shape[:2], -1, 2)) if adjacent else (
            lambda a: a.reshape(*a.shape[:2], 2, -1).swapaxes(-1, -2))
        E = np.repeat(np.abs(pair(n)).sum(-1), 2, -1) if adjacent else np.tile(np.abs(pair(n)).sum(-1), 2)
        res.append((f64(y), rope.rotate(n, pos.numpy()[None], f64(freq), None, adjacent), E))
    return res


@pytest.mark.parametrize("D,adjacent", [(64, False), (128, True)])
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-6, 1e-2, 1e12])
@pytest.mark.parametrize("size", [1e-38, 1e-25, 1e-16, 1.0, 1e18, 1e19, 1e25, 1e38])
def test_norm_of_any_size(D, adjacent, eps, size):
    """Squares that leave fp32 on either side; eps above, beside and below them."""
    g = gen(31)
    x = (torch.randn(5, 6, D, generator=g, dtype=torch.float64).clamp(-3, 3) * size).to(torch.bfloat16)
    w = 1 + 0.3 * torch.randn(D, generator=g)
    check_rope(normed(x, 4, w, eps, adjacent))


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
def test_norm_of_unlike_elements(eps):
    """One element sets the norm, the others are far below it, in heads of every size side by side."""
    x = normal(gen(32), 8, 6, 128, sigma=1.0)
    for t in range(8):
        x[t, :, t] = (-1.0) ** t * 10.0 ** (5 * t)         # 1 .. 1e35
        x[t, 5] = (x[t, 5].double() * 1e-30).to(torch.bfloat16)
    check_rope(normed(x, 4, torch.ones(128), eps))


def test_norm_of_zeros():
    x = normal(gen(33), 4, 4, 64)
    x[1], x[2, 3] = 0, 0
    (q, _, _), (k, _, _) = normed(x, 2, torch.ones(64), 1e-6)
    assert np.all(q[1] == 0) and np.all(k[1:3, 1] == 0) and np.all(np.isfinite(k))
    with np.errstate(invalid="ignore"):
        (q, ref, _), (k, _, _) = normed(x, 2, torch.ones(64), 0.0)
    assert np.isnan(q[1]).all() and np.isnan(ref[1]).all() and np.isnan(k[2, 1]).all() and np.isfinite(k[2, 0]).all()


# ---------------------------------------------------------------- a stream that has no store yet

@pytest.mark.parametrize("segs", [None, 2])
@pytest.mark.parametrize("stream", [False, True])
def test_attention_without_a_store(segs, stream, monkeypatch):
    """As vico_gather_attn takes it: None, with or without a table; through both paths of the binding."""
    import paper_2606_19849_amd._binding as binding
    g = gen(34)
    q, tk, tv, sk, sv = (normal(g, n, h, 64) for n, h in ((3, 8), (9, 2), (9, 2), (70, 2), (70, 2)))
    table = (None, None) if segs is None else (torch.tensor([0, 5], device=DEV), torch.tensor([7, 3], dtype=torch.int32, device=DEV))
    args = tuple(map(f64, (q, tk, tv, sk, sv))) + (np.zeros((0, 2, 64)),) * 2 + ([], [])
    ref, ref_lse = oracle.gather_attention(*args)
    dev = [t.to(DEV) for t in (q, tk, tv, sk, sv)]

    class Never:
        def __getattr__(self, name):
            return lambda *a: None

    for calls in (binding._fast(), Never()):
        monkeypatch.setattr(binding, "_calls", calls)
        out, lse = torch.empty(3, 8, 64, device=DEV), torch.empty(8, 3, device=DEV)
        torch.cuda.synchronize()
        vico.vico_gather_attn_q4(*dev, None, None, None, None, *table, out, lse=lse, num_splits=1,
                                 stream=torch.cuda.Stream() if stream else None)
        torch.cuda.synchronize()
        check_f32(f64(out), ref, gather_bound(*args), f64(lse), ref_lse)
        with pytest.raises(ValueError, match="all or none"):
            vico.vico_gather_attn_q4(*dev, torch.zeros(4, 2, 32, dtype=torch.uint8, device=DEV), None, None, None, *table, out)


# ---------------------------------------------------------------- scale bytes that the append never writes

def test_load_of_every_scale_byte_and_code():
    """256 slots, one for each scale byte, all 16 codes in either half of a byte: exact, subnormals too; from 2^128 on an
    infinity."""
    codes = torch.arange(16, dtype=torch.uint8).repeat(256, 1, 2)
    codes = codes | (15 - codes) << 4
    scales = torch.arange(256, dtype=torch.uint8).view(256, 1, 1).expand(256, 1, 2).contiguous()
    st = [t.to(DEV) for t in (codes, codes.flip(-1).contiguous(), scales, scales)]
    out = [torch.empty(256, 1, 64, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    vico.vico_kv_load_q4(*st, torch.tensor([0], device=DEV), torch.tensor([256], dtype=torch.int32, device=DEV), *out)
    torch.cuda.synchronize()
    for o, want in zip(out, store_values(st)):
        want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
        o = f64(o)
        assert np.array_equal(o, want, equal_nan=True) and np.array_equal(np.signbit(o[:255]), np.signbit(want[:255]))


@pytest.mark.parametrize("heads", [(8, 2, 64), (14, 2, 128)], ids=str)
def test_attention_over_slots_of_zeros_and_of_subnormal_values(heads):
    """Slots that nobody has written, in arrays of zeros, are keys and values of zero; bytes 0 to 3 with any codes are as
    small as makes no difference to the derived bounds."""
    def tweak(c):
        for t in c.store:
            t[20:40] = 0
        for t in c.store[2:]:
            t[50:80] = torch.arange(30, dtype=torch.uint8, device=DEV).view(30, 1, 1) % 4
    c = Case(35, *heads, 3, 9, 4, 100, [0], [95], tweak=tweak)
    for splits in (0, 1, 3):
        c.check(splits)
    c = Case(36, *heads, 300, 310, 4, 100, [0], [95], tweak=tweak)
    c.check(16)


# ---------------------------------------------------------------- the log-sum-exp of a row that is NaN

@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("q_len,pad,splits", [(1, 0, 1), (1, 0, 3), (1, 0, 20), (40, 70, 1), (40, 70, 3), (40, 70, 20),
                                              (300, 0, 1), (300, 0, 16)])
def test_log_sum_exp_of_nan_rows(q_len, pad, splits, bad):
    """NaN over the 4-bit store, -inf over the bf16 one, as the headers say; the outputs are NaN in both.  Query heads of
    the other KV head keep theirs."""
    q = normal(gen(40), q_len, 8, 64, sigma=1.0).abs().to(DEV)
    tail = [normal(gen(41 + i), q_len + 3, 2, 64).to(DEV) for i in range(2)]
    tail[0][0, 1] = bad                                    # a token that every row sees; logits of +inf where bad is
    seg = torch.zeros(1 + pad, dtype=torch.int64, device=DEV), torch.zeros(1 + pad, dtype=torch.int32, device=DEV)
    seg[1][0] = 700
    bf16 = [normal(gen(44 + i), 800, 2, 64).to(DEV) for i in range(2)]
    q4 = empty_store(800, 2, 64)
    vico.vico_kv_append_q4(*bf16, *q4, 0)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    for call, store, want in ((vico.vico_gather_attn_q4, q4, np.nan), (vico.vico_gather_attn, bf16, -np.inf)):
        out, lse = torch.empty(q_len, 8, 64, device=DEV), torch.empty(8, q_len, device=DEV)
        call(q, *tail, None, None, *store, *seg, out, lse=lse, workspace=ws, keys_hint=700, num_splits=splits)
        torch.cuda.synchronize()
        assert torch.isnan(out[:, 4:]).all() and torch.isfinite(out[:, :4]).all() and torch.isfinite(lse[:4]).all()
        assert np.array_equal(f64(lse[4:]), np.full((4, q_len), want), equal_nan=True)


# ---------------------------------------------------------------- strides and rotated widths

def test_rope_of_tokens_far_apart():
    """Token strides of 2^30 elements: offsets beyond 32 bits, in elements and in bytes."""
    T, Hq, Hkv, D, stride = 4, 3, 2, 64, 1 << 30
    buf = torch.empty((T - 1) * stride + (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device=DEV)
    x = normal(gen(50), T, Hq + 2 * Hkv, D)
    rows = buf.as_strided((T, Hq + 2 * Hkv, D), (stride, D, 1))
    rows.copy_(x)
    q, k, v = rows.split((Hq, Hkv, Hkv), 1)
    out = [torch.empty(T, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv)]
    w, pos, freq = torch.ones(D), torch.arange(T, dtype=torch.int32) * 1000, (1e4 ** (-torch.arange(32) / 32.0)).float()
    vico.vico_qk_norm_rope(q, k, pos.to(DEV), freq.to(DEV), out[0], out[1], v=v, v_out=out[2], q_weight=w.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(out[2].cpu(), x[:, Hq + Hkv:])
    res = []
    for y, xs, wi in ((out[0], x[:, :Hq], f64(w)), (out[1], x[:, Hq:Hq + Hkv], None)):
        n = rope.head_norm(f64(xs), wi, 1e-6)
        E = np.tile(np.abs(n[..., :32]) + np.abs(n[..., 32:]), 2)
        res.append((f64(y), rope.rotate(n, pos.numpy()[None], f64(freq)), E))
    check_rope(res)


@pytest.mark.parametrize("D,rot", [(64, 48), (128, 48), (128, 80), (128, 112)])
@pytest.mark.parametrize("kw", [dict(), dict(adjacent=True), dict(axes=3), dict(axes=3, strided=True)],
                         ids=lambda k: "-".join(k) or "plain")
def test_rope_of_other_widths(D, rot, kw):
    check_rope(rope_case(rot + D, 13, 5, 2, D, rot=rot, **kw))
