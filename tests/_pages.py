"""Caches in pages for tests: random sequences in a pool whose every other place holds NaN, and the derived
per-element bounds of tests/_bounds.py for attention over them."""
from __future__ import annotations

import numpy as np
import torch

import paper_2606_19849_amd as vico
from oracle import pages
from tests._bounds import Bound, _eta_dz

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


class Cache:
    """Sequences (new tokens n, cached tokens H) in pages.  Places that no sequence's tokens take are NaN, entries past
    a row's pages are numbers that are no page; `drop`: pages (row, entry) that the table does not have."""

    def __init__(self, seed, seqs, heads=(4, 2, 64), page=16, sink=0, window=-1, spare=3, width=None, drop=(), pad=2,
                 sigma=2.0, order=None):
        g = torch.Generator()
        g.manual_seed(seed)
        self.Hq, self.Hkv, self.D = heads
        self.n, self.H = [s[0] for s in seqs], [s[1] for s in seqs]
        self.page, self.sink, self.window = page, sink, window
        B = len(seqs)
        need = [pages.pages_of(n + H, page) for n, H in seqs]
        self.width = width or max(need + [1]) + 1
        N = sum(need) + spare
        ids = torch.randperm(N, generator=g).tolist() if order is None else order(N)
        bad = [-1, N, -7, 2 ** 31 - 1, -2 ** 31]
        self.table = [[bad[(b + j) % len(bad)] for j in range(self.width)] for b in range(B)]
        nan = float("nan")
        shape = (N, page, self.Hkv, self.D)
        self.k, self.v = torch.full(shape, nan, dtype=torch.bfloat16), torch.full(shape, nan, dtype=torch.bfloat16)
        self.q_start = np.cumsum([0] + self.n).tolist()
        rows = self.q_start[-1] + pad
        self.q = (torch.randn(rows, self.Hq, self.D, generator=g) * sigma).to(torch.bfloat16)
        for b, (n, H) in enumerate(seqs):
            for j in range(min(need[b], self.width)):
                p = ids.pop()
                m = min(page, H + n - j * page)
                self.k[p, :m] = (torch.randn(m, self.Hkv, self.D, generator=g) * sigma).to(torch.bfloat16)
                self.v[p, :m] = torch.randn(m, self.Hkv, self.D, generator=g).to(torch.bfloat16)
                lo = H - window if window >= 0 else 0
                gone = j * page >= min(sink, max(lo, 0)) and (j + 1) * page <= lo      # wholly between sink and window
                if (b, j) not in drop and not (gone and (b + j) % 2):     # half of the pages left behind are still there
                    self.table[b][j] = p
                if gone:
                    self.k[p], self.v[p] = nan, nan

    def device(self):
        self.dk, self.dv, self.dq = self.k.to(DEV), self.v.to(DEV), self.q.to(DEV)
        self.dt, self.ds, self.dl = i32(self.table), i32(self.q_start), i32(self.H)
        return self

    def place(self, b, p):
        return self.table[b][p // self.page], p % self.page

    def attention(self, dtype=torch.float32, flags=0, splits=0, scale=0.0, max_q=None, hint=0, stream=None, lse=True,
                  workspace=None):
        rows = self.q.shape[0]
        out = torch.full((rows, self.Hq, self.D), 7.25, dtype=dtype, device=DEV)
        lo = torch.full((self.Hq, rows), 7.25, dtype=torch.float32, device=DEV) if lse else None
        most = max(self.n + [0]) if max_q is None else max_q
        self.parts, wb = vico.vico_paged_attn_plan(len(self.n), rows, most, self.page, self.width, self.sink, self.window,
                                                   hint, self.Hq, self.Hkv, self.D, splits)
        if workspace is None and wb:
            workspace = torch.full((wb + 256,), 255, dtype=torch.uint8, device=DEV)       # NaN wherever nothing is written
        torch.cuda.synchronize()
        vico.vico_paged_attn(self.dq, self.ds, self.dl, self.dk, self.dv, self.dt, out, lse=lo, sink_len=self.sink,
                             window=self.window, max_q_len=most, keys_hint=hint, num_splits=splits, softmax_scale=scale,
                             flags=flags, workspace=workspace, stream=stream)
        torch.cuda.synchronize()
        if workspace is not None and wb and workspace.numel() == wb + 256:
            assert torch.all(workspace[wb:] == 255)
        return out, lo

    def oracle(self, bidirectional=False, scale=None, max_q=None, zero=()):
        """(out, lse, covered, Bound); zero: places of V taken as 0 (row, position, dim)."""
        q, k, v = f64(self.q), f64(self.k), f64(self.v)
        for b, p, h, d in zero:
            page, at = self.place(b, p)
            v[page, at, h, d] = 0.0
        rows = q.shape[0]
        A = np.zeros((rows, self.Hq, self.D))
        kmax, most = np.zeros((rows, self.Hq)), [1]
        s = self.D ** -0.5 if scale is None else scale

        def bound(rs, hq, K, V, p):
            A[rs, hq] = p @ np.abs(V)
            kmax[rs, hq] = np.sqrt((K ** 2).sum(-1)).max()
            most[0] = max(most[0], K.shape[0])

        out, lse, covered = pages.paged_attention(q, self.q_start, self.H, k, v, self.table, self.sink, self.window,
                                                  bidirectional, scale, max_q, bound)
        qn = np.sqrt((q ** 2).sum(-1))
        eta, dz = _eta_dz(qn * kmax, np.ones(self.Hq), s, self.D)
        return out, lse, covered, Bound(A, eta, dz, most[0], getattr(self, "parts", 1))


def check(cache, got, ref):
    """fp32 or bf16 output and the log-sum-exp within the bounds; rows of no sequence as they were; empty rows 0, -inf."""
    out, lse, covered, b = ref
    o = f64(got[0])
    assert np.all(o[~covered] == 7.25)
    bound = (b.f32 if got[0].dtype == torch.float32 else b.bf16)(out)
    err = np.abs(o - out)
    bad = ~(err <= bound) & covered[:, None, None]
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), float(err[bad].max()), int(bad.sum()))
    if got[1] is not None:
        l = f64(got[1])
        assert np.all(l[:, ~covered] == 7.25)
        empty = np.isneginf(lse) & covered[None]
        assert np.all(np.isneginf(l[empty])) and np.all(o[empty.T] == 0)
        fine = covered[None] & ~empty
        lb = b.lse(np.where(fine, lse, 0))
        assert np.all(np.abs(l - np.where(fine, lse, 0))[fine] <= lb[fine])
