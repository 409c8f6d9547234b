"""Performance cases of the paged cache: sequences of ragged length in one pool of pages.

Four kinds of pass, each what a program does with the cache in one step:

  attend   attention of every sequence's new tokens over its pages: decode steps, short queries, visual chunks and
           mixtures of them, with or without a window behind a fixed sink
  append   every sequence's new keys and values into its pages
  branch   questions branch off running streams: rows of the page table forked, room reserved for the question's
           tokens (a half-filled page that the stream holds too is replaced), pages copied in every layer
  compact  pages that the streams' windows have left are freed, the pages in use moved to the pool's low end

`own` false computes them from elementary torch operations, true by the package's entry points.  Head counts, head
sizes, sinks and windows are those of the repository's workloads (3B and 7B layers; small ones at head size 64).
"""
import math

import torch

own = False

# heads (query, key/value, size)
HEADS = {"3b": (16, 2, 128), "7b": (28, 4, 128), "small": (8, 2, 64)}
SIGMA_QK = 2.0 ** 0.5    # logits of standard deviation 2
DEV = "cuda"
FULL = -1                # a window that leaves nothing out
WORKSPACE = 64 << 20     # scratch that a program keeps for all its calls


# ---------------------------------------------------------------- the cases

def _attend(name, model, page, steps, chunks, n_lo, n_hi, h_lo, h_hi, window=FULL, sink=0, lse=False):
    """`steps` sequences with one new token, `chunks` with n_lo to n_hi; h_lo to h_hi tokens cached before."""
    return {"name": name, "kind": "attend", "model": model, "page": page, "steps": steps, "chunks": chunks, "n_lo": n_lo,
            "n_hi": n_hi, "h_lo": h_lo, "h_hi": h_hi, "window": window, "sink": sink, "lse": lse}


def _append(name, model, page, steps, chunks, n_lo, n_hi, h_lo, h_hi):
    return {"name": name, "kind": "append", "model": model, "page": page, "steps": steps, "chunks": chunks, "n_lo": n_lo,
            "n_hi": n_hi, "h_lo": h_lo, "h_hi": h_hi, "window": FULL, "sink": 0}


def _branch(name, model, page, streams, branches, layers, h_lo, h_hi, n_lo, n_hi):
    return {"name": name, "kind": "branch", "model": model, "page": page, "streams": streams, "branches": branches,
            "layers": layers, "h_lo": h_lo, "h_hi": h_hi, "n_lo": n_lo, "n_hi": n_hi}


def _compact(name, model, page, streams, layers, h_lo, h_hi, window, sink):
    return {"name": name, "kind": "compact", "model": model, "page": page, "streams": streams, "layers": layers,
            "h_lo": h_lo, "h_hi": h_hi, "window": window, "sink": sink}


def listed():
    return [
        # one answer token on a small layer, small pages: the smallest call there is
        _attend("decode_small", "small", 16, 1, 0, 1, 1, 200, 200),
        # answer tokens of 32 conversations in one step
        _attend("decode_7b_batch", "7b", 64, 32, 0, 1, 1, 1024, 16384),
        # one answer token over all of a long stream
        _attend("decode_7b_long", "7b", 256, 1, 0, 1, 1, 262143, 262143, lse=True),
        # a visual chunk of one stream beside the answer tokens of 31 others, bounded histories
        _attend("mixed_7b", "7b", 64, 31, 1, 1024, 1024, 500, 20000, window=8192, sink=64),
        # ragged visual chunks of four streams
        _attend("chunks_3b", "3b", 128, 0, 4, 256, 1024, 3000, 30000, window=8192, sink=64, lse=True),
        # the large visual chunk of one stream
        _attend("chunk_7b", "7b", 256, 0, 1, 2048, 2048, 50001, 50001, window=16384, sink=64),
        # the new tokens of 32 conversations into the cache
        _append("append_7b_batch", "7b", 64, 32, 0, 1, 1, 1024, 4096),
        # visual chunks of 16 streams into the cache
        _append("append_3b_chunks", "3b", 16, 0, 16, 256, 2048, 100, 3000),
        # one question to each of three short streams
        _branch("branch_small", "small", 16, 3, 3, 1, 100, 900, 5, 40),
        # questions to sixteen long streams, two layers' pages
        _branch("branch_7b", "7b", 64, 16, 16, 2, 2000, 12000, 16, 200),
        # windows of a few streams have moved on
        _compact("compact_3b", "3b", 64, 3, 1, 2000, 9000, 2048, 64),
        # a large pool after its streams' windows have moved on
        _compact("compact_7b", "7b", 64, 24, 1, 4000, 16000, 6144, 64),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = _draw(rng)
    case.pop("name")
    return case


def _draw(rng):
    kind = rng.choice(["decode", "decode", "short", "mixed", "chunks", "append", "branch", "compact"])
    model, page = rng.choice(["3b", "7b", "small"]), rng.choice([16, 32, 64, 128, 256])
    window, sink = (_log(rng, 64, 8192), rng.choice([0, 16, 64, 100])) if rng.random() < 0.4 else (FULL, 0)
    lse = rng.random() < 0.3
    lo = _log(rng, 1, 4096)
    h = (lo, lo + _log(rng, 1, 8192))
    if kind == "decode":
        return _attend("", model, page, _log(rng, 1, 64), 0, 1, 1, *h, window, sink, lse)
    if kind == "short":
        n = _log(rng, 2, 32)
        return _attend("", model, page, 0, _log(rng, 1, 8), n, n + rng.randrange(40), *h, window, sink, lse)
    if kind == "mixed":
        n = _log(rng, 2, 512)
        return _attend("", model, page, _log(rng, 1, 32), rng.choice([1, 2]), n, 2 * n, *h, window, sink, lse)
    if kind == "chunks":
        n = _log(rng, 64, 700)
        return _attend("", model, page, 0, rng.choice([1, 2, 4]), n, n + rng.randrange(320), *h, window, sink, lse)
    if kind == "append":
        n = _log(rng, 1, 1024)
        return _append("", model, page, rng.randrange(20), _log(rng, 1, 8), n, 2 * n, lo, lo + rng.randrange(2000))
    if kind == "branch":
        n = _log(rng, 1, 100)
        return _branch("", model, page, _log(rng, 1, 16), _log(rng, 1, 24), rng.choice([1, 2]), lo, h[1], n, 2 * n)
    return _compact("", model, page, _log(rng, 1, 24), 1, lo + 500, lo + 500 + _log(rng, 500, 8000), _log(rng, 200, 4096),
                    rng.choice([0, 64, 100]))


# ---------------------------------------------------------------- layouts: properties of the case, not of the seed

def _pages(tokens, page):
    return -(-tokens // page)


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g).tolist()


def _generator(case):
    g = torch.Generator()
    g.manual_seed(case["page"] * 7919 + case["h_lo"] * 31 + case["h_hi"])
    return g


def _sequences(case):
    """New tokens and cached tokens of every sequence, in an order that mixes the two sorts."""
    g = _generator(case)
    n = [1] * case["steps"] + _ints(g, case["n_lo"], case["n_hi"], case["chunks"])
    n = [n[i] for i in torch.randperm(len(n), generator=g).tolist()]
    return n, _ints(g, case["h_lo"], case["h_hi"], len(n)), g


def _spans(case, n, h):
    """The cached and new positions that a sequence's rows may see: the sink's, and those from the window on."""
    first = max(h - case["window"], 0) if case["window"] >= 0 else 0
    sink = min(case["sink"], first)
    return sink, first


def _table(rows, spare, g):
    """A page table for rows of wanted logical pages (lists of page numbers), scattered over a pool, and the pool's size."""
    total = sum(len(r) for r in rows)
    pool = total + spare
    order = torch.randperm(pool, generator=g).tolist()
    table = torch.full((len(rows), max(max(r, default=0) for r in rows) + 1), -1, dtype=torch.int32)
    for i, r in enumerate(rows):
        for j in r:
            table[i, j] = order.pop()
    return table, pool


def _starts(n):
    return torch.tensor([0] + n).cumsum(0).to(torch.int32)


def _sequence_layout(case):
    n, h, g = _sequences(case)
    P, rows = case["page"], []
    for a, b in zip(n, h):
        sink, first = _spans(case, a, b)
        rows.append(sorted(set(range(_pages(sink, P))) | set(range(first // P, _pages(a + b, P)))))
    return n, h, *_table(rows, 3, g)


def _branch_layout(case):
    """Streams' rows filled, branches' rows empty; new tokens of every row; the row that each is taken from."""
    g = _generator(case)
    S, B, P = case["streams"], case["branches"], case["page"]
    h = _ints(g, case["h_lo"], case["h_hi"], S)
    n = _ints(g, case["n_lo"], case["n_hi"], B)
    of = _ints(g, 0, S - 1, B)
    table, pool = _table([list(range(_pages(x, P))) for x in h], sum(_pages(x, P) + 2 for x in n), g)
    width = max(_pages(h[s] + x, P) for s, x in zip(of, n))
    full = torch.full((S + B, max(width, table.shape[1])), -1, dtype=torch.int32)
    full[:S, :table.shape[1]] = table
    return h + [0] * B, [0] * S + n, list(range(S)) + of, full, pool


def _compact_layout(case):
    g = _generator(case)
    h = _ints(g, case["h_lo"], case["h_hi"], case["streams"])
    table, pool = _table([list(range(_pages(x, case["page"]))) for x in h], 5, g)
    return h, [case["sink"]] * len(h), [max(x - case["window"], 0) for x in h], table, pool


# ---------------------------------------------------------------- inputs

def _normal(g, sigma, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16) * sigma


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    Hq, Hkv, D = HEADS[case["model"]]
    kind, P = case["kind"], case["page"]
    empty = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device=DEV)   # noqa: E731
    st = {"kind": kind, "case": case}
    if kind in ("attend", "append"):
        n, h, table, pool = _sequence_layout(case)
        total = sum(n)
        st.update(n=n, h=h, q_start=_starts(n).to(DEV), seq_len=torch.tensor(h, dtype=torch.int32, device=DEV),
                  table=table.to(DEV), k_pages=_normal(g, SIGMA_QK, pool, P, Hkv, D), v_pages=_normal(g, 1.0, pool, P, Hkv, D))
        if kind == "append":
            st.update(k=_normal(g, SIGMA_QK, total, Hkv, D), v=_normal(g, 1.0, total, Hkv, D))
        else:
            st.update(q=_normal(g, SIGMA_QK, total, Hq, D), out=empty(total, Hq, D),
                      lse=empty(Hq, total, dtype=torch.float32) if case["lse"] else None,
                      workspace=empty(WORKSPACE, dtype=torch.uint8))
        return st
    if kind == "branch":
        h, n, parent, table, pool = _branch_layout(case)
        st.update(q_start=_starts(n).to(DEV), parent=torch.tensor(parent, dtype=torch.int32, device=DEV),
                  moves=empty(len(h), 2, dtype=torch.int32), granted=empty(len(h), dtype=torch.int32))
    else:
        h, first, last, table, pool = _compact_layout(case)
        st.update(first=torch.tensor(first, dtype=torch.int32, device=DEV),
                  last=torch.tensor(last, dtype=torch.int32, device=DEV),
                  moves=empty(pool // 2, 2, dtype=torch.int32), count=empty(1, dtype=torch.int32))
    held = torch.bincount(table[table >= 0].long(), minlength=pool)
    st.update(seq_len=torch.tensor(h, dtype=torch.int32, device=DEV), table=table.to(DEV), refs=held.to(torch.int32).to(DEV),
              k_pages=_normal(g, SIGMA_QK, case["layers"], pool, P, Hkv, D),
              v_pages=_normal(g, 1.0, case["layers"], pool, P, Hkv, D), workspace=empty(WORKSPACE, dtype=torch.uint8))
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2606_19849_amd as vico
    case, kind = st["case"], st["kind"]
    P, table = case["page"], st["table"]
    if kind == "attend":
        vico.vico_paged_attn(st["q"], st["q_start"], st["seq_len"], st["k_pages"], st["v_pages"], table, st["out"],
                             lse=st["lse"], sink_len=case["sink"], window=case["window"], max_q_len=max(st["n"]),
                             keys_hint=max(st["h"]) + max(st["n"]), workspace=st["workspace"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "append":
        vico.vico_paged_append(st["k"], st["v"], st["q_start"], st["seq_len"], st["k_pages"], st["v_pages"], table)
        return {"k": st["k_pages"], "v": st["v_pages"]}
    if kind == "branch":       # the last questions' rows are given back as the rows are forked anew
        vico.vico_pages_fork(table, st["refs"], st["seq_len"], st["parent"], P)
        vico.vico_pages_reserve(table, st["refs"], st["seq_len"], st["q_start"], P, st["moves"], st["granted"],
                                st["workspace"])
        vico.vico_pages_copy(st["k_pages"], st["v_pages"], st["moves"])
        return {"table": table, "refs": st["refs"], "len": st["seq_len"], "moves": st["moves"], "granted": st["granted"],
                "k": st["k_pages"], "v": st["v_pages"]}
    table, refs = table.clone(), st["refs"].clone()
    vico.vico_pages_free(table, refs, st["first"], st["last"], P)
    vico.vico_pages_compact(table, refs, st["moves"], st["count"], st["workspace"])
    vico.vico_pages_copy(st["k_pages"], st["v_pages"], st["moves"], count=st["count"])
    return {"table": table, "refs": refs, "moves": st["moves"], "count": st["count"], "k": st["k_pages"], "v": st["v_pages"]}


def _slots(table_row, pos, page):
    """Token slots of the pool, pages one after the other, for positions of a sequence."""
    return table_row[pos // page].long() * page + pos % page


def _held(table, rows, pool, sign):
    """What the entries of some rows (a [rows, pages] mask) add to the pages' reference counts."""
    at = torch.where(rows & (table >= 0), table, pool).long().flatten()
    return sign * torch.zeros(pool + 1, dtype=torch.int32, device=DEV).scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:pool]


def _copy_pages(st, src, dst):
    """Pages src to pages dst in every layer; a negative source stands for no move."""
    real = (src >= 0).nonzero().flatten()
    src, dst = src[real].long(), dst[real].long()
    for x in (st["k_pages"], st["v_pages"]):
        x[:, dst] = x[:, src]


def _run_plain(st):
    case, kind = st["case"], st["kind"]
    Hq, Hkv, D = HEADS[case["model"]]
    P, table = case["page"], st["table"]
    if kind == "attend":
        return _plain_attend(st)
    if kind == "append":
        at = torch.cat([_slots(table[i], torch.arange(h, h + n, device=DEV), P) for i, (n, h) in enumerate(zip(st["n"], st["h"]))])
        st["k_pages"].view(-1, Hkv, D)[at] = st["k"]
        st["v_pages"].view(-1, Hkv, D)[at] = st["v"]
        return {"k": st["k_pages"], "v": st["v_pages"]}
    pool, refs = st["refs"].shape[0], st["refs"]
    rows, width = table.shape
    col = torch.arange(width, device=DEV)
    if kind == "branch":
        parent, length = st["parent"].long(), st["seq_len"]
        anew = (parent != torch.arange(rows, device=DEV))[:, None].expand(rows, width)
        forked = torch.where(col < ((length[parent] + P - 1) // P)[:, None], table[parent], -1)
        new = torch.where(anew, forked, table)
        refs += _held(table, anew, pool, -1) + _held(new, anew, pool, 1)
        length.copy_(length[parent])
        n = st["q_start"][1:] - st["q_start"][:-1]
        j0, j1 = (length // P)[:, None], ((length + n + P - 1) // P)[:, None]
        owned = (new >= 0) & (refs[new.clamp(min=0).long()] == 1)
        wants = (col >= j0) & (col < j1) & (n > 0)[:, None] & ~owned
        fits = j1[:, 0] <= width
        wants &= fits[:, None]
        need = wants.sum(1)
        free = refs == 0
        granted = fits & ((need == 0) | (need.cumsum(0) <= free.sum()))
        wants &= granted[:, None]
        rank = wants.flatten().cumsum(0).view(rows, width) - 1
        order = torch.argsort(~free, stable=True).to(torch.int32)            # the free pages first, lowest first
        fresh = order[rank.clamp(min=0, max=pool - 1)]
        shared = wants & (new >= 0)
        moved = shared & (col == j0) & (length % P != 0)[:, None]
        src = torch.where(moved, new, -1).amax(1)
        dst = torch.where(moved, fresh, -1).amax(1)
        refs += _held(new, shared, pool, -1) + _held(fresh, wants, pool, 1)
        table.copy_(torch.where(wants, fresh, new))
        st["moves"].copy_(torch.stack([src, dst], 1))
        st["granted"].copy_(granted)
        _copy_pages(st, src, dst)
        return {"table": table, "refs": refs, "len": length, "moves": st["moves"], "granted": st["granted"],
                "k": st["k_pages"], "v": st["v_pages"]}
    j0, j1 = ((st["first"] + P - 1) // P)[:, None], (st["last"] // P)[:, None]
    gone = (col >= j0) & (col < j1)
    refs = refs + _held(table, gone, pool, -1)
    table = torch.where(gone, -1, table)
    used = refs > 0
    n_used = used.sum()
    page = torch.arange(pool, device=DEV)
    src = torch.argsort(~(used & (page >= n_used)), stable=True)               # sources first, lowest first
    dst = torch.argsort(~(~used & (page < n_used)), stable=True)
    m = (used & (page >= n_used)).sum()
    k = torch.arange(pool // 2, device=DEV)
    src, dst = (torch.where(k < m, x[:pool // 2], -1).to(torch.int32) for x in (src, dst))
    to = torch.cat([page, page[:1]]).to(torch.int32)                           # a last entry for the moves that are none
    to[torch.where(src >= 0, src, pool).long()] = dst
    table = torch.where(table >= 0, to[table.clamp(min=0).long()], -1)
    taken = torch.cat([refs, refs[:1]])
    taken[torch.where(dst >= 0, dst, pool).long()] = refs[src.clamp(min=0).long()]
    taken[torch.where(src >= 0, src, pool).long()] = 0
    _copy_pages(st, src, dst)
    return {"table": table, "refs": taken[:pool], "moves": torch.stack([src, dst], 1), "count": m.to(torch.int32).view(1),
            "k": st["k_pages"], "v": st["v_pages"]}


def _plain_attend(st):
    case = st["case"]
    Hq, Hkv, D = HEADS[case["model"]]
    g, P = Hq // Hkv, case["page"]
    k_all, v_all = st["k_pages"].view(-1, Hkv, D), st["v_pages"].view(-1, Hkv, D)
    outs, lses, row0 = [], [], 0
    for b, (n, h) in enumerate(zip(st["n"], st["h"])):
        sink, first = _spans(case, n, h)
        pos = torch.cat([torch.arange(sink, device=DEV), torch.arange(first, h + n, device=DEV)])
        at = _slots(st["table"][b], pos, P)
        k, v = k_all[at].transpose(0, 1).float(), v_all[at].transpose(0, 1).float()            # [Hkv, keys, D]
        q = st["q"][row0:row0 + n].float().view(n, Hkv, g, D).permute(1, 2, 0, 3).reshape(Hkv, g * n, D)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(D ** -0.5).view(Hkv, g, n, -1)
        s = s.masked_fill_(pos > h + torch.arange(n, device=DEV)[:, None], -torch.inf).view(Hkv, g * n, -1)
        m = s.amax(-1, keepdim=True)
        p = s.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v.contiguous()) / total
        outs.append(o.view(Hkv, g, n, D).permute(2, 0, 1, 3).reshape(n, Hq, D).to(torch.bfloat16))
        lses.append((m + total.log()).view(Hq, n))
        row0 += n
    return {"out": torch.cat(outs), "lse": torch.cat(lses, 1) if case["lse"] else None}


# ---------------------------------------------------------------- the definition, in 64 bits where numbers are computed

def exact(case, seed):
    kind = case["kind"]
    return {"attend": _exact_attend, "append": _exact_append, "branch": _exact_branch, "compact": _exact_compact}[kind](
        case, prepare(case, seed))


def _exact_attend(case, st):
    Hq, Hkv, D = HEADS[case["model"]]
    P, n_all, h_all = case["page"], st["n"], st["h"]
    out = torch.empty(sum(n_all), Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(Hq, sum(n_all), dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, h) in enumerate(zip(n_all, h_all)):
        keys = [p for p in range(h + n) if p < case["sink"] or case["window"] < 0 or p >= h - case["window"]]
        wanted = torch.tensor(sorted({p // P for p in keys}), device=DEV)
        ids = st["table"][b][wanted].long()
        pos = (wanted[:, None] * P + torch.arange(P, device=DEV)).flatten()
        listed_keys = torch.zeros(int(wanted[-1] + 1) * P, dtype=torch.bool)
        listed_keys[keys] = True
        take = listed_keys.to(DEV)[pos]
        k, v, pos = (x[take] for x in (st["k_pages"][ids].flatten(0, 1), st["v_pages"][ids].flatten(0, 1), pos))
        hidden = pos[None] > h + torch.arange(n, device=DEV)[:, None]
        for head in range(Hq):
            kh, vh = k[:, head * Hkv // Hq].double(), v[:, head * Hkv // Hq].double()
            s = (st["q"][at:at + n, head].double() @ kh.T.contiguous()) / math.sqrt(D)
            s[hidden] = -math.inf
            lse[head, at:at + n] = torch.logsumexp(s, 1)
            out[at:at + n, head] = torch.exp(s - lse[head, at:at + n, None]) @ vh.contiguous()
        at += n
    return {"out": out, "lse": lse if case["lse"] else None}


def _exact_append(case, st):
    P, at, table = case["page"], 0, st["table"].tolist()
    for b, (n, h) in enumerate(zip(st["n"], st["h"])):
        p, end = h, h + n
        while p < end:         # a page at a time
            m = min(P - p % P, end - p)
            page = table[b][p // P]
            for x, y in ((st["k_pages"], st["k"]), (st["v_pages"], st["v"])):
                x[page, p % P:p % P + m] = y[at:at + m]
            p, at = p + m, at + m
    return {"k": st["k_pages"], "v": st["v_pages"]}


def _moved(st, moves):
    k, v = st["k_pages"].clone(), st["v_pages"].clone()
    for a, b in moves:
        if a >= 0:
            k[:, b], v[:, b] = st["k_pages"][:, a], st["v_pages"][:, a]
    return {"k": k, "v": v}


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _exact_branch(case, st):
    P = case["page"]
    before, length, parent = st["table"].tolist(), st["seq_len"].tolist(), st["parent"].tolist()
    start, refs = st["q_start"].tolist(), st["refs"].tolist()
    table, lens, width = [list(r) for r in before], list(length), len(before[0])
    for b, p in enumerate(parent):
        if p == b:
            continue
        for e in before[b]:
            if e >= 0:
                refs[e] -= 1
        keep = _pages(length[p], P)
        table[b], lens[b] = before[p][:keep] + [-1] * (width - keep), length[p]
        for e in table[b]:
            if e >= 0:
                refs[e] += 1
    at_first, free = list(refs), [i for i, x in enumerate(refs) if x == 0]
    left, moves, granted = len(free), [], []
    for b in range(len(table)):
        n, h = start[b + 1] - start[b], lens[b]
        span = range(h // P, _pages(h + n, P)) if n else range(0)
        want = [j for j in span if j < width and not (table[b][j] >= 0 and at_first[table[b][j]] == 1)]
        ok = (not n or span[-1] < width) and (not want or len(want) <= left)
        left -= len(want)
        granted.append(int(ok))
        moves.append((-1, -1))
        for j in want if ok else []:
            old, new = table[b][j], free.pop(0)
            table[b][j], refs[new] = new, refs[new] + 1
            if old >= 0:
                refs[old] -= 1
                if j == h // P and h % P:
                    moves[b] = (old, new)
    return {"table": _int(table), "refs": _int(refs), "len": _int(lens), "moves": _int(moves), "granted": _int(granted),
            **_moved(st, moves)}


def _exact_compact(case, st):
    P = case["page"]
    table, refs = st["table"].tolist(), st["refs"].tolist()
    for row, a, b in zip(table, st["first"].tolist(), st["last"].tolist()):
        for j in range(len(row)):
            if j * P >= a and (j + 1) * P <= b and row[j] >= 0:
                refs[row[j]] -= 1
                row[j] = -1
    used = sum(x > 0 for x in refs)
    holes = [i for i in range(used) if refs[i] <= 0]
    moves = [(a, holes[i]) for i, a in enumerate(a for a in range(used, len(refs)) if refs[a] > 0)]
    to = dict(moves)
    for a, b in moves:
        refs[b], refs[a] = refs[a], 0
    table = [[to.get(e, e) for e in row] for row in table]
    kv = _moved(st, moves)
    return {"table": _int(table), "refs": _int(refs), "moves": _int(moves + [(-1, -1)] * (len(refs) // 2 - len(moves))),
            "count": _int([len(moves)]), **kv}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    Hq, Hkv, D = HEADS[case["model"]]
    kind, P = case["kind"], case["page"]
    row = 4 * Hkv * D                                      # bytes of a token's key and value
    if kind in ("attend", "append"):
        n_all, h_all, table, _ = _sequence_layout(case)
        if kind == "append":
            return {"bytes": 2 * row * sum(n_all) + 12 * len(n_all), "flops": 0}
        nbytes = pairs = 0
        for n, h in zip(n_all, h_all):
            sink, first = _spans(case, n, h)
            keys = sink + h + n - first
            pairs += n * keys - n * (n - 1) // 2
            nbytes += keys * row + 4 * _pages(keys, P) + 12 + n * Hq * (4 * D + (4 if case["lse"] else 0))
        return {"bytes": nbytes, "flops": 4 * Hq * D * pairs}
    page = 2 * row * P * case["layers"]                    # a page moved: read and written in every layer
    if kind == "branch":
        h, n, parent, table, pool = _branch_layout(case)
        S = case["streams"]
        copied = sum(h[p] % P != 0 for p in parent[S:])
        entries = sum(_pages(h[p], P) + _pages(h[p] + x, P) for p, x in zip(parent[S:], n[S:]))
        return {"bytes": copied * page + 4 * entries + 4 * pool, "flops": 0}
    h, first, last, table, pool = _compact_layout(case)
    left = table.clone()
    for i, (a, b) in enumerate(zip(first, last)):
        left[i, _pages(a, P):max(b // P, _pages(a, P))] = -1
    left = left[left >= 0]
    moved = int((left >= left.numel()).sum())
    return {"bytes": moved * page + 8 * table.numel() + 8 * pool, "flops": 0}
