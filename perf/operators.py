"""Operators of the paged cache: attention of drafted token trees over pages, attention over selected pages, and the pages' upkeep.

A cache is a pool of pages k, v [layers, n_pages, Hkv, rows of a page, hd] that sequences share: table [S, max_pages] names a
sequence's pages in order (-1 = none), len [S] its rows, refs [n_pages] counts the table entries that name a page (0 = free).  New rows
(a token, a chain, a tree of drafts, the states of a block) of all sequences lie one behind the other, rows row_start[s] ..
row_start[s+1]-1 are those of sequence s, as q | k | v side by side, as a projection writes them.  Bit i of mask[t] says that row
t attends to the i-th new row of its sequence.  Heads and widths are those of the repository's workload configurations (32 heads of 128
without groups, 28 heads over 4, 4 heads of 64 in fp32) and generic ones (32 heads over 8, 16 over 4 of 64).
"""
import math
import random

import torch

own = False
DEV = "cuda"


def _case(name, kind, dtype="bf16", Hq=32, Hkv=8, hd=128, ps=64, S=1, lo=1024, hi=1024, nodes_lo=1, nodes_hi=1, shape="tree", n_sel=0, L=1, ragged=1):
    """lo, hi: rows cached for a sequence, nodes_lo, nodes_hi: its new rows; `ragged` seeds the sizes between them.  n_sel: pages
    that a kv head reads.  L: layers that the call is for."""
    c = dict(kind=kind, dtype=dtype, Hq=Hq, Hkv=Hkv, hd=hd, ps=ps, S=S, lo=lo, hi=hi, nodes_lo=nodes_lo, nodes_hi=nodes_hi,
             shape=shape, n_sel=n_sel, L=L, ragged=ragged)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One token of one conversation after 500 rows: latency.
        _case("one_token", "tree", lo=500, hi=500, ps=16),
        # Continuous batching, undrafted: 64 sequences of very different lengths, a token each.
        _case("one_token_64_sequences", "tree", ps=16, S=64, lo=64, hi=16384, ragged=5),
        # Drafted trees of 9 to 30 tokens of 8 sequences, grouped heads of the 28-head configuration.
        _case("trees_of_8_sequences", "tree", Hq=28, Hkv=4, ps=32, S=8, lo=300, hi=6000, nodes_lo=9, nodes_hi=30, ragged=2),
        # A tree of 63 tokens at the end of a document of 131000 rows.
        _case("tree_after_long_document", "tree", ps=64, lo=131001, hi=131001, nodes_lo=63, nodes_hi=63),
        # The draft graph of the headline configuration over pages: 32 states of a 32-token block, each sees the cache and itself.
        _case("states_of_a_block", "tree", Hq=32, Hkv=32, ps=64, lo=1024, hi=1024, nodes_lo=1024, nodes_hi=1024, shape="block"),
        # The fp32 configuration's heads, chains of drafts, pages that no tile divides.
        _case("fp32_chains", "tree", dtype="f32", Hq=4, Hkv=4, hd=64, ps=24, S=6, lo=64, hi=3000, nodes_lo=3, nodes_hi=13, shape="chain", ragged=3),
        # One token of a long conversation, 32 of about 520 pages read.
        _case("one_token_32_pages", "sparse", ps=64, lo=33333, hi=33333, n_sel=32),
        # Trees of up to 16 tokens of 16 long sequences, 64 pages each.
        _case("trees_64_pages", "sparse", ps=64, S=16, lo=5000, hi=65000, nodes_lo=5, nodes_hi=16, n_sel=64, ragged=4),
        # The summaries of 4 new prompts' pages.
        _case("summaries_of_prompts", "summary", ps=64, S=4, lo=9000, hi=50000, L=2, ragged=6),
        # Two continuations of one short prompt are forked and take their first accepted drafts: latency.
        _case("fork_two", "fork", ps=16, S=2, lo=37, hi=37, nodes_lo=8, nodes_hi=8, L=2),
        # 48 prompts are forked, every copy takes its accepted path in all 28 layers.
        _case("fork_48", "fork", Hq=28, Hkv=4, ps=64, S=48, lo=200, hi=2000, nodes_lo=12, nodes_hi=40, L=28, ragged=7),
        # Half of 40 sequences have ended: the pages of the others close ranks.
        _case("compact_40", "compact", ps=64, S=40, lo=500, hi=3000, L=8, ragged=8),
    ]


def _between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "sparse", "sparse", "summary", "fork", "compact"])
    Hq, Hkv, hd = rng.choice([(32, 8, 128), (28, 4, 128), (32, 32, 128), (16, 4, 64), (8, 2, 256), (6, 3, 80), (4, 4, 64), (16, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if dtype == "f32" and Hkv > 8:
        Hq, Hkv = 8, 4
    ps = rng.choice([16, 32, 64, 128, 1, 24, 57])
    S = _between(rng, 1, 24)
    hi = _between(rng, 1, max(64, 40000 // S))
    lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
    ragged = rng.randrange(1 << 30)
    if kind in ("tree", "sparse"):
        nodes_hi = _between(rng, 1, 80 if kind == "tree" else 24)
        shape = rng.choice(["tree", "chain", "full"])
        return _case(None, kind, dtype, Hq, Hkv, hd, ps if kind == "tree" else rng.choice([16, 32, 64, 100]), S, lo, hi, rng.randint(1, nodes_hi), nodes_hi, shape,
                     _between(rng, 3, 100) if kind == "sparse" else 0, 1, ragged)
    L = rng.randint(1, 6)
    if kind == "summary":
        return _case(None, kind, dtype, Hq, Hkv, hd, rng.choice([16, 32, 64, 128, 57]), S, lo, hi, L=L, ragged=ragged)
    ps = rng.choice([16, 32, 64, 128, 24, 57])
    hi = _between(rng, 2, max(8, min(4000, 1_500_000_000 // (2 * Hkv * hd * (4 if dtype == "f32" else 2) * L * max(2, S)))))
    lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
    nodes_hi = _between(rng, 1, 64)
    return _case(None, kind, dtype, Hq, Hkv, hd, ps, max(2, S), lo, hi, rng.randint(1, nodes_hi), nodes_hi, "tree", 0, L, ragged)


# ---- sizes, from the case alone --------------------------------------------------------------------------------------------


def _sizes(case):
    """Rows cached and new rows of every sequence, and each new row's bits (a list of Python integers a sequence)."""
    rng = random.Random(case["ragged"])
    lens = [_between(rng, case["lo"], case["hi"]) for _ in range(case["S"])]
    nodes = [rng.randint(case["nodes_lo"], case["nodes_hi"]) for _ in range(case["S"])]
    bits = []
    for n in nodes:
        if case["shape"] == "tree":          # a draft hangs under one of the eight before it
            rows = [1]
            for i in range(1, n):
                rows.append(rows[rng.randint(max(0, i - 8), i - 1)] | 1 << i)
        elif case["shape"] == "chain":
            rows = [(1 << i + 1) - 1 for i in range(n)]
        elif case["shape"] == "block":       # states of 32 tokens that see themselves
            rows = [((1 << 32) - 1) << 32 * (i // 32) & (1 << n) - 1 for i in range(n)]
        else:
            rows = [(1 << n) - 1] * n
        bits.append(rows)
    return lens, nodes, bits


def _pages(case, lens):
    return [-(-n // case["ps"]) for n in lens]


def _leaving(case):
    """compact: every second sequence has ended."""
    return [s for s in range(case["S"]) if s % 2 == 0]


def _kept(case, nodes, bits):
    """fork: the accepted node of every sequence and the new rows on its path."""
    rng = random.Random(case["ragged"] + 1)
    node = [rng.randrange(n) for n in nodes]
    return node, [bin(b[i]).count("1") for i, b in zip(node, bits)]


def work(case):
    lens, nodes, bits = _sizes(case)
    e, Hq, Hkv, hd, ps, L = 4 if case["dtype"] == "f32" else 2, case["Hq"], case["Hkv"], case["hd"], case["ps"], case["L"]
    pages, T = _pages(case, lens), sum(nodes)
    row = 2 * Hkv * hd * e
    if case["kind"] in ("tree", "sparse"):
        read = lens if case["kind"] == "tree" else [min(n, case["n_sel"] * ps) for n in lens]
        pairs = sum(n * r + sum(bin(b).count("1") for b in bs) for n, r, bs in zip(nodes, read, bits))
        nbytes, flops = row * (sum(read) + T) + 2 * T * Hq * hd * e, 4 * hd * Hq * pairs
        if case["kind"] == "sparse":
            nbytes += row * sum(pages) + 4 * Hkv * sum(min(p, case["n_sel"]) for p in pages)
            flops += 4 * hd * Hq * sum(n * p for n, p in zip(nodes, pages))
        return {"bytes": nbytes, "flops": flops}
    if case["kind"] == "summary":
        return {"bytes": L * (row // 2 * sum(lens) + row * sum(pages)), "flops": L * Hkv * hd * 2 * sum(lens)}
    if case["kind"] == "fork":
        kept = _kept(case, nodes, bits)[1]
        return {"bytes": 2 * L * row * (sum(n % ps for n in lens) + sum(kept)) + 8 * sum(pages), "flops": 0}
    gone = _leaving(case)
    left = sum(pages) - sum(pages[s] for s in gone)
    order = [s for s in range(case["S"]) for _ in range(pages[s])]      # pages lie in the pool as the sequences came
    moved = sum(1 for s in order[left:] if s not in gone)
    return {"bytes": 2 * L * row * ps * moved + 8 * sum(pages), "flops": 0}


# ---- inputs ----------------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    lens, nodes, bits = _sizes(case)
    pages, T, S, L = _pages(case, lens), sum(nodes), case["S"], case["L"]
    Hq, Hkv, hd, ps, kind = case["Hq"], case["Hkv"], case["hd"], case["ps"], case["kind"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    used, extra = sum(pages), -(-max(nodes) // ps) + 1
    n_seqs = 2 * S if kind == "fork" else S
    n_pages = used + (S * (extra + 1) if kind == "fork" else 3)
    max_pages = max(pages) + extra
    # in a pool that has been in use a sequence's pages lie anywhere; compact meets them as the prompts wrote them
    ids = torch.arange(n_pages) if kind == "compact" else torch.randperm(n_pages, generator=host)
    table, refs = torch.full((n_seqs, max_pages), -1, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32)
    at = 0
    for s, n in enumerate(pages):
        table[s, :n] = ids[at:at + n]
        at += n
    refs[ids[:used]] = 1
    length = torch.tensor(lens + [0] * (n_seqs - S), dtype=torch.int32)
    # one array holds refs, table and len, so that a program can keep or restore them together
    ints = torch.cat([refs, table.reshape(-1), length]).to(DEV)
    st = dict(case=case, S=S, max_rows=max(nodes), max_pages=max_pages, n_pages=n_pages, n_seqs=n_seqs, ints=ints, ints0=ints.clone(),
              refs=ints[:n_pages], table=ints[n_pages:n_pages + n_seqs * max_pages].view(n_seqs, max_pages), len=ints[n_pages + n_seqs * max_pages:],
              dtype=dt, scale=1.0 / math.sqrt(hd))
    for name in ("k", "v"):
        st[name] = torch.randn((L, n_pages, Hkv, ps, hd), generator=gen, device=DEV, dtype=dt)
    if kind in ("sparse", "summary"):
        st["summary"] = torch.zeros((L, n_pages, Hkv, 2, hd), device=DEV, dtype=dt)
        if kind == "sparse":                 # of pages in use; the last one of a sequence is filled in part
            _summaries(st)
    starts = [0]
    for n in nodes:
        starts.append(starts[-1] + n)
    st["row_start"] = torch.tensor(([0] * S if kind == "fork" else []) + starts, dtype=torch.int32, device=DEV)
    qkv = torch.randn((L, T, Hq + 2 * Hkv, hd), generator=gen, device=DEV, dtype=dt)
    if kind == "fork":
        st["rows_k"], st["rows_v"] = qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        st["src"] = torch.arange(S, dtype=torch.int32, device=DEV)
        st["dst"] = torch.arange(S, 2 * S, dtype=torch.int32, device=DEV)
        st["node"] = torch.tensor([-1] * S + _kept(case, nodes, bits)[0], dtype=torch.int32, device=DEV)
    else:
        st["q"], st["nk"], st["nv"] = qkv[0, :, :Hq], qkv[0, :, Hq:Hq + Hkv], qkv[0, :, Hq + Hkv:]
    if kind == "compact":
        st["gone"] = torch.tensor(_leaving(case), dtype=torch.int32, device=DEV)
    words = -(-max(nodes) // 64)
    flat = [[b >> 64 * w & (1 << 64) - 1 for w in range(words)] for rows in bits for b in rows]
    st["mask"] = torch.tensor([[x - (1 << 64) if x >> 63 else x for x in r] for r in flat], dtype=torch.int64, device=DEV)
    return st


# ---- plain forms -----------------------------------------------------------------------------------------------------------


def _new_rows(st):
    """Index [S, most rows] of every sequence's new rows, and which of them there are."""
    start = st["row_start"].long()
    i = torch.arange(st["max_rows"], device=DEV)
    there = i[None] < (start[1:] - start[:-1])[:, None]
    return torch.where(there, start[:-1, None] + i[None], 0), there


def _row_bits(st, rows):
    """[S, rows, most rows] truth values: whether a row attends to a new row of its sequence."""
    i = torch.arange(st["max_rows"], device=DEV)
    return (st["mask"][rows][..., i // 64] >> (i % 64) & 1).bool()


def _attention(st, slots):
    """slots [S, Hkv, n]: the pages that are read, -1 = none."""
    c = st["case"]
    S, Hq, Hkv, hd, ps = c["S"], c["Hq"], c["Hkv"], c["hd"], c["ps"]
    g, n = Hq // Hkv, st["max_rows"]
    page = torch.gather(st["table"].long()[:, None].expand(S, Hkv, -1), 2, slots.clamp(min=0))
    head = torch.arange(Hkv, device=DEV)[None, :, None]
    pos = slots[..., None] * ps + torch.arange(ps, device=DEV)
    seen = ((slots[..., None] >= 0) & (pos < st["len"].long()[:, None, None, None])).reshape(S, Hkv, 1, -1)
    k = st["k"][0, page.clamp(min=0), head].float().reshape(S, Hkv, -1, hd)
    v = st["v"][0, page.clamp(min=0), head].float().reshape(S, Hkv, -1, hd)
    rows, there = _new_rows(st)
    q = st["q"][rows].float().reshape(S, n, Hkv, g, hd).permute(0, 2, 1, 3, 4).reshape(S, Hkv, n * g, hd)
    nk = st["nk"][rows].float().permute(0, 2, 1, 3)
    nv = st["nv"][rows].float().permute(0, 2, 1, 3)
    bits = (_row_bits(st, rows) & there[:, None]).repeat_interleave(g, 1)[:, None]
    low = torch.tensor(-math.inf, device=DEV)
    a = torch.where(seen, torch.matmul(q, k.transpose(2, 3)) * st["scale"], low)
    b = torch.where(bits, torch.matmul(q, nk.transpose(2, 3)) * st["scale"], low)
    top = torch.maximum(a.amax(3, keepdim=True), b.amax(3, keepdim=True)).clamp(min=-3e38)
    a, b = torch.exp(a - top), torch.exp(b - top)
    total = a.sum(3, keepdim=True) + b.sum(3, keepdim=True)
    o = (torch.matmul(a, v) + torch.matmul(b, nv)) / torch.where(total > 0, total, 1.0)
    o = o.reshape(S, Hkv, n, g, hd).permute(0, 2, 1, 3, 4).reshape(S * n, Hq, hd)
    place = torch.where(there, rows, st["q"].shape[0]).reshape(-1)
    out = torch.zeros((st["q"].shape[0] + 1, Hq, hd), dtype=st["dtype"], device=DEV)
    out[place] = o.to(st["dtype"])
    return out[:-1]


def _used_pages(st):
    return (st["len"].long() + st["case"]["ps"] - 1) // st["case"]["ps"]


def _all_slots(st):
    j = torch.arange(st["max_pages"], device=DEV)
    return torch.where(j[None] < _used_pages(st)[:, None], j[None], -1)[:, None].expand(-1, st["case"]["Hkv"], -1)


def _summaries(st):
    """Least and greatest value of each channel over the rows of each page in use."""
    c = st["case"]
    slots = _all_slots(st)[:, 0]
    page = torch.where(slots >= 0, st["table"].long(), -1)
    rows = torch.where(slots >= 0, st["len"].long()[:, None] - slots * c["ps"], 0).clamp(0, c["ps"])
    rows_of = torch.zeros(st["n_pages"] + 1, dtype=torch.long, device=DEV)
    rows_of[page.reshape(-1)] = rows.reshape(-1)         # -1: the entry behind the last page
    there = (torch.arange(c["ps"], device=DEV)[None] < rows_of[:-1, None])[None, :, None, :, None]
    lo = torch.where(there, st["k"], math.inf).amin(3)
    hi = torch.where(there, st["k"], -math.inf).amax(3)
    in_use = (rows_of[:-1] > 0)[None, :, None, None, None]
    st["summary"].copy_(torch.where(in_use, torch.stack([lo, hi], 3), st["summary"]))


def _select(st):
    """The pages of the highest bounds.  The bounds are summed in 64 bits: which of two near ones is higher must not depend on the order of a sum."""
    c = st["case"]
    S, Hkv, g, n = c["S"], c["Hkv"], c["Hq"] // c["Hkv"], st["max_rows"]
    rows, there = _new_rows(st)
    q = st["q"][rows].double().reshape(S, n, Hkv, g, c["hd"]).permute(0, 2, 1, 3, 4).reshape(S, Hkv, n * g, c["hd"])
    s = st["summary"][0, st["table"].long().clamp(min=0)].double().permute(0, 2, 3, 4, 1)
    bound = torch.matmul(q.clamp(min=0), s[:, :, 1]) + torch.matmul(q.clamp(max=0), s[:, :, 0])
    bound = torch.where(there.repeat_interleave(g, 1)[:, None, :, None], bound, -math.inf).amax(2)
    j, used = torch.arange(st["max_pages"], device=DEV)[None], _used_pages(st)[:, None]
    always = (j < 1) | (j >= used - 1)
    bound = torch.where(always[:, None], math.inf, bound)
    bound = torch.where((j < used)[:, None], bound, -math.inf)
    best = torch.sort(bound, dim=2, descending=True, stable=True).indices[..., :c["n_sel"]]
    best = torch.where(best < used[:, None], best, st["max_pages"]).sort(2).values
    best = torch.nn.functional.pad(best, (0, c["n_sel"] - best.shape[2]), value=st["max_pages"])
    return torch.where(best < st["max_pages"], best, -1).int()


def _free_pages(st):
    return torch.argsort((st["refs"] > 0).int(), stable=True)


def _free(st, seqs):
    seqs = seqs.long()
    slots = _all_slots(st)[:, 0][seqs]
    page = torch.where(slots >= 0, st["table"][seqs].long(), 0)
    st["refs"].index_add_(0, page.reshape(-1), -(slots >= 0).int().reshape(-1))
    st["table"][seqs] = torch.where(slots >= 0, -1, st["table"][seqs])
    st["len"][seqs] = 0


def _fork(st):
    c = st["case"]
    src, dst = st["src"].long(), st["dst"].long()
    n = st["len"][src].long()
    full, rest = n // c["ps"], n % c["ps"]
    new = _free_pages(st)[(torch.cumsum((rest > 0).long(), 0) - 1).clamp(min=0)]
    j = torch.arange(st["max_pages"], device=DEV)[None]
    row = st["table"][src].long()
    shared = j < full[:, None]
    st["refs"].index_add_(0, torch.where(shared, row, 0).reshape(-1), shared.int().reshape(-1))
    last = torch.where(rest > 0, row.gather(1, full[:, None])[:, 0], row[:, 0])
    to = torch.where(rest > 0, new, last)                # without a page in part: onto itself
    in_use = (torch.arange(c["ps"], device=DEV) < rest[:, None])[None, :, None, :, None]
    st["k"][:, to] = torch.where(in_use, st["k"][:, last], st["k"][:, to])
    st["v"][:, to] = torch.where(in_use, st["v"][:, last], st["v"][:, to])
    st["refs"].index_add_(0, to, (rest > 0).int())
    at_end = (j == full[:, None]) & (rest > 0)[:, None]
    st["table"][dst] = torch.where(shared, row, torch.where(at_end, to[:, None], -1)).int()
    st["len"][dst] = n.int()


def _append(st):
    c = st["case"]
    ps, n = c["ps"], st["max_rows"]
    rows, there = _new_rows(st)
    node = st["node"].long()
    at = rows.gather(1, node.clamp(min=0)[:, None])
    kept = _row_bits(st, at)[:, 0] & there & (node >= 0)[:, None]
    had, length = _used_pages(st), st["len"].long()
    length2 = length + kept.sum(1)
    more = (length2 + ps - 1) // ps - had
    free = _free_pages(st)
    j = torch.arange(st["max_pages"], device=DEV)[None]
    rank = (torch.cumsum(more, 0) - more)[:, None] + j - had[:, None]
    fresh = (j >= had[:, None]) & (j < (had + more)[:, None])
    page = free[torch.where(fresh, rank, 0)]
    st["table"].copy_(torch.where(fresh, page, st["table"].long()))
    st["refs"].index_add_(0, page.reshape(-1), fresh.int().reshape(-1))
    # rows off the path: row 0 of their sequence, which stays what it is, is written again
    pos = torch.where(kept, length[:, None] + torch.cumsum(kept.long(), 1) - 1, 0)
    to, off = st["table"].long().gather(1, pos // ps), pos % ps
    for_all = kept[None, :, :, None, None]
    st["k"][:, to, :, off] = torch.where(for_all, st["rows_k"][:, rows], st["k"][:, to, :, off].permute(2, 0, 1, 3, 4)).permute(1, 2, 0, 3, 4)
    st["v"][:, to, :, off] = torch.where(for_all, st["rows_v"][:, rows], st["v"][:, to, :, off].permute(2, 0, 1, 3, 4)).permute(1, 2, 0, 3, 4)
    st["len"].copy_(length2)


def _compact(st):
    used = st["refs"] > 0
    i = torch.arange(st["n_pages"], device=DEV)
    count = used.sum()
    come, go = (~used & (i < count)).nonzero()[:, 0], (used & (i >= count)).nonzero()[:, 0]
    st["k"][:, come] = st["k"][:, go]
    st["v"][:, come] = st["v"][:, go]
    name = i.clone()
    name[go] = come
    st["refs"][come] = st["refs"][go]
    st["refs"][go] = 0
    st["table"].copy_(torch.where(st["table"] >= 0, name[st["table"].long().clamp(min=0)], -1))
    return count.int().reshape(1)


# ---- the framework's calls -------------------------------------------------------------------------------------------------


def _cache(st):
    """The handle on the pool that a program makes once."""
    if "cache" not in st:
        from paper_2509_18085_amd import spiffy as sp
        c = st["case"]
        cfg = sp.make_cfg(d=c["Hq"] * c["hd"], n_q_heads=c["Hq"], n_kv_heads=c["Hkv"], head_dim=c["hd"], ffn=8, vocab=2, mask_id=1, dtype=st["dtype"])
        st["cache"] = sp.PagedCache(cfg, st["k"], st["v"], st["refs"], st["table"], st["len"],
                                    summary=st.get("summary"))
    return st["cache"]


def _run_own(st):
    cache, kind = _cache(st), st["case"]["kind"]
    if kind == "tree":
        return cache.attend(0, st["q"], st["nk"], st["nv"], st["row_start"], st["max_rows"], mask=st["mask"], scale=st["scale"])
    if kind == "sparse":
        sel = cache.select(0, st["q"], st["row_start"], st["max_rows"], st["case"]["n_sel"], keep_first=1, keep_last=1)
        return sel, cache.attend(0, st["q"], st["nk"], st["nv"], st["row_start"], st["max_rows"], mask=st["mask"], selected=sel, scale=st["scale"])
    if kind == "summary":
        cache.summarize()
        return st["summary"]
    if kind == "fork":
        cache.free(st["dst"])                # the copies of the pass before
        cache.fork(st["src"], st["dst"])
        cache.append(st["rows_k"], st["rows_v"], st["row_start"], mask=st["mask"], node=st["node"])
        return st["k"], st["v"], st["refs"], st["table"], st["len"]
    st["ints"].copy_(st["ints0"])            # as it was before the sequences ended
    cache.free(st["gone"])
    return cache.compact(), st["k"], st["v"], st["refs"], st["table"], st["len"]


def _run_plain(st):
    kind = st["case"]["kind"]
    if kind == "tree":
        return _attention(st, _all_slots(st))
    if kind == "sparse":
        sel = _select(st)
        return sel, _attention(st, sel.long())
    if kind == "summary":
        _summaries(st)
        return st["summary"]
    if kind == "fork":
        _free(st, st["dst"])
        _fork(st)
        _append(st)
        return st["k"], st["v"], st["refs"], st["table"], st["len"]
    st["ints"].copy_(st["ints0"])
    _free(st, st["gone"])
    return _compact(st), st["k"], st["v"], st["refs"], st["table"], st["len"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------


def _exact_attention(st, case, lens, nodes, bits, chosen):
    """A sequence and a kv head at a time: the rows that are read, one behind the other, then a softmax over them."""
    Hq, Hkv, hd, ps = case["Hq"], case["Hkv"], case["hd"], case["ps"]
    g, out, t0 = Hq // Hkv, [], 0
    table = st["table"].cpu()
    for s, (length, n) in enumerate(zip(lens, nodes)):
        see = torch.tensor([[b >> i & 1 for i in range(n)] for b in bits[s]], dtype=torch.bool, device=DEV)
        heads = []
        for h in range(Hkv):
            pages = range(-(-length // ps)) if chosen is None else chosen[s][h]
            where = [(int(table[s, j]), min(ps, length - j * ps)) for j in pages]
            flat = torch.tensor([p * ps for p, _ in where], dtype=torch.long)[:, None] + torch.arange(ps)
            keep = torch.arange(ps)[None] < torch.tensor([m for _, m in where], dtype=torch.long)[:, None]
            flat = flat[keep].to(DEV)
            k = torch.cat([st["k"][0, flat // ps, h, flat % ps].double(), st["nk"][t0:t0 + n, h].double()])
            v = torch.cat([st["v"][0, flat // ps, h, flat % ps].double(), st["nv"][t0:t0 + n, h].double()])
            open_ = torch.cat([torch.ones((n, len(flat)), dtype=torch.bool, device=DEV), see], 1)
            parts = []
            for i in range(g):
                x = (st["q"][t0:t0 + n, h * g + i].double() @ k.T * st["scale"]).masked_fill(~open_, -math.inf)
                parts.append(torch.softmax(x, 1) @ v)
            heads.append(torch.stack(parts, 1))
        out.append(torch.cat(heads, 1))
        t0 += n
    return torch.cat(out)


def _exact_selection(st, case, lens, nodes):
    Hkv, ps, g, t0, chosen = case["Hkv"], case["ps"], case["Hq"] // case["Hkv"], 0, []
    for s, (length, n) in enumerate(zip(lens, nodes)):
        used, lists = -(-length // ps), []
        pages = st["table"][s, :used].long()
        for h in range(Hkv):
            lo, hi = st["summary"][0, pages, h, 0].double(), st["summary"][0, pages, h, 1].double()
            best = torch.full((used,), -math.inf, dtype=torch.float64, device=DEV)
            for q in st["q"][t0:t0 + n, h * g:(h + 1) * g].double().reshape(n * g, -1):
                best = torch.maximum(best, torch.maximum(q * lo, q * hi).sum(1))
            value = best.tolist()
            value[0] = value[used - 1] = math.inf
            order = sorted(range(used), key=lambda j: (-value[j], j))
            lists.append(sorted(order[:case["n_sel"]]))
        chosen.append(lists)
        t0 += n
    return chosen


def _exact_pages(st, case, lens, nodes, bits):
    """The pages' bookkeeping one page at a time in Python, and the moves of rows that follow from it."""
    ps, S = case["ps"], case["S"]
    refs, table, length = st["refs"].tolist(), st["table"].tolist(), st["len"].tolist()
    pools, first = [st["k"].double(), st["v"].double()], []
    if case["kind"] == "fork":
        for s in range(S):
            full, rest = divmod(length[s], ps)
            for j in range(full):
                refs[table[s][j]] += 1
                table[S + s][j] = table[s][j]
            if rest:
                new = refs.index(0)
                refs[new], table[S + s][full] = 1, new
                for pool in pools:
                    pool[:, new, :, :rest] = pool[:, table[s][full], :, :rest]
            length[S + s] = length[s]
        node, t0 = _kept(case, nodes, bits)[0], 0
        for s in range(S):
            for i in range(nodes[s]):
                if bits[s][node[s]] >> i & 1:
                    j, off = divmod(length[S + s], ps)
                    if not off:
                        table[S + s][j] = refs.index(0)
                        refs[table[S + s][j]] = 1
                    for pool, rows in zip(pools, (st["rows_k"], st["rows_v"])):
                        pool[:, table[S + s][j], :, off] = rows[:, t0 + i].double()
                    length[S + s] += 1
            t0 += nodes[s]
    else:
        for s in _leaving(case):
            for j in range(-(-length[s] // ps)):
                refs[table[s][j]] -= 1
                table[s][j] = -1
            length[s] = 0
        used = [p for p, r in enumerate(refs) if r]
        low, high = [p for p in range(len(used)) if not refs[p]], [p for p in used if p >= len(used)]
        name = dict(zip(high, low))
        for pool in pools:
            pool[:, low] = pool[:, high]
        for a, b in name.items():
            refs[b], refs[a] = refs[a], 0
        table = [[name.get(p, p) for p in row] for row in table]
        first = [torch.tensor([len(used)], dtype=torch.int32)]
    return tuple(first + pools + [torch.tensor(x, dtype=torch.int32) for x in (refs, table, length)])


def exact(case, seed):
    st = prepare(case, seed)
    lens, nodes, bits = _sizes(case)
    if case["kind"] == "tree":
        return _exact_attention(st, case, lens, nodes, bits, None)
    if case["kind"] == "sparse":
        chosen = _exact_selection(st, case, lens, nodes)
        lists = [[row + [-1] * (case["n_sel"] - len(row)) for row in heads] for heads in chosen]
        return torch.tensor(lists, dtype=torch.int32), _exact_attention(st, case, lens, nodes, bits, chosen)
    if case["kind"] == "summary":
        out = st["summary"].double()
        table = st["table"].tolist()
        for s, n in enumerate(lens):
            for j in range(-(-n // case["ps"])):
                rows = st["k"][:, table[s][j], :, :min(case["ps"], n - j * case["ps"])].double()
                out[:, table[s][j], :, 0] = rows.min(2).values
                out[:, table[s][j], :, 1] = rows.max(2).values
        return out
    return _exact_pages(st, case, lens, nodes, bits)
