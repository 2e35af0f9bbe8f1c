"""The paged cache against its plain form (tests/paged_reference.py): attention of drafted trees, selection of pages, and the pages' upkeep."""
import ctypes as C
import math
import os
import random
import subprocess
import sys

import numpy as np
import pytest
import torch

from paged_reference import PlainCache, Setup, mask_words, tree_rows
from paper_2509_18085_amd import spiffy as sp

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
gpu = pytest.mark.gpu


def _cfg(dtype, Hq, Hkv, hd):
    return sp.make_cfg(d=Hq * hd, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=hd, ffn=8, vocab=2, mask_id=1, dtype=dtype)


def _on_gpu(x, dtype):
    to = lambda t: None if t is None else t.to(DEV)
    return sp.PagedCache(_cfg(dtype, x.Hq, x.Hkv, x.hd), to(x.k), to(x.v), to(x.refs), to(x.table), to(x.len), to(x.summary))


def _close(got, want, dtype, n_keys, what):
    """Errors by arithmetic, relative to the largest |v| that a row can return (values are N(0,1): below 6).  fp32: a score is a sum of
    hd products (error below hd * 2^-24 of sum |q k| / sqrt(hd), some 1e-5 at most), a probability is off by that, and sums
    of n_keys terms in a tree of partial sums by far less than that again: 1e-4.  bf16: a probability is rounded by at most
    2^-8 of itself, so the sum of p v by at most 2^-8 max|v|, and the result by 2^-8 of itself."""
    far = (got.double().cpu() - want).abs()
    top = 6.0
    tol = 1e-4 * top if dtype == F32 else 2.0 ** -8 * top + 2.0 ** -8 * want.abs() + 1e-3
    assert not torch.isnan(got).any(), what
    bad = far > tol
    assert not bad.any(), (what, float(far.max()), int(bad.sum()), bad.nonzero()[:4].tolist())
    # and on average a tenth of that: roundings are not all at their worst and of one sign
    scale = want.pow(2).mean().sqrt().clamp(min=1e-30)
    assert (far.pow(2).mean().sqrt() / scale) < (2e-5 if dtype == F32 else 6e-3), what


# dtype, Hq, Hkv, hd, rows of a page, lengths, new rows
ATTEND = [
    (BF, 8, 2, 128, 16, [37, 0, 160, 5], [1, 1, 1, 1]),
    (BF, 8, 2, 128, 64, [500, 64, 63, 65, 1], [13, 1, 0, 30, 7]),
    (BF, 4, 4, 128, 32, [700, 31], [64, 65]),
    (BF, 7, 1, 128, 16, [1500, 3], [20, 2]),
    (BF, 28, 4, 128, 128, [300], [25]),
    (BF, 4, 1, 64, 16, [200, 1], [9, 33]),
    (BF, 8, 2, 64, 48, [200, 95], [1, 4]),
    (BF, 2, 1, 256, 16, [130, 17], [11, 1]),
    (BF, 4, 2, 256, 64, [300], [40]),
    (BF, 6, 3, 80, 24, [100, 24, 23], [5, 17, 1]),
    (BF, 2, 2, 8, 1, [70, 3], [3, 1]),
    (BF, 3, 1, 248, 57, [58, 57], [6, 2]),
    (BF, 16, 1, 128, 64, [2000], [1]),
    (BF, 6, 1, 80, 24, [333, 70, 2], [40, 11, 13]),
    (BF, 4, 1, 40, 7, [150, 0], [30, 3]),
    (BF, 2, 1, 64, 5, [3000, 1], [50, 64]),
    (BF, 2, 2, 128, 16, [5000, 40], [300, 128]),
    (BF, 16, 1, 128, 1, [900], [8]),
    (F32, 4, 4, 64, 24, [300, 7, 0], [8, 3, 2]),
    (F32, 8, 2, 128, 16, [500, 33], [1, 21]),
    (F32, 4, 1, 128, 64, [129], [70]),
    (F32, 2, 1, 256, 32, [90, 40], [3, 19]),
    (F32, 3, 3, 40, 5, [44, 1], [2, 18]),
    (F32, 5, 5, 16, 1, [17], [1]),
]


@gpu
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "-".join(str(x) for x in c[1:5]) + ("-f32" if c[0] == F32 else ""))
@pytest.mark.parametrize("kind", ["tree", "full", "random"])
def test_attention_of_trees(case, kind):
    dtype, Hq, Hkv, hd, ps, lens, nodes = case
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=len(lens) + hd, behind=2)
    words = -(-max(nodes) // 64)
    if kind == "tree":
        rows = x.tree()
    elif kind == "full":
        rows = None
    else:          # any bits, bits beyond the sequence's rows among them, and a row that attends to no new row
        rows = [x.rng.getrandbits(64 * words) for _ in range(x.T)]
        rows[0] = 0
    q, k, v = x.rows(0)
    want = x.plain().attend(0, q, k, v, x.start, rows, scale=hd ** -0.5)
    cache = _on_gpu(x, dtype)
    dq, dk, dv = x.rows(0, DEV)
    out = torch.full((x.T, Hq, hd), 7.0, dtype=dtype, device=DEV)
    mask = None if rows is None else mask_words(rows, words).to(DEV)
    got = cache.attend(0, dq, dk, dv, torch.tensor(x.start, dtype=torch.int32, device=DEV), max(nodes), mask=mask, out=out)
    n = x.start[-1]
    assert got is out and (out[n:] == 7).all()
    _close(got[:n], want[:n], dtype, max(lens) + max(nodes), (case[1:], kind))


@gpu
@pytest.mark.parametrize("case", [
    (BF, 8, 2, 128, 64, [500, 64, 63, 0, 3000], [13, 16, 1, 9, 7]),
    (BF, 4, 1, 64, 16, [200, 1], [9, 16]),
    (BF, 6, 3, 80, 24, [100, 24, 23], [25, 17, 32]),
    (BF, 28, 4, 128, 128, [300, 2000], [9, 5]),
    (BF, 3, 1, 40, 5, [700, 3], [20, 21]),
    (BF, 4, 1, 256, 16, [700, 5], [9, 2]),
    (F32, 8, 2, 128, 16, [500, 33], [16, 11]),
], ids=str)
@pytest.mark.parametrize("kind", ["tree", "full"])
def test_attention_under_a_long_table(case, kind):
    """Tables for hundreds of thousands of rows, few of them in use: the variants that are chosen by what a call may have to read."""
    dtype, Hq, Hkv, hd, ps, lens, nodes = case
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=len(lens) + hd, behind=2)
    entries = -(-(1 << 28) // (4 * hd * Hkv * len(lens) * ps))                # keys and values of 256 MB
    x.table = torch.nn.functional.pad(x.table, (0, entries), value=-1)
    rows = x.tree() if kind == "tree" else None
    want = x.plain().attend(0, *x.rows(0), x.start, rows, scale=hd ** -0.5)
    cache, start = _on_gpu(x, dtype), torch.tensor(x.start, dtype=torch.int32, device=DEV)
    out = torch.full((x.T, Hq, hd), 7.0, dtype=dtype, device=DEV)
    cache.attend(0, *x.rows(0, DEV), start, max(nodes), mask=None if rows is None else mask_words(rows, 1).to(DEV), out=out)
    n = x.start[-1]
    assert (out[n:] == 7).all()
    _close(out[:n], want[:n], dtype, max(lens) + max(nodes), (case[1:], kind))


@gpu
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_new_rows_that_are_not_finite_under_a_long_table(value):
    """As above, with a new row that only some rows attend to."""
    x = Setup(BF, 4, 1, 128, 16, [100, 40], [16, 12], seed=8)
    x.table = torch.nn.functional.pad(x.table, (0, 1 << 14), value=-1)
    rows = [1 << i for i in range(16)] + [1 << i | 1 for i in range(12)]
    x.qkv[0, 3, 5, ::3] = value                               # the value row of one new row
    want = x.plain().attend(0, *x.rows(0), x.start, rows, scale=0.1)
    got = _on_gpu(x, BF).attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), 16, mask=mask_words(rows, 1).to(DEV), scale=0.1)
    keep = [t for t in range(28) if t != 3]
    _close(got[keep], want[keep], BF, 120, value)
    assert not torch.isfinite(got[3, :, ::3]).any()


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S,n", [(8, 16), (42, 12), (43, 12), (128, 4), (129, 4), (171, 9), (60, 16)])
def test_many_short_trees(dtype, S, n):
    """Numbers of workgroups around those at which a workgroup takes more row tiles, 16 (row, head) a tile."""
    x = Setup(dtype, 16, 4, 64, 16, [7 + 5 * s % 90 for s in range(S)], [n - s % 3 for s in range(S)], seed=S)
    rows = x.tree()
    want = x.plain().attend(0, *x.rows(0), x.start, rows, scale=0.125)
    got = _on_gpu(x, dtype).attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), n, mask=mask_words(rows, 1).to(DEV))
    _close(got, want, dtype, 113, (S, n))


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_over_a_long_cache(dtype):
    """Many workgroups a sequence beside sequences of a few rows; the reference is computed in float64 on the GPU."""
    lens, nodes, Hq, Hkv, hd, ps = [20011, 3, 1200, 0], [7, 1, 16, 2], 8, 2, 128, 16
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=3)
    rows = x.tree()
    plain = x.plain()
    q, k, v = x.rows(0)
    cache = _on_gpu(x, dtype)
    got = cache.attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), 16, mask=mask_words(rows, 1).to(DEV))
    want = plain.attend(0, q, k, v, x.start, rows, scale=hd ** -0.5)
    _close(got, want, dtype, max(lens), dtype)
    again = cache.attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), 16, mask=mask_words(rows, 1).to(DEV))
    assert torch.equal(got, again)


@gpu
@pytest.mark.parametrize("dtype,hd,ps", [(BF, 128, 16), (BF, 80, 24), (F32, 64, 16), (F32, 128, 7)])
def test_attention_of_a_block_of_states(dtype, hd, ps):
    """The pattern of the block attention: 12 states of 16 tokens, each attends to the cache and to itself (192 new rows, three words)."""
    G, B = 12, 16
    x = Setup(dtype, 4, 2, hd, ps, [200], [G * B], seed=9)
    rows = [((1 << B) - 1) << (t // B * B) for t in range(G * B)]
    q, k, v = x.rows(0)
    want = x.plain().attend(0, q, k, v, x.start, rows, scale=0.1)
    got = _on_gpu(x, dtype).attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), G * B, mask=mask_words(rows, 3).to(DEV), scale=0.1)
    _close(got, want, dtype, 216, (dtype, hd, ps))


@gpu
@pytest.mark.parametrize("dtype,hd", [(BF, 128), (BF, 64), (F32, 128), (F32, 64), (BF, 40)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n,far", [(70, 40), (55, 40), (20, 18), (6, 5)])
def test_what_a_row_does_not_attend_to_does_not_show(dtype, hd, value, n, far):
    """Nodes 3 and `far` hold NaN or infinities; rows that see them get what the formula gives, all others are as if they were not there."""
    x = Setup(dtype, 4, 2, hd, 16, [50], [n], seed=4)
    rows = [r & ~(1 << 3) & ~(1 << far) if t % 7 else r | 1 << far for t, r in enumerate([x.rng.getrandbits(n) for _ in range(n)])]
    rows[4] = 0
    base = _on_gpu(x, dtype)
    start = torch.tensor(x.start, dtype=torch.int32, device=DEV)
    mask = mask_words(rows, -(-n // 64)).to(DEV)
    clean = base.attend(0, *x.rows(0, DEV), start, n, mask=mask)
    for part in (4, 6):                       # first kv head's keys, then its values; the second kv head's stay
        x.qkv[0, 3, part] = value
        x.qkv[0, far, part, hd // 2] = value
    got = base.attend(0, *x.rows(0, DEV), start, n, mask=mask).cpu()
    blind = [t for t in range(n) if not (rows[t] >> 3 & 1 or rows[t] >> far & 1)]
    assert blind and len(blind) < n
    assert torch.equal(got[blind], clean.cpu()[blind])
    assert torch.equal(got[:, 2:], clean.cpu()[:, 2:])
    q, k, v = x.rows(0)
    want = x.plain().attend(0, q, k, v, x.start, rows, scale=hd ** -0.5)
    seeing = [t for t in range(n) if t not in blind]
    assert torch.equal(torch.isnan(got[seeing, :2]), torch.isnan(want[seeing, :2]))


@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,ps,S,most", [(BF, 2, 1, 128, 16, 100, 3), (F32, 2, 2, 16, 3, 700, 2), (BF, 4, 1, 64, 8, 130, 20), (BF, 8, 1, 40, 5, 300, 9)])
def test_many_sequences_in_one_call(dtype, Hq, Hkv, hd, ps, S, most):
    """More sequences than lanes and than threads, some without rows or without cache, two long ones: attention, summaries and selection."""
    rng = random.Random(S)
    lens = [rng.choice([0, 1, rng.randint(1, 60)]) for _ in range(S)]
    lens[3], lens[S - 2] = 1500, 900
    nodes = [rng.randint(0, most) for _ in range(S)]
    nodes[5], nodes[3], nodes[S - 2] = most, 1, 1
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=S, summaries=True)
    rows = x.tree()
    plain, cache, start = x.plain(), _on_gpu(x, dtype), _ints(x.start)
    plain.summarize()
    cache.summarize()
    assert torch.equal(cache.summary.cpu(), plain.summary)
    q, k, v = x.rows(0)
    want = plain.attend(0, q, k, v, x.start, rows, scale=hd ** -0.5)
    _close(cache.attend(0, *x.rows(0, DEV), start, most, mask=mask_words(rows, 1).to(DEV)), want, dtype, 1600, S)
    sel = plain.select(0, q, x.start, 4, 1, 1)
    got = cache.select(0, x.rows(0, DEV)[0], start, most, 4, keep_first=1, keep_last=1)
    assert got.tolist() == sel
    want = plain.attend(0, q, k, v, x.start, rows, selected=sel, scale=hd ** -0.5)
    _close(cache.attend(0, *x.rows(0, DEV), start, most, mask=mask_words(rows, 1).to(DEV), selected=got), want, dtype, 100, (S, "selected"))


@gpu
@pytest.mark.parametrize("dtype,n", [(BF, 5), (BF, 60), (F32, 9)])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30])
def test_scales_of_zero_and_below(dtype, n, scale):
    x = Setup(dtype, 4, 2, 64, 16, [300], [n], seed=n)
    rows = x.tree()
    q, k, v = x.rows(0)
    want = x.plain().attend(0, q, k, v, x.start, rows, scale=scale)
    got = _on_gpu(x, dtype).attend(0, *x.rows(0, DEV), _ints(x.start), n, mask=mask_words(rows, 1).to(DEV), scale=scale)
    _close(got, want, dtype, 400, (dtype, n, scale))


@gpu
def test_extreme_scores_and_empty_rows():
    """Scores of +-1e4 (a running maximum that jumps), equal scores, and rows without any key."""
    x = Setup(F32, 2, 1, 64, 16, [100, 0], [20, 3], seed=5, garbage=False)
    x.k[0, :, :, :, 0] *= 1000.0
    x.qkv[0, :, :2, 0] *= 80.0
    rows = x.tree()
    rows[20] = rows[21] = 0
    q, k, v = x.rows(0)
    want = x.plain().attend(0, q, k, v, x.start, rows, scale=0.125)
    got = _on_gpu(x, F32).attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), 20, mask=mask_words(rows, 1).to(DEV), scale=0.125)
    assert (got[20:22] == 0).all()
    # a score of 1e4 in fp32 is off by some 64 * 2^-24 * 1e4 = 0.04 in the exponent
    far = (got.double().cpu() - want).abs()
    assert float(far.max()) < 0.25 and float(far.median()) < 1e-3


@gpu
@pytest.mark.parametrize("dtype,hd,ps", [(BF, 128, 64), (BF, 128, 16), (F32, 64, 24), (BF, 96, 5)])
def test_attention_over_selected_pages(dtype, hd, ps):
    lens, nodes = [900, 40, 0, 333], [6, 1, 2, 17]
    x = Setup(dtype, 8, 2, hd, ps, lens, nodes, seed=6)
    rows = x.tree()
    n_sel, sel = 11, []
    for n in lens:        # any order, gaps, entries beyond the pages in use; every page at most once
        used = -(-n // ps)
        sel.append([])
        for _ in range(2):
            p = x.rng.sample(range(used), min(used, 7)) + [-1, used, used + 1, 1 << 20]
            x.rng.shuffle(p)
            sel[-1].append((p + [-5] * n_sel)[:n_sel])
    q, k, v = x.rows(0)
    want = x.plain().attend(0, q, k, v, x.start, rows, selected=sel, scale=hd ** -0.5)
    got = _on_gpu(x, dtype).attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), 17, mask=mask_words(rows, 1).to(DEV),
                                   selected=torch.tensor(sel, dtype=torch.int32, device=DEV))
    _close(got, want, dtype, max(lens), (dtype, hd, ps))


@gpu
@pytest.mark.parametrize("ps", [16, 10])
def test_pages_that_do_not_exist_have_no_rows(ps):
    """Table entries outside the pool and lengths beyond the table: as documented, and nothing out of range is touched."""
    x = Setup(BF, 4, 2, 128, ps, [100, 50, 30], [3, 4, 5], seed=7)
    x.table[0, 1], x.table[1, 0], x.table[2, 1] = -7, 1 << 30, x.refs.numel()
    x.len[1] = 50 + (1 << 20)
    x.len[2] = -4
    plain = x.plain()
    plain.len[1], plain.len[2] = plain.max_pages * ps, 0
    plain.k[:], plain.v[:] = torch.nan_to_num(plain.k), torch.nan_to_num(plain.v)
    x.k, x.v = plain.k.clone(), plain.v.clone()
    q, k, v = x.rows(0)
    want = plain.attend(0, q, k, v, x.start, None, scale=0.1)
    got = _on_gpu(x, BF).attend(0, *x.rows(0, DEV), torch.tensor(x.start, dtype=torch.int32, device=DEV), 5, scale=0.1)
    _close(got, want, BF, 200, ps)


@gpu
def test_row_ranges_out_of_order_and_bounds_that_are_too_small():
    """row_start is taken within [0, T] and ascending; rows beyond max_rows are left as they were."""
    x = Setup(BF, 4, 2, 128, 16, [40, 20], [6, 6], seed=8)
    cache = _on_gpu(x, BF)
    rows = x.rows(0, DEV)
    out = torch.full((12, 4, 128), 7.0, dtype=BF, device=DEV)
    cache.attend(0, *rows, torch.tensor([-5, 1 << 30, 3], dtype=torch.int32, device=DEV), 4, out=out)
    assert not (out[:4] == 7).all(-1).any() and (out[4:] == 7).all()
    full = cache.attend(0, *rows, torch.tensor([0, 4, 12], dtype=torch.int32, device=DEV), 8)
    _close(out[:4], full[:4].double().cpu(), BF, 44, "fewer rows")


@gpu
def test_offsets_beyond_32_bits():
    """A pool of 4.3 GB of keys: the pages behind 2^32 bytes are read and written."""
    L, n_pages, Hkv, ps, hd = 1, 1 << 14, 8, 128, 128
    cfg = _cfg(BF, 8, Hkv, hd)
    cache = sp.PagedCache.empty(cfg, L, n_pages + 40, ps, 2, 64, summaries=True, device=DEV)
    assert cache.k.numel() * 2 > 1 << 32
    cache.refs[:n_pages] = 1
    gen = torch.Generator(device=DEV).manual_seed(1)
    rows = torch.randn((1, 1001, 2 * Hkv, hd), generator=gen, device=DEV).to(BF)
    cache.append(rows[:, :, :Hkv], rows[:, :, Hkv:], torch.tensor([0, 1000, 1001], dtype=torch.int32, device=DEV))
    cache.summarize()
    assert cache.table[0, :8].tolist() == list(range(n_pages, n_pages + 8)) and cache.table[1, 0] == n_pages + 8
    assert torch.equal(cache.k[0, n_pages + 7, :, 103], rows[0, 999, :Hkv])
    q = torch.randn((1, 8, hd), generator=gen, device=DEV).to(BF)
    z = torch.zeros((1, 8, hd), dtype=BF, device=DEV)
    start = torch.tensor([0, 1, 1], dtype=torch.int32, device=DEV)
    none = torch.zeros((1, 1), dtype=torch.int64, device=DEV)
    got = cache.attend(0, q, z, z, start, 1, mask=none)
    k, v = rows[0, :1000, :Hkv].double(), rows[0, :1000, Hkv:].double()
    p = torch.softmax((k * q.double()).sum(2) * hd ** -0.5, 0)
    _close(got[0], (p[:, :, None] * v).sum(0).cpu(), BF, 1000, "far pages")
    assert torch.equal(cache.summary[0, n_pages + 3, :, 0], rows[0, 384:512, :Hkv].amin(0))
    # many rows (tiles through LDS), a selection, a fork and its append
    T = 100
    q = torch.randn((T, 8, hd), generator=gen, device=DEV).to(BF)
    z, start, none = torch.zeros((T, 8, hd), dtype=BF, device=DEV), torch.tensor([0, T, T], dtype=torch.int32, device=DEV), torch.zeros((T, 2), dtype=torch.int64, device=DEV)
    want = torch.einsum("thj,jhd->thd", torch.softmax(torch.einsum("thd,jhd->thj", q.float(), k.float()).double() * hd ** -0.5, 2).float(), v.float())
    _close(cache.attend(0, q, z, z, start, T, mask=none), want.double().cpu(), BF, 1000, "far pages, many rows")
    sel = cache.select(0, q, start, T, 8)
    assert sel[0].tolist() == [list(range(8))] * Hkv and sel[1].tolist() == [[0] + [-1] * 7] * Hkv
    _close(cache.attend(0, q, z, z, start, T, mask=none, selected=sel), want.double().cpu(), BF, 1000, "far pages, selected")
    cache.free(torch.tensor([1], dtype=torch.int32, device=DEV))
    cache.fork(torch.tensor([0], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV))
    cache.append(rows[:, :3, :Hkv], rows[:, :3, Hkv:], torch.tensor([0, 0, 3], dtype=torch.int32, device=DEV))
    assert cache.table[1, :8].tolist() == [*range(n_pages, n_pages + 7), n_pages + 8] and cache.len.tolist() == [1000, 1003]
    assert torch.equal(cache.k[0, n_pages + 8, :, :104], cache.k[0, n_pages + 7, :, :104]) and torch.equal(cache.v[0, n_pages + 8, :, 106], rows[0, 2, Hkv:])
    cache.refs[:100] = 0                                        # pages 0 .. 99 go, and with them the need for the far ones
    assert cache.compact().item() == n_pages - 100 + 9 and int(cache.table.max()) < n_pages
    _close(cache.attend(0, q, z, z, start, T, mask=none), want.double().cpu(), BF, 1000, "after compaction")


# ---- selection --------------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,ps,lens,nodes", [
    (BF, 8, 2, 128, 16, [700, 3, 0, 160, 5000], [4, 1, 2, 0, 9]),
    (BF, 4, 4, 64, 64, [3000], [1]),
    (BF, 6, 3, 80, 24, [100, 1000], [33, 2]),
    (F32, 4, 1, 128, 10, [900, 77], [70, 3]),
    (F32, 2, 2, 8, 1, [1500], [5]),
    (BF, 2, 1, 256, 32, [3100], [2])])
@pytest.mark.parametrize("n_sel,first,last", [(1, 0, 0), (8, 1, 1), (40, 0, 3), (7, 9, 9), (3000, 1, 1)])
def test_selected_pages(dtype, Hq, Hkv, hd, ps, lens, nodes, n_sel, first, last):
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=n_sel + hd, summaries=True)
    plain = x.plain()
    plain.summarize()
    cache = _on_gpu(x, dtype)
    cache.summarize()
    assert torch.equal(cache.summary.cpu(), plain.summary)
    got = cache.select(0, x.rows(0, DEV)[0], torch.tensor(x.start, dtype=torch.int32, device=DEV), max(nodes), n_sel, keep_first=first, keep_last=last)
    assert got.tolist() == plain.select(0, x.rows(0)[0], x.start, n_sel, first, last)


@gpu
def test_selection_of_equal_infinite_and_nan_scores():
    """Equal scores go to the lower index; NaN is the lowest; queries and summaries of zeros, infinities and both signs of zero."""
    x = Setup(BF, 2, 1, 16, 4, [400], [2], seed=2, summaries=True)
    plain, cache = x.plain(), None
    plain.summarize()
    s = plain.summary
    for j in range(0, 100, 3):                                  # a third of the pages are alike
        s[0, plain.table[0][j]] = s[0, plain.table[0][0]]
    s[0, plain.table[0][50]] = math.nan
    s[0, plain.table[0][51]] = math.inf
    s[0, plain.table[0][52]] = -math.inf
    s[0, plain.table[0][53]] = 0.0
    s[0, plain.table[0][56]] = -0.0
    x.summary = s
    cache = _on_gpu(x, BF)
    start = torch.tensor(x.start, dtype=torch.int32, device=DEV)
    for n_sel in (1, 2, 20, 33, 34, 98, 99, 100):
        got = cache.select(0, x.rows(0, DEV)[0], start, 2, n_sel, keep_first=0, keep_last=0)
        assert got.tolist() == plain.select(0, x.rows(0)[0], x.start, n_sel, 0, 0), n_sel
    x.qkv.zero_()
    got = cache.select(0, x.rows(0, DEV)[0], start, 2, 9, keep_first=0, keep_last=2)
    assert got.tolist() == plain.select(0, x.rows(0)[0], x.start, 9, 0, 2)


@gpu
@pytest.mark.parametrize("hd,nodes", [(128, [1, 30]), (128, [22, 5]), (64, [40, 9]), (256, [7, 24]), (24, [33, 20]), (128, [2, 1])])
@pytest.mark.parametrize("kind", ["equal", "all equal", "last bit", "cancelling", "large", "infinite", "small"])
def test_selection_of_nearly_equal_scores(hd, nodes, kind):
    """Pages whose scores differ by less than fp32 sums tell apart, or not at all, among pages that are far from one another."""
    x = Setup(BF, 32, 2, hd, 4, [1500, 1203], nodes, seed=hd + nodes[0], summaries=True)
    plain = x.plain()
    plain.summarize()
    rng = torch.Generator().manual_seed(7)
    for s, n in ((0, 375), (1, 301)):
        alike = [plain.table[s][j] for j in torch.randperm(n, generator=rng)[:n if kind == "all equal" else n // 2].tolist()]
        for p in alike[1:]:
            plain.summary[0, p] = plain.summary[0, alike[0]]
            h, side, ch = (int(torch.randint(0, m, (1,), generator=rng)) for m in (2, 2, hd))
            y = plain.summary[0, p, h, side, ch:ch + 1]
            if kind == "last bit":                              # one channel by its last bit
                y.view(torch.int16)[0] += int(torch.randint(-1, 2, (1,), generator=rng))
            elif kind == "cancelling":                          # large terms of both signs: the sum is small beside them
                plain.summary[0, p, :, :, 0:2] = torch.tensor([4096.0, -4096.0])
                y.view(torch.int16)[0] += int(torch.randint(-1, 2, (1,), generator=rng))
            elif kind == "large":
                plain.summary[0, p, h, 0, ch], plain.summary[0, p, h, 1, ch] = -2.0 ** 70, 2.0 ** 70
            elif kind == "infinite":
                y[0] = math.inf if side else -math.inf
            elif kind == "small":
                plain.summary[0, p] *= 2.0 ** -128              # subnormal
    x.summary = plain.summary
    cache, start = _on_gpu(x, BF), torch.tensor(x.start, dtype=torch.int32, device=DEV)
    for n_sel, first, last in ((1, 0, 0), (40, 1, 1), (150, 0, 0), (200, 0, 2), (299, 3, 0), (301, 0, 1), (374, 0, 0)):
        got = cache.select(0, x.rows(0, DEV)[0], start, max(nodes), n_sel, keep_first=first, keep_last=last)
        assert got.tolist() == plain.select(0, x.rows(0)[0], x.start, n_sel, first, last), (kind, n_sel)


@gpu
def test_selection_without_new_rows():
    x = Setup(BF, 2, 1, 16, 4, [400, 9, 0], [2, 1, 1], seed=6, summaries=True)
    cache, start = _on_gpu(x, BF), torch.zeros(4, dtype=torch.int32, device=DEV)
    got = cache.select(0, x.rows(0, DEV)[0][:0], start, 2, 4, keep_first=0, keep_last=1).tolist()
    assert got == [[[0, 1, 2, 99]], [[0, 1, 2, -1]], [[-1] * 4]]


@gpu
@pytest.mark.parametrize("dtype,nodes", [(BF, 1), (BF, 40), (F32, 3)])
def test_pages_that_are_always_taken_come_before_infinite_bounds(dtype, nodes):
    """Bounds of +inf on every page: the first and the last pages are taken all the same, then the lowest indices."""
    x = Setup(dtype, 2, 1, 16, 4, [400], [nodes], seed=5, summaries=True)
    x.summary[:, :, :, 0], x.summary[:, :, :, 1] = -math.inf, math.inf
    cache, start = _on_gpu(x, dtype), torch.tensor(x.start, dtype=torch.int32, device=DEV)
    pick = lambda n, first, last: cache.select(0, x.rows(0, DEV)[0], start, nodes, n, keep_first=first, keep_last=last).tolist()[0][0]
    assert pick(1, 0, 1) == [99]
    assert pick(3, 0, 2) == [0, 98, 99]
    assert pick(4, 1, 1) == [0, 1, 2, 99]


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nodes", [[5, 1], [11, 20], [17, 3], [40, 33], [2, 70]])
def test_selection_with_summaries_that_are_not_finite(dtype, nodes):
    """Infinities on one side of a page's bounds: the channel's term is what the formula gives for each query's sign, for every row."""
    x = Setup(dtype, 4, 2, 24, 4, [300, 160], nodes, seed=sum(nodes), summaries=True)
    plain = x.plain()
    plain.summarize()
    for s, n in ((0, 75), (1, 40)):
        for i in range(25):
            j = x.rng.randrange(n)
            plain.summary[0, plain.table[s][j], x.rng.randrange(2), x.rng.randrange(2), x.rng.randrange(24)] = x.rng.choice([math.inf, -math.inf, math.nan])
    x.summary = plain.summary
    cache = _on_gpu(x, dtype)
    for n_sel in (3, 20):
        got = cache.select(0, x.rows(0, DEV)[0], torch.tensor(x.start, dtype=torch.int32, device=DEV), max(nodes), n_sel, keep_first=0, keep_last=0)
        assert got.tolist() == plain.select(0, x.rows(0)[0], x.start, n_sel, 0, 0), n_sel


@gpu
def test_summaries_of_new_rows_only():
    x = Setup(BF, 4, 2, 128, 16, [100, 33, 0, 16], [1, 1, 1, 1], layers=3, seed=3, summaries=True)
    plain, cache = x.plain(), _on_gpu(x, BF)
    for start in ([90, 32, 0, 16], [0, 40, -3, 1]):
        plain.summarize(start)
        cache.summarize(torch.tensor(start, dtype=torch.int32, device=DEV))
        assert torch.equal(cache.summary.cpu(), plain.summary)


# ---- pages ------------------------------------------------------------------------------------------------------------------

def _same(cache, plain, what=""):
    assert cache.refs.tolist() == plain.refs, what
    assert cache.len.tolist() == plain.len, what
    assert cache.table.tolist() == plain.table, what
    same = lambda a, b: torch.equal(torch.nan_to_num(a.cpu().float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0))
    assert same(cache.k, plain.k) and same(cache.v, plain.v), what
    assert plain.summary is None or torch.equal(cache.summary.cpu(), plain.summary), what


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


@gpu
@pytest.mark.parametrize("dtype,Hkv,hd,ps,layers", [(BF, 2, 128, 16, 3), (F32, 1, 24, 5, 1), (BF, 3, 8, 1, 2), (BF, 1, 16, 64, 70)])
def test_append_of_all_rows_and_of_paths(dtype, Hkv, hd, ps, layers):
    lens, nodes = [37, 0, 2 * ps, 2 * ps - 1, 5], [9, 40, 0, 1, 70]
    x = Setup(dtype, Hkv, Hkv, hd, ps, lens, nodes, layers=layers, spare=250, seed=ps)
    x.table = torch.nn.functional.pad(x.table, (0, 200), value=-1)
    plain, cache = x.plain(), _on_gpu(x, dtype)
    status = _ints([9] * 5)
    cache.append(*x.all_rows(DEV), _ints(x.start), status=status)
    assert status.tolist() == plain.append(*x.all_rows(), x.start)
    _same(cache, plain)
    rows = x.tree()
    for nodes_ in ([8, 39, -1, 0, 69], [0, 3, -1, -1, 20], [9, 12, 0, 1, 70]):      # the last: nodes that do not exist
        # nodes are read where a walk leaves them: column 0 of [n_seqs, 4]
        result = torch.full((5, 4), 77, dtype=torch.int32, device=DEV)
        result[:, 0] = _ints(nodes_)
        cache.append(*x.all_rows(DEV), _ints(x.start), mask=mask_words(rows, 2).to(DEV), node=result[:, 0], status=status)
        assert status.tolist() == plain.append(*x.all_rows(), x.start, rows, nodes_), nodes_
        _same(cache, plain, nodes_)


@gpu
def test_append_without_room():
    """Too few pages: the sequences in order, those that fit get theirs; too few table entries; a shared last page."""
    x = Setup(BF, 1, 1, 16, 4, [3, 4, 6, 1, 0], [9, 9, 1, 4, 40], spare=4, seed=2)
    plain, cache = x.plain(), _on_gpu(x, BF)
    status = _ints([9] * 5)
    cache.append(*x.all_rows(DEV), _ints(x.start), status=status)
    want = plain.append(*x.all_rows(), x.start)
    assert status.tolist() == want and set(want) == {0, 1, 2}
    _same(cache, plain)
    x = Setup(BF, 1, 1, 16, 4, [3, 4], [1, 1], seed=2)
    x.refs[x.table[0, 0]] = 2
    plain, cache = x.plain(), _on_gpu(x, BF)
    cache.append(*x.all_rows(DEV), _ints(x.start))
    assert plain.append(*x.all_rows(), x.start) == [3, 0]
    _same(cache, plain)


@gpu
def test_append_to_thousands_of_sequences():
    S, ps = 3000, 4
    rng = random.Random(1)
    lens, nodes = [rng.randint(0, 9) for _ in range(S)], [rng.randint(0, 7) for _ in range(S)]
    x = Setup(F32, 1, 1, 8, ps, lens, nodes, spare=6000, seed=1, garbage=False)
    for spare in (6000, 900):             # room for all; too few pages
        x.refs[:] = (x.refs == 1).int()
        if spare == 900:
            free = (x.refs == 0).nonzero()[spare:, 0]
            x.refs[free] = 1
        plain, cache = x.plain(), _on_gpu(x, F32)
        status = torch.zeros(S, dtype=torch.int32, device=DEV)
        cache.append(*x.all_rows(DEV), _ints(x.start), status=status)
        want = plain.append(*x.all_rows(), x.start)
        assert status.tolist() == want and (spare == 900) == (1 in want)
        _same(cache, plain)


@gpu
def test_fork_free_and_append_again():
    x = Setup(BF, 2, 2, 16, 8, [37, 16, 0, 0, 0, 0, 3, 0], [1] * 8, layers=2, spare=6, seed=5, summaries=True)
    plain, cache = x.plain(), _on_gpu(x, BF)
    plain.summarize()
    cache.summarize()
    steps = [("fork", [0, 1, 6], [2, 3, 4]), ("fork", [0, 0, 2, 5, 0, 6, 9, 0, -1], [5, 5, 7, 7, 1, 6, 1, 8, 7]), ("free", [0]),
             ("append",), ("fork", [2, 5], [0, 7]), ("free", [5, 5, 2, -3, 8, 1 << 30, 1]), ("append",), ("compact",), ("fork", [0], [1]),
             ("free", list(range(8))), ("compact",)]
    for i, (name, *args) in enumerate(steps):
        if name == "fork":
            status = _ints([9] * len(args[0]))
            cache.fork(_ints(args[0]), _ints(args[1]), status=status)
            assert status.tolist() == plain.fork(*args), (i, args)
        elif name == "free":
            cache.free(_ints(args[0]))
            plain.free(*args)
        elif name == "compact":
            assert cache.compact().item() == plain.compact()
        else:
            status = _ints([9] * 8)
            cache.append(*x.all_rows(DEV), _ints(x.start), status=status)
            assert status.tolist() == plain.append(*x.all_rows(), x.start), i
        _same(cache, plain, (i, name, args))
    assert not any(plain.refs)


@gpu
@pytest.mark.parametrize("n_pages,ps,layers", [(40, 4, 2), (20000, 1, 1), (300, 16, 66)])
def test_compaction_of_scattered_pages(n_pages, ps, layers):
    rng = random.Random(n_pages)
    S = 12
    used = [rng.randint(0, n_pages // S) for _ in range(S)]
    x = Setup(BF, 1, 1, 16, ps, [u * ps for u in used], [1] * S, layers=layers, spare=n_pages - sum(used), seed=n_pages, garbage=False, summaries=True)
    x.summary = torch.randn(x.summary.shape).to(BF)
    plain, cache = x.plain(), _on_gpu(x, BF)
    for gone in ([0, 3, 5], [], [1, 2, 4, 6, 7, 8, 9, 10, 11]):
        if gone:
            cache.free(_ints(gone))
        plain.free(gone)
        n_used = torch.zeros(1, dtype=torch.int32, device=DEV)
        assert cache.compact(n_used=n_used) is n_used and n_used.item() == plain.compact()
        _same(cache, plain, gone)
    cache.free(_ints(list(range(S))))
    assert cache.compact().item() == 0 and not cache.refs.any()


# ---- together ---------------------------------------------------------------------------------------------------------------

def _decode_step(cache, layers, rows, q, start, max_rows, mask, edges, drafts, targets, n_sel):
    """One step of drafted decoding over a paged cache, no host in between: attention in every layer (over selected pages), the walk down
    each sequence's tree (a node is a token), and the accepted path's rows into the cache."""
    outs, sels = [], []
    for l in range(layers):
        sel = cache.select(l, q[l], start, max_rows, n_sel, keep_first=1, keep_last=1)
        outs.append(cache.attend(l, q[l], rows[0][l], rows[1][l], start, max_rows, mask=mask, selected=sel))
        sels.append(sel)
    result = torch.empty((cache.n_seqs, 4), dtype=torch.int32, device=DEV)
    for s in range(cache.n_seqs):
        sp.graph_accept(edges[s], drafts[s], targets[s], res=result[s])
    before = cache.len.clone()
    cache.append(*rows, start, mask=mask, node=result[:, 0])
    cache.summarize(before)
    return outs, sels, result


@gpu
@pytest.mark.parametrize("dtype,hd,ps", [(BF, 128, 16), (F32, 64, 24)])
def test_drafted_decoding_over_a_paged_cache(dtype, hd, ps):
    """Fork a prompt, then steps of select, attend, walk, append; at the end one copy is freed and the pool compacted."""
    L, S, Hq, Hkv, n_sel, nodes = 2, 3, 4, 2, 4, [12, 5, 9]
    x = Setup(dtype, Hq, Hkv, hd, ps, [6 * ps + 3, 0, 0], nodes, layers=L, spare=40, seed=6, summaries=True)
    x.table = torch.nn.functional.pad(x.table, (0, 12), value=-1)
    plain, cache = x.plain(), _on_gpu(x, dtype)
    plain.summarize()
    cache.summarize()
    assert plain.fork([0, 0], [1, 2]) == [0, 0]
    cache.fork(_ints([0, 0]), _ints([1, 2]))
    start, rng = _ints(x.start), random.Random(3)
    for step in range(4):
        edges, drafts, targets, rows = [], [], [], []
        for n in nodes:
            parent = [rng.randint(0, i - 1) for i in range(1, n)]
            e = [(p, i + 1) for i, p in enumerate(parent)]
            m = sp.tree_mask(e, n, device="cpu")
            rows += [int(r[0]) for r in m]
            draft = list(range(100, 100 + n))                     # every node drafts a token of its own ...
            target = [draft[rng.choice([c for p, c in e if p == i] or [i])] if rng.random() < 0.8 else 7 for i in range(n)]
            edges.append(_ints(e).reshape(-1, 2))
            drafts.append(_ints(draft).reshape(-1, 1))
            targets.append(_ints(target).reshape(-1, 1))
        x.qkv = torch.randn(x.qkv.shape, generator=torch.Generator().manual_seed(step)).to(dtype)
        dq = [x.rows(l, DEV)[0] for l in range(L)]
        outs, sels, result = _decode_step(cache, L, x.all_rows(DEV), dq, start, 12, mask_words(rows, 1).to(DEV), edges, drafts, targets, n_sel)
        for l in range(L):
            q, k, v = x.rows(l)
            sel = plain.select(l, q, x.start, n_sel, 1, 1)
            assert sels[l].tolist() == sel
            _close(outs[l], plain.attend(l, q, k, v, x.start, rows, selected=sel, scale=hd ** -0.5), dtype, 200, (step, l))
        node = result[:, 0].tolist()
        for s in range(S):          # the walk's node is reached through targets that are its path's drafts
            d, t = drafts[s][:, 0].tolist(), targets[s][:, 0].tolist()
            at = 0
            while any(p == at and d[c] == t[at] for p, c in edges[s].tolist()):
                at = next(c for p, c in edges[s].tolist() if p == at and d[c] == t[at])
            assert at == node[s]
        before = list(plain.len)
        assert plain.append(*x.all_rows(), x.start, rows, node) == [0] * S
        plain.summarize(before)
        _same(cache, plain, step)
    plain.free([1])
    cache.free(_ints([1]))
    assert cache.compact().item() == plain.compact()
    _same(cache, plain)


@gpu
def test_captured_steps_replay_like_eager_ones():
    """A whole step in a HIP graph, replayed with the program's own work between: every replay equals the eager step on a second cache."""
    L, n_sel, nodes, hd = 2, 3, [5, 1], 128
    x = Setup(BF, 4, 2, hd, 16, [100, 20], nodes, layers=L, spare=60, seed=8, summaries=True)
    x.table = torch.nn.functional.pad(x.table, (0, 12), value=-1)
    rng = random.Random(1)
    rows = [r for n in nodes for r in tree_rows(n, rng)]
    node, start, mask = _ints([4, 0]), _ints(x.start), mask_words(rows, 1).to(DEV)
    new = x.qkv.to(DEV)
    q, k, v = new[:, :, :4], new[:, :, 4:6], new[:, :, 6:]

    def step(cache):
        outs = []
        for l in range(L):
            sel = cache.select(l, q[l], start, 5, n_sel)
            outs += [sel, cache.attend(l, q[l], k[l], v[l], start, 5, mask=mask, selected=sel), cache.attend(l, q[l], k[l], v[l], start, 5, mask=mask)]
        before = cache.len.clone()
        cache.append(k, v, start, mask=mask, node=node)
        cache.summarize(before)
        return outs

    a, b = _on_gpu(x, BF), _on_gpu(x, BF)
    for c in (a, b):
        c.summarize()
        step(c)                                  # once in front of the capture
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = step(a)
    for i in range(5):
        new.copy_(torch.randn(new.shape, generator=torch.Generator().manual_seed(i)).to(BF))
        torch.cuda.synchronize()
        g.replay()
        junk = torch.randn(1 << 20, device=DEV).sum().item()
        eager = step(b)
        for m, n in zip(captured, eager):
            assert torch.equal(m, n), (i, junk)
        assert torch.equal(a.len, b.len) and torch.equal(a.table, b.table) and torch.equal(a.summary, b.summary)


@gpu
def test_calls_on_two_streams_at_once():
    """Calls that only read the cache share nothing: two streams, each its own outputs and scratch."""
    x = Setup(BF, 8, 2, 128, 16, [9000, 300], [6, 9], seed=4, summaries=True)
    cache = _on_gpu(x, BF)
    cache.summarize()
    q, k, v = x.rows(0, DEV)
    q2 = torch.randn_like(q.float()).to(BF)
    start = _ints(x.start)

    def work(q, stream=None):
        sel = cache.select(0, q, start, 9, 20, stream=stream)
        return [sel, cache.attend(0, q, k, v, start, 9, selected=sel, stream=stream), cache.attend(0, q, k, v, start, 9, stream=stream)]

    want = [work(q), work(q2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(20):
        got = [work(y, s) for y, s in zip((q, q2), streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(m, n) for m, n in zip(g, w)), i
    raw = work(q, streams[0].cuda_stream)        # a raw handle, as everywhere in the binding
    torch.cuda.synchronize()
    assert all(torch.equal(m, n) for m, n in zip(raw, want[0]))


# ---- refusals (no GPU) ------------------------------------------------------------------------------------------------------

DUMMY = 0x10000


def _host(**kw):
    d = dict(n_pages=10, page_size=16, n_seqs=3, max_pages=7, refs=DUMMY, table=DUMMY, len=DUMMY)
    d.update(kw)
    return sp.PagedCacheStruct(d["n_pages"], d["page_size"], d["n_seqs"], d["max_pages"], d["refs"], d["table"], d["len"])


BAD_CACHES = [(dict(n_pages=0), -1), (dict(page_size=0), -1), (dict(n_seqs=0), -1), (dict(max_pages=0), -1), (dict(n_seqs=4097), -2),
              (dict(n_pages=1 << 27, page_size=16), -2), (dict(max_pages=(1 << 22) + 1, page_size=1), -2), (dict(max_pages=1 << 22, page_size=512), -2),
              (dict(max_pages=1 << 15, page_size=1 << 16), -2)]
BAD_POINTERS = [(dict(refs=None), -1), (dict(table=None), -1), (dict(len=None), -1), (dict(refs=DUMMY + 2), -3), (dict(len=DUMMY + 1), -3)]
BAD_HEADS = [(dict(Hkv=3), -2), (dict(hd=260), -2), (dict(hd=12), -2), (dict(hd=0), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(dtype=2), -1)]


def _heads(Hq=8, Hkv=2, hd=128, dtype=sp.SPIFFY_BF16):
    return sp.ModelCfg(64, Hq, Hkv, hd, 8, 2, 1, dtype, 1e-5, 1e4)


def _layer(**kw):
    d = dict(k=DUMMY, v=DUMMY, summary=DUMMY)
    d.update(kw)
    return sp.PageLayer(d["k"], d["v"], d["summary"])


def _attend(cfg=None, cache=None, layer=None, **kw):
    d = dict(q=DUMMY, qs=1024, k=DUMMY, v=DUMMY, ks=256, start=DUMMY, T=5, max_rows=5, mask=None, words=0, sel=None, n_sel=0, scale=1.0,
             out=DUMMY, os=1024, ws=DUMMY, wn=1 << 40)
    d.update(kw)
    return sp.lib.spiffy_tree_attention(C.byref(cfg or _heads()), C.byref(cache or _host()), C.byref(layer or _layer()), d["q"], d["qs"], d["k"], d["v"],
                                        d["ks"], d["start"], d["T"], d["max_rows"], d["mask"], d["words"], d["sel"], d["n_sel"], d["scale"], d["out"],
                                        d["os"], d["ws"], d["wn"], None)


def test_tree_attention_refuses():
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert _attend(cache=_host(**kw)) == want, kw
    for kw, want in BAD_HEADS:
        assert _attend(cfg=_heads(**kw)) == want, kw
    for kw, want in [(dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(out=None), -1), (dict(start=None), -1), (dict(T=0), -1),
                     (dict(max_rows=0), -1), (dict(max_rows=1025), -2), (dict(T=(1 << 20) + 1), -2), (dict(qs=1023), -1), (dict(qs=1028), -3),
                     (dict(ks=255), -1), (dict(ks=260), -3), (dict(os=1000), -1), (dict(os=1025), -3), (dict(q=DUMMY + 8), -3), (dict(k=DUMMY + 2), -3),
                     (dict(v=DUMMY + 4), -3), (dict(out=DUMMY + 8), -3), (dict(mask=DUMMY, words=0), -1), (dict(mask=DUMMY, words=17), -2),
                     (dict(mask=DUMMY + 4, words=1), -3), (dict(sel=DUMMY, n_sel=0), -1), (dict(sel=DUMMY + 2, n_sel=2), -3), (dict(sel=DUMMY, n_sel=1 << 28), -2),
                     (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(ws=None), -1), (dict(ws=DUMMY + 128), -3), (dict(wn=0), -4),
                     (dict(start=DUMMY + 1), -3)]:
        assert _attend(**kw) == want, kw
    for kw, want in [(dict(k=None), -1), (dict(v=None), -1), (dict(k=DUMMY + 8), -3), (dict(v=DUMMY + 8), -3)]:
        assert _attend(layer=_layer(**kw)) == want, kw
    size = lambda m, **kw: sp.lib.spiffy_tree_attention_workspace_bytes(C.byref(_heads()), C.byref(_host(**kw)), m)
    assert size(5) > 0 and size(0) == 0 and size(1025) == 0 and size(5, n_pages=0) == 0
    many = _heads(Hq=4096, Hkv=4096, hd=8)
    assert _attend(cfg=many, cache=_host(n_seqs=4096), qs=32768, ks=32768, os=32768) == -2
    assert sp.lib.spiffy_tree_attention_workspace_bytes(C.byref(many), C.byref(_host(n_seqs=4096)), 5) == 0


def _select(cfg=None, cache=None, layer=None, **kw):
    d = dict(q=DUMMY, qs=1024, start=DUMMY, T=5, max_rows=5, n_sel=4, first=1, last=1, out=DUMMY, ws=DUMMY, wn=1 << 40)
    d.update(kw)
    return sp.lib.spiffy_page_select(C.byref(cfg or _heads()), C.byref(cache or _host()), C.byref(layer or _layer()), d["q"], d["qs"], d["start"], d["T"],
                                     d["max_rows"], d["n_sel"], d["first"], d["last"], d["out"], d["ws"], d["wn"], None)


def test_page_select_and_summary_refuse():
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert _select(cache=_host(**kw)) == want, kw
        assert sp.lib.spiffy_page_summary(C.byref(_heads()), C.byref(_host(**kw)), 1, C.byref(_layer()), None, None) == want, kw
    for kw, want in BAD_HEADS:
        assert _select(cfg=_heads(**kw)) == want, kw
        assert sp.lib.spiffy_page_summary(C.byref(_heads(**kw)), C.byref(_host()), 1, C.byref(_layer()), None, None) == want, kw
    for kw, want in [(dict(q=None), -1), (dict(start=None), -1), (dict(out=None), -1), (dict(T=0), -1), (dict(max_rows=0), -1), (dict(max_rows=1025), -2),
                     (dict(n_sel=0), -1), (dict(n_sel=(1 << 22) + 1), -2), (dict(first=-1), -1), (dict(last=-1), -1), (dict(qs=8), -1), (dict(qs=1030), -3),
                     (dict(q=DUMMY + 8), -3), (dict(out=DUMMY + 2), -3), (dict(ws=None), -1), (dict(ws=DUMMY + 16), -3), (dict(wn=8), -4)]:
        assert _select(**kw) == want, kw
    assert _select(layer=_layer(summary=None)) == -1 and _select(layer=_layer(summary=DUMMY + 8)) == -3
    summary = lambda n, layer, start: sp.lib.spiffy_page_summary(C.byref(_heads()), C.byref(_host()), n, layer, start, None)
    assert summary(0, C.byref(_layer()), None) == -1 and summary(1, None, None) == -1 and summary(1, C.byref(_layer(k=None)), None) == -1
    assert summary(257, C.byref(_layer()), None) == -2 and summary(1, C.byref(_layer()), DUMMY + 2) == -3


def test_tables_of_more_than_31_bits_are_refused():
    big, fits = (dict(n_seqs=4096, max_pages=m, page_size=1) for m in (1 << 19, (1 << 19) - 1))
    assert _attend(cache=_host(**big)) == _select(cache=_host(**big)) == -2
    assert sp.lib.spiffy_page_summary(C.byref(_heads()), C.byref(_host(**big)), 1, C.byref(_layer()), None, None) == -2
    size = lambda kw: sp.lib.spiffy_pages_workspace_bytes(C.byref(_host(**kw)))
    assert size(big) == 0 and size(fits) > 0


def test_page_operations_refuse():
    one = (C.c_void_p * 1)(DUMMY)
    off = (C.c_void_p * 1)(DUMMY + 8)

    def append(cfg=None, cache=None, layer=None, **kw):
        d = dict(n=1, k=one, v=one, stride=256, start=DUMMY, T=5, mask=None, words=0, node=None, ns=1, status=None, ws=DUMMY, wn=1 << 40)
        d.update(kw)
        return sp.lib.spiffy_pages_append(C.byref(cfg or _heads()), C.byref(cache or _host()), d["n"], C.byref(layer or _layer()), d["k"], d["v"],
                                          d["stride"], d["start"], d["T"], d["mask"], d["words"], d["node"], d["ns"], d["status"], d["ws"], d["wn"], None)

    def fork(cfg=None, cache=None, layer=None, **kw):
        d = dict(n=1, src=DUMMY, dst=DUMMY, m=2, status=None, ws=DUMMY, wn=1 << 40)
        d.update(kw)
        return sp.lib.spiffy_pages_fork(C.byref(cfg or _heads()), C.byref(cache or _host()), d["n"], C.byref(layer or _layer()), d["src"], d["dst"], d["m"],
                                        d["status"], d["ws"], d["wn"], None)

    def compact(cfg=None, cache=None, layer=None, **kw):
        d = dict(n=1, used=None, ws=DUMMY, wn=1 << 40)
        d.update(kw)
        return sp.lib.spiffy_pages_compact(C.byref(cfg or _heads()), C.byref(cache or _host()), d["n"], C.byref(layer or _layer()), d["used"], d["ws"], d["wn"], None)

    free = lambda cache=None, seqs=DUMMY, n=1: sp.lib.spiffy_pages_free(C.byref(cache or _host()), seqs, n, None)
    for call in (append, fork, compact):
        for kw, want in BAD_CACHES + BAD_POINTERS:
            assert call(cache=_host(**kw)) == want, (call, kw)
        for kw, want in BAD_HEADS:
            assert call(cfg=_heads(**kw)) == want, (call, kw)
        for kw, want in [(dict(n=0), -1), (dict(n=257), -2), (dict(ws=None), -1), (dict(ws=DUMMY + 64), -3), (dict(wn=100), -4)]:
            assert call(**kw) == want, (call, kw)
        assert call(layer=_layer(k=None)) == -1 and call(layer=_layer(v=DUMMY + 8)) == -3 and call(layer=_layer(summary=DUMMY + 8)) == -3
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert free(cache=_host(**kw)) == want
    assert free(seqs=None) == -1 and free(n=0) == -1 and free(n=4097) == -2 and free(seqs=DUMMY + 2) == -3
    for kw, want in [(dict(k=None), -1), (dict(k=off), -3), (dict(v=off), -3), (dict(stride=255), -1), (dict(stride=260), -3), (dict(start=None), -1), (dict(T=0), -1),
                     (dict(T=(1 << 20) + 1), -2), (dict(mask=DUMMY, words=1), -1), (dict(node=DUMMY), -1), (dict(mask=DUMMY, words=0, node=DUMMY), -1),
                     (dict(mask=DUMMY, words=17, node=DUMMY), -2), (dict(mask=DUMMY, words=1, node=DUMMY, ns=0), -1), (dict(mask=DUMMY, words=1, node=DUMMY + 2), -3),
                     (dict(status=DUMMY + 2), -3), (dict(k=(C.c_void_p * 1)(None)), -1)]:
        assert append(**kw) == want, kw
    for kw, want in [(dict(src=None), -1), (dict(dst=None), -1), (dict(m=0), -1), (dict(m=4097), -2), (dict(src=DUMMY + 1), -3), (dict(status=DUMMY + 2), -3)]:
        assert fork(**kw) == want, kw
    assert compact(used=DUMMY + 2) == -3
    assert sp.lib.spiffy_pages_workspace_bytes(C.byref(_host())) > 0 and sp.lib.spiffy_pages_workspace_bytes(C.byref(_host(n_pages=0))) == 0


def _cpu_cache(**kw):
    """A PagedCache over CPU tensors: its checks run before anything is launched."""
    cfg = _cfg(BF, 4, 2, 16)
    t = dict(k=torch.zeros(2, 5, 2, 8, 16, dtype=BF), v=torch.zeros(2, 5, 2, 8, 16, dtype=BF), refs=torch.zeros(5, dtype=torch.int32),
             table=torch.zeros(3, 4, dtype=torch.int32), len=torch.zeros(3, dtype=torch.int32), summary=torch.zeros(2, 5, 2, 2, 16, dtype=BF))
    t.update(kw)
    return sp.PagedCache(cfg, t["k"], t["v"], t["refs"], t["table"], t["len"], summary=t["summary"])


def test_binding_checks_shapes_types_and_strides():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    for bad in (dict(k=torch.zeros(2, 5, 2, 8, 16)), dict(v=torch.zeros(2, 5, 2, 9, 16, dtype=BF)), dict(refs=i32(4)), dict(len=i32(4)), dict(table=i32(12)),
                dict(refs=torch.zeros(5, dtype=torch.int64)), dict(summary=torch.zeros(2, 5, 2, 16, dtype=BF)), dict(k=torch.zeros(2, 5, 1, 8, 16, dtype=BF)),
                dict(table=i32(4, 3).T)):
        with pytest.raises(ValueError):
            _cpu_cache(**bad)
    c = _cpu_cache()
    q, k, start = torch.zeros(6, 4, 16, dtype=BF), torch.zeros(6, 2, 16, dtype=BF), i32(4)
    for args, kw in [((q.float(), k, k, start, 3), {}), ((q, k[:5], k, start, 3), {}), ((q, k, k, i32(5), 3), {}), ((q[:, :3], k, k, start, 3), {}),
                     ((q, k, k, start, 3), dict(mask=torch.zeros(6, 1, dtype=torch.int32))), ((q, k, k, start, 3), dict(mask=torch.zeros(5, 1, dtype=torch.int64))),
                     ((q, k, k, start, 3), dict(selected=i32(3, 4, 2))), ((q, k, k, start, 3), dict(out=q[:5])), ((q, k, k.float(), start, 3), {}),
                     ((q, k, torch.zeros(6, 4, 16, dtype=BF)[:, :2], start, 3), {}), ((torch.zeros(6, 16, 4, dtype=BF).transpose(1, 2), k, k, start, 3), {})]:
        with pytest.raises(ValueError):
            c.attend(0, *args, **kw)
    with pytest.raises(IndexError):
        c.attend(2, q, k, k, start, 3)
    for call in (lambda: c.select(0, q, start, 0, 2), lambda: c.select(0, q, start, 1 << 32 | 3, 2), lambda: c.select(0, q, start, 3, 0),
                 lambda: c.select(0, q, start, 3, 2, keep_last=1 << 32), lambda: c.attend_workspace_bytes(1025), lambda: c.attend_workspace_bytes(1 << 32 | 3)):
        with pytest.raises(sp.SpiffyError):
            call()
    with pytest.raises(ValueError, match="not on a GPU"):      # host memory never reaches a kernel
        c.attend(0, q, k, k, start, 3)
    for call in (lambda: c.select(0, q, i32(3), 3, 2), lambda: c.select(0, q, start, 3, 2, out=i32(3, 2, 3)), lambda: c.summarize(i32(2)),
                 lambda: c.free(i32(2, 2)), lambda: c.fork(i32(2), i32(3)), lambda: c.fork(i32(2), i32(2), status=i32(1)),
                 lambda: c.append(k, k, start), lambda: c.append(k[None].repeat(2, 1, 1, 1), k[None].repeat(2, 1, 1, 1), start, node=i32(2)),
                 lambda: c.append(torch.zeros(2, 6, 2, 16), torch.zeros(2, 6, 2, 16), start)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sp.SpiffyError) as e:
        _cpu_cache(table=i32(4097, 4), len=i32(4097))
    assert e.value.status == sp.SPIFFY_ESHAPE
    # nothing to do is no error and launches nothing
    assert c.attend(0, q[:0], k[:0], k[:0], start, 3).shape == (0, 4, 16)
    c.free(i32(0))
    c.fork(i32(0), i32(0))
    c.append(torch.zeros(2, 0, 2, 16, dtype=BF), torch.zeros(2, 0, 2, 16, dtype=BF), start)


def test_tree_masks():
    m = sp.tree_mask([(0, 1), (0, 2), (2, 3), (1, 4)], 5, device="cpu")
    assert m[:, 0].tolist() == [1, 0b11, 0b101, 0b1101, 0b10011]
    chain = sp.tree_mask(torch.tensor([[i, i + 1] for i in range(99)]), 100, device="cpu")
    assert chain.shape == (100, 2) and chain[99].tolist() == [-1, (1 << 36) - 1] and chain[63].tolist() == [-1, 0]
    # several parents, edges in any order: all their ancestors
    assert sp.tree_mask([(2, 3), (1, 3), (0, 2)], 4, device="cpu")[:, 0].tolist() == [1, 0b10, 0b101, 0b1111]
    for bad in ([(1, 1)], [(2, 1)], [(0, 5)], [(-1, 1)]):
        with pytest.raises(ValueError):
            sp.tree_mask(bad, 5, device="cpu")


def test_plain_bookkeeping_stays_consistent():
    """The plain form itself: after any sequence of operations every page's count is the number of table entries that name it."""
    rng = random.Random(5)
    x = Setup(F32, 1, 1, 8, 4, [9, 0, 4, 0, 0, 2], [3, 3, 3, 3, 3, 3], spare=9, garbage=False)
    plain = x.plain()
    for _ in range(300):
        what = rng.randrange(4)
        if what == 0:
            plain.append(*x.all_rows(), x.start)
        elif what == 1:
            plain.fork([rng.randrange(6) for _ in range(3)], [rng.randrange(6) for _ in range(3)])
        elif what == 2:
            plain.free([rng.randrange(6)])
        else:
            assert plain.compact() == sum(r > 0 for r in plain.refs)
            assert all(r == 0 for r in plain.refs[plain.compact():])
        count = [0] * plain.n_pages
        for s in range(6):
            for j in range(plain.max_pages):
                assert (plain.table[s][j] >= 0) == (j < plain._used(s))
                if plain.table[s][j] >= 0:
                    count[plain.table[s][j]] += 1
        assert count == plain.refs


def test_host_checks_under_asan_and_ubsan():
    from paper_2509_18085_amd import build
    try:
        lib, rt = build.build_host_sanitized()
    except RuntimeError as e:
        pytest.skip("no sanitizer build: %s" % str(e)[:200])
    if not os.path.exists(rt):
        pytest.skip("no AddressSanitizer runtime to preload")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", SPIFFY_LIB=lib)
    env["LD_PRELOAD"] = " ".join(x for x in (rt, env.get("LD_PRELOAD", "")) if x)
    here = os.path.abspath(__file__)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", here, "-k", "refuse or binding"],
                       cwd=os.path.dirname(os.path.dirname(here)), env=env, capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-3000:]
    assert r.returncode == 0 and "passed" in r.stdout and "AddressSanitizer" not in tail and "runtime error" not in tail, tail
