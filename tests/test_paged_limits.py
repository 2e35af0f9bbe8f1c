"""The paged cache at the ends of what its calls take: pages of more rows than 32-bit offsets reach, scores of any size, calls without rows."""
import ctypes as C
import math
import os
import random
import shutil
import subprocess

import pytest
import torch

from paged_reference import Setup, mask_words
from paper_2509_18085_amd import build
from paper_2509_18085_amd import spiffy as sp

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
gpu = pytest.mark.gpu


def _cfg(dtype, Hq, Hkv, hd):
    return sp.make_cfg(d=Hq * hd, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=hd, ffn=8, vocab=2, mask_id=1, dtype=dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _host_program(tmp_path, text):
    """Compiles a program against the kernels' headers for the host alone and runs it; its output."""
    source, program = str(tmp_path / "p.hip"), str(tmp_path / "p")
    with open(source, "w") as f:
        f.write(text)
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    subprocess.run([hipcc, "-O1", "-std=c++17", "--offload-host-only", "-I", build.CSRC, source, "-o", program], check=True, capture_output=True, timeout=300)
    return subprocess.run([program], check=True, capture_output=True, text=True, timeout=120).stdout


def test_places_in_pages_of_more_than_2_24_rows(tmp_path):
    """Where a row lies in the pool, against 128-bit arithmetic: pages up to 2^31 - 1 rows, the last kv heads and rows among them."""
    out = _host_program(tmp_path, r"""
#include <cstdio>
#include "paged.h"
int main() {
  const int sizes[] = {1, 4, 48, (1 << 24) - 4, 1 << 24, (1 << 24) + 64, 1 << 25, 1 << 26, 1 << 30, 0x7fffffff};
  const unsigned heads[] = {0, 1, 7, 255, 4095, 1u << 20, 0x7fffffffu, 0xffffffffu};
  long long n = 0, bad = 0;
  for (int ps : sizes)
    for (unsigned h : heads)
      for (long long off : {0ll, 1ll, (1ll << 24) - 1, 1ll << 24, (1ll << 24) + 5, 1ll << 25, (long long)ps / 2, (long long)ps - 1})
        if (off < ps && (unsigned __int128)h * ps < ((unsigned __int128)1 << 55)) {
          ++n;
          for (int hd : {64, 128}) bad += spiffy::pool_row(h, ps, (int)off) * hd != (long long)(((unsigned __int128)h * ps + off) * hd);
        }
  printf("%lld %lld\n", n, bad);
}
""")
    n, bad = (int(x) for x in out.split())
    assert n > 300 and bad == 0, out


def test_pieces_of_pages_of_more_than_2_31(tmp_path):
    """The pieces that a thread copies, one after the other, against 128-bit arithmetic: few and many of a head, pages of up to 2^33
    pieces (128 GB of keys; the first and the last thread walk through them)."""
    out = _host_program(tmp_path, r"""
#include <cstdio>
#include "paged.h"
int main() {
  struct { long long heads, n, stride; } cases[] = {
      {8, 1, 1}, {3, 5, 16}, {4, 255, 256}, {4, 256, 256}, {4, 257, 1024}, {300, 1, 64}, {4096, 2, 16}, {2, 1023, 1024}, {2, 1024, 1024}, {2, 1025, 2048},
      {8, (1ll << 28) - 16, 1ll << 28}, {8, 1ll << 28, 1ll << 28}, {1, 1ll << 31, (1ll << 31) + 64}, {4, (1ll << 31) - 64, 1ll << 31}};
  long long walked = 0, bad = 0;
  for (auto& c : cases)
    for (int step : {256, 1024})
      for (int at : {0, 1, 37, 254, 255}) {
        const bool large = c.heads * c.n > 1 << 22;
        if (large && (step != 256 || (at && at != 255))) continue;
        spiffy::HeadPieces w(c.n, c.stride, at, step);
        for (__int128 u = at; u < (__int128)c.heads * c.n; u += step, w.next()) {
          ++walked;
          bad += w.place != (long long)(u / c.n * c.stride + u % c.n);
        }
        bad += w.place < c.heads * c.stride;             // the walk ends here
      }
  printf("%lld %lld\n", walked, bad);
}
""")
    walked, bad = (int(x) for x in out.split())
    assert walked > 1 << 26 and bad == 0, out


@gpu
@pytest.mark.parametrize("nodes", [1, 20, 70])
def test_attention_over_one_page_of_more_than_2_24_rows(nodes):
    """One page of one kv head, 4.3 GB of keys.  All rows but the last 61 have keys and values of zero, so their share of a softmax is
    their number; the last ones score 16 and some more."""
    ps, hd = (1 << 24) + 64, 128
    n, far = ps - 3, ps - 64
    gen = torch.Generator(device=DEV).manual_seed(2)
    k, v = (torch.zeros((1, 1, 1, ps, hd), dtype=BF, device=DEV) for _ in range(2))
    for t in (k, v):
        t[..., far:, :] = torch.randn((64, hd), generator=gen, device=DEV).to(BF)
    q = torch.randn((nodes, 1, hd), generator=gen, device=DEV).to(BF)
    q[..., 0], k[..., far:, 0] = 4.0, 4.0
    k[..., far:, 1:] *= 0.125
    k[..., n:, :] = float("nan")
    v[..., n:, :] = float("nan")
    new = torch.zeros((nodes, 1, hd), dtype=BF, device=DEV)
    cache = sp.PagedCache(_cfg(BF, 1, 1, hd), k, v, _ints([1]), _ints([[0]]), _ints([n]))
    got = cache.attend(0, q, new, new, _ints([0, nodes]), nodes, mask=torch.zeros((nodes, -(-nodes // 64)), dtype=torch.int64, device=DEV), scale=1.0)
    w = torch.exp(q[:, 0].double() @ k[0, 0, 0, far:n].double().T)
    want = w @ v[0, 0, 0, far:n].double() / (w.sum(1, keepdim=True) + far)
    # probabilities and the result are rounded to bf16 (2^-8 of |v| at most, and of the result); fp32 scores are off by less than 1e-4
    tol = 2.0 ** -8 * v[0, 0, 0, far:n].double().abs().amax() + 2.0 ** -8 * want.abs() + 1e-3
    assert ((got[:, 0].double() - want).abs() <= tol).all()
    assert want.abs().amax() > 0.1                           # not what zeros would give


# dtype, Hq, Hkv, hd, rows of a page, lengths, new rows: every kernel, in one piece and joined from units
LARGE = [
    (BF, 4, 2, 128, 16, [300, 33, 0], [1, 3, 2]),
    (BF, 4, 2, 128, 16, [3000, 33, 700], [9, 16, 2]),
    (BF, 4, 1, 80, 24, [900, 100], [13, 5]),
    (BF, 2, 1, 256, 16, [700, 40], [20, 3]),
    (BF, 2, 1, 128, 16, [1500, 60], [70, 66]),
    (BF, 2, 1, 64, 5, [700, 60], [64, 40]),
    (F32, 4, 2, 64, 24, [700, 33], [9, 3]),
    (F32, 2, 1, 128, 16, [200, 0], [5, 2]),
    (F32, 1, 1, 256, 16, [500, 10], [17, 3]),
]


@gpu
@pytest.mark.parametrize("case", LARGE, ids=str)
@pytest.mark.parametrize("size", [28, 29, 31, 36, 115])
@pytest.mark.parametrize("sign", ["mixed", "negative"])
def test_scores_of_any_finite_size(case, size, sign):
    """Scores of 0.75 times 2^size to 2^(size + 1), all exact in fp32 and 2^-7 of that apart or equal: a row gets the mean of the values
    of its highest keys.  Every highest key's probability is the same number, rounded to bf16 by 2^-8 of itself at most; the mean is rounded once
    more; the rest are sums in fp32."""
    dtype, Hq, Hkv, hd, ps, lens, nodes = case
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=size + hd)
    gen, rng = torch.Generator().manual_seed(size), random.Random(size)

    def keys(shape):
        y = (1 + torch.randint(0, 128, shape, generator=gen) / 128) * 2.0 ** (size - size // 2)
        return y * (torch.randint(0, 2, shape, generator=gen) * 2 - 1) if sign == "mixed" else -y

    one = torch.zeros_like(x.k)
    one[..., 3] = keys(x.k.shape[:-1]).to(dtype)
    x.k = torch.where(x.k.isnan(), x.k, one)
    x.qkv[:, :, :Hq + Hkv] = 0
    x.qkv[:, :, :Hq, 3] = 2.0 ** (size // 2)
    x.qkv[:, :, Hq:Hq + Hkv, 3] = keys((1, x.T, Hkv)).to(dtype)
    words = -(-max(nodes) // 64)
    rows = [rng.getrandbits(64 * words) | 1 << i for n in nodes for i in range(n)]
    want = x.plain().attend(0, *x.rows(0), x.start, rows, scale=0.75)
    cache = sp.PagedCache(_cfg(dtype, Hq, Hkv, hd), *(t.to(DEV) for t in (x.k, x.v, x.refs, x.table, x.len)))
    got = cache.attend(0, *x.rows(0, DEV), _ints(x.start), max(nodes), mask=mask_words(rows, words).to(DEV), scale=0.75).double().cpu()
    assert torch.isfinite(got).all()
    tol = 2.0 ** -20 * 6 + want.abs() * (0 if dtype == F32 else 2.0 ** -7 * (1 + 2.0 ** -8))
    assert ((got - want).abs() <= tol).all(), float((got - want).abs().max())


@gpu
@pytest.mark.parametrize("case", LARGE, ids=str)
def test_rows_of_large_scores_leave_other_rows_as_they_are(case):
    """Rows beside one another in a kernel: those whose queries are 2^40 times as large change no bit of the
    others' results."""
    dtype, Hq, Hkv, hd, ps, lens, nodes = case
    x = Setup(dtype, Hq, Hkv, hd, ps, lens, nodes, seed=5 + hd)
    cache = sp.PagedCache(_cfg(dtype, Hq, Hkv, hd), *(t.to(DEV) for t in (x.k, x.v, x.refs, x.table, x.len)))
    run = lambda: cache.attend(0, *x.rows(0, DEV), _ints(x.start), max(nodes))
    want = run()
    large = torch.arange(x.T) % 3 == 1
    x.qkv[:, large, :Hq] *= 2.0 ** 40
    got = run()
    assert torch.equal(got[~large.to(DEV)], want[~large.to(DEV)]) and torch.isfinite(got).all()
    assert not torch.equal(got, want)


@gpu
def test_the_documented_steps_leave_every_summary_up_to_date():
    """The example of the README as it stands, its step twice: what `select` will read is the least and greatest key of every page in use."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        lines = f.read().split("\n")
    first = next(i for i, x in enumerate(lines) if "PagedCache.empty" in x)
    block = []
    for x in lines[first:]:
        if not x.startswith("    "):
            break
        block.append(x[4:])
    step = next(i for i, x in enumerate(block) if x.startswith("mask ="))
    n_layers, Hq, Hkv, hd, ps, n = 2, 4, 2, 64, 4, 11
    rows = torch.randn((n_layers, n, Hq + 2 * Hkv, hd), generator=torch.Generator().manual_seed(3)).to(DEV, BF)
    env = dict(torch=torch, spiffy=sp, cfg=_cfg(BF, Hq, Hkv, hd), n_layers=n_layers, n_pages=40, page_size=ps, n_seqs=2, max_pages=20, layer=1, max_rows=n, n_sel=3,
               k_rows=rows[:, :, Hq:Hq + Hkv], v_rows=rows[:, :, Hq + Hkv:], q=rows[1, :, :Hq], k=rows[1, :, Hq:Hq + Hkv], v=rows[1, :, Hq + Hkv:],
               row_start=_ints([0, n, n]), src=_ints([0]), dst=_ints([1]), trees=[([(i, i + 1) for i in range(n - 1)], n)],
               results=_ints([[n - 1, 0, 0, 0], [-1, 0, 0, 0]]))
    exec("\n".join(block[:step]), env)
    for i in range(2):
        rows.copy_(rows.flip(1) * 1.5)
        exec("\n".join(block[step:]), env)
        cache = env["cache"]
        assert cache.len.tolist() == [n * (i + 2), n]
        for s, length in enumerate(cache.len.tolist()):
            for j in range(-(-length // ps)):
                p, used = int(cache.table[s, j]), min(ps, length - j * ps)
                keys = cache.k[:, p, :, :used].float()
                assert torch.equal(cache.summary[:, p].float(), torch.stack([keys.amin(2), keys.amax(2)], 2)), (i, s, j)


@gpu
def test_append_of_no_rows_reports():
    """Every status is written, as by a call in which no sequence has rows; the cache stays."""
    cache = sp.PagedCache.empty(_cfg(F32, 4, 2, 16), 2, 6, 4, 3, 5, device=DEV)
    cache.append(*torch.ones((2, 2, 5, 2, 16), device=DEV), _ints([0, 5, 5, 5]))
    none, kept = torch.zeros((2, 0, 2, 16), device=DEV), [t.clone() for t in (cache.k, cache.v, cache.refs, cache.table, cache.len)]
    for stream in (None, torch.cuda.Stream()):
        for start in ([0, 0, 0, 0], [0, 2, 2, 7]):                # row starts are taken within the rows that there are
            status = _ints([9, 9, 9])
            torch.cuda.synchronize()
            cache.append(none, none, _ints(start), status=status, stream=stream)
            torch.cuda.synchronize()
            assert status.tolist() == [sp.PAGES_DONE] * 3
            for words in (0, 1):
                status.fill_(9)
                torch.cuda.synchronize()
                cache.append(none, none, _ints(start), mask=torch.zeros((0, words), dtype=torch.int64, device=DEV), node=_ints([-1, 0, -1]), status=status, stream=stream)
                torch.cuda.synchronize()
                assert status.tolist() == [sp.PAGES_DONE, sp.PAGES_BAD, sp.PAGES_DONE]
    for t, was in zip((cache.k, cache.v, cache.refs, cache.table, cache.len), kept):
        assert torch.equal(t.nan_to_num(), was.nan_to_num())


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_selection_of_an_empty_batch_takes_row_starts_within_it(dtype):
    """No rows: by index alone, whatever row_start says, also where a row of zeros would tell pages apart (a page that is not there)."""
    cache = sp.PagedCache.empty(_cfg(dtype, 4, 2, 16), 1, 9, 4, 2, 8, summaries=True, device=DEV)
    rows = torch.ones((1, 50, 2, 16), dtype=dtype, device=DEV)
    cache.append(rows, rows, _ints([0, 30, 32]))
    cache.summarize()
    cache.table[0, 1] = -1
    q = torch.zeros((0, 4, 16), dtype=dtype, device=DEV)
    for start in ([0, 0, 0], [0, 1, 1], [0, 0, 1], [0, 3, 9]):
        got = cache.select(0, q, _ints(start), 3, 3, keep_first=1, keep_last=1)
        assert got.tolist() == [[[0, 1, 7]] * 2, [[0, -1, -1]] * 2], start


# ---- arguments (no GPU) -----------------------------------------------------------------------------------------------------


def _cpu_cache():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    return sp.PagedCache(_cfg(BF, 4, 2, 16), torch.zeros(2, 5, 2, 8, 16, dtype=BF), torch.zeros(2, 5, 2, 8, 16, dtype=BF), i32(5), i32(3, 4), i32(3),
                         summary=torch.zeros(2, 5, 2, 2, 16, dtype=BF))


def test_workspaces_count_the_bytes_that_they_have():
    """From the next multiple of 256 on: a view that ends in front of it has none (and no number that reads as a huge one), elements of any
    size, and no tensor whose elements share memory."""
    cache, base = _cpu_cache(), torch.zeros(4096, dtype=torch.uint8)
    skip = -base.data_ptr() % 256
    for first, n in ((0, 0), (8, 8), (8, 247), (8, 248), (8, 249), (0, 600), (256, 1000)):
        view = base[skip + first:skip + first + n]
        want = max(0, n - -first % 256)
        for p, have in (sp._ws(view), cache._scratch(1, view)[1:]):
            assert have == want and (n == 0 or p == base.data_ptr() + skip + first + -first % 256), (first, n)
    wide = torch.zeros(1024, dtype=torch.float32)
    assert sp._ws(wide)[1] == cache._scratch(1, wide)[2] == 4096 - -wide.data_ptr() % 256
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(4096), base[::2]):
        for call in (lambda: sp._ws(bad), lambda: cache._scratch(1, bad)):
            with pytest.raises(ValueError):
                call()


def _attend_status(scale):
    fake = 0x10000                                            # never reached: the call ends at its checks, a workspace of no bytes the last of them
    return sp.lib.spiffy_tree_attention(C.byref(_cfg(BF, 8, 2, 128)), C.byref(sp.PagedCacheStruct(10, 16, 3, 7, fake, fake, fake)), C.byref(sp.PageLayer(fake, fake, None)),
                                        fake, 1024, fake, fake, 256, fake, 5, 5, None, 0, None, 0, scale, fake, 1024, fake, 0, None)


def test_a_scale_whose_base_2_form_is_not_finite_is_refused():
    for scale in (2.4e38, -2.4e38, 3.4e38, math.inf, math.nan):
        assert _attend_status(scale) == sp.SPIFFY_EINVAL, scale
    for scale in (2.3e38, -2.3e38, 1.0, 0.0, 1e-45):
        assert _attend_status(scale) == sp.SPIFFY_EWORKSPACE, scale


def test_a_mask_of_no_words_is_refused():
    """It has no address, and without a mask a row attends to every new row of its sequence."""
    c, start = _cpu_cache(), torch.zeros(4, dtype=torch.int32)
    q, k, mask = torch.zeros(6, 4, 16, dtype=BF), torch.zeros(6, 2, 16, dtype=BF), torch.zeros(6, 0, dtype=torch.int64)
    with pytest.raises(ValueError, match="mask"):
        c.attend(0, q, k, k, start, 3, mask=mask)
    rows = torch.zeros(2, 6, 2, 16, dtype=BF)
    with pytest.raises(ValueError, match="mask"):
        c.append(rows, rows, start, mask=mask, node=torch.zeros(3, dtype=torch.int32))
    assert c.attend(0, q[:0], k[:0], k[:0], start, 3, mask=mask[:0]).shape == (0, 4, 16)


def test_masks_of_small_and_large_trees_lie_one_behind_the_other():
    trees = [([(i, i + 1) for i in range(n - 1)], n) for n in (3, 64, 65, 130, 1)]
    masks = [sp.tree_mask(e, n, device="cpu", words=3) for e, n in trees]
    both = torch.cat(masks)
    assert both.shape == (263, 3)
    for m, (e, n) in zip(masks, trees):
        own = sp.tree_mask(e, n, device="cpu")
        assert torch.equal(m[:, :own.shape[1]], own) and not m[:, own.shape[1]:].any()
    with pytest.raises(ValueError):
        sp.tree_mask([], 65, device="cpu", words=1)


def test_a_stream_of_another_device_is_refused():
    """Otherwise the call would run on the current stream of the cache's device, in no order with the stream that it was given."""
    class Elsewhere:
        device, cuda_stream = torch.device("cuda", 1), 0x10000

    cache, called = _cpu_cache(), []
    cache.device = torch.device("cuda", 0)
    with pytest.raises(ValueError, match="stream"):
        cache._there(Elsewhere(), called.append, 1)
    assert not called


def test_a_selection_of_no_pages_is_refused():
    """It has no address, and without a selection every page is read."""
    c, start = _cpu_cache(), torch.zeros(4, dtype=torch.int32)
    q, k, chosen = torch.zeros(6, 4, 16, dtype=BF), torch.zeros(6, 2, 16, dtype=BF), torch.zeros(3, 2, 5, dtype=torch.int32)
    assert chosen[:, :, :0].contiguous().data_ptr() == 0
    with pytest.raises(ValueError, match="selected"):
        c.attend(0, q, k, k, start, 3, selected=chosen[:, :, :0].contiguous())


def test_only_the_widest_kernels_of_the_paged_cache_use_scratch_memory():
    """bf16 heads of more than 128 channels in two row tiles have more accumulators than registers (they spill around the steps over new rows)."""
    found = {k for s in build.SOURCES if s.startswith("paged_") for k, n in build.scratch_bytes(s).items() if n}
    assert len(found) == 2 and all("tree_attn_kernelIDF16bLi256ELi2E" in k for k in found), found
