"""Caches of 8-bit codes: cells written and read back, sessions copied in and out, attention over
them, decode steps that append.

What is written is compared with the definition bit for bit: scales are powers of two, so a
quotient is exact, its rounding to a code is the definition's, and a code times its scale is
exact in 32 bits and in bf16.

The attention is compared with the formula in 64 bits over the values that the codes stand for.  Its
bound, with u = 2^-24: a score is off by at most A (dh + 4) u through its fp32 sum, A the largest sum
of |q k| scale, and by A 2^-17 more where q goes through two bf16 parts (each leaves at most 2^-9 of
what it rounds, twice 2^-18 in all); a probability is off by that, by the exponential's 2^-21 and by 2^-11 where the
output is bf16 (one fp16 rounding at the most), else by 2^-17; the sums over n cells by n u each.  The output is a
quotient of two such sums, so it is off by at most twice their relative errors times the
largest |v|, and then rounded to its type once."""
import math

import numpy as np
import pytest

import synth
from gpu_util import build_model, fill_synthetic_kv, log, max_abs, read_kv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
Q = {"i8": 127.0, "e4m3": 448.0}
BLOCK = 16


# ---- the definition, in 64 bits on the host ---------------------------------------------------


def _scale(top, code):
    """The smallest power of two s with top / s <= Q, at least 2^-100 (NaN for what is not finite)."""
    s = np.full_like(top, 2.0 ** -100)
    for _ in range(240):
        s = np.where(s * Q[code] < top, 2 * s, s)
    return np.where(np.isfinite(top), s, np.nan)


def _round(y, code):
    """y to the nearest code's value, ties to even."""
    if code == "i8":
        return np.rint(y)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.rint(y / step) * step


class Cache:
    """Values and scales of sequences of cells [cell][head][dim], blocks of 16 from cell 0."""

    def __init__(self, n, cells, nkv, dh, code):
        self.x = [np.zeros((n, cells, nkv, dh)) for _ in range(2)]          # K, V
        self.s = [np.zeros((n, cells // BLOCK, nkv)) for _ in range(2)]
        self.code = code

    def write(self, seq, first, k, v):
        if not len(k):
            return
        with np.errstate(all="ignore"):
            for which, rows in ((0, k), (1, v)):
                for b in range(first - first % BLOCK, first + len(rows), BLOCK):
                    lo, hi = max(b, first), min(b + BLOCK, first + len(rows))
                    new = rows[lo - first:hi - first].astype(np.float64)
                    fine = np.isfinite(new).all(axis=(0, 2))
                    s = _scale(np.where(fine, np.abs(np.nan_to_num(new)).max(axis=(0, 2)), np.inf), self.code)
                    if lo > b:
                        s = np.maximum(s, self.s[which][seq, b // BLOCK])   # (NaN stays NaN)
                        kept = self.x[which][seq, b:lo]
                        self.x[which][seq, b:lo] = _round(kept / s[:, None], self.code) * s[:, None]
                    self.s[which][seq, b // BLOCK] = s
                    self.x[which][seq, lo:hi] = _round(new / s[:, None], self.code) * s[:, None]


def _views(torch, pool, pages):
    """Codes of K [page, layer, head, cell, dim] and V [page, layer, head, dim, cell], scales of both
    [page, layer, head, block], as the pool's layouts say."""
    c, lay, sc = pool.cfg, pool.page_layout(), pool.scale_layout()
    fmt = torch.int8 if c.dtype == 8 else torch.float8_e4m3fn
    n, L, H, P, D = c.n_pages, c.n_layers, c.n_kv_heads, c.page_cells, c.head_dim
    assert lay.elem_bytes == 1 and sc.block_cells == BLOCK and lay.page_stride == L * lay.layer_stride
    at = lambda off, shape, strides, dt, e: torch.as_strided(  # noqa: E731
        pages.view(dt), shape, [lay.page_stride // e, lay.layer_stride // e, *strides], off // e)
    k = at(0, (n, L, H, P, D), list(lay.k_stride), fmt, 1)
    v = at(lay.v_offset, (n, L, H, D, P), [lay.v_stride[0], lay.v_stride[2], lay.v_stride[1]], fmt, 1)
    ks = at(sc.k_offset, (n, L, H, P // BLOCK), list(sc.stride), torch.float32, 4)
    vs = at(sc.v_offset, (n, L, H, P // BLOCK), list(sc.stride), torch.float32, 4)
    return k, v, ks, vs


def _scales(torch, pool, pages, layer):
    return [t[:, layer].cpu().numpy() for t in _views(torch, pool, pages)[2:]]


def _pool(torch, spp, layers, nkv, dh, code, page, n_pages, seed=0, max_seqs=64, fill=None):
    """A pool whose pages hold normal cells (or the byte `fill`)."""
    probe = spp.spp_pool_config(layers, nkv, dh, spp.CELL_CODES[code], page, n_pages, max_seqs)
    import ctypes
    nbytes = spp.lib().spp_pool_bytes(ctypes.byref(probe))
    pages = torch.full((nbytes,), 0 if fill is None else fill, dtype=torch.uint8, device="cuda")
    pool = spp.PagePool(layers, nkv, dh, True, page, n_pages, max_seqs=max_seqs, pages=pages, cells=code)
    g = torch.Generator(device="cuda").manual_seed(77 + seed)
    if fill is None:
        k, v, ks, vs = _views(torch, pool, pages)
        for t in (k, v):
            x = torch.empty(t.shape, device="cuda").normal_(0, 32 if code == "i8" else 80, generator=g)
            t.view(torch.uint8).copy_((x.round().clamp(-127, 127).to(torch.int8) if code == "i8" else x.to(t.dtype)).view(torch.uint8))
        for s in (ks, vs):
            s.copy_(torch.exp2(torch.randint(-8, -2, s.shape, generator=g, device="cuda").float()))
    return pool, pages, g


def _values(torch, pool, pages, layer):
    """K and V of a layer as values [page, head, cell, dim], fp64 on the host."""
    k, v, ks, vs = (t[:, layer] for t in _views(torch, pool, pages))
    k = k.contiguous().cpu().double() * ks.cpu().double().repeat_interleave(BLOCK, 2)[..., None]
    v = v.contiguous().cpu().double() * vs.cpu().double().repeat_interleave(BLOCK, 2)[:, :, None]
    return k, v.transpose(2, 3)


# ---- writing and reading ------------------------------------------------------------------------


WRITES = [
    # nkv, dh, code, io bf16, page, [spans of one call: (first, count) by sequence]...
    (1, 64, "i8", True, 16, [[(0, 1)], [(1, 1)], [(2, 13)], [(15, 1)], [(16, 1)], [(17, 40)]]),
    (2, 64, "e4m3", True, 16, [[(0, 5), (0, 33)], [(5, 1), (33, 1)], [(6, 60), (34, 0)]]),
    (8, 128, "i8", True, 64, [[(0, 100), (0, 64), (0, 17)], [(100, 1), (64, 1), (17, 1)], [(101, 27), (65, 130), (18, 1)]]),
    (4, 64, "i8", False, 32, [[(3, 30), (31, 2)], [(33, 1), (33, 1)]]),
    (3, 128, "e4m3", False, 128, [[(0, 129)], [(129, 1)], [(130, 100)]]),
    (2, 128, "e4m3", True, 256, [[(250, 20), (0, 1)], [(270, 2), (1, 1)]]),
    (5, 64, "e4m3", True, 64, [[(0, 1)] * 9, [(1, 1)] * 9, [(2, 1)] * 9]),
    # long spans that start and end anywhere in 64 cells
    (2, 64, "i8", True, 16, [[(0, 50), (0, 63)], [(50, 65), (63, 66)], [(115, 64), (129, 127)], [(179, 1), (256, 129)]]),
    (3, 128, "e4m3", False, 32, [[(47, 385), (0, 0), (63, 386)], [(432, 384), (63, 3), (449, 66)]]),
    (1, 64, "e4m3", True, 64, [[(63, 386)], [(449, 450)], [(899, 384)]]),
    (2, 64, "i8", True, 256, [[(0, 383), (0, 384)], [(383, 130), (384, 641)]]),
]


@pytest.mark.parametrize("nkv,dh,code,io_bf16,page,calls", WRITES)
def test_cells_written_are_the_definition(nkv, dh, code, io_bf16, page, calls):
    import torch
    import paper_2606_29565_amd as spp
    n = len(calls[0])
    most = max(f + c for spans in calls for f, c in spans)
    width = -(-most // page) + 1
    pool, pages, g = _pool(torch, spp, 2, nkv, dh, code, page, n * width + 1, seed=page + dh)
    table = torch.randperm(n * width + 1, generator=g, device="cuda")[:n * width].view(n, width).int()
    T = table.cpu().numpy()
    kv0, vv0 = _values(torch, pool, pages, 1)
    ks0, vs0 = _scales(torch, pool, pages, 1)
    cache = Cache(n, width * page, nkv, dh, code)
    for i in range(n):  # what the pages held before
        for x, was, s, old in ((cache.x[0], kv0, cache.s[0], ks0), (cache.x[1], vv0, cache.s[1], vs0)):
            x[i] = was[T[i]].transpose(1, 2).reshape(width * page, nkv, dh).numpy()
            s[i] = old[T[i]].transpose(0, 2, 1).reshape(-1, nkv)
    other = pages.clone()
    r = np.random.RandomState(3)
    dt = torch.bfloat16 if io_bf16 else torch.float32
    for spans in calls:
        first = torch.tensor([f for f, _ in spans], dtype=torch.int32, device="cuda")
        rows = torch.tensor(np.concatenate([[0], np.cumsum([c for _, c in spans])]), dtype=torch.int32, device="cuda")
        total = int(rows[-1])
        size = 2.0 ** r.uniform(-8, 6, (total, nkv, 1))                  # scales grow now and then
        k, v = (torch.from_numpy(r.randn(total, nkv, dh) * size).to("cuda", dt) for _ in range(2))
        cells = spp.PagedCells(pool, 1, table, first, rows, max(c for _, c in spans), io_bf16=io_bf16)
        cells.write(k, v)
        at = 0
        for i, (f, c) in enumerate(spans):
            cache.write(i, f, k[at:at + c].double().cpu().numpy(), v[at:at + c].double().cpu().numpy())
            at += c
        # everything up to the sequences' ends, read back
        ends = torch.tensor([f + c for f, c in spans], dtype=torch.int32)
        back = torch.cat([torch.zeros(1, dtype=torch.int32), ends.cumsum(0).int()]).cuda()
        out = [torch.full((int(back[-1]) + 2, nkv, dh), 7.0, dtype=dt, device="cuda") for _ in range(2)]
        spp.PagedCells(pool, 1, table, torch.zeros_like(first), back, int(ends.max()), io_bf16=io_bf16).read(*out)
        for which, got in enumerate(out):
            want = np.concatenate([cache.x[which][i, :f + c] for i, (f, c) in enumerate(spans)])
            assert np.array_equal(got[:-2].double().cpu().numpy(), want), (which, spans)
            assert bool((got[-2:] == 7).all())                           # rows behind the last sequence
        # scales where they lie
        ks, vs = _scales(torch, pool, pages, 1)
        for s, want in ((ks, cache.s[0]), (vs, cache.s[1])):
            for i, (f, c) in enumerate(spans):
                nb = -(-(f + c) // BLOCK)
                assert np.array_equal(s[T[i]].transpose(0, 2, 1).reshape(-1, nkv)[:nb], want[i, :nb])
    # the other layer and the page of no table stay as they were
    half = pages.numel() // (n * width + 1) // 2
    assert torch.equal(pages.view(-1, 2, half)[:, 0], other.view(-1, 2, half)[:, 0])
    spare = sorted(set(range(n * width + 1)) - set(T.reshape(-1).tolist()))[0]
    assert torch.equal(pages.view(-1, 2, half)[spare], other.view(-1, 2, half)[spare])


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_borders_ties_zeros_and_extremes(code):
    """Values at, below and above the border of a scale, ties between codes, blocks of zeros, the
    smallest and largest magnitudes, subnormal codes."""
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, _ = _pool(torch, spp, 1, 1, 64, code, 16, 40)
    q = Q[code]
    rows = []
    for top in (q, np.nextafter(np.float32(q), np.float32(1e9)), np.nextafter(np.float32(q), np.float32(0)), 1.0,
                2.0 ** -120, 2.0 ** -140, 0.0, 1.9921875 * 2.0 ** 126, 3.0, 2.0 ** -93 * q, q * 2.0 ** -100 * 1.5, 255.0):
        block = np.zeros((BLOCK, 1, 64), np.float32)
        block[0, 0, 0] = top
        block[1, 0, :] = top / 127 * (np.arange(64) - 31.5)          # halves: ties in i8
        block[2, 0, :] = top / 448 * 2.0 ** -np.arange(64).clip(0, 20)
        block[3, 0, :] = -top / 448 * 2.0 ** -8 * (np.arange(64) / 4)  # ties among subnormal codes
        rows.append(np.clip(block, -top, top))
    x = np.concatenate(rows).astype(np.float32)
    n = len(x)
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda").view(1, -1)
    z = torch.zeros(1, dtype=torch.int32, device="cuda")
    cells = spp.PagedCells(pool, 0, table, z, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, io_bf16=False)
    k = torch.from_numpy(x).cuda()
    cells.write(k, -k)
    gk, gv = cells.read(torch.empty_like(k), torch.empty_like(k))
    want = Cache(1, n, 1, 64, code)
    want.write(0, 0, x, -x)
    assert np.array_equal(gk.double().cpu().numpy(), want.x[0][0]) and np.array_equal(gv.double().cpu().numpy(), want.x[1][0])


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_infinities_and_nan_make_their_block_nan(code):
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 64, code, 32, 4)
    table = torch.tensor([[2, 0]], dtype=torch.int32, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.empty(40, 2, 64, device="cuda").normal_(generator=g)
    v = k.flip(0).contiguous()
    k[3, 1, 5], v[20, 0, 63] = float("inf"), float("nan")
    spp.PagedCells(pool, 0, table, i32(0), i32(0, 40), 40, io_bf16=False).write(k, v)
    read = spp.PagedCells(pool, 0, table, i32(0), i32(0, 40), 40, io_bf16=False)
    gk, gv = (t.clone() for t in read.read(torch.empty_like(k), torch.empty_like(v)))
    bad_k, bad_v = torch.isnan(gk), torch.isnan(gv)
    want_k, want_v = torch.zeros_like(bad_k), torch.zeros_like(bad_v)
    want_k[:16, 1], want_v[16:32, 0] = True, True
    assert torch.equal(bad_k, want_k) and torch.equal(bad_v, want_v)
    # appending to such a block leaves it so; writing it from its first cell makes it whole
    ones = torch.ones(1, 2, 64, device="cuda")
    spp.PagedCells(pool, 0, table, i32(15), i32(0, 1), 1, io_bf16=False).write(ones, ones)
    assert bool(torch.isnan(read.read(torch.empty_like(k), torch.empty_like(v))[0][:16, 1]).all())
    again = torch.ones(16, 2, 64, device="cuda")
    spp.PagedCells(pool, 0, table, i32(0), i32(0, 16), 16, io_bf16=False).write(again, again)
    assert bool((read.read(torch.empty_like(k), torch.empty_like(v))[0][:16] == 1).all())


def test_what_a_write_and_a_read_leave_out():
    """Negative starts and rows, rows past n_rows and max_cells, cells past the table, pages that are not
    listed; strided rows."""
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 64, "i8", 16, 20)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(4, 3)
    table[1, 1] = -1
    table[2, 1] = 20
    before = pages.clone()
    wide = torch.empty(60, 6, 64, device="cuda").normal_(generator=g).bfloat16()
    k, v = wide[:, 1:3], wide[:, 3:5]
    # nothing at all
    for first, rows, most in (((-1, -5, -2 ** 31, -1), (0, 9, 18, 27, 36), 9), ((0, 0, 0, 0), (60, 60, 60, 60, 60), 9),
                              ((0, 0, 0, 0), (-9, -8, -7, -6, -5), 9), ((48, 2 ** 31 - 1, 49, 2 ** 30), (0, 9, 18, 27, 36), 9),
                              ((0, 0, 0, 0), (9, 7, 5, 3, -2 ** 31), 9)):
        spp.PagedCells(pool, 0, table, i32(*first), i32(*rows), most).write(k, v)
        assert torch.equal(pages, before), (first, rows)
    # sequence 0 cut by max_cells, 1 and 2 with a page missing, 3 past its table and past n_rows
    first, rows = i32(14, 10, 0, 40), i32(0, 20, 32, 48, 70)
    c = spp.PagedCells(pool, 0, table, first, rows, 16)
    c.write(k, v)
    out = torch.full((60, 6, 64), 5.0, device="cuda").bfloat16()
    ok, ov = out[:, 1:3], out[:, 3:5]
    c.read(ok, ov)
    live = torch.zeros(60, dtype=torch.bool)
    live[:16] = True            # sequence 0: 16 of its 20 rows
    live[20:26] = True          # sequence 1: cells 10 .. 15, then its missing page
    live[32:48] = True          # sequence 2: cells 0 .. 15
    live[48:56] = True          # sequence 3: cells 40 .. 47
    zero = torch.zeros(60, dtype=torch.bool)
    zero[26:32] = True          # (cells 16 .. 21 of sequence 1 read as zeros)
    got = ok.float().cpu()
    assert bool((got[zero] == 0).all()) and bool((got[~live & ~zero] == 5).all())
    assert bool((out[:, 0] == 5).all()) and bool((out[:, 5] == 5).all())
    # half a step: new blocks of normal cells, max |x| below 8, have scales of at most 2^-4, but the cells that
    # a block kept have up to 2^-3, the largest that _pool gives, and new cells share it
    step = 2.0 ** -3
    assert float((got - k.float().cpu())[live].abs().max()) <= step / 2
    assert float((ov.float().cpu() - v.float().cpu())[live].abs().max()) <= step / 2
    # pages of no sequence
    lay = pool.page_layout().page_stride
    assert torch.equal(pages[12 * lay:], before[12 * lay:])


def test_written_and_read_from_a_graph():
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 128, "e4m3", 32, 16)
    eager_pool, eager_pages, _ = _pool(torch, spp, 1, 2, 128, "e4m3", 32, 16)
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    first, rows = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (3, 4))
    k, v = (torch.empty(30, 2, 128, device="cuda").bfloat16() for _ in range(2))
    ok, ov = torch.empty_like(k), torch.empty_like(v)
    c = spp.PagedCells(pool, 0, table, first, rows, 10)
    e = spp.PagedCells(eager_pool, 0, table, first, rows, 10)
    c.write(k, v)
    torch.cuda.synchronize()
    pages.copy_(eager_pages)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.write(k, v)
        c.read(ok, ov)
    at = torch.tensor([0, 3, 30], dtype=torch.int32)
    for counts in ((10, 1, 7), (1, 1, 1), (5, 10, 9), (1, 0, 1)):
        first.copy_(at)
        rows.copy_(torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32))
        for t in (k, v):
            t.copy_(torch.empty(t.shape, device="cuda").normal_(generator=g))
        ok.zero_(), ov.zero_()
        graph.replay()
        torch.cuda.synchronize()
        gk, gv = ok.clone(), ov.clone()
        e.write(k, v)
        wk, wv = e.read(torch.zeros_like(k), torch.zeros_like(v))
        assert torch.equal(gk, wk) and torch.equal(gv, wv)
        at += torch.tensor(counts, dtype=torch.int32)


# ---- attention --------------------------------------------------------------------------------


def _reference(torch, pool, pages, layer, nq, table, lengths, q, scale):
    """(output in 64 bits, largest sum of |q k| scale, largest |v|) over the live cells."""
    c = pool.cfg
    n, nkv, dh, page = q.shape[0], c.n_kv_heads, c.head_dim, c.page_cells
    G = nq // nkv
    out = torch.zeros(n, nq, dh, dtype=torch.float64)
    A = vmax = 0.0
    KV = _values(torch, pool, pages, layer)
    for i in range(n):
        at = np.arange(max(0, min(int(lengths[i]), table.shape[1] * page)))
        pg = table[i][at // page] if at.size else at
        ok = (pg >= 0) & (pg < c.n_pages)
        at, pg = at[ok], pg[ok]
        if not at.size:
            continue
        pgt, cell = torch.from_numpy(pg.astype(np.int64)), torch.from_numpy(at % page)
        K, V = KV[0][pgt, :, cell], KV[1][pgt, :, cell]                    # [cells, nkv, dh]
        for h in range(nq):
            k, v, qq = K[:, h // G], V[:, h // G], q[i, h].double().cpu()
            z = (k * qq).sum(1) * scale
            A = max(A, float((k * qq).abs().nan_to_num().sum(1).max()) * abs(scale))
            vmax = max(vmax, float(v.abs().nan_to_num().max()))
            p = torch.exp(z - z.max())
            out[i, h] = (p[:, None] * v).sum(0) / p.sum()
    return out, A, vmax


def _bound(A, vmax, dh, n, io_bf16, want):
    score = A * ((dh + 4) * U + (0.0 if io_bf16 else 2.0 ** -17))
    prob = score + 2.0 ** -21 + (2.0 ** -11 if io_bf16 else 2.0 ** -17)
    return 2 * (prob + n * U) * vmax + want.abs() * (2.0 ** -8 if io_bf16 else U) + 1e-30


CASES = [
    # nq, nkv, dh, code, io bf16, page, lengths, holes
    (4, 4, 64, "i8", False, 16, [1, 15, 16, 17, 63, 64, 65, 512], 0.0),
    (4, 2, 64, "e4m3", True, 16, [1, 2, 31, 32, 33, 127, 128, 129, 700], 0.0),
    (4, 2, 64, "i8", True, 32, [5, 0, 300, 1, 0, 1000], 0.3),
    (32, 8, 128, "i8", True, 64, [1, 8191, 4097], 0.0),
    (32, 8, 128, "e4m3", False, 128, [3, 130, 2049], 0.0),
    (64, 8, 128, "e4m3", True, 256, [600, 255, 257], 0.0),
    (20, 1, 128, "i8", True, 16, [40, 5000], 0.2),          # a second tile of 4 heads
    (40, 1, 64, "e4m3", False, 16, [77, 1, 300], 0.0),      # three tiles
    (6, 2, 64, "i8", True, 64, [129, 64], 0.0),
    (8, 8, 128, "i8", False, 16, [33, 200], 0.5),
    (16, 1, 64, "e4m3", False, 64, [16385], 0.0),
    (12, 4, 128, "i8", False, 64, [1, 500, 4500], 0.1),
    (32, 8, 128, "e4m3", False, 16, [700] * 20 + [1, 0, 1007], 0.0),   # one range to a sequence and head
]


@pytest.mark.parametrize("nq,nkv,dh,code,io_bf16,page,lengths,holes", CASES)
def test_attention_against_the_formula(nq, nkv, dh, code, io_bf16, page, lengths, holes):
    import torch
    import paper_2606_29565_amd as spp
    n = len(lengths)
    width = max(1, max(-(-l // page) for l in lengths)) + 1
    pool, pages, g = _pool(torch, spp, 2, nkv, dh, code, page, n * width + 2, seed=nq + page)
    table = torch.randperm(n * width + 2, generator=g, device="cuda")[:n * width].view(n, width).int()
    if holes:
        drop = torch.rand(n, width, generator=g, device="cuda") < holes
        drop[0] = True  # a sequence without a single listed page
        table[drop] = torch.tensor([-1, n * width + 2, 2 ** 31 - 1, -2 ** 31], device="cuda").int()[
            torch.randint(0, 4, (int(drop.sum()),), generator=g, device="cuda")]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    dt = torch.bfloat16 if io_bf16 else torch.float32
    q = torch.empty(n, nq, dh, device="cuda").normal_(0, 1.5, generator=g).to(dt)
    att = spp.PagedAttention(pool, 1, nq, table, lens, io_bf16=io_bf16)
    out = att(q, torch.full_like(q, 7.0))
    want, A, vmax = _reference(torch, pool, pages, 1, nq, table.cpu().numpy(), lengths, q, 1 / math.sqrt(dh))
    # (a few of the largest cases' codes are NaN: normal values past 448)
    assert torch.equal(torch.isnan(out).cpu(), torch.isnan(want))
    diff = (out.double().cpu() - want).abs().nan_to_num()
    assert bool((diff <= _bound(A, vmax, dh, max(lengths), io_bf16, want.nan_to_num())).all()), float(diff.max())
    log(f"attention {code} {nq}/{nkv}x{dh} page {page}: max diff {float(diff.max()):.2e}")
    # the same call again gives the same bits
    again = att(q, torch.empty_like(q))
    assert torch.equal(out.view(torch.int16 if io_bf16 else torch.int32), again.view(torch.int16 if io_bf16 else torch.int32))


@pytest.mark.parametrize("code,page", [("i8", 16), ("e4m3", 64), ("e4m3", 32), ("i8", 256)])
def test_attention_ignores_what_is_not_live(code, page):
    """Codes (NaN among them) and scales behind the last cell, in pages that are not listed and in the
    other layers change no bit; lengths past the table are cut to it, negative ones are zero."""
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 2, 2, 64, code, page, 24)
    k, v, ks, vs = _views(torch, pool, pages)
    table = torch.arange(20, device="cuda", dtype=torch.int32).view(4, 5)
    table[1, 2] = -1
    lens = [2 * page + page // 2 + 5, 5 * page, -7, 10 ** 9]
    q = torch.empty(4, 4, 64, device="cuda").normal_(generator=g)
    for io_bf16 in (False, True):
        qq = q.bfloat16() if io_bf16 else q
        att = spp.PagedAttention(pool, 0, 4, table, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                 io_bf16=io_bf16)
        a = att(qq, torch.empty_like(qq)).clone()
        assert not a[2].any() and bool(torch.isfinite(a).all())
        kept = pages.clone()
        for t in (k, v):
            t.view(torch.uint8)[:, 1] = 0x7F
            t.view(torch.uint8)[20:] = 0xFF
            for pg in (7, 3, 4):                                  # row 1's missing page, pages past row 0's
                t.view(torch.uint8)[pg] = 0x7F
        for s in (ks, vs):
            s[:, 1], s[20:] = float("nan"), float("inf")
            s[7], s[3], s[4] = float("nan"), float("nan"), float("nan")
            s[2, 0, :, (page // 2 + 5 + 15) // 16:] = float("nan")  # blocks past row 0's last
        rest = page // 2 + 5
        k.view(torch.uint8)[2, 0, :, rest:] = 0x7F
        v.view(torch.uint8)[2, 0, :, :, rest:] = 0x7F
        b = att(qq, torch.empty_like(qq))
        assert torch.equal(a, b)
        pages.copy_(kept)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_attention_of_a_nan_block_and_of_extreme_scales(code):
    """A live NaN scale of K makes the rows of its heads NaN, one of V likewise; blocks of the largest,
    smallest and very unequal scales keep the formula."""
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 64, code, 16, 12)
    k, v, ks, vs = _views(torch, pool, pages)
    table = torch.arange(12, device="cuda", dtype=torch.int32).view(2, 6)
    lens = torch.tensor([90, 96], dtype=torch.int32, device="cuda")
    q = torch.empty(2, 4, 64, device="cuda").normal_(generator=g).bfloat16()
    att = spp.PagedAttention(pool, 0, 4, table, lens)
    vs[0, 0, :, 0], vs[1, 0, :, 0], vs[2, 0, :, 0] = 2.0 ** -100, 2.0 ** 40, 2.0 ** -60
    vs[6:, 0] = 2.0 ** -100
    ks[3, 0], ks[7, 0] = 2.0 ** -100, 2.0 ** -30
    out = att(q, torch.empty_like(q)).clone()
    want, A, vmax = _reference(torch, pool, pages, 0, 4, table.cpu().numpy(), [90, 96], q, 0.125)
    diff = (out.double().cpu() - want).abs()
    assert bool((diff[0] <= _bound(A, vmax, 64, 96, True, want[0])).all())
    assert bool((diff[1] <= _bound(A, 448 * 2.0 ** -100, 64, 96, True, want[1])).all())   # 1e-30 is above it: zeros
    for s, page, head in ((ks, 4, 1), (vs, 9, 0)):
        was = s[page, 0, head].clone()
        s[page, 0, head] = float("nan")
        got = att(q, torch.empty_like(q))
        bad = torch.zeros_like(got, dtype=torch.bool)
        bad[page // 6, 2 * head:2 * head + 2] = True
        assert torch.equal(torch.isnan(got), bad)
        assert torch.equal(got[~bad], out[~bad])
        s[page, 0, head] = was


def test_attention_offsets_past_32_bits_and_a_scale():
    import torch
    import paper_2606_29565_amd as spp
    page, nkv, dh = 256, 8, 128
    n_pages = 9000                                                # 514 KiB each
    pool, pages, g = _pool(torch, spp, 1, nkv, dh, "i8", page, n_pages, fill=0)
    k, v, ks, vs = _views(torch, pool, pages)
    ids = [8999, 0, 8500]
    for i in ids:
        for t in (k, v):
            t[i] = torch.randint(-127, 128, t[i].shape, generator=g, device="cuda").to(torch.int8)
        ks[i], vs[i] = 2.0 ** -5, 2.0 ** -6
    assert 8500 * pool.page_layout().page_stride > 2 ** 32
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    lens = torch.tensor([700], dtype=torch.int32, device="cuda")
    q = torch.empty(1, 16, dh, device="cuda").normal_(generator=g)
    out = spp.PagedAttention(pool, 0, 16, table, lens, io_bf16=False, scale=0.05)(q, torch.empty_like(q))
    lay = pool.page_layout().page_stride
    small_pages = torch.cat([pages[i * lay:(i + 1) * lay] for i in ids])
    small = spp.PagePool(1, nkv, dh, True, page, 3, pages=small_pages, cells="i8")
    want, A, vmax = _reference(torch, small, small_pages, 0, 16, np.array([[0, 1, 2]]), [700], q, 0.05)
    diff = (out.double().cpu() - want).abs()
    assert bool((diff <= _bound(A, vmax, dh, 700, False, want)).all()), float(diff.max())
    # and cells there are written and read
    z = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    c = spp.PagedCells(pool, 0, table, z, rows, 20, io_bf16=False)
    x = torch.arange(20 * nkv * dh, device="cuda").float().view(20, nkv, dh) % 255 - 127
    x[0], x[16] = 127.0, 127.0                                    # a scale of 1 everywhere
    c.write(x, -x)
    a, b = c.read(torch.empty_like(x), torch.empty_like(x))
    assert torch.equal(a, x) and torch.equal(b, -x)


def test_attention_replayed_from_a_graph_with_strides():
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 128, "i8", 32, 64)
    table = torch.arange(60, device="cuda", dtype=torch.int32).view(3, 20)
    lens = torch.tensor([600, 64, 1], dtype=torch.int32, device="cuda")
    big = torch.empty(3, 12, 128, device="cuda").normal_(generator=g).bfloat16()
    q = big[:, 2:10]
    out = torch.empty(3, 8, 128, device="cuda").bfloat16()
    att = spp.PagedAttention(pool, 0, 8, table, lens)
    att._work.fill_(255)
    att(q, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att(q, out)
    eager = spp.PagedAttention(pool, 0, 8, table, lens)           # a workspace of its own
    for r in range(4):
        lens.copy_(torch.tensor([600 - 100 * r, 64 + r, 1 + 150 * r], dtype=torch.int32))
        table.copy_(table.roll(r, 0))
        big.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, eager(q.contiguous(), torch.empty_like(got))), r


# ---- sessions, forks and decode steps ---------------------------------------------------------


SESSIONS = [("bf16", "i8", 64, 1), ("bf16", "i8", 16, 203), ("bf16", "e4m3", 256, 1000), ("f32", "i8", 32, 97),
            ("bf16", "e4m3", 64, 576), ("f32", "e4m3", 128, 300), ("bf16", "i8", 16, 4200)]


@pytest.mark.parametrize("dtype,code,page,n", SESSIONS)
@pytest.mark.parametrize("dh", [64, 128])
def test_import_and_export_of_a_session(dtype, code, page, n, dh):
    """(4200 cells in pages of 16: more pages than one launch lists.)"""
    import torch
    import paper_2606_29565_amd as spp
    if dtype == "f32" and dh == 128:
        pytest.skip("fp32 models have heads of 64")
    shape = synth.Shape("pages", 2, 256, 4, 2, dh, 512, 2048, 1e4, dtype)
    b = build_model(shape, 3)
    cap = n + 37
    sess, into = spp.Session(b.model, cap), spp.Session(b.model, cap + 64)
    sess.kv.fill_(0xFF)                                           # NaN behind the cells
    into.kv.fill_(0x22)
    fill_synthetic_kv(b, sess, 5, n)
    sess.restore(n)
    pool, pages, _ = _pool(torch, spp, 2, 2, dh, code, page, -(-n // page) + 5, fill=0xFF)
    seq = pool.create(3)
    pool.import_session(seq, sess)
    pool.export_session(seq, into)
    torch.cuda.synchronize()
    assert pool.seq_info(seq).n_cells == n and into.info().n_committed == n
    for l in range(2):
        k, v = read_kv(b, sess, l, n)
        cache = Cache(1, -(-n // BLOCK) * BLOCK, 2, dh, code)
        cache.write(0, 0, k.transpose(1, 0, 2), v.transpose(1, 0, 2))
        k2, v2 = read_kv(b, into, l, n)
        assert np.array_equal(k2.transpose(1, 0, 2), cache.x[0][0, :n])
        assert np.array_equal(v2.transpose(1, 0, 2), cache.x[1][0, :n])
    # the session's cells behind the last one stay as they were
    for l in range(2):
        lay = b.model.kv_layout(into.capacity, l)
        eb = lay.elem_bytes
        kv = into.kv[lay.k_offset:lay.k_offset + 2 * lay.k_stride[0] * eb].view(2, -1, dh * eb)
        assert bool((kv[:, n:] == 0x22).all())
        vt = into.kv[lay.v_offset:lay.v_offset + 2 * lay.v_stride[0] * eb].view(2, dh, -1)
        assert bool((vt[:, :, n * eb:] == 0x22).all())
    pool.close()


def test_forks_write_pages_of_their_own():
    """Forks append cells of growing sizes to a shared partial block: each rounds its own copy."""
    import torch
    import paper_2606_29565_amd as spp
    for code, page in (("i8", 32), ("e4m3", 16)):
        n = 2 * page + 5
        pool, pages, g = _pool(torch, spp, 1, 2, 64, code, page, 64)
        base = pool.create(n)
        read = lambda s, m: [t.double().cpu().numpy() for t in spp.PagedCells(  # noqa: E731
            pool, 0, torch.tensor([pool.table(s)], dtype=torch.int32, device="cuda"),
            torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, m], dtype=torch.int32, device="cuda"), m,
            io_bf16=False).read(*(torch.empty(m, 2, 64, device="cuda") for _ in range(2)))]
        before = read(base, n)
        ks, vs = _scales(torch, pool, pages, 0)
        T = pool.table(base)
        forks = pool.fork(base, 6)
        pool.reserve(forks, 1)
        tables = torch.tensor([pool.table(f) for f in forks], dtype=torch.int32, device="cuda")
        first = torch.full((6,), n, dtype=torch.int32, device="cuda")
        rows = torch.arange(7, dtype=torch.int32, device="cuda")
        k = torch.empty(6, 2, 64, device="cuda").normal_(generator=g) * (4.0 ** torch.arange(6, device="cuda"))[:, None, None]
        spp.PagedCells(pool, 0, tables, first, rows, 1, io_bf16=False).write(k, 2 * k)
        for i, f in enumerate(forks):
            pool.commit(f, 1)
            cache = Cache(1, 3 * page, 2, 64, code)
            for x, was in zip(cache.x, before):
                x[0, :n] = was
            for s, old in ((cache.s[0], ks), (cache.s[1], vs)):
                s[0] = old[T].transpose(0, 2, 1).reshape(-1, 2)
            kk = k[i:i + 1].double().cpu().numpy()
            cache.write(0, n, kk, 2 * kk)
            got = read(f, n + 1)
            assert np.array_equal(got[0], cache.x[0][0, :n + 1]) and np.array_equal(got[1], cache.x[1][0, :n + 1])
        after = read(base, n)
        assert np.array_equal(before[0], after[0]) and np.array_equal(before[1], after[1])
        for f in forks[::2]:
            pool.free(f)
        kept = [read(f, n + 1) for f in forks[1::2]]
        pool.compact()
        for f, w in zip(forks[1::2], kept):
            assert all(np.array_equal(x, y) for x, y in zip(read(f, n + 1), w))
        pool.close()


@pytest.mark.parametrize("dtype,code,page,dh", [("bf16", "i8", 16, 64), ("bf16", "e4m3", 64, 128), ("f32", "i8", 32, 64),
                                                ("f32", "e4m3", 16, 64)])
def test_decode_steps_append_what_a_write_would(dtype, code, page, dh):
    """decode_batch over codes: layer 0's new cells do not depend on the cache, so those of a pool of values
    (the model's own dtype, or fp32) written through PagedCells are what the step has to append; and the
    logits are near those of the pool of values."""
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("codes", 2, 256, 4, 2, dh, 512, 2048, 1e4, dtype)
    b = build_model(shape, 3, max_sessions=8)
    n = 37
    sess = spp.Session(b.model, 100)
    fill_synthetic_kv(b, sess, 5, n)
    sess.restore(n)
    pool, pages, _ = _pool(torch, spp, 2, 2, dh, code, page, 64, fill=0xFF)
    plain = spp.PagePool(2, 2, dh, dtype == "bf16", page, 64)
    a, p = pool.create(), plain.create()
    pool.import_session(a, sess)
    plain.import_session(p, sess)
    forks, pforks = pool.fork(a, 5), plain.fork(p, 5)
    dists, pdists = (torch.empty(5, shape.vocab, device="cuda") for _ in range(2))
    ids = [3, 77, 1500, 8, 900]
    for step in range(14):                                        # past the end of a block and a page
        toks = [(t * (step + 1)) % shape.vocab for t in ids]
        spp.decode_batch(pool, b.model, forks, toks, list(dists))
        spp.decode_batch(plain, b.model, pforks, toks, list(pdists))
        diff, spread = max_abs(dists.cpu().numpy(), pdists.cpu().numpy()), float(pdists.std())
        assert diff < 0.2 * spread, (step, diff, spread)           # (8 bits a cell; a wrong cell is off by `spread`)
    log(f"decode over {code}: logits off by {diff:.3f} of a spread of {spread:.3f}")
    m = n + 14
    lay = plain.page_layout()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for f, pf in zip(forks, pforks):
        got = [t.double().cpu().numpy() for t in spp.PagedCells(
            pool, 0, torch.tensor([pool.table(f)], dtype=torch.int32, device="cuda"),
            torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, m], dtype=torch.int32, device="cuda"), m,
            io_bf16=False).read(*(torch.empty(m, 2, dh, device="cuda") for _ in range(2)))]
        pv = plain.pages.view(dt).view(64, 2, 2, -1)[torch.tensor(plain.table(pf), device="cuda"), 0]
        k = pv[:, 0].reshape(-1, 2, page, dh).transpose(1, 2).reshape(-1, 2, dh)[:m].double().cpu().numpy()
        v = pv[:, 1].reshape(-1, 2, dh, page).permute(0, 3, 1, 2).reshape(-1, 2, dh)[:m].double().cpu().numpy()
        assert lay.elem_bytes == dt.itemsize
        # each cell within the format's error of its block's largest magnitude: half a step, and a step
        # for cells that were rounded again as their block's scale grew; the values' own dtype on top
        for x, w in ((got[0], k), (got[1], v)):
            for c0 in range(0, m, BLOCK):
                blk = w[c0:c0 + BLOCK]
                s = _scale(np.abs(blk).max(axis=(0, 2)) * (1 + 2.0 ** -8), code)[None, :, None]
                tol = 1.5 * s if code == "i8" else 2 * (np.abs(blk) * 2.0 ** -4 + s * 2.0 ** -10) + np.abs(blk) * 2.0 ** -7
                assert bool((np.abs(x[c0:c0 + BLOCK] - blk) <= tol + np.abs(blk) * 2.0 ** -8).all()), c0
    # the best one goes back
    pool.export_session(forks[2], sess)
    assert sess.info().n_committed == m
    k0, _ = read_kv(b, sess, 0, m)
    torch.cuda.synchronize()
    assert np.isfinite(k0).all()
    pool.close(), plain.close()
