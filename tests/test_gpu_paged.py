"""Attention over paged caches, the pages' copies and the decode step of paged sequences.

The attention is compared with the formula in 64 bits over the cells the tables name.  Its bound,
with u = 2^-24: a score is off by at most A (dh + 4) u through its fp32 sum, A the largest sum of
|q k| scale, and by A 2^-17 more where q goes through two bf16 parts (each leaves at most
2^-9 of what it rounds, twice 2^-18 in all); a probability is off by that and by 2^-17 for its own two parts
(fp32 cells: by the exponential's 2^-21); the sums over n cells by n u each.  The output is a quotient of two
such sums, so it is off by at most twice their relative errors times the largest |v|, and then
rounded to its type once.  Copies are compared bit for bit."""
import math

import numpy as np
import pytest

import oracle
import synth
from gpu_util import build_model, fill_synthetic_kv, log, max_abs, read_kv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _pool(torch, spp, layers, nkv, dh, bf16, page, n_pages, max_seqs=64, seed=0):
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(1234 + seed)
    pages = torch.empty(n_pages, layers, 2, nkv * page * dh, dtype=dt, device="cuda").normal_(generator=g)
    return spp.PagePool(layers, nkv, dh, bf16, page, n_pages, max_seqs=max_seqs, pages=pages), pages, g


def _reference(torch, pages, layer, nq, nkv, dh, page, table, lengths, q, scale):
    """(output in 64 bits, largest sum of |q k| scale, largest |v|) over the live cells."""
    n, G = q.shape[0], nq // nkv
    out = torch.zeros(n, nq, dh, dtype=torch.float64)
    A = vmax = 0.0
    P = pages[:, layer].cpu()
    for i in range(n):
        at = np.arange(max(0, min(int(lengths[i]), table.shape[1] * page)))
        pg = table[i][at // page] if at.size else at
        ok = (pg >= 0) & (pg < pages.shape[0])
        at, pg = at[ok], pg[ok]
        if not at.size:
            continue
        pgt, cell = torch.from_numpy(pg.astype(np.int64)), torch.from_numpy(at % page)
        K = P[:, 0].view(-1, nkv, page, dh)[pgt, :, cell].double()       # [cells, nkv, dh]
        V = P[:, 1].view(-1, nkv, dh, page)[pgt, :, :, cell].double()
        for h in range(nq):
            k, v, qq = K[:, h // G], V[:, h // G], q[i, h].double().cpu()
            z = (k * qq).sum(1) * scale
            A = max(A, float((k * qq).abs().sum(1).max()) * abs(scale))
            vmax = max(vmax, float(v.abs().max()))
            p = torch.exp(z - z.max())
            out[i, h] = (p[:, None] * v).sum(0) / p.sum()
    return out, A, vmax


def _bound(A, vmax, dh, n, bf16, io_bf16, want):
    score = A * ((dh + 4) * U + (2.0 ** -17 if bf16 and not io_bf16 else 0.0))
    prob = score + (2.0 ** -17 if bf16 else 2.0 ** -21)
    return 2 * (prob + n * U) * vmax + want.abs() * (2.0 ** -8 if io_bf16 else U) + 1e-30


CASES = [
    # nq, nkv, dh, cells bf16, io bf16, page, lengths, holes
    (4, 4, 64, False, False, 16, [1, 15, 16, 17, 63, 64, 65, 512], 0.0),
    (4, 2, 64, True, True, 16, [1, 2, 31, 32, 33, 127, 128, 129, 700], 0.0),
    (4, 2, 64, True, False, 32, [5, 0, 300, 1, 0, 1000], 0.3),
    (32, 8, 128, True, True, 64, [1, 8191, 4097], 0.0),
    (32, 8, 128, True, False, 128, [3, 130, 2049], 0.0),
    (64, 8, 128, True, True, 256, [600, 255, 257], 0.0),
    (20, 1, 128, True, True, 16, [40, 5000], 0.2),          # a second tile of 4 heads
    (40, 1, 64, False, False, 16, [77, 1, 300], 0.0),       # three tiles
    (6, 2, 64, False, True, 64, [129, 64], 0.0),
    (8, 8, 128, False, False, 16, [33, 200], 0.5),
    (16, 1, 64, True, False, 64, [16385], 0.0),
    (12, 4, 128, False, False, 64, [1, 500, 4500], 0.1),
    (32, 8, 128, True, False, 16, [700] * 20 + [1, 0, 1007], 0.0),   # one range to a sequence and head
]


@pytest.mark.parametrize("nq,nkv,dh,bf16,io_bf16,page,lengths,holes", CASES)
def test_attention_against_the_formula(nq, nkv, dh, bf16, io_bf16, page, lengths, holes):
    import torch
    import paper_2606_29565_amd as spp
    n = len(lengths)
    width = max(1, max(-(-l // page) for l in lengths)) + 1
    pool, pages, g = _pool(torch, spp, 2, nkv, dh, bf16, page, n * width + 2, seed=nq + page)
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
    want, A, vmax = _reference(torch, pages, 1, nq, nkv, dh, page, table.cpu().numpy(), lengths, q,
                               1 / math.sqrt(dh))
    diff = (out.double().cpu() - want).abs()
    assert bool((diff <= _bound(A, vmax, dh, max(lengths), bf16, io_bf16, want)).all()), float(diff.max())
    log(f"attention {nq}/{nkv}x{dh} page {page}: max diff {float(diff.max()):.2e}")
    # the same call again gives the same bits
    again = att(q, torch.empty_like(q))
    assert torch.equal(out, again)


def test_attention_ignores_what_is_not_live():
    """NaN and infinities behind the last cell, in pages that are not listed and in the other
    layers change no bit; lengths past the table are cut to it, negative ones are zero."""
    import torch
    import paper_2606_29565_amd as spp
    for bf16, page in ((True, 16), (True, 64), (False, 32)):
        pool, pages, g = _pool(torch, spp, 2, 2, 64, bf16, page, 24)
        table = torch.arange(20, device="cuda", dtype=torch.int32).view(4, 5)
        table[1, 2] = -1
        lens = [3 * page + 5, 5 * page, -7, 10 ** 9]
        q = torch.empty(4, 4, 64, device="cuda").normal_(generator=g)
        att = spp.PagedAttention(pool, 0, 4, table, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                 io_bf16=False)
        a = att(q, torch.empty_like(q)).clone()
        assert not a[2].any() and bool(torch.isfinite(a).all())
        pages[:, 1] = float("nan")
        pages[20:] = float("inf")
        pages[7] = float("nan")                                   # row 1's page that is not listed
        pages[4] = float("nan")                                   # row 0's page past its length
        k = pages[3, 0, 0].view(2, page, 64)
        v = pages[3, 0, 1].view(2, 64, page)
        k[:, 5:] = float("nan")
        v[:, :, 5:] = float("inf")
        b = att(q, torch.empty_like(q))
        assert torch.equal(a, b)


def test_attention_rows_with_strides_and_workspace_of_garbage():
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 64, True, 16, 200)
    table = torch.randperm(200, generator=g, device="cuda")[:195].view(3, 65).int()[:, :60]
    assert table.stride(0) == 65
    lens = torch.tensor([900, 1, 333], dtype=torch.int32, device="cuda")
    big = torch.empty(3, 12, 64, device="cuda").normal_(generator=g).bfloat16()
    q = big[:, 4:8]                                               # rows 12 * 64 apart, offset 4 heads
    att = spp.PagedAttention(pool, 0, 4, table, lens)
    att._work.fill_(255)                                          # NaN patterns
    holder = torch.full((3, 6, 64), 9.0, device="cuda").bfloat16()
    att(q, holder[:, 1:5])
    plain = att(q.contiguous(), torch.empty(3, 4, 64, device="cuda").bfloat16())
    assert torch.equal(holder[:, 1:5], plain)
    assert bool((holder[:, 0] == 9).all()) and bool((holder[:, 5] == 9).all())


def test_attention_of_no_sequence():
    import torch
    import paper_2606_29565_amd as spp
    pool, _, _ = _pool(torch, spp, 1, 2, 64, True, 16, 4)
    q = torch.empty(0, 4, 64, device="cuda").bfloat16()
    table = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    att = spp.PagedAttention(pool, 0, 4, table, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert att(q, torch.empty_like(q)).shape == q.shape


def test_attention_scale_and_offsets_past_32_bits():
    """Pages whose byte offset passes 2^32 (and an explicit scale)."""
    import torch
    import paper_2606_29565_amd as spp
    page, nkv, dh = 256, 8, 128
    n_pages = 5000                                                # 1 MiB each in one layer
    pages = torch.zeros(n_pages, 1, 2, nkv * page * dh, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    ids = [4999, 0, 4500]
    for i in ids:
        pages[i].normal_(generator=g)
    pool = spp.PagePool(1, nkv, dh, True, page, n_pages, pages=pages)
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    lens = torch.tensor([700], dtype=torch.int32, device="cuda")
    q = torch.empty(1, 16, dh, device="cuda").normal_(generator=g)
    out = spp.PagedAttention(pool, 0, 16, table, lens, io_bf16=False, scale=0.05)(q, torch.empty_like(q))
    small = pages[ids].clone()
    want, A, vmax = _reference(torch, small, 0, 16, nkv, dh, page, np.array([[0, 1, 2]]), [700], q, 0.05)
    diff = (out.double().cpu() - want).abs()
    assert bool((diff <= _bound(A, vmax, dh, 700, True, False, want)).all()), float(diff.max())


def test_attention_replayed_from_a_graph_reads_the_tables_as_they_are():
    import torch
    import paper_2606_29565_amd as spp
    pool, pages, g = _pool(torch, spp, 1, 2, 128, True, 32, 64)
    table = torch.arange(60, device="cuda", dtype=torch.int32).view(3, 20)
    lens = torch.tensor([600, 64, 1], dtype=torch.int32, device="cuda")
    q = torch.empty(3, 8, 128, device="cuda").normal_(generator=g).bfloat16()
    out = torch.empty_like(q)
    att = spp.PagedAttention(pool, 0, 8, table, lens)
    att(q, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att(q, out)
    eager = spp.PagedAttention(pool, 0, 8, table, lens)           # a workspace of its own
    for k in range(4):
        lens.copy_(torch.tensor([600 - 100 * k, 64 + k, 1 + 150 * k], dtype=torch.int32))
        table.copy_(table.roll(k, 0))
        q.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, eager(q, torch.empty_like(q))), k


# ---- pages ----------------------------------------------------------------------------------


def _cells(torch, spp, pool, pages, seq, layer, n):
    """K, V [nkv][n][dh] of a sequence's first n cells."""
    c = pool.cfg
    t = pool.table(seq)
    k = torch.cat([pages[i, layer, 0].view(c.n_kv_heads, c.page_cells, c.head_dim) for i in t], 1)
    v = torch.cat([pages[i, layer, 1].view(c.n_kv_heads, c.head_dim, c.page_cells) for i in t], 2)
    return k[:, :n], v[:, :, :n].transpose(1, 2)


@pytest.mark.parametrize("bf16,page", [(True, 64), (True, 16), (False, 128)])
def test_forks_own_their_last_page_and_compaction_moves_it(bf16, page):
    import torch
    import paper_2606_29565_amd as spp
    n = 3 * page + 5
    pool, pages, g = _pool(torch, spp, 3, 2, 64, bf16, page, 300, max_seqs=64)
    base = pool.create(n)
    before = [tuple(x.clone() for x in _cells(torch, spp, pool, pages, base, l, n)) for l in range(3)]
    forks = pool.fork(base, 40)
    assert pool.info().used_pages == 4 and pool.info().shared_pages == 4
    pool.reserve(forks + [base], 1)
    assert pool.info().used_pages == 44 and pool.info().shared_pages == 3
    last = {pool.table(f)[-1] for f in forks + [base]}
    assert len(last) == 41
    for i, f in enumerate(forks):  # each writes its own cell
        pages[pool.table(f)[-1], :, 0].view(3, 2, page, 64)[:, :, n % page] = float(i)
    for f in forks[::3]:
        pool.free(f)
    keep = [f for i, f in enumerate(forks) if i % 3]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    moved = pool.compact(stream=other)
    torch.cuda.current_stream().wait_stream(other)
    used = pool.info().used_pages
    assert moved > 0 and used == 3 + len(keep) + 1
    assert all(t < used for f in keep + [base] for t in pool.table(f))
    for i, f in enumerate(forks):
        if i % 3 == 0:
            continue
        for l in range(3):
            k, v = _cells(torch, spp, pool, pages, f, l, n + 1)
            assert torch.equal(k[:, :n], before[l][0]) and torch.equal(v[:, :n], before[l][1])
            assert bool((k[:, n] == i).all())
    pool.close()


@pytest.mark.parametrize("bf16,page,n", [(True, 64, 1), (True, 16, 203), (True, 256, 1000),
                                         (False, 32, 97), (True, 64, 576), (True, 16, 4200)])
def test_import_and_export_of_a_session(bf16, page, n):
    """(4200 cells in pages of 16: more pages than one launch lists.)"""
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("pages", 2, 256, 4, 2, 64, 512, 2048, 1e4, "bf16" if bf16 else "f32")
    b = build_model(shape, 3)
    cap = n + 37
    sess, into = spp.Session(b.model, cap), spp.Session(b.model, cap + 64)
    sess.kv.fill_(0x11)
    into.kv.fill_(0x22)
    fill_synthetic_kv(b, sess, 5, n)
    sess.restore(n)
    pool, pages, _ = _pool(torch, spp, 2, 2, 64, bf16, page, -(-n // page) + 5)
    blank = pages.clone()
    seq = pool.create(3)
    pool.import_session(seq, sess)
    pool.export_session(seq, into)
    torch.cuda.synchronize()
    assert pool.seq_info(seq).n_cells == n and into.info().n_committed == n
    for l in range(2):
        k, v = read_kv(b, sess, l, n)
        pk, pv = _cells(torch, spp, pool, pages, seq, l, n)
        assert np.array_equal(pk.float().cpu().numpy(), k) and np.array_equal(pv.float().cpu().numpy(), v)
        k2, v2 = read_kv(b, into, l, n)
        assert np.array_equal(k, k2) and np.array_equal(v, v2)
    # what lies behind the last cell stays as it was, on both sides
    t = pool.table(seq)
    rest = n % page
    if rest:
        P = pages[t[-1]].view(2, 2, -1)
        Q = blank[t[-1]].view(2, 2, -1)
        assert torch.equal(P[:, 0].view(2, 2, page, 64)[:, :, rest:], Q[:, 0].view(2, 2, page, 64)[:, :, rest:])
        assert torch.equal(P[:, 1].view(2, 2, 64, page)[..., rest:], Q[:, 1].view(2, 2, 64, page)[..., rest:])
    for l in range(2):
        lay = b.model.kv_layout(into.capacity, l)
        eb = lay.elem_bytes
        kv = into.kv[lay.k_offset:lay.k_offset + 2 * lay.k_stride[0] * eb].view(2, -1, 64 * eb)
        assert bool((kv[:, n:] == 0x22).all())
        vt = into.kv[lay.v_offset:lay.v_offset + 2 * lay.v_stride[0] * eb].view(2, 64, -1)
        assert bool((vt[:, :, n * eb:] == 0x22).all())
    pool.close()


def test_a_session_changes_after_its_copy_on_another_stream():
    """A copy that starts late on one stream, then a shift of the same cells on another, and back."""
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("pages", 2, 256, 4, 2, 64, 512, 2048, 1e4, "bf16")
    b = build_model(shape, 3)
    n = 4000
    sess = spp.Session(b.model, n + 8)
    fill_synthetic_kv(b, sess, 5, n)
    sess.restore(n)
    pool, pages, _ = _pool(torch, spp, 2, 2, 64, True, 64, 200)
    first, second, third = (pool.create() for _ in range(3))
    pool.import_session(first, sess)
    want = [[c.clone() for c in _cells(torch, spp, pool, pages, first, l, n)] for l in range(2)]
    torch.cuda.synchronize()
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    a = torch.randn(4096, 4096, device="cuda")

    def delay():
        with torch.cuda.stream(late):
            x = a
            for _ in range(30):
                x = torch.tanh(x @ a)
        return x

    torch.cuda.synchronize()
    busy = delay()
    pool.import_session(second, sess, stream=late)
    sess.shift(1, stream=other)                            # waits for the copy
    pool.export_session(first, sess, stream=other)
    busy = delay()
    pool.compact(stream=late)
    pool.import_session(third, sess, stream=late)          # waits for the export
    torch.cuda.synchronize()
    assert bool(torch.isfinite(busy).all()) and sess.info().n_committed == n
    for seq in (second, third):
        for l in range(2):
            got = _cells(torch, spp, pool, pages, seq, l, n)
            assert all(torch.equal(x, y) for x, y in zip(got, want[l])), (seq, l)
    pool.close()


# ---- the decode step ------------------------------------------------------------------------


@pytest.mark.parametrize("fmt,max_sessions,page", [("f32", 1, 16), ("f32", 4, 64), ("bf16", 1, 64),
                                                   ("bf16", 8, 16), ("mxfp4", 4, 32)])
def test_forks_of_a_session_decode_like_the_oracle(fmt, max_sessions, page):
    """A session's state forked, each fork decoded three tokens of its own in batches, an adjusted greedy step read, the
    best exported into the session: every distribution against the oracle's over the same tokens."""
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("paged-" + fmt, 2, 256, 4, 2, 64, 512, 2048, 1e4, "f32" if fmt == "f32" else "bf16",
                        wfmt="mxfp4" if fmt == "mxfp4" else "dtype")
    b = build_model(shape, 21, max_sessions=max_sessions, max_tokens=64)
    n0, forks_n, steps = 100, 6, 3
    prefill = synth.cpu_tokens(n0, 21, 1, shape.vocab)
    sess = spp.Session(b.model, 160)
    sess.append_delta(prefill.tolist())
    bf16 = fmt != "f32"
    pool, pages, _ = _pool(torch, spp, 2, 2, 64, bf16, page, 40 * 16 // page + 12, max_seqs=8)
    base = pool.create()
    pool.import_session(base, sess)
    forks = pool.fork(base, forks_n)
    pool.free(base)
    toks = synth.cpu_tokens(forks_n * steps, 22, 2, shape.vocab).reshape(forks_n, steps)
    dists = [torch.empty(shape.vocab, dtype=torch.float32, device="cuda") for _ in forks]
    w = oracle.Weights(shape, 21)
    worst = 0.0
    for t in range(steps):
        spp.decode_batch(pool, b.model, forks, toks[:, t].tolist(), dists)
        if t == 1:
            pool.compact()
        summ = pool.summaries(forks)
        for i, f in enumerate(forks):
            kv = oracle.KVState(shape, n0 + steps)
            oracle.forward(w, kv, 0, prefill, logits=False)
            ref = oracle.forward(w, kv, n0, toks[i, :t + 1])
            got = dists[i].double().cpu().numpy()
            worst = max(worst, max_abs(got, ref))
            o = oracle.summary(got)
            assert (summ[i].argmax, summ[i].position, summ[i].flags) == (o.argmax, n0 + t + 1, 0)
            assert summ[i].top1 == np.float32(o.top1) and summ[i].top2 == np.float32(o.top2)
    log(f"paged decode {fmt}: max |logit - oracle| {worst:.2e}")
    assert worst <= (5e-2 if bf16 else 1e-4)
    # the greedy step of a grammar that allows four tokens and penalizes the last
    allowed = torch.from_numpy(synth.bitmap_from_ids(shape.vocab, [3, 700, 1500, 2047]).view(np.int32)).cuda()
    hist = torch.from_numpy(toks.astype(np.int32)).cuda()
    outs = [torch.empty_like(d) for d in dists]
    rows = [spp.AdjustRow(dists[i], outs[i], tokens=hist[i], repetition=1.5, allowed=allowed, fill=-3e38)
            for i in range(forks_n)]
    s = spp.LogitsAdjust(shape.vocab, rows)()
    for i in range(forks_n):
        assert int(s.argmax[i]) == int(torch.argmax(outs[i])) and int(s.argmax[i]) in (3, 700, 1500, 2047)
    # the second fork becomes the session's state; the next token there and in the pool agree
    pool.export_session(forks[1], sess)
    assert sess.info().n_committed == n0 + steps and not sess.info().valid
    d2 = torch.empty_like(dists[0])
    sess.resume([17], d2)
    spp.decode_batch(pool, b.model, [forks[1]], [17], [dists[1]])
    assert max_abs(d2.cpu().numpy(), dists[1].cpu().numpy()) <= (5e-2 if bf16 else 1e-4)
    pool.close()


def test_decode_on_two_streams_and_pools_of_one_model():
    """Two pools on two streams take turns at a model: the same bits as one after the other."""
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("paged-2", 2, 256, 4, 2, 64, 512, 2048, 1e4, "bf16")
    b = build_model(shape, 9, max_sessions=2, max_tokens=64)
    sess = spp.Session(b.model, 64)
    sess.append_delta(list(range(1, 51)))
    runs = []
    for apart in (False, True):
        got = []
        streams = [torch.cuda.current_stream()] * 2 if not apart else [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        pools = [_pool(torch, spp, 2, 2, 64, True, 16, 12)[0] for _ in range(2)]
        dists = [[torch.empty(shape.vocab, device="cuda") for _ in range(2)] for _ in range(2)]
        torch.cuda.synchronize()
        seqs = []
        for p, st in zip(pools, streams):
            q = p.create()
            p.import_session(q, sess, stream=st)
            seqs.append([q] + p.fork(q, 1))
        for t in range(4):
            for p, st, d, s in zip(pools, streams, dists, seqs):
                spp.decode_batch(p, b.model, s, [t + 3, 100 + t], d, stream=st)
        torch.cuda.synchronize()
        runs.append([x.clone() for d in dists for x in d])
    for a, c in zip(*runs):
        assert torch.equal(a, c)


def test_refusals_on_the_device():
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("paged-r", 2, 256, 4, 2, 64, 512, 2048, 1e4, "bf16")
    b = build_model(shape, 9, max_sessions=2, max_tokens=64)
    sess = spp.Session(b.model, 64)
    d = [torch.empty(shape.vocab, device="cuda") for _ in range(3)]
    pool, _, _ = _pool(torch, spp, 2, 2, 64, True, 16, 4, max_seqs=4)
    wrong, _, _ = _pool(torch, spp, 1, 2, 64, True, 16, 4, max_seqs=4)
    a = pool.create(16)

    def refused(rc, f, *args):
        with pytest.raises(spp.SppError) as e:
            f(*args)
        assert e.value.rc == rc

    refused(spp.SPP_E_INVALID_ARG, spp.decode_batch, pool, b.model, [a, a], [1, 2], d[:2])
    refused(spp.SPP_E_INVALID_ARG, spp.decode_batch, pool, b.model, [3], [1], d[:1])
    refused(spp.SPP_E_INVALID_ARG, spp.decode_batch, pool, b.model, [a], [shape.vocab], d[:1])
    q = wrong.create(5)
    refused(spp.SPP_E_INVALID_ARG, spp.decode_batch, wrong, b.model, [q], [1], d[:1])
    refused(spp.SPP_E_INVALID_ARG, wrong.import_session, q, sess)
    refused(spp.SPP_E_INVALID_ARG, wrong.export_session, q, sess)
    refused(spp.SPP_E_STATE, pool.summaries, [a])
    big = pool.create(48)
    refused(spp.SPP_E_CAPACITY, spp.decode_batch, pool, b.model, [a], [1], d[:1])  # no page left
    assert pool.seq_info(a).n_cells == 16 and pool.info().used_pages == 4
    pool.truncate(big, 20)
    spp.decode_batch(pool, b.model, [a, big], [1, 2], d[:2])
    assert pool.summaries([big, a])[0].position == 21
    pool.truncate(a, 16)
    refused(spp.SPP_E_STATE, pool.summaries, [a])
    sess.restore(40)
    refused(spp.SPP_E_CAPACITY, pool.import_session, a, sess)                      # 3 pages, 2 to be had
    assert pool.seq_info(a).n_cells == 16
    small = spp.Session(b.model, 8)
    refused(spp.SPP_E_CAPACITY, pool.export_session, a, small)
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    lens = torch.ones(1, dtype=torch.int32, device="cuda")
    x = torch.zeros(1, 4, 64, device="cuda").bfloat16()
    for kw in ({"n_q_heads": 3}, {"layer": 2}, {"layer": -1}, {"scale": math.inf}, {"scale": math.nan}):
        args = {"layer": 0, "n_q_heads": 4, "scale": 0.0, **kw}
        h = args["n_q_heads"]
        att = spp.PagedAttention(pool, args["layer"], h, table, lens, scale=args["scale"])
        refused(spp.SPP_E_INVALID_ARG, att, x[:, :h], torch.empty_like(x[:, :h]))
    att = spp.PagedAttention(pool, 0, 4, table, lens)
    with pytest.raises(ValueError):
        att(x.float(), x)
    flat = torch.zeros(4 * 64 + 8, device="cuda").bfloat16()
    refused(spp.SPP_E_INVALID_ARG, att, flat[1:257].view(1, 4, 64), torch.empty_like(x))  # misaligned
    for bad in ((table.cpu(), lens), (table, lens.cpu()), (table.long(), lens), (table, lens[:0]), (table[0], lens)):
        with pytest.raises(ValueError):
            spp.PagedAttention(pool, 0, 4, *bad)
    with pytest.raises(ValueError):
        att(x.cpu(), x)
    with pytest.raises(ValueError):
        spp.PagePool(2, 2, 64, True, 16, 4, pages=torch.zeros(4 * 2 * 2 * 2 * 16 * 64 * 2, dtype=torch.uint8))
    with pytest.raises(spp.SppError):
        spp.PagePool(2, 2, 64, True, 16, 4, pages=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(spp.SppError):
        spp.PagePool(2, 2, 64, True, 24, 4)
    pool.close()
    with pytest.raises(ValueError):
        att(x, torch.empty_like(x))
    refused(spp.SPP_E_INVALID_ARG, spp.decode_batch, pool, b.model, [a], [1], d[:1])
    with pytest.raises(ValueError):
        spp.PagedAttention(pool, 0, 4, table, lens)


def test_tables_of_any_length_and_numbers_of_any_kind():
    import numpy as np
    import paper_2606_29565_amd as spp
    pool = spp.PagePool(1, 1, 64, True, 16, 150, max_seqs=4)
    for n in (0, 1, 63, 64, 65):                   # pages
        q = pool.create(16 * n)
        assert pool.table(q) == pool.table(np.int64(q)) == list(range(n))
        pool.free(np.int32(q))
        for f in (pool.table, pool.free):
            with pytest.raises(spp.SppError):
                f(q)                               # given back
    q = pool.create(16 * 150)
    assert pool.table(q) == list(range(150)) and pool.info().used_pages == 150
    for f in (pool.table, pool.free):
        for bad in ("0", None, 0.0):
            with pytest.raises(TypeError):
                f(bad)
        for bad in (-1, 3, 4):
            with pytest.raises(spp.SppError):
                f(bad)
    pool.close()
    for f in (pool.table, pool.free):
        with pytest.raises(spp.SppError):
            f(q)
