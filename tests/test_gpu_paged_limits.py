"""Attention over paged caches where its rules change or reach their ends: workspaces of smaller
calls, infinities and NaN in live cells, the most ranges, the decode step over several of them.
The bound of a result is that of test_gpu_paged.py."""
import ctypes
import math

import pytest

from test_gpu_paged import _bound, _pool, _reference

pytestmark = pytest.mark.gpu


def _args(spp, torch, pool, n, n_q, table, lengths, q, out):
    row = n_q * pool.cfg.head_dim
    return spp.spp_paged_attn(pool.handle.value, 0, n, n_q, spp.SPP_DTYPE_BF16, q.data_ptr(), row, table.data_ptr(),
                              table.stride(0), table.shape[1], lengths.data_ptr(), 0.0, out.data_ptr(), row)


def test_a_workspace_of_the_largest_batch_serves_smaller_ones():
    """1000 cells of the 8B heads: from 16 sequences on one range each and no workspace, four ranges
    below; sizes do not fall with the sequences or the pages, and a batch that shrinks stays served."""
    import torch
    import paper_2606_29565_amd as spp
    nq, nkv, dh, page, width, n = 32, 8, 128, 64, 16, 40
    pool, pages, g = _pool(torch, spp, 1, nkv, dh, True, page, n * width)
    table = torch.randperm(n * width, generator=g, device="cuda").view(n, width).int()
    lengths = [1000 - 3 * i for i in range(n)]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.empty(n, nq, dh, device="cuda").normal_(0, 1.5, generator=g).bfloat16()
    size = lambda m, w: spp.lib().spp_paged_attention_work_bytes(  # noqa: E731
        ctypes.byref(_args(spp, torch, pool, m, nq, table[:, :w], lens, q, q)))
    for w in range(1, width + 1):
        sizes = [size(m, w) for m in range(1, n + 1)]
        assert sizes == sorted(sizes) and (w == 1 or size(n, w) >= size(n, w - 1))
    work = torch.empty(size(n, width), dtype=torch.uint8, device="cuda")
    want, A, vmax = _reference(torch, pages, 0, nq, nkv, dh, page, table.cpu().numpy(), lengths, q, 1 / math.sqrt(dh))
    for m in (n, 17, 16, 15, 5, 4, 1):
        work.fill_(255)
        out = torch.full_like(q, 7.0)
        a = _args(spp, torch, pool, m, nq, table, lens, q, out)
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        spp.check(spp.lib().spp_paged_attention(ctypes.byref(a), ctypes.c_void_p(work.data_ptr()), work.numel(),
                                                stream), "spp_paged_attention")
        diff = (out[:m].double().cpu() - want[:m]).abs()
        assert bool((diff <= _bound(A, vmax, dh, 1000, True, True, want[:m])).all()), (m, float(diff.max()))
        assert bool((out[m:] == 7).all())


@pytest.mark.parametrize("bf16,io_bf16,page,cells", [(True, True, 16, 100), (False, False, 32, 77), (True, True, 64, 3000),
                                                     (False, True, 16, 2500), (True, False, 64, 3000)])
def test_infinities_and_nan_in_live_cells(bf16, io_bf16, page, cells):
    """Of a live cell: a NaN of K makes the rows that use it NaN, one of V its dimension; an infinity
    of K makes scores of +inf (a NaN row) and -inf (no weight), one of V its dimension not finite.
    A row whose scores all are -inf is zero.  Nothing else changes a bit.  (fp32 queries over
    bf16 cells go through two parts, whose second is zero here: their infinite scores are NaN.)"""
    import torch
    import paper_2606_29565_amd as spp
    nq, nkv, dh, at, dim = 8, 2, 64, cells // 3, 37
    width = -(-cells // page)
    pool, pages, g = _pool(torch, spp, 1, nkv, dh, bf16, page, 2 * width)
    table = torch.randperm(2 * width, generator=g, device="cuda").view(2, width).int()
    lens = torch.full((2,), cells, dtype=torch.int32, device="cuda")
    q = torch.empty(2, nq, dh, device="cuda").normal_(0, 1.5, generator=g).bfloat16().to(
        torch.bfloat16 if io_bf16 else torch.float32)
    q[:, :, dim] = torch.tensor([2.0, -2.0] * (nq // 2), device="cuda")
    neg, pos = slice(1, nq // nkv, 2), slice(0, nq // nkv, 2)       # heads of kv head 0 by the sign
    att = spp.PagedAttention(pool, 0, nq, table, lens, io_bf16=io_bf16)
    run = lambda: att(q, torch.full_like(q, 7.0)).clone()  # noqa: E731
    keys = pages[:, 0, 0].view(-1, nkv, page, dh)
    vals = pages[:, 0, 1].view(-1, nkv, dh, page)
    pg, c = int(table[0, at // page]), at % page
    plain, clean = run(), pages.clone()
    split = bf16 and not io_bf16

    keys[pg, 0, c, dim] = float("nan")
    got = run()
    assert bool(got[0, :nq // nkv].isnan().all())
    assert torch.equal(got[0, nq // nkv:], plain[0, nq // nkv:]) and torch.equal(got[1], plain[1])
    pages.copy_(clean)

    for value in (float("nan"), float("inf"), -float("inf")):
        vals[pg, 0, dim, c] = value
        got = run()
        assert not bool(got[0, :nq // nkv, dim].isfinite().any())
        if math.isnan(value):
            assert bool(got[0, :nq // nkv, dim].isnan().all())
        got[0, :nq // nkv, dim] = plain[0, :nq // nkv, dim]
        assert torch.equal(got, plain)
        pages.copy_(clean)

    keys[pg, 0, c, dim] = float("inf")
    got = run()
    assert bool(got[0, pos].isnan().all())
    assert torch.equal(got[0, nq // nkv:], plain[0, nq // nkv:]) and torch.equal(got[1], plain[1])
    if split:
        assert bool(got[0, neg].isnan().all())
    else:                                                            # the cell is left out
        want, A, vmax = _reference_without(torch, pages, nq, nkv, dh, page, table, cells, q, at)
        diff = (got[0, neg].double().cpu() - want[neg]).abs()
        assert bool((diff <= _bound(A, vmax, dh, cells, bf16, io_bf16, want[neg])).all()), float(diff.max())
        keys[table[0].long(), 0, :, dim] = float("inf")
        got = run()
        assert bool((got[0, neg] == 0).all()) and bool(got[0, pos].isnan().all())
        assert torch.equal(got[0, nq // nkv:], plain[0, nq // nkv:]) and torch.equal(got[1], plain[1])


def _reference_without(torch, pages, nq, nkv, dh, page, table, cells, q, gone):
    """The formula for sequence 0 without cell `gone`: its cells moved together into pages of their own."""
    P = pages[table[0].long()].cpu()
    keep = [j for j in range(cells) if j != gone]
    K = P[:, 0, 0].view(-1, nkv, page, dh).transpose(1, 2).reshape(-1, nkv, dh)[keep]
    V = P[:, 0, 1].view(-1, nkv, dh, page).permute(0, 3, 1, 2).reshape(-1, nkv, dh)[keep]
    one = torch.stack([K.permute(1, 0, 2).reshape(-1), V.permute(1, 2, 0).reshape(-1)])[None, None]
    out, A, vmax = _reference(torch, one, 0, nq, nkv, dh, cells - 1, torch.zeros(1, 1, dtype=torch.int64).numpy(),
                              [cells - 1], q[:1], 1 / math.sqrt(dh))
    return out[0], A, vmax


@pytest.mark.parametrize("nq,dh,bf16,io_bf16,page,lengths", [
    (4, 64, False, False, 16, [32768 + 129, 100]),    # ranges of 128 cells: the most ranges, one of them longer
    (3, 128, False, True, 128, [129, 32768 * 2 + 1]),
    (5, 64, True, True, 64, [65536 + 257, 513]),      # ranges of 256
    (2, 128, True, False, 256, [300, 65536 + 257]),
    (4, 128, True, True, 32, [65536, 65537, 0]),
])
def test_as_many_ranges_as_there_are(nq, dh, bf16, io_bf16, page, lengths):
    """More cells than 256 ranges of one step hold: every thread of a join has a range, ranges are
    of several steps, and the other sequences of the call take a few ranges or one."""
    import torch
    import paper_2606_29565_amd as spp
    n, width = len(lengths), -(-max(lengths) // page)
    pool, pages, g = _pool(torch, spp, 1, 1, dh, bf16, page, n * width, seed=nq)
    table = torch.randperm(n * width, generator=g, device="cuda").view(n, width).int()
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.empty(n, nq, dh, device="cuda").normal_(0, 1.5, generator=g).to(
        torch.bfloat16 if io_bf16 else torch.float32)
    att = spp.PagedAttention(pool, 0, nq, table, lens, io_bf16=io_bf16)
    att._work.fill_(255)
    # as many ranges as the join has threads: each leaves dh sums, a maximum and a sum
    assert att._work.numel() == n * nq * 256 * (dh + 2) * 4
    out = att(q, torch.full_like(q, 7.0))
    want, A, vmax = _reference(torch, pages, 0, nq, 1, dh, page, table.cpu().numpy(), lengths, q, 1 / math.sqrt(dh))
    diff = (out.double().cpu() - want).abs()
    for i, m in enumerate(lengths):
        assert bool((diff[i] <= _bound(A, vmax, dh, m, bf16, io_bf16, want[i])).all()), (m, float(diff[i].max()))
    assert torch.equal(out, att(q, torch.empty_like(q)))


@pytest.mark.parametrize("fmt,max_sessions,page,heads", [("bf16", 4, 64, (4, 2, 64)), ("f32", 4, 16, (4, 2, 64)),
                                                         ("bf16", 1, 16, (2, 1, 128)), ("mxfp4", 3, 32, (4, 2, 64))])
def test_a_decode_step_over_several_ranges(fmt, max_sessions, page, heads):
    """Sequences of 1 to 1300 cells decoded together: the step joins its ranges (of 256 cells, 128 in
    fp32) and hands the attention on in its model's form.  Every distribution against the oracle's, where
    256 values less (the first, or the last of 1300 cells) are 0.2 and 0.14, one value less 5e-3."""
    import torch
    import oracle
    import paper_2606_29565_amd as spp
    import synth
    from gpu_util import build_model, log, max_abs
    nq, nkv, dh = heads
    bf16, steps = fmt != "f32", 2
    shape = synth.Shape("paged-long-" + fmt, 2, 256, nq, nkv, dh, 512, 2048, 1e4, "bf16" if bf16 else "f32",
                        wfmt="mxfp4" if fmt == "mxfp4" else "dtype")
    b = build_model(shape, 31, max_sessions=max_sessions, max_tokens=64)
    lengths = [1300, 1, 640, 255, 900]
    text = synth.cpu_tokens(max(lengths), 31, 1, shape.vocab)
    pool, _, _ = _pool(torch, spp, 2, nkv, dh, bf16, page, sum(-(-(m + steps) // page) for m in lengths), max_seqs=8)
    seqs, w = [], oracle.Weights(shape, 31)
    sess = spp.Session(b.model, max(lengths) + 8)
    sess.append_delta(text.tolist())
    for m in lengths:                                  # (a prefix's cells do not depend on what follows)
        sess.restore(m)
        seqs.append(pool.create())
        pool.import_session(seqs[-1], sess)
    toks = synth.cpu_tokens(len(lengths) * steps, 32, 2, shape.vocab).reshape(-1, steps)
    kv = oracle.KVState(shape, max(lengths) + steps)
    oracle.forward(w, kv, 0, text, logits=False)
    want = {}                                          # longest first: the cells overwritten are past the next ones'
    for i in sorted(range(len(lengths)), key=lambda i: -lengths[i]):
        for t in range(steps):
            want[i, t] = oracle.forward(w, kv, lengths[i] + t, toks[i, t:t + 1])
    dists = [torch.empty(shape.vocab, dtype=torch.float32, device="cuda") for _ in seqs]
    worst = 0.0
    for t in range(steps):
        spp.decode_batch(pool, b.model, seqs, toks[:, t].tolist(), dists)
        for i, d in enumerate(dists):
            worst = max(worst, max_abs(d.cpu().numpy(), want[i, t]))
        assert [s.position for s in pool.summaries(seqs)] == [m + t + 1 for m in lengths]
    log(f"paged decode {fmt} {heads} to {max(lengths)} cells: max |logit - oracle| {worst:.2e}")
    assert worst <= (5e-2 if bf16 else 1e-4)
