"""Log probabilities, entropy and alternatives against the definition in 64 bits.

Bounds, with u = 2^-24.  A term e^d, d = x - m, is formed in up to seven stages (against the thread's largest value so
far, three times brought to a new one, to the wave's, the workgroup's, the row's), whose d's add up to its own.  A stage
is off by a relative (3 |d| + 4) u: d and its product with log2 e round once each and the constant is off by less than
u, times the derivative's |d|; the exponential is off by one step; and by u for the product with it.  So e(d) = (3 |d| +
34) u.  R, a sum of terms of one sign, is off by their weighed mean of e(d) and by N u, N = 64 + the slices for the
additions on a term's way (32 and 3 in a thread, 6 in a wave, 4, then the slices' and 10); log(1 + R) by no more,
relatively, and 2 steps of its own.  Sums of e^d d likewise, with 3 u more a stage for the sum that it is brought to a new value by.  The
results round a few times more:
  lse: |lse| u + E log(1 + R);  log p: (|x - m| + |log p|) u + E log(1 + R);  H: (E' + 8 u) H."""
import math

import numpy as np
import pytest

from gpu_util import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _want(x, tokens, top):
    """(logprobs, lse, entropy, top tokens, top logprobs) of one row, and what each may be off by."""
    x = x.astype(np.float64)
    V = len(x)
    order = np.lexsort((np.arange(V), -x))                    # (NaN last)
    order = [i for i in order[:top] if x[i] > -np.inf]
    tt = np.full(top, -1, np.int64)
    tt[:len(order)] = order
    given = [x[t] if 0 <= t < V else np.nan for t in tokens]
    nan = np.full(len(tokens), np.nan)
    if np.isnan(x).any() or (x == np.inf).any():
        tl = np.where(tt >= 0, np.nan, -np.inf)
        return (nan, np.nan, np.nan, tt, tl), None
    if (x == -np.inf).all():
        return (nan, -np.inf, np.nan, tt, np.full(top, -np.inf)), None
    live = x[x > -np.inf]
    m = live.max()
    d = np.delete(live, int(live.argmax())) - m
    w = np.exp(d)
    R = w.sum()
    rest = math.log1p(R)
    lse, H = m + rest, rest - (w * d).sum() / (1 + R)
    N = 64 + V / 8192
    E = ((w * (3 * -d + 34)).sum() / R if R > 0 else 0.0) * U + (N + 4) * U
    T = (w * -d).sum()
    E2 = ((w * -d * (3 * -d + 57)).sum() / T if T > 0 else 0.0) * U + (N + 4) * U
    lp = np.array([g - m - rest for g in given])
    near = lambda v, l: (np.abs(v - m) + np.abs(l)) * U + E * rest + 1e-37  # noqa: E731
    tl = np.where(tt >= 0, x[tt] - m - rest, -np.inf)
    off = (near(np.array(given), lp), abs(lse) * U + E * rest, (max(E, E2) + 8 * U) * H + 1e-37,
           near(x[tt], tl) if top else np.zeros(0))
    return (lp, lse, H, tt, tl), off


def _check(r, rows, tokens, top):
    """Every result of a call against the definition; the largest share of its bound that one used."""
    used = 0.0
    for i, row in enumerate(rows):
        (lp, lse, H, tt, tl), off = _want(row.cpu().numpy(), [] if tokens is None else tokens[i].tolist(), top)
        got = [t[i].double().cpu().numpy() for t in (r.logprobs, r.lse, r.entropy, r.top_logprobs)]
        assert np.array_equal(r.top_tokens[i].cpu().numpy(), tt), (i, r.top_tokens[i].cpu().numpy()[:8], tt[:8])
        for k, (g, w) in enumerate(zip(got, (lp, lse, H, tl))):
            g, w = np.atleast_1d(g), np.atleast_1d(w)
            w = np.where(np.abs(w) > 2.0 ** 128, np.copysign(np.inf, w), w)  # (what fp32 rounds to an infinity)
            fine = np.isfinite(w)
            assert np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(g[~fine & ~np.isnan(w)], w[~fine & ~np.isnan(w)]), (i, k)
            if fine.any():
                share = np.abs(g[fine] - w[fine]) / np.broadcast_to(off[k], w.shape)[fine]
                assert (share <= 1).all(), (i, k, float(share.max()))
                used = max(used, float(share.max()))
    return used


CASES = [
    # vocab, rows, tokens, top, share of logits that are not -inf, offset of the rows in elements
    (1, 2, 1, 1, 1.0, 0),
    (2, 3, 2, 2, 1.0, 1),
    (3, 2, 1, 64, 1.0, 3),
    (65, 5, 3, 8, 0.3, 2),
    (4096, 1, 1, 0, 1.0, 0),
    (4099, 7, 300, 5, 1.0, 1),
    (8189, 4, 1, 64, 0.02, 3),
    (8192, 3, 0, 20, 1.0, 0),
    (8193, 3, 2, 20, 1.0, 2),
    (32000, 64, 4, 8, 1.0, 0),
    (128256, 1, 1, 20, 1.0, 0),
    (128256, 2, 1, 64, 0.001, 1),
    (152063, 17, 64, 50, 0.5, 0),
    (152063, 5, 5, 1, 1.0, 2),
    (5000, 200, 2, 3, 1.0, 0),                   # three launches
    (1 << 22, 1, 2, 64, 1.0, 0),                 # more groups than the merge holds
    (128256, 3, 300, 64, 1.0, 1),
    (300001, 2, 1, 33, 0.9, 3),
]


@pytest.mark.parametrize("V,n,m,top,share,offset", CASES)
def test_against_the_definition(V, n, m, top, share, offset):
    import torch
    import paper_2606_29565_amd as spp
    g = torch.Generator(device="cuda").manual_seed(V + n)
    buf = torch.empty(n, V + 4, device="cuda").normal_(0, 2, generator=g)
    x = buf[:, offset:offset + V]
    if share < 1:
        x[torch.rand(n, V, device="cuda", generator=g) >= share] = -math.inf
        x[:, V // 2] = 1.0
    tokens = torch.randint(0, V, (n, m), device="cuda", generator=g).int() if m else None
    if m > 1:
        tokens[0, 0], tokens[0, 1], tokens[-1, -1] = -1, V, -2 ** 31
    call = spp.LogProbs(V, list(x), tokens=tokens, top=top)
    call._work.fill_(255)
    r = call()
    used = _check(r, x, tokens, top)
    log(f"vocab {V}, {n} rows, top {top}: {used:.2f} of the bound")
    kept = [t.clone() for t in (r.logprobs, r.lse, r.entropy, r.top_tokens, r.top_logprobs)]
    r = call()                                   # the same bits again
    for a, b in zip(kept, (r.logprobs, r.lse, r.entropy, r.top_tokens, r.top_logprobs)):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))


def test_ties_and_rows_of_one_value():
    """Logits of few values, so that many are equal, sorted rows, and rows that are one value throughout."""
    import torch
    import paper_2606_29565_amd as spp
    g = torch.Generator(device="cuda").manual_seed(2)
    V = 20001                                     # (and 20000 of 8189: rows done in one launch)
    rows = [torch.randint(-3, 4, (V,), device="cuda", generator=g).float(),
            torch.randint(-300, 300, (V,), device="cuda", generator=g).float() / 16,
            torch.zeros(V, device="cuda"), torch.full((V,), -7.5, device="cuda"),
            torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0),   # one value: -0 is 0
            torch.arange(V, device="cuda").float() / 1000, -torch.arange(V, device="cuda").float() / 1000,
            (torch.arange(V, device="cuda") // 64).float(), torch.full((V,), -3.4e38, device="cuda"),
            (torch.arange(V, device="cuda") % 64 < 10).float() * 5]
    # few allowed, the others at the lowest number: fewer than are asked, then equal ones in order
    few = torch.full((V,), -3.402823466e38, device="cuda")
    few[torch.tensor([3, 19000, 700], device="cuda")] = torch.tensor([1.0, 2.0, 1.0], device="cuda")
    rows += [few, torch.where(torch.arange(V, device="cuda") < 19990, -math.inf, few)]
    for size in (V, 8189):
        for top in (1, 7, 64):
            part = [x[V - size:] for x in rows]
            _check(spp.LogProbs(size, part, top=top)(), part, None, top)


@pytest.mark.parametrize("V,offset", [(2500, 1), (8189, 0), (8193, 3), (40003, 2), (128256, 0), (300001, 1)])
def test_more_equals_than_a_list_holds(V, offset):
    """Some values above one that most of the row has: none, one or `top` - 1 of them, all in a group of 32 tokens or
    far apart, the equals from the start, behind what is masked, or every 33rd token; in infinities too."""
    import torch
    import paper_2606_29565_amd as spp
    g = torch.Generator(device="cuda").manual_seed(V)
    idx = torch.arange(V, device="cuda")
    for top in (1, 20, 64):
        rows = []
        for fill in (0.0, -3.402823466e38, math.inf):
            for above in sorted({0, 1, top - 1}):
                for how in range(4):
                    x = torch.full((V,), fill, device="cuda")
                    if how == 1:
                        x[:V * 5 // 8 - 3] = -math.inf
                    elif how == 2:
                        x[idx % 33 != 0] = -2.0
                    if above and fill != math.inf:
                        at = (torch.arange(above, device="cuda") + V // 3 if how == 3
                              else torch.randperm(V, device="cuda", generator=g)[:above])
                        x[at] = 1.0 + torch.rand(above, device="cuda", generator=g)
                    rows.append(x)
        buf = torch.empty(len(rows), V + 4, device="cuda")
        part = buf[:, offset:offset + V]
        part.copy_(torch.stack(rows))
        with np.errstate(all="ignore"):
            _check(spp.LogProbs(V, list(part), top=top)(), part, None, top)
    log(f"vocab {V}: in order")


def test_masked_rows_and_values_that_are_not_finite():
    import torch
    import paper_2606_29565_amd as spp
    V = 9000
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(12, V, device="cuda").normal_(generator=g)
    x[0] = -math.inf                                           # nothing is allowed
    x[1] = -math.inf
    x[1, 8999] = 3.0                                           # one token, in the last slice
    x[2, 8500] = math.nan
    x[3, 5], x[3, 8192] = math.inf, math.inf
    x[4] = math.nan
    x[5] = math.inf
    x[6, :8999] = -math.inf
    x[6, 8999] = math.nan
    x[7, 1:] = -math.inf
    x[8, 100] = 60.0                                           # near certain: log p about -e^-60 V
    x[9] = -math.inf
    x[9, 3], x[9, 8700] = -3.0e38, 3.0e38                      # further apart than an fp32 number is long
    x[10, 17] = -math.nan
    x[11] = torch.where(torch.arange(V, device="cuda") < 8192, -math.inf, x[11])
    tokens = torch.tensor([[3, 100, 8999, 8192, -5]] * 12, dtype=torch.int32, device="cuda")
    for top in (0, 3, 64):
        r = spp.LogProbs(V, list(x), tokens=tokens, top=top)()
        with np.errstate(all="ignore"):
            _check(r, x, tokens, top)
    assert -1e-20 < float(r.logprobs[8, 1]) < 0                # (kept, not rounded to 0)


def test_replayed_from_a_graph_and_on_another_stream():
    import torch
    import paper_2606_29565_amd as spp
    V, n, top = 40000, 6, 12
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(n, V, device="cuda").normal_(generator=g)
    tokens = torch.zeros(n, 3, dtype=torch.int32, device="cuda")
    call = spp.LogProbs(V, list(x), tokens=tokens, top=top)
    r = call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    eager = spp.LogProbs(V, list(x), tokens=tokens, top=top)
    side = torch.cuda.Stream()
    for k in range(4):
        x.normal_(generator=g)
        tokens.random_(0, V, generator=g)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (r.logprobs, r.lse, r.entropy, r.top_tokens, r.top_logprobs)]
        side.wait_stream(torch.cuda.current_stream())
        e = eager(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(got, (e.logprobs, e.lse, e.entropy, e.top_tokens, e.top_logprobs)):
            assert torch.equal(a, b), k
        _check(e, x, tokens, top)


def test_results_that_are_not_asked():
    """lse and entropy are each nullable, and rows may have lists of differing lengths."""
    import ctypes

    import torch
    import paper_2606_29565_amd as spp
    V = 700
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty(3, V, device="cuda").normal_(generator=g)
    tok = torch.tensor([5, 699, 0, 3], dtype=torch.int32, device="cuda")
    out = torch.full((4,), 9.0, device="cuda")
    ent = torch.full((3,), 9.0, device="cuda")
    rows = (spp.spp_logprob_row * 3)(
        spp.spp_logprob_row(x[0].data_ptr(), tok.data_ptr(), out.data_ptr(), 1),
        spp.spp_logprob_row(x[1].data_ptr(), None, None, 0),
        spp.spp_logprob_row(x[2].data_ptr(), tok.data_ptr() + 4, out.data_ptr() + 4, 2))
    nbytes = spp.lib().spp_logprobs_work_bytes(3, V, 0)
    work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    for lse, entropy in ((None, None), (None, ent.data_ptr())):
        spp.check(spp.lib().spp_logprobs(3, V, rows, 0, None, None, lse, entropy, work.data_ptr(), nbytes, st), "")
    want = torch.log_softmax(x.double(), 1)
    for got, w in ((out[0], want[0, 5]), (out[1], want[2, 699]), (out[2], want[2, 0])):
        assert abs(float(got) - float(w)) < 1e-5
    assert float(out[3]) == 9.0                                # past the last list
    assert float((ent.double() + (want.exp() * want).sum(1)).abs().max()) < 1e-5


def test_continuations_compared_after_decode_steps():
    """Operators together: a session's cells in 8 bits, forks decoded, their tokens' log probabilities summed,
    and the best one exported; the sums are those of the logits that the steps wrote."""
    import torch
    import paper_2606_29565_amd as spp
    import synth
    from gpu_util import build_model, fill_synthetic_kv
    for code in ("i8", "e4m3"):
        shape = synth.Shape("codes", 2, 256, 4, 2, 64, 512, 2048, 1e4, "bf16")
        b = build_model(shape, 3, max_sessions=4)
        sess = spp.Session(b.model, 80)
        fill_synthetic_kv(b, sess, 5, 30)
        sess.restore(30)
        pool = spp.PagePool(2, 2, 64, True, 16, 40, cells=code)
        seq = pool.create()
        pool.import_session(seq, sess)
        forks = pool.fork(seq, 4)
        dists = [torch.empty(2048, device="cuda") for _ in forks]
        chosen = torch.empty(4, 1, dtype=torch.int32, device="cuda")
        score = spp.LogProbs(2048, dists, tokens=chosen, top=4)
        spp.decode_batch(pool, b.model, forks, [1, 2, 3, 4], dists)
        total, plain = torch.zeros(4, device="cuda"), np.zeros(4)
        for step in range(5):
            r = score()
            # fork i takes its i-th alternative first, then the best
            pick = r.top_tokens[torch.arange(4), torch.arange(4) if step == 0 else 0]
            chosen.copy_(pick[:, None])
            r = score()
            total += r.logprobs[:, 0]
            for i, d in enumerate(dists):
                plain[i] += float(torch.log_softmax(d.double(), 0)[int(pick[i])])
            spp.decode_batch(pool, b.model, forks, pick.tolist(), dists)
        assert np.abs(total.cpu().numpy() - plain).max() < 5 * 2e-5
        best = forks[int(total.argmax())]
        pool.export_session(best, sess)
        assert sess.info().n_committed == 30 + 6
        pool.close()
