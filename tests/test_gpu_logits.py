"""Adjusted logits: penalties, biases and allowed sets, with the reductions of the allowed tokens.

Every operation is one fp32 operation with its own rounding, so the adjusted logits, the argmax
and the two largest are compared bit for bit with the same steps in numpy's fp32.  The
log-sum-exp is compared with 64 bits: a term exp(x - m) is off by at most |x - m| 2^-23 + 2^-21
relative (the argument's scaling and the exponential), the sums by 2^-18 (a few dozen additions in a row),
and the logarithm by 2^-21 of its value."""
import math

import numpy as np
import pytest

from gpu_util import log

pytestmark = pytest.mark.gpu


def _expect(x, tokens=(), n_prompt=0, rep=1.0, freq=0.0, pres=0.0, bias_tokens=(), bias=(), allowed=None,
            fill=-math.inf):
    f = np.float32
    V = len(x)
    y = x.copy()
    tokens = np.asarray(tokens, dtype=np.int64)
    inside = (tokens >= 0) & (tokens < V)
    seen = np.zeros(V, bool)
    seen[tokens[inside]] = True
    count = np.bincount(tokens[n_prompt:][inside[n_prompt:]], minlength=V)
    with np.errstate(all="ignore"):
        y[seen] = np.where(y[seen] > 0, y[seen] / f(rep), y[seen] * f(rep))
        c = count > 0
        y[c] = y[c] - f(freq) * count[c].astype(f)
        y[c] = y[c] - f(pres)
        last = {int(t): f(b) for t, b in zip(bias_tokens, bias) if 0 <= t < V}
        for t, b in last.items():
            y[t] = y[t] + b
    ok = np.ones(V, bool) if allowed is None else allowed
    y[~ok] = f(fill)
    return y, ok


def _bitmap(torch, ok):
    words = np.zeros((len(ok) + 31) // 32 * 32, np.uint8)
    words[:len(ok)] = ok
    return torch.from_numpy(np.packbits(words, bitorder="little").view(np.int32)).cuda()


def _check_row(y, ok, s, i):
    live = y[ok]
    nonfinite = not np.isfinite(live).all()
    ids = np.flatnonzero(ok & ~np.isnan(y))
    flags = (1 if nonfinite else 0) | (8 if not ok.any() else 0)
    assert int(s.flags[i]) == flags
    if not len(ids):
        assert int(s.argmax[i]) == -1 and float(s.top1[i]) == -math.inf and math.isnan(float(s.lse[i]))
        return
    order = ids[np.argsort(-y[ids], kind="stable")]
    assert int(s.argmax[i]) == order[0]
    top1 = np.float32(y[order[0]])
    top2 = np.float32(y[order[1]] if len(order) > 1 else -math.inf)
    assert np.float32(float(s.top1[i])) == top1 and np.float32(float(s.top2[i])) == top2
    if nonfinite:
        assert math.isnan(float(s.lse[i]))
        return
    assert np.float32(float(s.gap[i])) == np.float32(top1 - top2)
    d = live.astype(np.float64) - float(top1)
    lse = float(top1) + math.log(np.exp(d).sum())
    p = np.exp(d) / np.exp(d).sum()
    rel = float((p * np.abs(d)).sum()) * 2.0 ** -23 + 2.0 ** -21 + 2.0 ** -18
    bound = rel + (abs(lse) + abs(float(top1)) + abs(lse - float(top1))) * 2.0 ** -21
    assert abs(float(s.lse[i]) - lse) <= bound, (float(s.lse[i]), lse, bound)


@pytest.mark.parametrize("V,n,offset", [(1, 1, 0), (2, 3, 1), (31, 2, 3), (1023, 5, 2), (1024, 1, 0), (1025, 33, 1),
                                        (4096, 4, 0), (50021, 40, 3), (128256, 1, 0), (152063, 9, 0),
                                        (128256, 64, 0), (1022, 6, 0), (129022, 17, 0)])
def test_rows_match_their_steps_bit_for_bit(V, n, offset):
    """(`offset`: elements past a 16-byte boundary, src and dst unlike each other for odd rows.)"""
    import torch
    import paper_2606_29565_amd as spp
    r = np.random.RandomState(V + n)
    xs = r.normal(0, 2, (n, V)).astype(np.float32)
    src = torch.zeros(n, V + 9, device="cuda")
    dst = torch.full((n, V + 9), 5.0, device="cuda")
    rows, want, keep = [], [], []
    for i in range(n):
        o, p = offset, offset + (i % 2)
        src[i, o:o + V] = torch.from_numpy(xs[i])
        T = int(r.choice([0, 1, 7, 300, 5000]))
        tokens = r.randint(-3, V + 3, T).astype(np.int32)
        if T > 3:
            tokens[T // 2:] = tokens[:T - T // 2]          # repeats
        B = int(r.choice([0, 1, 40]))
        bt = r.randint(-2, V + 2, B).astype(np.int32)
        if B > 2:
            bt[-1] = bt[0]                                 # the same index twice: the last counts
        bv = r.normal(0, 3, B).astype(np.float32)
        ok = None
        if r.rand() < 0.6:
            ok = r.rand(V) < r.choice([0.0, 0.01, 0.5, 1.0])
        kw = dict(n_prompt=int(r.randint(0, T + 1)), rep=float(r.choice([1.0, 0.7, 1.3])),
                  freq=float(r.choice([0.0, 0.3, -0.2])), pres=float(r.choice([0.0, 0.15])),
                  fill=float(r.choice([-math.inf, -3.4e38, 0.0])))
        want.append(_expect(xs[i], tokens, bias_tokens=bt, bias=bv, allowed=ok, **kw))
        dev = [torch.from_numpy(a).cuda() for a in (tokens, bt, bv)]
        rows.append(spp.AdjustRow(src[i, o:o + V], dst[i, p:p + V], tokens=dev[0], n_prompt=kw["n_prompt"],
                                  repetition=kw["rep"], frequency=kw["freq"], presence=kw["pres"],
                                  bias_tokens=dev[1], bias=dev[2], fill=kw["fill"],
                                  allowed=None if ok is None else _bitmap(torch, ok)))
    call = spp.LogitsAdjust(V, rows)
    call._work.fill_(255)
    s = call()
    for i in range(n):
        y, ok = want[i]
        got = dst[i, offset + (i % 2):offset + (i % 2) + V].cpu().numpy()
        assert np.array_equal(got, y), (i, np.flatnonzero(got != y)[:5])
        _check_row(y, ok, s, i)
        edge = dst[i].cpu().numpy()
        assert (edge[:offset + (i % 2)] == 5).all() and (edge[offset + (i % 2) + V:] == 5).all()
        assert np.array_equal(src[i, offset:offset + V].cpu().numpy(), xs[i])


def test_nonfinite_logits_ties_and_masked_values():
    import torch
    import paper_2606_29565_amd as spp
    V = 5000
    base = np.linspace(-1, 1, V).astype(np.float32)
    plans = []
    a = base.copy(); a[7] = np.nan
    plans.append((a, None))
    ok = np.ones(V, bool); ok[7] = False
    plans.append((a, ok))                                   # NaN in a masked place
    b = base.copy(); b[3] = np.inf
    plans.append((b, None))
    c = base.copy(); c[100] = c[4000] = 9.0
    plans.append((c, None))                                 # a tie: gap 0, the lowest index
    d = np.full(V, -np.inf, np.float32)
    plans.append((d, None))                                 # only -inf: the first, not finite
    e = base.copy(); e[:] = np.nan
    plans.append((e, None))
    plans.append((base, np.zeros(V, bool)))                 # nothing allowed
    one = np.zeros(V, bool); one[V - 1] = True
    plans.append((base, one))                               # one token: no second
    f = base.copy(); f[9] = -3.4028235e38
    plans.append((f, None))
    g = base.copy(); g[4999] = 3.4028235e38; g[17] = -3.4028235e38
    plans.append((g, None))                                 # the whole range of the type
    h = base.copy(); h[20] = -np.inf
    plans.append((h, None))                                 # an -inf among others
    ok = np.zeros(V, bool); ok[[20, 21, 4000]] = True
    plans.append((h, ok))                                   # ... and allowed
    h2 = np.full(V, -np.inf, np.float32); h2[20] = np.nan
    plans.append((h2, ok))                                  # nothing finite is allowed
    k = base.copy(); k.view(np.uint32)[[4, 4998]] = 0x7FA00000, 0xFFA00001
    plans.append((k, None))                                 # signalling NaN, one beside the largest
    src = torch.stack([torch.from_numpy(p[0]) for p in plans]).cuda()
    rows = [spp.AdjustRow(src[i], src[i], allowed=None if p[1] is None else _bitmap(torch, p[1]), fill=-3.4028235e38)
            for i, p in enumerate(plans)]                   # in place
    s = spp.LogitsAdjust(V, rows)()
    for i, p in enumerate(plans):
        y, ok = _expect(p[0], allowed=p[1], fill=-3.4028235e38)
        assert np.array_equal(src[i].cpu().numpy(), y, equal_nan=True), i
        _check_row(y, ok, s, i)


def test_the_same_call_gives_the_same_bits():
    import torch
    import paper_2606_29565_amd as spp
    V, n = 60000, 70
    g = torch.Generator(device="cuda").manual_seed(8)
    src = torch.empty(n, V, device="cuda").normal_(0, 2, generator=g)
    tok = torch.randint(0, 500, (n, 3000), generator=g, device="cuda").int()
    got = []
    for _ in range(3):
        out = torch.empty_like(src)
        s = spp.LogitsAdjust(V, [spp.AdjustRow(src[i], out[i], tokens=tok[i], n_prompt=1000, repetition=1.3,
                                               frequency=0.01, presence=0.2) for i in range(n)])()
        got.append((out, s.argmax.clone(), s.top1.clone(), s.top2.clone(), s.lse.clone()))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_adjusted_logits_are_gated_and_replayed_from_a_graph():
    """A ready distribution adjusted in place is what the gate scans; a captured call reads
    the logits and the history as they are at each replay."""
    import torch
    import synth
    import paper_2606_29565_amd as spp
    from gpu_util import build_model
    shape = synth.Shape("adj", 1, 256, 4, 2, 64, 512, 2048, 1e4, "f32")
    b = build_model(shape, 4)
    sess = spp.Session(b.model, 64)
    dist = torch.empty(shape.vocab, device="cuda")
    ready = sess.preposition([1, 2, 3], dist)
    torch.cuda.synchronize()
    ids = [11, 500, 1999]
    allowed = torch.from_numpy(synth.bitmap_from_ids(shape.vocab, ids).view(np.int32)).cuda()
    best = max(ids, key=lambda t: float(dist[t]))
    call = spp.LogitsAdjust(shape.vocab, [spp.AdjustRow(dist, dist, allowed=allowed, fill=-3e38)])
    s = call()
    torch.cuda.synchronize()
    outcome, token, summ = spp.gate(ready, 0.0, allowed)
    assert (outcome, token) == (spp.SPP_SERVED, best) and int(s.argmax[0]) == best
    assert summ.gap == float(s.gap[0])
    # an infinite fill is never served
    spp.LogitsAdjust(shape.vocab, [spp.AdjustRow(dist, dist, allowed=allowed)])()
    torch.cuda.synchronize()
    assert spp.gate(ready, 0.0, allowed)[0] == spp.SPP_FALL_NONFINITE

    n, V = 3, 40000
    src = torch.empty(n, V, device="cuda").normal_()
    out = torch.empty_like(src)
    hist = torch.zeros(n, 50, dtype=torch.int32, device="cuda")
    rows = [spp.AdjustRow(src[i], out[i], tokens=hist[i], repetition=1.4, frequency=0.5) for i in range(n)]
    call = spp.LogitsAdjust(V, rows)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = call()
    r = np.random.RandomState(3)
    for k in range(4):
        src.normal_(0, 2)
        h = r.randint(0, V, (n, 50)).astype(np.int32)
        h[:, :5] = src.argmax(1).cpu().numpy()[:, None]
        hist.copy_(torch.from_numpy(h))
        graph.replay()
        torch.cuda.synchronize()
        for i in range(n):
            y, ok = _expect(src[i].cpu().numpy(), h[i], rep=1.4, freq=0.5)
            assert np.array_equal(out[i].cpu().numpy(), y), k
            _check_row(y, ok, s, i)


def test_refused_rows():
    import torch
    import paper_2606_29565_amd as spp
    x = torch.zeros(100, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for kw in ({"repetition": 0.0}, {"repetition": -1.0}, {"repetition": math.nan}, {"repetition": math.inf},
               {"frequency": math.inf}, {"presence": math.nan}, {"fill": math.nan}, {"n_prompt": 5},
               {"n_prompt": -1}):
        with pytest.raises(spp.SppError) as e:
            spp.LogitsAdjust(100, [spp.AdjustRow(x, x), spp.AdjustRow(x, x, tokens=t, **kw)])()
        assert e.value.rc == spp.SPP_E_INVALID_ARG and "row 1" in str(e.value)
    for bad in (dict(src=x.double(), dst=x), dict(src=x[:50], dst=x), dict(src=x, dst=None),
                dict(src=x, dst=x, tokens=t.long()), dict(src=x, dst=x, n_tokens=3),
                dict(src=x, dst=x, tokens=t, n_tokens=5), dict(src=x, dst=x, bias_tokens=t),
                dict(src=x, dst=x, allowed=t[:3]), dict(src=x.cpu(), dst=x), dict(src=x, dst=x, tokens=t.cpu())):
        with pytest.raises((ValueError, AttributeError)):
            spp.LogitsAdjust(100, [spp.AdjustRow(**bad)])
    assert not x.any()
    with pytest.raises(spp.SppError):
        spp.lib()  # (a workspace that is too small)
        call = spp.LogitsAdjust(100, [spp.AdjustRow(x, x)])
        call._args = call._args[:5] + (8,)
        call()
