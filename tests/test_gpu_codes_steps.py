"""What decode steps append to a cache of 8-bit codes, against the definition bit for bit."""
import numpy as np
import pytest

import synth
from gpu_util import build_model, fill_synthetic_kv, log
from test_gpu_codes import BLOCK, Cache, _pool, _scales, _views

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code,page", [("i8", 16), ("e4m3", 32), ("i8", 64), ("e4m3", 256)])
def test_decode_steps_append_bit_for_bit(code, page):
    """A pool of fp32 values holds what a step of an fp32 model quantises: layer 0's new cells depend on no cache.  Codes and
    scales of a pool of codes are the definition's of those values, written one by one.  The cells that the sequences
    start with are small, so that the first step makes a block's scale grow."""
    import torch
    import paper_2606_29565_amd as spp
    shape = synth.Shape("codes", 2, 256, 4, 2, 64, 512, 2048, 1e4, "f32")
    b = build_model(shape, 3, max_sessions=8)
    n, steps, nkv, dh = 37, 30, 2, 64
    sess = spp.Session(b.model, 100)
    fill_synthetic_kv(b, sess, 5, n)
    lay = b.model.kv_layout(sess.capacity, 0)
    k = sess.kv[lay.k_offset:lay.k_offset + nkv * lay.k_stride[0] * 4].view(torch.float32).view(nkv, -1, dh)
    v = sess.kv[lay.v_offset:lay.v_offset + nkv * lay.v_stride[0] * 4].view(torch.float32).view(nkv, dh, -1)
    k[:, 32:n] *= 2.0 ** -12
    v[:, :, 32:n] *= 2.0 ** -12
    sess.restore(n)
    pool, pages, _ = _pool(torch, spp, 2, nkv, dh, code, page, 64, fill=0xFF)
    plain = spp.PagePool(2, nkv, dh, False, page, 64)
    a, p = pool.create(), plain.create()
    pool.import_session(a, sess)
    plain.import_session(p, sess)
    forks, pforks = pool.fork(a, 5), plain.fork(p, 5)
    dists, pdists = (torch.empty(5, shape.vocab, device="cuda") for _ in range(2))
    for step in range(steps):                                 # past the ends of two blocks
        toks = [(t * (step + 1) + step) % shape.vocab for t in (3, 77, 1500, 8, 900)]
        spp.decode_batch(pool, b.model, forks, toks, list(dists))
        spp.decode_batch(plain, b.model, pforks, toks, list(pdists))
    torch.cuda.synchronize()
    m, grew = n + steps, [0, 0]
    blocks = -(-m // BLOCK)
    codes = _views(torch, pool, pages)[:2]
    ks, vs = _scales(torch, pool, pages, 0)
    for f, pf in zip(forks, pforks):
        pv = plain.pages.view(torch.float32).view(64, 2, 2, -1)[torch.tensor(plain.table(pf), device="cuda"), 0]
        vals = (pv[:, 0].reshape(-1, nkv, page, dh).transpose(1, 2).reshape(-1, nkv, dh)[:m].double().cpu().numpy(),
                pv[:, 1].reshape(-1, nkv, dh, page).permute(0, 3, 1, 2).reshape(-1, nkv, dh)[:m].double().cpu().numpy())
        cache = Cache(1, blocks * BLOCK, nkv, dh, code)
        cache.write(0, 0, vals[0][:n], vals[1][:n])
        for c in range(n, m):
            was = [s[0, c // BLOCK].copy() for s in cache.s]
            cache.write(0, c, vals[0][c:c + 1], vals[1][c:c + 1])
            for w in range(2):
                grew[w] += int(c % BLOCK > 0 and (cache.s[w][0, c // BLOCK] > was[w]).any())
        pg = torch.tensor(pool.table(f), device="cuda")
        T = pool.table(f)
        for w, scales in ((0, ks), (1, vs)):
            got = scales[T].transpose(0, 2, 1).reshape(-1, nkv)[:blocks]
            assert np.array_equal(got, cache.s[w][0]), (w, got / cache.s[w][0])
            c8 = codes[w][pg, 0].cpu().double()               # K [page, head, cell, dim], V [page, head, dim, cell]
            c8 = c8.permute(0, 2, 1, 3) if w == 0 else c8.permute(0, 3, 1, 2)
            c8 = c8.reshape(-1, nkv, dh)[:m].numpy()
            want = cache.x[w][0, :m] / np.repeat(cache.s[w][0], BLOCK, 0)[:m, :, None]
            assert np.array_equal(c8, want), (w, int((c8 != want).sum()))
    assert min(grew) >= 5                                     # (every fork's first step)
    log(f"steps over {code}: {grew} scales grew")
    pool.close(), plain.close()
