"""Attention over caches of 8-bit codes with a bound for each element (attention_parts.py), which the low bf16 parts of the
query and of the probabilities are well above: rows whose roundings line up, and ordinary ones."""
import math

import numpy as np
import pytest

from attention_parts import aligned_case, row
from gpu_util import log
from test_gpu_codes import _pool, _values, _views

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("io_bf16", [False, True])
def test_attention_of_rows_whose_roundings_line_up(code, dh, io_bf16):
    import torch
    import paper_2606_29565_amd as spp
    heads, page, lengths = 4, 32, [17, 40, 64]
    pool, pages, _ = _pool(torch, spp, 1, heads, dh, code, page, 6, fill=0)
    k, v, ks, vs = _views(torch, pool, pages)
    table = torch.tensor([[4, 1], [0, 5], [3, 2]], dtype=torch.int32, device="cuda")
    q = torch.empty(3, heads, dh, device="cuda", dtype=torch.bfloat16 if io_bf16 else torch.float32)
    want, off = np.empty((3, heads, dh)), np.empty((3, heads, dh))
    for i, n in enumerate(lengths):
        for h in range(heads):
            qq, K, sk, V, sv, scale = aligned_case(code, dh, io_bf16, n, seed=10 * n + h)
            want[i, h], off[i, h] = row(qq, K * sk, V * sv, scale, io_bf16)
            q[i, h] = torch.from_numpy(qq).to(q)
            for j in range(0, n, page):
                pg, m = int(table[i, j // page]), min(page, n - j)
                k[pg, 0, h, :m] = torch.from_numpy(K[j:j + m]).cuda().to(k.dtype)
                v[pg, 0, h, :, :m] = torch.from_numpy(V[j:j + m].T.copy()).cuda().to(v.dtype)
            ks[table[i].long(), 0, h], vs[table[i].long(), 0, h] = sk, sv
    att = spp.PagedAttention(pool, 0, heads, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), io_bf16=io_bf16)
    got = att(q, torch.empty_like(q)).double().cpu().numpy()
    share = np.abs(got - want) / off
    log(f"aligned roundings {code} x{dh} {'bf16' if io_bf16 else 'fp32'}: {share.max():.2f} of the bound")
    assert (share <= 1).all(), float(share.max())


ROWS = [
    # nq, nkv, dh, code, io bf16, page, lengths
    (4, 4, 64, "i8", False, 16, [1, 2, 15, 16, 17, 63, 64, 65, 512]),
    (6, 2, 64, "e4m3", False, 16, [3, 31, 129, 255, 257, 700]),
    (6, 2, 64, "i8", True, 64, [5, 64, 300, 1000]),
    (32, 8, 128, "i8", False, 64, [1, 40, 600]),
    (20, 1, 128, "e4m3", True, 128, [9, 130, 511]),
    (40, 2, 128, "e4m3", False, 32, [33, 1000]),
]


@pytest.mark.parametrize("nq,nkv,dh,code,io_bf16,page,lengths", ROWS)
def test_attention_with_a_bound_for_each_row(nq, nkv, dh, code, io_bf16, page, lengths):
    import torch
    import paper_2606_29565_amd as spp
    n, width = len(lengths), -(-max(lengths) // page)
    pool, pages, g = _pool(torch, spp, 1, nkv, dh, code, page, n * width, seed=nq + page)
    if code == "e4m3":                                        # (no code that is NaN)
        k, v, _, _ = _views(torch, pool, pages)
        for t in (k, v):
            bits = t.view(torch.uint8)
            bits[(bits & 0x7F) == 0x7F] = 0x30
    table = torch.randperm(n * width, generator=g, device="cuda").view(n, width).int()
    q = torch.empty(n, nq, dh, device="cuda").normal_(0, 1.5, generator=g).to(torch.bfloat16 if io_bf16 else torch.float32)
    att = spp.PagedAttention(pool, 0, nq, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), io_bf16=io_bf16)
    got = att(q, torch.empty_like(q)).double().cpu().numpy()
    K, V = (t.numpy() for t in _values(torch, pool, pages, 0))
    T, qq, most = table.cpu().numpy(), q.double().cpu().numpy(), 0.0
    for i, m in enumerate(lengths):
        at = np.arange(m)
        for h in range(nq):
            k1, v1 = (x[T[i][at // page], h // (nq // nkv), at % page] for x in (K, V))
            want, off = row(qq[i, h], k1, v1, 1 / math.sqrt(dh), io_bf16)
            share = np.abs(got[i, h] - want) / off
            assert (share <= 1).all(), (m, h, float(share.max()))
            most = max(most, float(share.max()))
    log(f"attention {code} {nq}/{nkv}x{dh}: {most:.2f} of the bound")


@pytest.mark.parametrize("nq,nkv,dh,page,cells,ranges", [
    (32, 8, 128, 64, 512, 1), (32, 8, 128, 64, 513, 3), (32, 8, 128, 64, 768, 3), (32, 8, 128, 256, 1000, 4),
    (4, 2, 64, 16, 513, 1), (4, 2, 64, 16, 768, 1), (4, 2, 64, 16, 769, 4),
])
@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_a_short_sequence_alone_is_dealt_out_by_its_head_size(code, nq, nkv, dh, page, cells, ranges):
    """One sequence of three steps of 256 cells: a workgroup for each step of heads of 128, one for all of heads of 64; and
    what it gives."""
    import ctypes

    import torch
    import paper_2606_29565_amd as spp
    width = -(-cells // page)
    pool, pages, g = _pool(torch, spp, 1, nkv, dh, code, page, width, seed=cells)
    if code == "e4m3":
        for t in _views(torch, pool, pages)[:2]:
            bits = t.view(torch.uint8)
            bits[(bits & 0x7F) == 0x7F] = 0x30
    table = torch.randperm(width, generator=g, device="cuda").view(1, width).int()
    att = spp.PagedAttention(pool, 0, nq, table, torch.tensor([cells], dtype=torch.int32, device="cuda"), io_bf16=False)
    nbytes = spp.lib().spp_paged_attention_work_bytes(ctypes.byref(att._a))
    assert nbytes == (0 if ranges == 1 else nq * ranges * (dh + 2) * 4)
    q = torch.empty(1, nq, dh, device="cuda").normal_(0, 1.5, generator=g)
    got = att(q, torch.empty_like(q))[0].double().cpu().numpy()
    K, V = (t.numpy() for t in _values(torch, pool, pages, 0))
    at, T = np.arange(cells), table[0].cpu().numpy()
    for h in range(nq):
        k1, v1 = (x[T[at // page], h // (nq // nkv), at % page] for x in (K, V))
        want, off = row(q[0, h].double().cpu().numpy(), k1, v1, 1 / math.sqrt(dh), False)
        assert (np.abs(got[h] - want) <= off).all(), h
