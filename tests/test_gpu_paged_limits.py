"""Attention over paged caches where its rules change or reach their ends: workspaces of smaller
calls.  The bound of a result is that of test_gpu_paged.py."""
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
