"""What the calls of 8-bit caches and of log probabilities refuse, and what they answer without a device:
layouts and workspace sizes.  (Device pointers are made up: nothing runs.)"""
import ctypes
import math
import types

import pytest
import torch

import paper_2606_29565_amd as spp

P = 1 << 20  # some device pointer, aligned


def _refused(rc):
    assert rc == spp.SPP_E_INVALID_ARG and spp.lib().spp_last_error()


# ---- pools of codes ----------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [8, 9])
@pytest.mark.parametrize("layers,heads,dh,page", [(1, 1, 64, 16), (2, 3, 128, 64), (4, 8, 128, 256), (3, 5, 64, 32)])
def test_layout_of_a_pool_of_codes(dtype, layers, heads, dh, page):
    cfg = spp.spp_pool_config(layers, heads, dh, dtype, page, 7, 4)
    lay, sc = spp.spp_page_layout(), spp.spp_scale_layout()
    spp.check(spp.lib().spp_pool_page_layout(ctypes.byref(cfg), ctypes.byref(lay)), "")
    spp.check(spp.lib().spp_pool_scale_layout(ctypes.byref(cfg), ctypes.byref(sc)), "")
    codes, blocks = heads * dh * page, page // 16
    assert lay.elem_bytes == 1 and lay.v_offset == codes and sc.block_cells == 16
    assert list(lay.k_stride) == [page * dh, dh, 1] and list(lay.v_stride) == [page * dh, 1, page]
    assert sc.k_offset == 2 * codes and sc.v_offset == 2 * codes + 4 * heads * blocks
    assert list(sc.stride) == [blocks, 1]
    assert lay.layer_stride == 2 * codes + math.ceil(8 * heads * blocks / 128) * 128
    assert lay.page_stride == layers * lay.layer_stride
    assert spp.lib().spp_pool_bytes(ctypes.byref(cfg)) == 7 * lay.page_stride


def test_pools_that_are_no_pools_of_codes():
    sc = spp.spp_scale_layout()
    for dtype in (0, 1):                                     # values: no scales
        cfg = spp.spp_pool_config(1, 1, 64, dtype, 16, 7, 4)
        assert spp.lib().spp_pool_bytes(ctypes.byref(cfg))
        _refused(spp.lib().spp_pool_scale_layout(ctypes.byref(cfg), ctypes.byref(sc)))
    for dtype in (2, 7, 10, -1):
        cfg = spp.spp_pool_config(1, 1, 64, dtype, 16, 7, 4)
        assert spp.lib().spp_pool_bytes(ctypes.byref(cfg)) == 0
        _refused(spp.lib().spp_pool_scale_layout(ctypes.byref(cfg), ctypes.byref(sc)))
    cfg = spp.spp_pool_config(1, 1, 64, 8, 16, 7, 4)
    _refused(spp.lib().spp_pool_scale_layout(ctypes.byref(cfg), None))
    # a page of 2 GiB with its scales, though not without them
    cfg = spp.spp_pool_config(1, (1 << 31) // (2 * 128 * 16) - 1, 128, 8, 16, 1, 4)
    assert spp.lib().spp_pool_bytes(ctypes.byref(cfg)) == 0
    with pytest.raises(ValueError, match="cells"):
        spp.PagePool(1, 1, 64, True, 16, 4, cells="fp8")


def _cells(dev=-1, n=2, width=3, **over):
    """A PagedCells over a stand-in for a pool (-1 is the host's number)."""
    pool = types.SimpleNamespace(handle=ctypes.c_void_p(0), device=dev)
    args = dict(table=torch.zeros(n, width, dtype=torch.int32), first=torch.zeros(n, dtype=torch.int32),
                rows=torch.zeros(n + 1, dtype=torch.int32))
    args.update(over)
    pool.handle = types.SimpleNamespace(value=None) if over.pop("open", True) else None
    pool.cfg = spp.spp_pool_config(1, 2, 64, 8, 16, 7, 4)
    pool.pages = torch.zeros(16, dtype=torch.uint8)
    return spp.PagedCells(pool, 0, args["table"], args["first"], args["rows"], 1)


@pytest.mark.parametrize("over", [
    {"table": torch.zeros(2, 3)}, {"table": torch.zeros(6, dtype=torch.int32)},
    {"table": torch.zeros(3, 2, dtype=torch.int32).t()}, {"first": torch.zeros(3, dtype=torch.int32)},
    {"first": torch.zeros(2, dtype=torch.int64)}, {"first": torch.zeros(4, dtype=torch.int32)[::2]},
    {"rows": torch.zeros(2, dtype=torch.int32)}, {"rows": torch.zeros(6, dtype=torch.int32)[::2]},
], ids=lambda o: "-".join(f"{k}{tuple(v.shape)}{v.dtype}" for k, v in o.items()))
def test_cells_refuse_tables_they_cannot_read(over):
    with pytest.raises(ValueError):
        _cells(**over)
    with pytest.raises(ValueError, match="device"):
        _cells(dev=0)


def test_cells_past_the_checks_need_a_pool():
    with pytest.raises(spp.SppError) as e:
        _cells()
    assert e.value.rc == spp.SPP_E_INVALID_ARG


# ---- log probabilities -----------------------------------------------------------------------------


def _rows(n=2, **over):
    rows = (spp.spp_logprob_row * n)()
    for i in range(n):
        rows[i] = spp.spp_logprob_row(P, P, P, 1)
    for k, v in over.items():
        setattr(rows[n - 1], k, v)
    return rows


def _call(n=2, vocab=100, rows=None, top=3, tt=P, tl=P, lse=P, ent=P, work=P, nbytes=1 << 20):
    return spp.lib().spp_logprobs(n, vocab, _rows() if rows is None else rows, top, tt, tl, lse, ent, work, nbytes, None)


@pytest.mark.parametrize("over", [
    {"n": -1}, {"n": (1 << 20) + 1}, {"vocab": 0}, {"vocab": (1 << 24) + 1}, {"top": -1}, {"top": 65}, {"tt": None},
    {"tl": None}, {"tt": P + 2}, {"tl": P + 1}, {"lse": P + 2}, {"ent": P + 3}, {"work": None}, {"work": P + 8},
    {"nbytes": 16}, {"rows": _rows(logits=None)}, {"rows": _rows(tokens=None)}, {"rows": _rows(logprobs=None)},
    {"rows": _rows(n_tokens=-1)}, {"rows": _rows(n_tokens=(1 << 30) + 1)}, {"rows": _rows(logits=P + 1)},
    {"rows": _rows(tokens=P + 2)}, {"rows": _rows(logprobs=P + 3)},
], ids=lambda o: ",".join(o))
def test_logprobs_refuse(over):
    _refused(_call(**over))


def test_logprobs_of_no_row_and_without_rows():
    assert _call(n=0) == spp.SPP_OK
    _refused(spp.lib().spp_logprobs(1, 100, None, 0, None, None, None, None, P, 1 << 20, None))


@pytest.mark.parametrize("vocab", [1, 100, 8192, 8193, 128256, 1 << 24])
@pytest.mark.parametrize("top", [0, 1, 64])
def test_logprobs_workspace_does_not_fall_with_the_rows(vocab, top):
    sizes = [spp.lib().spp_logprobs_work_bytes(n, vocab, top) for n in range(1, 300)]
    assert all(s > 0 for s in sizes) and sizes == sorted(sizes)
    assert spp.lib().spp_logprobs_work_bytes(1 << 20, vocab, top) >= sizes[-1]
    for bad in ((0, vocab, top), (-1, vocab, top), (1, 0, top), (1, vocab, -1), (1, vocab, 65), ((1 << 20) + 1, vocab, top)):
        assert spp.lib().spp_logprobs_work_bytes(*bad) == 0


ROW = torch.zeros(100)
BAD = {
    "no rows": ([], None, 0), "none": ([None], None, 0), "short": ([torch.zeros(99)], None, 0),
    "bf16": ([ROW.bfloat16()], None, 0), "strided": ([torch.zeros(200)[::2]], None, 0), "on the host": ([ROW], None, 0),
    "tokens of fp32": ([ROW], torch.zeros(1, 2), 0), "tokens of another number": ([ROW], torch.zeros(2, 2, dtype=torch.int32), 0),
    "tokens flat": ([ROW], torch.zeros(1, dtype=torch.int32), 0),
    "tokens strided": ([ROW], torch.zeros(1, 4, dtype=torch.int32)[:, ::2], 0),
}


@pytest.mark.parametrize("what", sorted(BAD))
def test_the_binding_refuses_rows_it_cannot_read(what):
    rows, tokens, top = BAD[what]
    with pytest.raises(ValueError):
        spp.LogProbs(100, rows, tokens=tokens, top=top)
