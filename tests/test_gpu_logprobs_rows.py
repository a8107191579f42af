"""Log probabilities of rows whose logits have a common offset or a small spread, and of the longest rows, against the
definition in 64 bits and with the bounds of test_gpu_logprobs.py.  An offset does not change a row's probabilities, so neither does it change how
its alternatives are found."""
import math

import numpy as np
import pytest

from gpu_util import log
from test_gpu_logprobs import _check, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [2500, 8189, 8193, 32000, 128256])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_rows_with_an_offset(V, top):
    import torch
    import paper_2606_29565_amd as spp
    g = torch.Generator(device="cuda").manual_seed(V + top)
    rows = []
    for offset, spread in ((300, 2), (-300, 2), (1000, 2), (-1000, 2), (300, 0.01), (1e6, 3), (0, 1e-3), (0, 1e4)):
        rows.append(torch.empty(V, device="cuda").normal_(offset, spread, generator=g))
    half = rows[0].clone()
    half[torch.rand(V, device="cuda", generator=g) >= 0.5] = -math.inf
    few = rows[3].clone()
    few[torch.rand(V, device="cuda", generator=g) >= 0.02] = -math.inf
    few[V // 2] = -1000.0
    rows += [half, few, torch.sort(rows[0])[0], torch.sort(rows[1], descending=True)[0]]
    tokens = torch.randint(0, V, (len(rows), 2), device="cuda", generator=g).int()
    used = _check(spp.LogProbs(V, rows, tokens=tokens, top=top)(), rows, tokens, top)
    log(f"vocab {V}, top {top}: {used:.2f} of the bound")


def test_rows_of_more_slices_than_the_merge_has_threads():
    """2^21 and 2^24 tokens: over 1024 slices, and more groups than are held in registers.  The largest logit in a slice
    past the 1024th and far above the rest, in two slices, one value over and over, and behind a mask."""
    import torch
    import paper_2606_29565_amd as spp
    g = torch.Generator(device="cuda").manual_seed(21)
    V = 1 << 21
    x = torch.empty(5, V + 1, device="cuda").normal_(0, 2, generator=g)[:, 1:]
    x[1, V - 1] = 60.0
    x[2] = -7.5
    x[2, [3, V - 2, V // 2]] = torch.tensor([1.0, 2.0, 1.0], device="cuda")
    x[3, :V - 70] = -math.inf
    x[4, 9], x[4, V - 9] = 60.0, 60.0
    tokens = torch.tensor([[V - 1, 0, V]] * 5, dtype=torch.int32, device="cuda")
    _check(spp.LogProbs(V, list(x[1:2]), tokens=tokens[1:2], top=64)(), x[1:2], tokens[1:2], 64)   # short slices
    for top in (0, 64):
        used = _check(spp.LogProbs(V, list(x), tokens=tokens, top=top)(), x, tokens, top)
    log(f"vocab {V}: {used:.2f} of the bound")
    V = 1 << 24
    y = torch.empty(1, V, device="cuda").normal_(100, 2, generator=g)
    y[0, V - 3] = 200.0
    tokens = torch.tensor([[V - 3, 7]], dtype=torch.int32, device="cuda")
    r = spp.LogProbs(V, list(y), tokens=tokens, top=20)()
    (lp, lse, H, tt, tl), off = _want(y[0].cpu().numpy(), tokens[0].tolist(), 20)
    # a term e^d, here d < -80, below 2^-126 may be lost, once on its way, and is less than that: V of them are less than
    # V 2^-126, and times their -d, at most 120 here, so are what H loses
    lost = V * 2.0 ** -126
    assert np.array_equal(r.top_tokens[0].cpu().numpy(), tt)
    for got, want, o in ((r.logprobs, lp, off[0] + lost), (r.lse, lse, off[1] + lost), (r.entropy, H, off[2] + 121 * lost),
                         (r.top_logprobs, tl, off[3] + lost)):
        assert (np.abs(got[0].double().cpu().numpy() - want) <= o).all(), (want, got)
    assert float(H) < 1e-30 and -1e-34 < lp[0] < 0
