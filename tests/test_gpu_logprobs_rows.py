"""Log probabilities of rows whose logits have a common offset or a small spread, against the definition in 64 bits and
with the bounds of test_gpu_logprobs.py.  An offset does not change a row's probabilities, so neither does it change how
its alternatives are found."""
import math

import pytest

from gpu_util import log
from test_gpu_logprobs import _check

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
