"""What decode_batch refuses before it calls the library: logits that the step would write past or
into other memory.  (No device: the pool and the model are stand-ins, and -1 is the host's number.)"""
import types

import pytest
import torch

import paper_2606_29565_amd as spp

VOCAB = 64
BAD = {
    "on the host": (torch.empty(VOCAB), 0),
    "without memory": (torch.empty(VOCAB, device="meta"), 0),
    "bf16": (torch.empty(VOCAB, dtype=torch.bfloat16), -1),
    "fp64": (torch.empty(VOCAB, dtype=torch.float64), -1),
    "short": (torch.empty(VOCAB - 1), -1),
    "strided": (torch.empty(2 * VOCAB)[::2], -1),
}


def _decode(dists, device):
    pool = types.SimpleNamespace(handle=None, device=device)
    model = types.SimpleNamespace(handle=None, vocab=VOCAB)
    spp.decode_batch(pool, model, list(range(len(dists))), [1] * len(dists), dists, stream=0)


@pytest.mark.parametrize("what", sorted(BAD))
def test_decode_refuses_logits_it_cannot_write(what):
    dist, device = BAD[what]
    for dists in ([dist], [1 << 20, dist]):
        with pytest.raises(ValueError, match=f"dist {len(dists) - 1} "):
            _decode(dists, device)


@pytest.mark.parametrize("dist", [1 << 20, torch.empty(VOCAB), torch.empty(1, VOCAB + 1)], ids=["pointer", "vocabulary", "longer"])
def test_decode_takes_pointers_and_tensors_that_fit(dist):
    with pytest.raises(spp.SppError) as e:     # (past the checks, there is no pool)
        _decode([dist], -1)
    assert e.value.rc == spp.SPP_E_INVALID_ARG
