"""Workspace sizes of the operators on logits: a workspace for n rows serves fewer of them."""
import pytest

import paper_2606_29565_amd as spp


@pytest.mark.parametrize("vocab", [1, 1000, 1025, 4096, 32000, 128256, 152063, 2 ** 20 + 1, 2 ** 24])
def test_adjust_workspace_does_not_fall_with_the_rows(vocab):
    most = 0
    for n in range(1, 200):
        nbytes = spp.lib().spp_adjust_logits_work_bytes(n, vocab)
        assert nbytes >= most, n
        most = nbytes
        # slices of 1024 tokens at most, one more for a row that starts between 16-byte boundaries
        assert nbytes <= n * ((vocab + 3) // 1024 + 1) * 16
