"""The bound of attention_parts.py on the CPU: what the kernel's roundings give is inside it, and each of the mistakes that
it is there to see -- a bf16 part of the query or of the probabilities gone missing, probabilities cut off -- is
outside, with bf16 and fp32 outputs."""
import numpy as np
import pytest

from attention_parts import MISTAKES, aligned_case, emulate, row


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("io_bf16", [False, True])
@pytest.mark.parametrize("n", [17, 40, 64])
def test_the_bound_tells_parts_from_their_absence(code, dh, io_bf16, n):
    q, K, ks, V, vs, scale = aligned_case(code, dh, io_bf16, n, seed=n)
    want, off = row(q, K * ks, V * vs, scale, io_bf16)
    share = lambda plant: float((np.abs(emulate(q, K * ks, V * vs, scale, io_bf16, plant) - want) / off).max())  # noqa: E731
    assert share(None) <= 1
    for plant in MISTAKES[io_bf16]:
        assert share(plant) > 2, (plant, share(plant))
