"""Limits of the block-8 calls, at both sides, before anything is enqueued (no GPU is needed)."""

import pytest

from paper_2607_16248_gb300 import build, kvq
from test_block8_refusals import ARG, CAPACITY, _attn


@pytest.fixture(scope="module")
def L():
    build.build()
    return kvq.lib()


def test_softmax_scales(L):
    """A scale whose product with log2 e is no fp32 number is refused."""
    for scale in (0.0, 1e-45, 2.0 ** 127):
        assert _attn(L, scale=scale) == CAPACITY, kvq.last_error()
    for scale in (2.0 ** 127 * (1 + 2.0 ** -23), 3.4e38):
        assert _attn(L, scale=scale) == ARG and "softmax_scale" in kvq.last_error()
