"""CPU tests: what an attention description may say, which needs no GPU to be refused."""
import pytest

import paper_2002_05645_amd as P


@pytest.mark.parametrize("scale,held", [(2.0 ** -64, True), (0.125, True), (1.0, True), (1024.0, True), (1024.001, False), (2.0 ** 30, False), (2.0 ** 64, False), (2.0 ** -65, False)])
def test_attention_scales_beyond_what_the_gradients_hold_are_refused(scale, held):
    # the backward pass takes e^(score - lse) from an lse in fp32: no input's score times 2^30 leaves it a digit
    a = P.make_attention(dtype="bf16", heads=4, kv_heads=2, head_dim=64, sequences=3, max_len=100, scale=scale)
    assert (P.attention_work_bytes(a) > 0) == held
