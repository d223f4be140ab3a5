"""The serving example: append, read-back, prompt and prefix attention together.

Bar: attention on the codes against fp64 attention over the read-back fp16 K
and V.  K and V are rounded to fp16 by the read-back (2^-11 each, the scores by
2^-11 of |q| |k| scale), the kernel rounds the weights and the output (2^-11
each): under 2^-8 in norm."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("kw", [dict(requests=5, shared=333, steps=3), dict(requests=40, shared=1000, steps=2, heads=8,
                                                                           kv_heads=8, dim=64, page=16)])
def test_example_decodes_what_the_read_back_cache_says(kw):
    import paged_serving
    from paper_2405_16406_gb300 import spinq
    outs, q, layer, text, tables, length = paged_serving.serve(**kw)
    ref = paged_serving.attention_over_read_back(q, layer, text, kw["shared"], tables, length)
    assert outs.shape[0] == kw["steps"]
    assert float((outs[-1].double() - ref).norm() / ref.norm()) < 2.0 ** -8
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
