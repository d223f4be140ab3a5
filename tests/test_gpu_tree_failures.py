"""The bounded waits of the tree attention kernel: a launch that issues no copies
gives up, reports the time-out, frees its tensor memory, and the next call is right."""
import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu

DEFAULT_NS = 2_000_000_000


@pytest.mark.parametrize("nodes,D", [(6, 128), (16, 64), (40, 128)])
def test_tree_attention_gives_up_and_recovers(nodes, D):
    from paper_2405_16406_gb300 import spinq
    rng = np.random.default_rng(nodes)
    cache = ku.random_cache(spinq, rng, 40, 64, 2, D)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    q = torch.from_numpy(rng.standard_normal((2 * nodes, 8, D)).astype(np.float16)).cuda()
    table = torch.randperm(40, generator=torch.Generator().manual_seed(0)).to(torch.int32).view(2, 20).cuda()
    call = lambda: spinq.tree_attention_kv4(q, cache, table, i32(1000, 300), i32(0, nodes, 2 * nodes), nodes)   # noqa: E731
    good = call()
    torch.cuda.synchronize()
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
    try:
        assert spinq.spinq_debug_set_wait_limit_ns(1_000_000) == spinq.SPINQ_OK
        assert spinq.spinq_debug_stall_launches(1) == 0
        call()
        torch.cuda.synchronize()
        st, site = spinq.spinq_device_status()
        assert spinq.spinq_debug_stall_launches(0) == 0
    finally:
        spinq.spinq_debug_stall_launches(0)
        assert spinq.spinq_debug_set_wait_limit_ns(DEFAULT_NS) == spinq.SPINQ_OK
    assert st == spinq.SPINQ_ETIMEOUT and site > 0
    again = call()
    torch.cuda.synchronize()
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
    assert torch.equal(good, again)
