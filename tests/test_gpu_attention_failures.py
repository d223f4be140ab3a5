"""The bounded waits of the attention kernels: a launch that issues no copies
gives up, reports the time-out, frees its tensor memory, and the next call is right."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEFAULT_NS = 2_000_000_000


@pytest.mark.parametrize("n,D", [(300, 128), (40, 64)])
def test_prompt_attention_gives_up_and_recovers(n, D):
    from paper_2405_16406_gb300 import spinq
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v = (torch.randn((n, h, D), generator=g, device="cuda").half() for h in (8, 2, 2))
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    good = spinq.prompt_attention(q, k, v, cu, cu, n, n)
    torch.cuda.synchronize()
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
    try:
        assert spinq.spinq_debug_set_wait_limit_ns(1_000_000) == spinq.SPINQ_OK
        assert spinq.spinq_debug_stall_launches(1) == 0
        spinq.prompt_attention(q, k, v, cu, cu, n, n)
        torch.cuda.synchronize()
        st, site = spinq.spinq_device_status()
        assert spinq.spinq_debug_stall_launches(0) == 0
    finally:
        spinq.spinq_debug_stall_launches(0)
        assert spinq.spinq_debug_set_wait_limit_ns(DEFAULT_NS) == spinq.SPINQ_OK
    assert st == spinq.SPINQ_ETIMEOUT and site > 0
    again = spinq.prompt_attention(q, k, v, cu, cu, n, n)
    torch.cuda.synchronize()
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
    assert torch.equal(good, again)


def test_prefix_attention_gives_up_and_recovers():
    import numpy as np

    import kv4_util as ku
    from paper_2405_16406_gb300 import spinq
    rng = np.random.default_rng(0)
    cache = ku.random_cache(spinq, rng, 20, 64, 2, 128)
    q = torch.from_numpy(rng.standard_normal((3, 8, 128)).astype(np.float16)).cuda()
    args = (q, cache, torch.arange(16, dtype=torch.int32, device="cuda"), 1000,
            torch.tensor([[16], [17], [18]], dtype=torch.int32, device="cuda"),
            torch.tensor([5, 0, 64], dtype=torch.int32, device="cuda"))
    good = spinq.prefix_attention_kv4(*args)
    torch.cuda.synchronize()
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
    try:
        assert spinq.spinq_debug_set_wait_limit_ns(1_000_000) == spinq.SPINQ_OK
        assert spinq.spinq_debug_stall_launches(1) == 0
        spinq.prefix_attention_kv4(*args)
        torch.cuda.synchronize()
        st, site = spinq.spinq_device_status()
        assert spinq.spinq_debug_stall_launches(0) == 0
    finally:
        spinq.spinq_debug_stall_launches(0)
        assert spinq.spinq_debug_set_wait_limit_ns(DEFAULT_NS) == spinq.SPINQ_OK
    assert st == spinq.SPINQ_ETIMEOUT and site > 0
    again = spinq.prefix_attention_kv4(*args)
    torch.cuda.synchronize()
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
    assert torch.equal(good, again)
