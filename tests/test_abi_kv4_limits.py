"""What the paged cache's calls and their workspace queries do past their limits, on
the host: nothing is launched and no pointer is followed."""
import pytest


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import build
    build.build()
    from paper_2405_16406_gb300 import spinq
    return spinq


SHAPE = dict(B=3, prefix_len=100, table_width=2, page_size=64, Hq=128, Hkv=1, D=128)


@pytest.mark.parametrize("kw", [dict(Hq=129), dict(Hq=256), dict(Hq=512, Hkv=2), dict(Hq=1 << 20, Hkv=1 << 19),
                                dict(B=65536), dict(B=1 << 60), dict(prefix_len=1 << 31), dict(prefix_len=(1 << 63) - 1),
                                dict(table_width=1 << 25), dict(table_width=(1 << 63) - 1), dict(page_size=0),
                                dict(page_size=-16), dict(page_size=8), dict(page_size=48), dict(page_size=512),
                                dict(Hq=127, Hkv=2), dict(D=96)])
def test_no_workspace_for_a_prefix_call_that_is_refused(S, kw):
    """A query past the limits answers 0, as for other arguments that the call refuses (Hq / Hkv over 128 divided
    by zero)."""
    query = lambda f: S.spinq_prefix_attention_workspace_bytes(*f.values())   # noqa: E731
    assert query(SHAPE) > 0
    assert query({**SHAPE, **kw}) == 0


@pytest.mark.gpu
def test_too_many_query_heads_for_a_kv_head_are_refused(S):
    import torch
    cache = S.kv4_pages(2, 16, 1, 128)
    one = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(S.SpinqError) as e:
        S.prefix_attention_kv4(torch.zeros((1, 256, 128), dtype=torch.float16, device="cuda"), cache, one[0], 16, one, one[0])
    assert e.value.status == S.SPINQ_EUNSUPPORTED


def test_prompt_attention_wants_no_workspace(S):
    for shape in ((1, 1, 1, 8, 8, 64), (16, 4096, 100000, 32, 8, 128), (1, 0, 0, 0, 0, 0)):
        assert S.spinq_prompt_attention_workspace_bytes(*shape) == 0
