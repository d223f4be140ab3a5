"""spinq_prompt_attention with offsets outside the rows: clamped, so that nothing
before or after `out` is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("first,last", [(-7, 30), (-1000, 4000), (0, 31)])
def test_offsets_outside_the_rows_are_clamped(D, first, last):
    from paper_2405_16406_gb300 import spinq as S
    g = torch.Generator(device="cuda").manual_seed(0)
    n, room = 30, 1100   # rows on either side of out, wider than any offset here reaches
    q, k, v = (torch.randn((n, h, D), generator=g, device="cuda").half() for h in (8, 2, 2))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    want = S.prompt_attention(q, k, v, ints(0, n), ints(0, n), n, n)
    wide = torch.full((room + n + room, 8, D), 7.0, dtype=torch.float16, device="cuda")
    S.prompt_attention(q, k, v, ints(first, last), ints(first, last), n, n, out=wide[room:room + n])
    torch.cuda.synchronize()
    assert torch.equal(wide[room:room + n], want)
    assert bool((wide[:room] == 7).all()) and bool((wide[room + n:] == 7).all())
    assert S.spinq_device_status()[0] == S.SPINQ_OK
