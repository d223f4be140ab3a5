"""A key or value that is not a number, through the paged cache: Eq. 1 of its row is
NaN, so the row reads back as NaN and attention over it is NaN, while other rows,
heads and sequences keep their values exactly."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("clip", [1.0, 0.9])
@pytest.mark.parametrize("value", [0, 7, 40, 63])
def test_a_row_with_nan_stays_one(D, clip, value):
    from paper_2405_16406_gb300 import spinq as S
    rng = np.random.default_rng(value)
    T, Hq, Hkv, P = 40, 8, 2, 16
    q, k, v = (torch.from_numpy(rng.standard_normal((T, h, D)).astype(np.float16)).cuda() for h in (Hq, Hkv, Hkv))
    slots, cu = torch.arange(T, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda")
    table = torch.arange(3, dtype=torch.int32, device="cuda")
    own, lens = table[:2, None].contiguous(), torch.tensor([16, 16], dtype=torch.int32, device="cuda")

    def run():
        cache = S.kv4_pages(3, P, Hkv, D)
        S.kv4_append(None, k, v, cache, slots, clip=clip)
        kr, vr = S.kv4_read(cache, table[None], cu, T)
        behind = S.prefix_attention_kv4(q[:2].contiguous(), cache, table[2:], 8, own, lens)
        shared = S.prefix_attention_kv4(q[:2].contiguous(), cache, table, 32, own[:, :0].contiguous(), lens)
        torch.cuda.synchronize()
        return kr, vr, behind, shared
    clean = run()
    k[3, 1, value] = float("nan")    # sequence 0, head 1
    v[20, 0, value] = float("nan")   # sequence 1, head 0
    kr, vr, behind, shared = run()
    rows = torch.zeros((T, Hkv), dtype=torch.bool, device="cuda")
    rows[3, 1] = True
    assert kr[rows].isnan().all() and torch.equal(kr[~rows], clean[0][~rows])
    rows[3, 1], rows[20, 0] = False, True
    assert vr[rows].isnan().all() and torch.equal(vr[~rows], clean[1][~rows])
    bad = torch.zeros((2, Hq), dtype=torch.bool, device="cuda")
    bad[0, 4:] = bad[1, :4] = True
    assert behind[bad].isnan().all() and torch.equal(behind[~bad], clean[2][~bad])
    assert shared.isnan().all() and not clean[3].isnan().any()
