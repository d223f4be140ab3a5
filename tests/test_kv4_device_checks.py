"""The paged cache's tensor calls take no host tensor for a GPU address: refused before
anything is launched."""
import pytest
import torch


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import build
    build.build()
    from paper_2405_16406_gb300 import spinq
    return spinq


def _calls(S, dev):
    """(call, its tensor arguments) for each of the four; the tensors on `dev`."""
    half = lambda *s: torch.zeros(s, dtype=torch.float16, device=dev)   # noqa: E731
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev)    # noqa: E731
    pages = dict(zip(("k_codes", "v_codes", "scales"), (lambda c: (c.k_codes, c.v_codes, c.scales))(S.kv4_pages(2, 16, 1, 64, dev))))
    cache = lambda a: S.KV4Pages(a.pop("k_codes"), a.pop("v_codes"), a.pop("scales").fill_(0))   # noqa: E731
    append = dict(pages, q=half(3, 2, 64), k=half(3, 1, 64), v=half(3, 1, 64), slots=torch.arange(3, device=dev),
                  positions=ints(0, 1, 2), cos_sin=torch.zeros((4, 32, 2), device=dev), q_weight=half(64), k_weight=half(64),
                  q_out=half(3, 2, 64))
    read = dict(pages, page_table=ints(0, 1)[None], cu_tokens=ints(0, 5), starts=ints(1), k=half(5, 1, 64), v=half(5, 1, 64))
    prompt = dict(q=half(3, 2, 64), k=half(3, 1, 64), v=half(3, 1, 64), cu_q=ints(0, 3), cu_k=ints(0, 3), out=half(3, 2, 64),
                  workspace=torch.zeros(16, dtype=torch.uint8, device=dev))
    prefix = dict(pages, q=half(1, 2, 64), prefix_table=ints(0), page_table=ints(1)[None], lens=ints(4), out=half(1, 2, 64),
                  workspace=torch.zeros(1 << 20, dtype=torch.uint8, device=dev))
    return {"append": (lambda a: S.kv4_append(cache=cache(a), **a), append),
            "read": (lambda a: S.kv4_read(cache(a), total=5, **a), read),
            "prompt": (lambda a: S.prompt_attention(max_q=3, max_k=3, **a), prompt),
            "prefix": (lambda a: S.prefix_attention_kv4(cache=cache(a), prefix_len=16, **a), prefix)}


@pytest.mark.parametrize("name", ["append", "read", "prompt", "prefix"])
def test_host_tensors_are_refused(S, name):
    call, args = _calls(S, "cpu")[name]
    with pytest.raises(ValueError, match="GPU"):
        call(dict(args))


def test_host_addresses_are_not_taken(S):
    with pytest.raises(ValueError):
        S._full(torch.zeros(3, dtype=torch.int32), torch.int32, (3,), 0)
    with pytest.raises(ValueError):
        S._token_rows(torch.zeros((3, 2, 64), dtype=torch.float16), 0)
    with pytest.raises(ValueError):
        S._space(torch.zeros(3), 0)
    with pytest.raises(ValueError):
        S._pages(S.kv4_pages(1, 16, 1, 64, "cpu"), 0)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["append", "read", "prompt", "prefix"])
def test_one_host_tensor_among_the_arguments_is_refused(S, name):
    call, args = _calls(S, "cuda")[name]
    call(dict(args))
    torch.cuda.synchronize()
    for arg, x in args.items():
        with pytest.raises(ValueError):
            call({**args, arg: x.cpu()})
    torch.cuda.synchronize()
    assert S.spinq_device_status()[0] == S.SPINQ_OK


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["append", "read", "prompt", "prefix"])
def test_wrong_types_and_layouts_are_refused(S, name):
    call, args = _calls(S, "cuda")[name]
    for arg, x in args.items():
        if arg == "workspace":
            continue
        bad = [x.double()]
        if x.numel() > 1:
            bad.append(torch.stack([x, x], -1)[..., 0])   # every other element
        if arg != "page_table":   # a table without pages is one
            bad.append(x[..., :0])
        for y in bad:
            with pytest.raises(ValueError):
                call({**args, arg: y})
