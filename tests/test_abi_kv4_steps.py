"""Refusals of the page plan, the kept paths, and windowed and tree attention, on
the host: nothing is launched and no pointer is followed."""
import ctypes

import pytest
import torch

from test_abi_kv4_pages import BAD_PAGES, FAKE, ODD, pages


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import build
    build.build()
    from paper_2405_16406_gb300 import spinq
    return spinq


HALF = ctypes.c_void_p((1 << 20) + 2)
FOUR = ctypes.c_void_p((1 << 20) + 4)


def plan(S, **kw):
    f = dict(lens=FAKE, drop=FAKE, add=FAKE, batch=3, table=FAKE, width=4, page=64, free=FAKE, count=FAKE, capacity=9,
             depths=FAKE, offset=0, total=7, cu=FAKE, positions=FAKE, slots=FAKE, granted=FAKE)
    f.update(kw)
    return S.spinq_kv4_plan(*f.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(lens=None), "SPINQ_EINVAL"), (dict(table=None), "SPINQ_EINVAL"), (dict(free=None), "SPINQ_EINVAL"),
    (dict(count=None), "SPINQ_EINVAL"), (dict(cu=None), "SPINQ_EINVAL"), (dict(positions=None), "SPINQ_EINVAL"),
    (dict(slots=None), "SPINQ_EINVAL"), (dict(batch=-1), "SPINQ_EINVAL"), (dict(width=-1), "SPINQ_EINVAL"),
    (dict(capacity=-1), "SPINQ_EINVAL"), (dict(total=-1), "SPINQ_EINVAL"), (dict(page=0), "SPINQ_EINVAL"),
    (dict(lens=HALF), "SPINQ_EINVAL"), (dict(slots=FOUR), "SPINQ_EINVAL"), (dict(depths=HALF), "SPINQ_EINVAL"),
    (dict(granted=HALF), "SPINQ_EINVAL"),
    (dict(page=48), "SPINQ_EUNSUPPORTED"), (dict(page=512), "SPINQ_EUNSUPPORTED"), (dict(batch=4097), "SPINQ_EUNSUPPORTED"),
    (dict(width=1 << 26), "SPINQ_EUNSUPPORTED"), (dict(total=1 << 31), "SPINQ_EUNSUPPORTED"),
    (dict(capacity=1 << 31), "SPINQ_EUNSUPPORTED"), (dict(offset=1 << 31), "SPINQ_EUNSUPPORTED"),
])
def test_plan_refuses(S, kw, want):
    assert plan(S, **kw) == getattr(S, want)


def keep(S, **kw):
    f = dict(pages={}, table=FAKE, batch=2, width=3, starts=FAKE, path=FAKE, n=4, counts=FAKE)
    f.update(kw)
    return S.spinq_kv4_keep(None if f["pages"] is None else pages(S, **f["pages"]), f["table"], f["batch"], f["width"],
                            f["starts"], f["path"], f["n"], f["counts"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(pages=None), "SPINQ_EINVAL"), (dict(table=None), "SPINQ_EINVAL"), (dict(batch=-1), "SPINQ_EINVAL"),
    (dict(width=-1), "SPINQ_EINVAL"), (dict(starts=None), "SPINQ_EINVAL"), (dict(path=None), "SPINQ_EINVAL"),
    (dict(counts=None), "SPINQ_EINVAL"), (dict(n=-1), "SPINQ_EINVAL"), (dict(batch=1 << 31), "SPINQ_EUNSUPPORTED"),
    (dict(n=1 << 31), "SPINQ_EUNSUPPORTED"),
] + [(dict(pages=p), w) for p, w in BAD_PAGES])
def test_keep_refuses(S, kw, want):
    assert keep(S, **kw) == getattr(S, want)


def prompt(S, **kw):
    f = dict(q=FAKE, ldq=1024, k=FAKE, ldk=256, v=FAKE, ldv=256, cu_q=FAKE, cu_k=FAKE, batch=2, total_q=9, total_k=9,
             max_q=5, max_k=5, Hq=8, Hkv=2, D=128, window=7, sinks=1, scale=0.1, out=ctypes.c_void_p(2 << 20))
    f.update(kw)
    return S.spinq_window_prompt_attention(*f.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(window=0), "SPINQ_EINVAL"), (dict(window=-1), "SPINQ_EINVAL"), (dict(sinks=-1), "SPINQ_EINVAL"),
    (dict(q=None), "SPINQ_EINVAL"), (dict(v=ODD), "SPINQ_EINVAL"), (dict(out=None), "SPINQ_EINVAL"),
    (dict(ldq=1000), "SPINQ_EINVAL"), (dict(batch=0), "SPINQ_EINVAL"), (dict(Hq=9), "SPINQ_EINVAL"),
    (dict(scale=float("nan")), "SPINQ_EINVAL"), (dict(D=96, ldq=1024), "SPINQ_EUNSUPPORTED"),
    (dict(Hq=258, ldq=258 * 128), "SPINQ_EUNSUPPORTED"), (dict(total_k=1 << 40), "SPINQ_EUNSUPPORTED"),
])
def test_window_prompt_refuses(S, kw, want):
    assert prompt(S, **kw) == getattr(S, want)


def tree(S, **kw):
    f = dict(q=FAKE, pages={}, table=FAKE, width=4, lens=FAKE, cu=FAKE, parents=FAKE, B=3, total=20, most=9, Hq=8, window=0,
             sinks=0, scale=0.1, out=ctypes.c_void_p(2 << 20), ws=FAKE, ws_bytes=1 << 40)
    f.update(kw)
    f["pages"] = None if f["pages"] is None else pages(S, **f["pages"])
    return S.spinq_tree_attention_kv4(*f.values(), None)


def decode(S, **kw):
    f = dict(q=FAKE, pages={}, table=FAKE, width=4, lens=FAKE, B=3, Hq=8, window=0, sinks=0, scale=0.1,
             out=ctypes.c_void_p(2 << 20), ws=FAKE, ws_bytes=1 << 40)
    f.update(kw)
    f["pages"] = None if f["pages"] is None else pages(S, **f["pages"])
    return S.spinq_window_attention_kv4(*f.values(), None)


BOTH = [(dict(q=None), "SPINQ_EINVAL"), (dict(pages=None), "SPINQ_EINVAL"), (dict(table=None), "SPINQ_EINVAL"),
        (dict(lens=None), "SPINQ_EINVAL"), (dict(out=None), "SPINQ_EINVAL"), (dict(q=ODD), "SPINQ_EINVAL"),
        (dict(out=ODD), "SPINQ_EINVAL"), (dict(B=-1), "SPINQ_EINVAL"), (dict(width=-1), "SPINQ_EINVAL"),
        (dict(Hq=9), "SPINQ_EINVAL"), (dict(Hq=0), "SPINQ_EINVAL"), (dict(window=-1), "SPINQ_EINVAL"),
        (dict(sinks=-1), "SPINQ_EINVAL"), (dict(scale=float("inf")), "SPINQ_EINVAL"),
        (dict(pages=dict(num_pages=0)), "SPINQ_EINVAL"), (dict(ws=None), "SPINQ_EINVAL"), (dict(ws=ODD), "SPINQ_EINVAL"),
        (dict(ws_bytes=100), "SPINQ_EINVAL"), (dict(Hq=512), "SPINQ_EUNSUPPORTED"), (dict(B=70000), "SPINQ_EUNSUPPORTED"),
        (dict(width=1 << 30), "SPINQ_EUNSUPPORTED")] + [(dict(pages=p), w) for p, w in BAD_PAGES]


@pytest.mark.parametrize("kw,want", BOTH + [
    (dict(cu=None), "SPINQ_EINVAL"), (dict(B=0), "SPINQ_EINVAL"), (dict(most=0), "SPINQ_EINVAL"),
    (dict(total=-1), "SPINQ_EINVAL"), (dict(most=-1), "SPINQ_EINVAL"), (dict(most=129), "SPINQ_EUNSUPPORTED"),
    (dict(total=1 << 31), "SPINQ_EUNSUPPORTED")])
def test_tree_refuses(S, kw, want):
    assert tree(S, **kw) == getattr(S, want)


@pytest.mark.parametrize("kw,want", BOTH)
def test_window_decode_refuses(S, kw, want):
    assert decode(S, **kw) == getattr(S, want)


SHAPE = dict(B=3, max_q=9, table_width=2, page_size=64, Hq=128, Hkv=1, D=128)


@pytest.mark.parametrize("kw", [dict(B=0), dict(B=65536), dict(max_q=0), dict(max_q=129), dict(table_width=-1),
                                dict(table_width=1 << 25), dict(page_size=48), dict(Hq=129), dict(Hq=127, Hkv=2), dict(D=96),
                                dict(B=65535, max_q=128, table_width=1 << 22, Hq=65535, Hkv=65535)])
def test_no_workspace_for_a_call_that_is_refused(S, kw):
    query = lambda f: S.spinq_tree_attention_workspace_bytes(*f.values())   # noqa: E731
    assert query(SHAPE) > 0
    assert query({**SHAPE, **kw}) == 0


def test_nothing_to_do_is_ok(S):
    assert keep(S, batch=0, starts=None, path=None, counts=None, table=None) == S.SPINQ_OK
    assert keep(S, n=0, path=None) == S.SPINQ_OK
    assert prompt(S, total_q=0, q=None, out=None) == S.SPINQ_OK
    assert tree(S, total=0, q=None, out=None, lens=None, cu=None, ws=None, ws_bytes=0) == S.SPINQ_OK
    assert decode(S, B=0, q=None, out=None, lens=None, ws=None, ws_bytes=0) == S.SPINQ_OK


# ------------------------------------------------------------ tensors
def _calls(S, dev):
    """(call, its tensor arguments) for each of the five; the tensors on `dev`."""
    half = lambda *s: torch.zeros(s, dtype=torch.float16, device=dev)   # noqa: E731
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev)    # noqa: E731
    c = S.kv4_pages(2, 16, 1, 64, dev)
    pages = dict(k_codes=c.k_codes, v_codes=c.v_codes, scales=c.scales)
    cache = lambda a: S.KV4Pages(a.pop("k_codes"), a.pop("v_codes"), a.pop("scales").fill_(0))   # noqa: E731
    plan = dict(lens=ints(4, 5), add=ints(1, 1), page_table=ints(0, 1).view(2, 1), free_pages=ints(2, 3, 4), free_count=ints(3),
                drop=ints(0, 0), depths=ints(0, 0))
    keep = dict(pages, page_table=ints(0, 1)[None], starts=ints(3), path=ints(0, 2)[None], counts=ints(2))
    prompt = dict(q=half(3, 2, 64), k=half(3, 1, 64), v=half(3, 1, 64), cu_q=ints(0, 3), cu_k=ints(0, 3), out=half(3, 2, 64))
    space = torch.zeros(64 << 20, dtype=torch.uint8, device=dev)
    tree = dict(pages, q=half(3, 2, 64), page_table=ints(0, 1)[None], lens=ints(20), cu_q=ints(0, 3), parents=ints(-1, 0, 0),
                out=half(3, 2, 64), workspace=space)
    decode = dict(pages, q=half(1, 2, 64), page_table=ints(0, 1)[None], lens=ints(20), out=half(1, 2, 64), workspace=space)
    return {"plan": (lambda a: S.kv4_plan(page_size=16, total=2, **a), plan),
            "keep": (lambda a: S.kv4_keep(cache(a), **a), keep),
            "prompt": (lambda a: S.window_prompt_attention(max_q=3, max_k=3, window=2, **a), prompt),
            "tree": (lambda a: S.tree_attention_kv4(cache=cache(a), max_q=3, **a), tree),
            "decode": (lambda a: S.window_attention_kv4(cache=cache(a), window=5, **a), decode)}


NAMES = ["plan", "keep", "prompt", "tree", "decode"]


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_refused(S, name):
    call, args = _calls(S, "cpu")[name]
    with pytest.raises(ValueError, match="GPU"):
        call(dict(args))


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
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
@pytest.mark.parametrize("name", NAMES)
def test_wrong_types_and_layouts_are_refused(S, name):
    call, args = _calls(S, "cuda")[name]
    for arg, x in args.items():
        if arg in ("workspace", "free_pages"):   # of any type; of any length
            continue
        bad = [x.double()]
        if x.numel() > 1:
            bad.append(torch.stack([x, x], -1)[..., 0])   # every other element
        if arg not in ("page_table", "path"):   # a table without pages and a path without nodes are one
            bad.append(x[..., :0])
        for y in bad:
            with pytest.raises(ValueError):
                call({**args, arg: y})
