"""Refusals of the paged cache's entry points, on the host: nothing is launched
and no pointer is followed."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 8)


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import build
    build.build()
    from paper_2405_16406_gb300 import spinq
    return spinq


def pages(S, **kw):
    f = dict(k_codes=1 << 20, v_codes=1 << 20, scales=1 << 20, num_pages=4, page_size=64, kv_heads=2, head_dim=128)
    f.update(kw)
    return ctypes.byref(S.Kv4PagesCfg(**f))


BAD_PAGES = [(dict(k_codes=None), "SPINQ_EINVAL"), (dict(v_codes=None), "SPINQ_EINVAL"), (dict(scales=None), "SPINQ_EINVAL"),
             (dict(scales=(1 << 20) + 4), "SPINQ_EINVAL"), (dict(k_codes=(1 << 20) + 8), "SPINQ_EINVAL"),
             (dict(num_pages=-1), "SPINQ_EINVAL"), (dict(kv_heads=0), "SPINQ_EINVAL"), (dict(page_size=0), "SPINQ_EINVAL"),
             (dict(page_size=48), "SPINQ_EUNSUPPORTED"), (dict(page_size=8), "SPINQ_EUNSUPPORTED"),
             (dict(page_size=512), "SPINQ_EUNSUPPORTED"), (dict(head_dim=96), "SPINQ_EUNSUPPORTED"),
             (dict(head_dim=256), "SPINQ_EUNSUPPORTED")]


def append(S, **kw):
    f = dict(q=FAKE, ldq=1024, q_out=ctypes.c_void_p(2 << 20), k=FAKE, ldk=256, v=FAKE, ldv=256, T=3, Hq=8, qw=FAKE,
             kw=FAKE, eps=1e-6, rope=dict(rotary_dim=128, interleaved=0, positions=1 << 20, cos_sin=1 << 20, max_pos=9),
             bits=4, sym=False, group=128, clip=1.0, pages={}, slots=FAKE)
    f.update(kw)
    rope = None if f["rope"] is None else ctypes.byref(S.RopeCfg(**f["rope"]))
    kvq = S.quant_cfg(f["bits"], f["sym"], S.SPINQ_PER_GROUP, f["group"], f["clip"])
    return S.spinq_kv4_append(f["q"], f["ldq"], f["q_out"], f["k"], f["ldk"], f["v"], f["ldv"], f["T"], f["Hq"], f["qw"],
                              f["kw"], f["eps"], rope, ctypes.byref(kvq),
                              None if f["pages"] is None else pages(S, **f["pages"]), f["slots"], None)


def rope(**kw):
    f = dict(rotary_dim=128, interleaved=0, positions=1 << 20, cos_sin=1 << 20, max_pos=9)
    f.update(kw)
    return dict(rope=f)


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), "SPINQ_EINVAL"), (dict(Hq=-1), "SPINQ_EINVAL"), (dict(q=None), "SPINQ_EINVAL"),
    (dict(q_out=None), "SPINQ_EINVAL"), (dict(k=None), "SPINQ_EINVAL"), (dict(v=None), "SPINQ_EINVAL"),
    (dict(slots=None), "SPINQ_EINVAL"), (dict(q=ODD), "SPINQ_EINVAL"), (dict(k=ODD), "SPINQ_EINVAL"),
    (dict(qw=ODD), "SPINQ_EINVAL"), (dict(ldq=1016), "SPINQ_EINVAL"), (dict(ldk=260), "SPINQ_EINVAL"),
    (dict(ldv=248), "SPINQ_EINVAL"), (dict(eps=-1.0), "SPINQ_EINVAL"), (dict(eps=float("nan")), "SPINQ_EINVAL"),
    (dict(clip=0.0), "SPINQ_EINVAL"), (dict(clip=1.5), "SPINQ_EINVAL"), (dict(pages=None), "SPINQ_EINVAL"),
    (dict(q_out=FAKE, ldq=2048), "SPINQ_EINVAL"),
    (rope(rotary_dim=-2), "SPINQ_EINVAL"), (rope(rotary_dim=160), "SPINQ_EINVAL"), (rope(interleaved=2), "SPINQ_EINVAL"),
    (rope(positions=None), "SPINQ_EINVAL"), (rope(cos_sin=None), "SPINQ_EINVAL"), (rope(max_pos=0), "SPINQ_EINVAL"),
    (rope(cos_sin=(1 << 20) + 8), "SPINQ_EINVAL"), (rope(rotary_dim=16), "SPINQ_EUNSUPPORTED"),
    (dict(bits=8), "SPINQ_EUNSUPPORTED"), (dict(sym=True), "SPINQ_EUNSUPPORTED"), (dict(group=64), "SPINQ_EUNSUPPORTED"),
    (dict(T=1 << 33), "SPINQ_EUNSUPPORTED"),
] + [(dict(pages=p), w) for p, w in BAD_PAGES])
def test_append_refuses(S, kw, want):
    assert append(S, **kw) == getattr(S, want)


def read(S, **kw):
    f = dict(pages={}, table=FAKE, batch=2, width=3, starts=None, cu=FAKE, total=10, k=FAKE, v=FAKE)
    f.update(kw)
    return S.spinq_kv4_read(None if f["pages"] is None else pages(S, **f["pages"]), f["table"], f["batch"], f["width"],
                            f["starts"], f["cu"], f["total"], f["k"], f["v"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(pages=None), "SPINQ_EINVAL"), (dict(table=None), "SPINQ_EINVAL"), (dict(batch=-1), "SPINQ_EINVAL"),
    (dict(batch=0), "SPINQ_EINVAL"), (dict(width=-1), "SPINQ_EINVAL"), (dict(cu=None), "SPINQ_EINVAL"),
    (dict(total=-1), "SPINQ_EINVAL"), (dict(k=None), "SPINQ_EINVAL"), (dict(v=ODD), "SPINQ_EINVAL"),
    (dict(total=1 << 40), "SPINQ_EUNSUPPORTED"),
] + [(dict(pages=p), w) for p, w in BAD_PAGES])
def test_read_refuses(S, kw, want):
    assert read(S, **kw) == getattr(S, want)


def prompt(S, **kw):
    f = dict(q=FAKE, ldq=1024, k=FAKE, ldk=256, v=FAKE, ldv=256, cu_q=FAKE, cu_k=FAKE, batch=2, total_q=9, total_k=9,
             max_q=5, max_k=5, Hq=8, Hkv=2, D=128, causal=1, scale=0.1, out=ctypes.c_void_p(2 << 20), ws=FAKE,
             ws_bytes=1 << 40)
    f.update(kw)
    return S.spinq_prompt_attention(*[f[n] for n in ("q", "ldq", "k", "ldk", "v", "ldv", "cu_q", "cu_k", "batch", "total_q",
                                                     "total_k", "max_q", "max_k", "Hq", "Hkv", "D", "causal", "scale",
                                                     "out", "ws", "ws_bytes")], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), "SPINQ_EINVAL"), (dict(k=None), "SPINQ_EINVAL"), (dict(v=None), "SPINQ_EINVAL"),
    (dict(out=None), "SPINQ_EINVAL"), (dict(cu_q=None), "SPINQ_EINVAL"), (dict(cu_k=None), "SPINQ_EINVAL"),
    (dict(q=ODD), "SPINQ_EINVAL"), (dict(v=ODD), "SPINQ_EINVAL"), (dict(out=ODD), "SPINQ_EINVAL"),
    (dict(ldq=1000), "SPINQ_EINVAL"), (dict(ldk=257), "SPINQ_EINVAL"), (dict(batch=-1), "SPINQ_EINVAL"),
    (dict(batch=0), "SPINQ_EINVAL"), (dict(max_q=0), "SPINQ_EINVAL"), (dict(total_q=-1), "SPINQ_EINVAL"),
    (dict(Hq=9), "SPINQ_EINVAL"), (dict(Hkv=0), "SPINQ_EINVAL"), (dict(causal=2), "SPINQ_EINVAL"),
    (dict(scale=float("inf")), "SPINQ_EINVAL"), (dict(scale=float("nan")), "SPINQ_EINVAL"),
    (dict(D=96, ldq=1024), "SPINQ_EUNSUPPORTED"), (dict(Hq=258, ldq=258 * 128), "SPINQ_EUNSUPPORTED"),
    (dict(total_k=1 << 40), "SPINQ_EUNSUPPORTED"), (dict(batch=70000), "SPINQ_EUNSUPPORTED"),
])
def test_prompt_refuses(S, kw, want):
    assert prompt(S, **kw) == getattr(S, want)


def prefix(S, **kw):
    f = dict(q=FAKE, pages={}, ptab=FAKE, prefix=100, table=FAKE, width=2, lens=FAKE, B=3, Hq=8, scale=0.1,
             out=ctypes.c_void_p(2 << 20), ws=FAKE, ws_bytes=1 << 40)
    f.update(kw)
    return S.spinq_prefix_attention_kv4(f["q"], None if f["pages"] is None else pages(S, **f["pages"]), f["ptab"],
                                        f["prefix"], f["table"], f["width"], f["lens"], f["B"], f["Hq"], f["scale"],
                                        f["out"], f["ws"], f["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), "SPINQ_EINVAL"), (dict(pages=None), "SPINQ_EINVAL"), (dict(ptab=None), "SPINQ_EINVAL"),
    (dict(table=None), "SPINQ_EINVAL"), (dict(lens=None), "SPINQ_EINVAL"), (dict(out=None), "SPINQ_EINVAL"),
    (dict(q=ODD), "SPINQ_EINVAL"), (dict(out=ODD), "SPINQ_EINVAL"), (dict(B=-1), "SPINQ_EINVAL"),
    (dict(prefix=-1), "SPINQ_EINVAL"), (dict(width=-1), "SPINQ_EINVAL"), (dict(Hq=9), "SPINQ_EINVAL"),
    (dict(Hq=0), "SPINQ_EINVAL"), (dict(scale=float("nan")), "SPINQ_EINVAL"), (dict(pages=dict(num_pages=0)), "SPINQ_EINVAL"),
    (dict(Hq=512), "SPINQ_EUNSUPPORTED"), (dict(B=70000), "SPINQ_EUNSUPPORTED"), (dict(prefix=1 << 40), "SPINQ_EUNSUPPORTED"),
    (dict(width=1 << 30), "SPINQ_EUNSUPPORTED"),
] + [(dict(pages=p), w) for p, w in BAD_PAGES])
def test_prefix_refuses(S, kw, want):
    assert prefix(S, **kw) == getattr(S, want)


def test_workspaces_that_are_missing_or_small_are_refused(S):
    need = S.spinq_prefix_attention_workspace_bytes(3, 100, 2, 64, 8, 2, 128)
    for ws, n in ((None, need), (FAKE, need - 1), (ODD, need)):
        if need:
            assert prefix(S, ws=ws, ws_bytes=n) == S.SPINQ_EINVAL
    need = S.spinq_prompt_attention_workspace_bytes(1, 5, 100000, 8, 2, 128)
    for ws, n in ((None, need), (FAKE, need - 1), (ODD, need)):
        if need:
            assert prompt(S, batch=1, max_k=100000, ws=ws, ws_bytes=n) == S.SPINQ_EINVAL


def test_nothing_to_do_is_ok(S):
    assert append(S, T=0, q=None, q_out=None, k=None, v=None, slots=None) == S.SPINQ_OK
    assert read(S, total=0, k=None, v=None, cu=None, batch=0) == S.SPINQ_OK
    assert prompt(S, total_q=0, q=None, out=None) == S.SPINQ_OK
    assert prefix(S, B=0, q=None, out=None, lens=None) == S.SPINQ_OK
