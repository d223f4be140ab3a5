"""Operators of the paged 4-bit cache: the cases they are measured on, and
their plain form.

* ``write``: norms of queries and keys for each head, the position rotation,
  the online Hadamard R3 and the 4-bit quantizer in one pass, K and V written
  into the pages of the cache (``spinq.kv4_append``); the written tokens are
  read back (``spinq.kv4_read``), as a prompt that arrives in chunks does.
* ``read``: cached tokens of a batch of sequences expanded to packed fp16 K
  and V (``spinq.kv4_read``).
* ``prompt``: attention over whole prompts, packed sequences of different
  lengths with grouped heads, causal, also where each prompt continues a
  cached context (``spinq.prompt_attention``).
* ``prefix``: one query per sequence and head over a prefix that the whole
  batch shares and the sequence's own tokens, straight on the 4-bit pages
  (``spinq.prefix_attention_kv4``).

``own`` false computes them in elementary torch operations in 32 bits, rounded
once at the end; ``own`` true calls the library.  Lengths of a case come from
its own numbers (``lens_seed``), everything else from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
MAX_POS = 32768


# ------------------------------------------------------------------ the cases
def listed():
    heads = {"heads": 32, "kv_heads": 8, "head_dim": 128}
    return [
        # one decode step of eight sequences: a token each, the call's latency counts
        {"name": "write one token x 8", "op": "write", "batch": 8, "shortest": 1, "longest": 1, "lens_seed": 0,
         "context": 4096, **heads, "rotary": 128, "interleaved": False, "norm": True, "page": 64},
        # a chunk of packed prompts of ragged length, part of the head rotated, neighbouring pairs
        {"name": "write ragged chunk", "op": "write", "batch": 7, "shortest": 1, "longest": 611, "lens_seed": 3,
         "context": 1000, "heads": 24, "kv_heads": 8, "head_dim": 128, "rotary": 64, "interleaved": True,
         "norm": True, "page": 16},
        # the prompts of the 8 x 4096 cache workload, no head norms
        {"name": "write 8 x 4096", "op": "write", "batch": 8, "shortest": 4096, "longest": 4096, "lens_seed": 0,
         "context": 0, **heads, "rotary": 128, "interleaved": False, "norm": False, "page": 64},
        # one short sequence with small heads read back before its next chunk
        {"name": "read 777 tokens", "op": "read", "batch": 1, "shortest": 777, "longest": 777, "lens_seed": 0,
         "kv_heads": 8, "head_dim": 64, "page": 32},
        # the contexts of a batch of long sequences
        {"name": "read long contexts", "op": "read", "batch": 8, "shortest": 4001, "longest": 30011, "lens_seed": 1,
         "kv_heads": 8, "head_dim": 128, "page": 64},
        # a few short prompts with small heads
        {"name": "prompt few short", "op": "prompt", "batch": 3, "shortest": 1, "longest": 61, "lens_seed": 2,
         "context": 0, "heads": 8, "kv_heads": 2, "head_dim": 64},
        # packed prompts of many lengths
        {"name": "prompt packed ragged", "op": "prompt", "batch": 16, "shortest": 1, "longest": 1537, "lens_seed": 4,
         "context": 0, **heads},
        # a chunk of two prompts over their cached contexts
        {"name": "prompt chunk over 16384", "op": "prompt", "batch": 2, "shortest": 389, "longest": 512,
         "lens_seed": 5, "context": 16384, **heads},
        # whole prompts of the length of the cache workload
        {"name": "prompt 4 x 4096", "op": "prompt", "batch": 4, "shortest": 4096, "longest": 4096, "lens_seed": 0,
         "context": 0, **heads},
        # a few sequences that share an instruction text
        {"name": "prefix 1000 x 4", "op": "prefix", "batch": 4, "prefix": 1000, "shortest": 1, "longest": 77,
         "lens_seed": 6, **heads, "page": 16},
        # a serving batch behind one long document
        {"name": "prefix 8191 x 64", "op": "prefix", "batch": 64, "prefix": 8191, "shortest": 0, "longest": 517,
         "lens_seed": 7, **heads, "page": 64},
        # the largest batch and document, many answers in parallel
        {"name": "prefix 32768 x 256", "op": "prefix", "batch": 256, "prefix": 32768, "shortest": 64,
         "longest": 1024, "lens_seed": 8, **heads, "page": 64},
    ]


def _spread(rng, low, high):
    """A whole number from low to high, spread over the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(("write", "read", "prompt", "prefix"))
    heads, kv_heads, dim = rng.choice(((32, 8, 128), (24, 8, 128), (8, 8, 64), (16, 2, 64), (20, 4, 128),
                                       (32, 8, 64), (8, 1, 128)))
    page = rng.choice((16, 32, 64, 128, 256))
    case = {"op": op, "kv_heads": kv_heads, "head_dim": dim, "lens_seed": rng.randrange(1 << 20)}
    if op in ("write", "read"):
        batch = _spread(rng, 1, 8)
        longest = _spread(rng, 1, (4096 if op == "write" else 20000))
        case.update(batch=batch, longest=longest, shortest=_spread(rng, 1, longest), page=page)
        if op == "write":
            case.update(heads=heads, context=rng.choice((0, _spread(rng, 1, 8000))),
                        rotary=rng.choice((dim, dim, dim // 2, dim // 4)), interleaved=rng.random() < 0.5,
                        norm=rng.random() < 0.5)
    elif op == "prompt":
        longest = _spread(rng, 1, 4096)
        context = rng.choice((0, 0, _spread(rng, 1, 4096)))
        # no more pairs of a query and a key than four prompts of 4096 have
        most = max(1, min(16, int(4 * 4096 * 2048 * 32 / (longest * (longest / 2 + context) * heads))))
        case.update(batch=_spread(rng, 1, most), longest=longest, shortest=_spread(rng, 1, longest),
                    context=context, heads=heads)
    else:
        longest = _spread(rng, 1, 1024)
        case.update(batch=_spread(rng, 1, 200), prefix=rng.choice((0, _spread(rng, 1, 24000), _spread(rng, 64, 24000))),
                    longest=longest, shortest=rng.choice((0, _spread(rng, 1, longest))), heads=heads, page=page)
    return case


def _lengths(case):
    r = random.Random(case["lens_seed"])
    return [r.randint(case["shortest"], case["longest"]) for _ in range(case["batch"])]


# ----------------------------------------------------------------- the inputs
def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _pages_of(gen, lens, page):
    """Page tables of sequences of the given lengths, pages in random order, and the number of pages."""
    need = [(n + page - 1) // page for n in lens]
    total = max(1, sum(need))
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((len(lens), max(1, max(need))), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def _random_pages(gen, pages, case):
    """Pages as the quantizer leaves them: codes spread like a normal row's, scales of rows of unit variance."""
    shape = (pages, case["kv_heads"], case["page"], case["head_dim"] // 2)

    def codes():
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        for at in range(0, pages, 512):   # a part at a time: the normal draws are 16 times the codes
            part = (min(512, pages - at),) + shape[1:]
            low = (torch.randn(part, generator=gen, device="cuda") * 2.7 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            high = (torch.randn(part, generator=gen, device="cuda") * 2.7 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            out[at:at + 512] = low | (high << 4)
        return out

    scales = torch.empty((pages, case["kv_heads"], case["page"], 4), device="cuda")
    for at in (0, 2):
        step = 0.36 * (1 + 0.1 * torch.randn(shape[:3], generator=gen, device="cuda")).clamp_(0.5, 2)
        scales[..., at] = step
        scales[..., at + 1] = -7.5 * step + 0.1 * torch.randn(shape[:3], generator=gen, device="cuda")
    return codes(), codes(), scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).half()

    lens = _lengths(case)
    dim, hk, hq = case["head_dim"], case["kv_heads"], case.get("heads")
    s = dict(case)
    if case["op"] == "write":
        total = sum(lens)
        s["table"], pages = _pages_of(gen, [case["context"] + n for n in lens], case["page"])
        s["fused"] = normal(total, (hq + 2 * hk) * dim)   # the output of one q, k, v projection
        s["starts"] = _ints([case["context"]] * case["batch"])
        s["cu"] = _ints(_offsets(lens))
        s["total"] = total
        row = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), _ints(lens, torch.int64))
        s["positions"] = (torch.arange(total, device="cuda") - s["cu"].long()[row] + case["context"]).int()
        p = s["positions"].long()
        s["slots"] = s["table"].long()[row, p // case["page"]] * case["page"] + p % case["page"]
        half = case["rotary"] // 2
        theta = 500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        angle = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * theta
        s["cos_sin"] = torch.stack((angle.cos(), angle.sin()), -1).float()
        s["q_weight"] = (1 + 0.1 * normal(dim).float()).half() if case["norm"] else None
        s["k_weight"] = (1 + 0.1 * normal(dim).float()).half() if case["norm"] else None
        s["k_codes"] = torch.zeros((pages, hk, case["page"], dim // 2), dtype=torch.uint8, device="cuda")
        s["v_codes"] = torch.zeros_like(s["k_codes"])
        s["scales"] = torch.zeros((pages, hk, case["page"], 4), device="cuda")
    elif case["op"] == "read":
        s["table"], pages = _pages_of(gen, lens, case["page"])
        s["k_codes"], s["v_codes"], s["scales"] = _random_pages(gen, pages, case)
        s["cu"] = _ints(_offsets(lens))
        s["total"] = sum(lens)
    elif case["op"] == "prompt":
        total = sum(lens)
        keys = [n + case["context"] for n in lens]
        fused = normal(total, (hq + 2 * hk) * dim)   # strided rows, as the projection leaves them
        s["q"] = fused[:, :hq * dim].view(total, hq, dim)
        s["q"].mul_(2)
        if case["context"]:
            s["k"], s["v"] = normal(sum(keys), hk, dim), normal(sum(keys), hk, dim)
        else:
            s["k"] = fused[:, hq * dim:(hq + hk) * dim].view(total, hk, dim)
            s["v"] = fused[:, (hq + hk) * dim:].view(total, hk, dim)
        s["cu_q"], s["cu_k"] = _ints(_offsets(lens)), _ints(_offsets(keys))
        s["max_q"], s["max_k"] = max(lens), max(keys)
    else:
        prefix = case["prefix"]
        table, pages = _pages_of(gen, [prefix] + lens, case["page"])
        used = (prefix + case["page"] - 1) // case["page"]
        wide = max(1, (max(lens) + case["page"] - 1) // case["page"])
        s["prefix_table"] = table[0, :max(1, used)].contiguous()
        s["table"] = table[1:, :wide].contiguous()
        s["k_codes"], s["v_codes"], s["scales"] = _random_pages(gen, pages, case)
        s["lens"] = _ints(lens)
        s["most"] = max(lens)
        s["q"] = normal(case["batch"], hq, dim, scale=2.0)
    return s


# ------------------------------------------------------------- the plain form
def _tree_sum(x):
    """Sums of the last dimension (a power of two), neighbours first."""
    return x[..., 0] if x.shape[-1] == 1 else _tree_sum(x[..., 0::2] + x[..., 1::2])


def _hadamard(x, bit=1):
    """The Sylvester-Hadamard transform of the last dimension, unnormalised."""
    if bit == x.shape[-1]:
        return x
    y = x.unflatten(-1, (-1, 2, bit))
    a, b = y[..., 0, :], y[..., 1, :]
    return _hadamard(torch.stack((a + b, a - b), -2).flatten(-3), 2 * bit)


def _rotated(x, weight, s):
    """Norm of each head, position rotation and Hadamard (unnormalised) of x [T, H, D] in 32 bits."""
    x = x.float()
    if weight is not None:
        x = (x * (1 / torch.sqrt(_tree_sum(x * x) / x.shape[-1] + EPS))[..., None]) * weight.float()
    part, rest = x[..., :s["rotary"]], x[..., s["rotary"]:]
    cs = s["cos_sin"][s["positions"].long()][:, None]
    cos, sin = cs[..., 0], cs[..., 1]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = part.chunk(2, -1)
        part = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return _hadamard(torch.cat((part, rest), -1))


def _quantized(y, norm):
    """The values that the 4-bit codes of rows y stand for."""
    low, high = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    span = high - low
    inv = torch.where(span > 0, 15.0 / span, torch.zeros_like(span))
    code = torch.round((y - low) * inv).clamp(0, 15)
    return (code * (span / 15.0 * norm) + low * norm).half()


def _expanded(s, table, token, which):
    """Values [..., Hkv, D] of the tokens at positions `token` of the page tables `table` (same leading shape)."""
    page, slot = token // s["page"], token % s["page"]
    at = table.long().gather(-1, page) if table.dim() == page.dim() else table.long()[page]
    packed = s["k_codes" if which == 0 else "v_codes"][at, :, slot]
    scale = s["scales"][at, :, slot]
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2).float()
    return code * scale[..., 2 * which, None] + scale[..., 2 * which + 1, None]


def _softmax_parts(scores):
    """exp(scores - row maximum) and the row sums; a row without a visible key gives zeros."""
    top = scores.amax(-1, keepdim=True)
    weight = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    return weight, weight.sum(-1, keepdim=True)


def _plain_write(s):
    dim, hq, hk = s["head_dim"], s["heads"], s["kv_heads"]
    q, k, v = (x.unflatten(-1, (-1, dim)) for x in s["fused"].split((hq * dim, hk * dim, hk * dim), -1))
    norm = 1 / math.sqrt(dim)
    return {"q": (_rotated(q, s["q_weight"], s) * norm).half(), "k": _quantized(_rotated(k, s["k_weight"], s), norm),
            "v": _quantized(v.float(), 1.0)}


def _plain_read(s):
    at = torch.arange(s["total"], device="cuda")
    row = torch.bucketize(at, s["cu"][1:].long(), right=True)
    token = (at - s["cu"].long()[row])[:, None]
    table = s["table"][row]
    return {"k": _expanded(s, table, token, 0)[:, 0].half(), "v": _expanded(s, table, token, 1)[:, 0].half()}


def _plain_prompt(s):
    hk, dim = s["kv_heads"], s["head_dim"]
    group = s["heads"] // hk
    cu_q, cu_k = s["cu_q"].long(), s["cu_k"].long()
    nq, nk = (cu_q[1:] - cu_q[:-1])[:, None], (cu_k[1:] - cu_k[:-1])[:, None]
    i, j = torch.arange(s["max_q"], device="cuda"), torch.arange(s["max_k"], device="cuda")
    at_q = (cu_q[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    at_k = (cu_k[:-1, None] + j).clamp(max=s["k"].shape[0] - 1)
    q = s["q"][at_q].float().unflatten(2, (hk, group)).permute(0, 2, 3, 1, 4)          # B, hk, group, max_q, dim
    k = s["k"][at_k].float().permute(0, 2, 3, 1)[:, :, None]                             # B, hk, 1, dim, max_k
    v = s["v"][at_k].float().permute(0, 2, 1, 3)[:, :, None]
    seen = (j[None, None] <= i[None, :, None] + (nk - nq)[:, :, None]) & (j[None, None] < nk[:, :, None])
    scores = torch.matmul(q, k) * (1 / math.sqrt(dim))
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    weight, total = _softmax_parts(scores)
    out = torch.where(total > 0, torch.matmul(weight, v) / total, torch.zeros_like(total))
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)                                        # B, max_q, heads, dim
    return {"out": out[i[None] < nq].half()}


def _plain_prefix(s):
    hk, dim, batch = s["kv_heads"], s["head_dim"], s["batch"]
    group = s["heads"] // hk
    q = s["q"].float().view(batch, hk, group, dim) * (1 / math.sqrt(dim))
    first = torch.arange(s["prefix"], device="cuda")
    k, v = (_expanded(s, s["prefix_table"], first, w).permute(1, 0, 2) for w in (0, 1))     # hk, prefix, dim
    shared = torch.matmul(q.permute(1, 0, 2, 3).flatten(1, 2), k.transpose(1, 2))
    shared = shared.unflatten(1, (batch, group)).permute(1, 0, 2, 3)                        # batch, hk, group, prefix
    last = torch.arange(s["most"], device="cuda")[None].expand(batch, -1)
    ks, vs = (_expanded(s, s["table"], last, w).permute(0, 2, 1, 3) for w in (0, 1))        # batch, hk, most, dim
    mine = torch.matmul(q, ks.transpose(2, 3)).masked_fill_((last >= s["lens"][:, None])[:, None, None], -math.inf)
    scores = torch.cat((shared, mine, torch.full_like(q[..., :1], -math.inf)), -1)
    weight, total = _softmax_parts(scores)
    front = weight[..., :s["prefix"]].permute(1, 0, 2, 3).flatten(1, 2)
    out = torch.matmul(front, v).unflatten(1, (batch, group)).permute(1, 0, 2, 3)
    out = out + torch.matmul(weight[..., s["prefix"]:-1], vs)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return {"out": out.flatten(1, 2).half()}


# -------------------------------------------------------- the framework's own
def _own_write(s, spinq):
    dim, hq, hk = s["head_dim"], s["heads"], s["kv_heads"]
    q, k, v = (x.unflatten(-1, (-1, dim)) for x in s["fused"].split((hq * dim, hk * dim, hk * dim), -1))
    cache = spinq.KV4Pages(s["k_codes"], s["v_codes"], s["scales"])
    q_out = spinq.kv4_append(q, k, v, cache, s["slots"], s["positions"], s["cos_sin"], q_weight=s["q_weight"],
                             k_weight=s["k_weight"], eps=EPS, interleaved=s["interleaved"])
    k_out, v_out = spinq.kv4_read(cache, s["table"], s["cu"], s["total"], starts=s["starts"])
    return {"q": q_out, "k": k_out, "v": v_out}


def _own_read(s, spinq):
    cache = spinq.KV4Pages(s["k_codes"], s["v_codes"], s["scales"])
    k, v = spinq.kv4_read(cache, s["table"], s["cu"], s["total"])
    return {"k": k, "v": v}


def _own_prompt(s, spinq):
    return {"out": spinq.prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["max_q"], s["max_k"])}


def _own_prefix(s, spinq):
    cache = spinq.KV4Pages(s["k_codes"], s["v_codes"], s["scales"])
    return {"out": spinq.prefix_attention_kv4(s["q"], cache, s["prefix_table"], s["prefix"], s["table"], s["lens"])}


def run(state):
    if own:
        from paper_2405_16406_gb300 import spinq
        return {"write": _own_write, "read": _own_read, "prompt": _own_prompt,
                "prefix": _own_prefix}[state["op"]](state, spinq)
    return {"write": _plain_write, "read": _plain_read, "prompt": _plain_prompt,
            "prefix": _plain_prefix}[state["op"]](state)


# ------------------------------------------------------------ the unavoidable
def work(case):
    lens = _lengths(case)
    dim, hk, hq = case["head_dim"], case["kv_heads"], case.get("heads", 0)
    row4 = hk * (dim + 16)        # a token's codes and scales of K and V
    row16 = hk * dim * 4          # a token's K and V in fp16
    n = sum(lens)
    if case["op"] == "write":
        # projection in, rotated queries and pages out, then the pages in and fp16 K and V out; a token's slot
        # and position; the rotation table's rows once
        rows = hq + hk
        flops = n * rows * dim * (math.log2(dim) + (4 if case["norm"] else 0) + 3 * case["rotary"] / dim)
        flops += n * 2 * hk * dim * 6
        return {"bytes": n * ((2 * hq + 2 * hk) * dim * 2 + row4 + row4 + row16 + 12) + max(lens) * 4 * case["rotary"],
                "flops": flops}
    if case["op"] == "read":
        return {"bytes": n * (row4 + row16), "flops": n * hk * dim * 4}
    if case["op"] == "prompt":
        pairs = sum(m * case["context"] + m * (m + 1) // 2 for m in lens)
        keys = n + case["context"] * len(lens)
        return {"bytes": n * hq * dim * 4 + keys * row16, "flops": 4 * pairs * hq * dim}
    keys = case["batch"] * case["prefix"] + n
    return {"bytes": (case["prefix"] + n) * row4 + case["batch"] * hq * dim * 4, "flops": 4 * keys * hq * dim}


# ------------------------------------------------------------------ 64 bits
def _sylvester(n):
    i = torch.arange(n)
    bits = i[:, None] & i[None]
    parity = sum((bits >> b) & 1 for b in range(8)) & 1
    return (1.0 - 2.0 * parity.double()).cuda()


def _exact_rows(x, weight, case, positions):
    x = x.double()
    dim, part = x.shape[-1], case["rotary"]
    if weight is not None:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * weight.double()
    theta = 500000.0 ** (-2.0 * torch.arange(part // 2, device="cuda", dtype=torch.float64) / part)
    # the table that the call takes holds 32-bit values
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), positions.double()[:, None] * theta)
    turn = torch.complex(turn.real.float().double(), turn.imag.float().double())[:, None]
    y = x.clone()
    if case["interleaved"]:
        y[..., :part] = torch.view_as_real(torch.complex(x[..., 0:part:2], x[..., 1:part:2]) * turn).flatten(-2)
    else:
        z = torch.complex(x[..., :part // 2], x[..., part // 2:part]) * turn
        y[..., :part // 2], y[..., part // 2:part] = z.real, z.imag
    return y @ _sylvester(dim) / math.sqrt(dim)


def _exact_codes(y):
    beta = y.amin(-1, keepdim=True)
    alpha = (y.amax(-1, keepdim=True) - beta) / 15
    u = torch.where(alpha > 0, ((y - beta) / alpha).round(), torch.zeros_like(y))
    return u * alpha + beta


def _exact_tokens(s, pages, n):
    """K and V [n, Hkv, D] in 64 bits of the first n tokens of one sequence's pages."""
    out = []
    used = pages[:(n + s["page"] - 1) // s["page"]].long()
    for which, name in ((0, "k_codes"), (1, "v_codes")):
        c = s[name][used].transpose(1, 2).flatten(0, 1)[:n].int()
        f = s["scales"][used].transpose(1, 2).flatten(0, 1)[:n].double()
        u = torch.empty(c.shape[:2] + (s["head_dim"],), dtype=torch.float64, device="cuda")
        u[..., 0::2], u[..., 1::2] = (c % 16).double(), (c // 16).double()
        out.append(u * f[..., 2 * which:2 * which + 1] + f[..., 2 * which + 1:2 * which + 2])
    return out


def _exact_attention(q, k, v, seen=None):
    """q [n, Hq, D], k and v [m, Hkv, D] in 64 bits; seen [n, m] or None."""
    out = torch.zeros_like(q)
    if k.shape[0] == 0:
        return out
    group = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        a = q[:, h] @ k[:, h // group].T / math.sqrt(q.shape[-1])
        if seen is not None:
            a = a.masked_fill(~seen, -math.inf)
        out[:, h] = torch.softmax(a, -1) @ v[:, h // group]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    dim, hk, hq, lens = case["head_dim"], case["kv_heads"], case.get("heads"), _lengths(case)
    if case["op"] == "write":
        x = s["fused"].view(s["total"], hq + 2 * hk, dim)
        k = _exact_codes(_exact_rows(x[:, hq:hq + hk], s["k_weight"], case, s["positions"]))
        return {"q": _exact_rows(x[:, :hq], s["q_weight"], case, s["positions"]), "k": k,
                "v": _exact_codes(x[:, hq + hk:].double())}
    if case["op"] == "read":
        every = [_exact_tokens(s, s["table"][b], n) for b, n in enumerate(lens)]
        return {"k": torch.cat([e[0] for e in every]), "v": torch.cat([e[1] for e in every])}
    if case["op"] == "prompt":
        out, at, ak = [], 0, 0
        for n in lens:
            m = n + case["context"]
            seen = torch.ones((n, m), dtype=torch.bool, device="cuda").tril(m - n)
            out.append(_exact_attention(s["q"][at:at + n].double(), s["k"][ak:ak + m].double(),
                                        s["v"][ak:ak + m].double(), seen))
            at, ak = at + n, ak + m
        return {"out": torch.cat(out)}
    # the prefix for every sequence at once, then each sequence's own tokens, joined by their sums
    q = s["q"].double()
    pk, pv = _exact_tokens(s, s["prefix_table"], case["prefix"])
    group, scale = hq // hk, 1 / math.sqrt(dim)
    out = torch.zeros_like(q)
    score = [q[:, h] @ pk[:, h // group].T * scale for h in range(hq)] if case["prefix"] else None
    for b, n in enumerate(lens):
        k, v = _exact_tokens(s, s["table"][b], n)
        for h in range(hq if n + case["prefix"] else 0):
            a = k[:, h // group] @ q[b, h] * scale
            if score is not None:
                a = torch.cat((score[h][b], a))
            w = torch.softmax(a, 0)
            out[b, h] = w[case["prefix"]:] @ v[:, h // group]
            if score is not None:
                out[b, h] += w[:case["prefix"]] @ pv[:, h // group]
    return {"out": out}
