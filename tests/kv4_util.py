"""Plain 64-bit forms of the paged cache's operators, and case builders."""
import numpy as np
import torch


def sylvester(n):
    h = np.ones((1, 1))
    while h.shape[0] < n:
        h = np.block([[h, h], [h, -h]])
    return h


def cos_sin(max_pos, rotary, base=10000.0):
    th = base ** (-2.0 * np.arange(rotary // 2) / rotary)
    ang = np.arange(max_pos)[:, None] * th[None, :]
    return np.stack([np.cos(ang), np.sin(ang)], axis=-1).astype(np.float32)


def rotated_rows(x, weight, eps, positions, table, interleaved):
    """Norm, rotary embedding and H_D / sqrt(D) of x [T, H, D] (float64)."""
    x = np.array(x, dtype=np.float64)
    D = x.shape[-1]
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if table is not None:
        half = table.shape[1]
        cs = table[np.clip(positions, 0, table.shape[0] - 1)].astype(np.float64)
        c, s = cs[:, None, :, 0], cs[:, None, :, 1]
        if interleaved:
            a, b = x[..., 0:2 * half:2].copy(), x[..., 1:2 * half:2].copy()
            x[..., 0:2 * half:2], x[..., 1:2 * half:2] = a * c - b * s, a * s + b * c
        else:
            a, b = x[..., :half].copy(), x[..., half:2 * half].copy()
            x[..., :half], x[..., half:2 * half] = a * c - b * s, a * s + b * c
    return x @ sylvester(D) / np.sqrt(D)


def codes_of(y, clip=1.0):
    """(u, alpha, beta) of Eq. 1, asymmetric, 4 bits, of rows y."""
    beta = clip * y.min(-1, keepdims=True)
    alpha = (clip * y.max(-1, keepdims=True) - beta) / 15
    safe = np.where(alpha > 0, alpha, 1)
    u = np.where(alpha > 0, np.clip(np.rint((y - beta) / safe), 0, 15), 0)
    return u, alpha[..., 0], beta[..., 0]


def unpack(codes):
    c = codes.astype(np.int64)
    return np.stack([c & 15, c >> 4], -1).reshape(c.shape[:-1] + (2 * c.shape[-1],)).astype(np.float64)


def slot_values(cache, slots):
    """(codes, alpha, beta) of K and of V at the slots [T]: [T, Hkv, D] and [T, Hkv]."""
    P = cache.k_codes.shape[2]
    page = torch.as_tensor(slots).long().to(cache.k_codes.device) // P
    at = torch.as_tensor(slots).long().to(cache.k_codes.device) % P
    sc = cache.scales[page, :, at].double().cpu().numpy()
    out = []
    for w, c in ((0, cache.k_codes), (1, cache.v_codes)):
        out.append((unpack(c[page, :, at].cpu().numpy()), sc[..., 2 * w], sc[..., 2 * w + 1]))
    return out


def token_slots(table, P, start, n):
    """Slot numbers of tokens start .. start + n - 1 of a page list."""
    t = np.arange(start, start + n)
    return np.asarray(table, dtype=np.int64)[t // P] * P + t % P


def attention(q, k, v, scale, visible=None):
    """o and sum p |v| of q [n, Hq, D] over k, v [m, Hkv, D] (float64); visible [n, m] or None."""
    n, Hq, D = q.shape
    o, size = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    if k.shape[0] == 0:
        return o, size
    G = Hq // k.shape[1]
    for h in range(Hq):
        s = scale * (q[:, h] @ k[:, h // G].T)
        if visible is not None:
            s = np.where(visible, s, -np.inf)
        top = s.max(-1, keepdims=True)
        p = np.exp(s - np.where(np.isinf(top), 0, top))
        tot = p.sum(-1, keepdims=True)
        p = np.where(tot > 0, p / np.where(tot > 0, tot, 1), 0)
        o[:, h], size[:, h] = p @ v[:, h // G], p @ np.abs(v[:, h // G])
    return o, size


def random_cache(spinq, rng, pages, P, Hkv, D, poison=True):
    """A cache of random codes and scales on the GPU; unwritten slots are the caller's to poison."""
    kc = rng.integers(0, 256, (pages, Hkv, P, D // 2)).astype(np.uint8)
    vc = rng.integers(0, 256, (pages, Hkv, P, D // 2)).astype(np.uint8)
    sc = np.empty((pages, Hkv, P, 4), np.float32)
    for a in (0, 2):
        sc[..., a] = 0.2 * (1 + rng.random((pages, Hkv, P)))
        sc[..., a + 1] = -7.5 * sc[..., a] + 0.3 * rng.standard_normal((pages, Hkv, P))
    return spinq.KV4Pages(torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), torch.from_numpy(sc).cuda())


def page_tables(rng, lens, P, extra=2):
    """Page lists of sequences of the given lengths over shuffled pages: (table [B, W] int32, pages)."""
    need = [-(-n // P) for n in lens]
    total = sum(need) + extra
    order = rng.permutation(total).astype(np.int32)
    table = np.full((len(lens), max(need + [1])), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total
