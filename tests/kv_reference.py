"""Plain 64-bit forms of the rotary positions, the paged cache and attention over it (tests only)."""
import math

import torch

PAGE = 64
F8 = torch.float8_e4m3fn


def turned(x, cs, interleaved=False, inverse=False):
    """x[T, H, d] with rows cs[T, rot/2, 2] of the table, fp64."""
    x, cs = x.double(), cs.double()
    half = cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * (-1.0 if inverse else 1.0)
    y = x.clone()
    p = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    q = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    y[..., p] = x[..., p] * c - x[..., q] * s
    y[..., q] = x[..., p] * s + x[..., q] * c
    return y


def k_byte(o, x, d, e):
    """Byte of token o, dimension x of K in a block, e bytes an element (the documented layout)."""
    E = 16 // e
    u, a, j, t, i = o // (4 * E), o // E % 4, o % E // 8, o % 8 // 4, o % 4
    c, g, r = x // (4 * E), x // E % 4, x % E
    return (((((E // 8 * u + j) * 2 + t) * (d // (4 * E)) + c) * 4 + g) * 16 + 4 * a + i) * 16 + r * e


def v_byte(o, x, d, e):
    E = 16 // e
    u, g, r = o // (4 * E), o // E % 4, o % E
    return (((u * (d // 16) + x // 16) * 4 + g) * 16 + x % 16) * 16 + r * e


def held(data, d, fmt):
    """(K codes, V codes, K scales, V scales): fp32 [pages, heads, 64, d] and [pages, heads, 64]."""
    data = data.cpu()
    e = 2 if fmt == "bf16" else 1
    n = PAGE * d
    out = []
    for at, byte in ((0, k_byte), (n * e, v_byte)):
        idx = torch.tensor([byte(o, x, d, e) // e for o in range(PAGE) for x in range(d)])
        part = data[..., at:at + n * e].contiguous().view(torch.bfloat16 if e == 2 else F8).float()
        out.append(part[..., idx].view(*part.shape[:-1], PAGE, d))
    for at in (2 * n * e, 2 * n * e + 4 * PAGE):
        out.append(data[..., at:at + 4 * PAGE].contiguous().view(torch.float32))
    return out


def fill(data, d, fmt, pages, K, V):
    """Puts K, V [len(pages) * 64 at most, heads, d] into the pages in order: codes, by the layout."""
    e = 2 if fmt == "bf16" else 1
    n = PAGE * d
    ki = torch.tensor([k_byte(o, x, d, e) // e for o in range(PAGE) for x in range(d)]).view(PAGE, d)
    vi = torch.tensor([v_byte(o, x, d, e) // e for o in range(PAGE) for x in range(d)]).view(PAGE, d)
    word = torch.int16 if e == 2 else torch.uint8
    for at, idx, rows, scale_at in ((0, ki, K, 2 * n * e), (n * e, vi, V, 2 * n * e + 4 * PAGE)):
        if fmt == "bf16":
            codes, scale = rows.to(torch.bfloat16), torch.ones(rows.shape[:-1])
        else:
            scale = torch.clamp(rows.float().abs().amax(-1) / 448.0, min=2.0 ** -120)
            codes = (rows.float() / scale[..., None]).to(F8)
        for k in range(0, rows.shape[0], PAGE):
            m = min(PAGE, rows.shape[0] - k)
            block = data[pages[k // PAGE]]
            lie = block[:, at:at + n * e].contiguous().view(word)
            lie[:, idx[:m].reshape(-1)] = codes[k:k + m].view(word).permute(1, 0, 2).reshape(rows.shape[1], -1)
            block[:, at:at + n * e] = lie.view(torch.uint8)
            s = block[:, scale_at:scale_at + 4 * PAGE].contiguous().view(torch.float32)
            s[:, :m] = scale[k:k + m].t()
            block[:, scale_at:scale_at + 4 * PAGE] = s.view(torch.uint8)


def attend(q, K, V, scale, last):
    """q[n, Hq, d] against K, V[L, Hkv, d] (fp64): query i sees keys 0 .. last[i].  (out, absolute),
    `absolute` the same sum over |V|: what a relative error of the numerators is measured against."""
    n, Hq, d = q.shape
    g = Hq // K.shape[1]
    out, absolute = torch.zeros((n, Hq, d), dtype=torch.float64), torch.zeros((n, Hq, d), dtype=torch.float64)
    for i in range(n):
        m = last[i] + 1
        if m <= 0:
            continue
        for h in range(Hq):
            p = torch.softmax(K[:m, h // g] @ q[i, h].double() * scale, 0)
            out[i, h], absolute[i, h] = p @ V[:m, h // g], p @ V[:m, h // g].abs()
    return out, absolute


def attention_error(got, out, absolute):
    """Largest error over its bound.  A numerator is rounded to bf16 (8 significant bits: 2^-8 of itself at most),
    so the sum may be off by 2^-8 of the sum over |V|; half as much again for the scores, which are
    fp32 sums; the result is rounded once (2^-8)."""
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(out)), "NaN in other places than the plain form"
    bound = (2.0 ** -8 + 2.0 ** -9) * absolute + (2.0 ** -8 + 2.0 ** -15) * out.abs() + 1e-30
    err = ((got - out).abs() / bound).nan_to_num(0.0)
    return float(err.max())


def inv_sqrt(d):
    return 1.0 / math.sqrt(d)
