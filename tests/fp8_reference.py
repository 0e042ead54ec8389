"""Plain 64-bit forms of the 8-bit products, what feeds them and the token log probabilities, and the
bounds that their tests use (rounding counted in half steps: bf16 2^-8, fp32 2^-24, e4m3 2^-4)."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F8 = torch.float8_e4m3fn
LEAST = 2.0 ** -120

ACT = {
    "none": lambda z: z,
    "relu": lambda z: torch.where(z < 0, torch.zeros_like(z), z),
    "silu": lambda z: z * torch.sigmoid(z),
    "gelu": lambda z: z * torch.special.ndtr(z),
    "gelu_tanh": lambda z: 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))),
}


def quantised(a):
    """(unrounded codes, scale) of the rows of a (fp64), and which rows hold a NaN or an infinity."""
    bad = ~torch.isfinite(a).all(-1)
    a = torch.where(bad[:, None], torch.zeros_like(a), a)
    scale = (a.abs().amax(-1) / 448.0).clamp(min=LEAST)
    return a / scale[:, None], scale, bad


def rmsnorm(x, residual, gamma, eps):
    """(h = x + residual, 1 / rms, h gamma) in fp64."""
    h = x.double() if residual is None else x.double() + residual.double()
    r = 1.0 / torch.sqrt((h * h).mean(-1) + eps)
    return h, r, h if gamma is None else h * gamma.double()


def half_step_e4m3(v):
    """Half the distance of neighbouring e4m3 values at v."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    return torch.exp2(e - 4)


def assert_codes(codes, v):
    """codes are v to the nearest, but for 1e-4 of a half step: v itself is a few fp32 roundings off, each 2^-24 of
    v, and a half step is 2^-5 of v at least."""
    got = codes.double()
    assert torch.isfinite(got).all()
    assert ((got - v).abs() <= half_step_e4m3(v) * (1 + 1e-4)).all()


def assert_within(got, ref, bound):
    """|got - ref| <= bound where ref is finite, the same infinities and NaN elsewhere."""
    got, ref = got.double(), ref.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), "NaN pattern"
    inf = ~fine & ~torch.isnan(ref)
    assert torch.equal(got[inf], ref[inf]), "infinities"
    off = (got - ref).abs()[fine] - (bound if not isinstance(bound, torch.Tensor) else bound[fine])
    assert off.numel() == 0 or off.max().item() <= 0, f"{off.max().item():.3e} past the bound"


def linear(x, xs, w, ws, b, act, up=None, us=None, ub=None, residual=None, f32=True):
    """(result, bound of the error before the output's rounding) of codes x[M, K], w[K, N] in fp64.  A sum of K
    products in fp32 is off by at most K 2^-24 of the sum of their magnitudes; scales and bias add 3 roundings.
    The 8-bit instructions (f32 false) drop at most 2^-13 of the largest of 16 products from each of the 15
    others: 15 2^-13 of the sum of magnitudes."""
    K = x.shape[1]
    parts = (K + 3) * 2.0 ** -24 + (0.0 if f32 else 15 * 2.0 ** -13)

    def product(w, ws, b):
        z = (x.double() @ w.double()) * xs.double()[:, None] * ws.double()
        size = (x.double().abs() @ w.double().abs()) * xs.double()[:, None] * ws.double()
        if b is not None:
            z, size = z + b.double(), size + b.double().abs()
        return z, size * parts

    z, e = product(w, ws, b)
    y = ACT[act](z)
    # no activation is steeper than 1.2; its own evaluation: 16 roundings of its value or, where it
    # cancels (1 + erf or tanh near -1), of its argument
    e = 1.2 * e + (16 * 2.0 ** -24 * z.abs() if act not in ("none", "relu") else 0.0)
    if up is not None:
        u, eu = product(up, us, ub)
        y, e = y * u, e * u.abs() + y.abs() * eu + e * eu + (y * u).abs() * 2.0 ** -24
    if residual is not None:
        y = y + residual.double()
        e = e + y.abs() * 2.0 ** -24
    return y, e


def logprobs(logits, targets, top, scale=1.0):
    """{"logprobs", "entropy", "top_logprobs", "top_ids"} in fp64; ids by the logits, the lowest first among equals."""
    x = logits.double()
    y = x * scale
    y = y - y.amax(1, keepdim=True)  # first: at 1e38 even 64 bits have no room for ln V beside y
    logp = y - torch.logsumexp(y, 1, keepdim=True)
    bad = torch.isnan(x).any(1) | (x == math.inf).any(1) | (x == -math.inf).all(1)
    p = logp.exp()
    entropy = -torch.special.xlogy(p, p).sum(1)
    entropy[bad] = math.nan
    logp[bad] = math.nan
    out = {"entropy": entropy, "logprobs": None, "top_logprobs": None, "top_ids": None}
    if targets is not None and targets.shape[1]:
        t = targets.long()
        given = logp.gather(1, t.clamp(0, x.shape[1] - 1))
        given[t >= x.shape[1]] = math.nan
        given[t < 0] = 0.0
        out["logprobs"] = given
    if top:
        key = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
        order = torch.sort(key, dim=1, descending=True, stable=True)[1]
        ids = order[:, :top]
        out["top_ids"], out["top_logprobs"] = ids, logp.gather(1, ids)
    return out
