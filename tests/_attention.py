"""Plain float64 forms of the attention operators, and how far a result may be from them.

Bounds follow from the roundings that the operators state.  With u = 2^-8 (bf16, eight significant bits, round to nearest: half the spacing 2^-7 above a power of two) an
element of a bf16 result is within u |ref| of its sum, and a sum over rounded probabilities (or score gradients) within
u sum |p| |v| of the exact one; the delta of the backward is taken from the rounded o, which moves each score gradient
by up to u p sum |do| |o|.  Float32 sums and exponentials are below that by more than 2^-10.  In float32 the scores
carry a rounding error of about sqrt(D) 2^-24 sum |q_d k_d| scale (1e-6 at the sizes here), which is the relative error
of the probabilities, and the score gradients that of their own sums: 2e-5 of the sums of magnitudes leaves a factor of
ten."""

import math

import torch

U16, U32 = 2.0 ** -8 * 1.1, 2e-5


def dense_mask(Tq, Tk, lo=None, hi=None, causal=False, offset=None):
    j = torch.arange(Tk)
    seen = torch.ones(Tq, Tk, dtype=torch.bool)
    if lo is not None:
        seen &= (j >= lo[:, None]) & (j < hi[:, None])
    if causal:
        seen &= j <= (torch.arange(Tq) + (Tk - Tq if offset is None else offset))[:, None]
    return seen


def attention(q, k, v, seen, scale=None, softcap=0.0, slopes=None, offset=None, do=None):
    """o, lse, and with do the gradients; each result with the sum of magnitudes that its rounding scales with."""
    q, k, v = (t.detach().double().cpu() for t in (q, k, v))
    Tq, H, D = q.shape
    Tk, K, _ = k.shape
    g = H // K
    scale = D ** -0.5 if scale is None else scale
    q, k, v = q.transpose(0, 1), k.transpose(0, 1).repeat_interleave(g, 0), v.transpose(0, 1).repeat_interleave(g, 0)
    z = scale * q @ k.transpose(1, 2)
    slope = torch.ones_like(z)
    if softcap:
        t = torch.tanh(z / softcap)
        z, slope = softcap * t, 1 - t * t
    if slopes is not None:
        at = torch.arange(Tq) + (Tk - Tq if offset is None else offset)
        z = z - slopes.double().cpu()[:, None, None] * (at[:, None] - torch.arange(Tk)).abs()
    z = z.masked_fill(~seen, -math.inf)
    empty = ~seen.any(1)
    lse = torch.logsumexp(z, 2) if Tk else torch.full((H, Tq), -math.inf, dtype=torch.float64)
    p = torch.where(seen, torch.exp(z - torch.where(empty, 0.0, lse)[..., None]), 0.0)
    o = p @ v
    rows = lambda t: t.transpose(0, 1)  # noqa: E731
    out = {"o": (rows(o), rows(p @ v.abs())), "lse": (lse, lse.abs().nan_to_num(posinf=0.0))}
    if do is None:
        return out
    do = do.detach().double().cpu().transpose(0, 1)
    dp = do @ v.transpose(1, 2)
    ds = p * (dp - (do * o).sum(-1, keepdim=True))
    dz = scale * ds * slope
    mag = scale * slope * p * (dp.abs() + 2 * (do.abs() * o.abs()).sum(-1, keepdim=True))
    shared = lambda t: rows(t.view(K, g, Tk, D).sum(1))  # noqa: E731
    out["dq"] = (rows(dz @ k), rows(mag @ k.abs()))
    out["dk"] = (shared(dz.transpose(1, 2) @ q), shared(mag.transpose(1, 2) @ q.abs()))
    out["dv"] = (shared(p.transpose(1, 2) @ do), shared(p.transpose(1, 2) @ do.abs()))
    return out


def check(name, got, want, dtype):
    """Every element within the bound of its type; infinities and NaN nowhere but where the reference has them."""
    ref, mag = want
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert bool((torch.isfinite(got) == fine).all()), f"{name}: infinities or NaN in other places"
    assert bool((got[~fine & ~torch.isnan(ref)] == ref[~fine & ~torch.isnan(ref)]).all()), name
    u = U16 if dtype == torch.bfloat16 and name != "lse" else U32
    off = (got - ref).abs() - u * (ref.abs() + mag)
    worst = float(off[fine].max()) if bool(fine.any()) else 0.0
    assert worst <= 1e-30 + 1e-7 * float(mag[fine].max() if bool(fine.any()) else 0), f"{name}: {worst} past its bound"


def rotated(x, cos, sin, interleaved):
    """x [T, heads, D] with the first 2 cos.shape[1] elements of each head turned, as complex numbers."""
    rot = 2 * cos.shape[1]
    turn = torch.complex(cos.double(), sin.double())[:, None]
    if interleaved:
        pairs = x[..., :rot].reshape(*x.shape[:2], rot // 2, 2)
    else:
        pairs = x[..., :rot].reshape(*x.shape[:2], 2, rot // 2).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    if not interleaved:
        y = y.transpose(-1, -2)
    return torch.cat([y.reshape(*x.shape[:2], rot), x[..., rot:]], -1)


def heads_norm_rope(x, weight, cos, sin, interleaved, eps):
    x = x.double()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    return x if cos is None else rotated(x, cos, sin, interleaved)


def close(name, got, ref, dtype, scale=None):
    """Elementwise: half an ulp of bf16, or float32 rounding, against the larger of the element and `scale` (the
    magnitude of the sums behind it; its row's root mean square where none is given)."""
    got, ref = got.detach().double().cpu(), ref.detach().double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    if not ref.numel():
        return
    rms = ref.square().mean(-1, keepdim=True).sqrt() if scale is None else scale
    bound = (2.0 ** -8 * ref.abs() + 1e-5 * rms) if dtype == torch.bfloat16 else 4e-6 * torch.maximum(ref.abs(), rms)
    worst = float(((got - ref).abs() - bound).max())
    assert worst <= 1e-30, f"{name}: {worst} past its bound"
