"""Rotary positions and attention over a paged cache in float64 (torch, on the
tensors' device), from the definitions, for the tests.  Shares no code with the
CUDA path."""
import torch


def rotate(x, positions, frequencies, interleaved, scale=1.0, backward=False):
    """Rows x [rows, heads, 128] turned by their positions: pairs of the first 2
    len(frequencies) channels, as complex numbers."""
    y = x.double().clone()
    f = torch.as_tensor(frequencies, dtype=torch.float64, device=x.device)
    n = f.numel()
    angle = positions.double()[:, None, None] * f * (-1 if backward else 1)
    first = torch.arange(n, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.full_like(angle, scale), angle)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def rows_of(pages, table_row, first, count):
    """Slots first .. first + count - 1 of a sequence, [count, heads, 128]."""
    page = pages.shape[1]
    slot = torch.arange(first, first + count, device=pages.device)
    at = table_row.long()[torch.div(slot, page, rounding_mode="floor")]
    inside = (at >= 0) & (at < pages.shape[0])
    rows = pages[torch.where(inside, at, 0), slot % page]
    return torch.where(inside[:, None, None], rows, torch.zeros_like(rows))


def attend(q, k, v, start, causal, scale):
    """One sequence: q [n, Hq, 128] whose token i stands at slot start + i, k and v
    [length, H, 128].  Returns out, lse [Hq, n], and for tolerances the sums over
    the slots seen of p |v| and of |v|, the largest p, and the largest sum |q k| a
    row.  What a token does not see is not touched."""
    n, hq, d = q.shape
    length, h = k.shape[:2]
    group = hq // h
    out = torch.zeros(n, hq, d, dtype=torch.float64, device=q.device)
    lse = torch.full((hq, n), -float("inf"), dtype=torch.float64, device=q.device)
    pv, sv = torch.zeros_like(out), torch.zeros_like(out)
    top, mass = torch.ones_like(lse), torch.zeros_like(lse)
    for i in range(n):
        seen = max(min(length, start + i + 1), 0) if causal else length
        if not seen:
            continue
        kk = k[:seen].double().repeat_interleave(group, 1)  # [seen, Hq, d]
        vv = v[:seen].double().repeat_interleave(group, 1)
        x = q[i].double()
        z = torch.einsum("hd,shd->hs", x, kk) * scale
        lse[:, i] = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[:, i, None])
        out[i] = torch.einsum("hs,shd->hd", p, vv)
        pv[i] = torch.einsum("hs,shd->hd", p, vv.abs())
        sv[i] = vv.abs().sum(0)
        top[:, i] = p.amax(1)
        mass[:, i] = torch.einsum("hd,shd->hs", x.abs(), kk.abs()).amax(1) * scale
    return out, lse, {"pv": pv, "sv": sv, "top": top, "mass": mass}


def tolerance(dtype, slots, out, lse, parts):
    """How far out [n, Hq, 128] and lse [Hq, n] of the kernel may be off, from what
    it rounds: a logit by 2^-20 of its terms' magnitudes (fp32 sums of the tensor
    cores, and the scale), so p by twice that and as much again for the sum of
    exponentials; an exponential and the sums of it by 2^-20; a probability to the
    dtype, half a step (and for f16, which it enters times 2^7, below 2^-21 of the
    largest, 2^-32 of that); the output's fp32 sums by 2^-23 for every 16 slots; and
    the output to the dtype."""
    half = torch.finfo(dtype).eps / 2
    logit = parts["mass"] * 2.0 ** -20
    per = (4 * logit + 2.0 ** -19).T[..., None] + half + (slots / 16 + 16) * 2.0 ** -23
    tol = parts["pv"] * per + half * out.abs() + torch.finfo(dtype).smallest_normal * half
    if dtype == torch.float16:
        tol = tol + parts["sv"] * parts["top"].T[..., None] * 2.0 ** -32
    seen = torch.isfinite(lse)
    ltol = 2 * logit + 2.0 ** -19 + torch.where(seen, lse, 0).abs() * 2.0 ** -22
    return tol, ltol
