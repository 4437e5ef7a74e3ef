"""How exactly the 4-bit cache's attention adds up V: cases whose logits are
exact, so that only the sum over the slots is at stake, with a bound that has no
room for an operand rounded once to fp16 where the kernel keeps what the
rounding left.

Logits: K's groups are constant (scale 0) and zero but for the first, and a
query has one channel, so z is one product: off by 2^-22 of itself (|z| <= 8
here) and its exponential by 2^-22: 2^-19 of a probability.  Sums: a product of
the tensor cores adds 16 numbers to a sum, each cut off at 2^-25 of the largest's
power of two, and cuts the result off at 2^-23 (measured: 2^-25 added to 1 sixteen
times in one product is 2^-21, 2^-26 nothing; 2^-24 added once is nothing): at
most (17/4 + 1) 2^-23 of what the sum holds.  A warp has one tile here, four steps
with two products each, 8 x 5.25 x 2^-23 = 2^-17.6: of 15 p s a slot before the
middle comes off, and of p (|m'| + 7.5 s) for the middles and the codes' own; with
the joins' roundings at most 2^-17 of sum p (15 s + |m'|).  Rests: two fp16
numbers hold p, p s and m' to 2^-21.  So
  |error| <= half a step of the output + 2^-17 sum p (15 s + |m'|)
             + (2^-19 + 2^-20) sum p (s |c| + |m'|),   c = n - 7.5, m' = m + 7.5 s,
and for bf16 outputs, whose p and p s are rounded once,
             + 2^-11 (sum p s |c| + sum p |s c + m'|).
"""
import numpy as np
import pytest
import torch

from oracle import q4_oracle as q4

SLOTS = (64, 300)
QUERIES = (1.0, 0.7, -1.3, 0.3)


def v_rows(kind, n, gen):
    """Codes, scales and minima (bf16 numbers) of V."""
    if kind == "wide":         # one channel a hundred times wider than the others
        x = torch.randn((n, 128), generator=gen)
        x[:, 5::32] *= 100.0
        return q4.quantise(x.bfloat16().float().numpy())
    codes = torch.randint(0, 16, (n, 128), generator=gen).numpy()
    s = 2.0 ** torch.randint(-2, 3, (n, 4), generator=gen).double().numpy()
    s *= 1 + torch.randint(0, 8, (n, 4), generator=gen).double().numpy() / 8  # (15 s / 2: bf16 numbers)
    if kind == "centred":      # middles of 0: the codes' sum alone
        return codes, s, -7.5 * s
    m = 80 + 60 * torch.rand((n, 4), generator=gen)  # kind "opposite": in pairs that cancel
    m[1::2] = -m[::2]
    return codes, s * 2.0 ** -6, m.bfloat16().double().numpy()


def logits(kind, n, gen):
    """x [n] (bf16 numbers) and a [4] with z = a x; uniform for the pairs."""
    x = (1.5 * torch.randn(n, generator=gen)).clamp(-6, 6).bfloat16().double().numpy()
    a = torch.tensor(QUERIES).half().double().numpy()
    return x, a * (kind != "opposite")


def bound(dtype, p, codes, s, m, want):
    s, m = np.repeat(s, 32, -1).astype(float), np.repeat(m, 32, -1).astype(float)
    c, mid = codes - 7.5, m + 7.5 * s
    half, floor = (2.0 ** -11, 2.0 ** -24) if dtype == torch.float16 else (2.0 ** -8, 2.0 ** -132)
    tol = half * np.abs(want) + 2.0 ** -17 * (p @ (15 * s + np.abs(mid)))
    tol += (2.0 ** -19 + 2.0 ** -20) * (p @ (s * np.abs(c) + np.abs(mid))) + floor
    if dtype == torch.bfloat16:
        tol += 2.0 ** -11 * (p @ (s * np.abs(c)) + p @ np.abs(s * c + mid))
    return tol


def exact(kind, n, gen):
    codes, s, m = v_rows(kind, n, gen)
    x, a = logits(kind, n, gen)
    e = np.exp(a[:, None] * x)
    p = e / e.sum(-1, keepdims=True)
    return codes, s, m, x, a, p, p @ q4.values(codes, s, m)


def emulated(codes, s, m, z, lost=()):
    """The kernel's operands in fp16, exact sums; `lost`: rests that are left out."""
    h = lambda v: np.asarray(v).astype(np.float16).astype(float)  # noqa: E731
    s, m = np.asarray(s, float), np.asarray(m, float)
    e = np.floor(np.log2(np.maximum(16 * s.max(-1), np.abs(m).max(-1))))
    s1, mid = s * 2.0 ** (3 - e)[:, None], (m + 7.5 * s) * 2.0 ** (3 - e)[:, None]
    p = 2.0 ** (z * np.log2(np.e))
    w = p * 2.0 ** e
    gain = 2.0 ** (2 - np.floor(np.log2(w.max())))
    w, back = w * gain, 8 * gain
    hi = h(w)
    lo = 0 if "p" in lost else h(w - hi)
    mh = h(mid)
    ml = 0 if "middles" in lost else h(mid - mh)
    out = np.zeros(128)
    for J in range(4):
        ps = h(hi * s1[:, J])
        rest = 0 if "p s" in lost else h(hi * s1[:, J] - ps + lo * s1[:, J])
        ml_j = ml if np.isscalar(ml) else ml[:, J]
        out[32 * J:32 * J + 32] = (ps + rest) @ (codes[:, 32 * J:32 * J + 32] - 7.5)
        # (what is left of p s comes off with the middle as well: sum p s is of the same operands)
        out[32 * J:32 * J + 32] += (hi + lo) @ mh[:, J] + hi @ (ml_j + np.zeros(len(w)))
    return out / back / p.sum()


@pytest.mark.parametrize("kind,lost", [("wide", ["middles"]), ("opposite", ["middles"]), ("centred", ["p"]),
                                       ("centred", ["p s"]), ("wide", ["p s"])])
def test_the_bound_sees_an_operand_rounded_once(kind, lost):
    for n in SLOTS:
        gen = torch.Generator().manual_seed(n)
        codes, s, m, x, a, p, want = exact(kind, n, gen)
        tol = bound(torch.float16, p, codes, s, m, want)
        with_all, without = [], []
        for r in range(4):
            for left_out, said in (((), with_all), (lost, without)):
                got = emulated(codes, s, m, a[r] * x, left_out)
                got = torch.from_numpy(got).half().double().numpy()
                said.append(np.abs(got - want[r]) <= tol[r])
        assert np.all(with_all)
        assert not np.all(without), (kind, lost, n)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["wide", "opposite", "centred"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_adds_up_exactly(cuda_device, kind, dtype):
    import paper_2606_24467_gb300 as ckv

    dev = cuda_device
    c = ckv.q4_cache(1, len(SLOTS), max(SLOTS), dev)
    c.weights.zero_()
    wanted = []
    q = torch.zeros((1, 4 * len(SLOTS), 1, 128))
    for g, n in enumerate(SLOTS):
        codes, s, m, x, a, p, want = exact(kind, n, torch.Generator().manual_seed(n))
        c.v_codes[0, g, :n] = torch.from_numpy(q4.pack(codes)).to(dev)
        c.v_params[0, g, :n] = torch.from_numpy(np.concatenate([s, m], -1)).bfloat16().to(dev)
        assert np.array_equal(c.v_params[0, g, :n, 4:].double().cpu().numpy(), m)
        c.k_codes[0, g, :n] = 0
        c.k_params[0, g, :n] = 0
        c.k_params[0, g, :n, 4] = torch.from_numpy(x).bfloat16().to(dev)
        c.lengths[0, g] = n
        q[0, 4 * g:4 * g + 4, 0, 3] = torch.from_numpy(a)
        wanted.append((codes, s, m, p, want))
    if dtype == torch.bfloat16:  # the queries' own rounding, first
        q = q.to(dtype)
        for g, (codes, s, m, p, want) in enumerate(wanted):
            x = c.k_params[0, g, :SLOTS[g], 4].double().cpu().numpy()
            e = np.exp(q[0, 4 * g:4 * g + 4, 0, 3].double().numpy()[:, None] * x)
            p = e / e.sum(-1, keepdims=True)
            wanted[g] = (codes, s, m, p, p @ q4.values(codes, s, m))
    q = q.to(dtype).to(dev)
    out = torch.empty_like(q)
    ckv.q4_attend(c, q, out, ckv.q4_workspace(c, q.shape[1], 1), scale=1.0)
    for g, (codes, s, m, p, want) in enumerate(wanted):
        got = out[0, 4 * g:4 * g + 4, 0].double().cpu().numpy()
        tol = bound(dtype, p, codes, s, m, want)
        assert (np.abs(got - want) <= tol).all(), (g, (np.abs(got - want) / tol).max())
