"""The 4-bit cache on the device against the float64 oracle: rows appended and
gathered bit by bit, attention, eviction, and the decode loop that runs them
together (needs a GB300).

Tolerances of the attention, derived from what it rounds.  Logits: the codes
and the queries enter the products exactly; at most 32 roundings of at most
2^-23 (sums that the tensor core truncates) of S, the sum of the magnitudes of
a row's products, so |dz| <= 2^-18 S.  Probabilities: relative 2 |dz| + 2^-20.
Output, as sum p s c + sum p m' with c = n - 7.5 and m' = m + 7.5 s: a 16-bit
rounding (2^-8 or 2^-11 of the value); p in fp16 and once more p s, or m', in
fp16: two roundings of 2^-11 of each term, 2^-10 (sum p s |c| + sum p |m'|);
truncated sums: a step of 16 slots cuts at most 2^-23 of what its sum holds, so
350 steps at most 2^-14 of the terms' magnitudes, and the four steps of a tile,
which hold up to 15 p s a slot before the middle comes off, 2^-19 of sum p s;
and the probabilities' error on both terms.
"""
import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
import workloads as wl
from oracle import q4_oracle as q4
from paper_2606_24467_gb300 import compresskv as B

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
BYTES = ("k_codes", "v_codes", "k_params", "v_params", "positions", "weights", "lengths")


def host(cache):
    """A cache's buffers as numpy arrays (params as float32)."""
    c = {n: getattr(cache, n).cpu() for n in BYTES if getattr(cache, n) is not None}
    return {n: (t.float() if t.dtype == torch.bfloat16 else t).numpy() for n, t in c.items()}


def bits(cache):
    return {n: getattr(cache, n).clone().view(torch.uint8) for n in BYTES if getattr(cache, n) is not None}


def blank(b, h, cap, dev, weights=True):
    """A cache whose free slots hold what must not be read as data."""
    c = ckv.q4_cache(b, h, cap, dev, weights=weights)
    for n in ("k_codes", "v_codes"):
        getattr(c, n).fill_(0xA7)
    for n in ("k_params", "v_params"):
        getattr(c, n).fill_(float("nan"))
    c.positions.fill_(-7)
    if weights:
        c.weights.fill_(float("nan"))
    return c


def random_cache(b, h, cap, lens, dev, gen, weights=True, scale=1.0):
    """A cache with quantised random rows in its first slots."""
    c = blank(b, h, cap, dev, weights)
    cap = c.capacity
    lens = np.broadcast_to(np.asarray(lens), (b, h))
    for part in ("k", "v"):
        x = torch.randn((b, h, cap, 128), generator=gen) * scale
        codes, s, m = q4.quantise(x.numpy())
        par = torch.from_numpy(np.concatenate([s, m], -1)).bfloat16()
        for i in range(b):
            for g in range(h):
                n = lens[i, g]
                getattr(c, part + "_codes")[i, g, :n] = torch.from_numpy(q4.pack(codes[i, g, :n])).to(dev)
                getattr(c, part + "_params")[i, g, :n] = par[i, g, :n].to(dev)
    c.lengths.copy_(torch.from_numpy(lens.astype(np.int32)))
    order = torch.rand((b, h, cap), generator=gen).argsort(-1).int() * 2
    c.positions.copy_(order)
    if weights:
        c.weights.copy_(torch.rand((b, h, cap), generator=gen) * 3)
    return c


def stored(c, part, i, g, n):
    """Float64 values of a unit's first n slots (of host(cache))."""
    par = c[part + "_params"][i, g, :n]
    return q4.values(q4.unpack(c[part + "_codes"][i, g, :n]), par[:, :4], par[:, 4:])


def check_rows(c, i, g, slots, k, v):
    """The cache's slots hold the quantised rows (float32 arrays), bit by bit."""
    for part, x in (("k", k), ("v", v)):
        codes, s, m = q4.quantise(x)
        assert np.array_equal(c[part + "_codes"][i, g][slots], q4.pack(codes)), part
        want = np.concatenate([s, m], -1)
        assert np.array_equal(c[part + "_params"][i, g][slots], want, equal_nan=True), part


def check_values(back, x, dtype):
    codes, s, m = q4.quantise(x)
    want = q4.values(codes, s, m)
    got = back.float().cpu().numpy().astype(np.float64)
    # one rounding to fp32 (2^-24) and one to the rows' type
    tol = (HALF_STEP[dtype] + 2.0 ** -22) * np.abs(want) + (2.0 ** -25 if dtype == torch.float16 else 0)
    assert np.array_equal(np.isnan(want), np.isnan(got))
    ok = np.isnan(want) | (np.abs(got - want) <= tol)
    assert ok.all()


# ------------------------------------------------------------------ append
KINDS = ["normal", "offset", "constant", "tiny", "wide", "ties", "zeros", "non_finite"]


def make_rows(kind, shape, gen, dtype):
    x = torch.randn(shape, generator=gen)
    if kind == "offset":
        x = x * 0.03 + 7.5
    elif kind == "constant":
        x = torch.full(shape, -1.375)
    elif kind == "tiny":
        x = x * (2.0 ** -20 if dtype == torch.float16 else 2.0 ** -128)  # subnormal spreads
    elif kind == "wide":
        x = x * (2.0 ** 12 if dtype == torch.float16 else 2.0 ** 120)
    elif kind == "ties":
        x = torch.randint(0, 31, shape, generator=gen).float() / 2  # scale 1, half-way values
        x[..., 0::32] = 0.0
        x[..., 1::32] = 15.0
    elif kind == "zeros":
        x = torch.where(torch.rand(shape, generator=gen) < 0.7, 0.0, x)
        x = torch.where(torch.rand(shape, generator=gen) < 0.2, -0.0, x)
    x = x.to(dtype)
    if kind == "non_finite":
        flat = x.view(-1, 128)
        flat[0, 5], flat[1, 40], flat[2, 127] = float("nan"), float("inf"), float("-inf")
        if dtype == torch.bfloat16:
            flat[3, 64], flat[3, 65] = 3e38, -3e38  # a spread beyond fp32
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [1, 5, 70])
def test_append_quantises_bit_by_bit(cuda_device, dtype, kind, rows):
    gen = torch.Generator().manual_seed(rows)
    b, h = 3, 4
    k = make_rows(kind, (b * rows, h, 128), gen, dtype)
    v = make_rows(kind, (b * rows, h, 128), gen, dtype)
    c = blank(b, h, 96, cuda_device)
    c.lengths.copy_(torch.tensor([[0, 1, 2, 3], [9, 0, 26, 13], [26, 26, 26, 0]], dtype=torch.int32))
    old = host(c)
    pos = torch.arange(b * rows, dtype=torch.int32) + 100
    kd, vd = k.to(cuda_device), v.to(cuda_device)
    kv, vv = torch.empty_like(kd), torch.empty_like(vd)
    ckv.q4_append(c, kd, vd, pos.to(cuda_device), k_values=kv, v_values=vv)
    new = host(c)
    for i in range(b):
        for g in range(h):
            n0 = int(old["lengths"][i, g])
            at = slice(n0, n0 + rows)
            part = slice(i * rows, (i + 1) * rows)
            check_rows(new, i, g, at, k[part, g].float().numpy(), v[part, g].float().numpy())
            assert np.array_equal(new["positions"][i, g, at], pos[part].numpy())
            assert (new["weights"][i, g, at] == 0).all() and new["lengths"][i, g] == n0 + rows
            for n in BYTES[:-1]:  # every other slot as it was
                o, w = np.delete(old[n][i, g], np.r_[at], 0), np.delete(new[n][i, g], np.r_[at], 0)
                assert np.array_equal(o, w, equal_nan=o.dtype.kind == "f"), n
    check_values(kv, k.float().numpy(), dtype)
    check_values(vv, v.float().numpy(), dtype)


@pytest.mark.parametrize("most", [3, 80])
def test_append_ragged_padded_and_full(cuda_device, most):
    """cu_rows with an empty sequence, padding by negative positions, a unit
    without room and one whose start is outside; strided rows; no weights."""
    gen = torch.Generator().manual_seed(9)
    n = [most, 0, 2, most, 1]
    cu = np.concatenate([[0], np.cumsum(n)])
    b, h, cap = 5, 2, 96
    big = torch.randn((int(cu[-1]), 3, 2 * 128), generator=gen).bfloat16().to(cuda_device)
    k, v = big[:, :2, :128], big[:, :2, 128:]
    c = blank(b, h, cap, cuda_device, weights=False)
    start = torch.tensor([[4, 0], [7, 8], [95, 94], [10, 20], [-1, 97]], dtype=torch.int32)
    c.lengths.fill_(50)
    pos = torch.arange(int(cu[-1]), dtype=torch.int32)
    pos[cu[3] + 2:cu[4]] = -1  # two rows of sequence 3 are real
    status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    old = host(c)
    ckv.q4_append(c, k, v, pos.to(cuda_device), cu_rows=cu, start=start.to(cuda_device),
                  device_status=status)
    new = host(c)
    assert int(status) == B.CKV_ERR_DEVICE_INDEX
    real = [most, 0, 2, 2, 1]
    for i in range(b):
        for g in range(h):
            at = int(start[i, g])
            if not 0 <= at <= cap:
                assert new["lengths"][i, g] == 50
                assert np.array_equal(old["k_codes"][i, g], new["k_codes"][i, g])
                continue
            used = min(real[i], cap - at)
            assert new["lengths"][i, g] == at + used
            rows = slice(cu[i], cu[i] + used)
            check_rows(new, i, g, slice(at, at + used), k[rows, g].float().cpu().numpy(),
                       v[rows, g].float().cpu().numpy())
            assert np.array_equal(old["k_codes"][i, g, :at], new["k_codes"][i, g, :at])
    # without a status word, and with room for all: none is needed
    ckv.q4_append(c, k, v, pos.to(cuda_device), cu_rows=cu, start=torch.zeros_like(c.lengths))
    assert c.lengths.cpu()[:, 0].tolist() == real


def test_append_of_no_rows(cuda_device):
    c = blank(2, 3, 32, cuda_device)
    c.lengths.fill_(9)
    k = torch.empty((0, 3, 128), dtype=torch.float16, device=cuda_device)
    pos = torch.empty(0, dtype=torch.int32, device=cuda_device)
    ckv.q4_append(c, k, k, pos)
    assert (c.lengths == 9).all()
    ckv.q4_append(c, k, k, pos, start=torch.full_like(c.lengths, 4))  # a rollback alone
    assert (c.lengths == 4).all()


def test_append_to_many_sequences(cuda_device):
    """More sequences than a table of rows may have."""
    b, h = 700, 2
    gen = torch.Generator().manual_seed(2)
    k = torch.randn((b, h, 128), generator=gen).half()
    c = blank(b, h, 32, cuda_device)
    ckv.q4_append(c, k.to(cuda_device), k.to(cuda_device),
                  torch.zeros(b, dtype=torch.int32, device=cuda_device))
    new = host(c)
    assert (new["lengths"] == 1).all()
    codes, s, m = q4.quantise(k.float().numpy())
    assert np.array_equal(new["k_codes"][:, :, 0], q4.pack(codes))
    assert np.array_equal(new["v_params"][:, :, 0], np.concatenate([s, m], -1))
    ckv.q4_append(c, k[:0].to(cuda_device), k[:0].to(cuda_device),
                  torch.zeros(0, dtype=torch.int32, device=cuda_device), start=torch.zeros_like(c.lengths))
    assert (c.lengths == 0).all()


# ------------------------------------------------------------------ gather
def test_gather_of_a_compression(cuda_device):
    """The retained rows of a ragged batch (one sequence empty, one shorter than
    the window) as compress_layer chose them, weights from the raw scores."""
    dev = cuda_device
    lens = [900, 0, 20, 333]
    cfg = wl.get("c1").scaled(dtype="bf16", batch=4, seq_len=0, srh_per_group=(1, 2))
    d = wl.make_layer(cfg, 0, lengths=lens, budgets=np.full((1, 4), 100, np.int32))
    q, k, v = d["q_win"].to(dev), d["k"].to(dev), d["v"].to(dev)
    p = ckv.Problem(q, k, d["cu_seqlens"], cfg.window, cfg.pool_width)
    out = ckv.LayerOutputs(p, d["budgets"], 128, k.dtype, dev)
    ws = ckv.workspace(p, dev)
    cu_out = ckv.compress_layer(p, q, k, v, d["srh_mask"], d["budgets"], out.indices, out.k_out,
                                out.v_out, ws, raw=out.raw)
    c = blank(4, 8, 110, dev)
    kv, vv = torch.empty_like(out.k_out), torch.empty_like(out.v_out)
    ckv.q4_gather(p, c, out.indices, cu_out, k, v, raw=out.raw, k_values=kv, v_values=vv, ws=ws)
    assert ckv.read_device_status(ws) == 0
    new, idx, raw = host(c), out.indices.cpu().numpy(), out.raw.cpu().numpy()
    ko, vo = out.k_out.float().cpu().numpy(), out.v_out.float().cpu().numpy()
    for s in range(4):
        o0, o1 = int(cu_out[s]), int(cu_out[s + 1])
        for g in range(8):
            assert new["lengths"][s, g] == o1 - o0
            check_rows(new, s, g, slice(0, o1 - o0), ko[o0:o1, g], vo[o0:o1, g])
            assert np.array_equal(new["positions"][s, g, :o1 - o0], idx[g, o0:o1])
            at = idx[g, o0:o1]
            n = max(lens[s] - cfg.window, 0)
            want = np.where(at < n, np.append(raw[g, out.cu_prefix[s]:], 0.)[np.minimum(at, max(n - 1, 0))], 0)
            assert np.array_equal(new["weights"][s, g, :o1 - o0], want.astype(np.float32))
            assert (new["positions"][s, g, o1 - o0:] == -7).all()
    check_values(kv, ko, torch.bfloat16)
    check_values(vv, vo, torch.bfloat16)
    ckv.q4_gather(p, c, out.indices, cu_out, k, v)  # without raw scores: weight 0
    assert (c.weights[0, :, :100] == 0).all()


def test_gather_of_head_budgets(cuda_device):
    dev, cfg = cuda_device, wl.get("c1").scaled(seq_len=600)
    d = wl.make_layer(cfg, 0)
    q, k, v = d["q_win"].to(dev), d["k"].to(dev), d["v"].to(dev)
    p = ckv.Problem(q, k, d["cu_seqlens"], cfg.window, cfg.pool_width)
    gb = np.array([[32, 40, 600, 77, 64, 90, 33, 128]], np.int32)
    cu, rows = ckv.head_budget_layout(p, gb)
    idx = torch.empty(rows, dtype=torch.int32, device=dev)
    ko = torch.empty((rows, 128), dtype=k.dtype, device=dev)
    vo = torch.empty_like(ko)
    ws = ckv.workspace(p, dev)
    cu_out = ckv.compress_layer_head_budgets(p, q, k, v, d["srh_mask"], gb, idx, ko, vo, ws)
    c = blank(1, 8, 600, dev)
    kv, vv = torch.empty_like(ko), torch.empty_like(vo)
    ckv.q4_gather(p, c, idx, cu_out, k, v, k_values=kv, v_values=vv)
    new, at = host(c), idx.cpu().numpy()
    for g in range(8):
        o0, o1 = int(cu_out[g, 0]), int(cu_out[g, 1])
        assert new["lengths"][0, g] == gb[0, g] == o1 - o0
        check_rows(new, 0, g, slice(0, o1 - o0), ko[o0:o1].float().cpu().numpy(),
                   vo[o0:o1].float().cpu().numpy())
        assert np.array_equal(new["positions"][0, g, :o1 - o0], at[o0:o1])
    check_values(kv, ko.float().cpu().numpy(), k.dtype)


def test_gather_reports_an_index_outside(cuda_device):
    dev = cuda_device
    k = torch.randn((50, 2, 128), device=dev).half()
    q = torch.zeros((1, 4, 16, 128), dtype=torch.float16, device=dev)
    p = ckv.Problem(q, k, [0, 50], 16, 7)
    idx = torch.tensor([[0, 50, 2], [1, -1, 49]], dtype=torch.int32, device=dev)
    c = blank(1, 2, 32, dev)
    ws = ckv.q4_workspace(c)
    ckv.q4_gather(p, c, idx, [0, 3], k, k, ws=ws)
    assert ckv.read_device_status(ws) == B.CKV_ERR_DEVICE_INDEX
    new = host(c)
    assert new["positions"][0, :, :3].tolist() == [[0, -7, 2], [1, -7, 49]]
    kk = k.float().cpu().numpy()
    check_rows(new, 0, 1, [0, 2], kk[[1, 49], 1], kk[[1, 49], 1])


# ------------------------------------------------------------------ attention
def check_attend(c, q, out, lse, before, after, scale, q_positions=None, weights=True):
    """Against the oracle, unit by unit (c: host(cache) before the call)."""
    b, hq, n, _ = q.shape
    h = c["lengths"].shape[1]
    group = hq // h
    qd = q.double().cpu().numpy()
    got, gl = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    half = HALF_STEP[q.dtype]
    floor = 2.0 ** -24 if q.dtype == torch.float16 else 2.0 ** -132  # of the type's subnormals
    for i in range(b):
        for g in range(h):
            used = int(np.clip(c["lengths"][i, g], 0, c["positions"].shape[2]))
            k, v = stored(c, "k", i, g, used), stored(c, "v", i, g, used)
            par = c["v_params"][i, g, :used].astype(np.float64)
            sc = np.repeat(par[:, :4], 32, -1)
            m = np.abs(np.repeat(par[:, 4:], 32, -1) + 7.5 * sc)
            code = np.abs(q4.unpack(c["v_codes"][i, g, :used]) - 7.5) * sc
            kp = c["k_params"][i, g, :used].astype(np.float64)
            kmag = (q4.unpack(c["k_codes"][i, g, :used]) * np.repeat(kp[:, :4], 32, -1)
                    + np.abs(np.repeat(kp[:, 4:], 32, -1)))
            for x in (m, code, kmag, sc):
                x[np.isnan(x)] = 0
            add, slack = np.zeros(used), np.zeros(used)
            for hh in range(g * group, (g + 1) * group):
                vis = np.ones((n, used), bool)
                if q_positions is not None:
                    vis = c["positions"][i, g, :used][None] <= q_positions[i].cpu().numpy()[:, None]
                ro, rl, p = q4.attend(qd[i, hh], k, v, vis, scale)
                for t in range(n):
                    S = scale * (kmag[vis[t]] @ np.abs(qd[i, hh, t])).max(initial=0.0)
                    dz = 2.0 ** -18 * S
                    dp = 2 * dz + 2.0 ** -20
                    terms = p[t][vis[t]] @ (code + m)[vis[t]]
                    tol = (half * np.abs(ro[t]) + (2.0 ** -10 + 2.0 ** -14 + dp) * terms
                           + 2.0 ** -19 * (p[t][vis[t]] @ sc[vis[t]]) + floor)
                    same_nan = np.isnan(ro[t]) & np.isnan(got[i, hh, t])
                    assert ((np.abs(got[i, hh, t] - ro[t]) <= tol) | same_nan).all(), (i, hh, t)
                    if gl is not None:
                        if np.isfinite(rl[t]):
                            assert abs(gl[i, hh, t] - rl[t]) <= dz + 2.0 ** -20 * max(1, abs(rl[t]))
                        else:
                            assert np.array_equal(gl[i, hh, t], rl[t], equal_nan=True)
                    add += p[t]
                    slack += p[t] * dp
            if weights:
                w0, w1 = before[i, g].astype(np.float64), after[i, g].astype(np.float64)
                tol = slack + 2.0 ** -21 * (np.abs(w0[:used]) + add) + 1e-30
                bad = np.isnan(add)
                assert (np.abs(w1[:used] - w0[:used] - add) <= tol)[~bad].all(), (i, g)
                assert np.array_equal(w0[used:], w1[used:], equal_nan=True)


def run_attend(c, q, scale=0.0, q_positions=None, accumulate=True, with_lse=True, out=None):
    dev = q.device
    ws = ckv.q4_workspace(c, q.shape[1], q.shape[2])
    out = torch.full_like(q, float("nan")) if out is None else out
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=dev) if with_lse else None
    before = host(c)
    ckv.q4_attend(c, q, out, ws, q_positions=q_positions, scale=scale, lse=lse, accumulate=accumulate)
    assert ckv.read_device_status(ws) == 0
    after = host(c)
    for n in BYTES:
        if n != "weights":
            assert np.array_equal(before[n], after[n], equal_nan=before[n].dtype.kind == "f"), n
    check_attend(before, q, out, lse, before.get("weights"), after.get("weights"),
                 scale or 128 ** -0.5, q_positions, accumulate)
    if not accumulate and "weights" in before:
        assert np.array_equal(before["weights"], after["weights"], equal_nan=True)
    return out, lse


LENS = {"one": [[1, 1]], "empty": [[0, 0], [5, 0]], "tile": [[31, 32], [33, 64]],
        "ragged": [[1000, 3], [517, 640]], "long": [[5000, 4999]]}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("group,n", [(1, 1), (4, 1), (7, 1), (8, 1), (4, 2), (7, 4), (3, 5), (16, 1), (2, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend(cuda_device, lens, group, n, dtype):
    le = np.array(LENS[lens])
    b, h = le.shape
    gen = torch.Generator().manual_seed(group * 100 + n)
    c = random_cache(b, h, int(le.max()) + 40, le, cuda_device, gen)
    q = torch.randn((b, h * group, n, 128), generator=gen).to(dtype).to(cuda_device)
    run_attend(c, q)


@pytest.mark.parametrize("group,n", [(4, 1), (8, 1), (7, 4), (4, 16)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_attend_by_position(cuda_device, group, n, accumulate):
    """Slots above a query's position are not seen; rows that see one slot, or none."""
    le = np.array([[700, 64], [33, 1]])
    gen = torch.Generator().manual_seed(n)
    c = random_cache(2, 2, 704, le, cuda_device, gen, weights=accumulate)
    q = torch.randn((2, 2 * group, n, 128), generator=gen).bfloat16().to(cuda_device)
    at = torch.randint(0, 1400, (2, n), generator=gen).int()
    at[0, 0] = -1                                   # sees nothing
    if n > 2:
        at[0, 1] = 2 ** 31 - 1                      # sees all
        at[0, 2] = int(c.positions[0, 0, :700].min())
    out, lse = run_attend(c, q, q_positions=at.to(cuda_device), accumulate=accumulate)
    assert not out[0, :, 0].any() and (lse[0, :, 0] == float("-inf")).all()


def test_attend_strides_scale_and_broadcast(cuda_device):
    gen = torch.Generator().manual_seed(4)
    c = random_cache(3, 2, 128, [[100, 90], [1, 128], [64, 65]], cuda_device, gen)
    base = torch.randn((3, 4, 10, 136), generator=gen).bfloat16().to(cuda_device)
    q = base.transpose(1, 2)[..., :128]                       # [3, 10, 4, 128]
    hold = torch.full((3, 4, 10, 136), 7.0, device=cuda_device).bfloat16()
    run_attend(c, q, scale=0.3, out=hold.transpose(1, 2)[..., :128])
    assert (hold[..., 128:] == 7).all()
    one = torch.randn((1, 1, 1, 128), generator=gen).half().to(cuda_device).expand(3, 10, 2, 128)
    run_attend(c, one, out=torch.empty((3, 10, 2, 128), dtype=torch.float16, device=cuda_device))


@pytest.mark.parametrize("scale", [1e-3, 30.0, 2.0 ** 60, 2.0 ** -100])
def test_attend_value_ranges(cuda_device, scale):
    """Rows far from 1: all of one magnitude, and of magnitudes that differ by slot."""
    gen = torch.Generator().manual_seed(6)
    c = random_cache(1, 2, 320, [[300, 77]], cuda_device, gen)
    c.v_params.copy_((c.v_params.double() * scale).bfloat16())
    c.v_params[0, 1, 5] *= 2.0 ** -12                 # a token of small values
    q = torch.randn((1, 8, 1, 128), generator=gen).bfloat16().to(cuda_device)
    run_attend(c, q)


def test_attend_large_logits_and_small_queries(cuda_device):
    gen = torch.Generator().manual_seed(8)
    c = random_cache(1, 1, 640, [[640]], cuda_device, gen, scale=4.0)
    for f in (40.0, 1e-4, 2.0 ** -120, 0.0):
        q = (torch.randn((1, 4, 1, 128), generator=gen) * f).bfloat16().to(cuda_device)
        run_attend(c, q)
    run_attend(c, (torch.randn((1, 4, 1, 128), generator=gen) * 6e-8).half().to(cuda_device))


def test_attend_non_finite_slots(cuda_device):
    """A NaN group is seen by the rows that see its slot and by no other."""
    gen = torch.Generator().manual_seed(10)
    c = random_cache(1, 2, 96, [[90, 80]], cuda_device, gen)
    c.positions.copy_(torch.arange(96, dtype=torch.int32).expand(1, 2, 96))
    c.v_params[0, 0, 50, [1, 5]] = float("nan")
    c.k_params[0, 1, 60, [2, 6]] = float("nan")
    q = torch.randn((1, 8, 2, 128), generator=gen).bfloat16().to(cuda_device)
    at = torch.tensor([[40, 85]], dtype=torch.int32, device=cuda_device)
    out, lse = run_attend(c, q, q_positions=at)
    assert torch.isfinite(out[:, :, 0]).all() and torch.isfinite(lse[:, :, 0]).all()
    nan = torch.isnan(out[0, :4, 1])
    assert nan[:, 32:64].all() and not nan[:, :32].any() and not nan[:, 64:].any()
    assert torch.isnan(out[0, 4:, 1]).all() and torch.isnan(lse[0, 4:, 1]).all()
    # an odd number of rows, none of which sees the slot
    c.weights.zero_()
    q3 = torch.randn((1, 6, 1, 128), generator=gen).bfloat16().to(cuda_device)
    run_attend(c, q3, q_positions=at[:, :1].contiguous())
    assert torch.isfinite(c.weights[0, 1, :80]).all() and (c.weights[0, 1, 41:80] == 0).all()
    # a query that holds a NaN or an infinity stays alone
    c = random_cache(1, 2, 96, [[90, 80]], cuda_device, gen)
    for bad in (float("nan"), float("inf")):
        q = torch.randn((1, 8, 1, 128), generator=gen).half().to(cuda_device)
        clean = torch.empty_like(q)
        ws = ckv.q4_workspace(c, 8, 1)
        ckv.q4_attend(c, q, clean, ws)
        q2 = q.clone()
        q2[0, 3, 0, 77] = bad
        got = torch.empty_like(q)
        ckv.q4_attend(c, q2, got, ws)
        keep = [0, 1, 2, 4, 5, 6, 7]
        assert torch.equal(got[:, keep], clean[:, keep])
        assert not torch.isfinite(got[0, 3]).any()


def test_attend_is_the_same_on_every_call(cuda_device):
    gen = torch.Generator().manual_seed(12)
    c = random_cache(4, 2, 1500, [[1500, 1], [20, 900], [0, 33], [1499, 1031]], cuda_device, gen)
    q = torch.randn((4, 14, 3, 128), generator=gen).half().to(cuda_device)
    w0 = c.weights.clone()
    ws = ckv.q4_workspace(c, 14, 3)
    got = []
    for _ in range(3):
        c.weights.copy_(w0)
        out = torch.empty_like(q)
        ckv.q4_attend(c, q, out, ws, accumulate=True)
        got.append((out, c.weights.clone()))
    for o, w in got[1:]:
        assert torch.equal(o.view(torch.int16), got[0][0].view(torch.int16))
        assert torch.equal(w.view(torch.int32), got[0][1].view(torch.int32))


@pytest.mark.parametrize("b,h,most", [(140, 1, 300), (70, 4, 200), (129, 1, 2000), (500, 5, 90), (3, 1, 9000)])
def test_attend_many_units(cuda_device, b, h, most):
    """Units by the hundred, some empty: whole in a warp, in a CTA, or shared."""
    gen = torch.Generator().manual_seed(b)
    le = torch.randint(0, most, (b, h), generator=gen).numpy()
    le[::7] = 0
    le[-1, -1] = most
    c = random_cache(b, h, most, le, cuda_device, gen)
    run_attend(c, torch.randn((b, 2 * h, 1, 128), generator=gen).bfloat16().to(cuda_device))
    run_attend(c, torch.randn((b, 9 * h, 1, 128), generator=gen).half().to(cuda_device))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_averages_many_slots(cuda_device, dtype):
    """Attention spread over 64K slots, each warp summing thousands: the output
    is small against its terms, and keeps its precision.  Bound: 2^-8 or 2^-11 of
    the value; eight standard deviations of the independent roundings of p, p s
    and m' (at most 2^-11 each, of p s c or p m'); 2^-19 of sum p s for the tiles'
    sums and, for a bias along the 432 steps of a warp, 2^-14 of the value."""
    units, cap = 128, 65536
    gen = torch.Generator(device=cuda_device).manual_seed(61)
    c = ckv.q4_cache(16, 8, cap, cuda_device, weights=False)
    for part in ("k", "v"):
        getattr(c, part + "_codes").random_(0, 256, generator=gen)
        par = getattr(c, part + "_params")
        par[..., :4] = 0.1 + 0.05 * torch.rand((16, 8, cap, 4), generator=gen, device=cuda_device)
        par[..., 4:] = -7.5 * par[..., :4].float() + 0.05 * torch.randn((16, 8, cap, 4), generator=gen,
                                                                        device=cuda_device)
    c.lengths.fill_(cap)
    q = (0.7 * torch.randn((16, 32, 1, 128), generator=gen, device=cuda_device)).to(dtype)
    out = torch.empty_like(q)
    ckv.q4_attend(c, q, out, ckv.q4_workspace(c, 32, 1))
    for b, g in ((0, 0), (7, 3), (15, 7)):
        def term(part):
            raw = getattr(c, part + "_codes")[b, g].int()
            n = torch.stack([raw & 15, raw >> 4], -1).flatten(-2).double()
            par = getattr(c, part + "_params")[b, g].double().repeat_interleave(32, -1)
            return par[:, :128] * (n - 7.5), par[:, 128:] + 7.5 * par[:, :128], par[:, :128]
        kc, km, _ = term("k")
        vc, vm, vs = term("v")
        for h in range(4 * g, 4 * g + 4):
            p = ((kc + km) @ q[b, h, 0].double() * 128 ** -0.5).softmax(0)
            want = p @ (vc + vm)
            sd = 2.0 ** -11 * (2 * (p.square() @ (vc.square() + vm.square()))).sqrt()
            tol = (HALF_STEP[dtype] + 2.0 ** -14) * want.abs() + 8 * sd + 2.0 ** -19 * (p @ vs)
            assert ((out[b, h, 0].double() - want).abs() <= tol).all(), (b, h)


def test_attend_with_256_rows_a_unit(cuda_device):
    gen = torch.Generator().manual_seed(71)
    c = random_cache(1, 1, 500, [[490]], cuda_device, gen)
    q = torch.randn((1, 16, 16, 128), generator=gen).bfloat16().to(cuda_device)
    run_attend(c, q, q_positions=torch.randint(0, 1000, (1, 16), generator=gen).int().to(cuda_device))


@pytest.mark.parametrize("lens", ["empty", "tile", "ragged", "long"])
@pytest.mark.parametrize("group,n,causal", [(12, 1, False), (7, 4, True), (3, 5, False), (16, 16, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_of_a_large_cache(cuda_device, lens, group, n, causal, dtype):
    """More than 2^20 slots, where row blocks have 16 rows, few of them in use."""
    le = np.array(LENS[lens])
    gen = torch.Generator().manual_seed(group + n)
    small = random_cache(*le.shape, int(le.max()) + 40, le, cuda_device, gen)
    c = blank(*le.shape, 2 ** 20 // le.size + 32, cuda_device)
    used = small.capacity
    for name in BYTES[:-1]:
        getattr(c, name)[:, :, :used] = getattr(small, name)
    c.lengths.copy_(small.lengths)
    q = torch.randn((le.shape[0], le.shape[1] * group, n, 128), generator=gen).to(dtype).to(cuda_device)
    at = None
    if causal:
        at = torch.randint(-1, 2 * used, (le.shape[0], n), generator=gen).int().to(cuda_device)
    ws = ckv.q4_workspace(c, q.shape[1], n)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float32, device=cuda_device)
    ckv.q4_attend(c, q, out, ws, q_positions=at, lse=lse, accumulate=True)
    assert ckv.read_device_status(ws) == 0
    assert torch.isnan(c.weights[:, :, used:]).all() and (c.positions[:, :, used:] == -7).all()
    after = c.weights[:, :, :used].cpu().numpy()
    check_attend(host(small), q, out, lse, host(small)["weights"], after, 128 ** -0.5, at)


def test_attend_all_empty(cuda_device):
    c = blank(3, 2, 64, cuda_device)
    q = torch.randn((3, 8, 2, 128), device=cuda_device).half()
    out, lse = run_attend(c, q)
    assert not out.any() and (lse == float("-inf")).all()


def test_attend_with_one_workspace_for_calls_of_many_shapes(cuda_device):
    """Calls in turn, and captured graphs in turn, share a workspace."""
    gen = torch.Generator().manual_seed(19)
    calls = []
    for b, h, n, group, le in ((1, 2, 1, 4, 9000), (2, 4, 3, 3, 700), (4, 1, 1, 16, 40), (1, 1, 1, 1, 20000)):
        c = random_cache(b, h, le, le, cuda_device, gen)
        q = torch.randn((b, h * group, n, 128), generator=gen).bfloat16().to(cuda_device)
        want = torch.empty_like(q)
        ckv.q4_attend(c, q, want, ckv.q4_workspace(c, h * group, n), accumulate=False)
        calls.append((c, q, want, torch.empty_like(q)))
    most = max(ckv.q4_workspace_size(c, q.shape[1], q.shape[2]) for c, q, _, _ in calls)
    ws = torch.zeros(most, dtype=torch.uint8, device=cuda_device)
    for c, q, want, got in calls * 2:
        got.zero_()
        ckv.q4_attend(c, q, got, ws)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    graphs = []
    for c, q, want, got in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ckv.q4_attend(c, q, got, ws)
        graphs.append(g)
    for _ in range(2):
        for g, (c, q, want, got) in zip(graphs, calls):
            got.zero_()
            g.replay()
            assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_steps_on_a_share_of_the_sms(cuda_device):
    """The stream of a green context: fewer CTAs, the same values."""
    from test_gpu_shared_sms import GreenStream
    try:
        green = GreenStream(16)
    except (OSError, AttributeError, RuntimeError) as e:
        pytest.skip(f"no green contexts here: {e}")
    gen = torch.Generator().manual_seed(23)
    c = random_cache(2, 2, 5000, [[5000, 3000], [100, 0]], cuda_device, gen)
    q = torch.randn((2, 8, 1, 128), generator=gen).bfloat16().to(cuda_device)
    ws, out = ckv.q4_workspace(c, 8, 1), torch.empty_like(q)
    lse = torch.empty((2, 8, 1), device=cuda_device)
    before = host(c)
    torch.cuda.synchronize()
    ckv.q4_attend(c, q, out, ws, lse=lse, accumulate=True, stream=green.stream)
    torch.cuda.synchronize()
    after = host(c)
    check_attend(before, q, out, lse, before["weights"], after["weights"], 128 ** -0.5)
    ckv.q4_evict(c, 1000, ws, sinks=2, recent=5, stream=green.stream)
    torch.cuda.synchronize()
    check_evict(after, host(c), np.full((2, 2), 1000), 2, 5)


def test_attend_lengths_outside_the_cache(cuda_device):
    gen = torch.Generator().manual_seed(13)
    c = random_cache(1, 3, 64, [[64, 64, 64]], cuda_device, gen)
    c.lengths.copy_(torch.tensor([[-5, 1000, 64]], dtype=torch.int32))
    run_attend(c, torch.randn((1, 3, 1, 128), generator=gen).bfloat16().to(cuda_device))


def test_attend_and_append_behind_2_gib(cuda_device):
    """A unit whose codes and params lie behind 2^31 bytes (and 2^31 params)."""
    cap, h = 1 << 20, 40
    gen = torch.Generator().manual_seed(14)
    c = ckv.q4_cache(1, h, cap, cuda_device)
    c.lengths.zero_()
    n = 700
    x = torch.randn((1, 1, n, 128), generator=gen)
    codes, s, m = q4.quantise(x.numpy())
    for part in ("k", "v"):
        getattr(c, part + "_codes")[0, h - 1, cap - n:] = torch.from_numpy(q4.pack(codes[0, 0])).to(cuda_device)
        getattr(c, part + "_params")[0, h - 1, cap - n:] = torch.from_numpy(
            np.concatenate([s, m], -1)[0, 0]).bfloat16().to(cuda_device)
        getattr(c, part + "_codes")[0, h - 1, :cap - n] = 0
        getattr(c, part + "_params")[0, h - 1, :cap - n] = 0
    c.positions[0, h - 1] = torch.arange(cap, dtype=torch.int32, device=cuda_device)
    c.weights[0, h - 1] = 0
    c.lengths[0, h - 1] = cap - 1
    k = torch.randn((1, h, 128), generator=gen).bfloat16()
    ckv.q4_append(c, k.to(cuda_device), k.to(cuda_device),
                  torch.tensor([cap], dtype=torch.int32, device=cuda_device))
    assert int(c.lengths[0, h - 1]) == cap and int(c.lengths[0, 0]) == 1
    q = torch.randn((1, h, 1, 128), generator=gen).bfloat16().to(cuda_device)
    out = torch.empty_like(q)
    ws = ckv.q4_workspace(c, h, 1)
    ckv.q4_attend(c, q, out, ws, accumulate=True)
    tail = slice(cap - n, cap)
    kv = stored(host_slice(c, h - 1, tail), "k", 0, 0, n)
    vv = stored(host_slice(c, h - 1, tail), "v", 0, 0, n)
    z = np.zeros(cap)
    z[cap - n:] = 128 ** -0.5 * (kv @ q[0, h - 1, 0].double().cpu().numpy())
    p = np.exp(z - z.max())
    p /= p.sum()
    want = p[cap - n:] @ vv
    got = out[0, h - 1, 0].double().cpu().numpy()
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * (p[cap - n:] @ np.abs(vv) + p[cap - n:].sum() * 4)
    assert (np.abs(got - want) <= tol).all()
    w = c.weights[0, h - 1].double().cpu().numpy()
    assert np.allclose(w, p, rtol=1e-3, atol=1e-12)


def host_slice(c, unit, cut):
    out = {}
    for part in ("k", "v"):
        out[part + "_codes"] = getattr(c, part + "_codes")[:, unit:unit + 1, cut].cpu().numpy()
        out[part + "_params"] = getattr(c, part + "_params")[:, unit:unit + 1, cut].float().cpu().numpy()
    return out


# ------------------------------------------------------------------ eviction
def check_evict(c0, c1, budgets, sinks, recent):
    """host(cache) before and after, budgets [B, H]."""
    b, h, cap = c0["positions"].shape
    for i in range(b):
        for g in range(h):
            n = int(np.clip(c0["lengths"][i, g], 0, cap))
            to, frm, left = q4.evict(c0["positions"][i, g, :n], c0["weights"][i, g, :n],
                                     int(budgets[i, g]), sinks, recent)
            assert c1["lengths"][i, g] == (left if left < n else c0["lengths"][i, g])
            for name in BYTES[:-1]:
                want = c0[name][i, g].copy()
                want[to] = want[frm]
                # slots behind the new length are free
                assert np.array_equal(want[:left], c1[name][i, g, :left],
                                      equal_nan=want.dtype.kind == "f"), (i, g, name)


@pytest.mark.parametrize("n,budget,sinks,recent", [
    (40, 39, 0, 0), (40, 32, 4, 8), (1025, 1024, 4, 32), (1152, 1024, 0, 0), (700, 0, 0, 0),
    (700, 1, 1, 0), (700, 36, 4, 32), (3000, 1500, 4, 100), (33000, 16500, 4, 32), (64, 64, 1, 1),
    (300, 299, 299, 0)])
def test_evict(cuda_device, n, budget, sinks, recent):
    gen = torch.Generator().manual_seed(n)
    c = random_cache(2, 2, n, [[n, max(n - 7, 0)], [n // 2, 0]], cuda_device, gen)
    w0 = host(c)
    ws = ckv.q4_workspace(c)
    ckv.q4_evict(c, budget, ws, sinks=sinks, recent=recent)
    assert ckv.read_device_status(ws) == 0
    check_evict(w0, host(c), np.full((2, 2), budget), sinks, recent)


@pytest.mark.parametrize("n", [2000, 5000])
@pytest.mark.parametrize("kind", ["ties", "equal", "zeros", "nan", "inf", "negative", "close"])
def test_evict_weights(cuda_device, kind, n):
    gen = torch.Generator().manual_seed(3)
    c = random_cache(1, 3, n, [[n, n - 1, 77]], cuda_device, gen)
    w = torch.rand((1, 3, c.capacity), generator=gen)
    w = {"ties": (w * 4).floor(), "equal": torch.full_like(w, 0.25),
         "zeros": torch.where(w < 0.5, 0.0, -0.0), "nan": torch.where(w < 0.3, float("nan"), w),
         "inf": torch.where(w < 0.1, float("inf"), torch.where(w < 0.2, float("-inf"), w)),
         "negative": w - 0.5, "close": 1 + (w * 8).floor() * 2.0 ** -23}[kind]
    c.weights.copy_(w)
    for budget in (n * 3 // 4, 60):
        c0 = host(c)
        ckv.q4_evict(c, budget, ckv.q4_workspace(c), sinks=3, recent=20)
        check_evict(c0, host(c), np.full((1, 3), budget), 3, 20)


@pytest.mark.parametrize("units,n", [(80, 5000), (2, 210001), (80, 26001), (20, 9000), (1, 26000),
                                     (80, 1250), (3, 70000), (80, 9000)])
def test_evict_of_long_units(cuda_device, units, n):
    """Units that a CTA or a cluster of them holds in shared memory, or does not
    (the first and the last unit are compared)."""
    gen = torch.Generator(device=cuda_device).manual_seed(n)
    c = blank(units, 1, n, cuda_device)
    for part in ("k", "v"):
        getattr(c, part + "_codes").random_(0, 256, generator=gen)
        getattr(c, part + "_params").normal_(generator=gen)
    order = torch.rand((units, 1, c.capacity), generator=gen, device=cuda_device)
    order[:, :, n:] = 2
    c.positions.copy_(order.argsort(-1).int())
    c.weights.copy_((torch.rand((units, 1, c.capacity), generator=gen, device=cuda_device) * 500).floor())
    c.lengths.fill_(n)
    c.lengths[-1] = n - 37
    pick = [0, units - 1]
    c0 = {k: v[pick] for k, v in host(c).items()}
    budget, recent = n // 3, n // 25
    ckv.q4_evict(c, budget, ckv.q4_workspace(c), sinks=5, recent=recent)
    check_evict(c0, {k: v[pick] for k, v in host(c).items()}, np.full((2, 1), budget), 5, recent)


def test_evict_budgets_per_unit(cuda_device):
    gen = torch.Generator().manual_seed(5)
    c = random_cache(3, 4, 500, 500, cuda_device, gen)
    c.lengths[1, 2] = 9999
    b = torch.randint(-2, 560, (3, 4), generator=gen).int()
    b[0, 0], b[0, 1] = 0, 3     # below the protected slots
    c0 = host(c)
    ckv.q4_evict(c, b.to(cuda_device), ckv.q4_workspace(c), sinks=8, recent=8)
    check_evict(c0, host(c), b.numpy(), 8, 8)


def test_evict_as_a_sliding_window_with_sinks(cuda_device):
    """budget = sinks + recent: the first tokens and the newest, whatever the weights."""
    gen = torch.Generator().manual_seed(6)
    c = random_cache(1, 2, 256, 256, cuda_device, gen)
    c.positions.copy_(torch.arange(256, dtype=torch.int32).expand(1, 2, 256))
    ckv.q4_evict(c, 4 + 60, ckv.q4_workspace(c), sinks=4, recent=60)
    want = set(range(4)) | set(range(196, 256))
    for g in range(2):
        assert set(c.positions[0, g, :64].tolist()) == want and int(c.lengths[0, g]) == 64


# ------------------------------------------------------------------ together
def decode_inputs(b, h, group, steps, gen, dtype, dev):
    q = torch.randn((steps, b, h * group, 1, 128), generator=gen).to(dtype).to(dev)
    k = torch.randn((steps, b, h, 128), generator=gen).to(dtype).to(dev)
    v = torch.randn((steps, b, h, 128), generator=gen).to(dtype).to(dev)
    return q, k, v


def test_decode_loop(cuda_device):
    """gather -> (append, attend, evict) steps; every step against the oracle on
    what the cache then holds, the evictions exactly."""
    dev, cfg = cuda_device, wl.get("c1").scaled(dtype="bf16", seq_len=500)
    d = wl.make_layer(cfg, 0)
    q, k, v = d["q_win"].to(dev), d["k"].to(dev), d["v"].to(dev)
    p = ckv.Problem(q, k, d["cu_seqlens"], cfg.window, cfg.pool_width)
    out = ckv.LayerOutputs(p, [128], 128, k.dtype, dev)
    ws = ckv.workspace(p, dev)
    cu_out = ckv.compress_layer(p, q, k, v, d["srh_mask"], [128], out.indices, out.k_out, out.v_out,
                                ws, raw=out.raw)
    c = blank(1, 8, 150, dev)
    ckv.q4_gather(p, c, out.indices, cu_out, k, v, raw=out.raw, ws=ws)
    gen = torch.Generator().manual_seed(1)
    qs, ks, vs = decode_inputs(1, 8, 4, 12, gen, torch.bfloat16, dev)
    ws4 = ckv.q4_workspace(c, 32, 1)
    for t in range(12):
        pos = torch.tensor([500 + t], dtype=torch.int32, device=dev)
        ckv.q4_append(c, ks[t], vs[t], pos)
        run_attend(c, qs[t])
        if t % 3 == 2:
            c0 = host(c)
            ckv.q4_evict(c, 128, ws4, sinks=4, recent=16)
            check_evict(c0, host(c), np.full((1, 8), 128), 4, 16)
            assert (c.lengths == 128).all()


def _step(c, q, k, v, pos, out, lse, ws, budget):
    ckv.q4_append(c, k, v, pos)
    ckv.q4_attend(c, q, out, ws, lse=lse, accumulate=True)
    ckv.q4_evict(c, budget, ws, sinks=2, recent=8)


def test_decode_step_in_a_graph_and_on_a_side_stream(cuda_device):
    """A captured step, replayed with new inputs, gives the bits of eager calls;
    so do eager calls on another stream than the tensors'."""
    dev = cuda_device
    gen = torch.Generator().manual_seed(21)
    lens = [[200, 190], [100, 199]]
    qs, ks, vs = decode_inputs(2, 2, 7, 6, gen, torch.float16, dev)

    def fresh():
        g2 = torch.Generator().manual_seed(22)
        c = random_cache(2, 2, 256, lens, dev, g2)
        for n in ("k_codes", "v_codes"):
            getattr(c, n)[:, :, 200:] = 0
        return c

    def eager(c):
        ws = ckv.q4_workspace(c, 14, 1)
        got = []
        for t in range(6):
            pos = torch.full((2,), 1000 + t, dtype=torch.int32, device=dev)
            out, lse = torch.empty_like(qs[t]), torch.empty((2, 14, 1), device=dev)
            _step(c, qs[t], ks[t], vs[t], pos, out, lse, ws, 198)
            got.append((out, lse))
        return got

    c0 = fresh()
    want = eager(c0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c1 = fresh()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = eager(c1)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for (a, b), (x, y) in zip(want, got):
        assert torch.equal(a.view(torch.int16), x.view(torch.int16)) and torch.equal(b, y)
    c2 = fresh()
    ws = ckv.q4_workspace(c2, 14, 1)
    q, k, v = qs[0].clone(), ks[0].clone(), vs[0].clone()
    pos = torch.full((2,), 1000, dtype=torch.int32, device=dev)
    out, lse = torch.empty_like(q), torch.empty((2, 14, 1), device=dev)
    scratch = fresh()
    _step(scratch, q, k, v, pos, out, lse, ckv.q4_workspace(scratch, 14, 1), 198)  # first use is eager
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(c2, q, k, v, pos, out, lse, ws, 198)
    for t in range(6):
        q.copy_(qs[t])
        k.copy_(ks[t])
        v.copy_(vs[t])
        pos.fill_(1000 + t)
        graph.replay()
        assert torch.equal(out.view(torch.int16), want[t][0].view(torch.int16))
        assert torch.equal(lse, want[t][1])
    for n in BYTES:
        a, b = getattr(c0, n), getattr(c2, n)
        for i in range(2):
            for g in range(2):
                m = int(c0.lengths[i, g]) if n != "lengths" else None
                x, y = (a, b) if m is None else (a[i, g, :m], b[i, g, :m])
                assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)), n


def test_two_calls_at_once(cuda_device):
    """Two layers of a packed cache on two streams, each with its own workspace."""
    dev = cuda_device
    gen = torch.Generator().manual_seed(31)
    c = random_cache(2, 4, 4000, 4000, dev, gen)
    q = torch.randn((2, 16, 1, 128), generator=gen).bfloat16().to(dev)
    want = torch.empty_like(q)
    w0 = c.weights.clone()
    ckv.q4_attend(c, q, want, ckv.q4_workspace(c, 16, 1), accumulate=True)
    w1 = c.weights.clone()
    c.weights.copy_(w0)
    parts = [c.sequences(i, 1) for i in range(2)]
    wss = [ckv.q4_workspace(x, 16, 1) for x in parts]
    outs = [torch.empty_like(q[i:i + 1]) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        ckv.q4_attend(parts[i], q[i:i + 1], outs[i], wss[i], accumulate=True, stream=streams[i])
    torch.cuda.synchronize()
    # another split of the work over the SMs: not the same bits, the same values
    for i in range(2):
        assert torch.allclose(outs[i].float(), want[i:i + 1].float(), rtol=2.0 ** -7, atol=1e-3)
        assert torch.allclose(c.weights[i], w1[i], rtol=1e-4, atol=1e-6)


def test_layers_packed_in_one_cache(cuda_device):
    """A layer's block of a packed cache gives what a cache of its own gives."""
    dev = cuda_device
    gen = torch.Generator().manual_seed(41)
    c = random_cache(6, 2, 300, 280, dev, gen)
    part = c.sequences(2, 2)
    own = ckv.Q4Cache(*(getattr(part, n).clone() for n in BYTES[:5]), part.lengths.clone(),
                      part.weights.clone())
    before = bits(c)
    q = torch.randn((2, 4, 1, 128), generator=gen).half().to(dev)
    k = torch.randn((2, 2, 128), generator=gen).half().to(dev)
    pos = torch.full((2,), 900, dtype=torch.int32, device=dev)
    got = []
    for x in (part, own):
        out, lse = torch.empty_like(q), torch.empty((2, 4, 1), device=dev)
        ws = ckv.q4_workspace(x, 4, 1)
        ckv.q4_append(x, k, k, pos)
        ckv.q4_attend(x, q, out, ws, lse=lse, accumulate=True)
        ckv.q4_evict(x, 200, ws, sinks=1, recent=5)
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    for n in BYTES:
        a = getattr(c, n).view(torch.uint8)
        assert torch.equal(a[2:4], getattr(own, n).view(torch.uint8)), n
        assert torch.equal(a[:2], before[n][:2]) and torch.equal(a[4:], before[n][4:]), n


def test_trace_names_the_kernels(cuda_device):
    dev = cuda_device
    t = ckv.Trace(16)
    c = ckv.q4_cache(1, 2, 64, dev, trace=t)
    k = torch.randn((1, 2, 128), device=dev).half()
    pos = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = ckv.q4_workspace(c, 2, 1)
    q = torch.randn((1, 2, 1, 128), device=dev).half()
    ckv.q4_append(c, k, k, pos)
    ckv.q4_attend(c, q, torch.empty_like(q), ws)
    ckv.q4_evict(c, 0, ws)
    torch.cuda.synchronize()
    names = [n for n, _ in t.records()]
    assert names[0] == "q4_write" and "q4_attend" in names and names[-1] == "q4_evict"
    assert t.launches == len(names)


def test_refuses_tensors_of_another_device(cuda_device):
    c = ckv.q4_cache(1, 2, 64, cuda_device)
    ws = ckv.q4_workspace(c, 2, 1)
    k = torch.randn((1, 2, 128)).half()
    pos = torch.zeros(1, dtype=torch.int32)
    q = torch.randn((1, 2, 1, 128)).half()
    for call in (lambda: ckv.q4_append(c, k, k, pos.to(cuda_device)),
                 lambda: ckv.q4_append(c, k.to(cuda_device), k, pos.to(cuda_device)),
                 lambda: ckv.q4_attend(c, q, q, ws),
                 lambda: ckv.q4_evict(c, torch.zeros((1, 2), dtype=torch.int32), ws),
                 lambda: ckv.q4_attend(c, q.to(cuda_device), q.to(cuda_device), ws.cpu())):
        with pytest.raises(ckv.CompressKVError) as e:
            call()
        assert e.value.code == B.CKV_ERR_INVALID_ARG


def test_scores_of_the_values_that_an_append_returns(cuda_device):
    """A scoring call right behind an append reads the append's k_values."""
    dev, cfg = cuda_device, wl.get("c1").scaled(dtype="bf16", seq_len=3001)
    d = wl.make_layer(cfg, 0)
    q, k, v = d["q_win"].to(dev), d["k"].to(dev), d["v"].to(dev)
    pos = torch.arange(3001, dtype=torch.int32, device=dev)
    c = ckv.q4_cache(1, 8, 3001, dev)
    kv, vv = torch.zeros_like(k), torch.zeros_like(v)
    p = ckv.Problem(q, kv, d["cu_seqlens"], cfg.window, cfg.pool_width)
    ws = ckv.workspace(p, dev)
    raw = torch.empty((8, 3001 - cfg.window), device=dev)

    def step(wait):
        kv.zero_()
        ckv.q4_append(c, k, v, pos, start=torch.zeros_like(c.lengths), k_values=kv, v_values=vv)
        if wait:
            torch.cuda.synchronize()
        ckv.score(p, q, kv, d["srh_mask"], raw, ws)
        return raw.clone()

    want = step(True)
    for _ in range(5):
        assert torch.equal(step(False), want)


def test_values_in_page_locked_host_memory(cuda_device):
    """V rows that the device reads over the host link."""
    gen = torch.Generator().manual_seed(51)
    k = torch.randn((5, 2, 128), generator=gen).half()
    v = torch.randn((5, 2, 128), generator=gen).half()
    c = blank(1, 2, 32, cuda_device)
    ckv.q4_append(c, k.to(cuda_device), v.pin_memory(), torch.arange(5, dtype=torch.int32, device=cuda_device))
    new = host(c)
    for g in range(2):
        check_rows(new, 0, g, slice(0, 5), k[:, g].float().numpy(), v[:, g].float().numpy())
