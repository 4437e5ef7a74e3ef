"""The 4-bit cache without a GPU: the oracle against exact fractions and closed
forms, and every refusal of the entry points (argument checks come before any
launch)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from oracle import q4_oracle as q4
from paper_2606_24467_gb300 import compresskv as B


# ------------------------------------------------------------------ the oracle
def _bf16_grid():
    """All finite non-negative bf16 numbers, ascending."""
    return (np.arange(0x7F80, dtype=np.uint32) << 16).view(np.float32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", ["normal", "offset", "tiny", "wide"])
def test_oracle_quantisation_against_fractions(dtype, kind):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((6, 128), generator=gen)
    x = {"normal": x, "offset": x * 0.05 + 9, "tiny": x * 1e-6, "wide": x * 300}[kind].to(dtype)
    x[0, 40] = 0.0
    codes, s, m = q4.quantise(x.float().numpy())
    grid = _bf16_grid()
    for row in range(6):
        for J in range(4):
            g = x[row, 32 * J:32 * J + 32].float().numpy()
            lo = g.min()
            # minimum: the largest bf16 not above it
            below = (-grid[::-1])[-grid[::-1] <= lo] if lo < 0 else grid[grid <= lo]
            assert Fraction(float(m[row, J])) == Fraction(float(below.max()))
            top = Fraction(float(np.float32(g.max() - m[row, J])))
            k = int(np.searchsorted(grid.astype(np.float64) * 15, float(top)))
            assert 15 * Fraction(float(grid[k])) >= top > 15 * Fraction(float(grid[k - 1]))
            assert Fraction(float(s[row, J])) == Fraction(float(grid[k]))
            for i in range(32):
                d = Fraction(float(np.float32(g[i] - m[row, J])))
                assert codes[row, 32 * J + i] == round(d / Fraction(float(s[row, J])))  # ties to even
    assert codes.min() >= 0 and codes.max() <= 15


def test_oracle_quantisation_of_constant_and_non_finite_groups():
    x = np.zeros((1, 128), np.float32)
    x[0, :32] = 2.5
    x[0, 40] = np.nan
    x[0, 70] = -np.inf
    codes, s, m = q4.quantise(x)
    assert s[0, 0] == 0 and m[0, 0] == 2.5 and not codes[0, :32].any()
    assert np.isnan(s[0, 1:3]).all() and np.isnan(m[0, 1:3]).all()
    assert s[0, 3] == 0 and m[0, 3] == 0
    back = q4.values(codes, s, m)
    assert (back[0, :32] == 2.5).all() and np.isnan(back[0, 32:96]).all() and not back[0, 96:].any()


def test_oracle_packing():
    codes = np.arange(256).reshape(2, 128) % 16
    packed = q4.pack(codes)
    assert packed.shape == (2, 64) and packed[0, 0] == 0x10
    assert np.array_equal(q4.unpack(packed), codes)


def test_oracle_attention_against_torch():
    gen = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((n, 128), generator=gen, dtype=torch.float64) for n in (3, 40, 40))
    vis = np.ones((3, 40), bool)
    vis[1, 5:] = False
    vis[2] = False
    k[39] = float("nan")
    vis[:, 39] = False
    out, lse, p = q4.attend(q.numpy(), k.numpy(), v.numpy(), vis, 0.1)
    for r, n in ((0, 39), (1, 5)):
        z = 0.1 * (k[:n] @ q[r])
        assert np.allclose(out[r], (z.softmax(0) @ v[:n]).numpy(), atol=1e-12)
        assert np.isclose(lse[r], float(z.logsumexp(0)), atol=1e-12)
        assert np.isclose(p[r].sum(), 1)
    assert not out[2].any() and lse[2] == -np.inf and not p[2].any()


def test_oracle_eviction_by_hand():
    #        slot      0  1  2  3  4  5  6
    pos = np.array([10, 0, 11, 3, 12, 5, 13])
    w = np.array([.5, 0, np.nan, .5, 9, .2, 0])
    # sink: slot 1; recent (two newest): slots 4, 6; then weights: .5 (slot 0), .5 (slot 3), .2, NaN
    to, frm, n = q4.evict(pos, w, 4, 1, 2)
    assert n == 4 and to.tolist() == [2, 3] and frm.tolist() == [4, 6]
    assert q4.evict(pos, w, 7, 1, 2)[2] == 7 and q4.evict(pos, w, -1, 1, 2)[2] == 7
    to, frm, n = q4.evict(pos, w, 0, 0, 0)
    assert n == 0 and to.size == 0


# ------------------------------------------------------------------ refusals
def _cache(b=2, h=4, cap=64, **kw):
    return ckv.q4_cache(b, h, cap, device="cpu", **kw)


def _refused(code, fn, *a, **kw):
    with pytest.raises(ckv.CompressKVError) as e:
        fn(*a, **kw)
    assert e.value.code == code


def test_cache_tensors_are_checked():
    c = _cache()
    t = {n: getattr(c, n) for n in ("k_codes", "v_codes", "k_params", "v_params", "positions",
                                    "lengths", "weights")}
    ckv.Q4Cache(**t)
    for name, bad in (("k_codes", t["k_codes"].view(torch.int8)), ("v_codes", t["v_codes"][:, :, :32]),
                      ("k_params", t["k_params"].float()), ("v_params", t["v_params"][..., :4]),
                      ("positions", t["positions"].long()), ("lengths", t["lengths"].T),
                      ("weights", t["weights"].double()), ("k_codes", t["k_codes"][0])):
        _refused(B.CKV_ERR_INVALID_ARG, ckv.Q4Cache, **{**t, name: bad})
    assert _cache(cap=33).capacity == 64
    part = c.sequences(1, 1)
    assert part.k_codes.data_ptr() == c.k_codes[1].data_ptr() and part.batch == 1
    _refused(B.CKV_ERR_INVALID_ARG, c.sequences, 1, 2)
    _refused(B.CKV_ERR_INVALID_ARG, c.sequences, -1, 1)


def test_workspace_size():
    c = _cache()
    rows = 2 * 32
    assert ckv.q4_workspace_size(c, 32, 1) >= rows * 4
    assert ckv.q4_workspace_size(c, 32, 16) > ckv.q4_workspace_size(c, 32, 1)
    assert ckv.q4_workspace_size(c) >= 256
    for hq, n in ((30, 1), (32, 17), (32, 0), (0, 1), (512, 1), (-4, 1)):
        _refused(B.CKV_ERR_INVALID_ARG, ckv.q4_workspace_size, c, hq, n)
    for field, value in (("capacity", 40), ("capacity", 0), ("capacity", 1 << 25), ("batch", 0),
                         ("batch", 20000), ("num_kv_heads", 65), ("head_dim", 64)):
        old = getattr(c.struct, field)
        setattr(c.struct, field, value)
        _refused(B.CKV_ERR_INVALID_ARG, ckv.q4_workspace_size, c)
        setattr(c.struct, field, old)


def test_append_refusals():
    c = _cache()
    k = torch.zeros((6, 4, 128), dtype=torch.bfloat16)
    pos = torch.zeros(6, dtype=torch.int32)
    bad = B.CKV_ERR_INVALID_ARG
    _refused(bad, ckv.q4_append, c, k.float(), k.float(), pos)
    _refused(bad, ckv.q4_append, c, k, k.half(), pos)
    _refused(bad, ckv.q4_append, c, k[:, :2], k[:, :2], pos)
    _refused(bad, ckv.q4_append, c, k, k.transpose(0, 1).contiguous().transpose(0, 1), pos)
    _refused(bad, ckv.q4_append, c, k, k, pos.long())
    _refused(bad, ckv.q4_append, c, k, k, pos[:4])
    _refused(bad, ckv.q4_append, c, k[:5], k[:5], pos[:5])           # 5 rows of 2 sequences
    _refused(bad, ckv.q4_append, c, k, k, pos, cu_rows=[0, 3])
    _refused(bad, ckv.q4_append, c, k, k, pos, cu_rows=[0, 3, 5])
    _refused(bad, ckv.q4_append, c, k, k, pos, start=torch.zeros(2, dtype=torch.int32))
    _refused(bad, ckv.q4_append, c, k, k, pos, k_values=k.float())
    _refused(bad, ckv.q4_append, c, k, k, pos)                       # not in device memory


def _rows(**kw):
    r = B.CkvQ4Rows(B.CKV_DTYPE_BF16, 3, None, 512, 128)
    for n, v in kw.items():
        setattr(r, n, v)
    return ctypes.addressof(r), r


def test_append_refusals_of_the_library():
    c = _cache()
    lib = ckv.load()
    fake = 1 << 30

    def call(r=None, k=fake, v=fake, pos=fake, cache=c, values=None):
        at, keep = r or _rows()
        return lib.compresskv_q4_append(cache.addr, at, k, v, pos, None, values, None, None, None)

    bad = B.CKV_ERR_INVALID_ARG
    assert call(_rows(dtype=2)) == bad
    assert call(_rows(rows_per_seq=-1)) == bad
    assert call(_rows(token_stride=100)) == bad and call(_rows(head_stride=0)) == bad
    assert call(k=None) == bad and call(pos=None) == bad and call(k=fake + 8) == bad
    assert call(values=fake + 4) == bad
    cu = np.array([0, 4, 2], np.int32)
    assert call(_rows(cu_rows=cu.ctypes.data)) == bad
    cu1 = np.array([1, 2, 3], np.int32)
    assert call(_rows(cu_rows=cu1.ctypes.data)) == bad
    wide = _cache(b=600, h=1, cap=32)
    cu = np.arange(601, dtype=np.int32)
    assert call(_rows(cu_rows=cu.ctypes.data), cache=wide) == B.CKV_ERR_UNSUPPORTED
    assert call(_rows(rows_per_seq=0)) == B.CKV_OK  # nothing to do: no CUDA call
    old = c.struct.k_codes
    c.struct.k_codes = None
    assert call() == bad
    c.struct.k_codes = old + 8
    assert call() == bad
    c.struct.k_codes = old


def test_gather_refusals():
    c = _cache()
    cu = [0, 100, 150]
    k = torch.zeros((150, 4, 128), dtype=torch.float16)
    q = torch.zeros((2, 8, 32, 128), dtype=torch.float16)
    p = ckv.Problem(q, k, cu, 32, 7)
    idx = torch.zeros((4, 90), dtype=torch.int32)
    bad = B.CKV_ERR_INVALID_ARG
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 50, 91], k, k)       # indices of 90 rows
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 90], k, k)
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 50, 90], k.bfloat16(), k.bfloat16())
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 50, 90], k[:140], k[:140])
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 50, 90], k, k, raw=torch.zeros((4, 7)))
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 50, 90], k, k, k_values=torch.zeros_like(k))
    _refused(bad, ckv.q4_gather, p, _cache(b=3), idx, [0, 50, 90], k, k)
    _refused(bad, ckv.q4_gather, p, c, idx, [0, 50, 90], k, k)       # not in device memory
    lib = ckv.load()

    def call(cu_out, cache=c, group=0, ws=None, kk=1 << 30):
        a = np.asarray(cu_out, np.int32)
        return lib.compresskv_q4_gather(
            p.ref, cache.addr, group, 1 << 30, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), kk,
            1 << 30, None, None, None, ws, None)

    assert call([0, 65, 90]) == bad                   # more than the capacity
    assert call([0, 50, 110]) == bad                  # more than the sequence (50)
    assert call([0, 50, 40]) == bad and call([1, 50, 90]) == bad
    assert call([0, 50, 90], ws=(1 << 30) + 4) == B.CKV_ERR_WORKSPACE
    assert call([0, 50, 90], cache=_cache(h=2)) == bad
    assert call([0, 50, 90], kk=None) == bad
    assert call([0, 5, 9] * 4, group=1) == bad        # group 1 does not begin where group 0 ends


def test_attend_refusals():
    c = _cache()
    q = torch.zeros((2, 8, 5, 128), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    bad = B.CKV_ERR_INVALID_ARG
    _refused(bad, ckv.q4_attend, c, q[0], q[0], ws)
    _refused(bad, ckv.q4_attend, c, q, q[:, :4], ws)
    _refused(bad, ckv.q4_attend, c, q, q.half(), ws)
    _refused(bad, ckv.q4_attend, c, q.float(), q.float(), ws)
    _refused(bad, ckv.q4_attend, c, q, q, ws, q_positions=torch.zeros((2, 2), dtype=torch.int32))
    _refused(bad, ckv.q4_attend, c, q, q, ws, lse=torch.zeros((2, 8)))
    _refused(bad, ckv.q4_attend, c, q, q, ws)                        # not in device memory
    lib = ckv.load()

    def call(cache=c, ws=1 << 30, n=1 << 30, q=1 << 30, **kw):
        a = B.CkvQ4Queries(8, 5, B.CKV_DTYPE_BF16, 0, 0.0, 5120, 640, 128, 5120, 640, 128)
        for f, v in kw.items():
            setattr(a, f, v)
        return lib.compresskv_q4_attend(cache.addr, ctypes.addressof(a), q, None, 1 << 30, None, ws, n,
                                        None)

    assert call(num_q_heads=6) == bad and call(num_queries=0) == bad and call(dtype=7) == bad
    assert call(num_queries=17) == B.CKV_ERR_UNSUPPORTED
    assert call(num_q_heads=260) == B.CKV_ERR_UNSUPPORTED
    assert call(num_q_heads=256, num_queries=5) == B.CKV_ERR_UNSUPPORTED  # 320 rows a unit
    assert call(scale=-1.0) == bad and call(scale=float("inf")) == bad and call(scale=float("nan")) == bad
    assert call(q=None) == bad and call(q=(1 << 30) + 8) == bad
    assert call(q_head_stride=100) == bad and call(out_query_stride=0) == bad
    assert call(out_head_stride=64) == bad and call(out_batch_stride=-128) == bad
    assert call(cache=_cache(weights=False), accumulate=1) == bad
    assert call(ws=None) == B.CKV_ERR_WORKSPACE and call(ws=(1 << 30) + 16) == B.CKV_ERR_WORKSPACE
    assert call(n=256) == B.CKV_ERR_WORKSPACE


def test_evict_refusals():
    c = _cache()
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    _refused(B.CKV_ERR_INVALID_ARG, ckv.q4_evict, c, 10, ws)         # not in device memory
    _refused(B.CKV_ERR_INVALID_ARG, ckv.q4_evict, c, torch.zeros(2, dtype=torch.int32), ws)
    lib = ckv.load()

    def call(cache=c, budget=10, sinks=0, recent=0, ws=1 << 30, n=1 << 30):
        return lib.compresskv_q4_evict(cache.addr, budget, None, sinks, recent, ws, n, None)

    assert call(budget=-1) == B.CKV_ERR_INVALID_ARG and call(sinks=-1) == B.CKV_ERR_INVALID_ARG
    assert call(recent=-5) == B.CKV_ERR_INVALID_ARG
    assert call(sinks=4, recent=7) == B.CKV_ERR_BUDGET
    assert call(recent=2 ** 31 - 1, sinks=2 ** 31 - 1) == B.CKV_ERR_BUDGET
    assert call(cache=_cache(weights=False)) == B.CKV_ERR_INVALID_ARG
    assert call(n=300) == B.CKV_ERR_WORKSPACE and call(ws=None) == B.CKV_ERR_WORKSPACE
    assert lib.compresskv_q4_workspace_init(None, 1 << 20, None) == B.CKV_ERR_WORKSPACE
    assert lib.compresskv_q4_workspace_init(1 << 30, 100, None) == B.CKV_ERR_WORKSPACE
