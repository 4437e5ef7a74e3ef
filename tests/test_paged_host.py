"""Rotary tables, and the arguments that the rotary and paged-cache calls refuse
before any launch (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from oracle import paged_oracle as po
from paper_2606_24467_gb300 import compresskv as B

OK, BAD, NOT, WS = B.CKV_OK, B.CKV_ERR_INVALID_ARG, B.CKV_ERR_UNSUPPORTED, B.CKV_ERR_WORKSPACE
AT = 1 << 30  # an address that no call reads before its launch


def refused(code, call, *args, **kw):
    with pytest.raises(ckv.CompressKVError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


# ------------------------------------------------------------------- rotary
def test_frequencies():
    i = np.arange(64)
    plain = ckv.rope_frequencies(128, 10000.0)
    np.testing.assert_allclose(plain, 10000.0 ** (-i / 64), rtol=1e-14)
    np.testing.assert_allclose(ckv.rope_frequencies(128, 10000.0, "linear", 8.0), plain / 8, rtol=1e-14)
    base = ckv.rope_frequencies(128, 10000.0, "base", 8.0)
    assert base[0] == 1.0 and abs(base[-1] * 8 / plain[-1] - 1) < 1e-12  # shortest wave, longest wave
    waves = ckv.rope_frequencies(128, 10000.0, "waves", 8.0, 8192.0, 1.0, 4.0)
    turns = 8192 * plain / (2 * np.pi)
    np.testing.assert_allclose(waves[turns >= 4], plain[turns >= 4], rtol=1e-14)
    np.testing.assert_allclose(waves[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and ((waves < plain) & (waves > plain / 8))[mid].all()
    ramp = ckv.rope_frequencies(128, 10000.0, "ramp", 4.0, 4096.0, 1.0, 32.0)
    turns = 4096 * plain / (2 * np.pi)
    first, last = np.searchsorted(-turns, [-32.0, -1.0])  # the first pairs with no more turns than that
    np.testing.assert_allclose(ramp[:first], plain[:first], rtol=1e-14)
    np.testing.assert_allclose(ramp[last:], plain[last:] / 4, rtol=1e-14)
    keep = (ramp / plain - 0.25) / 0.75
    step = -np.diff(keep[first:last])
    assert (step > 0).all() and np.allclose(step[:-1], step[0], rtol=1e-9)
    f = np.linspace(0.1, -0.3, 8)
    np.testing.assert_array_equal(ckv.Rope(16, frequencies=f).frequencies, f)


def test_table_holds_turns():
    f = np.array([1.0, 0.0, -1.0, 2 * np.pi, 1e-6, 100.0, 2.0 ** 20, -1e-300])
    r = ckv.Rope(16, frequencies=f, scale=0.5, interleaved=True)
    turns = [int(x) for x in r.struct.turns[:8]]
    for x, t in zip(f, turns):
        want = (x / (2 * np.pi)) % 1.0
        gap = abs(t / 2.0 ** 64 - want)
        assert min(gap, 1 - gap) < 2.0 ** -50
    assert r.struct.scale == 0.5 and r.struct.interleaved == 1 and r.struct.rot_dim == 16


def test_bad_tables_are_refused():
    for rot in (0, 1, 3, 130, -2):
        refused(BAD, ckv.rope_frequencies, rot)
        refused(BAD, ckv.Rope, rot)
    for base in (0.0, -1.0, float("nan"), float("inf")):
        refused(BAD, ckv.rope_frequencies, 128, base)
    for factor in (0.5, float("nan"), float("inf")):
        refused(BAD, ckv.rope_frequencies, 128, 1e4, "linear", factor)
    refused(BAD, ckv.rope_frequencies, 2, 1e4, "base", 2.0)
    for kw in (dict(original_length=0.0), dict(original_length=8192.0, low=4.0, high=4.0),
               dict(original_length=8192.0, low=0.0), dict(original_length=float("nan"))):
        refused(BAD, ckv.rope_frequencies, 128, 1e4, "waves", 2.0, **kw)
    refused(BAD, ckv.rope_frequencies, 128, 1.0, "ramp", 2.0, 4096.0)
    refused(BAD, ckv.rope_frequencies, 128, 1e4, "other")
    refused(BAD, ckv.Rope, 16, frequencies=np.ones(7))
    for f in (np.nan, np.inf, 2.0 ** 21):
        refused(BAD, ckv.Rope, 2, frequencies=np.array([f]))
    for scale in (float("nan"), float("inf"), 1e39):
        refused(BAD, ckv.Rope, 128, scale=scale)
    refused(BAD, ckv.Rope, 2 ** 32 + 128)


def rope_code(rope=None, q=AT, k=AT, q_out=AT, k_out=AT, positions=AT, **kw):
    x = B.CkvRopeRows(4, 3, 2, B.CKV_DTYPE_BF16, 0, 0, 384, 128, 256, 128, 384, 128, 256, 128)
    for name, value in kw.items():
        setattr(x, name, value)
    r = rope or ckv.Rope(128)
    return ckv.load().compresskv_rope_apply(r.addr, ctypes.addressof(x), positions, q, k, q_out, k_out, None)


def test_rope_apply_refusals():
    for kw in (dict(rows=-1), dict(dtype=2), dict(num_q_heads=-1), dict(q_token_stride=380),
               dict(q_head_stride=-128), dict(q=None), dict(q_out=None), dict(k=AT + 2), dict(positions=None),
               dict(positions=AT + 2), dict(k_out_head_stride=120), dict(q_out_token_stride=0),
               dict(num_k_heads=0), dict(q_token_stride=1 << 45),
               dict(q_out=AT + 256),                       # its input, moved by a head
               dict(q_out_token_stride=512)):              # in place, but with another stride
        assert rope_code(**kw) == BAD, kw
    assert rope_code(num_q_heads=257) == NOT
    assert rope_code(rows=0) == OK
    r = ckv.Rope(128)
    r.struct.rot_dim = 7
    assert rope_code(r) == BAD
    assert ckv.load().compresskv_rope_apply(None, None, None, None, None, None, None, None) == BAD


def test_rope_apply_binding():
    rope, pos = ckv.Rope(128), torch.zeros(4, dtype=torch.int32)
    q = torch.zeros(4, 2, 128, dtype=torch.float16)
    refused(BAD, ckv.rope_apply, rope, pos, q)                         # host memory
    refused(BAD, ckv.rope_apply, rope, pos.long(), q)
    refused(BAD, ckv.rope_apply, rope, pos[:3], q)
    refused(BAD, ckv.rope_apply, rope, pos, q.float())
    refused(BAD, ckv.rope_apply, rope, pos, q, q.bfloat16())
    refused(BAD, ckv.rope_apply, rope, pos, q[..., :64])
    refused(BAD, ckv.rope_apply, rope, pos, q, None, torch.zeros(4, 3, 128, dtype=torch.float16))
    refused(BAD, ckv.rope_apply, rope, pos, q, None, None, q)


# -------------------------------------------------------------------- cache
def cache_struct(**kw):
    c = B.CkvPagedCache(2, 2, 128, B.CKV_DTYPE_F16, 16, 10, 4, 0, AT, 2 * AT, 16 * 256, 256, 128, 3 * AT, 4,
                        3 * AT + 4096)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


BAD_CACHES = [(BAD, dict(batch=0)), (BAD, dict(num_kv_heads=0)), (BAD, dict(dtype=2)), (BAD, dict(page_size=8)),
              (BAD, dict(page_size=24)), (BAD, dict(page_size=512)), (BAD, dict(num_pages=0)),
              (BAD, dict(table_width=0)), (NOT, dict(batch=513)), (NOT, dict(head_dim=64)),
              (NOT, dict(num_kv_heads=65)), (NOT, dict(table_width=(1 << 20) + 1, table_stride=1 << 21)),
              (BAD, dict(k_pages=None)), (BAD, dict(v_pages=2 * AT + 8)), (BAD, dict(table=None)),
              (BAD, dict(table=3 * AT + 2)), (BAD, dict(lengths=None)), (BAD, dict(table_stride=3)),
              (BAD, dict(page_stride=128)), (BAD, dict(slot_stride=120)), (BAD, dict(head_stride=0)),
              (BAD, dict(head_stride=-128)), (BAD, dict(slot_stride=128, head_stride=128))]


def append_code(c, k=AT * 8, v=AT * 9, start=None, rope=None, positions=None, q=None, q_out=None, status=None, **kw):
    r = B.CkvPagedRows(3, 0, None, 256, 128, 256, 128, 256, 128)
    for name, value in kw.items():
        setattr(r, name, value)
    return ckv.load().compresskv_paged_append(ctypes.addressof(c), ctypes.addressof(r), k, v, start,
                                              rope.addr if rope else None, positions, q, q_out, status, None)


def attend_code(c, q=AT * 8, out=AT * 9, start=None, lse=None, ws=0, size=0, **kw):
    a = B.CkvPagedQueries(4, 3, None, 1, 0.0, 512, 128, 512, 128)
    for name, value in kw.items():
        setattr(a, name, value)
    return ckv.load().compresskv_paged_attend(ctypes.addressof(c), ctypes.addressof(a), q, start, out, lse,
                                              ws or None, size, None)


@pytest.mark.parametrize("code, kw", BAD_CACHES)
def test_bad_caches_are_refused(code, kw):
    c = cache_struct(**kw)
    assert append_code(c) == code and attend_code(c) == code
    assert ckv.load().compresskv_paged_gather(ctypes.addressof(c), None, 3, None, AT, AT, None, None) == code


def cu(*values):
    a = np.array(values, np.int32)
    return a, a.ctypes.data


def test_append_refusals():
    c, rope = cache_struct(), ckv.Rope(128)
    lengths = 3 * AT + 4096
    down, at_down = cu(0, 5, 3)
    late, at_late = cu(1, 2, 3)
    for kw in (dict(k=None), dict(v=AT + 8), dict(kv_token_stride=100), dict(rows_per_seq=-1), dict(num_q_heads=-1),
               dict(cu_rows=at_down), dict(cu_rows=at_late), dict(q=AT), dict(num_q_heads=2, q=AT, q_out=AT),
               dict(num_q_heads=2, rope=rope), dict(num_q_heads=2, rope=rope, q=AT, q_out=AT + 256),
               dict(start=AT + 1), dict(positions=AT + 3), dict(status=AT + 2),
               dict(start=lengths + 4)):                    # overlaps the lengths without being them
        assert append_code(c, **kw) == BAD, kw
    assert append_code(c, num_q_heads=257, rope=rope) == NOT
    assert append_code(c, rows_per_seq=(1 << 30) + 1) == NOT
    assert append_code(c, rows_per_seq=0) == OK
    assert append_code(c, rows_per_seq=0, start=lengths) == OK


def test_gather_refusals():
    f, c = ckv.load().compresskv_paged_gather, cache_struct()
    at = ctypes.addressof(c)
    assert f(at, None, -1, None, AT, AT, None, None) == BAD
    assert f(at, None, 1, None, AT + 8, AT, None, None) == BAD
    assert f(at, None, 1, AT + 2, AT, AT, None, None) == BAD
    assert f(at, None, 1, None, AT, AT, AT + 1, None) == BAD
    assert f(at, None, 0, None, AT, AT, None, None) == OK
    assert f(at, None, 1, None, None, None, None, None) == OK


def test_attend_refusals():
    c = cache_struct()
    for kw in (dict(num_q_heads=0), dict(num_q_heads=3), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(scale=2.0 ** 97), dict(q=None), dict(out=AT + 8), dict(lse=AT + 2),
               dict(start=AT + 2), dict(q_token_stride=0), dict(q_token_stride=100), dict(out_head_stride=64),
               dict(out_token_stride=0), dict(rows_per_seq=-1), dict(out=AT * 8), dict(out=AT * 8 + 1024)):
        assert attend_code(c, **kw) == BAD, kw
    assert attend_code(c, num_q_heads=258) == NOT and attend_code(c, rows_per_seq=1 << 24, out=AT * 1000) == NOT
    assert attend_code(cache_struct(num_kv_heads=1), num_q_heads=129) == NOT
    assert attend_code(c) == WS and attend_code(c, ws=AT, size=16) == WS
    assert attend_code(c, ws=AT + 128, size=1 << 40) == WS


def test_stall_hook_limits():
    for bad in (-1, 99_999, 2_000_000_001):
        refused(BAD, ckv.debug_stall_next_paged_attend, bad)
    ckv.debug_stall_next_paged_attend(1_000_000)
    ckv.debug_stall_next_paged_attend(0)  # cancelled: no later call stalls


def test_workspace_size():
    f, c = ckv.load().compresskv_paged_workspace_size, cache_struct()
    at = ctypes.addressof(c)
    assert f(at, 4, 1) > 0 and f(at, 4, 0) > 0 and f(at, 4, 1000) >= f(at, 4, 1)
    assert f(at, 3, 1) == 0 and f(at, 0, 1) == 0 and f(at, 4, -1) == 0 and f(None, 4, 1) == 0
    assert f(ctypes.addressof(cache_struct(page_size=17)), 4, 1) == 0
    assert ckv.load().compresskv_paged_workspace_init(None, 1 << 20, None) == WS
    assert ckv.load().compresskv_paged_workspace_init(AT, 16, None) == WS


def test_binding_refusals():
    c = ckv.paged_cache(2, 2, 50, page_size=16, device="cpu")
    assert c.capacity == 64 and c.num_pages == 8 and tuple(c.k_pages.shape) == (8, 16, 2, 128)
    assert c.sequences(1, 1).table.tolist() == [[4, 5, 6, 7]]
    refused(BAD, c.sequences, 1, 2)
    kp, vp, table, lengths = c.k_pages, c.v_pages, c.table, c.lengths
    refused(BAD, ckv.PagedCache, kp.float(), vp, table, lengths)
    refused(BAD, ckv.PagedCache, kp, vp.contiguous(), table, lengths)   # other strides
    refused(BAD, ckv.PagedCache, kp[..., :64], vp[..., :64], table, lengths)
    refused(BAD, ckv.PagedCache, kp, vp, table.long(), lengths)
    refused(BAD, ckv.PagedCache, kp, vp, table.T, lengths)
    refused(BAD, ckv.PagedCache, kp, vp, table, lengths[:1])
    k = torch.zeros(6, 2, 128, dtype=torch.bfloat16)
    q = torch.zeros(6, 4, 128, dtype=torch.bfloat16)
    refused(BAD, ckv.paged_append, c, k, k)                              # host memory
    refused(BAD, ckv.paged_append, c, k[:5], k[:5])
    refused(BAD, ckv.paged_append, c, k, k, [0, 2, 5])
    refused(BAD, ckv.paged_append, c, k.half(), k)
    refused(BAD, ckv.paged_append, c, k, k[:, :1].expand(6, 2, 128))
    refused(BAD, ckv.paged_append, c, k, k, q=q)
    refused(BAD, ckv.paged_append, c, k, k, rope=ckv.Rope(), q_out=q)
    refused(BAD, ckv.paged_append, c, k, k, start=torch.zeros(3, dtype=torch.int32))
    refused(BAD, ckv.paged_gather, c, None)
    refused(BAD, ckv.paged_gather, c, k.transpose(0, 1))
    refused(BAD, ckv.paged_gather, c, k, k[:5])
    refused(BAD, ckv.paged_attend, c, q, q[:, :2], None)
    for scale in (float("nan"), float("inf"), 1e39, -1e39):
        refused(BAD, ckv.paged_attend, c, q, q.clone(), torch.empty(16, dtype=torch.uint8), scale=scale)
    long = torch.zeros(1, 4, 128, dtype=torch.bfloat16).expand(1 << 32, 4, 128)
    refused(BAD, ckv.paged_attend, c, long, long, torch.empty(16, dtype=torch.uint8))
    refused(BAD, ckv.paged_workspace, c, 4, 1)
    refused(BAD, ckv.paged_workspace_size, c, 3, 1)


# ------------------------------------------------------------------- oracle
def test_oracle_rotation_by_hand():
    x = torch.arange(1, 9, dtype=torch.float64).view(1, 1, 8)
    f = np.array([np.pi / 2, np.pi])                       # at position 1: a quarter and half a turn
    pos = torch.tensor([1])
    half = po.rotate(x, pos, f, False)[0, 0]
    torch.testing.assert_close(half, torch.tensor([-3.0, -2, 1, -4, 5, 6, 7, 8], dtype=torch.float64))
    near = po.rotate(x, pos, f, True)[0, 0]
    torch.testing.assert_close(near, torch.tensor([-2.0, 1, -3, -4, 5, 6, 7, 8], dtype=torch.float64))
    back = po.rotate(half.view(1, 1, 8), pos, f, False, backward=True)
    torch.testing.assert_close(back, x)


def test_oracle_attention_by_softmax():
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((3, 4, 128), (7, 2, 128), (7, 2, 128)))
    out, lse, parts = po.attend(q, k, v, 4, True, 0.1)
    z = torch.einsum("nhd,shd->hns", q, k.repeat_interleave(2, 1)) * 0.1
    z = z.masked_fill(torch.arange(7) > 4 + torch.arange(3)[:, None], -float("inf"))
    torch.testing.assert_close(out, torch.einsum("hns,shd->nhd", z.softmax(-1), v.repeat_interleave(2, 1)))
    torch.testing.assert_close(lse, z.logsumexp(-1))
    none, lse, _ = po.attend(q, k, v, -2, True, 0.1)
    assert (none[:2] == 0).all() and torch.isinf(lse[:, :2]).all() and torch.isfinite(lse[:, 2]).all()
