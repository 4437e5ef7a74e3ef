"""Arguments of the 4-bit cache's calls that the library takes or refuses before
any launch (no GPU)."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from paper_2606_24467_gb300 import compresskv as B


def test_stall_hook_limits():
    for bad in (-1, 99_999, 2_000_000_001):
        with pytest.raises(ckv.CompressKVError):
            ckv.debug_stall_next_q4_attend(bad)
    ckv.debug_stall_next_q4_attend(1_000_000)
    ckv.debug_stall_next_q4_attend(0)  # cancelled: no later call stalls


def attend_code(dims, strides):
    """What q4_attend says of an output of these dimensions and strides, with a
    workspace of no bytes (the check that follows the strides')."""
    b, hq, n = dims
    c = ckv.q4_cache(b, 1, 32, device="cpu")
    a = B.CkvQ4Queries(hq, n, B.CKV_DTYPE_BF16, 0, 0.0, 128 * hq * n, 128 * n, 128, *strides)
    return ckv.load().compresskv_q4_attend(c.addr, ctypes.addressof(a), 1 << 30, None, 1 << 30, None,
                                           1 << 30, 0, None)


def overlap(dims, strides):
    at = np.zeros(1, np.int64)
    for n, s in zip(dims, strides):
        at = (at[:, None] + np.arange(n) * s).ravel()
    at.sort()
    return bool((np.diff(at) < 128).any())


@pytest.mark.parametrize("dims", [(1, 1, 1), (3, 1, 1), (1, 4, 2), (2, 4, 1), (2, 4, 3), (5, 6, 2), (40, 3, 2)])
def test_outputs_whose_rows_overlap_are_refused(dims):
    steps = (0, 8, 128, 136, 256, 264, 384, 512, 640, 1024, 1032, 5120, 5248)
    said = {True: 0, False: 0}
    for strides in itertools.product(steps, repeat=3):
        bad = overlap(dims, strides)
        want = B.CKV_ERR_INVALID_ARG if bad else B.CKV_ERR_WORKSPACE
        assert attend_code(dims, strides) == want, strides
        said[bad] += 1
    assert said[False] > 0


def test_output_strides_that_interleave_or_are_far_apart():
    free, bad = B.CKV_ERR_WORKSPACE, B.CKV_ERR_INVALID_ARG
    assert attend_code((2, 2, 1), (128, 256, 8)) == free
    assert attend_code((2, 3, 1), (384, 256, 8)) == free     # 0 256 512 / 384 640 896: side by side
    assert attend_code((3, 4, 1), (384, 256, 8)) == bad      # 768 twice
    assert attend_code((2, 4, 5), (128, 128, 128)) == bad    # each alone would do
    assert attend_code((2, 4, 5), (1 << 44, 1 << 40, 1 << 36)) == free
    assert attend_code((2, 4, 5), ((1 << 44) + 8, 640, 128)) == bad
    assert attend_code((60000, 1, 1), (120, 8, 8)) == bad and attend_code((60000, 1, 1), (128, 8, 8)) == free


def test_rows_whose_strides_differ_where_they_mean_nothing():
    """One row, or one KV head: K and V cut out of different tensors."""
    c = ckv.q4_cache(1, 4, 32, device="cpu")
    k = torch.zeros((1, 4, 128)).bfloat16()
    v = torch.zeros((9, 4, 256)).bfloat16()[::3, :, :128]
    assert B._q4_rows(c, k, v[:1].as_strided((1, 4, 128), (999, 128, 1)))[1] == (1, 4, 128)
    with pytest.raises(ckv.CompressKVError):
        B._q4_rows(c, k, v[:1])  # the heads' strides differ
    one = ckv.q4_cache(1, 1, 32, device="cpu")
    a, b = torch.zeros((5, 1, 128)).half(), torch.zeros((5, 2, 128)).half()[:, :1]
    with pytest.raises(ckv.CompressKVError):
        B._q4_rows(one, a, b)    # the rows' strides differ
    assert B._q4_rows(one, a, a.as_strided((5, 1, 128), (128, 999, 1)))[2] == (128, 128, 1)


def test_numbers_beyond_32_bits_are_refused():
    """(a budget of 2^40 slots would otherwise have been one of 0)"""
    c = ckv.q4_cache(2, 4, 64, device="cpu")
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for kw in ({"budget": 2 ** 40}, {"budget": 10, "sinks": 2 ** 32}, {"budget": 10, "recent": -2 ** 33}):
        with pytest.raises(ckv.CompressKVError, match="32 bits"):
            ckv.q4_evict(c, ws=ws, **kw)
    with pytest.raises(ckv.CompressKVError, match="32 bits"):
        ckv.q4_workspace_size(c, 2 ** 32 + 8, 1)


def test_softmax_scales_that_overflow_are_refused():
    c = ckv.q4_cache(1, 1, 32, device="cpu")
    a = B.CkvQ4Queries(1, 1, B.CKV_DTYPE_BF16, 0, 0.0, 128, 128, 128, 128, 128, 128)
    for scale, code in ((2.0 ** 96, B.CKV_ERR_WORKSPACE), (2.0 ** 97, B.CKV_ERR_INVALID_ARG),
                        (3e38, B.CKV_ERR_INVALID_ARG)):
        a.scale = scale
        assert ckv.load().compresskv_q4_attend(c.addr, ctypes.addressof(a), 1 << 30, None, 1 << 30, None,
                                               1 << 30, 0, None) == code
