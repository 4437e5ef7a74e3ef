"""Outputs of the rotary and paged-cache calls that share memory with another tensor of
the call are refused before any launch (no GPU)."""
import ctypes

import pytest

import paper_2606_24467_gb300 as ckv
from paper_2606_24467_gb300 import compresskv as B

OK, BAD = B.CKV_OK, B.CKV_ERR_INVALID_ARG
AT, ROW = 1 << 30, 256  # an address that no call reads before its launch; bytes of a row


def rope_code(q, k, q_out, k_out, token, rows=4, hq=3, hk=2, k_token=None, head=128):
    """All strides alike, but K's token stride where given."""
    kt = token if k_token is None else k_token
    x = B.CkvRopeRows(rows, hq, hk, B.CKV_DTYPE_BF16, 0, 0, token, head, kt, head, token, head, kt, head)
    return ckv.load().compresskv_rope_apply(ckv.Rope(128).addr, ctypes.addressof(x), AT, q, k, q_out, k_out, None)


@pytest.mark.parametrize("q, k, q_out, k_out, kw", [
    (0, 0, 0, 0, dict(token=384)),                      # one tensor for both, in place
    (0, 100, 0, 101, dict(token=384)),                  # (k_out meets its input)
    (0, 2, 0, 2, dict(token=640)),                      # q's last head is k's first
    (0, 5 * 4 + 2, 0, 5 * 4 + 2, dict(token=640)),      # only of the last token
    (0, 100, 200, 201, dict(token=384)),                # the two outputs
    (0, 100, 101, 200, dict(token=384)),                # q_out over k
    (0, 100, 200, 1, dict(token=384)),                  # k_out over q
    (0, 1, 0, 1, dict(token=2048, head=128)),           # wide tokens
    (0, 2, 0, 2, dict(token=384, k_token=256, rows=1)),  # one row: the token strides mean nothing
])
def test_rotary_outputs_that_meet_are_refused(q, k, q_out, k_out, kw):
    assert rope_code(*(AT + ROW * x for x in (q, k, q_out, k_out)), **kw) == BAD


def append_code(k, v, q_out, kv_token, q_token, rows=2):
    c = B.CkvPagedCache(2, 2, 128, B.CKV_DTYPE_F16, 16, 10, 4, 0, AT, 2 * AT, 16 * 256, 256, 128, 3 * AT, 4,
                        3 * AT + 4096)
    r = B.CkvPagedRows(rows, 3, None, kv_token, 128, q_token, 128, q_token, 128)
    return ckv.load().compresskv_paged_append(ctypes.addressof(c), ctypes.addressof(r), 8 * AT + ROW * k,
                                              8 * AT + ROW * v, None, ckv.Rope(128).addr, None, 8 * AT + ROW * q_out,
                                              8 * AT + ROW * q_out, None, None)


def test_appended_queries_that_meet_rows_are_refused():
    for k, v, q_out in ((2, 100, 0), (100, 2, 0), (0, 100, 1), (100, 0, 0)):
        assert append_code(k, v, q_out, 7 * 128, 7 * 128) == BAD, (k, v, q_out)


def test_heads_of_other_strides_that_meet_are_refused():
    x = B.CkvRopeRows(4, 3, 2, B.CKV_DTYPE_BF16, 0, 0, 4096, 256, 4096, 384, 4096, 256, 4096, 384)
    # q at rows 0, 2, 4 of a token; k at first and first + 3
    for first in (0, 1, 2, 4, 32 + 1):
        k = AT + ROW * first
        assert ckv.load().compresskv_rope_apply(ckv.Rope(128).addr, ctypes.addressof(x), AT, AT, k, AT, k, None) == BAD
