"""Calls of the 4-bit cache at the edges of what its documentation allows (needs
a GB300)."""
import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from paper_2606_24467_gb300 import compresskv as B
from test_gpu_q4 import blank, check_rows, host, random_cache, run_attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2, 40])
def test_append_behind_lengths_outside_the_cache(cuda_device, rows):
    """A length below 0 counts as 0, one beyond the capacity as the capacity."""
    gen = torch.Generator().manual_seed(rows)
    c = blank(1, 3, 64, cuda_device)
    c.lengths.copy_(torch.tensor([[-5, 1000, 3]], dtype=torch.int32))
    old = host(c)
    k, v = (torch.randn((rows, 3, 128), generator=gen).half() for _ in range(2))
    pos = torch.arange(rows, dtype=torch.int32, device=cuda_device)
    status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    ckv.q4_append(c, k.to(cuda_device), v.to(cuda_device), pos, device_status=status)
    new = host(c)
    assert new["lengths"].tolist() == [[rows, 64, 3 + rows]]
    assert int(status) == B.CKV_ERR_DEVICE_INDEX  # the second unit's rows have no room
    for g, at in ((0, 0), (2, 3)):
        check_rows(new, 0, g, slice(at, at + rows), k[:, g].float().numpy(), v[:, g].float().numpy())
        assert np.array_equal(new["positions"][0, g, at:at + rows], np.arange(rows))
    assert np.array_equal(old["k_codes"][0, 1], new["k_codes"][0, 1])
    assert np.array_equal(old["positions"][0, 1], new["positions"][0, 1])


@pytest.mark.parametrize("lens", [[[1, 20]], [[300, 700]], [[20000, 1500]]])
def test_attend_values_near_the_largest_number(cuda_device, lens):
    """V up to 2^127: by a warp alone, joined in a CTA, and joined by CTAs, no
    sum on the way may pass what fp32 holds."""
    gen = torch.Generator().manual_seed(91)
    c = random_cache(1, 2, max(lens[0]), lens, cuda_device, gen)
    for g in range(2):  # (behind the length there are NaN)
        n = lens[0][g]
        c.v_params[0, g, :n] = (c.v_params[0, g, :n].double() * 2.0 ** 124).bfloat16()
    out, _ = run_attend(c, torch.randn((1, 8, 2, 128), generator=gen).bfloat16().to(cuda_device))
    assert torch.isfinite(out).all()
