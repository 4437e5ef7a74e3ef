"""The 4-bit cache's attention in row blocks of 16 (more than 8 query rows a
unit, more than 2^20 slots) where CTAs take equal runs of all tiles: a CTA ends
one row block and starts another, row blocks are joined over CTAs, and the CTA
that comes last joins two of them at once (needs a GB300)."""
import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from test_gpu_q4 import BYTES, blank, check_attend, host, random_cache

pytestmark = pytest.mark.gpu


# 100 units of two row blocks are more than the SMs, so no row block has CTAs of
# its own; more than 128 units are added up by the whole CTA instead of by a warp.
@pytest.mark.parametrize("units,most", [(100, 900), (200, 400), (40, 6000)])
@pytest.mark.parametrize("group,n,causal", [(5, 4, False), (7, 4, True), (20, 1, True), (9, 1, False)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_in_row_blocks_of_16(cuda_device, units, most, group, n, causal, dtype):
    gen = torch.Generator().manual_seed(units + group)
    b, h = units // 2, 2
    le = (most * torch.rand((b, h), generator=gen) ** 2).int().numpy()
    le[::9] = 0
    le[1::9, 1] = 1
    le[-1, -1] = most
    small = random_cache(b, h, most, le, cuda_device, gen)
    c = blank(b, h, 2 ** 20 // units + 64, cuda_device)
    used = small.capacity
    for name in BYTES[:-1]:
        getattr(c, name)[:, :, :used] = getattr(small, name)
    c.lengths.copy_(small.lengths)
    q = torch.randn((b, h * group, n, 128), generator=gen).to(dtype).to(cuda_device)
    at = torch.randint(-1, 3 * used, (b, n), generator=gen).int().to(cuda_device) if causal else None
    ws = ckv.q4_workspace(c, q.shape[1], n)
    before = host(small)
    w0 = c.weights.clone()
    for _ in range(2):  # (and the tickets are ready for the next call)
        c.weights.copy_(w0)
        out, lse = torch.full_like(q, float("nan")), torch.empty(q.shape[:3], device=cuda_device)
        ckv.q4_attend(c, q, out, ws, q_positions=at, lse=lse, accumulate=True)
        assert ckv.read_device_status(ws) == 0
    assert torch.isnan(c.weights[:, :, used:]).all()
    pick = np.r_[0:4, b // 2, b - 3:b]  # sequences that are compared
    part = {k: v[pick] for k, v in before.items()}
    check_attend(part, q[pick], out[pick], lse[pick], part["weights"],
                 c.weights[pick, :, :used].cpu().numpy(), 128 ** -0.5, None if at is None else at[pick])
    # every other one is finite, and empty where nothing is seen
    assert torch.isfinite(out).all()
    assert not out[0].any() and (lse[0] == float("-inf")).all()
