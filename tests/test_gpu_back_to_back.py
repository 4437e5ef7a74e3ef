"""Calls that read what the call right before them on the stream has written
(needs a GB300)."""
import pytest
import torch

import paper_2606_24467_gb300 as ckv
import workloads as wl

pytestmark = pytest.mark.gpu


def test_scores_of_a_cache_that_was_just_gathered(cuda_device):
    """Scoring kernels follow a gather that lets its successor start early; with
    two gathers in a row the writer may still run when the second one starts."""
    dev, cfg = cuda_device, wl.get("c1").scaled(dtype="bf16", seq_len=6000)
    d = wl.make_layer(cfg, 0)
    q, k, v = d["q_win"].to(dev), d["k"].to(dev), d["v"].to(dev)
    H, rows = k.shape[1], 5000
    p = ckv.Problem(q, k, d["cu_seqlens"], cfg.window, cfg.pool_width)
    gen = torch.Generator().manual_seed(3)
    idx = torch.stack([torch.randperm(6000, generator=gen)[:rows] for _ in range(H)]).int().to(dev)
    ko, vo, ko2, vo2 = (torch.empty((rows, H, 128), dtype=k.dtype, device=dev) for _ in range(4))
    small = ckv.Problem(q, ko, [0, rows], cfg.window, cfg.pool_width)
    ws = ckv.workspace(small, dev)

    def step(twice, wait):
        ko.zero_()
        raw = torch.full((H, rows - cfg.window), float("nan"), device=dev)
        ckv.gather(p, idx, [0, rows], k, v, ko, vo)
        if twice:
            ckv.gather(p, idx[:, :64].contiguous(), [0, 64], k, v, ko2, vo2)
        if wait:
            torch.cuda.synchronize()
        ckv.score(small, q, ko, d["srh_mask"], raw, ws)
        torch.cuda.synchronize()
        return raw

    want = step(False, True)
    assert torch.isfinite(want).all()
    for i in range(6):
        assert torch.equal(step(bool(i & 1), False), want)
