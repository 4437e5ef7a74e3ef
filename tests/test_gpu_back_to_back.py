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


def test_rows_that_were_just_gathered_go_into_the_4_bit_cache(cuda_device):
    """compresskv_gather, then its k_out and v_out appended and attended to right
    behind it."""
    from oracle import q4_oracle as q4

    dev, rows = cuda_device, 5000
    gen = torch.Generator().manual_seed(5)
    k, v = (torch.randn((6000, 2, 128), generator=gen).bfloat16().to(dev) for _ in range(2))
    q = torch.randn((1, 4, 16, 128), generator=gen).bfloat16().to(dev)
    p = ckv.Problem(q, k, [0, 6000], 16, 7)
    idx = torch.stack([torch.randperm(6000, generator=gen)[:rows] for _ in range(2)]).int().to(dev)
    pos = torch.arange(rows, dtype=torch.int32, device=dev)
    c = ckv.q4_cache(1, 2, rows, dev)
    ws = ckv.q4_workspace(c, 4, 1)
    start = torch.zeros_like(c.lengths)
    ko, vo = (torch.empty((rows, 2, 128), dtype=k.dtype, device=dev) for _ in range(2))
    q1, outs = q[:, :, :1].contiguous(), []
    for _ in range(5):
        c.lengths.zero_()
        ko.zero_()
        vo.zero_()
        ckv.gather(p, idx, [0, rows], k, v, ko, vo)
        ckv.q4_append(c, ko, vo, pos, start=start)
        out = torch.empty_like(q1)
        ckv.q4_attend(c, q1, out, ws)
        outs.append(out)
    torch.cuda.synchronize()
    for g in range(2):
        codes, s, m = q4.quantise(k[idx[g].long(), g].float().cpu().numpy())
        assert torch.equal(c.k_codes[0, g, :rows].cpu(), torch.from_numpy(q4.pack(codes)))
    for out in outs[1:]:
        assert torch.equal(out.view(torch.int16), outs[0].view(torch.int16))
