"""Calls of the 4-bit cache's attention whose bounded wait runs out (a one-shot
hook makes one warp wait for a barrier that nothing completes): the call ends,
the context stays usable, and the workspace's set-up makes it good again (needs
a GB300)."""
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from paper_2606_24467_gb300 import compresskv as B
from test_gpu_q4 import random_cache

pytestmark = pytest.mark.gpu


def call(c, q, ws, accumulate=True):
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    ckv.q4_attend(c, q, out, ws, lse=lse, accumulate=accumulate)
    return out, lse


def init(ws):
    code = ckv.load().compresskv_q4_workspace_init(ws.data_ptr(), ws.numel(), None)
    assert code == B.CKV_OK
    torch.cuda.synchronize()


# units of one CTA each, shared by several CTAs, and in equal runs of tiles over
# the CTAs (each CTA ends one row block and starts another)
@pytest.mark.parametrize("lens,group,n", [([[700, 64]], 4, 1), ([[30000, 20000]], 4, 1),
                                          ([[9000, 300], [5000, 1], [2500, 7777]], 7, 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_wait_runs_out(cuda_device, lens, group, n, dtype):
    gen = torch.Generator().manual_seed(81)
    c = random_cache(len(lens), 2, max(map(max, lens)), lens, cuda_device, gen)
    q = torch.randn((len(lens), 2 * group, n, 128), generator=gen).to(dtype).to(cuda_device)
    ws = ckv.q4_workspace(c, 2 * group, n)
    w0 = c.weights.clone()
    out, lse = call(c, q, ws)
    w1 = c.weights.clone()
    c.weights.copy_(w0)
    torch.cuda.synchronize()
    ckv.debug_stall_next_q4_attend(2_000_000)
    call(c, q, ws)
    assert ckv.read_device_status(ws) == B.CKV_ERR_DEVICE_TIMEOUT
    # no weight of logits and sums that were not made, by this call or the next
    assert torch.equal(w0.view(torch.int32), c.weights.view(torch.int32))
    call(c, q, ws)
    assert torch.equal(w0.view(torch.int32), c.weights.view(torch.int32))
    init(ws)
    assert ckv.read_device_status(ws) == 0
    for _ in range(2):  # (tickets of the row blocks that were left half done start again)
        c.weights.copy_(w0)
        again, lse2 = call(c, q, ws)
        assert ckv.read_device_status(ws) == 0
        assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)
        assert torch.equal(w1.view(torch.int32), c.weights.view(torch.int32))


def test_attend_stops_while_other_warps_work(cuda_device):
    """The wait runs out after 0.1 ms of a call that takes longer."""
    gen = torch.Generator(device=cuda_device).manual_seed(83)
    c = ckv.q4_cache(4, 8, 131072, cuda_device, weights=False)
    for part in ("k", "v"):
        getattr(c, part + "_codes").random_(0, 256, generator=gen)
        getattr(c, part + "_params").uniform_(0, 0.1, generator=gen)
    c.lengths.fill_(131072)
    q = torch.randn((4, 64, 1, 128), generator=gen, device=cuda_device).bfloat16()
    ws = ckv.q4_workspace(c, 64, 1)
    want = call(c, q, ws, accumulate=False)
    for _ in range(10):
        torch.cuda.synchronize()
        ckv.debug_stall_next_q4_attend(100_000)
        call(c, q, ws, accumulate=False)
        assert ckv.read_device_status(ws) == B.CKV_ERR_DEVICE_TIMEOUT
        init(ws)
    got = call(c, q, ws, accumulate=False)
    assert ckv.read_device_status(ws) == 0
    assert torch.equal(want[0].view(torch.int16), got[0].view(torch.int16)) and torch.equal(want[1], got[1])


def test_a_call_without_slots_does_not_stall(cuda_device):
    gen = torch.Generator().manual_seed(82)
    c = random_cache(1, 2, 64, [[0, 0]], cuda_device, gen)
    q = torch.randn((1, 4, 1, 128), generator=gen).half().to(cuda_device)
    ws = ckv.q4_workspace(c, 4, 1)
    ckv.debug_stall_next_q4_attend(2_000_000)
    out, lse = call(c, q, ws)
    assert ckv.read_device_status(ws) == 0 and not out.any() and (lse == float("-inf")).all()


def test_weights_stay_whatever_the_status_said_before(cuda_device):
    """The status keeps its first error, here an index that a gather skipped; a
    call that does not stop adds its weights all the same, one that does does not."""
    gen = torch.Generator().manual_seed(84)
    c = random_cache(1, 2, 96, [[90, 70]], cuda_device, gen)
    q = torch.randn((1, 8, 1, 128), generator=gen).half().to(cuda_device)
    ws = ckv.q4_workspace(c, 8, 1)
    ws[:4].view(torch.int32).fill_(B.CKV_ERR_DEVICE_INDEX)
    w0 = c.weights.clone()
    call(c, q, ws)
    torch.cuda.synchronize()
    assert (c.weights[0, 0, :90] > w0[0, 0, :90]).all()
    w1 = c.weights.clone()
    ckv.debug_stall_next_q4_attend(1_000_000)
    call(c, q, ws)
    assert ckv.read_device_status(ws) == B.CKV_ERR_DEVICE_INDEX
    assert torch.equal(w1.view(torch.int32), c.weights.view(torch.int32))
