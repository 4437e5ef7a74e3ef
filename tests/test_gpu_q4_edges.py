"""Calls of the 4-bit cache at the edges of what its documentation allows (needs
a GB300)."""
import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from oracle import q4_oracle as q4
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


def spread(c, i, g, slots, power):
    """Multiplies the values of a unit's slots by 2^power (numbers or one)."""
    f = torch.as_tensor(2.0 ** np.asarray(power, np.float64), device=c.v_params.device)
    rows = c.v_params[i, g, slots].double()
    c.v_params[i, g, slots] = (rows * (f[:, None] if f.dim() else f)).bfloat16()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group,n", [(4, 1), (3, 2), (7, 4)])
@pytest.mark.parametrize("kind", ["large", "lowest", "constant", "infinite"])
def test_attend_beside_slots_that_are_not_seen(cuda_device, dtype, group, n, kind):
    """Behind a query's position stand rows of V up to the type's lowest number,
    and infinities: they take no bits from what the row sees, also where another
    row of the same block sees them, in the same tile or an earlier one."""
    gen = torch.Generator().manual_seed(7 * group + n)
    lens = [[200, 90], [64, 3000]]
    c = random_cache(2, 2, 3008, lens, cuda_device, gen)
    last = torch.finfo(dtype).min
    at = torch.full((2, n), 10 ** 6, dtype=torch.int32)
    for i in range(2):
        for g in range(2):
            m = lens[i][g]
            hidden = torch.randperm(m, generator=gen)[:m // 3].to(cuda_device)
            hidden = torch.cat([hidden[hidden > 0], torch.zeros(1, dtype=torch.long, device=cuda_device)])
            c.positions[i, g, :m] = torch.arange(m, dtype=torch.int32, device=cuda_device)
            c.positions[i, g, hidden] += 2 ** 30
            if kind == "large":      # values of about 2^15, or 2^100
                spread(c, i, g, hidden, 15 if dtype == torch.float16 else 100)
            elif kind == "lowest":   # from the lowest number to 0
                c.v_params[i, g, hidden, :4] = abs(last) / 16
                c.v_params[i, g, hidden, 4:] = last
            elif kind == "constant":
                c.v_params[i, g, hidden, :4] = 0.0
                c.v_params[i, g, hidden, 4:] = last
            else:
                c.v_params[i, g, hidden, 4:] = float("inf")
            spread(c, i, g, torch.arange(1, m, 2, device=cuda_device), -9)
    if n > 1:
        at[0, 1] = 2 ** 31 - 1  # sees all
    q = torch.randn((2, 2 * group, n, 128), generator=gen).to(dtype).to(cuda_device)
    if kind == "infinite":  # the cache's own mark for such groups
        c.v_params[torch.isinf(c.v_params)] = float("nan")
        c.v_params[..., :4][torch.isnan(c.v_params[..., 4:])] = float("nan")
    out, _ = run_attend(c, q, q_positions=at.to(cuda_device))
    assert torch.isfinite(out[:, :, 0]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_values_of_many_magnitudes(cuda_device, dtype):
    """V's rows from 2^-60 to 2^60 (f16: 2^-12 to 2^12) by slot, against logits
    that make every magnitude matter somewhere: rows of 2^e get probabilities of
    about 2^-e, slots in rising and in falling order."""
    gen = torch.Generator().manual_seed(17)
    m, most = 400, 60 if dtype == torch.bfloat16 else 12
    c = random_cache(1, 4, m, [[m] * 4], cuda_device, gen)
    power = np.linspace(-most, most, m).round()
    u = torch.randn(128, generator=gen).double()
    for g, p in enumerate((power, power[::-1], np.roll(power, 131), 0 * power + most)):
        # keys along u, so that q = u gives logits of -p ln 2
        k = (-p * np.log(2) * 128 ** 0.5)[:, None] * (u / (u @ u)).numpy() + 0.01 * torch.randn(
            (m, 128), generator=gen).numpy()
        codes, s, mn = q4.quantise(k.astype(np.float32))
        c.k_codes[0, g, :m] = torch.from_numpy(q4.pack(codes)).to(cuda_device)
        c.k_params[0, g, :m] = torch.from_numpy(np.concatenate([s, mn], -1)).bfloat16().to(cuda_device)
        spread(c, 0, g, torch.arange(m, device=cuda_device), p.copy())
    q = torch.stack([u, 0.5 * u, 0 * u, -0.5 * u]).repeat(4, 1)[None, :, None]
    run_attend(c, q.to(dtype).to(cuda_device))


def test_attend_when_a_later_slot_outweighs_large_values(cuda_device):
    """A slot of huge values and small logit first, then one that takes all the
    attention, by more than the values' ratio."""
    gen = torch.Generator().manual_seed(18)
    for first, later in ((100, 0), (100, -90), (0, 110), (-110, 100)):
        c = random_cache(1, 1, 192, [[192]], cuda_device, gen)
        c.k_params[0, 0, 100:, 4:] += 400.0  # logits some hundreds above the others'
        spread(c, 0, 0, torch.arange(0, 100, device=cuda_device), first)
        spread(c, 0, 0, torch.arange(100, 192, device=cuda_device), later)
        q = (0.2 + 0.05 * torch.randn((1, 4, 1, 128), generator=gen)).bfloat16().to(cuda_device)
        run_attend(c, q)


def test_values_beyond_the_largest_f16_number(cuda_device):
    """A group from -65504 to 65504: its top code stands for more than f16 holds."""
    k = torch.zeros((1, 1, 128)).half()
    k[0, 0, 0], k[0, 0, 1], k[0, 0, 2] = 65504.0, -65504.0, 60000.0
    c = blank(1, 1, 32, cuda_device)
    kd = k.to(cuda_device)
    kv, vv = torch.empty_like(kd), torch.empty_like(kd)
    c.lengths.zero_()
    ckv.q4_append(c, kd, kd, torch.zeros(1, dtype=torch.int32, device=cuda_device), k_values=kv, v_values=vv)
    codes, s, m = q4.quantise(k[0].float().numpy())
    want = q4.values(codes, s, m)
    assert 65520 < want[0, 0] < 65504 * (1 + 2.0 ** -6)
    assert torch.equal(kv.cpu()[0], torch.from_numpy(want).half()) and torch.isinf(kv[0, 0, 0])
    q = torch.zeros((1, 1, 1, 128), device=cuda_device).bfloat16()
    out, _ = run_attend(c, q, accumulate=False)
    assert torch.isfinite(out).all()
