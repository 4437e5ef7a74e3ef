"""Rotary positions (rope_apply) on the GPU against float64."""
import numpy as np
import pytest
import torch

import paper_2606_24467_gb300 as ckv
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu


def near(got, x, positions, rope, scale=1.0, backward=False, angle=2.0 ** -21):
    """Half a step of the dtype, and fp32 cosines and sines (2^-21 of the pair; more
    where the float64 angles themselves are rounded by more)."""
    want = po.rotate(x, positions, rope.frequencies, rope.interleaved, scale, backward)
    n = rope.rot_dim
    assert torch.equal(got[..., n:], x[..., n:])
    ahead = po.rotate(x.abs().double(), torch.zeros_like(positions), rope.frequencies, rope.interleaved)
    pair = ahead[..., :n].unflatten(-1, (-1, 2) if rope.interleaved else (2, -1))
    both = pair.sum(-1 if rope.interleaved else -2, keepdim=True).expand_as(pair).flatten(-2)
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * half
    w = want[..., :n]
    tol = half * w.abs() + abs(scale) * both * angle * (1 + half) + tiny
    bad = (got[..., :n].double() - w).abs() > tol
    assert not bad.any(), (got[..., :n].double() - w).abs().max()


def rows(gen, shape, dtype):
    return torch.randn(shape, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot_dim", [128, 96, 64, 20, 2])
def test_layouts(rot_dim, interleaved, dtype):
    gen = torch.Generator().manual_seed(rot_dim)
    rope = ckv.Rope(rot_dim, base=10000.0, interleaved=interleaved)
    for n, hq, hk in ((1, 1, 0), (3, 28, 4), (37, 32, 8), (700, 5, 3)):
        q, k = rows(gen, (n, hq, 128), dtype), rows(gen, (n, hk, 128), dtype) if hk else None
        pos = torch.randint(0, 40000, (n,), generator=gen).int().cuda()
        qo, ko = torch.empty_like(q), torch.empty_like(k) if hk else None
        ckv.rope_apply(rope, pos, q, k, qo, ko)
        near(qo, q, pos, rope)
        if hk:
            near(ko, k, pos, rope)
        ckv.rope_apply(rope, pos, q, k, qo, ko, backward=True)
        near(qo, q, pos, rope, backward=True)
        q0 = q.clone()
        ckv.rope_apply(rope, pos, q)  # in place, q alone
        near(q, q0, pos, rope)


def test_far_and_negative_positions():
    gen = torch.Generator().manual_seed(1)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, -987654321, 2 ** 24 + 1],
                       dtype=torch.int32)
    q = rows(gen, (8, 4, 128), torch.float16)
    for scaling in (dict(), dict(scaling="linear", factor=7.0), dict(scaling="base", factor=16.0),
                    dict(scaling="waves", factor=8.0, original_length=8192.0),
                    dict(scaling="ramp", factor=4.0, original_length=4096.0, low=1.0, high=32.0)):
        rope = ckv.Rope(128, base=500000.0, scale=1.25, **scaling)
        out = torch.empty_like(q)
        ckv.rope_apply(rope, pos.cuda(), q, q_out=out)
        # three float64 roundings (the frequency over 2 pi, 2 pi, the oracle's angle), each
        # up to 2^-53 of 2^31 radians
        near(out, q, pos.cuda(), rope, scale=1.25, angle=2.0 ** -19)


def test_strides_and_views():
    gen = torch.Generator().manual_seed(2)
    rope = ckv.Rope(128)
    qkv = rows(gen, (50, 6 + 2 + 2, 128), torch.bfloat16)
    before = qkv.clone()
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    ckv.rope_apply(rope, pos, qkv[:, :6], qkv[:, 6:8])  # in place inside a fused projection
    near(qkv[:, :6], before[:, :6], pos, rope)
    near(qkv[:, 6:8], before[:, 6:8], pos, rope)
    assert torch.equal(qkv[:, 8:], before[:, 8:])
    x = rows(gen, (3, 50, 128), torch.bfloat16).transpose(0, 1)  # head-major
    out = torch.empty(50, 3, 256, dtype=x.dtype, device="cuda")[..., 128:]
    ckv.rope_apply(rope, pos, x, q_out=out)
    near(out, x, pos, rope)
    one = rows(gen, (50, 1, 128), torch.bfloat16)
    out = torch.empty(50, 3, 128, dtype=x.dtype, device="cuda")
    ckv.rope_apply(rope, pos, one.expand(50, 3, 128), q_out=out)  # a row shared by heads is read as often
    near(out, one.expand(50, 3, 128), pos, rope)


def test_gradient_by_differences_and_round_trip():
    """<g, R x> = <R^T g, x>; and the rotation back gives the rows again."""
    gen = torch.Generator().manual_seed(3)
    for interleaved in (False, True):
        rope = ckv.Rope(64, interleaved=interleaved)
        pos = torch.randint(0, 100000, (40,), generator=gen).int().cuda()
        x, g = rows(gen, (40, 8, 128), torch.float16), rows(gen, (40, 8, 128), torch.float16)
        y, gx = torch.empty_like(x), torch.empty_like(x)
        ckv.rope_apply(rope, pos, x, q_out=y)
        ckv.rope_apply(rope, pos, g, q_out=gx, backward=True)
        left, right = (g.double() * y.double()).sum(-1), (gx.double() * x.double()).sum(-1)
        # two rounded vectors of 128: at most half a step of each product's magnitude
        size = (g.double().norm(dim=-1) * x.double().norm(dim=-1))
        assert ((left - right).abs() <= 2.2 * 2.0 ** -11 * size).all()
        # a difference along one channel is that channel's column
        step = torch.zeros_like(x)
        step[..., 5] = 1.0
        moved = torch.empty_like(x)
        ckv.rope_apply(rope, pos, step, q_out=moved)
        want = (g.double() * moved.double()).sum(-1)
        tol = 2.0 ** -11 * (gx[..., 5].double().abs() + 2 * g.double().abs().amax(-1)) + 2.0 ** -20
        assert ((gx[..., 5].double() - want).abs() <= tol).all()
        ckv.rope_apply(rope, pos, y, backward=True)
        pair = x.double().abs().amax(-1, keepdim=True) * 2
        assert ((y.double() - x.double()).abs() <= 2.0 ** -10 * pair).all()


def test_nan_stays_in_its_pair_and_what_is_not_rotated_is_copied():
    rope = ckv.Rope(32)
    x = torch.ones(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 3] = float("nan")
    x[1, 1, 100] = float("inf")
    x[1, 1, 101] = float("nan")
    out = torch.empty_like(x)
    ckv.rope_apply(rope, torch.tensor([5, 6], dtype=torch.int32, device="cuda"), x, q_out=out)
    bad = torch.isnan(out)
    assert bad[0, 0, 3] and bad[0, 0, 19] and bad[1, 1, 101] and int(bad.sum()) == 3
    assert out[1, 1, 100] == float("inf")


def test_graph_and_side_stream():
    gen = torch.Generator().manual_seed(4)
    rope = ckv.Rope(128)
    q = rows(gen, (16, 8, 128), torch.bfloat16)
    pos = torch.zeros(16, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        ckv.rope_apply(rope, pos, q, q_out=out)
    torch.cuda.synchronize()
    near(out, q, pos, rope)
    with torch.cuda.graph(graph):
        ckv.rope_apply(rope, pos, q, q_out=out)
    for p in (3, 70000):
        pos.fill_(p)
        graph.replay()
        torch.cuda.synchronize()
        near(out, q, pos, rope)


def test_rows_of_no_heads_and_no_rows():
    rope = ckv.Rope(128)
    q = torch.empty(0, 4, 128, dtype=torch.float16, device="cuda")
    ckv.rope_apply(rope, torch.empty(0, dtype=torch.int32, device="cuda"), q)
    q = torch.ones(3, 0, 128, dtype=torch.float16, device="cuda")
    ckv.rope_apply(rope, torch.zeros(3, dtype=torch.int32, device="cuda"), q)
    torch.cuda.synchronize()


def test_launches_are_traced():
    rope, trace = ckv.Rope(128), ckv.Trace(4)
    q = torch.ones(3, 2, 128, dtype=torch.float16, device="cuda")
    ckv.rope_apply(rope, torch.zeros(3, dtype=torch.int32, device="cuda"), q, trace=trace)
    torch.cuda.synchronize()
    assert [k for k, _ in trace.records()] == ["rope"] and trace.launches == 1
    assert np.isfinite(trace.records()[0][1])
