"""Q, K and V that lie between one another in memory, rotated in place and appended, give
what separate tensors give."""
import pytest
import torch

import paper_2606_24467_gb300 as ckv

pytestmark = pytest.mark.gpu


def between(n, h, how):
    """q, k and v [n, h, 128] in one buffer."""
    gen = torch.Generator().manual_seed(n)
    if how == "heads of a token in turn":
        x = torch.randn((n, h, 3, 128), generator=gen).bfloat16().cuda()
        return [x[:, :, i] for i in range(3)]
    if how == "tokens of a head in turn":
        x = torch.randn((3 * h, n, 128), generator=gen).bfloat16().cuda()
        return [x[i::3].transpose(0, 1) for i in range(3)]
    if how == "heads in turn, tokens apart":
        x = torch.randn((n, 3 * h + 1, 128), generator=gen).bfloat16().cuda()
        return [x[:, i:3 * h:3] for i in range(3)]
    x = torch.randn((n, 3 * h, 128), generator=gen).bfloat16().cuda()  # a fused projection
    return [x[:, i * h:(i + 1) * h] for i in range(3)]


@pytest.mark.parametrize("how", ["heads of a token in turn", "tokens of a head in turn", "heads in turn, tokens apart",
                                 "side by side"])
@pytest.mark.parametrize("n, h", [(1, 4), (1, 1), (37, 4), (37, 1)])
def test_between_one_another(how, n, h):
    rope = ckv.Rope(128)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    apart = [x.clone() for x in between(n, h, how)]
    ckv.rope_apply(rope, pos, apart[0], apart[1])
    q, k, v = between(n, h, how)
    ckv.rope_apply(rope, pos, q, k)
    assert torch.equal(q, apart[0]) and torch.equal(k, apart[1]) and torch.equal(v, apart[2])
    q, k, v = between(n, h, how)
    cache = ckv.paged_cache(1, h, n, 16)
    ckv.paged_append(cache, k, v, rope=rope, q=q)
    back = [torch.empty((n, h, 128), dtype=v.dtype, device="cuda") for _ in range(2)]
    ckv.paged_gather(cache, *back)
    assert torch.equal(q, apart[0]) and torch.equal(back[0], apart[1]) and torch.equal(back[1], apart[2])
