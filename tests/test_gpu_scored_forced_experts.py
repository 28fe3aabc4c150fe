"""A bias of +infinity forces an expert into every choice that its group is part of; a group of fewer eligible experts than its value
sums is -infinity all the same, as mcft.h defines it, and no NaN that ranks by its bits."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M

from .test_gpu_route_scored import desc_of

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,d", [(3, 64, 128), (90, 64, 128), (5, 256, 1024), (300, 256, 256)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups_of_a_forced_and_no_other_expert(T, E, d, score, dtype):
    G, g = 8, torch.Generator().manual_seed(T)
    size = E // G
    x, w = torch.randn(T, d, generator=g).to(dtype).cuda(), (torch.randn(E, d, generator=g) * 0.05).to(dtype).cuda()
    lone = torch.zeros(E)
    lone[5 * size:6 * size] = -INF
    lone[5 * size + 3] = INF  # alone in group 5: its group's value is -infinity, and seven groups have better ones
    masked = lone.clone()
    masked[5 * size + 3] = -INF
    D = desc_of(d, E, 4, dtype, score, n_group=G, topk_group=7, group_top=2)
    got, want = (M.mcft_route_scored(D, x, w, b.cuda()) for b in (lone, masked))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert not (got[0] == 5 * size + 3).any()
    # with company the group's value is +infinity, and the expert is chosen first
    lone[5 * size + 1] = 0.0
    D = desc_of(d, E, 4, dtype, score, n_group=G, topk_group=2, group_top=2)
    idx, gate = M.mcft_route_scored(D, x, w, lone.cuda())
    M.mcft_device_error()
    assert (idx[:, 0] == 5 * size + 3).all() and torch.isfinite(gate).all()
    # by its best alone it needs none
    D = desc_of(d, E, 4, dtype, score, n_group=G, topk_group=1, group_top=1)
    lone[5 * size + 1] = -INF
    idx, gate = M.mcft_route_scored(D, x, w, lone.cuda())
    M.mcft_device_error()
    assert (idx[:, 0] == 5 * size + 3).all() and (idx[:, 1:] == -1).all() and (gate[:, 0] == 1).all()
