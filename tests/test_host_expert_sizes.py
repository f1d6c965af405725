"""Sizes of the experts' products that a device's memory could hold and one launch
could not: refused by the call, before anything is launched (no GPU needed)."""
import os

import pytest

P = 0x10000  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def cl():
    from paper_2609_04609_amd import build, ciera
    if not os.path.exists(ciera.LIB_PATH):
        build.build()
    ciera.lib()
    return ciera


@pytest.mark.parametrize("dtype,E,N,C", [
    (2, 1024, 1, 1 << 20),  # 4 GB of results, 2^23 workgroups of 512
    (0, 1024, 1, (1 << 20) + 1),  # no whole octets: the same tiles
    (1, 512, 3, (1 << 21) + 4),
    (2, 1024, 1 << 20, 1),  # one column of tiles
])
def test_weight_grad(cl, dtype, E, N, C):
    assert cl.ciera_expert_weight_grad(P, P, 4, P, P, 4, 128, E, N, C, P, P,
                                       dtype, 0) == cl.EINVAL


@pytest.mark.parametrize("dtype,R,N", [(2, 1 << 30, 100), (0, 1 << 30, 101),
                                       (1, (1 << 30) + 5, 7)])
def test_products(cl, dtype, R, N):
    assert cl.ciera_expert_matmul(P, 128, P, 4, R, P, 128, P, 4, 1, N, 128, 0,
                                  P, dtype, N, 0) == cl.EINVAL


def test_plan_of_experts_past_int32(cl):
    """No id names them, and a negative id must not."""
    need = cl.ciera_plan_workspace_bytes(10, 2, 64)
    for first in ((1 << 31) - 63, (1 << 31) - 1):
        assert cl.ciera_route_plan(P, 10, 2, first, 64, P, P, P, P, need,
                                   0) == cl.EINVAL


@pytest.mark.parametrize("train", [False, True])
def test_layer_of_a_type_without_kernels(cl, train):
    import torch

    from paper_2609_04609_amd.experts import ExpertLayer
    with pytest.raises(ValueError, match="dtype is torch.float64"):
        ExpertLayer(4, 2, 4, 16, 16, dtype=torch.float64, device="cpu",
                    train=train)
    m = ExpertLayer(4, 2, 4, 16, 16, dtype=torch.float16, device="cpu",
                    train=train)
    assert m.out.dtype == torch.float16
    with pytest.raises(ValueError, match="grad_dtype is torch.int32"):
        ExpertLayer(4, 2, 4, 16, 16, device="cpu", train=train,
                    grad_dtype=torch.int32)
