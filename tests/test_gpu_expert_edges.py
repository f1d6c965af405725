"""The experts' operators at the edges of what their calls allow: offsets that a
caller got wrong, saturated scores, biases far apart, sums that cancel."""
import math

import pytest
import torch

from tests import expert_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def cl():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04609_amd import ciera
    ciera.lib()
    return ciera


def randn(*shape, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * std


# ------------------------------------------------------ offsets that fall ----

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16,
                                   torch.float32])
@pytest.mark.parametrize("E,top", [(4, 2 ** 31 - 1), (7, 300),
                                   (1000, 2 ** 31 - 1)])
def test_weight_grad_of_offsets_that_fall(cl, dtype, E, top):
    """Offsets 0, top, 0, top ...: an expert has at most all columns, those that
    start behind the last column have none, nothing outside is read, and the call
    ends. (Rows of 2^31 in 500 experts add up to 2^33 blocks.)"""
    N, C, L = 24, 40, 640
    g = torch.Generator().manual_seed(E)
    dy = torch.randint(-4, 5, (N, L), generator=g).float()
    x = torch.randint(-4, 5, (C, L), generator=g).float()
    one = torch.full((max(N, C), 8), 127, dtype=torch.uint8, device=DEV)
    off = torch.tensor([top * (e % 2) for e in range(E + 1)],
                       dtype=torch.int32)
    dw = torch.full((E, N, C), 9.0, dtype=dtype, device=DEV)
    cl.expert_weight_grad_t(dy.to(E4M3).to(DEV), one[:N].contiguous(),
                            x.to(E4M3).to(DEV), one[:C].contiguous(),
                            off.to(DEV), dw)
    start = 0
    for e in range(E):
        n = -(-max(0, min(int(off[e + 1]), L) - min(int(off[e]), L)) // 128) * 128
        a, b = min(start, L), min(start + n, L)
        expect = dy[:, a:b] @ x[:, a:b].t()  # whole numbers below 2^14
        assert torch.equal(dw[e].cpu(), expect.to(dtype)), e
        start += n
