"""The experts' operators on matrices of more than 2^32 bytes: what lies in front of
the last rows is zeros, the last rows are compared with 64 bits."""
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
    if torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("less than 64 GiB of memory")
    from paper_2609_04609_amd import ciera
    ciera.lib()
    yield ciera
    torch.cuda.empty_cache()


def randn(*shape, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g)


def zeros8(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device=DEV).view(E4M3)


def eights(R, C, seed):
    """Whole numbers in e4m3 and scales that leave them as they are."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(-8, 9, (R, C), generator=g).float()
    return v, v.to(E4M3).to(DEV)


def test_rows_and_columns(cl):
    R, C = 530_001, 4224  # 4.5 GB of bf16; 8-bit columns 2.2 GB
    x = torch.zeros(R, C, dtype=torch.bfloat16, device=DEV)
    last = randn(200, C, seed=1).bfloat16()
    x[-200:] = last.to(DEV)
    q = zeros8(2 * R, C)  # 4.5 GB
    s = torch.zeros(2 * R, 36, dtype=torch.uint8, device=DEV)
    at = torch.full((R, 1), -1, dtype=torch.int32, device=DEV)
    at[-200:, 0] = torch.arange(2 * R - 200, 2 * R, device=DEV).int()
    cl.quantize_rows_t(x, q, s, position=at)
    qr, sr = ref.quantize(last, 1, 128)
    assert torch.equal(q[-200:].float().cpu().double(), qr)
    assert torch.equal(s[-200:, :33].cpu().long(), sr)
    del q, s
    off = torch.tensor([0, R - 100, R], dtype=torch.int32, device=DEV)
    L = cl.ciera_columns_length(R, 2) * 2  # columns of 1.06 MB: 4.5 GB
    qt = zeros8(C, L)
    st = torch.zeros(C, -(-L // 512) * 4, dtype=torch.uint8, device=DEV)
    cl.quantize_columns_t(x, off, qt, st)
    start = -(-(R - 100) // 128) * 128
    qr, sr = ref.quantize(last[100:], 128, 1)
    assert torch.equal(qt[:, start:start + 100].float().cpu().double(), qr.t())
    assert torch.equal(st[:, start // 128].cpu().long(), sr[0])
    # the last columns' rows' gradient with themselves, of the last expert
    dw = torch.empty(2, C, C, device=DEV)
    cl.expert_weight_grad_t(qt, st, qt, st, off, dw)
    v = ref.values(*ref.quantize(last[100:], 128, 1), 128, 1)
    bound = 100 * 2.0 ** -23 * (v.abs().t() @ v.abs())
    assert ((dw[1].cpu().double() - v.t() @ v).abs() <= bound).all()


@pytest.mark.parametrize("P", [3, 700])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights(cl, P, dtype):
    E, N, D = 65, 8200, 8192  # 4.4 GB
    v, rows = eights(P, D, 1)
    b, last = eights(N, D, 2)
    w = zeros8(E, N, D)
    w[-1] = last
    sa = torch.full((P, 64), 127, dtype=torch.uint8, device=DEV)
    sb = torch.full((E, 65, 64), 127, dtype=torch.uint8, device=DEV)
    off = torch.tensor([0] * E + [P], dtype=torch.int32, device=DEV)
    out = torch.empty(P, N, dtype=dtype, device=DEV)
    cl.expert_matmul_t(rows, sa, w, sb, off, out)
    exact = (v.double() @ b.double().t())  # whole numbers below 2^24
    assert torch.equal(out.cpu(), exact.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_and_results_of_products(cl, dtype):
    P, N, D = 1_050_000, 4104, 4224  # rows 4.4 GB, results 8.6 or 17 GB
    v, last = eights(300, D, 1)
    b, w = eights(N, D, 2)
    rows = zeros8(P, D)
    rows[-300:] = last
    sa = torch.full((P, 36), 127, dtype=torch.uint8, device=DEV)
    sb = torch.full((1, 33, 36), 127, dtype=torch.uint8, device=DEV)
    out = torch.empty(P, N, dtype=dtype, device=DEV)
    out[-301:] = 7
    cl.expert_matmul_t(rows, sa, w[None], sb, None, out)
    exact = (v.double() @ b.double().t()).to(dtype)
    assert torch.equal(out[-300:].cpu(), exact)
    assert (out[-301] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weight_grad_past_the_caches(cl, dtype):
    """Results of more than 256 MiB, of ragged tiles; no row twice alike."""
    E, N, C = 19, 2600, 2824
    counts = [(7 * e) % 13 * 20 for e in range(E)]
    off = torch.tensor([0] + counts).cumsum(0).int()
    P = int(off[-1])
    g = torch.Generator().manual_seed(1)
    dy = torch.randint(-2, 3, (P, N), generator=g).to(dtype)
    x = torch.randint(-2, 3, (P, C), generator=g).to(dtype)
    L = cl.ciera_columns_length(P, E)
    S = -(-L // 512) * 4
    yt, xt = zeros8(N, L), zeros8(C, L)
    ys = torch.zeros(N, S, dtype=torch.uint8, device=DEV)
    xs = torch.zeros(C, S, dtype=torch.uint8, device=DEV)
    at = off.to(DEV)
    cl.quantize_columns_t(dy.to(DEV), at, yt, ys)
    cl.quantize_columns_t(x.to(DEV), at, xt, xs)
    dw = torch.full((E, N, C), 7, dtype=dtype, device=DEV)
    cl.expert_weight_grad_t(yt, ys, xt, xs, at, dw)
    for e in range(E):
        rows = slice(int(off[e]), int(off[e + 1]))
        exact = dy[rows].float().t() @ x[rows].float()  # below 4 * 240
        assert torch.equal(dw[e].cpu(), exact.to(dtype)), e


def test_blocks(cl):
    E, N, C = 130, 4100, 8200  # 8.7 GB, 8 bits 4.4 GB each way
    w = torch.zeros(E, N, C, dtype=torch.bfloat16, device=DEV)
    last = randn(N, C, seed=1).bfloat16()
    w[-1] = last.to(DEV)
    (_, Cq), (_, Cs) = cl.quantized_shapes(N, C)
    (_, Nq), (_, Ns) = cl.quantized_shapes(C, N)
    q, qt = zeros8(E, N, Cq), zeros8(E, C, Nq)
    s = torch.empty(E, 33, Cs, dtype=torch.uint8, device=DEV)
    st = torch.empty(E, 65, Ns, dtype=torch.uint8, device=DEV)
    cl.quantize_blocks_t(w, q, s, qt, st)
    qr, sr = ref.quantize(last, 128, 128)
    assert torch.equal(q[-1, :, :C].float().cpu().double(), qr)
    assert torch.equal(qt[-1, :, :N].float().cpu().double(), qr.t())
    assert torch.equal(s[-1, :, :65].cpu().long(), sr)
    assert torch.equal(st[-1, :, :33].cpu().long(), sr.t())


def test_combine(cl):
    T, k, P, C = 530_000, 2, 530_002, 4104  # 4.35 GB each
    rows = torch.zeros(P, C, dtype=torch.bfloat16, device=DEV)
    last = randn(2, C, seed=1).bfloat16()
    rows[-2:] = last.to(DEV)
    at = torch.full((T, k), -1, dtype=torch.int32, device=DEV)
    at[-1] = torch.tensor([P - 2, P - 1], device=DEV).int()
    w = torch.full((T, k), 0.5, device=DEV)
    out = torch.full((T, C), 3.0, dtype=torch.bfloat16, device=DEV)
    cl.combine_t(rows, at, out, weights=w)
    y = last.double().sum(0) / 2
    assert ((out[-1].cpu().double() - y).abs() <=
            2.0 ** -8 * y.abs() + 2.0 ** -22 * last.double().abs().sum(0)).all()
    assert (out[-2] == 0).all()
    g = torch.zeros(T, C, dtype=torch.bfloat16, device=DEV)
    g[-1] = last[0].to(DEV)
    d_w = torch.empty(T, k, device=DEV)
    d_rows = torch.full((P, C), 3.0, dtype=torch.bfloat16, device=DEV)
    cl.combine_backward_t(g, rows, w, at, d_rows, d_w)
    assert torch.equal(d_rows[-2:].cpu(), (last[:1] / 2).expand(2, C))
    assert (d_rows[-3] == 3).all()
    dots = (last[:1].double() * last.double())
    bound = (C / 64 + 16) * 2.0 ** -23 * dots.abs().sum(1)
    assert ((d_w[-1].cpu().double() - dots.sum(1)).abs() <= bound).all()


def test_logits(cl):
    """Rows 4 KB apart: the last ones lie behind 2^32 bytes."""
    T, E = 1_100_000, 8
    wide = torch.zeros(T, 2048, dtype=torch.bfloat16, device=DEV)
    l, d = wide[:, :E], wide[:, E:2 * E]
    last = randn(70, E, seed=1).bfloat16()
    l[-70:] = last.to(DEV)
    ids = torch.empty(T, 2, dtype=torch.int32, device=DEV)
    w = torch.empty(T, 2, device=DEV)
    cl.route_t(l, ids, w, normalize=True)
    i, x = ref.route(last, 2, normalize=True)
    assert torch.equal(ids[-70:].cpu().long(), i)
    assert ((w[-70:].cpu().double() - x).abs() <= 2.0 ** -19).all()
    cl.route_backward_t(l, ids, torch.ones_like(w), d)
    z = last.double().requires_grad_()
    torch.softmax(z, 1).gather(1, i).sum().backward()
    assert ((d[-70:].cpu().double() - z.grad).abs() <=
            2.0 ** -8 * z.grad.abs() + 2.0 ** -18).all()
