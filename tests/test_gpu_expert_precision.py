"""How exact the experts' products and weight gradients of ordinary values are, in
every kernel that takes them, against 64 bits.

16-bit results come from a matrix instruction that cuts each of eight
neighbouring products, toward zero, to a multiple of 2^-13 of the power of two
that the largest one's factors have (an e4m3 subnormal counts as 2^-6), before
fp32 sums take over. The test computes these cut products in 64 bits; what is left are
fp32 roundings, of at most 2^-23 of a partial sum each: a group of eight and a sum
makes one, and no partial sum of n products of random signs leaves 6 times the root
of the products' squares (Hoeffding: 2 exp(-18) of them). The cuts themselves are
2^-15 of that root, which the mean square of all errors must show.

fp32 results come from exact products and fp32 sums: an addition rounds by 2^-24 of
a partial sum, K of them in any order by sqrt(K) 2^-24 of the root in the mean
square."""
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


def randn(*shape, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV)


def rows8(cl, x):
    q, s = cl.quantized_shapes(*x.shape)
    q = torch.empty(q, dtype=E4M3, device=DEV)
    s = torch.empty(s, dtype=torch.uint8, device=DEV)
    cl.quantize_rows_t(x, q, s)
    return q, s


def picked(n, most, seed):
    """Some of n, the first and the last among them."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randperm(n, generator=g)[:most]
    return torch.unique(torch.cat([at, torch.tensor([0, n - 1])]))


def power(v):
    """Exponents of e4m3 values; a subnormal's is that of the smallest normal."""
    return torch.frexp(v)[1].sub(1).clamp(min=-6).double()


def sums(qa, sa, qb, sb):
    """Of rows qa [n, K] and qb [m, K] (doubles) with scales a block of 128: the sums
    of products, of cut products, and the root of the products' squares."""
    n, K = qa.shape
    blocks = K // 128
    scale = 2.0 ** (sa[:, None, :blocks].double() +
                    sb[None, :, :blocks].double() - 254)
    exact, cut, squares = (torch.zeros(n, qb.shape[0], dtype=torch.float64)
                           for _ in range(3))
    for k in range(blocks):
        part = slice(128 * k, 128 * (k + 1))
        a, b = qa[:, part], qb[:, part]
        p = (a[:, None] * b[None]).view(n, -1, 16, 8)
        e = (power(a)[:, None] + power(b)[None]).view(n, -1, 16, 8)
        e = torch.where(p != 0, e, torch.full_like(e, -60.0))
        unit = 2.0 ** (e.amax(3, keepdim=True) - 13)
        c = torch.trunc(p / unit) * unit
        f = scale[:, :, k]
        exact += p.sum((2, 3)) * f
        cut += c.sum((2, 3)) * f
        squares += (p * p).sum((2, 3)) * f * f
    return exact, cut, squares.sqrt()


def check(out, exact, cut, root, K):
    """`out`: the kernel's results, on the CPU."""
    dtype, out = out.dtype, out.double()
    once = (exact.to(dtype).double() - exact) / root
    err = (out - exact) / root
    if dtype == torch.float32:
        assert float(err.pow(2).mean().sqrt()) <= K ** 0.5 * 2.0 ** -24
        return
    half = torch.finfo(dtype).eps / 2
    bound = half * cut.abs() + (1 + half) * K / 8 * 2.0 ** -23 * 6 * root
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25
    assert ((out - cut).abs() <= bound).all()
    # 1.05: the mean of some thousand squares is known to some hundredths
    most = 1.05 * (float(once.pow(2).mean()) + 2.0 ** -30) ** 0.5
    assert float(err.pow(2).mean().sqrt()) <= most


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16,
                                   torch.float32])
@pytest.mark.parametrize("P,N,K,E", [
    (8, 2048, 1024, 1),     # few rows
    (2, 517, 512, 2),       # few rows of two experts
    (2100, 1032, 1024, 3),  # 16 bits: streaming tiles; fp32: tiles of 128
    (600, 264, 2176, 2),    # the same, an odd number of blocks
    (3000, 261, 1024, 2),   # tiles of 128
    (4200, 4101, 640, 1),   # tiles of 256
])
def test_products(cl, dtype, P, N, K, E):
    a, sa = rows8(cl, randn(P, K, seed=1))
    w = 0.02 * randn(E, N, K, seed=2)
    b = torch.empty(E, N, K, dtype=E4M3, device=DEV)
    sb = torch.empty(E, -(-N // 128), -(-K // 512) * 4, dtype=torch.uint8,
                     device=DEV)
    cl.quantize_blocks_t(w, b, sb)
    step = P // E
    off = torch.tensor([step * e for e in range(E)] + [P], dtype=torch.int32)
    out = torch.full((P, N), 7.0, dtype=dtype, device=DEV)
    cl.expert_matmul_t(a, sa, b, sb, off.to(DEV), out)
    parts = []
    for e in range(E):
        r = picked(int(off[e + 1] - off[e]), 40, 3) + int(off[e])
        c = picked(N, 50, 4)
        scales = sb[e].cpu()[c // 128]
        parts.append((out[r][:, c].cpu(),) + sums(
            a[r].cpu().double(), sa[r].cpu(), b[e, c].cpu().double(), scales))
    check(*(torch.cat([p[i].reshape(-1) for p in parts]) for i in range(4)), K)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16,
                                   torch.float32])
@pytest.mark.parametrize("N,C,counts", [
    (264, 328, [700, 0, 1300]),   # 16 bits: streaming tiles; fp32: tiles of 128
    (131, 261, [1000, 300]),      # tiles of 128
    (4100, 4101, [640]),          # tiles of 256
])
def test_weight_gradients(cl, dtype, N, C, counts):
    P, E = sum(counts), len(counts)
    off = torch.tensor([0] + counts).cumsum(0).int()
    L = cl.ciera_columns_length(P, E)
    both = []
    for n, seed, std in ((N, 1, 0.01), (C, 2, 1.0)):
        x = std * randn(P, n, seed=seed)
        (_, _), (_, S) = cl.quantized_shapes(1, L)
        q = torch.zeros(n, L, dtype=torch.uint8, device=DEV).view(E4M3)
        s = torch.full((n, S), 127, dtype=torch.uint8, device=DEV)
        cl.quantize_columns_t(x, off.to(DEV), q, s)
        both += [q, s]
    out = torch.full((E, N, C), 7.0, dtype=dtype, device=DEV)
    cl.expert_weight_grad_t(*both, off.to(DEV), out)
    y, ys, x, xs = both
    parts, start = [], 0
    for e, n in enumerate(counts):
        end = start + -(-n // 128) * 128
        if n:
            r, c = picked(N, 40, 3), picked(C, 50, 4)
            blocks = slice(start // 128, end // 128)
            parts.append((out[e][r][:, c].cpu(),) + sums(
                y[r, start:end].cpu().double(), ys[r, blocks].cpu(),
                x[c, start:end].cpu().double(), xs[c, blocks].cpu()))
        else:
            assert (out[e] == 0).all()
        start = end
    check(*(torch.cat([p[i].reshape(-1) for p in parts]) for i in range(4)),
          max(counts))


def test_sixteen_bit_sums_that_cancel(cl):
    """What the header says of them: a product 2^14 below the largest of its eight is
    lost, in the next eight it is not; fp32 results keep it."""
    def product(at, dtype):
        a, b = torch.zeros(1, 128), torch.zeros(1, 128)
        a[0, 0], b[0, 0] = 256.0, 256.0
        a[0, 64], b[0, 64] = 256.0, -256.0
        a[0, at], b[0, at] = 2.0, 2.0
        one = torch.full((1, 4), 127, dtype=torch.uint8, device=DEV)
        out = torch.empty(1, 1, dtype=dtype, device=DEV)
        cl.expert_matmul_t(a.to(E4M3).to(DEV), one, b.to(E4M3).to(DEV)[None],
                           one[None], None, out)
        return float(out)

    for dtype in (torch.bfloat16, torch.float16):
        assert product(7, dtype) == 0 and product(8, dtype) == 4
    assert product(7, torch.float32) == 4 == product(8, torch.float32)


@pytest.mark.parametrize("P", [1, 300])
def test_scales_that_fp32_results_hold(cl, P):
    """Every value of the smallest and the largest scale that bf16 holds, with a
    factor that brings the product back."""
    bits = torch.arange(256).to(torch.uint8)
    v = bits.view(E4M3).float()
    v = v[torch.isfinite(v)]
    a = torch.zeros(P, 128)
    b = torch.zeros(v.numel(), 128)
    a[:, 5], b[:, 5] = 1.0, v
    for byte, back in ((3, 200), (246, 20)):
        sa = torch.full((P, 4), back, dtype=torch.uint8, device=DEV)
        sb = torch.full((1, 2, 4), byte, dtype=torch.uint8, device=DEV)
        out = torch.empty(P, v.numel(), device=DEV)
        cl.expert_matmul_t(a.to(E4M3).to(DEV), sa, b.to(E4M3).to(DEV)[None], sb,
                           None, out)
        expect = v.double() * 2.0 ** (byte + back - 254)
        assert torch.equal(out.cpu().double(), expect.expand(P, -1))
