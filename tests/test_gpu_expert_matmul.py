"""Quantisation, the experts' products, their gradients and the combination
against 64-bit definitions (tests/expert_ref.py). Quantisation has one right
answer and is compared exactly. Products of small integers with small
power-of-two scales are exact in fp32 whatever the order of the sum, so the
results must be the exact sum rounded once to the output's type."""
import math

import pytest
import torch

from tests import expert_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
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


def same(a, b):
    """Equal values, NaN at the same places."""
    a, b = a.double().cpu(), b.double().cpu()
    assert a.shape == b.shape
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0))


def narrow(rows, cols, fill=0xA5):
    """An 8-bit matrix and its scales with old bytes in them."""
    blocks = -(-cols // 128)
    q = torch.full((rows, 128 * blocks), fill, dtype=torch.uint8, device=DEV)
    s = torch.full((rows, -(-blocks // 4) * 4), fill, dtype=torch.uint8,
                   device=DEV)
    return q.view(E4M3), s


def hard_values(rows, cols, dtype, seed):
    """Values over many magnitudes, with zeros, subnormals, the type's extremes
    and what is not finite in places."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    x *= 2.0 ** torch.randint(-12, 12, (rows, cols), generator=g).double()
    x = x.to(dtype)
    flat = x.view(-1)
    i = torch.randperm(flat.numel(), generator=g)
    f = torch.finfo(dtype)
    for j, v in enumerate([0.0, -0.0, f.max, f.min, f.tiny, f.tiny / 4,
                           math.inf, -math.inf, math.nan, 448.0, 449.0,
                           1.75 * 2 ** 9, 240.0, 464.0]):
        if j < flat.numel() // 8:
            flat[i[j]] = v
    if rows > 2:
        x[1] = 0
        x[2, :] = f.tiny / 8
    return x


# ---------------------------------------------------------- quantisation ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,C", [(1, 1), (3, 127), (5, 128), (7, 129),
                                 (16, 512), (9, 513), (4, 1100), (2, 4097)])
def test_rows(cl, dtype, R, C):
    x = hard_values(R, C, dtype, R * 1000 + C)
    q, s = narrow(R, C)
    cl.quantize_rows_t(x.to(DEV), q, s)
    qr, sr = ref.quantize(x, 1, 128)
    same(q[:, :C].float(), qr)
    assert (q.view(torch.uint8)[:, C:] == 0).all()
    n = sr.shape[1]
    assert torch.equal(s[:, :n].cpu().long(), sr)
    assert (s[:, n:] == 127).all()


def test_every_bf16_rounds_right(cl):
    """All finite bf16 values, each in a block whose scale it sets and in one
    whose maximum is 448 times a power of two next to it."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16)
    x = x[torch.isfinite(x)]
    rows = torch.zeros(x.numel(), 128, dtype=torch.bfloat16)
    rows[:, 5] = x
    rows2 = rows.clone()
    a = x.abs().double()
    near = torch.where((a > 1e-30) & (a < 1e30), a, torch.ones_like(a))
    rows2[:, 77] = (448 * 2.0 ** (torch.floor(torch.log2(near)) - 6)).to(
        torch.bfloat16)
    for r in (rows, rows2):
        q, s = narrow(r.shape[0], 128)
        cl.quantize_rows_t(r.to(DEV), q, s)
        qr, sr = ref.quantize(r, 1, 128)
        same(q.float(), qr)
        assert torch.equal(s[:, :1].cpu().long(), sr)


@pytest.mark.parametrize("k", [1, 3, 8])
def test_rows_by_position(cl, k):
    """A token goes to every row that it names; rows that none names stay."""
    T, C, P = 40, 300, 41 * k
    x = randn(T, C, seed=k).to(torch.bfloat16)
    g = torch.Generator().manual_seed(k)
    pos = torch.randperm(P, generator=g)[:T * k].view(T, k).int()
    pos[3] = -1
    pos[5, 0] = P  # out of range
    pos[6, k - 1] = -2 ** 31
    q, s = narrow(P, C)
    cl.quantize_rows_t(x.to(DEV), q, s, position=pos.to(DEV))
    qr, sr = ref.quantize(x, 1, 128)
    named = torch.zeros(P, dtype=torch.bool)
    for t in range(T):
        for j in range(k):
            p = int(pos[t, j])
            if 0 <= p < P:
                named[p] = True
                same(q[p, :C].float(), qr[t])
                assert torch.equal(s[p, :3].cpu().long(), sr[t])
    assert (q.view(torch.uint8).cpu()[~named] == 0xA5).all()
    assert (s.cpu()[~named] == 0xA5).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,N,C", [(1, 1, 1), (2, 128, 128), (3, 130, 257),
                                   (1, 300, 100), (2, 64, 700), (1, 513, 1)])
@pytest.mark.parametrize("both", [False, True])
def test_blocks(cl, dtype, E, N, C, both):
    w = torch.stack([hard_values(N, C, dtype, e + N) for e in range(E)])
    nb, cb = -(-N // 128), -(-C // 128)

    def buffers(rows, blocks, cols):
        q = torch.full((E, rows, 128 * cols), 0xA5, dtype=torch.uint8,
                       device=DEV).view(E4M3)
        return q, torch.full((E, blocks, -(-cols // 4) * 4), 0xA5,
                             dtype=torch.uint8, device=DEV)

    q, s = buffers(N, nb, cb)
    qt, st = buffers(C, cb, nb) if both else (None, None)
    cl.quantize_blocks_t(w.to(DEV), q, s, qt, st)
    for e in range(E):
        qr, sr = ref.quantize(w[e], 128, 128)
        same(q[e, :, :C].float(), qr)
        assert (q[e, :, C:].view(torch.uint8) == 0).all()
        assert torch.equal(s[e, :, :cb].cpu().long(), sr)
        assert (s[e, :, cb:] == 127).all()
        if both:
            same(qt[e, :, :N].float(), qr.t())
            assert (qt[e, :, N:].view(torch.uint8) == 0).all()
            assert torch.equal(st[e, :, :nb].cpu().long(), sr.t())
            assert (st[e, :, nb:] == 127).all()


def offsets_of(counts):
    return torch.tensor([0] + counts).cumsum(0).int()


COUNTS = [[1], [0, 1, 0], [128, 0, 129, 1], [0, 0], [300, 5, 0, 127, 260],
          [3] * 70, [0] * 100 + [200] + [0] * 30]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("C", [1, 100, 300])
@pytest.mark.parametrize("gather", [False, True])
def test_columns(cl, dtype, counts, C, gather):
    off = offsets_of(counts)
    held = int(off[-1])
    P = held + 5  # rows behind the last expert's are not read
    k = 3
    if gather:
        x = hard_values(17, C, dtype, 1)
        g = torch.Generator().manual_seed(2)
        src = torch.randint(0, 17 * k, (P,), generator=g).int()
        rows = x[(src // k).long()]
    else:
        x = hard_values(P, C, dtype, 1)
        src, rows = None, x
    L = cl.ciera_columns_length(P, len(counts)) + 128
    qt, st = narrow(C, L)
    cl.quantize_columns_t(x.to(DEV), off.to(DEV), qt, st,
                          source=None if src is None else src.to(DEV),
                          top_k=k if gather else 1)
    at = 0
    for e, n in enumerate(counts):
        end = at + -(-n // 128) * 128
        part = rows[off[e]:off[e + 1]]
        if n:
            qr, sr = ref.quantize(part, 128, 1)
            same(qt[:, at:at + n].float(), qr.t())
            assert (qt[:, at + n:end].contiguous().view(torch.uint8) == 0).all()
            assert torch.equal(st[:, at // 128:end // 128].cpu().long(),
                               sr.t())
        at = end
    assert (qt[:, at:].contiguous().view(torch.uint8) == 0xA5).all()
    assert (st[:, at // 128:] == 0xA5).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_every_value_rounds_right_in_columns(cl, dtype):
    """All finite 16-bit values (of fp32: bits at random, the upper half counted
    through), each in a column whose scale it sets, next to an infinity, and in one
    whose maximum is some powers of two larger."""
    bits = torch.arange(65536, dtype=torch.int64)
    if dtype == torch.float32:
        g = torch.Generator().manual_seed(1)
        bits = bits * 65536 + torch.randint(0, 65536, (65536,), generator=g)
        bits = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits)
        v = bits.to(torch.int32).view(dtype)
    else:
        v = bits.to(torch.int16).view(dtype)
    v = v[torch.isfinite(v)]
    n = v.numel()
    x = torch.zeros(3 * 130, n, dtype=dtype)
    x[5] = v
    x[130 + 127] = v
    x[130 + 8, ::2] = math.inf
    x[130 + 9, 1::3] = -math.inf
    x[260 + 64] = v
    a = v.abs().double()
    f = torch.finfo(dtype)
    x[260 + 77] = torch.where((a > 0) & (a < f.max / 2.0 ** 9), a * 2.0 ** 7,
                              a).to(dtype)
    off = torch.tensor([0, 130, 260, 390], dtype=torch.int32)
    qt, st = narrow(n, cl.ciera_columns_length(390, 3))
    cl.quantize_columns_t(x.to(DEV), off.to(DEV), qt, st)
    for e in range(3):
        qr, sr = ref.quantize(x[130 * e:130 * (e + 1)], 128, 1)
        same(qt[:, 256 * e:256 * e + 130].float(), qr.t())
        assert torch.equal(st[:, 2 * e:2 * e + 2].cpu().long(), sr.t())


# -------------------------------------------------------------- products ----

def whole_values(rows, cols, filled, seed, per_row=1):
    """Integers of -8 ... 8 as e4m3 (0 from cols on) and scales of 1/2, 1, 2."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(-8, 9, (rows, filled), generator=g).float()
    q[:, cols:] = 0
    s = torch.randint(126, 129, (-(-rows // per_row), -(-filled // 512) * 4),
                      generator=g).to(torch.uint8)
    return q.to(E4M3), s


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,N,D", [
    ([1], 1, 128), ([1], 200, 256), ([0, 1, 0], 64, 128), ([17], 16, 384),
    ([128, 0, 129, 1], 128, 640), ([0, 0], 130, 128),
    ([300, 5, 0, 127, 260], 257, 1024), ([3] * 70, 100, 256),
    ([0] * 100 + [200] + [0] * 30, 36, 512), ([1, 2, 3, 4, 0, 5, 1, 9], 511, 1920),
    ([2000, 700, 33], 700, 512),
    # results of whole octets: even, odd and few blocks of the depth, tiles cut in
    # rows and columns, experts without rows, several tiles a workgroup
    ([300, 5, 0, 127, 260], 264, 1024), ([1], 8, 512), ([0, 0], 128, 640),
    ([256, 255, 257], 256, 640), ([70, 0, 513], 1096, 896),
    ([40] * 90, 1032, 512), ([0] * 100 + [200] + [0] * 30, 40, 2176),
    ([1500, 0, 900, 257], 1032, 640), ([2000, 700, 33], 704, 1024),
    ([0] * 10 + [2000] + [0] * 3, 1032, 2176), ([5000, 3200], 2052, 128),
    ([60] * 8, 300, 3200)])
def test_matmul(cl, dtype, counts, N, D):
    off = offsets_of(counts)
    E, held = len(counts), int(off[-1])
    P = held + 3
    a, sa = whole_values(P, D - 5, D, 1)
    b, sb = zip(*[whole_values(N, D - 5, D, 2 + e, 128) for e in range(E)])
    out = torch.full((P, N), 77.0, dtype=dtype, device=DEV)
    cl.expert_matmul_t(a.to(DEV), sa.to(DEV), torch.stack(b).to(DEV),
                       torch.stack(sb).to(DEV), off.to(DEV), out)
    torch.cuda.synchronize()
    av = ref.values(a, sa, 1, 128)
    for e in range(E):
        r = slice(int(off[e]), int(off[e + 1]))
        y = av[r] @ ref.values(b[e], sb[e], 128, 128).t()
        same(out[r], y.to(dtype))
    assert (out[held:] == 77).all()


@pytest.mark.parametrize("P", [1, 2, 16, 17, 100, 513])
def test_matmul_of_one_expert_without_offsets(cl, P):
    N, D = 300, 768
    a, sa = whole_values(P, D, D, 1)
    b, sb = whole_values(N, D, D, 2, 128)
    out = torch.empty(P, N, device=DEV)
    cl.expert_matmul_t(a.to(DEV), sa.to(DEV), b[None].to(DEV),
                       sb[None].to(DEV), None, out)
    same(out, ref.values(a, sa, 1, 128) @ ref.values(b, sb, 128, 128).t())


def test_matmul_strided_and_unaligned_output(cl):
    """Rows of wider buffers: the operand's, its scales' and the output's, whose
    rows start at odd places."""
    P, N, D = 37, 61, 256
    a, sa = whole_values(P, D, D, 1)
    b, sb = whole_values(N, D, D, 2, 128)
    wide = torch.zeros(P, D + 144, dtype=torch.uint8, device=DEV)
    wide[:, 16:16 + D] = a.view(torch.uint8).to(DEV)
    ws = torch.zeros(P, 12, dtype=torch.uint8, device=DEV)
    ws[:, 4:8] = sa.to(DEV)
    y = ref.values(a, sa, 1, 128) @ ref.values(b, sb, 128, 128).t()
    for dtype in TYPES:
        out = torch.full((P, N + 6), 5.0, dtype=dtype, device=DEV)
        cl.expert_matmul_t(wide[:, 16:16 + D].view(E4M3), ws[:, 4:8],
                           b[None].to(DEV), sb[None].to(DEV), None,
                           out[:, 3:3 + N])
        same(out[:, 3:3 + N], y.to(dtype))
        assert (out[:, :3] == 5).all() and (out[:, 3 + N:] == 5).all()


def test_matmul_scales_far_from_one(cl):
    """Scale bytes whose products stay within fp32, to both sides."""
    P, N, D = 16, 16, 256
    a, _ = whole_values(P, D, D, 1)
    b, _ = whole_values(N, D, D, 2, 128)
    for ea, eb in ((-100, 90), (100, -90), (50, 60), (-60, -40), (-127, 120),
                   (120, -127)):
        sa = torch.full((P, 4), ea + 127, dtype=torch.uint8)
        sb = torch.full((1, 4), eb + 127, dtype=torch.uint8)
        out = torch.empty(P, N, device=DEV)
        cl.expert_matmul_t(a.to(DEV), sa.to(DEV), b[None].to(DEV),
                           sb[None].to(DEV), None, out)
        same(out, ref.values(a, sa, 1, 128) @ ref.values(b, sb, 128, 128).t())


def test_matmul_nan_stays_in_its_row(cl):
    P, N, D = 40, 130, 256
    a, sa = whole_values(P, D, D, 1)
    a = a.float()
    a[7, 200] = math.nan
    a = a.to(E4M3)
    b, sb = whole_values(N, D, D, 2, 128)
    out = torch.empty(P, N, device=DEV)
    cl.expert_matmul_t(a.to(DEV), sa.to(DEV), b[None].to(DEV),
                       sb[None].to(DEV), None, out)
    bad = torch.isnan(out).cpu()
    assert bad[7].all() and int(bad.sum()) == N


def test_matmul_of_random_values(cl):
    """Sums that round: D fp32 roundings (or truncations, 2^-23) of partial
    sums of at most sum |a b|."""
    P, N, D = 64, 256, 2048
    x, w = randn(P, D, seed=1), randn(N, D, seed=2, std=0.02)
    a, sa = narrow(P, D)
    cl.quantize_rows_t(x.to(DEV), a, sa)
    b, sb = narrow(N, D)
    sb = torch.empty(1, N // 128, D // 128, dtype=torch.uint8, device=DEV)
    cl.quantize_blocks_t(w[None].to(DEV), b[None], sb)
    out = torch.empty(P, N, device=DEV)
    cl.expert_matmul_t(a, sa, b[None], sb, None, out)
    av, bv = ref.values(a, sa, 1, 128), ref.values(b, sb[0], 128, 128)
    bound = D * 2.0 ** -23 * (av.abs() @ bv.abs().t())
    assert ((out.cpu().double() - av @ bv.t()).abs() <= bound).all()


def test_fp32_results_keep_small_products(cl):
    """A product of 2^16 and one of 2^-6 next to it: 23 bits that an fp32 sum
    holds. With neighbours of every distance within a block of 128."""
    D = 128
    a = torch.zeros(D - 1, D)
    for j in range(1, D):
        a[j - 1, 0], a[j - 1, j] = 256.0, 0.125
    b = torch.full((1, D), 0.125)
    b[0, 0] = 256.0
    one = torch.full((D - 1, 4), 127, dtype=torch.uint8, device=DEV)
    out = torch.empty(D - 1, 1, device=DEV)
    cl.expert_matmul_t(a.to(E4M3).to(DEV), one, b[None].to(E4M3).to(DEV),
                       one[:1, None].contiguous(), None, out)
    assert (out == 65536.0 + 2.0 ** -6).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,N,C", [
    ([1], 1, 1), ([0, 1, 0], 100, 130), ([128, 0, 129, 1], 129, 64),
    ([0, 0], 20, 30), ([300, 5, 0, 127, 260], 257, 300), ([3] * 70, 33, 40),
    ([700], 256, 384)])
def test_weight_grad(cl, dtype, counts, N, C):
    off = offsets_of(counts)
    E = len(counts)
    L = cl.ciera_columns_length(int(off[-1]) + 4, E) + 128

    def columns(rows, seed):
        g = torch.Generator().manual_seed(seed)
        q = torch.randint(-8, 9, (rows, L), generator=g).float()
        at = 0
        for n in counts:
            end = at + -(-n // 128) * 128
            q[:, at + n:end] = 0
            at = end
        q[:, at:] = math.nan  # nothing behind the last expert counts
        s = torch.randint(126, 129, (rows, -(-L // 512) * 4),
                          generator=g).to(torch.uint8)
        return q.to(E4M3), s

    dy, sdy = columns(N, 1)
    x, sx = columns(C, 2)
    dw = torch.full((E, N, C), 9.0, dtype=dtype, device=DEV)
    cl.expert_weight_grad_t(dy.to(DEV), sdy.to(DEV), x.to(DEV), sx.to(DEV),
                            off.to(DEV), dw)
    dyv, xv = ref.values(dy, sdy, 1, 128), ref.values(x, sx, 1, 128)
    at = 0
    for e, n in enumerate(counts):
        same(dw[e], (dyv[:, at:at + n] @ xv[:, at:at + n].t()).to(dtype))
        at += -(-n // 128) * 128


# --------------------------------------------------------------- combine ----

def positions(T, k, P, seed):
    g = torch.Generator().manual_seed(seed)
    pos = torch.full((T * k,), -1)
    n = min(T * k, P)
    at = torch.randperm(T * k, generator=g)[:n]
    pos[at] = torch.randperm(P, generator=g)[:n]
    return pos.view(T, k).int()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,P,C", [(1, 1, 1, 1), (1, 8, 8, 2048),
                                     (9, 8, 40, 7), (33, 3, 99, 513),
                                     (5, 64, 320, 100), (70, 2, 100, 4099)])
def test_combine(cl, dtype, T, k, P, C):
    rows = randn(P, C, seed=1).to(dtype)
    w = randn(T, k, seed=2)
    pos = positions(T, k, P, 3)
    pos[0, 0] = -1 if T > 1 else pos[0, 0]
    if T > 4:
        pos[4, k - 1] = P
    held = ((pos >= 0) & (pos < P)).double()
    r = rows.double()[pos.long().clamp(0, P - 1)]
    for weights in (w, None):
        out = torch.full((T, C), 3.0, dtype=dtype, device=DEV)
        cl.combine_t(rows.to(DEV), pos.to(DEV), out,
                     weights=None if weights is None else w.to(DEV))
        f = held if weights is None else held * w.double()
        y = (r * f.unsqueeze(2)).sum(1)
        size = (r.abs() * f.abs().unsqueeze(2)).sum(1)
        # k multiply-adds in fp32, then one rounding
        bound = k * 2.0 ** -23 * size + torch.finfo(dtype).eps / 2 * y.abs()
        if dtype == torch.float16:
            bound = bound + 2.0 ** -25
        assert ((out.cpu().double() - y).abs() <= bound).all()


def test_combine_nan_weight(cl):
    rows = randn(6, 20, seed=1).to(DEV)
    pos = torch.tensor([[0, 1], [-1, 2], [-1, -1]], dtype=torch.int32)
    w = torch.tensor([[1.0, 2.0], [math.nan, 1.0], [0.5, 0.5]])
    out = torch.empty(3, 20, device=DEV)
    cl.combine_t(rows, pos.to(DEV), out, weights=w.to(DEV))
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all()
    assert (out[2] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,P,C", [(1, 1, 1, 1), (1, 8, 8, 2048),
                                     (9, 8, 40, 7), (33, 3, 99, 513),
                                     (5, 64, 320, 100), (30, 2, 60, 4099)])
def test_combine_backward(cl, dtype, T, k, P, C):
    rows = randn(P, C, seed=1).to(dtype)
    w, g = randn(T, k, seed=2), randn(T, C, seed=4).to(dtype)
    pos = positions(T, k, P, 3)
    if T > 4:
        pos[4, 0] = P
    d_rows = torch.full((P, C), 5.0, dtype=dtype, device=DEV)
    d_w = torch.full((T, k), 5.0, device=DEV)
    cl.combine_backward_t(g.to(DEV), rows.to(DEV), w.to(DEV), pos.to(DEV),
                          d_rows, d_w)
    expect = torch.full((P, C), 5.0, dtype=torch.float64)
    named = torch.zeros(P, dtype=torch.bool)
    for t in range(T):
        for j in range(k):
            p = int(pos[t, j])
            if not 0 <= p < P:
                assert d_w[t, j] == 0
                continue
            expect[p] = w[t, j].double() * g[t].double()
            named[p] = True
            dot = (g[t].double() * rows[p].double()).sum()
            size = (g[t].double() * rows[p].double()).abs().sum()
            # C multiply-adds in fp32 over at least 64 lanes: C / 64 + 8
            # of them one after the other
            assert abs(float(d_w[t, j]) - float(dot)) <= \
                (C / 64 + 16) * 2.0 ** -23 * float(size)
    # The product is rounded to fp32 and then to its type, or to its type at once
    # (the multiply-add of fp16): y (1 + a)(1 + b) with |a| <= 2^-24 and |b| <=
    # eps / 2, so |error| <= |y| (eps / 2 + 2^-24 (1 + eps / 2)), or, below
    # fp16's normal values, half a step of 2^-24 and 2^-24 |y|.
    half = torch.finfo(dtype).eps / 2
    bound = expect.abs() * (half + 2.0 ** -24 * (1 + half))
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25
    got = d_rows.cpu().double()
    assert ((got - expect).abs()[named] <= bound[named]).all()
    assert (got[~named] == 5).all()


def test_combine_of_differences(cl):
    """<d_out, combine> changes with rows and weights as the gradients say: it
    is linear in each, so differences are exact but for fp32's roundings."""
    T, k, P, C = 6, 3, 14, 50
    rows, w = randn(P, C, seed=1), randn(T, k, seed=2)
    pos, g = positions(T, k, P, 3), randn(T, C, seed=4)
    d_rows = torch.zeros(P, C, device=DEV)
    d_w = torch.zeros(T, k, device=DEV)
    cl.combine_backward_t(g.to(DEV), rows.to(DEV), w.to(DEV), pos.to(DEV),
                          d_rows, d_w)

    def loss(rows, w):
        out = torch.empty(T, C, device=DEV)
        cl.combine_t(rows.to(DEV), pos.to(DEV), out, weights=w.to(DEV))
        return float((out.cpu().double() * g.double()).sum())

    base = loss(rows, w)
    for i in range(4):
        dr, dw = randn(P, C, seed=20 + i), randn(T, k, seed=30 + i)
        moved = loss(rows + dr, w) - base
        expect = float((d_rows.cpu().double() * dr.double()).sum())
        assert abs(moved - expect) <= 1e-3 * T * C ** 0.5
        moved = loss(rows, w + dw) - base
        expect = float((d_w.cpu().double() * dw.double()).sum())
        assert abs(moved - expect) <= 1e-3 * T * C ** 0.5


# -------------------------------------------------------------- refusals ----

def test_tensors_that_do_not_fit(cl):
    """Every call names the tensor that does not fit; nothing is enqueued."""
    T, k, E, C, P = 4, 2, 3, 256, 8
    f = torch.zeros(T, C, device=DEV)
    i = torch.zeros(T, k, dtype=torch.int32, device=DEV)
    w = torch.zeros(T, k, device=DEV)
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    rows = torch.zeros(P, C, device=DEV)
    q, s = narrow(P, C)
    b = torch.zeros(E, 128, C, device=DEV).to(E4M3)
    sb = torch.zeros(E, 1, 4, dtype=torch.uint8, device=DEV)
    qt, st = narrow(C, 512)
    dw = torch.zeros(E, C, C, device=DEV)
    out = torch.zeros(P, 128, device=DEV)
    bad = [
        ("weights has type", lambda: cl.route_t(f, i, w.half())),
        ("weights has shape", lambda: cl.route_t(f, i, w[:3])),
        ("expert_ids has type", lambda: cl.route_t(f, i.long(), w)),
        ("logits is not contiguous", lambda: cl.route_t(f.t()[:T], i, w)),
        ("logits is not contiguous",
         lambda: cl.route_t(f[:1].expand(T, C), i, w)),
        ("bias has shape", lambda: cl.route_t(f, i, w, bias=f[0, :5])),
        ("bias is on cpu", lambda: cl.route_t(f, i, w, bias=torch.zeros(C))),
        ("d_logits has type",
         lambda: cl.route_backward_t(f, i, w, f.half())),
        ("offsets has shape", lambda: cl.route_plan_t(
            i, E, off[:3], i.view(-1), i, cl.PlanWorkspace(T, k, E))),
        ("position has shape",
         lambda: cl.quantize_rows_t(f, q, s, position=i[:2])),
        ("q has shape", lambda: cl.quantize_rows_t(f[:, :100], q, s)),
        ("do not fit", lambda: cl.quantize_rows_t(f, q, s[:, :1].contiguous())),
        ("w is not contiguous",
         lambda: cl.quantize_blocks_t(dw.transpose(1, 2), b, sb)),
        ("go together",
         lambda: cl.quantize_blocks_t(dw, b, sb, q_t=b)),
        ("offsets has shape",
         lambda: cl.quantize_columns_t(rows, off[:1], qt, st)),
        ("scales of b has shape",
         lambda: cl.expert_matmul_t(q, s, b, sb[:2], off, out)),
        ("out has shape", lambda: cl.expert_matmul_t(q, s, b, sb, off, rows)),
        ("offsets has type",
         lambda: cl.expert_matmul_t(q, s, b, sb, off.long(), out)),
        ("x_t has shape",
         lambda: cl.expert_weight_grad_t(qt, st, qt[:5], st, off, dw)),
        ("out has type",
         lambda: cl.combine_t(rows, i, f.half())),
        ("d_rows has shape",
         lambda: cl.combine_backward_t(f, rows, w, i, rows[:3], w)),
    ]
    for what, call in bad:
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(cl.CieraError):  # one expert's rows need no offsets
        cl.expert_matmul_t(q, s, b, sb, None, out)
    with pytest.raises(cl.CieraError):  # more experts a token than experts
        cl.route_t(f[:, :1].contiguous(), i, w)


def test_one_column_and_one_row_views(cl):
    """Matrices of one column or row keep their strides."""
    wide = randn(6, 9, seed=1).to(DEV)
    pos = torch.arange(6, dtype=torch.int32, device=DEV).view(3, 2)
    out = torch.full((3, 4), 7.0, device=DEV)
    cl.combine_t(wide[:, 2:3], pos, out[:, 1:2])
    y = wide[:, 2].view(3, 2).sum(1)
    assert torch.equal(out[:, 1], y) and (out[:, 0] == 7).all()
    assert (out[:, 2:] == 7).all()
