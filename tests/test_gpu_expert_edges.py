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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_grad_of_offsets_that_start_late(cl, dtype):
    """The experts' columns alone, of rows that lie behind many others."""
    N, C, counts = 24, 40, [100, 0, 200]
    off = torch.tensor([5000] + counts).cumsum(0).int()
    L = cl.ciera_columns_length(300, 3)
    g = torch.Generator().manual_seed(3)
    dy = torch.randint(-4, 5, (N, L), generator=g).float()
    x = torch.randint(-4, 5, (C, L), generator=g).float()
    one = torch.full((C, 8), 127, dtype=torch.uint8, device=DEV)
    dw = torch.full((3, N, C), 9.0, dtype=dtype, device=DEV)
    cl.expert_weight_grad_t(dy.to(E4M3).to(DEV), one[:N].contiguous(),
                            x.to(E4M3).to(DEV), one, off.to(DEV), dw)
    for e, part in enumerate((slice(0, 128), slice(0, 0), slice(128, 384))):
        expect = dy[:, part] @ x[:, part].t()
        assert torch.equal(dw[e].cpu(), expect.to(dtype)), e


# ------------------------------------------------------- saturated scores ----

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16,
                                   torch.float32])
@pytest.mark.parametrize("times", [1, 90])  # 90: several tokens share a wave
@pytest.mark.parametrize("normalize", [False, True])
def test_gradient_of_saturated_sigmoids(cl, dtype, times, normalize):
    """c s (1 - s) g relative to its own size, for logits of -30 to 30. s and 1 - s
    are each an exponential (its argument is the logit itself; 1 ulp), a sum and a
    division (2.5 ulp at most): 4 ulps of 2^-23. Scale, two products: 1.5 more. Two
    chosen logits that are equal have weights of a half each (their scores are
    the same number) and, with gradients g and -g, a mean of 0."""
    l = torch.linspace(-30, 30, 61).to(dtype).view(-1, 1).repeat(times, 2)
    T = l.shape[0]
    k = 2 if normalize else 1
    ids = torch.arange(k, dtype=torch.int32).repeat(T, 1)
    g = randn(T, 1, seed=1)
    dw = torch.cat([g, -g], 1)[:, :k].contiguous()
    d = torch.full((T, 2), 7.0, dtype=dtype, device=DEV)
    cl.route_backward_t(l.to(DEV), ids.to(DEV), dw.to(DEV), d, sigmoid=True,
                        normalize=normalize, scale=2.5)
    x, g = l[:, 0].double(), 2.5 * g[:, 0].double()
    rest = 1 / (1 + torch.exp(x))
    exact = rest * g * (0.5 if normalize else 1 / (1 + torch.exp(-x)))
    bound = exact.abs() * (9.5 * 2.0 ** -23 + torch.finfo(dtype).eps / 2)
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25  # half a step of its subnormal values
    d = d.double().cpu()
    assert ((d[:, 0] - exact).abs() <= bound).all()
    if normalize:
        assert ((d[:, 1] + exact).abs() <= bound).all()
    else:
        assert (d[:, 1] == 0).all()


@pytest.mark.parametrize("times", [1, 1100])  # 1100: several tokens share a wave
@pytest.mark.parametrize("o", [dict(), dict(normalize=True),
                               dict(sigmoid=True),
                               dict(sigmoid=True, normalize=True)])
def test_gradient_of_slots_without_an_expert(cl, o, times):
    """Slots whose id is out of range add nothing, whatever their weight's gradient
    is: the bits are those of gradients of 0 there."""
    E, k = 20, 4
    l = randn(4, E, seed=1).repeat(times, 1).to(DEV)
    ids = torch.tensor([[3, -1, 7, 20], [-1, -1, -1, -1], [0, 19, -5, 2],
                        [1, 2, 3, 4]], dtype=torch.int32)
    dw = randn(4, k, seed=2)
    clean = torch.where((ids >= 0) & (ids < E), dw, torch.zeros(4, k))
    for bad in (math.nan, math.inf, -math.inf):
        got = []
        for g in (torch.where(clean == 0, torch.full_like(dw, bad), dw), clean):
            d = torch.full_like(l, 7.0)
            cl.route_backward_t(l, ids.repeat(times, 1).to(DEV),
                                g.repeat(times, 1).to(DEV), d, **o)
            got.append(d)
        assert torch.isfinite(got[0]).all()
        assert torch.equal(got[0], got[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16,
                                   torch.float32])
@pytest.mark.parametrize("times", [1, 110])  # 110: several tokens share a wave
@pytest.mark.parametrize("o", [dict(), dict(normalize=True),
                               dict(sigmoid=True, normalize=True)])
def test_gradient_of_saturated_weights(cl, dtype, times, o):
    """One score of nearly 1, by a logit of 0 to 40 above the others, relative to the
    gradients' own size. An exponential is off by 1 ulp of 2^-23, a sum of the seven
    others by 3 more, of all by half, a division by 2.5: a score by 8 ulps, the
    others' share by 11. 1 - s of a sigmoid is off by 4. The slots' gradients have
    opposite signs, so that no difference between them is smaller than they are, and
    the mean's error is at most its 9 ulps: with products and the scale 40 in all."""
    E, scale = 8, 2.5
    t = torch.arange(41).double().repeat(times)
    T = t.numel()
    l = torch.zeros(T, E, dtype=torch.float64)
    l[:, 5] = t  # whole numbers to 40, which every type holds
    k = 2 if o.get("normalize") else 1
    ids = torch.tensor([5, 2][:k], dtype=torch.int32).repeat(T, 1)
    a, b = randn(T, 1, seed=1).abs() + 0.1, -randn(T, 1, seed=2).abs() - 0.1
    dw = torch.cat([a, b], 1)[:, :k].contiguous()
    d = torch.full((T, E), 7.0, dtype=dtype, device=DEV)
    cl.route_backward_t(l.to(dtype).to(DEV), ids.to(DEV), dw.to(DEV), d,
                        scale=scale, **o)
    a, b = scale * a[:, 0].double(), scale * b[:, 0].double()
    exact = torch.zeros(T, E, dtype=torch.float64)
    if not o:
        p = 1 / (1 + 7 * torch.exp(-t))
        q = torch.exp(-t) * p
        exact[:] = (-q * p * a).unsqueeze(1)
        exact[:, 5] = p * 7 * q * a
    else:
        s, r = 1 / (1 + torch.exp(-t)), 1 / (1 + torch.exp(t))
        if o.get("sigmoid"):
            w = 0.5 / (s + 0.5)  # the other's score is 1/2
            exact[:, 5] = (1 - w) * r * w * (a - b)
            exact[:, 2] = -w * 0.5 * (1 - w) * (a - b)
        else:
            exact[:, 5] = s * r * (a - b)
            exact[:, 2] = -exact[:, 5]
    bound = exact.abs() * (40 * 2.0 ** -23 + torch.finfo(dtype).eps / 2)
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25  # half a step of its subnormal values
    assert ((d.double().cpu() - exact).abs() <= bound).all()


@pytest.mark.parametrize("times", [1, 1500])
@pytest.mark.parametrize("o", [dict(), dict(normalize=True)])
def test_gradient_of_the_largest_score_named_twice(cl, o, times):
    """Twice in the slots, or equal to another's, or with every score chosen: the
    derivative in 64 bits, off by some 20 ulps of the largest term."""
    l = torch.tensor([[9.0, 1.0, 0.0, 2.0], [3.0, 3.0, 3.0, -1.0],
                      [-math.inf, 5.0, -math.inf, 5.0]])
    ids = torch.tensor([[0, 0, 2, 0], [1, 0, 1, 3], [3, 1, 3, 1]])
    dw = randn(3, 4, seed=4)
    d = torch.full((3 * times, 4), 7.0, device=DEV)
    cl.route_backward_t(l.repeat(times, 1).to(DEV),
                        ids.int().repeat(times, 1).to(DEV),
                        dw.repeat(times, 1).to(DEV), d, **o)
    x = l.double().clamp(min=-2000).requires_grad_()
    (ref.weights_of(x, ids, False, o.get("normalize", False), 1.0) *
     dw.double()).sum().backward()
    bound = 4 * 20 * 2.0 ** -23 * float(dw.abs().max())
    assert ((d.double().cpu() - x.grad.repeat(times, 1)).abs() <= bound).all()


# ------------------------------------------------------- the layer's inputs ----

def layer(*args, **o):
    from paper_2609_04609_amd.experts import ExpertLayer
    return ExpertLayer(*args, **o)


@pytest.mark.parametrize("dtype,other", [
    (torch.bfloat16, torch.float32), (torch.bfloat16, torch.float16),
    (torch.float16, torch.float32), (torch.float32, torch.bfloat16)])
def test_layer_with_logits_of_another_type(cl, dtype, other):
    """A router in fp32 beside 16-bit tokens, and others. With logits that both types
    hold everything has the bits of logits of the layer's type, and the
    logits' gradient is the same fp32 number, rounded to their type."""
    T, k, E, N, C = 70, 3, 12, 64, 136
    m = layer(T, k, E, N, C, dtype=dtype, sigmoid=True, normalize=True)
    m.load(randn(E, N, C, seed=1).to(dtype).to(DEV))
    x, g = (randn(T, n, seed=n).to(dtype).to(DEV) for n in (C, N))
    l = (randn(T, E, seed=3) * 64).round() / 64  # some 8 bits
    l = l.to(torch.bfloat16).to(torch.float16)
    runs = []
    for t in (other, dtype, other):
        y = m.forward(x, l.to(t).to(DEV))
        grads = m.backward(g, x, l.to(t).to(DEV))
        assert grads[2].dtype == t and grads[2] is m.d_logits
        runs.append([v.clone() for v in (y,) + grads])
    for a, b in zip(runs[0], runs[2]):
        assert torch.equal(a, b)
    for a, b in zip(runs[0][:3], runs[1][:3]):
        assert torch.equal(a, b)
    a, b = runs[0][3], runs[1][3]
    wide, narrow = (a, b) if a.dtype == torch.float32 else (b, a)
    if torch.float32 in (dtype, other):
        assert torch.equal(wide.to(narrow.dtype), narrow)
    assert float(a.float().abs().sum()) > 0


def test_layer_refuses_before_it_runs(cl):
    """An input that an operator in the middle of a call would refuse leaves the
    layer's buffers as they were."""
    T, k, E, N, C = 9, 2, 4, 40, 50
    m = layer(T, k, E, N, C)
    m.load(randn(E, N, C, seed=1).bfloat16().to(DEV))
    x, g = (randn(T, n, seed=n).bfloat16().to(DEV) for n in (C, N))
    l = randn(T, E, seed=3).to(DEV)
    y = m.forward(x, l)
    m.backward(g, x, l)
    kept = [m.ids, m.weights, m.position, m.x, m.out, m.d_rows, m.d_weights,
            m.d_x, m.d_w, m.d_logits]
    before = [t.view(torch.uint8).clone() if t.dtype == E4M3 else t.clone()
              for t in kept]
    new = randn(T, E, seed=4).to(DEV)
    bad = [
        ("x has type", lambda: m.forward(x.int(), new)),
        ("x is on cpu", lambda: m.forward(x.cpu(), new)),
        ("x is not contiguous", lambda: m.forward(x.t().contiguous().t(), new)),
        ("logits has type", lambda: m.forward(x, new.double())),
        ("d_out has type", lambda: m.backward(g.float(), x, new)),
        ("x has type", lambda: m.backward(2 * g, x.double(), new)),
        ("logits has type", lambda: m.backward(2 * g, x, new.double())),
        ("logits is on cpu", lambda: m.backward(2 * g, x, new.cpu())),
        ("logits is not contiguous",
         lambda: m.backward(2 * g, x, new.t().contiguous().t())),
    ]
    for what, call in bad:
        with pytest.raises(ValueError, match=what):
            call()
    torch.cuda.synchronize()
    for t, b in zip(kept, before):
        t = t.view(torch.uint8) if t.dtype == E4M3 else t
        assert torch.equal(t, b)
    assert m.out is y


@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, torch.float32),
                                        (torch.float16, torch.float32),
                                        (torch.float32, torch.bfloat16)])
def test_layer_with_weight_gradients_of_another_type(cl, dtype, grad):
    """Everything else has the bits of a layer without; the gradients are those of
    the 8-bit operands that the layer left, off by a rounding of 2^-23 for each of n
    sums (16-bit ones by the half step and 2^-10 of the products' sizes)."""
    T, k, E, N, C = 90, 3, 5, 72, 136
    args = [randn(T, C, seed=1).to(dtype), randn(T, E, seed=2).to(dtype),
            randn(T, N, seed=3).to(dtype)]
    x, l, g = (t.to(DEV) for t in args)
    w = randn(E, N, C, seed=4).to(dtype).to(DEV)
    runs = []
    for o in (dict(grad_dtype=grad), dict()):
        m = layer(T, k, E, N, C, dtype=dtype, normalize=True, **o)
        m.load(w)
        runs.append([m, m.forward(x, l)] + list(m.backward(g, x, l)))
    (m, y, d_x, d_w, d_l), other = runs
    assert d_w.dtype == grad and other[3].dtype == dtype
    for a, b in ((y, other[1]), (d_x, other[2]), (d_l, other[4])):
        assert torch.equal(a, b)
    off, start = m.offsets.tolist(), 0
    half = torch.finfo(grad).eps / 2
    for e in range(E):
        n = off[e + 1] - off[e]
        end = start + -(-n // 128) * 128
        at = slice(start // 128, end // 128)
        a = ref.values(m.dy_t[:, start:end], m.dy_t_scales[:, at], 1, 128)
        b = ref.values(m.x_t[:, start:end], m.x_t_scales[:, at], 1, 128)
        size = a.abs() @ b.abs().t()
        bound = half * (a @ b.t()).abs() + n * 2.0 ** -23 * size
        if grad != torch.float32:
            bound = bound + 2.0 ** -10 * size
        assert ((d_w[e].double().cpu() - a @ b.t()).abs() <= bound).all()
        start = end


# ---------------------------------------------------- groups and far biases ----

@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,G,far", [(64, 32, 1000.0), (64, 16, 1000.0),
                                     (60, 20, 1000.0), (256, 32, 3000.0)])
def test_groups_whose_two_values_cancel(cl, E, G, far, sigmoid):
    """Groups rank by the sum of two values of some +far and -far, each of which is
    held to 2^-24 of far, so that ranks a thousandth apart may be in the wrong order
    in fp32. Few and many tokens; chosen as 64 bits choose."""
    T, k, S = 60_000, 4, E // G
    l = randn(T, E, seed=E)
    bias = randn(E, seed=G, std=0.02) - 4 * far
    bias[0::S] += 5 * far
    bias[1::S] += 3 * far
    s = torch.sigmoid(l.double()) if sigmoid else torch.softmax(l.double(), 1)
    v = s + bias.double()
    rank = v.view(T, G, S)[:, :, :2].sum(2)
    kept = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :5]
    out = torch.ones(T, G, dtype=torch.bool).scatter_(1, kept, False)
    v = v.masked_fill(out.repeat_interleave(S, 1), -math.inf)
    expect = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    l, bias = l.to(DEV), bias.to(DEV)
    for n in (T, 4000):
        ids = torch.full((T, k), -7, dtype=torch.int32, device=DEV)
        w = torch.empty(T, k, device=DEV)
        for at in range(0, T, n):
            cl.route_t(l[at:at + n], ids[at:at + n], w[at:at + n], bias=bias,
                       groups=G, top_groups=5, group_top_two=True,
                       sigmoid=sigmoid)
        assert torch.equal(ids.cpu().long(), expect)


@pytest.mark.parametrize("T", [1, 5000])
def test_group_sums_past_fp32(cl, T):
    """Two finite biases whose sum no float holds."""
    l = torch.zeros(T, 12, device=DEV)
    b = torch.tensor([2e38, 2.1e38, 0, 0, 3e38, 2.9e38, 0, 0, -3e38, -2e38,
                      -3.1e38, -2.2e38], device=DEV)
    ids = torch.full((T, 2), -7, dtype=torch.int32, device=DEV)
    w = torch.empty(T, 2, device=DEV)
    cl.route_t(l, ids, w, bias=b, groups=3, top_groups=1, group_top_two=True)
    assert (ids == torch.tensor([4, 5], device=DEV)).all()
    b = b - 0.0
    b[:8] = torch.tensor([-3e38, -2.9e38, -3.1e38, -3.2e38] * 2)
    b[4] = -2.8e38
    b[8:] = b[0]
    # sums -5.9e38, -5.7e38, -6e38; of the first two groups -2.8e38 is the highest,
    # then -2.9e38, which experts 1 and 5 have
    cl.route_t(l, ids, w, bias=b, groups=3, top_groups=2, group_top_two=True)
    assert (ids == torch.tensor([4, 1], device=DEV)).all()


@pytest.mark.parametrize("E", [64, 256, 1024])
def test_close_softmax_scores_beside_a_large_one(cl, E):
    """One score ahead of many that are all but equal, where the sum's own error is
    the largest: scores some 2^-20 of themselves apart, with biases that order
    them by halves of that. Chosen as 64 bits choose, few and many tokens."""
    T, k = 4200, 7
    l = randn(T, E, seed=E) * 2.0 ** -20
    l[:, 3] = torch.linspace(0, 11, T)
    bias = randn(E, seed=1) * 2.0 ** -21 / E
    v = torch.softmax(l.double(), 1) + bias.double()
    expect = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    l, bias = l.to(DEV), bias.to(DEV)
    for n in (T, 600):
        ids = torch.full((T, k), -7, dtype=torch.int32, device=DEV)
        w = torch.empty(T, k, device=DEV)
        for at in range(0, T, n):
            cl.route_t(l[at:at + n], ids[at:at + n], w[at:at + n], bias=bias)
        assert torch.equal(ids.cpu().long(), expect)


# ------------------------------------------------------------------- sizes ----

def test_few_rows_of_wide_weights(cl):
    """131 GB of weights, for whose columns the kernel of few rows would need 2^32
    threads and more: another takes them."""
    if torch.cuda.get_device_properties(0).total_memory < 200 << 30:
        pytest.skip("less than 200 GiB of memory")
    E, N, D, P = 1024, 1_000_003, 128, 2048
    w = torch.zeros(E, N, D, dtype=torch.uint8, device=DEV)
    g = torch.Generator().manual_seed(1)
    last = torch.randint(-8, 9, (300, D), generator=g).float()
    w[-1, -300:] = last.to(E4M3).view(torch.uint8).to(DEV)
    a = torch.randint(-8, 9, (P, D), generator=g).float()
    sa = torch.full((P, 4), 127, dtype=torch.uint8, device=DEV)
    sb = torch.full((E, -(-N // 128), 4), 127, dtype=torch.uint8, device=DEV)
    off = torch.arange(0, P + 1, 2, dtype=torch.int32)  # two rows an expert
    out = torch.full((P, N), 7.0, dtype=torch.bfloat16, device=DEV)
    cl.expert_matmul_t(a.to(E4M3).to(DEV), sa, w.view(E4M3), sb, off.to(DEV),
                       out)
    expect = (a[-2:] @ last.t()).bfloat16()  # whole numbers below 2^24
    assert torch.equal(out[-2:, -300:].cpu(), expect)
    assert (out[-2:, :-300] == 0).all()
    for rows in out[:-2].split(256):
        assert not rows.any()
    del w, out, rows
    torch.cuda.empty_cache()


def test_plan_of_the_last_experts(cl):
    """Ids up to 2^31 - 1, beside negative ones whose difference wraps."""
    E, first = 8, 2 ** 31 - 8
    ids = torch.tensor([[2 ** 31 - 1, -1], [-2 ** 31, 2 ** 31 - 8],
                        [-2 ** 31 + 3, 2 ** 31 - 2], [0, 2 ** 31 - 8]])
    off = torch.full((E + 1,), -9, dtype=torch.int32, device=DEV)
    src = torch.full((8,), -9, dtype=torch.int32, device=DEV)
    pos = torch.full((4, 2), -9, dtype=torch.int32, device=DEV)
    cl.route_plan_t(ids.int().to(DEV), E, off, src, pos,
                    cl.PlanWorkspace(4, 2, E), first_expert=first)
    o, s, p = ref.plan(ids, E, first)
    assert torch.equal(off.cpu().long(), o)
    assert torch.equal(src.cpu().long(), s)
    assert torch.equal(pos.cpu().long(), p)
