"""Routing to experts, its gradient and the plan against 64-bit definitions
(tests/expert_ref.py): ids and plans exactly, weights and gradients within
bounds that count fp32 roundings."""
import math

import numpy as np
import pytest
import torch

from tests import expert_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


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


def route(cl, logits, k, **o):
    T = logits.shape[0]
    ids = torch.full((T, k), -7, dtype=torch.int32, device=DEV)
    w = torch.full((T, k), 7.0, device=DEV)
    bias = o.pop("bias", None)
    cl.route_t(logits, ids, w, bias=None if bias is None else bias.to(DEV),
               groups=o.get("groups", 1), top_groups=o.get("top_groups", 1),
               group_top_two=o.get("two", False),
               sigmoid=o.get("sigmoid", False),
               normalize=o.get("normalize", False), scale=o.get("scale", 1.0))
    torch.cuda.synchronize()
    return ids.cpu().long(), w.cpu().double()


def check(cl, logits, k, **o):
    """ids equal, weights within the fp32 roundings of their computation: an
    exponential's argument is off by at most half an ulp of its size (|l -
    top|, or |l|), the exponential by 1 ulp, a sum of n by n half ulps, a
    division by 1.5 ulp and the scale by half: (|x| + 2 + n + 3 + 1) 2^-24,
    twice for numerator and sum."""
    ids, w = route(cl, logits.to(DEV), k, **dict(o))
    ids_r, w_r = ref.route(logits, k, **dict(o))
    assert torch.equal(ids, ids_r)
    l = logits.double()
    live = torch.isfinite(l)
    x = torch.where(live, l, torch.zeros_like(l))
    size = x.abs().amax() * 2 if live.any() else torch.tensor(0.0).double()
    size = min(float(size), 110.0)  # beyond, the exponential is 0
    bound = 2 * (size + 6 + logits.shape[1]) * 2.0 ** -24
    nan = torch.isnan(w_r)
    assert torch.equal(torch.isnan(w), nan)
    err = (w - w_r).abs()[~nan]
    # below 2^-126 fp32 may hold 0
    assert (err <= bound * w_r.abs()[~nan] + 2.0 ** -125).all(), err.max()


OPTIONS = [
    dict(),
    dict(normalize=True, scale=2.5),
    dict(sigmoid=True),
    dict(sigmoid=True, normalize=True),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (3, 5, 5),
                                   (130, 60, 6), (65, 64, 64), (66, 65, 3),
                                   (33, 128, 8), (40, 256, 8), (9, 257, 16),
                                   (5, 1024, 64)])
@pytest.mark.parametrize("o", OPTIONS)
def test_no_bias(cl, dtype, T, E, k, o):
    check(cl, randn(T, E, seed=E, std=2.0).to(dtype), k, **o)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,k,G,t,two", [
    (256, 8, 8, 4, True), (256, 8, 8, 4, False), (64, 6, 4, 2, True),
    (60, 4, 4, 3, True), (64, 8, 64, 8, True), (64, 8, 64, 9, False),
    (1024, 16, 8, 2, True), (1020, 5, 60, 7, True), (6, 3, 2, 1, False),
    (12, 2, 4, 4, True)])
@pytest.mark.parametrize("o", OPTIONS)
def test_bias_and_groups(cl, dtype, E, k, G, t, two, o):
    logits = randn(77, E, seed=E + k).to(dtype)
    bias = randn(E, seed=5, std=0.05)
    check(cl, logits, k, bias=bias, groups=G, top_groups=t, two=two, **o)
    check(cl, logits, k, groups=G, top_groups=t, two=two, **o)


@pytest.mark.parametrize("o", OPTIONS)
@pytest.mark.parametrize("E,G,t", [(64, 1, 1), (256, 8, 4), (60, 4, 2)])
def test_ties_go_to_the_lowest_index(cl, o, E, G, t):
    g = torch.Generator().manual_seed(3)
    logits = torch.randint(-2, 3, (60, E), generator=g).to(torch.bfloat16)
    logits[0] = 0.5
    check(cl, logits, 8, groups=G, top_groups=t, **o)
    check(cl, logits, 8, groups=G, top_groups=t, two=True,
          bias=torch.zeros(E), **o)
    check(cl, logits, 8, groups=G, top_groups=t, two=True,
          bias=torch.randint(0, 2, (E,), generator=g).float(), **o)


def test_values_closer_than_fp32_tells_apart(cl):
    """Sigmoids that differ by some 2^-30 and biases that cancel them."""
    T, E = 64, 64
    l = torch.zeros(T, E)
    l += randn(T, E, seed=9) * 2.0 ** -20
    check(cl, l, 8, bias=torch.zeros(E), sigmoid=True, normalize=True)
    s = torch.sigmoid(randn(E, seed=4).double())
    bias = (1 - s).float()
    l = randn(E, seed=4).repeat(T, 1)
    check(cl, l, 8, bias=bias, sigmoid=True)
    check(cl, l, 8, bias=bias, sigmoid=True, groups=8, top_groups=3, two=True)


@pytest.mark.parametrize("o", OPTIONS)
@pytest.mark.parametrize("E", [60, 256])
@pytest.mark.parametrize("bias", [False, True])
def test_masked_logits(cl, o, E, bias):
    """-inf (some, all but two, all of a row), the lowest finite value, NaN
    and +inf, and biases that are not finite."""
    l = randn(9, E, seed=1)
    l[0, ::2] = -math.inf
    l[1] = -math.inf
    l[1, 7] = 0.5
    l[1, 33] = -4.0
    l[2] = -math.inf
    l[3] = torch.finfo(torch.float32).min
    l[4, 5:] = torch.finfo(torch.float32).min
    l[5, 11] = math.nan
    l[6, 12] = math.inf
    l[7] = -200.0 + randn(E, seed=2)
    o = dict(o)
    if bias:
        b = randn(E, seed=8, std=0.02)
        b[3], b[4], b[5] = -math.inf, math.nan, math.inf
        o["bias"] = b
    check(cl, l, 6, **o)
    check(cl, l, 6, groups=4, top_groups=2, two=True, **o)


def check_many(cl, rows, k, **o):
    """As check(), with the rows again and again until there are so many tokens
    that several share a wave, and every copy the same."""
    R = rows.shape[0]
    n = -(-4200 // R)
    check(cl, rows, k, **o)
    many = rows.repeat(n, 1)[:n * R - 3]
    ids, w = route(cl, many.to(DEV), k, **dict(o))
    ids_r, w_r = ref.route(rows, k, **dict(o))
    assert torch.equal(ids, ids_r.repeat(n, 1)[:n * R - 3])
    w_r = w_r.repeat(n, 1)[:n * R - 3]
    assert torch.equal(torch.isnan(w), torch.isnan(w_r))
    fine = ~torch.isnan(w_r)
    # the bound of check(), with arguments of at most 110
    bound = 2 * (116 + rows.shape[1]) * 2.0 ** -24
    err = (w - w_r).abs()[fine]
    assert (err <= bound * w_r.abs()[fine] + 2.0 ** -125).all()
    first = torch.nan_to_num(w[:R])
    for i in range(1, n - 1):  # a copy's bits do not depend on its place
        assert torch.equal(torch.nan_to_num(w[i * R:(i + 1) * R]), first)


@pytest.mark.parametrize("o", OPTIONS)
@pytest.mark.parametrize("dtype,E,k,G,t,two", [
    (torch.bfloat16, 8, 2, 1, 1, False), (torch.float32, 1, 1, 1, 1, False),
    (torch.float16, 61, 6, 1, 1, False), (torch.bfloat16, 64, 16, 4, 3, True),
    (torch.float32, 64, 8, 16, 5, True), (torch.bfloat16, 100, 17, 1, 1, False),
    (torch.float32, 128, 16, 2, 1, True), (torch.float16, 130, 3, 1, 1, True),
    (torch.float32, 256, 8, 8, 4, True), (torch.float32, 256, 16, 16, 9, False),
    (torch.bfloat16, 252, 4, 12, 5, True), (torch.bfloat16, 257, 8, 1, 1, False),
    (torch.float32, 160, 4, 2, 1, True), (torch.bfloat16, 192, 7, 4, 2, False),
    (torch.float16, 24, 3, 2, 1, True), (torch.float32, 240, 16, 3, 2, True)])
def test_many_tokens(cl, o, dtype, E, k, G, t, two):
    rows = randn(29, E, seed=E + k, std=2.0)
    if E > 8:
        rows[2, ::3] = -math.inf
        rows[3] = -math.inf
        rows[4, E - 2] = math.nan
        rows[5, 1] = math.inf
        rows[6:9] = rows[6:9].round()  # equals
        rows[9] = 0.25
        rows[10] = randn(E, seed=3) * 2.0 ** -20
        rows[11] = -torch.finfo(dtype).max
        rows[12, 2:] = -math.inf
    rows = rows.to(dtype)
    bias = randn(E, seed=5, std=0.05)
    if E > 8:
        bias[7] = math.nan
    check_many(cl, rows, k, groups=G, top_groups=t, two=two, **o)
    check_many(cl, rows, k, bias=bias, groups=G, top_groups=t, two=two, **o)
    check_many(cl, rows, k, bias=torch.zeros(E), groups=G, top_groups=t,
               two=two, **o)


def test_strided_logits_and_a_side_stream(cl):
    wide = randn(50, 100, seed=1).to(torch.bfloat16).to(DEV)
    l = wide[:, 3:67]
    ids = torch.empty(50, 8, dtype=torch.int32, device=DEV)
    w = torch.empty(50, 8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cl.route_t(l, ids, w)
    side.synchronize()
    r, _ = ref.route(l.cpu(), 8)
    assert torch.equal(ids.cpu().long(), r)


def test_no_tokens(cl):
    e = torch.empty(0, 64, device=DEV)
    ids = torch.empty(0, 8, dtype=torch.int32, device=DEV)
    cl.route_t(e, ids, torch.empty(0, 8, device=DEV))
    off = torch.full((5,), 9, dtype=torch.int32, device=DEV)
    cl.route_plan_t(ids, 4, off, torch.empty(0, dtype=torch.int32, device=DEV),
                    ids, cl.PlanWorkspace(1, 8, 4))
    assert off.tolist() == [0] * 5


# ------------------------------------------------------------- gradient ----

def backward(cl, logits, ids, dw, **o):
    d = torch.full_like(logits, 3.0, device=DEV)
    cl.route_backward_t(logits.to(DEV), ids.int().to(DEV), dw.to(DEV), d, **o)
    torch.cuda.synchronize()
    return d.cpu().double()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (67, 60, 6),
                                   (20, 128, 8), (15, 256, 64), (6, 1024, 9)])
@pytest.mark.parametrize("o", OPTIONS)
def test_gradient_of_the_formula_and_of_differences(cl, dtype, T, E, k, o):
    """Against the derivative in 64 bits: a weight's own error is (|x| + E + 9)
    2^-24 relative (see check), it meets gradients of size max |dw|, and the
    result is rounded once. Against central differences with h = 2^-12: their
    own error is h^2 / 6 of a third derivative that is at most 6 max |dw| k."""
    logits = randn(T, E, seed=T + E, std=1.5).to(dtype)
    dw = randn(T, k, seed=2)
    ids = torch.stack([torch.randperm(E, generator=torch.Generator(
    ).manual_seed(t))[:k] for t in range(T)])
    o = dict(dict(sigmoid=False, normalize=False, scale=1.0), **o)
    got = backward(cl, logits, ids, dw, **o)
    l = logits.double().requires_grad_()
    f = (ref.weights_of(l, ids, o["sigmoid"], o["normalize"], o["scale"]) *
         dw.double()).sum()
    f.backward()
    eps = torch.finfo(dtype).eps / 2
    size = float(dw.abs().max()) * o["scale"]
    atol = 4 * size * (12 + E + 9) * 2.0 ** -24
    bound = atol + eps * l.grad.abs()
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25  # fp16's subnormal half step
    assert ((got - l.grad).abs() <= bound).all()
    h, at = 2.0 ** -12, [0, E // 2, E - 1]
    for e in at:
        for sign in (1,):
            p, m = l.detach().clone(), l.detach().clone()
            p[:, e] += h
            m[:, e] -= h
            fp = (ref.weights_of(p, ids, o["sigmoid"], o["normalize"],
                                 o["scale"]) * dw.double()).sum(1)
            fm = (ref.weights_of(m, ids, o["sigmoid"], o["normalize"],
                                 o["scale"]) * dw.double()).sum(1)
            diff = (fp - fm) / (2 * h)
            assert ((got[:, e] - diff).abs() <=
                    bound[:, e] + h * h * size * k).all()


@pytest.mark.parametrize("o", OPTIONS)
def test_gradient_of_odd_rows(cl, o):
    """Masked logits get 0; a row that is masked whole gets zeros; ids out of
    range add nothing; an id named twice counts twice."""
    E, k = 60, 4
    l = randn(6, E, seed=6)
    l[0, 10:40] = -math.inf
    l[1] = -math.inf
    ids = torch.tensor([[1, 2, 45, 50], [-1, -1, -1, -1], [3, 60, -5, 7],
                        [8, 8, 8, 9], [0, 1, 2, 3], [59, 58, 57, 56]])
    dw = randn(6, k, seed=3)
    got = backward(cl, l, ids, dw, **o)
    assert torch.isfinite(got).all()
    assert (got[0, 10:40] == 0).all() and (got[1] == 0).all()
    for t in (0, 2, 3, 4, 5):
        ok = (ids[t] >= 0) & (ids[t] < E)
        x = l[t:t + 1].double().requires_grad_()
        w = ref.weights_of(x, ids[t:t + 1, ok], o.get("sigmoid", False),
                           o.get("normalize", False), o.get("scale", 1.0))
        (w * dw[t:t + 1, ok].double()).sum().backward()
        bound = 4 * float(dw.abs().max()) * 2.5 * (12 + E + 9) * 2.0 ** -24
        assert ((got[t] - x.grad[0]).abs() <= bound).all(), t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,k,pad", [(8, 2, 0), (61, 16, 0), (64, 8, 0),
                                     (64, 8, 3), (128, 17, 0), (100, 5, 4),
                                     (256, 8, 0), (250, 12, 1)])
@pytest.mark.parametrize("o", OPTIONS)
def test_gradient_of_many_tokens(cl, dtype, E, k, pad, o):
    """Enough tokens that several share a wave, rows `pad` values apart:
    against the formula, with the bound of the few."""
    R, T = 23, 4201
    l = randn(R, E, seed=E, std=1.5).to(dtype)
    l[1, E // 2:] = -math.inf
    dw = randn(R, k, seed=2)
    ids = torch.stack([torch.randperm(E, generator=torch.Generator(
    ).manual_seed(t))[:k] for t in range(R)])
    ids[1] = torch.arange(k) % (E // 2)  # of those not masked, some twice
    at = torch.arange(T) % R
    wide = torch.zeros(T, E + pad, dtype=dtype, device=DEV)
    out = torch.full((T, E + pad), 3.0, dtype=dtype, device=DEV)
    wide[:, :E] = l[at].to(DEV)
    cl.route_backward_t(wide[:, :E], ids[at].int().to(DEV), dw[at].to(DEV),
                        out[:, :E], **o)
    got = out[:, :E].cpu().double()
    assert (out[:, E:] == 3).all()
    x = l.double().requires_grad_()
    (ref.weights_of(x, ids, o.get("sigmoid", False), o.get("normalize", False),
                    o.get("scale", 1.0)) * dw.double()).sum().backward()
    exact = torch.nan_to_num(x.grad)
    size = float(dw.abs().max()) * o.get("scale", 1.0)
    bound = 4 * size * (12 + E + 9) * 2.0 ** -24 + \
        torch.finfo(dtype).eps / 2 * exact.abs()
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25
    assert ((got - exact[at]).abs() <= bound[at]).all()


# ----------------------------------------------------------------- plan ----

@pytest.mark.parametrize("T,k,E,first", [
    (1, 8, 64, 0), (1, 1, 1, 0), (7, 3, 5, 0), (64, 8, 16, 24), (256, 8, 64, 0),
    (257, 8, 64, 0), (1000, 2, 1000, 0), (5000, 6, 1024, 100),
    (20001, 8, 32, 64), (70000, 1, 3, 1)])
def test_plan(cl, T, k, E, first):
    g = torch.Generator().manual_seed(T)
    ids = torch.randint(-1, first + E + 3, (T, k), generator=g,
                        dtype=torch.int32)
    ids[T // 2:] = ids[T // 2:].clamp(max=first)  # many of one expert
    ids[0, 0] = 2 ** 31 - 1
    ids[-1, -1] = -2 ** 31
    off = torch.full((E + 1,), -9, dtype=torch.int32, device=DEV)
    src = torch.full((T * k,), -9, dtype=torch.int32, device=DEV)
    pos = torch.full((T, k), -9, dtype=torch.int32, device=DEV)
    ws = cl.PlanWorkspace(T, k, E)
    ws.buf.fill_(0xA5)
    for _ in range(2):
        cl.route_plan_t(ids.to(DEV), E, off, src, pos, ws, first_expert=first)
        o, s, p = ref.plan(ids, E, first)
        assert torch.equal(off.cpu().long(), o)
        assert torch.equal(src.cpu().long(), s)
        assert torch.equal(pos.cpu().long(), p)


@pytest.mark.parametrize("T,k,E", [(129, 2, 3), (1023, 2, 64), (1025, 2, 64),
                                   (40_000, 3, 256), (70_001, 8, 65)])
def test_plan_of_every_tile(cl, T, k, E):
    """Few pairs shared by all waves, and both sizes of tiles."""
    g = torch.Generator().manual_seed(T)
    ids = torch.randint(-1, E + 1, (T, k), generator=g, dtype=torch.int32)
    off = torch.full((E + 1,), -9, dtype=torch.int32, device=DEV)
    src = torch.full((T * k,), -9, dtype=torch.int32, device=DEV)
    pos = torch.full((T, k), -9, dtype=torch.int32, device=DEV)
    cl.route_plan_t(ids.to(DEV), E, off, src, pos, cl.PlanWorkspace(T, k, E))
    o, s, p = ref.plan(ids, E)
    assert torch.equal(off.cpu().long(), o)
    assert torch.equal(src.cpu().long(), s)
    assert torch.equal(pos.cpu().long(), p)


def test_route_and_plan_in_a_graph(cl):
    T, E, k = 300, 64, 8
    l = randn(T, E, seed=1).to(DEV)
    ids = torch.zeros(T, k, dtype=torch.int32, device=DEV)
    w = torch.zeros(T, k, device=DEV)
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    src = torch.zeros(T * k, dtype=torch.int32, device=DEV)
    pos = torch.zeros(T, k, dtype=torch.int32, device=DEV)
    ws = cl.PlanWorkspace(T, k, E)

    def step():
        cl.route_t(l, ids, w, sigmoid=True, normalize=True)
        cl.route_plan_t(ids, E, off, src, pos, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        new = randn(T, E, seed=10 + seed)
        l.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        r, _ = ref.route(new, k, sigmoid=True)
        assert torch.equal(ids.cpu().long(), r)
        o, s, p = ref.plan(r, E)
        assert torch.equal(off.cpu().long(), o)
        assert torch.equal(src.cpu().long(), s)
        assert torch.equal(pos.cpu().long(), p)


def test_same_bits_twice(cl):
    l = randn(500, 256, seed=3).to(DEV)
    a = route(cl, l, 8, sigmoid=True, normalize=True, bias=randn(256, seed=1))
    b = route(cl, l, 8, sigmoid=True, normalize=True, bias=randn(256, seed=1))
    assert np.array_equal(a[1].numpy().view(np.int64),
                          b[1].numpy().view(np.int64))
    assert torch.equal(a[0], b[0])
