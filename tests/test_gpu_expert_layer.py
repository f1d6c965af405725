"""The experts' operators run together, as a layer uses them: forward and
backward against 64 bits, against differences, captured into graphs, and behind the
codec's decode in both schedules of the pipeline."""
import math

import pytest
import torch

from tests import expert_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def cl():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04609_amd import ciera
    ciera.lib()
    return ciera


def layer(*args, **o):
    from paper_2609_04609_amd.experts import ExpertLayer
    return ExpertLayer(*args, **o)


def randn(*shape, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * std


def whole(*shape, seed, most=4):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).float()


def pairs_of_experts(T, E, seed):
    """[T, 2] different experts a token, and logits for which softmax gives
    each of them half."""
    g = torch.Generator().manual_seed(seed)
    e = torch.stack([torch.randperm(E, generator=g)[:2].sort().values
                     for _ in range(T)])
    return e, torch.full((T, E), -30.0).scatter(1, e, 30.0)


@pytest.mark.parametrize("T,E,N,C", [(1, 2, 1, 1), (5, 9, 130, 200),
                                     (150, 6, 160, 72), (700, 3, 264, 520)])
def test_whole_numbers_are_exact(cl, T, E, N, C):
    """Inputs that e4m3 holds and weights of a half: every product and sum is a
    multiple of a half below 2^24, so the layer has one right answer, and being
    linear in x and in W, its gradients are its differences."""
    e, logits = pairs_of_experts(T, E, 1)
    x, w = whole(T, C, seed=2), whole(E, N, C, seed=3)
    d_out = 2 * whole(T, N, seed=4)
    m = layer(T, 2, E, N, C, dtype=torch.float32, normalize=True)
    on = [t.to(DEV) for t in (x, w, d_out, logits)]

    def out(x, w, logits=logits):
        m.load(w.to(DEV))
        return m.forward(x.to(DEV), logits.to(DEV)).double().cpu()

    y = out(x, w)
    assert torch.equal(m.ids.cpu().long(), e)
    assert (m.weights == 0.5).all()
    W, X, G = w.double(), x.double(), d_out.double()
    rows = torch.matmul(W[e].reshape(T * 2, N, C),
                        X.repeat_interleave(2, 0).unsqueeze(2))
    rows = rows.view(T, 2, N)
    assert torch.equal(y, rows.sum(1) / 2)
    d_x, d_w, d_l = (g.double().cpu() for g in
                     m.backward(on[2], on[0], on[3]))
    half = G / 2
    back = torch.matmul(half.view(T, 1, 1, N), W[e]).view(T, 2, C)
    assert torch.equal(d_x, back.sum(1))
    expect = torch.zeros(E, N, C, dtype=torch.float64)
    for t in range(T):
        for s in range(2):
            expect[e[t, s]] += half[t].unsqueeze(1) * X[t].unsqueeze(0)
    assert torch.equal(d_w, expect)
    g = (rows * G.unsqueeze(1)).sum(2)
    assert torch.equal(m.d_weights.double().cpu(), g)
    diff = (g[:, 0] - g[:, 1]) / 4  # w (g_s - sum w g)
    expect = torch.zeros(T, E, dtype=torch.float64)
    expect.scatter_(1, e, torch.stack([diff, -diff], 1))
    # a handful of fp32 roundings of the weights and products
    bound = 8 * 2.0 ** -23 * g.abs().sum(1, keepdim=True)
    assert ((d_l - expect).abs() <= bound).all()

    dx, dw = whole(T, C, seed=5), whole(E, N, C, seed=6)
    assert float(((out(x + dx, w) - y) * G).sum()) == float((d_x * dx).sum())
    assert float(((out(x, w + dw) - y) * G).sum()) == float((d_w * dw).sum())
    # the logits' way is curved: sigma(u + h v) of a token's two logits has a
    # third derivative of at most |v|^3 / 8; the outputs are off by 2^-22 of themselves
    h, v = 2.0 ** -6, whole(T, E, seed=7)
    up, down = out(x, w, logits + h * v), out(x, w, logits - h * v)
    slope = float(((up - down) * G).sum()) / (2 * h)
    dv = (v.gather(1, e)[:, 0] - v.gather(1, e)[:, 1]).abs().double()
    bound = (h * h / 6 * dv ** 3 / 8 * (g[:, 0] - g[:, 1]).abs()).sum()
    bound += 2.0 ** -22 / h * (rows.abs().sum(1) * G.abs()).sum()
    bound += 8 * 2.0 ** -23 * (g.abs().sum(1, keepdim=True) * v.abs()).sum()
    assert abs(slope - float((d_l * v).sum())) <= float(bound)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("dtype,o,T,E,k,N,C", [
    (torch.bfloat16, dict(sigmoid=True, normalize=True, scale=2.5, groups=4,
                          top_groups=2, group_top_two=True), 300, 16, 3, 264,
     200),
    (torch.bfloat16, dict(), 1, 5, 5, 96, 640),
    (torch.float16, dict(normalize=True), 77, 40, 2, 130, 72),
])
def test_against_64_bits(cl, dtype, o, T, E, k, N, C):
    """Every step against its definition, from the tensors that the step
    before it left: some tokens have no expert, some experts are masked."""
    m = layer(T, k, E, N, C, dtype=dtype, **o)
    x = randn(T, C, seed=1).to(dtype)
    w = randn(E, N, C, seed=2, std=C ** -0.5).to(dtype)
    logits = randn(T, E, seed=3).to(dtype)
    d_out = randn(T, N, seed=4).to(dtype)
    bias = randn(E, seed=5, std=0.1) if "groups" in o else None
    if T > 10:
        logits[3:5] = -math.inf  # no expert
        logits[:, 1] = -math.inf  # no token
    X, L, G = x.to(DEV), logits.to(DEV), d_out.to(DEV)
    m.load(w.to(DEV))
    y = m.forward(X, L, None if bias is None else bias.to(DEV))
    grads = m.backward(G, X, L)
    torch.cuda.synchronize()
    eps = half_step(dtype)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0

    def near(got, exact, bound):
        got = got.double().cpu()
        assert torch.isfinite(got).all()
        err = (got - exact).abs() - bound - eps * exact.abs() - tiny
        assert (err <= 0).all(), float(err.max())

    r = dict(o)
    r["two"] = r.pop("group_top_two", False)
    ids, wt = ref.route(logits, k, bias=bias, **r)
    assert torch.equal(m.ids.cpu().long(), ids)
    assert ((m.weights.double().cpu() - wt).abs() <= 2.0 ** -17 * wt).all()
    offsets, source, position = ref.plan(ids, E)
    assert torch.equal(m.offsets.cpu().long(), offsets)
    assert torch.equal(m.source.cpu().long(), source)
    assert torch.equal(m.position.cpu().long(), position)
    held = int(offsets[-1])
    token, expert = source[:held] // k, ids.view(-1)[source[:held]]
    wt = m.weights.double().cpu()

    def product(a, b, pick):
        """Rows of a times their experts' b, with the bound of a sum whose
        neighbours, eight at a time, are added with 14 bits."""
        out = torch.empty(held, b.shape[1], dtype=torch.float64)
        size = torch.empty_like(out)
        for e in range(E):
            at = pick == e
            out[at] = a[at] @ b[e].t()
            size[at] = a[at].abs() @ b[e].abs().t()
        return out, size * (2.0 ** -10 + a.shape[1] * 2.0 ** -23)

    def of(q, s):
        return ref.values(q, s, 1, 128)

    qx = of(*ref.quantize(x[token], 1, 128))
    qw = [ref.values(*ref.quantize(w[e], 128, 128), 128, 128)
          for e in range(E)]
    qw = torch.stack(qw)
    near(m.rows[:held], *product(qx, qw, expert))
    rows = m.rows[:held].double().cpu()
    exact = torch.zeros(T, N, dtype=torch.float64)
    size = torch.zeros_like(exact)
    flat = wt.view(-1)[source[:held]].unsqueeze(1)
    exact.index_add_(0, token, flat * rows)
    size.index_add_(0, token, flat * rows.abs())
    near(y, exact, k * 2.0 ** -23 * size)
    assert (y[position.lt(0).all(1).to(DEV)] == 0).all()

    g = d_out.double()[token]
    near(m.d_rows[:held], flat * g, 2.0 ** -23 * (flat * g).abs())
    d_weights = torch.zeros(T * k, dtype=torch.float64)
    d_weights[source[:held]] = (g * rows).sum(1)
    size = torch.zeros_like(d_weights)
    size[source[:held]] = (g * rows).abs().sum(1)
    got = m.d_weights.double().cpu().view(-1)
    assert ((got - d_weights).abs() <= N * 2.0 ** -23 * size).all()
    d_rows = m.d_rows[:held].cpu()
    dy = of(*ref.quantize(d_rows, 1, 128))
    near(m.d_x_rows[:held], *product(dy, qw.transpose(1, 2), expert))
    back = m.d_x_rows[:held].double().cpu()
    exact = torch.zeros(T, C, dtype=torch.float64).index_add_(0, token, back)
    size = torch.zeros_like(exact).index_add_(0, token, back.abs())
    d_x, d_w, d_logits = grads
    near(d_x, exact, k * 2.0 ** -23 * size)
    for e in range(E):
        at = slice(int(offsets[e]), int(offsets[e + 1]))
        if at.start == at.stop:
            assert (d_w[e] == 0).all()
            continue
        q = [ref.values(*ref.quantize(t, 128, 1), 128, 1)
             for t in (d_rows[at], x[token[at]])]
        n = at.stop - at.start
        near(d_w[e], q[0].t() @ q[1],
             (2.0 ** -10 + n * 2.0 ** -23) * (q[0].abs().t() @ q[1].abs()))
    l = torch.where(torch.isfinite(logits), logits, torch.tensor(-60.0,
                    dtype=dtype)).double().requires_grad_()
    own = ref.weights_of(l, ids.clamp(0), o.get("sigmoid", False), False, 1.0)
    if o.get("normalize", False):
        own = own / own.sum(1, keepdim=True)
    own = own * o.get("scale", 1.0)
    gw = m.d_weights.double().cpu() * (ids >= 0)
    (own * gw).sum().backward()
    exact = torch.where(torch.isfinite(logits), l.grad,
                        torch.zeros_like(l.grad))
    # the weights (2^-17) times the gradients, and sums of E terms
    near(d_logits, exact, 2.0 ** -16 * o.get("scale", 1.0) *
         gw.abs().sum(1, keepdim=True).expand(T, E))


def test_captured_layers(cl):
    """Two layers, each captured on a side stream and replayed in turn with new
    inputs; eager work of a third between the replays, which also gives the
    right bits."""
    T, k, E, N, C = 130, 4, 24, 320, 256
    bf16 = torch.bfloat16
    make = [layer(T, k, E, N, C, sigmoid=True, normalize=True)
            for _ in range(3)]
    x, w, l, g = ([torch.empty(s, dtype=bf16, device=DEV) for _ in range(2)]
                  for s in ((T, C), (E, N, C), (T, E), (T, N)))

    def fill(i, seed):
        for j, t in enumerate((x, w, l, g)):
            t[i].copy_(randn(*t[i].shape, seed=100 * seed + 10 * i + j))

    def run(m, i):
        m.load(w[i])
        return (m.forward(x[i], l[i]),) + m.backward(g[i], x[i], l[i])

    graphs, outs = [], []
    for i in range(2):
        fill(i, 0)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            run(make[i], i)
        torch.cuda.current_stream().wait_stream(st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            outs.append(run(make[i], i))
        graphs.append(graph)
    for seed in range(1, 4):
        for i in range(2):
            fill(i, seed)
            for t in outs[i]:
                t.fill_(7)
        for i in range(2):
            graphs[i].replay()
        got = [[t.clone() for t in o] for o in outs]
        for i in range(2):
            expect = run(make[2], i)
            torch.cuda.synchronize()
            for a, b in zip(got[i], expect):
                assert torch.equal(a, b)
            assert float(expect[0].float().abs().sum()) > 0


def test_without_train(cl):
    m = layer(9, 2, 4, 40, 50, train=False)
    x, w = randn(9, 50, seed=1).bfloat16(), randn(4, 40, 50, seed=2).bfloat16()
    l = randn(9, 4, seed=3).bfloat16()
    m.load(w.to(DEV))
    y = m.forward(x.to(DEV), l.to(DEV)).clone()
    both = layer(9, 2, 4, 40, 50)
    both.load(w.to(DEV))
    assert torch.equal(y, both.forward(x.to(DEV), l.to(DEV)))
    with pytest.raises(ValueError, match="backward"):
        m.backward(y, x.to(DEV), l.to(DEV))
    with pytest.raises(ValueError, match="x has shape"):
        both.backward(both.forward(x.to(DEV), l.to(DEV)), x[:, :49].to(DEV),
                      l.to(DEV))


def test_experts_behind_the_decode(cl):
    """The pipeline's layers as layers of experts: both schedules decode the
    same bits as before, and every layer's results are those of its decoded
    weights."""
    import bench
    from paper_2609_04609_amd import synth
    from paper_2609_04609_amd.pipeline import OverlapPipeline
    S = bench.Setup(synth.WORKLOADS["olmoe_expert"], 512,
                    torch.device("cuda:0"))
    with pytest.raises(ValueError, match="not 8 experts of 1000"):
        OverlapPipeline(S, 2, 1e12, tokens=64, experts=(8, 2, 1000))
    P = OverlapPipeline(S, 3, 1e12, tokens=64, experts=(8, 2, 512))
    assert [tuple(y.shape) for y in P.y] == [(64, 512)] * 3
    alone = layer(64, 2, 8, 512, 512, normalize=True)
    seen = []
    for overlapped in (False, True, True, True):
        P.step(overlapped)
        assert P.check(), f"overlapped={overlapped}"
        for i in range(3):
            alone.load(P.outs[i].view(torch.bfloat16).view(8, 512, 512))
            y = alone.forward(P.act, P.logits)
            expect = (y,) + alone.backward(P.d_y, P.act, P.logits)
            m = P.experts[i]
            for a, b in zip((P.y[i], m.d_x, m.d_w, m.d_logits), expect):
                assert torch.equal(a, b)
                assert torch.isfinite(a).all()
        seen.append(P.y[0].clone())
    assert not torch.equal(seen[0], seen[1])  # the weights moved
    assert torch.equal(seen[1], seen[3])  # and came back
    assert set(P.component_us(reps=2)) == {"encode", "link", "decode",
                                           "compute"}
