"""Refusals of the experts' operators, and their sizes, without a GPU: every
call below fails its checks before anything is enqueued (the pointers are never
followed), or has nothing to do."""
import pytest
import torch

from tests import expert_ref as ref

P = 0x10000  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def cl():
    import os

    from paper_2609_04609_amd import build, ciera
    if not os.path.exists(ciera.LIB_PATH):
        build.build()
    ciera.lib()
    return ciera


def refused(cl, fn, good, changes, code=None):
    """`good` arguments with one change each are refused."""
    for change in changes:
        args = dict(good, **change)
        rc = getattr(cl, fn)(*args.values())
        assert rc == (cl.EINVAL if code is None else code), (fn, change, rc)


def test_route(cl):
    good = dict(logits=P, dtype=0, T=4, E=64, stride=64, bias=P, groups=8,
                top_groups=4, k=8, flags=7, scale=1.0, ids=P, w=P, stream=0)
    refused(cl, "ciera_route", good, [
        dict(logits=0), dict(logits=P + 1), dict(dtype=3), dict(E=0),
        dict(E=1025), dict(stride=63), dict(bias=P + 2), dict(groups=0),
        dict(groups=7), dict(groups=128, E=128), dict(top_groups=0),
        dict(top_groups=9), dict(k=0), dict(k=33), dict(k=65), dict(flags=8),
        dict(ids=0), dict(w=0), dict(ids=P + 2), dict(T=1 << 28),
        dict(T=1 << 31), dict(T=(1 << 61) + 1)])
    assert cl.ciera_route(*dict(good, T=0, logits=0, ids=0, w=0).values()) == 0


def test_route_backward(cl):
    good = dict(logits=P, dtype=2, T=4, E=64, stride=64, k=8, flags=3,
                scale=1.0, ids=P, dw=P, d=P, ds=64, stream=0)
    refused(cl, "ciera_route_backward", good, [
        dict(logits=0), dict(logits=P + 2), dict(dtype=3), dict(E=0),
        dict(E=1025), dict(stride=1), dict(ds=63), dict(k=0), dict(k=65),
        dict(flags=4), dict(ids=0), dict(dw=0), dict(d=0), dict(d=P + 2),
        dict(T=1 << 28)])
    assert cl.ciera_route_backward(*dict(good, T=0).values()) == 0


def test_plan(cl):
    assert cl.ciera_plan_workspace_bytes(10, 8, 0) == 0
    assert cl.ciera_plan_workspace_bytes(10, 8, 1025) == 0
    assert cl.ciera_plan_workspace_bytes(10, 0, 4) == 0
    assert cl.ciera_plan_workspace_bytes(1 << 28, 8, 4) == 0
    assert cl.ciera_plan_workspace_bytes((1 << 61) + 1, 8, 4) == 0
    need = cl.ciera_plan_workspace_bytes(5000, 8, 64)
    assert need >= 4 * (5000 * 8 // 2048 * 64 + 1)
    good = dict(ids=P, T=5000, k=8, first=0, E=64, off=P, src=P, pos=P, ws=P,
                n=need, stream=0)
    refused(cl, "ciera_route_plan", good, [
        dict(ids=0), dict(k=0), dict(k=65), dict(E=0), dict(E=1025),
        dict(off=0), dict(src=0), dict(pos=0), dict(ws=0), dict(off=P + 1),
        dict(first=1 << 31)])
    refused(cl, "ciera_route_plan", good, [dict(n=need - 1)], cl.ENOSPC)
    with pytest.raises(cl.CieraError):
        cl.PlanWorkspace(10, 8, 2000, device="cpu")


def test_quantize(cl):
    good = dict(x=P, dtype=0, R=5, C=300, stride=300, pos=P, k=2, Q=10, q=P,
                qs=384, s=P, ss=4, stream=0)
    refused(cl, "ciera_quantize_rows", good, [
        dict(x=0), dict(x=P + 1), dict(dtype=3), dict(stride=299),
        dict(pos=P + 1), dict(k=0), dict(k=65), dict(q=0), dict(q=P + 8),
        dict(qs=300), dict(qs=392), dict(s=0), dict(s=P + 1), dict(ss=3),
        dict(ss=5), dict(pos=0), dict(pos=0, k=1, Q=4), dict(R=1 << 31),
        dict(Q=1 << 31), dict(C=1 << 30)])
    for zero in (dict(R=0), dict(C=0), dict(Q=0)):
        assert cl.ciera_quantize_rows(*dict(good, **zero).values()) == 0
    good = dict(w=P, dtype=2, E=2, N=130, C=300, q=P, qs=384, s=P, ss=4, qt=P,
                qts=256, st=P, sts=4, stream=0)
    refused(cl, "ciera_quantize_blocks", good, [
        dict(w=0), dict(w=P + 2), dict(dtype=7), dict(q=0), dict(qs=300),
        dict(s=0), dict(ss=0), dict(qt=0), dict(st=0), dict(qts=128),
        dict(qts=200), dict(sts=1), dict(E=1 << 31), dict(N=1 << 30),
        dict(E=1 << 30, N=1 << 20)])
    for zero in (dict(E=0), dict(N=0), dict(C=0)):
        assert cl.ciera_quantize_blocks(*dict(good, **zero).values()) == 0
    need = cl.ciera_columns_length(1000, 64)
    good = dict(x=P, dtype=0, X=125, R=1000, C=300, stride=300, src=P, k=8,
                off=P, E=64, q=P, L=need, s=P, ss=need // 128 + 3 & ~3,
                stream=0)
    refused(cl, "ciera_quantize_columns", good, [
        dict(x=0), dict(dtype=3), dict(stride=299), dict(src=0), dict(k=0),
        dict(off=0), dict(off=P + 2), dict(E=0), dict(E=1025), dict(q=0),
        dict(q=P + 4), dict(L=need + 64), dict(s=0), dict(ss=4),
        dict(X=1 << 31), dict(R=1 << 31)])
    refused(cl, "ciera_quantize_columns", good, [dict(L=need - 128)],
            cl.ENOSPC)


@pytest.mark.parametrize("counts", [[0], [1], [5, 0, 200], [1] * 9,
                                    [128, 128], [129, 127, 1, 0]])
def test_columns_length_is_enough(cl, counts):
    need = sum(-(-n // 128) * 128 for n in counts)
    L = cl.ciera_columns_length(sum(counts), len(counts))
    assert L >= need and L % 128 == 0
    # and not more than the worst split of as many rows needs
    some = min(len(counts), sum(counts))
    worst = [1] * (some - 1) + [sum(counts) - some + 1] if some else []
    assert L <= 128 * len(worst) + sum(counts)


def test_products(cl):
    good = dict(a=P, as_=256, sa=P, ssa=4, R=10, b=P, bs=256, sb=P, ssb=4, E=2,
                N=100, D=256, off=P, out=P, dtype=0, os=100, stream=0)
    refused(cl, "ciera_expert_matmul", good, [
        dict(a=0), dict(a=P + 8), dict(as_=255), dict(as_=264), dict(sa=0),
        dict(sa=P + 2), dict(ssa=1), dict(b=0), dict(bs=128), dict(sb=0),
        dict(ssb=6), dict(E=0), dict(E=1025), dict(D=0), dict(D=200),
        dict(D=1 << 24), dict(off=0), dict(off=P + 1), dict(out=0),
        dict(out=P + 1), dict(dtype=3), dict(os=99), dict(R=1 << 31),
        dict(N=1 << 30), dict(R=1 << 30, N=1 << 20)])
    for zero in (dict(R=0), dict(N=0)):
        assert cl.ciera_expert_matmul(*dict(good, **zero).values()) == 0
    good = dict(dy=P, sdy=P, ssdy=4, x=P, sx=P, ssx=4, L=512, E=2, N=10, C=20,
                off=P, dw=P, dtype=2, stream=0)
    refused(cl, "ciera_expert_weight_grad", good, [
        dict(dy=0), dict(sdy=0), dict(ssdy=0), dict(x=P + 4), dict(sx=P + 1),
        dict(ssx=7), dict(L=500), dict(L=1 << 31), dict(E=0), dict(E=1025),
        dict(off=0), dict(dw=0), dict(dw=P + 2), dict(dtype=3),
        dict(N=1 << 30), dict(N=1 << 29, C=1 << 29)])
    for zero in (dict(N=0), dict(C=0)):
        assert cl.ciera_expert_weight_grad(*dict(good, **zero).values()) == 0


def test_combine(cl):
    good = dict(rows=P, dtype=0, R=10, C=100, stride=100, w=P, pos=P, T=5, k=2,
                out=P, os=100, stream=0)
    refused(cl, "ciera_combine", good, [
        dict(rows=0), dict(rows=P + 1), dict(dtype=3), dict(stride=99),
        dict(w=P + 1), dict(pos=0), dict(k=0), dict(k=65), dict(out=0),
        dict(os=99), dict(R=1 << 31), dict(T=1 << 31), dict(C=1 << 30)])
    for zero in (dict(T=0), dict(C=0)):
        assert cl.ciera_combine(*dict(good, **zero).values()) == 0
    good = dict(g=P, gs=100, rows=P, dtype=0, R=10, C=100, stride=100, w=P,
                pos=P, T=5, k=2, d=P, ds=100, dw=P, stream=0)
    refused(cl, "ciera_combine_backward", good, [
        dict(g=0), dict(gs=99), dict(rows=0), dict(dtype=3), dict(stride=99),
        dict(w=0), dict(pos=0), dict(k=0), dict(k=65), dict(d=0), dict(ds=99),
        dict(dw=0), dict(d=P + 1), dict(T=1 << 30)])
    assert cl.ciera_combine_backward(*dict(good, T=0).values()) == 0


def test_tensors_are_checked(cl):
    """A tensor that is not on the current device is refused by name."""
    x = torch.zeros(4, 8)
    i = torch.zeros(4, 2, dtype=torch.int32)
    w = torch.zeros(4, 2)
    with pytest.raises(ValueError, match="logits is on cpu"):
        cl.route_t(x, i, w)
    with pytest.raises(ValueError, match="rows is on cpu"):
        cl.combine_t(x, i, x)
    with pytest.raises(ValueError, match="logits has 1 dimensions"):
        cl.route_t(x[0], i, w)


def test_the_reference_itself():
    """tests/expert_ref.py against what torch and hand arithmetic say."""
    bits = torch.arange(256).to(torch.uint8)
    v = bits.view(torch.float8_e4m3fn).double()
    v = v[torch.isfinite(v)]
    assert torch.equal(ref.e4m3_round(v), v)  # its own values stay
    assert ref.e4m3_round(torch.tensor([17.0, 19.0, -17.5], dtype=torch.float64)
                          ).tolist() == [16.0, 20.0, -18.0]
    top = torch.tensor([0.0, 448.0, 448.1, 1.0, 3.5, 3.6, 2.0 ** -140]).double()
    # 1 <= 448 * 2^-8 = 1.75 and 3.5 = 448 * 2^-7
    assert ref.exponent_of(top).tolist() == [0, 0, 1, -8, -7, -6, -127]
    ids, w = ref.route(torch.tensor([[1.0, 3.0, 3.0, 0.0]]), 2, normalize=True)
    assert ids.tolist() == [[1, 2]] and w.tolist() == [[0.5, 0.5]]
    o, s, p = ref.plan(torch.tensor([[1, 0], [5, 1]]), 2)
    assert o.tolist() == [0, 1, 3] and s.tolist() == [1, 0, 3, -1]
    assert p.tolist() == [[1, 0], [-1, 2]]


def test_plan_workspace_grows(cl):
    """A workspace for some tokens is enough for fewer."""
    for k, E in ((1, 3), (8, 64)):
        last = 0
        for n in sorted({0, 1, 100, 255, 256, 257, 2047, 2048, 2049, 65535,
                         65536, 65537, 70000, 131072, 131073, 524287, 524288,
                         524289, 600000, 1048576, 1048577, 1 << 24}):
            need = cl.ciera_plan_workspace_bytes(n, k, E)
            assert need >= last, (k, n)
            last = need


def test_launches_past_32_bits_of_threads(cl):
    """Sizes that a device's memory could hold but one launch could not cover."""
    big = 1 << 26
    assert cl.ciera_route(P, 0, big, 1, 1, 0, 1, 1, 1, 0, 1.0, P, P,
                          0) == cl.EINVAL
    assert cl.ciera_route_backward(P, 0, big, 1, 1, 1, 0, 1.0, P, P, P, 1,
                                   0) == cl.EINVAL
    assert cl.ciera_quantize_rows(P, 0, big, 128, 128, 0, 1, big, P, 128, P, 4,
                                  0) == cl.EINVAL
    assert cl.ciera_quantize_blocks(P, 0, 1 << 24, 1, 128, P, 128, P, 4, 0, 0,
                                    0, 0, 0) == cl.EINVAL
    assert cl.ciera_combine(P, 0, 1, 8, 8, P, P, big, 1, P, 8, 0) == cl.EINVAL
    assert cl.ciera_combine_backward(P, 8, P, 0, 1, 8, 8, P, P, big // 8, 8, P,
                                     8, P, 0) == cl.EINVAL
