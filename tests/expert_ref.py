"""The experts' operators in 64 bits, from their definitions: plain torch on
the CPU, sharing no code with the library."""
import math

import torch

INF = math.inf


def top_of(values, n):
    """Indices of the n largest of a 1-D double tensor, lowest first among
    equals; entries of -inf are not taken."""
    order = sorted(range(values.numel()),
                   key=lambda i: (-values[i].item(), i))
    return [i for i in order if values[i].item() > -INF][:n]


def scores(l, sigmoid):
    """Softmax (of a row whose -inf entries are masked) or sigmoid of a row, value
    by value: torch's own may give equal logits scores that differ in the last
    bit, by their place in the row."""
    x = l.tolist()
    top = max(x)
    if sigmoid:
        s = [1 / (1 + math.exp(-v)) if v > 0 else
             math.exp(v) / (1 + math.exp(v)) for v in x]
    elif top == -INF:
        s = [0.0] * len(x)
    else:
        e = [math.exp(v - top) for v in x]
        total = math.fsum(e)
        s = [v / total for v in e]
    return torch.tensor(s, dtype=torch.float64)


def route(logits, k, bias=None, groups=1, top_groups=1, two=False,
          sigmoid=False, normalize=False, scale=1.0):
    """ids (int64) and weights (double), row by row."""
    T, E = logits.shape
    ids = torch.full((T, k), -1)
    w = torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        l = logits[t].double().cpu()
        if torch.isnan(l).any() or (l == INF).any():
            w[t] = math.nan
            continue
        s = scores(l, sigmoid)
        v = s.clone()
        if bias is not None:
            b = bias.double().cpu()
            v = torch.where(torch.isfinite(b), v + b, torch.tensor(-INF).double())
        elif top_groups == groups or not two:
            v = l.clone()  # the scores' own order
        v[l == -INF] = -INF
        if top_groups < groups:
            S = E // groups
            rank = torch.full((groups,), -INF, dtype=torch.float64)
            for g in range(groups):
                live = sorted((x for x in v[g * S:(g + 1) * S].tolist()
                               if x > -INF), reverse=True)
                if live:
                    rank[g] = sum(live[:2]) if two else live[0]
            kept = top_of(rank, top_groups)
            for g in range(groups):
                if g not in kept:
                    v[g * S:(g + 1) * S] = -INF
        chosen = top_of(v, k)
        n = len(chosen)
        ids[t, :n] = torch.tensor(chosen, dtype=torch.int64)
        if n == 0:
            continue
        c = torch.tensor(chosen)
        if normalize and sigmoid:
            x = torch.softmax(torch.nn.functional.logsigmoid(l[c]), 0)
        elif normalize:
            x = torch.softmax(l[c], 0)
        else:
            x = s[c]
        w[t, :n] = x * scale
    return ids, w


def weights_of(l, ids, sigmoid, normalize, scale):
    """The weights as a function of double logits, for fixed ids (>= 0)."""
    s = torch.sigmoid(l) if sigmoid else torch.softmax(l, 1)
    w = s.gather(1, ids)
    if normalize:
        w = w / w.sum(1, keepdim=True)
    return w * scale


def plan(ids, n_experts, first=0):
    """(offsets, source, position) by a Python sort."""
    T, k = ids.shape
    flat = [e - first for e in ids.reshape(-1).tolist()]
    held = [i for i, e in enumerate(flat) if 0 <= e < n_experts]
    held.sort(key=lambda i: flat[i])  # stable
    source = held + [-1] * (T * k - len(held))
    position = [-1] * (T * k)
    for p, i in enumerate(held):
        position[i] = p
    offsets = [0] * (n_experts + 1)
    for i in held:
        offsets[flat[i] + 1] += 1
    for e in range(n_experts):
        offsets[e + 1] += offsets[e]
    return (torch.tensor(offsets), torch.tensor(source, dtype=torch.int64),
            torch.tensor(position, dtype=torch.int64).view(T, k))


def exponent_of(top):
    """Smallest integer e >= -127 with top <= 448 * 2^e (0 for no value), of a
    double tensor of maxima that 32-bit floats hold."""
    e = torch.full(top.shape, -127.0, dtype=torch.float64)
    for c in range(-126, 122):
        e = torch.where(top > 448 * 2.0 ** (c - 1),
                        torch.full_like(e, float(c)), e)
    return torch.where(top == 0, torch.zeros_like(e), e)


def e4m3_round(y):
    """Nearest e4m3 value, ties to even, of doubles within +-448."""
    a = y.abs()
    step = torch.full_like(a, 2.0 ** -9)
    for p in range(-5, 9):  # a >= 2^p: steps of 2^(p - 3)
        step = torch.where(a >= 2.0 ** p, torch.full_like(a, 2.0 ** (p - 3)),
                           step)
    return torch.round(y / step) * step


def quantize(x, rows, cols):
    """Blocks of rows x cols of a 2-D tensor -> (held values as doubles, NaN
    where not finite, scale bytes as int64 [row blocks, col blocks])."""
    x = x.double().cpu()
    R, C = x.shape
    q = torch.empty_like(x)
    s = torch.empty(-(-R // rows), -(-C // cols), dtype=torch.int64)
    fine = torch.isfinite(x)
    top = torch.where(fine, x.abs(), torch.zeros_like(x))
    pad = torch.nn.functional.pad(top, (0, -C % cols, 0, -R % rows))
    m = pad.view(s.shape[0], rows, s.shape[1], cols).amax((1, 3))
    e = exponent_of(m)
    s = (e + 127).long()
    full = e.repeat_interleave(rows, 0)[:R].repeat_interleave(cols, 1)[:, :C]
    q = e4m3_round(torch.where(fine, x, torch.zeros_like(x)) * 2.0 ** -full)
    return torch.where(fine, q, torch.full_like(q, math.nan)), s


def values(q, s, rows, cols):
    """Doubles that 8-bit values (any float type) and scale bytes stand for."""
    q = q.double().cpu()
    f = 2.0 ** (s.double().cpu() - 127)
    f = f.repeat_interleave(rows, 0)[:q.shape[0]]
    return q * f.repeat_interleave(cols, 1)[:, :q.shape[1]]
