"""Plain 64-bit oracle of the layer operators in ``include/poseidon_layers.h`` (numpy, row by row definitions).

Test infrastructure: shares no code with the HIP path.
"""
import numpy as np

GROUP = 64
EXPONENTS = {"f32": (-126, 121), "bf16": (-126, 121), "f16": (-24, 9)}


def stash(x, kind):
    """(codes int8 [n, groups * 64], scale bytes uint8 [n, groups]) of float64 rows x that hold values of type `kind`."""
    n, d = x.shape
    g = -(-d // GROUP)
    low, high = EXPONENTS[kind]
    codes = np.zeros((n, g * GROUP), np.int8)
    scales = np.zeros((n, g), np.uint8)
    for b in range(g):
        v = x[:, b * GROUP:(b + 1) * GROUP]
        a = np.abs(v).max(axis=1)
        for r in range(n):
            if not np.isfinite(a[r]):
                scales[r, b] = 255
                continue
            e = low
            if a[r] > 0:
                e = int(np.floor(np.log2(a[r]))) - 8
                while a[r] > 127 * 2.0 ** e:
                    e += 1
            e = min(max(e, low), high)
            scales[r, b] = e + 127
            codes[r, b * GROUP:b * GROUP + v.shape[1]] = np.clip(np.round(v[r] / 2.0 ** e), -127, 127)
    return codes, scales


def restore(codes, scales, d):
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (codes.astype(np.float64) * np.repeat(unit, GROUP, axis=1))[:, :d]


def sigmoid(z):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-z))


def gated_forward(gate, up):
    return gate * sigmoid(gate) * up


def gated_backward(dout, gate, up):
    s = sigmoid(gate)
    return dout * up * s * (1 + gate * (1 - s)), dout * gate * s


def weight_gradient(dy, x, offsets):
    return np.stack([dy[a:b].T @ x[a:b] for a, b in zip(offsets[:-1], offsets[1:])])


def expert_sort(choice, experts):
    """(order, position, offsets) of the flat choices, by insertion into the experts' lists."""
    lists = [[] for _ in range(experts + 1)]
    for i, c in enumerate(choice.reshape(-1).tolist()):
        lists[c if 0 <= c < experts else experts].append(i)
    order = np.array([i for one in lists for i in one], np.int64)
    offsets = np.concatenate([[0], np.cumsum([len(one) for one in lists[:experts]])])
    position = np.full(choice.size, -1, np.int64)
    position[order[:offsets[-1]]] = np.arange(offsets[-1])
    return order, position.reshape(choice.shape), offsets


def expert_gather(x, position):
    n, k = position.shape
    xs = np.zeros((n * k, x.shape[1]))
    for t in range(n):
        for j in range(k):
            if position[t, j] >= 0:
                xs[position[t, j]] = x[t]
    return xs


def expert_combine(ys, position, weights):
    n, k = position.shape
    out = np.zeros((n, ys.shape[1]))
    for t in range(n):
        for j in range(k):
            if position[t, j] >= 0:
                out[t] += weights[t, j] * ys[position[t, j]]
    return out


def expert_combine_backward(dout, ys, position, weights):
    n, k = position.shape
    dys, dw = np.zeros_like(ys), np.zeros((n, k))
    for t in range(n):
        for j in range(k):
            p = position[t, j]
            if p >= 0:
                dys[p] = weights[t, j] * dout[t]
                dw[t, j] = dout[t] @ ys[p]
    return dys, dw


def embed(ids, table, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids.tolist()):
        if 0 <= i < len(table):
            out[t] = scale * table[i]
    return out


def embed_backward(ids, dout, vocab, scale):
    d = np.zeros((vocab, dout.shape[1]))
    for t, i in enumerate(ids.tolist()):
        if 0 <= i < vocab:
            d[i] += scale * dout[t]
    return d


def norm_forward(x, residual, weight, eps):
    """(out, sum, 1 / root of the mean square of each row)"""
    h = x if residual is None else x + residual
    rstd = 1 / np.sqrt((h * h).sum(axis=1) / h.shape[1] + eps)
    return h * rstd[:, None] * weight, h, rstd


def norm_backward(dout, h, rstd, weight, dsum):
    """(dx, dweight) for the rstd that is given"""
    n, g = h * rstd[:, None], dout * weight
    dx = rstd[:, None] * (g - n * (n * g).sum(axis=1, keepdims=True) / h.shape[1])
    return dx if dsum is None else dx + dsum, (dout * n).sum(axis=0)


def expert_product(x, weights, offsets, transposed):
    out = np.zeros((x.shape[0], weights.shape[2] if transposed else weights.shape[1]))
    for w, a, b in zip(weights, offsets, offsets[1:]):
        out[a:b] = x[a:b] @ (w if transposed else w.T)
    return out


def attention_forward(q, k, v, offsets, scale):
    """(out [tokens, heads, dim], lse [heads, tokens]), a query at a time."""
    n, heads, _ = q.shape
    group = heads // k.shape[1]
    out, lse = np.zeros(q.shape[:2] + v.shape[2:]), np.full((heads, n), -np.inf)
    for a, b in zip(offsets, offsets[1:]):
        for h in range(heads):
            for i in range(a, b):
                s = scale * (k[a:i + 1, h // group] @ q[i, h])
                p = np.exp(s - s.max())
                out[i, h] = p @ v[a:i + 1, h // group] / p.sum()
                lse[h, i] = s.max() + np.log(p.sum())
    return out, lse


def attention_backward(dout, q, k, v, out, offsets, scale):
    """(dq, dk, dv), a sequence and a head at a time."""
    heads = q.shape[1]
    group = heads // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for a, b in zip(offsets, offsets[1:]):
        later = np.triu(np.ones((b - a, b - a), bool), 1)
        for h in range(heads):
            j = h // group
            s = np.where(later, -np.inf, scale * q[a:b, h] @ k[a:b, j].T)
            p = np.exp(s - s.max(axis=1, keepdims=True)) if b > a else s
            p /= p.sum(axis=1, keepdims=True)
            ds = p * (dout[a:b, h] @ v[a:b, j].T - (dout[a:b, h] * out[a:b, h]).sum(axis=1, keepdims=True))
            dq[a:b, h] = scale * ds @ k[a:b, j]
            dk[a:b, j] += scale * ds.T @ q[a:b, h]
            dv[a:b, j] += p.T @ dout[a:b, h]
    return dq, dk, dv
