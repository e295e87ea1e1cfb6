"""Plain 64-bit forms of the operators of a step over drafted tokens, on the CPU, for their tests."""
import math

import numpy as np
import torch


def lora(A, W, La, Lb, adapter, scale):
    """(C, sum of absolute products) in fp64."""
    A, W = A.double(), W.double()
    C, S = A @ W.T, A.abs() @ W.abs().T
    for a in range(La.shape[0]):
        rows = (adapter == a).nonzero()[:, 0]
        la, lb, s = La[a].double(), Lb[a].double(), float(scale[a])
        C[rows] += s * (A[rows] @ la.T) @ lb.T
        S[rows] += abs(s) * (A[rows].abs() @ la.abs().T) @ lb.abs().T
    return C, S


def rope_frequencies(rot, base, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=8192):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        turns = original_len * f / (2 * math.pi)
        keep = 1.0 if scaling == "none" else 0.0 if scaling == "linear" else min(1.0, max(0.0, (turns - low) / (high - low)))
        out.append(f * keep + f / factor * (1.0 - keep))
    return torch.tensor(out, dtype=torch.float64)


def rope(x, positions, rot, layout, freq, amplitude=1.0, inverse=False):
    x = x.double()
    half = rot // 2
    i = torch.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + half)
    t = (positions.double()[:, None] * freq)[:, None]
    c, s = amplitude * t.cos(), amplitude * t.sin() * (-1 if inverse else 1)
    a, b = x[..., ia], x[..., ib]
    y = x.clone()
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    return y


def tree_attention(q, k, v, pool, table, lens, offs, mask, scale, max_nodes=None, max_len=None):
    """out, lse, what the weights' errors are measured by (sum of weight * |v|), the largest sum of |q k| scale of a row; fp64.  Rows of
    nodes that are not computed: NaN."""
    N, hq, hd = q.shape
    G = hq // k.shape[1]
    out = torch.full((N, hq, hd), float("nan"), dtype=torch.float64)
    lse, mag, size = torch.full((N, hq), float("nan"), dtype=torch.float64), torch.zeros_like(out), torch.zeros((N, hq), dtype=torch.float64)
    for b in range(len(lens)):
        o0, o1 = int(offs[b]), int(offs[b + 1])
        n = o1 - o0 if max_nodes is None else min(o1 - o0, max_nodes)
        length = max(0, int(lens[b]))
        if max_len is not None:
            length = min(length, max_len)
        if table is not None:
            length = min(length, 16 * table.shape[1])
        pos = [p for p in range(length) if 0 <= int(table[b, p // 16]) < pool.shape[0]]
        page = torch.tensor([int(table[b, p // 16]) for p in pos], dtype=torch.long)
        slot = torch.tensor([p % 16 for p in pos], dtype=torch.long)
        for i in range(o0, o0 + n):
            seen = [j for j in range(n) if (j <= i - o0 if mask is None else int(mask[i, j // 64]) >> (j % 64) & 1)]
            at = torch.tensor([o0 + j for j in seen], dtype=torch.long)
            for h in range(hq):
                g = h // G
                K, V = k[at, g].double(), v[at, g].double()
                if len(pos):
                    K, V = torch.cat((pool[page, 0, g, slot].double(), K)), torch.cat((pool[page, 1, g, slot].double(), V))
                if K.shape[0] == 0:
                    out[i, h], lse[i, h] = 0.0, -math.inf
                    continue
                s = K @ q[i, h].double() * scale
                w = torch.softmax(s, 0)
                out[i, h], mag[i, h] = w @ V, w @ V.abs()
                lse[i, h] = torch.logsumexp(s, 0)
                size[i, h] = (K.abs() @ q[i, h].double().abs() * abs(scale)).max()
    return out, lse, mag, size


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log share, kept, distance of the nearest border of a decision, relative to the mass).  All by their definition in fp64."""
    l = np.asarray(logits, dtype=np.float64)
    order = np.argsort(np.where(np.isnan(l), np.inf, -l), kind="stable")
    order = [int(i) for i in order if l[i] > -np.inf]
    if not order:
        return -1, -math.inf, 0, 1.0
    if not temperature > 0:
        return order[0], 0.0, 1, 1.0
    x = np.array([0.0 if l[i] == l[order[0]] else (l[i] - l[order[0]]) / temperature for i in order])
    w = np.exp(x)
    w = w[w > 0]
    n, margin = len(w), 1.0
    if top_k > 0:
        n = min(n, top_k)
    k = n
    if top_p < 1:
        before = np.cumsum(w[:k]) - w[:k]
        edge = before / w[:k].sum() - max(top_p, 0.0)
        n = min(n, max(1, int((edge < 0).sum())))
        margin = min(margin, float(np.abs(edge[1:]).min()) if k > 1 else 1.0)
    if min_p > 0:
        n = min(n, max(1, int((w >= min_p).sum())))
        near = np.abs(w[1:] - min_p)
        margin = min(margin, float(near.min()) if len(near) else 1.0)
    cum = np.cumsum(w[:n])
    target = min(max(u, 0.0), 1.0) * cum[-1]
    j = min(int((cum <= target).sum()), n - 1)
    if n > 1:
        margin = min(margin, float(np.abs(cum[:-1] - target).min() / cum[-1]))
    return order[j], math.log(w[j] / cum[-1]), n, margin
