"""The attention operators from their definitions, in 64 bits on the CPU, one query at a
time; nothing here is shared with the library."""
from __future__ import annotations

import math

import torch


def sees(i, j, start, end, causal, prefix, window):
    """Whether query i sees key j, both tokens of the document [start, end)."""
    if causal and not (j <= i or j < start + prefix):
        return False
    if window and i - j >= window:
        return False
    return not (window and not causal and j - i >= window)


def masks(T, doc_start, causal=True, prefix=None, window=0):
    """[T][T] of what each query sees."""
    m = torch.zeros((T, T), dtype=torch.bool)
    for n, (a, b) in enumerate(zip(doc_start, doc_start[1:])):
        i = torch.arange(a, b)[:, None]
        j = torch.arange(a, b)[None, :]
        ok = torch.ones((b - a, b - a), dtype=torch.bool)
        if causal:
            ok = j <= i
            if prefix is not None:
                ok = ok | (j < a + prefix[n])
        if window:
            ok = ok & (i - j < window)
            if not causal:
                ok = ok & (j - i < window)
        m[a:b, a:b] = ok
    return m


def attention(q, k, v, seen, scale, softcap=0.0, slope=None, d_o=None):
    """o, lse and, given d_o, dq, dk, dv; only visible places are looked at."""
    q, k, v = q.double(), k.double(), v.double()
    T, nq, d = q.shape
    G = nq // k.shape[1]
    o, lse = torch.zeros_like(q), torch.full((nq, T), -math.inf, dtype=torch.float64)
    grads = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)] if d_o is not None else None
    for i in range(T):
        js = seen[i].nonzero()[:, 0]
        if not len(js):
            continue
        kk, vv = (x[js].repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))      # [h][n][d]
        z = (kk @ q[i][:, :, None])[..., 0] * scale
        t = torch.tanh(z / softcap) if softcap else None
        s = softcap * t if softcap else z
        if slope is not None:
            s = s - slope.double()[:, None] * (i - js).abs()
        lse[:, i] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[:, i, None])
        o[i] = (p[:, None, :] @ vv)[:, 0]
        if d_o is None:
            continue
        g = d_o[i].double()                                                           # [h][d]
        dp = (vv @ g[:, :, None])[..., 0]
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        if softcap:
            ds = ds * (1 - t * t)
        grads[0][i] = scale * (ds[:, None, :] @ kk)[:, 0]
        dk = scale * ds[:, :, None] * q[i][:, None, :]
        dv = p[:, :, None] * g[:, None, :]
        for x, dx in ((1, dk), (2, dv)):
            grads[x][js] += dx.view(-1, G, len(js), d).sum(1).transpose(0, 1)
    return (o, lse, *grads) if grads else (o, lse)


def rope(x, pos, table, rot, interleaved, gain=None, eps=1e-6, norm=True, dy=None):
    """y, and given dy: dx and dgain; x [T][h][d]."""
    x = x.double()
    T, h, d = x.shape
    r = torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps) if norm else torch.ones(T, h, 1, dtype=torch.float64)
    g = gain.double() if norm and gain is not None else torch.ones(d, dtype=torch.float64)
    xn = x / r
    turn = torch.eye(d, dtype=torch.float64).repeat(T, 1, 1)                           # y = turn n
    half = rot // 2
    for t in range(T):
        c = table[int(pos[t])].double()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            turn[t, a, a] = turn[t, b, b] = c[i]
            turn[t, a, b], turn[t, b, a] = -c[half + i], c[half + i]
    y = torch.einsum("tij,thj->thi", turn, xn * g)
    if dy is None:
        return y
    w = torch.einsum("tij,thi->thj", turn, dy.double())
    if not norm:
        return y, w, None
    gw = g * w
    return y, (gw - xn * (gw * xn).mean(-1, keepdim=True)) / r, (w * xn).sum((0, 1))


def paged(q, k_cache, v_cache, page_table, kv_len, q_len, scale, window=0, softcap=0.0, slope=None):
    """o [rows][h][d] and lse [rows][h]."""
    rows, nq, d = q.shape
    page, G = k_cache.shape[1], nq // k_cache.shape[2]
    o, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full((rows, nq), -math.inf, dtype=torch.float64)
    for r in range(rows):
        n, length = r // q_len, int(kv_len[r // q_len])
        at = length - q_len + r % q_len
        if at < 0:
            continue
        js = torch.arange(max(0, at - window + 1) if window else 0, at + 1)
        ids = page_table[n, js // page].long()
        kk, vv = (c[ids, js % page].double().repeat_interleave(G, 1).transpose(0, 1) for c in (k_cache, v_cache))
        s = (kk @ q[r].double()[:, :, None])[..., 0] * scale
        if softcap:
            s = softcap * torch.tanh(s / softcap)
        if slope is not None:
            s = s - slope.double()[:, None] * (at - js)
        lse[r] = torch.logsumexp(s, 1)
        o[r] = (torch.exp(s - lse[r][:, None])[:, None] @ vv)[:, 0]
    return o, lse
