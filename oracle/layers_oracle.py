"""Float64 numpy implementation of the layers of include/rnngraph_layers.h, from their definitions: linear attention
frame by frame, the residual sum with dropout and root-mean-square norm row by row, the dropout generator."""
import numpy as np


def attention_forward(q, k, v, log_decay, scale, state=None, lengths=None):
    """q [T][N][H][dk], k, v with H / group heads.  Returns o (zeros behind a stream's length) and the final state."""
    T, N, H, dk = q.shape
    rep = H // k.shape[2]
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    k, v = np.repeat(k, rep, 2), np.repeat(v, rep, 2)
    L = np.full(N, T) if lengths is None else np.clip(lengths, 0, T)
    g = np.exp(np.minimum(np.asarray(log_decay, np.float64), 0.0))[:, None, None]
    S = np.zeros((N, H, dk, v.shape[3])) if state is None else np.array(state, np.float64)
    o = np.zeros((T, N, H, v.shape[3]))
    for n in range(N):
        for t in range(L[n]):
            S[n] = g * S[n] + k[t, n, :, :, None] * v[t, n, :, None, :]
            o[t, n] = scale * np.einsum("hi,hij->hj", q[t, n], S[n])
    return o, S


def attention_backward(q, k, v, log_decay, scale, do, state=None, dstate_out=None, lengths=None):
    """(dq, dk, dv, dstate_in): the chain rule through attention_forward's loop, backwards."""
    T, N, H, dk = q.shape
    Hk = k.shape[2]
    rep = H // Hk
    q, k, v, do = (np.asarray(x, np.float64) for x in (q, k, v, do))
    k, v = np.repeat(k, rep, 2), np.repeat(v, rep, 2)
    L = np.full(N, T) if lengths is None else np.clip(lengths, 0, T)
    g = np.exp(np.minimum(np.asarray(log_decay, np.float64), 0.0))[:, None, None]
    S = np.zeros((N, H, dk, v.shape[3])) if state is None else np.array(state, np.float64)
    G = np.zeros_like(S) if dstate_out is None else np.array(dstate_out, np.float64)
    dq, dkk, dvv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for n in range(N):
        for t in range(L[n]):
            S[n] = g * S[n] + k[t, n, :, :, None] * v[t, n, :, None, :]
            dq[t, n] = scale * np.einsum("hij,hj->hi", S[n], do[t, n])
        for t in range(L[n] - 1, -1, -1):
            G[n] += scale * q[t, n, :, :, None] * do[t, n, :, None, :]
            dkk[t, n] = np.einsum("hij,hj->hi", G[n], v[t, n])
            dvv[t, n] = np.einsum("hij,hi->hj", G[n], k[t, n])
            G[n] *= g
    shared = lambda x: x.reshape(T, N, Hk, rep, -1).sum(3)  # noqa: E731
    return dq, shared(dkk), shared(dvv), G


def philox4x32(counter, key, rounds):
    """counter [..., 4], key [2]: uint32 words.  Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3 (2011)."""
    c = [np.asarray(counter)[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> sh) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1).astype(np.uint32)


def dropout_factor(rows, dim, p, seed, offset, first_row=0):
    """[rows][dim]: 0 where an element is dropped, 1 / (1 - p) where it is kept, p rounded to a multiple of 2^-16."""
    cut = int(np.floor(p * 65536 + 0.5))
    if cut == 0:
        return np.ones((rows, dim))
    if cut == 65536:
        return np.zeros((rows, dim))
    groups = -(-dim // 8)
    at = (np.arange(rows, dtype=np.uint64)[:, None] + np.uint64(first_row)) * np.uint64(groups) + np.arange(groups, dtype=np.uint64)
    ctr = np.empty((rows, groups, 4), np.uint32)
    ctr[..., 0], ctr[..., 1] = at & np.uint64(0xFFFFFFFF), at >> np.uint64(32)
    ctr[..., 2], ctr[..., 3] = offset & 0xFFFFFFFF, offset >> 32
    w = philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32), 7)
    u = np.stack([w & 0xFFFF, w >> 16], -1).reshape(rows, groups * 8)[:, :dim]
    return np.where(u >= cut, 65536.0 / (65536 - cut), 0.0)


def add_norm(x, residual, gain, eps, factor):
    """h, y, rstd of rows [rows][dim]; dropped elements count as 0 whatever they hold."""
    h = np.where(factor > 0, np.asarray(x, np.float64) * factor, 0.0) + (0.0 if residual is None else np.asarray(residual, np.float64))
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h, h * rstd[:, None] * (1.0 if gain is None else np.asarray(gain, np.float64)), rstd


def add_norm_backward(dy, dh, h, rstd, gain, factor):
    """dx, dresidual, dgain."""
    dy, h, r = np.asarray(dy, np.float64), np.asarray(h, np.float64), np.asarray(rstd, np.float64)[:, None]
    n, gd = h * r, dy * (1.0 if gain is None else np.asarray(gain, np.float64))
    s = (0.0 if dh is None else np.asarray(dh, np.float64)) + r * (gd - n * (gd * n).mean(1, keepdims=True))
    return np.where(factor > 0, s * factor, 0.0), s, (dy * n).sum(0)
