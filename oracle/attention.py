"""Plain 64-bit forms of the attention and public-weight calls, words mod 2^64 in numpy: test infrastructure, as the rest of
this package.  A sharing is a pair of uint64 arrays.  Products are the literal Alg. 1; the folded addends of the library's
material are unfolded first."""
from __future__ import annotations

import numpy as np

U64 = np.uint64
CHUNK = 64


def trunc(z, bits):
    """Local rescale of a sharing."""
    return z[0] >> U64(bits), -(-z[1] >> U64(bits))


def beaver(x, y, a, b, c_folded):
    """Alg. 1 on matrices: e = x - a, f = y - b opened; c_folded[0] = c_0 - a_0 b_0."""
    c0 = c_folded[0] + a[0] @ b[0]
    e = (x[0] - a[0]) + (x[1] - a[1])
    f = (y[0] - b[0]) + (y[1] - b[1])
    return c0 + e @ b[0] + a[0] @ f + e @ f, c_folded[1] + e @ b[1] + a[1] @ f


def position_bias(x, table, buckets, n_buckets=None):
    Tq, Tk = x[0].shape[-2:]
    n = table[0].shape[0] if n_buckets is None else n_buckets
    out = tuple(np.zeros_like(w) for w in x)
    for p in range(2):
        for i in range(Tq):
            for j in range(Tk):
                u = int(buckets[j - i + Tq - 1])
                if 0 <= u < n:
                    out[p][..., i, j] = x[p][..., i, j] + table[p][u]
    return out


def position_bias_grad(g, buckets, n_buckets):
    """(table gradient, scores gradient)"""
    Tq, Tk = g[0].shape[-2:]
    grad = tuple(np.zeros((n_buckets, g[0].shape[1]), U64) for _ in range(2))
    scores = tuple(np.zeros_like(w) for w in g)
    for p in range(2):
        for i in range(Tq):
            for j in range(Tk):
                u = int(buckets[j - i + Tq - 1])
                if 0 <= u < n_buckets:
                    grad[p][u] += g[p][..., i, j].sum(0, dtype=U64)
                    scores[p][..., i, j] = g[p][..., i, j]
    return grad, scores


def matvec4(x, q, scales, group, scale_bits):
    """x [M, K] by integers q [N, K] in [-8, 7] times scales [N, groups]"""
    w = q.astype(np.int64) * np.repeat(scales.astype(np.int64), group, axis=1)[:, :q.shape[1]]
    z = tuple(s @ w.view(U64).T for s in x)
    return trunc(z, scale_bits)


def step(q, k, v, decay, m, state, bits=16):
    """One token; q, k [B, H, dk], v [B, H, dv], state [B, H, dk, dv]."""
    B, H, dk, dv = state[0].shape
    o, new = tuple(np.empty((B, H, dv), U64) for _ in range(2)), tuple(np.empty_like(s) for s in state)
    for b in range(B):
        for h in range(H):
            col = lambda s: tuple(w[b, h][:, None] for w in s)
            row = lambda s: tuple(w[b, h][None] for w in s)
            mat = lambda s: tuple(w[b, h] for w in s)
            u = beaver(col(k), row(v), col(m["a_k"]), row(m["a_v"]), mat(m["c_u"]))
            g = U64(int(decay[h, 1]))
            S = trunc(tuple(s * g + w for s, w in zip(mat(state), u)), bits)
            z = trunc(beaver(row(q), S, row(m["a_q"]), mat(m["a_s"]), row(m["c_o"])), bits)
            for p in range(2):
                o[p][b, h] = z[p][0]; new[p][b, h] = S[p]
    return o, new


def linear_attention(q, k, v, decay, m, state, bits=16):
    """Chunks of 64 tokens; q, k [B, T, H, dk], v [B, T, H, dv], state [B, H, dk, dv]."""
    B, T, H, dk = q[0].shape
    dv = v[0].shape[-1]
    o, new = tuple(np.empty((B, T, H, dv), U64) for _ in range(2)), tuple(np.empty((B, H, dk, dv), U64) for _ in range(2))
    for b in range(B):
        for h in range(H):
            n, pw = b * H + h, [U64(int(d)) for d in decay[h]]
            S = tuple(s[b, h] for s in state)
            for c, t0 in enumerate(range(0, T, CHUNK)):
                L = min(CHUNK, T - t0)
                tok = slice(t0, t0 + L)
                a = {name: tuple(w[n, c] if name in ("a_s", "c_u") else w[n, tok] for w in s) for name, s in m.items()}
                Q, K, V = (tuple(w[b, tok, h] for w in s) for s in (q, k, v))
                T_ = lambda s: tuple(w.T for w in s)
                P = trunc(beaver(Q, T_(K), a["a_q"], T_(a["a_k"]), tuple(w[:, :L] for w in a["c_p"])), bits)
                D = np.zeros((L, L), U64)
                for i in range(L):
                    for j in range(i + 1):
                        D[i, j] = pw[i - j]
                low = np.tril(np.ones((L, L), U64))
                W = tuple(w * low for w in trunc(tuple(w * D for w in P), bits))
                aw = tuple(w[:, :L] * low for w in a["a_w"])
                rise, fall = np.array(pw[1:L + 1], U64)[:, None], np.array(pw[L - 1::-1][:L], U64)[:, None]
                Qd, Kd = trunc(tuple(w * rise for w in Q), bits), trunc(tuple(w * fall for w in K), bits)
                O = trunc(beaver(tuple(np.hstack(s) for s in zip(W, Qd)), tuple(np.vstack(s) for s in zip(V, S)),
                                 tuple(np.hstack(s) for s in zip(aw, a["a_qd"])), tuple(np.vstack(s) for s in zip(a["a_v"], a["a_s"])),
                                 a["c_o"]), bits)
                U = beaver(T_(Kd), V, T_(a["a_kd"]), a["a_v"], a["c_u"])
                S = trunc(tuple(s * pw[L] + u for s, u in zip(S, U)), bits)
                for p in range(2):
                    o[p][b, tok, h] = O[p]
            for p in range(2):
                new[p][b, h] = S[p]
    return o, new
