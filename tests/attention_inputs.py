"""Seeded inputs of the attention and public-weight calls, in numpy; shared by the tests of this group."""
import numpy as np

from paper_2209_13643_amd import synth

U64 = np.uint64
CHUNK = 64


def words(rng, *shape):
    return synth.rand_words(rng, shape)


def share(rng, value):
    return synth.share_additive(rng, value)


def fixed(rng, std, *shape):
    return synth.normal_fixed(rng, shape, std)


def masks(rng, *shape):
    return words(rng, *shape), words(rng, *shape)


def folded(rng, total, own):
    c0, c1 = share(rng, total)
    return c0 - own, c1


def step_material(rng, B, H, dk, dv):
    m = dict(a_q=masks(rng, B, H, dk), a_k=masks(rng, B, H, dk), a_v=masks(rng, B, H, dv), a_s=masks(rng, B, H, dk, dv))
    outer = lambda a, b: a[..., :, None] * b[..., None, :]
    m["c_u"] = folded(rng, outer(sum(m["a_k"]), sum(m["a_v"])), outer(m["a_k"][0], m["a_v"][0]))
    times = lambda a, b: (a[..., :, None] * b).sum(-2, dtype=U64)
    m["c_o"] = folded(rng, times(sum(m["a_q"]), sum(m["a_s"])), times(m["a_q"][0], m["a_s"][0]))
    return m


def prompt_material(rng, B, H, T, dk, dv):
    N, nc = B * H, -(-T // CHUNK)
    m = {n: masks(rng, N, T, dk) for n in ("a_q", "a_k", "a_qd", "a_kd")}
    m["a_v"], m["a_w"], m["a_s"] = masks(rng, N, T, dv), masks(rng, N, T, CHUNK), masks(rng, N, nc, dk, dv)
    cp, cu, co = ([np.zeros(s, U64) for _ in range(2)] for s in ((N, T, CHUNK), (N, nc, dk, dv), (N, T, dv)))
    for i, take in enumerate((sum, lambda s: s[0])):          # the whole product, party 0's own
        for n in range(N):
            for c in range(nc):
                t = slice(c * CHUNK, min(T, (c + 1) * CHUNK))
                L = t.stop - t.start
                a = {x: take([w[n, t] for w in m[x]]) for x in ("a_q", "a_k", "a_qd", "a_kd", "a_v", "a_w")}
                s = take([w[n, c] for w in m["a_s"]])
                cp[i][n, t, :L] = a["a_q"] @ a["a_k"].T
                cu[i][n, c] = a["a_kd"].T @ a["a_v"]
                co[i][n, t] = np.tril(a["a_w"][:, :L]) @ a["a_v"] + a["a_qd"] @ s
    for name, (total, own) in (("c_p", cp), ("c_u", cu), ("c_o", co)):
        m[name] = folded(rng, total, own)
    return m


def prompt(rng, B, H, T, dk, dv, state=True):
    d = dict(q=share(rng, fixed(rng, 0.125, B, T, H, dk)), k=share(rng, fixed(rng, 0.125, B, T, H, dk)),
             v=share(rng, fixed(rng, 1.0, B, T, H, dv)), mat=prompt_material(rng, B, H, T, dk, dv))
    d["state"] = share(rng, fixed(rng, 0.5, B, H, dk, dv)) if state else None
    return d


def one_token(rng, B, H, dk, dv):
    return dict(q=share(rng, fixed(rng, 0.125, B, H, dk)), k=share(rng, fixed(rng, 0.125, B, H, dk)), v=share(rng, fixed(rng, 1.0, B, H, dv)),
                mat=step_material(rng, B, H, dk, dv), state=share(rng, fixed(rng, 0.5, B, H, dk, dv)))
