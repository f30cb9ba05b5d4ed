"""Attention without a softmax and 4-bit public weights on secret shares, as timed cases.

A sharing is a pair of arrays of 64-bit words, x = x_0 + x_1 mod 2^64, of fixed-point values with 16 fraction bits; here
a pair is one tensor whose first axis is the party.  All results are ring words, the same in every bit however they are
computed.  The offline material (masks a_*, addends c_*, party 0's with its local product folded in), decays, bucket maps
and public weights are what a program holds before the shares arrive.

  bias         scores[b,h,i,j] + table[bucket[j - i + Tq - 1], h]; pairs without a bucket become zero
  bias-grad    the table's gradient (sums over batch and pairs) and, under a mask, the scores' (zero where there is no bucket)
  matvec4      x W^T, W public: 4-bit integers times one fixed-point scale for each row and group of columns
  step         one token of linear attention: S <- trunc(decay S + k v^T), o = trunc(q S)
  prompt       the same over chunks of 64 tokens
"""
import functools
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
FRAC = 16
CHUNK = 64
MAX_PAIRS = 8 * 12 * 512 * 512           # pairs of the largest listed bias
MAX_WEIGHTS = 25088 * 4096
MAX_STATE = 128 * 16 * 64 * 64
MAX_PROMPT = 8 * 12 * 512 * (64 + 64)


def listed():
    return [
        # encoder layer of 512 tokens: batch 8, 12 heads, both directions
        dict(name="bias-encoder", kind="bias", B=8, H=12, Tq=512, Tk=512, buckets=32, far=128, causal=False),
        # one new token against what came before, 16 heads: launch and latency
        dict(name="bias-one-token", kind="bias", B=1, H=16, Tq=1, Tk=577, buckets=32, far=128, causal=True),
        # training step of the encoder layer, and of a causal one with an odd length
        dict(name="bias-grad-encoder", kind="bias-grad", B=8, H=12, Tq=512, Tk=512, buckets=32, far=128, causal=False),
        dict(name="bias-grad-causal-odd", kind="bias-grad", B=2, H=12, Tq=197, Tk=197, buckets=48, far=200, causal=True),
        # the encoder's QKV projection of one token, the image classifier's first dense layer of one image,
        # and a few tokens at once through a 1024-wide layer with small groups
        dict(name="matvec4-qkv", kind="matvec4", M=1, K=768, N=2304, group=64),
        dict(name="matvec4-classifier", kind="matvec4", M=1, K=25088, N=4096, group=128),
        dict(name="matvec4-8rows", kind="matvec4", M=8, K=1024, N=4096, group=32),
        # one token of every sequence: the encoder's heads, and a large serving batch of 16 heads
        dict(name="step-encoder", kind="step", B=8, H=12, dk=64, dv=64),
        dict(name="step-batch", kind="step", B=128, H=16, dk=64, dv=64),
        # prompts: the encoder layer at its 512 tokens, one ragged sequence with narrow heads, long sequences with wide ones
        dict(name="prompt-encoder", kind="prompt", B=8, T=512, H=12, dk=64, dv=64),
        dict(name="prompt-odd", kind="prompt", B=1, T=205, H=12, dk=48, dv=40),
        dict(name="prompt-wide-long", kind="prompt", B=1, T=1500, H=8, dk=128, dv=128),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["bias", "bias-grad", "matvec4", "step", "prompt"])
    while True:
        if kind in ("bias", "bias-grad"):
            Tk = _log(rng, 1, 1500)
            Tq = rng.choice([1, Tk, Tk, rng.randint(1, Tk)])
            c = dict(kind=kind, B=_log(rng, 1, 32), H=rng.choice([1, 6, 12, 16]), Tq=Tq, Tk=Tk, buckets=2 * rng.randint(4, 32),
                     far=rng.randint(64, 400), causal=rng.random() < 0.5)
            if c["B"] * c["H"] * Tq * Tk <= MAX_PAIRS:
                return c
        elif kind == "matvec4":
            c = dict(kind=kind, M=_log(rng, 1, 16), K=_log(rng, 32, 25088), N=_log(rng, 10, 4096), group=rng.choice([32, 64, 128, 256]))
            if c["K"] * c["N"] * max(1, c["M"] // 4) <= MAX_WEIGHTS:
                return c
        elif kind == "step":
            c = dict(kind=kind, B=_log(rng, 1, 128), H=rng.choice([1, 5, 12, 16]), dk=rng.randint(8, 128), dv=rng.randint(8, 128))
            if c["B"] * c["H"] * c["dk"] * c["dv"] <= MAX_STATE:
                return c
        else:
            c = dict(kind=kind, B=_log(rng, 1, 16), T=_log(rng, 1, 1500), H=rng.choice([1, 5, 12, 16]), dk=rng.randint(8, 128),
                     dv=rng.randint(8, 128))
            if c["B"] * c["T"] * c["H"] * (c["dk"] + c["dv"]) <= MAX_PROMPT:
                return c


# ------------------------------------------------------------------------------------------------ states
def _words(g, *shape):
    hi = torch.randint(-(1 << 31), 1 << 31, shape, generator=g, device=DEVICE, dtype=torch.int64)
    return (hi << 32) | torch.randint(0, 1 << 32, shape, generator=g, device=DEVICE, dtype=torch.int64)


def _share(g, value):
    first = _words(g, *value.shape)
    return torch.stack((first, value - first))


def _fixed(g, std, *shape):
    return torch.round(torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float64) * (std * (1 << FRAC))).to(torch.int64)


def _bucket_map(c):
    """Bucket of every relative position j - i (the last query stands at the last key): near ones each have their own, far
    ones share by their logarithm; -1 for a key behind its query in a causal map."""
    rel = torch.arange(c["Tq"] + c["Tk"] - 1) - (c["Tq"] - 1) - (c["Tk"] - c["Tq"])
    n = c["buckets"] if c["causal"] else c["buckets"] // 2
    near = n // 2
    d = rel.abs()
    log = torch.log(d.clamp(min=1).double() / near) / math.log(c["far"] / near) * (n - near)
    at = torch.where(d < near, d, (near + log.clamp(min=0).long()).clamp(max=n - 1))
    at = torch.where(rel > 0, -1 if c["causal"] else at + n, at)
    return at.to(torch.int32).to(DEVICE)


def _decays(H):
    """Powers 0..64 of every head's decay, 16 fraction bits: 1 - 2^-5, 1 - 2^-6, ... as heads look further back."""
    decay = 1 - 2.0 ** (-5 - torch.arange(H, dtype=torch.float64) % 8)
    return torch.round(decay[:, None] ** torch.arange(CHUNK + 1) * (1 << FRAC)).to(torch.int32).to(DEVICE)


def _addend(g, *products):
    """Shares of the sum of A B over the given (a, b) masks, with party 0's own a_0 b_0 taken off."""
    c = _share(g, sum(_matmul(a[0] + a[1], b[0] + b[1]) for a, b in products))
    c[0] -= sum(_matmul(a[0], b[0]) for a, b in products)
    return c


def _prompt_state(g, c):
    B, T, H, dk, dv = (c[n] for n in ("B", "T", "H", "dk", "dv"))
    N, chunks = B * H, -(-T // CHUNK)
    s = {}
    if dk == dv:                          # as the QKV projection leaves them: one row of 3 H d words a token
        qkv = _share(g, _fixed(g, 1.0, B, T, 3, H, dk) // torch.tensor([8, 8, 1], device=DEVICE)[:, None, None])
        s["q"], s["k"], s["v"] = qkv[:, :, :, 0], qkv[:, :, :, 1], qkv[:, :, :, 2]
    else:
        s["q"], s["k"], s["v"] = (_share(g, _fixed(g, std, B, T, H, d)) for std, d in ((0.125, dk), (0.125, dk), (1.0, dv)))
    s["state"] = _share(g, _fixed(g, 0.5, B, H, dk, dv))
    mat = {n: _words(g, 2, N, T, dk) for n in ("a_q", "a_k", "a_qd", "a_kd")}
    mat["a_v"], mat["a_s"], mat["a_w"] = _words(g, 2, N, T, dv), _words(g, 2, N, chunks, dk, dv), _words(g, 2, N, T, CHUNK)
    # nothing above a chunk's diagonal is masked or opened
    mat["a_w"] *= torch.arange(CHUNK, device=DEVICE) <= (torch.arange(T, device=DEVICE) % CHUNK)[:, None]
    q, k, kd, v, w = (_chunks(mat[n]) for n in ("a_q", "a_k", "a_kd", "a_v", "a_w"))
    mat["c_p"] = _tokens(_addend(g, (q, k.transpose(-1, -2))), T)
    mat["c_u"] = _addend(g, (kd.transpose(-1, -2), v))
    mat["c_o"] = _tokens(_addend(g, (w, v), (_chunks(mat["a_qd"]), mat["a_s"])), T)
    s.update(mat=mat, decay=_decays(H), o=torch.empty(2, B, T, H, dv, dtype=torch.int64, device=DEVICE), new=torch.empty_like(s["state"]))
    return s


def _step_state(g, c):
    B, H, dk, dv = (c[n] for n in ("B", "H", "dk", "dv"))
    s = {n: _share(g, _fixed(g, std, B, H, d)) for n, std, d in (("q", 0.125, dk), ("k", 0.125, dk), ("v", 1.0, dv))}
    s["state"] = _share(g, _fixed(g, 0.5, B, H, dk, dv))
    mat = {"a_q": _words(g, 2, B, H, dk), "a_k": _words(g, 2, B, H, dk), "a_v": _words(g, 2, B, H, dv), "a_s": _words(g, 2, B, H, dk, dv)}
    mat["c_u"] = _addend(g, (mat["a_k"].unsqueeze(-1), mat["a_v"].unsqueeze(-2)))
    mat["c_o"] = _addend(g, (mat["a_q"].unsqueeze(-2), mat["a_s"])).squeeze(-2)
    s.update(mat=mat, decay=_decays(H), o=torch.empty(2, B, H, dv, dtype=torch.int64, device=DEVICE), new=torch.empty_like(s["state"]))
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    kind = case["kind"]
    s = dict(kind=kind)
    if kind in ("bias", "bias-grad"):
        B, H, Tq, Tk, n = (case[x] for x in ("B", "H", "Tq", "Tk", "buckets"))
        scores = _words(g, 2, B, H, Tq, Tk)
        scores[1] = torch.round(torch.randn(B, H, Tq, Tk, generator=g, device=DEVICE) * (1 << FRAC)).to(torch.int64) - scores[0]
        s.update(x=scores, buckets=_bucket_map(case), n=n)
        if kind == "bias":
            s["table"] = _share(g, _fixed(g, 0.5, n, H))
        else:
            s["grad"] = torch.empty(2, n, H, dtype=torch.int64, device=DEVICE)
        if kind == "bias" or case["causal"]:                 # without masked pairs the scores' gradient is the given one
            s["y"] = torch.empty_like(scores)
    elif kind == "matvec4":
        M, K, N, group = (case[x] for x in ("M", "K", "N", "group"))
        # rows of 16 bytes for every 32 columns, the even column of a byte in its low half
        w = torch.randint(0, 256, (N, -(-K // 32) * 16), generator=g, device=DEVICE, dtype=torch.uint8)
        scale = torch.rand(N, -(-K // group), generator=g, device=DEVICE, dtype=torch.float64) * 0.4 + 0.8
        s.update(x=_share(g, _fixed(g, 1.0, M, K)), w=w, scales=torch.round(scale * (K ** -0.5 / 4.6) * (1 << 20)).to(torch.int32), group=group,
                 y=torch.empty(2, M, N, dtype=torch.int64, device=DEVICE))
    elif kind == "step":
        s.update(_step_state(g, case))
    else:
        s.update(_prompt_state(g, case))
    # the same tensors as a pair of shares each, as the framework's calls take them
    s["pair"] = {n: tuple(t.unbind(0)) for n, t in s.items() if isinstance(t, torch.Tensor) and t.dtype == torch.int64}
    s["pair"]["mat"] = {n: tuple(t.unbind(0)) for n, t in s.get("mat", {}).items()}
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------ plain form
def _matmul(a, b):
    """Product mod 2^64 from 16-bit limbs: their products and the sums over up to 2^19 terms are exact in float64."""
    a, b = ([((x >> (16 * i)) & 0xFFFF).double() for i in range(4)] for x in (a, b))
    return sum((torch.cat(a[:s + 1], -1) @ torch.cat(b[s::-1], -2)).to(torch.int64) << (16 * s) for s in range(4))


def _rescale(z, bits=FRAC):
    """z_0 >> bits and -((-z_1) >> bits), logical shifts."""
    mask = (1 << (64 - bits)) - 1
    return torch.stack(((z[0] >> bits) & mask, -((-z[1] >> bits) & mask)))


def _product(x, y, a, b, c):
    """Shares of x y: e = x - a and f = y - b are opened; party 0 has c_0 + (x_0 + e_1)(y_0 + f_1), party 1 c_1 + e b_1 + a_1 f."""
    e, f = x - a, y - b
    return torch.stack((c[0] + _matmul(x[0] + e[1], y[0] + f[1]),
                        c[1] + _matmul(torch.cat((e[0] + e[1], a[1]), -1), torch.cat((b[1], f[0] + f[1]), -2))))


def _chunks(t):
    """[2, N, T, d] as [2, N, chunks, 64, d], zeros behind the last token."""
    T = t.shape[2]
    return torch.nn.functional.pad(t, (0, 0, 0, -T % CHUNK)).unflatten(2, (-1, CHUNK))


def _tokens(t, T):
    return t.flatten(2, 3)[:, :, :T].contiguous()


def _by_pair(of_distance, Tq, Tk):
    """[..., Tq + Tk - 1] by distance as [..., Tq, Tk]."""
    at = torch.arange(Tk, device=DEVICE) - torch.arange(Tq, device=DEVICE)[:, None] + Tq - 1
    return of_distance[..., at]


def _plain_bias(s):
    Tq, Tk = s["x"].shape[-2:]
    kept = _by_pair(s["buckets"] >= 0, Tq, Tk)
    of_distance = s["table"][:, s["buckets"].clamp(min=0).long()].transpose(1, 2)
    return (s["x"] + _by_pair(of_distance, Tq, Tk)[:, None]) * kept


def _plain_bias_grad(s):
    Tq, Tk = s["x"].shape[-2:]
    bucket = _by_pair(s["buckets"].long(), Tq, Tk).flatten()
    kept = bucket >= 0
    by_pair = s["x"].sum(1).flatten(2)                                      # [2, H, Tq Tk]
    grad = torch.zeros(2, by_pair.shape[1], s["n"], dtype=torch.int64, device=DEVICE)
    grad.index_add_(2, bucket.clamp(min=0), by_pair * kept)
    grad = grad.transpose(1, 2).contiguous()
    return (grad, s["x"] * kept.view(Tq, Tk)) if "y" in s else grad


def _plain_matvec4(s):
    K, group = s["x"].shape[-1], s["group"]
    groups = -(-K // group)
    w = torch.stack((s["w"] & 15, s["w"] >> 4), -1).flatten(1)[:, :K]
    w = torch.nn.functional.pad((w ^ 8).double() - 8, (0, groups * group - K)).view(-1, groups, group).transpose(0, 1)
    x = torch.nn.functional.pad(s["x"], (0, groups * group - K)).view(2, -1, groups, group)
    x = torch.stack([(x >> (16 * i)) & 0xFFFF for i in range(4)]).double().permute(3, 4, 0, 1, 2)        # [groups, group, 4, 2, M]
    z = (w.contiguous() @ x.flatten(2)).to(torch.int64).view(groups, -1, 4, *x.shape[3:])
    z = (z << torch.tensor([0, 16, 32, 48], device=DEVICE).view(4, 1, 1)).sum(2)                         # [groups, N, 2, M]
    return _rescale((z * s["scales"].t().long()[..., None, None]).sum(0).permute(1, 2, 0), 20)


def _plain_step(s):
    m, one = s["mat"], s["decay"][:, 1].long()[:, None, None]
    u = _product(s["k"].unsqueeze(-1), s["v"].unsqueeze(-2), m["a_k"].unsqueeze(-1), m["a_v"].unsqueeze(-2), m["c_u"])
    new = _rescale(s["state"] * one + u)
    o = _product(s["q"].unsqueeze(-2), new, m["a_q"].unsqueeze(-2), m["a_s"], m["c_o"].unsqueeze(-2))
    return _rescale(o.squeeze(-2)), new


def _plain_prompt(s):
    _, B, T, H, dv = s["o"].shape
    m = {n: t if n in ("a_s", "c_u") else _chunks(t) for n, t in s["mat"].items()}
    q, k, v = (_chunks(t.transpose(2, 3).flatten(1, 2)) for t in (s["q"], s["k"], s["v"]))
    power = s["decay"].long().repeat(B, 1)                                  # [N, 65]
    chunks, at = q.shape[2], torch.arange(CHUNK, device=DEVICE)
    length = (T - torch.arange(chunks, device=DEVICE) * CHUNK).clamp(max=CHUNK)
    within = power[:, (at[:, None] - at).clamp(min=0)] * (at <= at[:, None])
    left = power[:, (length[:, None] - 1 - at).clamp(min=0)]                # from a token to its chunk's end
    w = _rescale(_rescale(_product(q, k.transpose(-1, -2), m["a_q"], m["a_k"].transpose(-1, -2), m["c_p"])) * within[:, None])
    qd, kd = _rescale(q * power[:, 1:][:, None, :, None]), _rescale(k * left[..., None])
    u = _product(kd.transpose(-1, -2), v, m["a_kd"].transpose(-1, -2), m["a_v"], m["c_u"])
    state = [s["state"].flatten(1, 2)]
    for i in range(chunks):
        state.append(_rescale(state[-1] * power[:, length[i]][:, None, None] + u[:, :, i]))
    o = _product(torch.cat((w, qd), -1), torch.cat((v, torch.stack(state[:-1], 2)), -2), torch.cat((m["a_w"], m["a_qd"]), -1),
                 torch.cat((m["a_v"], m["a_s"]), -2), m["c_o"])
    return _tokens(_rescale(o), T).view(2, B, H, T, dv).transpose(2, 3), state[-1].view_as(s["state"])


# ------------------------------------------------------------------------------------------------ the framework's calls
@functools.lru_cache(None)
def _lane():
    from paper_2209_13643_amd import mpc
    return mpc.Lane(0, single_queue=True)


def _own(s):
    """The calls write into the state's outputs; both shares come back as one tensor, as from the plain form."""
    lane, kind, t = _lane(), s["kind"], s["pair"]
    if kind == "bias":
        lane.position_bias(t["x"], t["table"], s["buckets"], out=t["y"])
        return s["y"]
    if kind == "bias-grad":
        lane.position_bias_grad(t["x"], s["buckets"], s["n"], out=t["grad"], scores_out=t.get("y"))
        return (s["grad"], s["y"]) if "y" in s else s["grad"]
    if kind == "matvec4":
        lane.matvec4(t["x"], s["w"], s["scales"], s["group"], scale_bits=20, out=t["y"])
        return s["y"]
    call = lane.linear_attention_step if kind == "step" else lane.linear_attention
    call(t["q"], t["k"], t["v"], s["decay"], t["mat"], t["state"], out=t["o"], state_out=t["new"])
    return s["o"], s["new"]


def run(state):
    if own:
        return _own(state)
    return {"bias": _plain_bias, "bias-grad": _plain_bias_grad, "matvec4": _plain_matvec4, "step": _plain_step,
            "prompt": _plain_prompt}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
WORD = 8
RING = 2 * 15            # 8-bit products and sums of one multiplication mod 2^64: the bilinear rank of eight digits mod x^8


def work(case):
    kind = case["kind"]
    if kind in ("bias", "bias-grad"):
        B, H, Tq, Tk, n = (case[x] for x in ("B", "H", "Tq", "Tk", "buckets"))
        pairs = B * H * Tq * Tk
        written = kind == "bias" or case["causal"]
        return {"bytes": 2 * WORD * ((1 + written) * pairs + n * H) + 4 * (Tq + Tk - 1), "flops": 2 * pairs}
    if kind == "matvec4":
        M, K, N, group = (case[x] for x in ("M", "K", "N", "group"))
        # a 4-bit integer times eight digits, both parties
        return {"bytes": N * K // 2 + 4 * N * -(-K // group) + 2 * WORD * M * (K + N), "flops": 2 * 16 * M * K * N}
    B, H, dk, dv = (case[x] for x in ("B", "H", "dk", "dv"))
    if kind == "step":
        # state, its mask and the outer product's addend in, the new state out; q, k, v, their masks, o and its addend
        return {"bytes": 2 * WORD * B * H * (4 * dk * dv + 4 * dk + 4 * dv), "flops": B * H * dk * dv * (2 + 3 + 3) * 2}
    T, N, chunks = case["T"], B * H, -(-case["T"] // CHUNK)
    pairs = sum(min(CHUNK, T - c * CHUNK) * (min(CHUNK, T - c * CHUNK) + 1) // 2 for c in range(chunks))
    words = T * (6 * dk + 4 * dv) + 2 * pairs + 2 * (chunks + 1) * dk * dv
    return {"bytes": 2 * WORD * N * words, "flops": RING * 3 * N * (pairs * (dk + dv) + 2 * T * dk * dv)}


# ------------------------------------------------------------------------------------------------ the definitions, word by word
def _np(t):
    return t.cpu().numpy().view(np.uint64) if t.dtype == torch.int64 else t.cpu().numpy()


def _shift(party, z, bits):
    return z >> np.uint64(bits) if party == 0 else -(-z >> np.uint64(bits))


def _sharing(L, R, a, b, c):
    """Party 0 and party 1 of Alg. 1 for z = L R, with a_0 b_0 already taken off c_0."""
    e, f = L[0] - a[0] + L[1] - a[1], R[0] - b[0] + R[1] - b[1]
    return [c[0] + a[0] @ b[0] + e @ b[0] + a[0] @ f + e @ f, c[1] + e @ b[1] + a[1] @ f]


def exact(case, seed):
    kind = case["kind"]
    if kind == "prompt" and case["B"] * case["H"] * case["T"] * (CHUNK * (case["dk"] + case["dv"]) + 2 * case["dk"] * case["dv"]) > 2e9:
        return None
    s = prepare(case, seed)
    s = {n: {m: _np(t) for m, t in v.items()} if n == "mat" else _np(v) if isinstance(v, torch.Tensor) else v for n, v in s.items()}
    if kind in ("bias", "bias-grad"):
        x = s["x"]
        Tq, Tk = x.shape[-2:]
        out, grad = np.zeros_like(x), np.zeros((2, s["n"], x.shape[2]), np.uint64)
        for i in range(Tq):
            bucket = s["buckets"][Tq - 1 - i:Tq - 1 - i + Tk]
            js = np.flatnonzero(bucket >= 0)
            out[..., i, js] = x[..., i, js]
            if kind == "bias":
                out[..., i, js] += s["table"][:, bucket[js]].swapaxes(1, 2)[:, None]
            else:
                np.add.at(grad, (slice(None), bucket[js]), x[..., i, js].sum(1).swapaxes(1, 2))
        out = torch.from_numpy(out.view(np.int64))
        if kind == "bias":
            return out
        grad = torch.from_numpy(grad.view(np.int64))
        return (grad, out) if case["causal"] else grad
    if kind == "matvec4":
        K = s["x"].shape[-1]
        w = np.empty((s["w"].shape[0], 2 * s["w"].shape[1]), np.int64)
        w[:, 0::2], w[:, 1::2] = s["w"] & 15, s["w"] >> 4
        w = np.where(w > 7, w - 16, w)[:, :K] * np.repeat(s["scales"].astype(np.int64), s["group"], 1)[:, :K]
        z = [_shift(p, s["x"][p] @ w.view(np.uint64).T, 20) for p in (0, 1)]
        return torch.from_numpy(np.stack(z).view(np.int64))
    m, H, dk, dv = s["mat"], case["H"], case["dk"], case["dv"]
    power = s["decay"].astype(np.uint64)
    T, C = (1, 1) if kind == "step" else (case["T"], CHUNK)
    o, new = np.empty_like(s["o"]), np.empty_like(s["state"])
    for b in range(case["B"]):
        for h in range(H):
            S = [s["state"][p, b, h] for p in (0, 1)]
            if kind == "step":
                row = lambda n: m[n][:, b, h][:, None]  # noqa: E731
                q, k, v = (s[n][:, b, h][:, None] for n in "qkv")
                u = _sharing(k.swapaxes(1, 2), v, row("a_k").swapaxes(1, 2), row("a_v"), m["c_u"][:, b, h])
                S = [_shift(p, S[p] * power[h, 1] + u[p], FRAC) for p in (0, 1)]
                z = _sharing(q, S, row("a_q"), m["a_s"][:, b, h], row("c_o"))
                o[:, b, h] = [_shift(p, z[p], FRAC)[0] for p in (0, 1)]
            for c in range(0 if kind == "step" else -(-T // C)):
                t = slice(c * C, min(T, c * C + C))
                L, n = t.stop - t.start, b * H + h
                a = {x: m[x][:, n, t] for x in m if x not in ("a_s", "c_u")}
                q, k, v = (s[x][:, b, t, h] for x in "qkv")
                P = _sharing(q, k.swapaxes(1, 2), a["a_q"], a["a_k"].swapaxes(1, 2), a["c_p"][..., :L])
                D = np.array([[power[h, i - j] if i >= j else 0 for j in range(L)] for i in range(L)], np.uint64)
                W = [np.tril(_shift(p, _shift(p, P[p], FRAC) * D, FRAC)) for p in (0, 1)]
                qd = [_shift(p, q[p] * power[h, 1:L + 1, None], FRAC) for p in (0, 1)]
                kd = [_shift(p, k[p] * power[h, L - 1::-1, None], FRAC).T for p in (0, 1)]
                z = _sharing([np.hstack((W[p], qd[p])) for p in (0, 1)], [np.vstack((v[p], S[p])) for p in (0, 1)],
                             [np.hstack((a["a_w"][p][:, :L], a["a_qd"][p])) for p in (0, 1)],
                             [np.vstack((a["a_v"][p], m["a_s"][p, n, c])) for p in (0, 1)], a["c_o"])
                o[:, b, t, h] = [_shift(p, z[p], FRAC) for p in (0, 1)]
                u = _sharing(kd, v, a["a_kd"].swapaxes(1, 2), a["a_v"], m["c_u"][:, n, c])
                S = [_shift(p, S[p] * power[h, L] + u[p], FRAC) for p in (0, 1)]
            new[:, b, h] = S
    return torch.from_numpy(o.view(np.int64)), torch.from_numpy(new.view(np.int64))
