"""Attention layers on shares: host helpers of the attention calls (bucket maps, decay tables, 4-bit weights), the scores
form with a learned position bias and its backward pass, and a layer that serves prompts and single tokens through linear
attention with public 4-bit projections.  Every protocol step runs in the library; this module orders its calls."""
from __future__ import annotations

import dataclasses

import torch

from . import mpc


# ------------------------------------------------------------------------------------------------ host helpers
def relative_buckets(Tq: int, Tk: int, n_buckets: int, max_distance: int, causal: bool = False) -> torch.Tensor:
    """Bucket of every relative position, int32 [Tq + Tk - 1], entry j - i + Tq - 1 of query i and key j; the last query
    stands at the last key.  Causal: keys behind a query are masked (-1) and all buckets serve the distances before it; else
    half of the buckets serve each side.  The nearer half of a side's distances have a bucket each, the others share by the
    logarithm of their distance up to max_distance, all beyond it share the last.  Exact: bucket near + m starts at the first
    distance d with (d / near)^(n - near) >= (max_distance / near)^m, compared in whole numbers."""
    if min(Tq, Tk, n_buckets) <= 0:
        raise ValueError("Tq, Tk and n_buckets have to be positive")
    if not causal and n_buckets % 2:
        raise ValueError("both directions take half of the buckets each: an even number expected")
    n = n_buckets if causal else n_buckets // 2
    near = max(n // 2, 1)
    if max_distance <= near:
        raise ValueError(f"max_distance has to be beyond the {near} distances that have a bucket each")
    top = Tq + Tk
    side, m = [], 0                                  # bucket of distance 0, 1, ...
    for d in range(min(top, max_distance + 1)):
        if d < near:
            side.append(min(d, n - 1))
            continue
        while m + 1 < n - near and d ** (n - near) * near ** (m + 1) >= max_distance ** (m + 1) * near ** (n - near):
            m += 1
        side.append(min(near + m, n - 1))
    side = torch.tensor(side, dtype=torch.int32)
    rel = torch.arange(Tq + Tk - 1) - (Tk - 1)       # j - i with the last query at the last key
    at = side[rel.abs().clamp(max=len(side) - 1)]
    return torch.where(rel > 0, torch.full_like(at, -1) if causal else at + n, at)


def decay_powers(decay, frac_bits: int = 16) -> torch.Tensor:
    """Powers 0..64 of every head's decay in [0, 1] as fixed point, int32 [H, 65], on the device of a tensor; formed on the host,
    where all devices' tables are the same."""
    given = torch.as_tensor(decay, dtype=torch.float64)
    d = given.cpu()
    if d.ndim != 1 or not bool(((d >= 0) & (d <= 1)).all()):
        raise ValueError("one decay in [0, 1] for each head expected")
    if not 0 <= frac_bits <= 30:
        raise ValueError("frac_bits in [0, 30] expected: a decay of one has to fit 31 bits")
    return torch.round(d[:, None] ** torch.arange(mpc.ATTENTION_CHUNK + 1) * 2.0 ** frac_bits).to(torch.int32).to(given.device)


def pack_weights4(q: torch.Tensor) -> torch.Tensor:
    """Integers [N, K] in [-8, 7] as uint8 [N, 16 ceil(K / 32)]: an even column in a byte's low half, the odd one after it in
    its high half, zeros behind column K."""
    if q.ndim != 2 or q.is_floating_point() or int(q.min()) < -8 or int(q.max()) > 7:
        raise ValueError("integers in [-8, 7] of shape [N, K] expected")
    q = torch.nn.functional.pad(q.to(torch.int16), (0, -q.shape[1] % 32)) & 15
    return (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8).contiguous()


def quantize4(w: torch.Tensor, group: int, scale_bits: int = 20):
    """Nearest 4-bit form of real weights [N, K]: (packed weights, int32 scales [N, ceil(K / group)]); a group's scale is its
    largest magnitude over 7.  The product takes the same scale_bits (Lane.matvec4's own default is 16)."""
    N, K = w.shape
    if group <= 0 or not bool((w.abs().double() * 2.0 ** scale_bits / 7 < 2 ** 31 - 1).all()):
        raise ValueError("a positive group and finite weights whose scales fit 31 bits expected")
    g = torch.nn.functional.pad(w.double(), (0, -K % group)).view(N, -1, group)
    scales = torch.round(g.abs().amax(-1) / 7 * 2.0 ** scale_bits).clamp(min=1, max=2 ** 31 - 1)
    q = torch.round(g / (scales[..., None] * 2.0 ** -scale_bits)).clamp(-8, 7).view(N, -1)[:, :K]
    return pack_weights4(q.to(torch.int16)), scales.to(torch.int32).contiguous()


# ------------------------------------------------------------------------------------------------ scores form, with training
def scores_forward(lane: "mpc.Lane", q, k, v, table, buckets, t_qk, t_av):
    """O = (Q K^T + bias) V per head, q, k, v [B, H, T, d] sharings; t_qk, t_av = (a, b, c) triples of the two products over
    B*H matrices (b of t_qk masks K as it is stored, [B*H, Tk, d]).  Returns (o [B, H, Tq, dv], biased scores for backward)."""
    B, H, Tq, d = q[0].shape
    flat = lambda s: tuple(t.view((-1,) + tuple(t.shape[-2:])) for t in s)
    scores = lane.beaver_matmul(flat(q), flat(k), *t_qk, flags=mpc.MPC_TRUNCATE | mpc.MPC_TRANS_Y)
    scores = tuple(t.view(B, H, Tq, -1) for t in scores)
    lane.position_bias(scores, table, buckets, out=scores)
    o = lane.beaver_matmul(flat(scores), flat(v), *t_av)
    return tuple(t.view(B, H, Tq, -1) for t in o), scores


def scores_backward(lane: "mpc.Lane", go, q, k, v, scores, buckets, n_buckets, t_gs, t_gv, t_gq, t_gk):
    """Gradients (q, k, v, table) of scores_forward for its output's gradient go; one triple for each of the four products
    gO V^T, A^T gO, gS K and gS^T Q, masks stored as their operands are."""
    B, H = go[0].shape[:2]
    flat = lambda s: tuple(t.view((-1,) + tuple(t.shape[-2:])) for t in s)
    heads = lambda s: tuple(t.view((B, H) + tuple(t.shape[-2:])) for t in s)
    T = mpc.MPC_TRUNCATE
    gv = lane.beaver_matmul(flat(scores), flat(go), *t_gv, flags=T | mpc.MPC_TRANS_X)
    gs = heads(lane.beaver_matmul(flat(go), flat(v), *t_gs, flags=T | mpc.MPC_TRANS_Y))
    table, gs = lane.position_bias_grad(gs, buckets, n_buckets, scores_out=gs)
    gq = lane.beaver_matmul(flat(gs), flat(k), *t_gq)
    gk = lane.beaver_matmul(flat(gs), flat(q), *t_gk, flags=T | mpc.MPC_TRANS_X)
    return heads(gq), heads(gk), heads(gv), table


# ------------------------------------------------------------------------------------------------ prompts and single tokens
_ROWS = 16384                     # of a projection at a time


@dataclasses.dataclass
class TokenLayer:
    """Attention layer with public 4-bit projections: x -> [q | k | v] -> linear attention -> out projection.  Results are new
    tensors: a graph is recorded of the lane's calls with out arguments instead."""
    heads: int
    dk: int
    dv: int
    w_qkv: torch.Tensor            # [heads (2 dk + dv)] rows: q of all heads, k of all heads, v of all heads
    s_qkv: torch.Tensor
    w_out: torch.Tensor            # rows of heads * dv columns
    s_out: torch.Tensor
    group: int
    decay: torch.Tensor            # [heads, 65]
    scale_bits: int = 20

    def _product(self, lane, x, w, scales):
        """x [M, K] by one projection, in blocks of rows: the call takes 65535, and its workspace has up to 4 KB for each row and
        256 columns."""
        M = x[0].shape[0]
        if M <= _ROWS:
            return lane.matvec4(x, w, scales, self.group, self.scale_bits)
        out = tuple(torch.empty((M, w.shape[0]), dtype=torch.int64, device=x[0].device) for _ in range(2))
        for r in range(0, M, _ROWS):
            rows = lambda s: tuple(t[r:r + _ROWS] for t in s)
            lane.matvec4(rows(x), w, scales, self.group, self.scale_bits, out=rows(out))
        return out

    def _project(self, lane, x, shape):
        """x [M, width] -> q, k, v as views [*shape, heads, d] of one product"""
        qkv = self._product(lane, x, self.w_qkv, self.s_qkv)
        nk = self.heads * self.dk
        part = lambda a, b, d: tuple(t[:, a:b].unflatten(0, shape).unflatten(-1, (self.heads, d)) for t in qkv)
        return part(0, nk, self.dk), part(nk, 2 * nk, self.dk), part(2 * nk, 2 * nk + self.heads * self.dv, self.dv)

    def _out(self, lane, o, rows):
        return self._product(lane, tuple(t.view(rows, -1) for t in o), self.w_out, self.s_out)

    def prompt(self, lane: "mpc.Lane", x, mat, state=None):
        """x [B, T, width] sharing -> (y [B, T, rows of w_out], state after the last token)"""
        B, T, _ = x[0].shape
        q, k, v = self._project(lane, tuple(t.view(B * T, -1) for t in x), (B, T))
        o, state = lane.linear_attention(q, k, v, self.decay, mat, state)
        return tuple(t.view(B, T, -1) for t in self._out(lane, o, B * T)), state

    def token(self, lane: "mpc.Lane", x, mat, state):
        """x [B, width] sharing, one token of every sequence -> y [B, rows of w_out]; state is brought up to date in place"""
        B = x[0].shape[0]
        q, k, v = self._project(lane, x, (B,))
        o, _ = lane.linear_attention_step(q, k, v, self.decay, mat, state, state_out=state)
        return self._out(lane, o, B)
