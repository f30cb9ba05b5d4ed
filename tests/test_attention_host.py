"""The attention and public-weight calls on the host: what they refuse, what their helpers compute, and the plain 64-bit forms
against real arithmetic.  No GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import attention_inputs as inputs
import fake_hip
from oracle import attention as plain
from paper_2209_13643_amd import attention

U64 = np.uint64


def real(pair):
    return (pair[0] + pair[1]).view(np.int64).astype(np.float64) / 65536.0


@pytest.mark.parametrize("T,dk,dv", [(1, 3, 5), (64, 8, 4), (70, 5, 9), (130, 4, 4)])
def test_plain_prompt_is_decayed_linear_attention(T, dk, dv):
    """Decoded against float64.  Every trunc is off by less than 2 steps of 2^-16 (floor, plus one from the shares); the
    decay's 16 bits by 2^-17.  O has L P's and dk Qd's terms: with |V|, |S| < 8 and sums of up to 64 + dk terms an error of
    (64 + 9) * 8 * (2 + 2 + 1) * 2^-16 + the states' (3 chunks of 64 terms) stays below 2^-3; a wrong term is of order one."""
    rng = np.random.default_rng(T)
    B, H = 1, 2
    d = inputs.prompt(rng, B, H, T, dk, dv)
    decay = [0.9, 1.0]
    o, new = plain.linear_attention(d["q"], d["k"], d["v"], attention.decay_powers(decay).numpy(), d["mat"], d["state"])
    q, k, v, s0 = (real(d[n]) for n in ("q", "k", "v", "state"))
    for h in range(H):
        S = s0[0, h]
        for t in range(T):
            S = decay[h] * S + np.outer(k[0, t, h], v[0, t, h])
            assert np.abs(q[0, t, h] @ S - real(o)[0, t, h]).max() < 2 ** -7
        assert np.abs(S - real(new)[0, h]).max() < 2 ** -7


def test_plain_step_follows_the_recurrence():
    rng = np.random.default_rng(3)
    d = inputs.one_token(rng, 2, 3, 5, 4)
    powers = attention.decay_powers([0.5, 0.97, 1.0])
    o, new = plain.step(d["q"], d["k"], d["v"], powers.numpy(), d["mat"], d["state"])
    q, k, v, s = (real(d[n]) for n in ("q", "k", "v", "state"))
    want = np.array([0.5, 0.97, 1.0])[None, :, None, None] * s + k[..., :, None] * v[..., None, :]
    assert np.abs(real(new) - want).max() < 2 ** -13 and np.abs(real(o) - (q[..., None] * want).sum(-2)).max() < 2 ** -12


def test_plain_matvec4_is_the_real_product():
    rng = np.random.default_rng(4)
    q, scales = rng.integers(-8, 8, (7, 70)), rng.integers(1, 1 << 17, (7, 3))
    x = inputs.share(rng, inputs.fixed(rng, 1.0, 2, 70))
    w = q * np.repeat(scales, 32, 1)[:, :70] / 2.0 ** 20
    assert np.abs(real(plain.matvec4(x, q, scales, 32, 20)) - real(x) @ w.T).max() < 2 ** -14      # floor, plus one


def test_plain_bias_gradient_is_the_transposed_map():
    """<bias(t), g> = <t, grad(g)> for every table t and gradient g, exactly in the ring."""
    rng = np.random.default_rng(5)
    buckets = np.array([-1, 0, 3, 1, 1, 7, 2, -5, 0, 3, 2], np.int32)
    t, g = inputs.masks(rng, 4, 3), inputs.masks(rng, 2, 3, 5, 7)
    zero = tuple(np.zeros_like(w) for w in g)
    y, (grad, _) = plain.position_bias(zero, t, buckets), plain.position_bias_grad(g, buckets, 4)
    for p in range(2):
        assert (y[p] * g[p]).sum(dtype=U64) == (t[p] * grad[p]).sum(dtype=U64)


# ------------------------------------------------------------------------------------------------ helpers
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Tq,Tk,n,far", [(1, 1, 8, 20), (5, 9, 8, 20), (64, 64, 32, 128), (1, 300, 32, 128), (9, 5, 2, 3)])
def test_relative_buckets(Tq, Tk, n, far, causal):
    at = attention.relative_buckets(Tq, Tk, n, far, causal).tolist()
    assert len(at) == Tq + Tk - 1
    half = n if causal else n // 2
    near = max(half // 2, 1)
    for i in range(Tq):
        for j in range(Tk):
            d, u = j - (i + Tk - Tq), at[j - i + Tq - 1]
            if causal and d > 0:
                assert u == -1
                continue
            if not causal and d > 0:
                assert u >= half
                u -= half
            d = abs(d)
            assert 0 <= u < half
            if d < near:
                assert u == min(d, half - 1)
            elif d >= far:
                assert u == half - 1
            else:
                exact = near + math.log(d / near) / math.log(far / near) * (half - near)
                assert abs(min(exact, half - 1) - u) <= 1 + 1e-9 and u <= exact + 1e-9


def test_helpers_refuse():
    for bad in [(0, 1, 8, 20), (1, 1, 7, 20), (1, 1, 8, 2)]:
        with pytest.raises(ValueError):
            attention.relative_buckets(*bad)
    for bad in [[1.5], [-0.1], [[0.5]]]:
        with pytest.raises(ValueError):
            attention.decay_powers(bad)
    for bad in [torch.tensor([[8]]), torch.tensor([[-9]]), torch.tensor([0]), torch.tensor([[0.5]])]:
        with pytest.raises(ValueError):
            attention.pack_weights4(bad)


def test_packed_weights_and_quantisation():
    q = torch.arange(-8, 8).repeat(3, 3)[:, :37]
    p = attention.pack_weights4(q)
    assert p.shape == (3, 32) and p.dtype == torch.uint8
    for k in range(37):
        half = (int(p[1, k // 2]) >> (4 * (k % 2))) & 15
        assert (half ^ 8) - 8 == int(q[1, k])
    assert int(p[1, 18]) >> 4 == 0 and int(p[:, 19:].max()) == 0
    w = torch.randn(5, 100, generator=torch.Generator().manual_seed(0))
    packed, s = attention.quantize4(w, 32)
    assert s.shape == (5, 4) and packed.shape == (5, 64)
    lo = torch.stack((packed & 15, packed >> 4), -1).flatten(1)[:, :100].int()
    back = ((lo ^ 8) - 8) * s.double().repeat_interleave(32, 1)[:, :100] * 2.0 ** -20
    assert ((back - w).abs() <= s.double().repeat_interleave(32, 1)[:, :100] * 2.0 ** -20 * (0.5 + 1e-3)).all()


def test_decay_powers():
    t = attention.decay_powers([1.0, 0.0, 0.5])
    assert t.shape == (3, 65) and t[0].eq(65536).all() and t[1].tolist() == [65536] + [0] * 64 and t[2, 3] == 8192


# ------------------------------------------------------------------------------------------------ refusals of the C calls
REFUSALS = r'''
class Strides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]
class Operands(ctypes.Structure):
    _fields_ = [("q", Share), ("k", Share), ("v", Share), ("sq", Strides), ("sk", Strides), ("sv", Strides), ("decay", c_void_p), ("state", Share), ("o", Share),
                ("so", Strides), ("state_out", Share)]
class Material(ctypes.Structure):
    _fields_ = [("s", Share * 10)]
class StepMaterial(ctypes.Structure):
    _fields_ = [("s", Share * 6)]
for n in ("mpc_linear_attention_workspace_bytes", "mpc_linear_attention_step_workspace_bytes"):
    getattr(lib, n).restype = c_size_t
P = c_void_p
lib.mpc_position_bias.argtypes = [P, Share, Share, P, Share] + [c_int] * 5
lib.mpc_position_bias_grad.argtypes = [P, Share, P, Share, Share] + [c_int] * 5
lib.mpc_matvec4_workspace_bytes.restype = lib.mpc_position_bias_grad_workspace_bytes.restype = c_size_t
lib.mpc_matvec4.argtypes = [P, Share, P, P, Share] + [c_int] * 5
lib.mpc_linear_attention.argtypes = [P, P, P] + [c_int] * 5
lib.mpc_linear_attention_step.argtypes = [P, P, P] + [c_int] * 4
def share(nbytes): return Share((c_void_p * 2)(array(nbytes), array(nbytes)))
none, half = Share(), Share((c_void_p * 2)(array(64), None))
big = 1 << 24

def bias(x=None, t=None, m=None, o=None, B=2, H=3, Tq=8, Tk=8, n=4, c=None):
    x, t, o = x or share(big), t or share(big), o or share(big)
    return lib.mpc_position_bias(c if c is not None else ctx, x, t, array(big) if m is None else m or None, o, B, H, Tq, Tk, n)
x = share(big)
shifted = Share((c_void_p * 2)(x.p[0] + 8, x.p[1] + 8)); crossed = Share((c_void_p * 2)(x.p[1], x.p[0]))
same = Share((c_void_p * 2)(x.p[0], x.p[0]))
result["bias"] = [bias(), bias(x=x, o=x), bias(x=none), bias(t=half), bias(o=none), bias(m=0), bias(B=0), bias(H=-1), bias(Tq=0), bias(Tk=0), bias(n=0),
                  bias(n=4097), bias(Tq=1 << 30, Tk=(1 << 30) + 2), bias(x=x, o=shifted), bias(x=x, o=crossed), bias(x=x, o=same), bias(t=x, o=x)]
def grad(g=None, m=None, t=None, s=None, B=2, H=3, Tq=8, Tk=8, n=4):
    return lib.mpc_position_bias_grad(ctx, g or share(big), array(big) if m is None else m or None, t or share(big), s or none, B, H, Tq, Tk, n)
lib.mpc_ctx_set_workspace(ctx, array(big), big)
result["grad"] = [grad(), grad(g=x, s=x), grad(g=none), grad(t=none), grad(s=half), grad(m=0), grad(B=0), grad(n=5000), grad(g=x, s=shifted), grad(g=x, t=x), grad(s=x, t=x)]
def mv(x=None, w=None, s=None, z=None, M=2, K=100, N=5, group=32, bits=16):
    return lib.mpc_matvec4(ctx, x or share(big), array(big) if w is None else w or None, array(big) if s is None else s or None, z or share(big), M, K, N, group, bits)
result["matvec4"] = [mv(), mv(group=64), mv(group=128), mv(group=384), mv(bits=0), mv(bits=31), mv(x=none), mv(z=half), mv(w=0), mv(s=0), mv(M=0), mv(K=0), mv(N=0),
                     mv(group=0), mv(group=16), mv(group=96), mv(group=192), mv(bits=-1), mv(bits=32), mv(w=array(64) + 8), mv(s=array(64) + 2), mv(M=65536),
                     mv(K=(1 << 22) + 1), mv(x=x, z=x), mv(w=x.p[0], z=x), mv(s=x.p[1], z=x)]
B, T, H, dk, dv = 2, 70, 3, 8, 6
nat = lambda T, d: Strides(T * H * d, H * d, d)
def prompt(q=None, sq=None, so=None, m=None, state=None, o=None, out=None, decay=None, ws=True, B=B, T=T, H=H, dk=dk, dv=dv, drop=None):
    need = lib.mpc_linear_attention_workspace_bytes(B, T, H, dk, dv)
    lib.mpc_ctx_set_workspace(ctx, array(max(need, 1)), need - (0 if ws else 1) if need else 0)
    mat = Material((Share * 10)(*[none if i == drop else share(big) for i in range(10)]))
    x = Operands(q or share(big), share(big), share(big), sq or nat(T, dk), nat(T, dk), nat(T, dv), array(big) if decay is None else decay or None,
                 share(big) if state is None else state, o or share(big), so or nat(T, dv), share(big) if out is None else out)
    return lib.mpc_linear_attention(ctx, ctypes.byref(x), ctypes.byref(mat) if m is None else None, B, T, H, dk, dv)
result["prompt"] = [prompt(), prompt(state=none), prompt(out=none), prompt(state=x, out=x), prompt(sq=Strides(0, 0, 0)), prompt(T=1), prompt(dk=128, dv=128),
                    prompt(q=none), prompt(m=0), prompt(decay=0), prompt(state=half), prompt(out=half), prompt(o=none), prompt(B=0), prompt(T=0), prompt(H=0), prompt(dk=0),
                    prompt(dv=0), prompt(dk=129), prompt(dv=200), prompt(ws=False), prompt(sq=Strides(-1, 8, 8)), prompt(so=Strides(0, 18, 6)), prompt(so=Strides(1260, 18, 5)),
                    prompt(so=Strides(1259, 18, 6)), prompt(q=x, o=x), prompt(q=x, out=x), prompt(state=x, o=x), prompt(o=x, out=x), prompt(state=x, out=shifted),
                    prompt(B=1 << 20, H=1 << 12)]
need = lib.mpc_position_bias_grad_workspace_bytes(2, 3, 8, 8, 4)
lib.mpc_ctx_set_workspace(ctx, array(need), need - 1)
result["grad without room"] = grad()
lib.mpc_ctx_set_workspace(ctx, array(need), need)
result["grad with room"] = grad()
lib.mpc_ctx_set_workspace(ctx, array(4096), 4096)
result["matvec4 without room"] = [mv(M=16, K=4096, N=4096), mv(M=16, K=4096, N=100)]
result["drops"] = [prompt(drop=i) for i in range(10)]
def step(q=None, so=None, state=None, o=None, out=None, ws=True, B=B, H=H, dk=dk, dv=dv, drop=None):
    need = lib.mpc_linear_attention_step_workspace_bytes(B, H, dk, dv)
    lib.mpc_ctx_set_workspace(ctx, array(max(need, 1)), need - (0 if ws else 1) if need else 0)
    mat = StepMaterial((Share * 6)(*[none if i == drop else share(big) for i in range(6)]))
    n = lambda d: Strides(H * d, -7, d)                     # the token's stride is not used
    x = Operands(q or share(big), share(big), share(big), n(dk), n(dk), n(dv), array(big), share(big) if state is None else state, o or share(big), so or n(dv),
                 share(big) if out is None else out)
    return lib.mpc_linear_attention_step(ctx, ctypes.byref(x), ctypes.byref(mat), B, H, dk, dv)
result["step"] = [step(), step(state=x, out=x), step(B=1, H=1, dk=1, dv=1), step(dk=128, dv=128),
                  step(q=none), step(state=none), step(out=none), step(o=none), step(B=0), step(dk=129), step(ws=False), step(so=Strides(0, 0, 6)), step(q=x, o=x),
                  step(state=x, o=x), step(state=x, out=shifted), step(o=x, out=x)]
result["step_drops"] = [step(drop=i) for i in range(6)]
fine = c_void_p()
assert lib.mpc_ctx_create_single_queue(ctypes.byref(fine), 0, 31) == 0
old, ctx = ctx, fine
result["frac"] = [prompt(), step()]
ctx = old
launches()
result["null"] = [lib.mpc_linear_attention(ctx, None, ctypes.byref(Material()), 1, 1, 1, 1, 1), lib.mpc_linear_attention_step(ctx, None, ctypes.byref(StepMaterial()), 1, 1, 1, 1), lib.mpc_position_bias(None, x, x, array(8), share(8), 1, 1, 1, 1, 1), lib.mpc_matvec4(None, x, array(8), array(8), share(8), 1, 1, 1, 32, 1)]
bias(n=0); grad(g=none); mv(K=0); prompt(T=0); step(dk=129)
result["launched by refused calls"] = launches()
'''


def test_refusals(tmp_path):
    r = fake_hip.run(tmp_path, REFUSALS)
    E, M, R = -1, -2, -4
    assert r["bias"] == [0, 0] + [E] * 9 + [R, R] + [E] * 4
    assert r["grad"] == [0, 0] + [E] * 5 + [R] + [E] * 3
    assert r["matvec4"] == [0] * 6 + [E] * 15 + [R, R] + [E] * 3
    assert r["prompt"] == [0] * 7 + [E] * 11 + [R, R, M] + [E] * 9 + [R]
    assert r["grad without room"] == M and r["grad with room"] == 0
    assert r["matvec4 without room"] == [M, 0]
    assert r["drops"] == [E] * 10 and r["step_drops"] == [E] * 6
    assert r["step"] == [0] * 4 + [E] * 5 + [R, M] + [E] * 5
    assert r["frac"] == [R, R] and r["null"] == [E, E, E, E] and r["launched by refused calls"] == []


SIZES_AND_OVERLAPS = r'''
result["bias"] = [bias(B=1 << 24, H=1, Tq=1, Tk=1), bias(B=1, H=1, Tq=1, Tk=(1 << 31) - 1), bias(o=x, m=x.p[0]), bias(o=x, m=x.p[1] + 16)]
result["grad"] = [grad(B=1, H=1, Tq=1, Tk=(1 << 31) - 2), grad(H=1 << 14, n=4096), grad(B=1, H=1 << 25, Tq=1, Tk=1, n=1), grad(t=x, m=x.p[1]), grad(s=x, m=x.p[0])]
result["matvec4"] = [mv(M=1, K=1, N=(1 << 25) + 1), mv(M=1, K=1, N=(1 << 31) - 1)]
result["prompt"] = [prompt(B=1, H=1 << 26, T=1, dk=1, dv=1), prompt(B=1, H=1, T=(1 << 31) - 1), prompt(o=x, decay=x.p[0]), prompt(out=x, decay=x.p[1])]
result["step"] = [step(B=1, H=1 << 26, dk=1, dv=1)]
result["queries"] = [lib.mpc_linear_attention_workspace_bytes(1 << 15, (1 << 31) - 100, 1 << 15, 128, 128), lib.mpc_matvec4_workspace_bytes(8, 64, (1 << 31) - 1)]
result["refused calls launched"] = launches()
'''


def test_sizes_beyond_a_launch_and_outputs_on_public_arrays(tmp_path):
    r = fake_hip.run(tmp_path, REFUSALS + "lib.mpc_ctx_set_workspace(ctx, array(big), big); launches()\n" + SIZES_AND_OVERLAPS)
    E, R = -1, -4
    assert r["bias"] == [R, R, E, E] and r["grad"] == [R, R, R, E, E] and r["matvec4"] == [R, R]
    assert r["prompt"] == [R, R, E, E] and r["step"] == [R]
    assert r["queries"] == [0, 0] and r["refused calls launched"] == []


def test_helpers_refuse_what_is_not_finite():
    for bad in [[float("nan")], [0.5, float("inf")]]:
        with pytest.raises(ValueError):
            attention.decay_powers(bad)
    with pytest.raises(ValueError):
        attention.decay_powers([0.5], 31)
    for bad in [float("nan"), float("inf"), -1e6]:
        with pytest.raises(ValueError):
            attention.quantize4(torch.tensor([[0.5, bad]]), 32)
    with pytest.raises(ValueError):
        attention.quantize4(torch.ones(2, 2), 0)


def test_workspace_queries_refuse():
    from paper_2209_13643_amd import mpc
    L = mpc.lib()
    assert L.mpc_linear_attention_workspace_bytes(1, 0, 1, 8, 8) == 0 and L.mpc_linear_attention_workspace_bytes(1, 1, 1, 129, 8) == 0
    assert L.mpc_matvec4_workspace_bytes(0, 1 << 14, 1 << 14) == 0 and L.mpc_matvec4_workspace_bytes(1, 1 << 14, 1 << 14) == 0
    assert L.mpc_matvec4_workspace_bytes(16, 4100, 4096) == 16 * 17 * 4096
    assert L.mpc_linear_attention_step_workspace_bytes(0, 1, 8, 8) == 0 and L.mpc_linear_attention_step_workspace_bytes(1, 1, 8, 8) > 0
    assert L.mpc_linear_attention_workspace_bytes(1, 65, 1, 8, 8) > L.mpc_linear_attention_workspace_bytes(1, 64, 1, 8, 8) > 0
