"""The attention and public-weight calls against their plain 64-bit forms, every share of both parties, bit for bit."""
import numpy as np
import pytest
import torch

import attention_inputs as inputs
from oracle import attention as plain

pytestmark = pytest.mark.gpu
U64 = np.uint64


@pytest.fixture(scope="module")
def mpc():
    from paper_2209_13643_amd import mpc as m
    return m


@pytest.fixture(scope="module")
def attention():
    from paper_2209_13643_amd import attention as a
    return a


@pytest.fixture(scope="module")
def lane(mpc):
    ln = mpc.Lane(0, single_queue=True)
    yield ln
    ln.close()


def dev(mpc, pair):
    return tuple(mpc.to_device(s) for s in pair)


def dev_all(mpc, d):
    return {n: dev(mpc, s) for n, s in d.items()}


def equal(mpc, got, want, what=""):
    for p in range(2):
        h = mpc.to_host(got[p].contiguous())
        assert h.shape == want[p].shape, what
        bad = np.flatnonzero((h != want[p]).ravel())
        assert bad.size == 0, f"{what} party {p}: {bad.size} of {h.size} words differ, first at {np.unravel_index(bad[0], h.shape)}"


def filled(shape, value=-0x5A5A5A5A5A5A5A5A):
    pair = tuple(torch.full(shape, value, dtype=torch.int64, device="cuda:0") for _ in range(2))
    torch.cuda.synchronize()                                 # torch's stream is not the lane's
    return pair


# ------------------------------------------------------------------------------------------------ position bias
BIAS = [(1, 1, 1, 1), (2, 3, 1, 9), (1, 2, 5, 1), (2, 2, 7, 13), (1, 1, 64, 64), (2, 1, 33, 130), (1, 2, 3, 1025), (1, 1, 2, 2051),
        (1, 1, 600, 2), (1, 1, 530, 16), (1, 1, 521, 17), (3, 1, 40, 255)]


def bias_map(rng, kind, Tq, Tk, n, attention):
    if kind == "buckets":
        return attention.relative_buckets(Tq, Tk, n, 20 + n, causal=False).numpy()
    if kind == "causal":
        return attention.relative_buckets(Tq, Tk, n, 20 + n, causal=True).numpy()
    if kind == "all masked":
        return np.full(Tq + Tk - 1, -1, np.int32)
    return rng.integers(-3, n + 3, Tq + Tk - 1).astype(np.int32)          # "any": entries outside [0, n) mask


@pytest.mark.parametrize("kind", ["buckets", "causal", "any", "all masked"])
@pytest.mark.parametrize("B,H,Tq,Tk", BIAS)
def test_position_bias_and_gradient(mpc, lane, attention, B, H, Tq, Tk, kind):
    print(f"bias {B}x{H}x{Tq}x{Tk} {kind}", flush=True)
    rng = np.random.default_rng(B * Tq + Tk)
    n = 8
    m = bias_map(rng, kind, Tq, Tk, n, attention)
    x, t = inputs.masks(rng, B, H, Tq, Tk), inputs.masks(rng, n, H)
    xd, md = dev(mpc, x), mpc.to_device(m)
    out, grad, scores = filled((B, H, Tq, Tk)), filled((n, H)), filled((B, H, Tq, Tk))
    assert lane.position_bias(xd, dev(mpc, t), md, out=out) is out
    lane.position_bias_grad(xd, md, n, out=grad, scores_out=scores)
    alone, none = lane.position_bias_grad(xd, md, n)
    lane.sync()
    assert none is None
    equal(mpc, out, plain.position_bias(x, t, m), "bias")
    wg, ws = plain.position_bias_grad(x, m, n)
    equal(mpc, grad, wg, "table gradient"); equal(mpc, alone, wg, "table gradient alone"); equal(mpc, scores, ws, "scores gradient")
    # in place
    lane.position_bias(xd, dev(mpc, t), md, out=xd)
    again = dev(mpc, x)
    lane.position_bias_grad(again, md, n, out=grad, scores_out=again)
    lane.sync()
    equal(mpc, xd, plain.position_bias(x, t, m), "bias in place"); equal(mpc, again, ws, "scores in place"); equal(mpc, grad, wg, "gradient in place")


def test_position_bias_many_buckets_and_heads(mpc, lane):
    rng = np.random.default_rng(0)
    B, H, Tq, Tk, n = 2, 5, 31, 67, 4096
    m = rng.permutation(4096)[:Tq + Tk - 1].astype(np.int32); m[0] = 4095; m[1] = 4096
    x, t = inputs.masks(rng, B, H, Tq, Tk), inputs.masks(rng, n, H)
    out, (grad, _) = lane.position_bias(dev(mpc, x), dev(mpc, t), mpc.to_device(m)), lane.position_bias_grad(dev(mpc, x), mpc.to_device(m), n)
    lane.sync()
    equal(mpc, out, plain.position_bias(x, t, m)); equal(mpc, grad, plain.position_bias_grad(x, m, n)[0])


def test_position_bias_on_words_that_are_not_16_byte_aligned(mpc, lane):
    rng = np.random.default_rng(1)
    B, H, Tq, Tk, n = 1, 2, 9, 32, 4
    m = rng.integers(-1, n, Tq + Tk - 1).astype(np.int32)
    x, t = inputs.masks(rng, B, H, Tq, Tk), inputs.masks(rng, n, H)
    size = B * H * Tq * Tk
    buf = tuple(torch.empty(size + 1, dtype=torch.int64, device="cuda:0") for _ in range(2))
    at = tuple(b[1:].view(B, H, Tq, Tk) for b in buf)
    for a, w in zip(at, x):
        a.copy_(mpc.to_device(w))
    torch.cuda.synchronize()
    lane.position_bias(at, dev(mpc, t), mpc.to_device(m), out=at)
    lane.sync()
    equal(mpc, at, plain.position_bias(x, t, m))


def test_position_bias_large(mpc, lane, attention):
    """96 heads of 512 x 512 (as int64 tensors: the same sums mod 2^64)."""
    B, H, T, n = 8, 12, 512, 32
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = tuple(torch.randint(-2 ** 63, 2 ** 63 - 1, (B, H, T, T), generator=g, device="cuda:0") for _ in range(2))
    t = tuple(torch.randint(-2 ** 63, 2 ** 63 - 1, (n, H), generator=g, device="cuda:0") for _ in range(2))
    for causal in (False, True):
        m = attention.relative_buckets(T, T, n, 128, causal).cuda()
        torch.cuda.synchronize()
        y = lane.position_bias(x, t, m)
        grad, gs = lane.position_bias_grad(x, m, n, scores_out=filled((B, H, T, T)))
        lane.sync()
        at = m.long()[torch.arange(T, device="cuda:0") - torch.arange(T, device="cuda:0")[:, None] + T - 1]
        kept = at >= 0
        for p in range(2):
            assert torch.equal(y[p], (x[p] + t[p][at.clamp(min=0)].permute(2, 0, 1)) * kept)
            assert torch.equal(gs[p], x[p] * kept)
            want = torch.zeros(n, H, dtype=torch.int64, device="cuda:0")
            want.index_add_(0, at.clamp(min=0).flatten(), (x[p] * kept).sum(0).flatten(1).t().contiguous())
            assert torch.equal(grad[p], want)


def test_position_bias_beyond_32_bit_offsets(mpc, lane, attention):
    """Shares of more than 2^32 bytes each, compared at the ends and across the border; the gradient as sums of int64 tensors."""
    B, H, T, n = 2, 48, 2400, 8
    g = torch.Generator(device="cuda:0").manual_seed(2)
    x = tuple(torch.randint(-2 ** 63, 2 ** 63 - 1, (B, H, T, T), generator=g, device="cuda:0") for _ in range(2))
    t = tuple(torch.randint(-2 ** 63, 2 ** 63 - 1, (n, H), generator=g, device="cuda:0") for _ in range(2))
    assert x[0].numel() * 8 > 2 ** 32
    m = attention.relative_buckets(T, T, n, 40, True).cuda()
    torch.cuda.synchronize()
    y = lane.position_bias(x, t, m)
    grad, _ = lane.position_bias_grad(x, m, n)
    lane.sync()
    at = m.long()[torch.arange(T, device="cuda:0") - torch.arange(T, device="cuda:0")[:, None] + T - 1]
    kept = at >= 0
    for p in range(2):
        for b, h in ((0, 0), (1, 44), (1, 45), (1, 46), (1, 47)):
            assert torch.equal(y[p][b, h], (x[p][b, h] + t[p][at.clamp(min=0), h]) * kept)
            want = torch.zeros(n, dtype=torch.int64, device="cuda:0")
            want.index_add_(0, at.clamp(min=0).flatten(), ((x[p][0, h] + x[p][1, h]) * kept).flatten())
            assert torch.equal(grad[p][:, h], want)


@pytest.mark.parametrize("B,H,T,n,causal", [(1, 2, 1175, 32, True), (1, 1, 6000, 300, False), (2, 3, 1100, 257, True), (5, 2, 1030, 7, False)])
def test_position_bias_shared_out(mpc, lane, attention, B, H, T, n, causal):
    """Several shares of the diagonals, several items to a workgroup: table and scores against sums of int64 tensors."""
    g = torch.Generator(device="cuda:0").manual_seed(T)
    x = tuple(torch.randint(-2 ** 63, 2 ** 63 - 1, (B, H, T, T), generator=g, device="cuda:0") for _ in range(2))
    t = tuple(torch.randint(-2 ** 63, 2 ** 63 - 1, (n, H), generator=g, device="cuda:0") for _ in range(2))
    m = torch.randint(-1, n, (2 * T - 1,), generator=g, device="cuda:0", dtype=torch.int32)
    if causal:
        m[T:] = -1                                           # entry j - i + T - 1
    torch.cuda.synchronize()
    y, gx = lane.position_bias(x, t, m), tuple(torch.empty_like(w) for w in x)
    only, _ = lane.position_bias_grad(x, m, n)
    both, _ = lane.position_bias_grad(x, m, n, scores_out=gx)
    lane.sync()
    i = torch.arange(T, device="cuda:0")
    at = m.long()[i - i[:, None] + T - 1]
    kept, at = at >= 0, at.clamp(min=0)
    for p in range(2):
        assert torch.equal(gx[p], x[p] * kept)
        for h in range(H):
            assert torch.equal(y[p][:, h], (x[p][:, h] + t[p][at, h]) * kept)
            want = torch.zeros(n, dtype=torch.int64, device="cuda:0")
            want.index_add_(0, at.flatten(), (x[p][:, h].sum(0) * kept).flatten())
            assert torch.equal(only[p][:, h], want) and torch.equal(both[p][:, h], want)


# ------------------------------------------------------------------------------------------------ 4-bit weights
@pytest.mark.parametrize("M,K,N,group", [(1, 1, 1, 32), (1, 32, 16, 32), (2, 33, 5, 32), (1, 64, 17, 64), (3, 100, 40, 64), (1, 127, 15, 128), (4, 129, 33, 128),
                                         (1, 700, 64, 128), (5, 1000, 50, 32), (8, 513, 31, 64), (9, 300, 20, 256), (17, 96, 70, 32), (1, 2500, 130, 32),
                                         (2, 5000, 3, 128), (1, 40, 9, 4096), (33, 256, 16, 128), (1, 4100, 257, 64)])
@pytest.mark.parametrize("bits", [16, 0])
def test_matvec4(mpc, lane, attention, M, K, N, group, bits):
    print(f"matvec4 {M}x{K}x{N} group {group}", flush=True)
    rng = np.random.default_rng(M * K + N)
    q = rng.integers(-8, 8, (N, K))
    scales = rng.integers(-(1 << 31), 1 << 31, (N, -(-K // group))).astype(np.int32)     # the whole range
    x = inputs.masks(rng, M, K)
    w = attention.pack_weights4(torch.from_numpy(q))
    if K % 32:                                               # what lies behind the last column is not used
        w[:, (K + 1) // 2:] = 0xA7
        if K % 2:
            w[:, K // 2] |= 0x90
    z = filled((M, N))
    lane.matvec4(dev(mpc, x), w.cuda(), mpc.to_device(scales), group, bits, out=z)
    lane.sync()
    equal(mpc, z, plain.matvec4(x, q, scales, group, bits))


@pytest.mark.parametrize("M,K,N,group", [(9, 4100, 3700, 32), (8, 4097, 4100, 64), (17, 2050, 3900, 128), (5, 10241, 2630, 1024)])
def test_matvec4_many_rows(mpc, lane, attention, M, K, N, group):
    """Products whose digits are made once for all workgroups, on a workspace of exactly the size of the query."""
    print(f"matvec4 {M}x{K}x{N} group {group}", flush=True)
    rng = np.random.default_rng(M)
    q, scales, x = rng.integers(-8, 8, (N, K)), rng.integers(-(1 << 31), 1 << 31, (N, -(-K // group))).astype(np.int32), inputs.masks(rng, M, K)
    need = mpc.lib().mpc_matvec4_workspace_bytes(M, K, N)
    assert need > 0
    from test_gpu_workspace_bounds import Guarded
    g = Guarded(mpc, need)
    g.lane._ws_bytes = need                                  # what the library was told: not to be grown
    z = g.lane.matvec4(dev(mpc, x), attention.pack_weights4(torch.from_numpy(q)).cuda(), mpc.to_device(scales), group, 20)
    g.check()
    equal(mpc, z, plain.matvec4(x, q, scales, group, 20))


@pytest.mark.parametrize("M,K,N,group", [(1, 25088, 10, 32), (1, 16417, 100, 64), (2, 9000, 33, 128), (3, 8197, 40, 64), (9, 8200, 17, 256), (16, 25088, 400, 128)])
def test_matvec4_columns_split_over_workgroups(mpc, attention, M, K, N, group):
    """Long rows of few weights: the sums of several workgroups are joined, in a workspace of exactly the queried size."""
    from test_gpu_workspace_bounds import Guarded
    rng = np.random.default_rng(K + N)
    need = mpc.lib().mpc_matvec4_workspace_bytes(M, K, N)
    assert need >= 2 * 16 * M * N
    g = Guarded(mpc, need)
    g.lane._ws_bytes = need
    x, q, s = inputs.masks(rng, M, K), rng.integers(-8, 8, (N, K)), rng.integers(-(1 << 31), 1 << 31, (N, -(-K // group))).astype(np.int32)
    z = g.lane.matvec4(dev(mpc, x), attention.pack_weights4(torch.from_numpy(q)).cuda(), mpc.to_device(s), group, 16)
    g.check()
    equal(mpc, z, plain.matvec4(x, q, s, group, 16))


def test_matvec4_recorded(mpc, attention):
    """One graph of products that take a workspace (digits in memory, columns split, both): replays with eager work between."""
    rng, ln, calls = np.random.default_rng(8), mpc.Lane(0, single_queue=True), []
    for M, K, N, group in [(8, 4097, 4100, 64), (1, 16417, 40, 32), (16, 25088, 400, 128)]:
        q, s = rng.integers(-8, 8, (N, K)), rng.integers(-(1 << 31), 1 << 31, (N, -(-K // group))).astype(np.int32)
        calls.append((dev(mpc, inputs.masks(rng, M, K)), attention.pack_weights4(torch.from_numpy(q)).cuda(), mpc.to_device(s), group, filled((M, N)), q, s))
    def run():
        for x, w, s, group, z, _, _ in calls:
            ln.matvec4(x, w, s, group, 16, out=z)
    torch.cuda.synchronize()
    run(); ln.sync()
    with ln.capture() as cap:
        run()
    for _ in range(3):
        for x, *_, q, s in calls:                            # other words for every replay
            for t in x:
                t.add_(t << 7)
        torch.cuda.synchronize()
        cap.graph.launch(ln)
        ln.sync()
        for x, w, _, group, z, q, s in calls:
            equal(mpc, z, plain.matvec4(tuple(mpc.to_host(t) for t in x), q, s, group, 16))
    cap.graph.close()
    ln.close()


def test_matvec4_extreme_weights(mpc, lane, attention):
    """Every weight -8, every scale -2^31 and words whose digits are all -128: the largest sums there are."""
    M, K, N = 2, 20000, 3
    x = tuple(np.full((M, K), 0x7F7F7F7F7F7F7F80, U64) for _ in range(2))
    q, s = np.full((N, K), -8), np.full((N, 1), -(1 << 31), np.int32)
    z = lane.matvec4(dev(mpc, x), attention.pack_weights4(torch.from_numpy(q)).cuda(), mpc.to_device(s), 1 << 20, 31)
    lane.sync()
    equal(mpc, z, plain.matvec4(x, q, s, 1 << 20, 31))


def test_matvec4_long_rows(mpc, lane, attention):
    rng = np.random.default_rng(2)
    M, K, N = 1, 25088, 24
    q, s, x = rng.integers(-8, 8, (N, K)), rng.integers(1, 1 << 17, (N, K // 128)).astype(np.int32), inputs.masks(rng, M, K)
    z = lane.matvec4(dev(mpc, x), attention.pack_weights4(torch.from_numpy(q)).cuda(), mpc.to_device(s), 128, 20)
    lane.sync()
    equal(mpc, z, plain.matvec4(x, q, s, 128, 20))


# ------------------------------------------------------------------------------------------------ linear attention
STEP = [(1, 1, 1, 1), (2, 3, 64, 64), (1, 2, 16, 128), (3, 1, 128, 16), (2, 2, 17, 33), (1, 5, 100, 7), (1, 1, 128, 128), (1, 1, 3, 40), (40, 2, 8, 24)]


@pytest.mark.parametrize("B,H,dk,dv", STEP)
def test_step(mpc, lane, attention, B, H, dk, dv):
    print(f"step {B}x{H}x{dk}x{dv}", flush=True)
    rng = np.random.default_rng(dk * dv)
    d = inputs.one_token(rng, B, H, dk, dv)
    decay = attention.decay_powers([1.0, 0.0, 0.97, 0.5, 0.999][:H])
    want_o, want_s = plain.step(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], d["state"])
    q, k, v, state = (dev(mpc, d[n]) for n in ("q", "k", "v", "state"))
    mat = dev_all(mpc, d["mat"])
    out, new = filled((B, H, dv)), filled((B, H, dk, dv))
    lane.linear_attention_step(q, k, v, decay.cuda(), mat, state, out=out, state_out=new)
    lane.sync()
    equal(mpc, out, want_o, "o"); equal(mpc, new, want_s, "state"); equal(mpc, state, d["state"], "old state")
    lane.linear_attention_step(q, k, v, decay.cuda(), mat, state, out=out, state_out=state)      # in place
    lane.sync()
    equal(mpc, out, want_o, "o"); equal(mpc, state, want_s, "state in place")


@pytest.mark.parametrize("seed", range(3))
def test_step_on_any_words(mpc, lane, seed):
    """Shares, states and decays over their whole ranges: the ring's arithmetic alone."""
    rng = np.random.default_rng(seed)
    B, H, dk, dv = 2, 2, 20, 19
    d = inputs.one_token(rng, B, H, dk, dv)
    for n, shape in (("q", (B, H, dk)), ("k", (B, H, dk)), ("v", (B, H, dv)), ("state", (B, H, dk, dv))):
        d[n] = inputs.masks(rng, *shape)
    decay = rng.integers(0, 1 << 31, (H, 65)).astype(np.int32); decay[0, 1] = 2 ** 31 - 1
    out, new = lane.linear_attention_step(*(dev(mpc, d[n]) for n in ("q", "k", "v")), mpc.to_device(decay), dev_all(mpc, d["mat"]), dev(mpc, d["state"]))
    lane.sync()
    want_o, want_s = plain.step(d["q"], d["k"], d["v"], decay, d["mat"], d["state"])
    equal(mpc, out, want_o); equal(mpc, new, want_s)


PROMPT = [(1, 1, 1, 1, 1), (1, 2, 2, 5, 3), (2, 63, 1, 16, 16), (1, 64, 2, 64, 64), (1, 65, 1, 64, 64), (2, 130, 2, 48, 40), (1, 200, 1, 33, 70), (1, 128, 1, 128, 128),
          (1, 100, 1, 100, 65), (1, 320, 1, 64, 64), (3, 7, 3, 17, 15), (1, 90, 1, 65, 127),
          (9, 100, 3, 70, 72)]                               # one job for all of W V, two tiles


@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("B,T,H,dk,dv", PROMPT)
def test_prompt(mpc, lane, attention, B, T, H, dk, dv, state):
    print(f"prompt {B}x{T}x{H}x{dk}x{dv}", flush=True)
    rng = np.random.default_rng(T * dk + dv)
    d = inputs.prompt(rng, B, H, T, dk, dv)
    decay = attention.decay_powers([0.97, 1.0, 0.0][:H])
    zero = tuple(np.zeros_like(s) for s in d["state"])
    want_o, want_s = plain.linear_attention(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], d["state"] if state else zero)
    q, k, v, s = (dev(mpc, d[n]) for n in ("q", "k", "v", "state"))
    mat = dev_all(mpc, d["mat"])
    out, new = filled((B, T, H, dv)), filled((B, H, dk, dv))
    lane.linear_attention(q, k, v, decay.cuda(), mat, s if state else None, out=out, state_out=new)
    lane.sync()
    equal(mpc, out, want_o, "o"); equal(mpc, new, want_s, "state")
    if state:
        lane.linear_attention(q, k, v, decay.cuda(), mat, s, out=out, state_out=s)                # in place
        lane.sync()
        equal(mpc, out, want_o, "o"); equal(mpc, s, want_s, "state in place")


@pytest.mark.parametrize("layout", ["fused projection", "heads first", "odd strides", "one head for all"])
def test_prompt_and_step_layouts(mpc, lane, attention, layout):
    rng = np.random.default_rng(7)
    B, T, H, d_ = 2, 70, 3, 24
    d = inputs.prompt(rng, B, H, T, d_, d_)
    t = inputs.one_token(rng, B, H, d_, d_)
    if layout == "one head for all":                         # keys and values shared by all heads
        for x, axis in ((d, 2), (t, 1)):
            for n in ("k", "v"):
                x[n] = tuple(np.repeat(s.take([0], axis), H, axis) for s in x[n])
    decay = attention.decay_powers([0.9, 0.99, 1.0])

    def laid(x, token):
        tensors = {n: dev(mpc, x[n]) for n in ("q", "k", "v")}
        if layout == "fused projection":
            both = [torch.stack([tensors[n][p] for n in ("q", "k", "v")], -3) for p in range(2)]          # [.., 3, H, d]
            return {n: tuple(b.select(-3, i) for b in both) for i, n in enumerate(("q", "k", "v"))}
        if layout == "heads first":
            return {n: tuple(w.transpose(-2, 0 if token else 1).contiguous().transpose(-2, 0 if token else 1) for w in s) for n, s in tensors.items()}
        if layout == "odd strides":
            res = {}
            for n, s in tensors.items():
                res[n] = ()
                for w in s:
                    buf = torch.zeros(w.shape[:-2] + (H + 2, d_ + 1), dtype=torch.int64, device="cuda:0")
                    buf[..., 1:H + 1, 1:] = w
                    res[n] += (buf[..., 1:H + 1, 1:],)
            return res
        return {n: tuple(w[..., :1, :].expand(w.shape) if n != "q" else w for w in s) for n, s in tensors.items()}

    for x, token, call, want in ((d, False, lane.linear_attention, plain.linear_attention), (t, True, lane.linear_attention_step, plain.step)):
        w_o, w_s = want(x["q"], x["k"], x["v"], decay.numpy(), x["mat"], x["state"])
        a = laid(x, token)
        torch.cuda.synchronize()
        shape = (B, H, d_) if token else (B, T, H, d_)
        out = filled(shape[:-1] + (d_ + 3,)); view = tuple(o[..., 1:d_ + 1] for o in out)
        o, s = call(a["q"], a["k"], a["v"], decay.cuda(), dev_all(mpc, x["mat"]), dev(mpc, x["state"]), out=view)
        lane.sync()
        equal(mpc, o, w_o, "o"); equal(mpc, s, w_s, "state")
        for w in out:                                        # nothing beside the rows
            assert (w[..., 0] == -0x5A5A5A5A5A5A5A5A).all() and (w[..., d_ + 1:] == -0x5A5A5A5A5A5A5A5A).all()


def test_prompt_goes_on_where_another_ended(mpc, lane, attention):
    """Two prompts one after the other and then a token, the state handed on, on any words."""
    rng = np.random.default_rng(9)
    B, H, dk, dv = 1, 2, 20, 12
    decay = attention.decay_powers([0.95, 0.99])
    first, second, last = inputs.prompt(rng, B, H, 70, dk, dv, state=False), inputs.prompt(rng, B, H, 5, dk, dv), inputs.one_token(rng, B, H, dk, dv)
    zero = tuple(np.zeros((B, H, dk, dv), U64) for _ in range(2))
    _, s = plain.linear_attention(first["q"], first["k"], first["v"], decay.numpy(), first["mat"], zero)
    _, s = plain.linear_attention(second["q"], second["k"], second["v"], decay.numpy(), second["mat"], s)
    want, s = plain.step(last["q"], last["k"], last["v"], decay.numpy(), last["mat"], s)
    dd, state = decay.cuda(), None
    for x in (first, second):
        _, state = lane.linear_attention(*(dev(mpc, x[n]) for n in ("q", "k", "v")), dd, dev_all(mpc, x["mat"]), state, state_out=state)
    out, state = lane.linear_attention_step(*(dev(mpc, last[n]) for n in ("q", "k", "v")), dd, dev_all(mpc, last["mat"]), state, state_out=state)
    lane.sync()
    equal(mpc, out, want, "o"); equal(mpc, state, s, "state")


@pytest.mark.parametrize("bits", [8, 30])
def test_other_fixed_points(mpc, attention, bits):
    rng = np.random.default_rng(bits)
    ln = mpc.Lane(0, frac_bits=bits)                         # three streams
    B, T, H, dk, dv = 1, 66, 2, 9, 10
    d, t = inputs.prompt(rng, B, H, T, dk, dv), inputs.one_token(rng, B, H, dk, dv)
    decay = attention.decay_powers([0.9, 1.0], bits)
    for x, call, want in ((d, ln.linear_attention, plain.linear_attention), (t, ln.linear_attention_step, plain.step)):
        w_o, w_s = want(x["q"], x["k"], x["v"], decay.numpy(), x["mat"], x["state"], bits)
        o, s = call(*(dev(mpc, x[n]) for n in ("q", "k", "v")), decay.cuda(), dev_all(mpc, x["mat"]), dev(mpc, x["state"]))
        ln.sync()
        equal(mpc, o, w_o, "o"); equal(mpc, s, w_s, "state")
    ln.close()


@pytest.mark.parametrize("call", ["prompt", "step", "bias gradient"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1, 1), (1, 70, 3, 40, 65), (2, 130, 2, 128, 128)])
def test_workspaces_of_exactly_the_queried_size(mpc, attention, call, size):
    from test_gpu_workspace_bounds import Guarded
    B, T, H, dk, dv = size
    rng, L = np.random.default_rng(T), mpc.lib()
    need = {"prompt": lambda: L.mpc_linear_attention_workspace_bytes(*size), "step": lambda: L.mpc_linear_attention_step_workspace_bytes(B, H, dk, dv),
            "bias gradient": lambda: L.mpc_position_bias_grad_workspace_bytes(B, H, T, T, 5)}[call]()
    g = Guarded(mpc, need)
    g.lane._ws_bytes = need                                  # not to be grown
    decay = attention.decay_powers([0.9, 0.97, 1.0][:H])
    if call == "bias gradient":
        x, m = inputs.masks(rng, B, H, T, T), rng.integers(-1, 5, 2 * T - 1).astype(np.int32)
        grad, _ = g.lane.position_bias_grad(dev(mpc, x), mpc.to_device(m), 5)
        got, want = (grad,), (plain.position_bias_grad(x, m, 5)[0],)
    else:
        d = inputs.prompt(rng, B, H, T, dk, dv) if call == "prompt" else inputs.one_token(rng, B, H, dk, dv)
        run, form = (g.lane.linear_attention, plain.linear_attention) if call == "prompt" else (g.lane.linear_attention_step, plain.step)
        got = run(*(dev(mpc, d[n]) for n in ("q", "k", "v")), decay.cuda(), dev_all(mpc, d["mat"]), dev(mpc, d["state"]))
        want = form(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], d["state"])
    g.check()
    for a, w in zip(got, want):
        equal(mpc, a, w, call)


def test_calls_follow_the_lanes_stream(mpc, attention):
    """Inputs made by torch right before the call, ordered by wait_torch alone."""
    rng = np.random.default_rng(13)
    ln = mpc.Lane(0)
    d = inputs.one_token(rng, 2, 3, 33, 20)
    decay = attention.decay_powers([0.9, 0.97, 1.0])
    want = plain.step(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], d["state"])
    host = [dev(mpc, d[n]) for n in ("q", "k", "v", "state")]
    mat, dd = dev_all(mpc, d["mat"]), decay.cuda()
    slow = torch.randn(4096, 4096, device="cuda:0")
    torch.cuda.synchronize()
    for _ in range(8):
        slow = slow @ slow * 1e-3
    late = [tuple(w + 0 * slow[0, :1].long() for w in pair) for pair in host]          # written behind the products
    ln.wait_torch()
    o, s = ln.linear_attention_step(*late[:3], dd, mat, late[3])
    ln.sync()
    equal(mpc, o, want[0]); equal(mpc, s, want[1])
    ln.close()


# ------------------------------------------------------------------------------------------------ together
def test_recorded_graphs_and_two_lanes(mpc, attention):
    """A token's calls recorded on two lanes and replayed in turn, with eager work between: every replay gives the eager words
    (the state runs on, so each replay has another answer)."""
    rng = np.random.default_rng(11)
    B, H, d_ = 2, 2, 32
    lanes, runs = [mpc.Lane(0, single_queue=True) for _ in range(2)], []
    decay = attention.decay_powers([0.9, 0.99])
    for ln in lanes:
        d, p = inputs.one_token(rng, B, H, d_, d_), inputs.prompt(rng, B, H, 66, d_, d_)
        q, w = rng.integers(-8, 8, (20, H * d_)), None
        x = dict(d=d, p=p, q=q, s=rng.integers(1, 1 << 18, (20, 1)).astype(np.int32), state=d["state"])
        t = dict(arg=[dev(mpc, d[n]) for n in ("q", "k", "v")], mat=dev_all(mpc, d["mat"]), state=dev(mpc, d["state"]), o=filled((B, H, d_)), z=filled((B, 20)),
                 w=attention.pack_weights4(torch.from_numpy(q)).cuda(), s=mpc.to_device(x["s"]), decay=decay.cuda(),
                 parg=[dev(mpc, p[n]) for n in ("q", "k", "v")], pmat=dev_all(mpc, p["mat"]), po=filled((B, 66, H, d_)),
                 m=attention.relative_buckets(2, H, 4, 20).cuda(), table=filled((4, 1), 5), b=filled((B, 1, 2, H)), g=filled((4, 1)))

        def call(ln=ln, t=t):
            ln.linear_attention(*t["parg"], t["decay"], t["pmat"], t["state"], out=t["po"], state_out=t["state"])
            ln.linear_attention_step(*t["arg"], t["decay"], t["mat"], t["state"], out=t["o"], state_out=t["state"])
            ln.matvec4(tuple(o.view(B, H * d_) for o in t["o"]), t["w"], t["s"], 64, 18, out=t["z"])
            four = tuple(z[:, :2 * H].reshape(B, 1, 2, H) for z in t["b"])
            ln.position_bias(four, t["table"], t["m"], out=four)
            ln.position_bias_grad(four, t["m"], 4, out=t["g"])
        runs.append((x, t, call))
    torch.cuda.synchronize()

    def expect(x):
        p, d = x["p"], x["d"]
        po, s = plain.linear_attention(p["q"], p["k"], p["v"], decay.numpy(), p["mat"], x["state"])
        o, x["state"] = plain.step(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], s)
        return po, o, plain.matvec4(tuple(w.reshape(B, -1) for w in o), x["q"], x["s"], 64, 18)
    graphs = []
    for ln, (x, t, call) in zip(lanes, runs):
        call(); ln.sync(); expect(x)
        with ln.capture() as cap:
            call()
        graphs.append(cap.graph)
    for _ in range(3):
        for ln, g in zip(lanes, graphs):
            g.launch(ln)
        torch.ones(1000, device="cuda:0").sum().item()
        for ln in lanes:
            ln.sync()
        for x, t, _ in runs:
            po, o, z = expect(x)
            equal(mpc, t["po"], po, "prompt"); equal(mpc, t["o"], o, "o"); equal(mpc, t["z"], z, "z"); equal(mpc, t["state"], x["state"], "state")
    for g in graphs:
        g.close()
    for ln in lanes:
        ln.close()


@pytest.mark.parametrize("B,H,T,dk,dv", [(2, 2, 70, 16, 24), (1, 1, 1, 1, 1), (1, 3, 64, 5, 7)])
def test_dealt_material_unfolds_to_the_masks_products(mpc, lane, B, H, T, dk, dv):
    from paper_2209_13643_amd import dealer
    g = dealer.gen(1, "cuda:0")
    host = lambda m: {n: tuple(mpc.to_host(t.contiguous()) for t in s) for n, s in m.items()}
    m = host(dealer.attention_step_material(lane, g, B, H, dk, dv))
    whole, own = lambda s: s[0] + s[1], lambda s: s[0]
    outer, times = lambda a, b: a[..., :, None] * b[..., None, :], lambda a, b: (a[..., :, None] * b).sum(-2, dtype=U64)
    assert np.array_equal(sum(m["c_u"]), outer(whole(m["a_k"]), whole(m["a_v"])) - outer(m["a_k"][0], m["a_v"][0])), "c_u of a token"
    assert np.array_equal(sum(m["c_o"]), times(whole(m["a_q"]), whole(m["a_s"])) - times(m["a_q"][0], m["a_s"][0])), "c_o of a token"
    m = host(dealer.attention_material(lane, g, B, H, T, dk, dv))
    for n in range(B * H):
        for c in range(-(-T // 64)):
            t = slice(c * 64, min(T, c * 64 + 64))
            L = t.stop - t.start
            p, u, o = (0, 0, 0)
            for take, sign in ((whole, U64(1)), (own, ~U64(0))):
                a = {x: take([w[n, t] for w in m[x]]) for x in ("a_q", "a_k", "a_qd", "a_kd", "a_v", "a_w")}
                p = p + sign * (a["a_q"] @ a["a_k"].T)
                u = u + sign * (a["a_kd"].T @ a["a_v"])
                o = o + sign * (np.tril(a["a_w"][:, :L]) @ a["a_v"] + a["a_qd"] @ take([w[n, c] for w in m["a_s"]]))
            assert np.array_equal(sum(m["c_p"])[n, t, :L], p) and np.array_equal(sum(m["c_u"])[n, c], u) and np.array_equal(sum(m["c_o"])[n, t], o)


def test_layer_serves_a_prompt_and_tokens(mpc, lane, attention):
    """TokenLayer on dealt material: a prompt, then two tokens, decoded, against float64 with the quantised weights."""
    from paper_2209_13643_amd import dealer
    g = dealer.gen(3, "cuda:0")
    rng = np.random.default_rng(3)
    B, T, H, dk, dv, D = 2, 70, 2, 16, 24, 48
    wq, wo = rng.normal(0, D ** -0.5, (H * (2 * dk + dv), D)), rng.normal(0, (H * dv) ** -0.5, (D, H * dv))
    (pq, sq), (po, so) = (attention.quantize4(torch.from_numpy(w), 32) for w in (wq, wo))
    decay = [0.9, 0.99]
    layer = attention.TokenLayer(H, dk, dv, pq.cuda(), sq.cuda(), po.cuda(), so.cuda(), 32, attention.decay_powers(decay).cuda())
    unpack = lambda p, s, K: ((torch.stack((p & 15, p >> 4), -1).flatten(1)[:, :K].int() ^ 8) - 8).numpy() * np.repeat(s.numpy() / 2.0 ** 20, 32, 1)[:, :K]
    Wq, Wo = unpack(pq, sq, D), unpack(po, so, H * dv)
    X = inputs.fixed(rng, 1.0, B, T + 2, D)
    xs = inputs.share(rng, X)
    real = lambda s: (mpc.to_host(s[0]) + mpc.to_host(s[1])).view(np.int64).astype(np.float64) / 65536
    x = X.view(np.int64) / 65536.0
    qkv = x @ Wq.T
    q, k, v = (qkv[..., a:b].reshape(B, T + 2, H, -1) for a, b in ((0, H * dk), (H * dk, 2 * H * dk), (2 * H * dk, H * (2 * dk + dv))))
    S, want = np.zeros((B, H, dk, dv)), np.zeros((B, T + 2, D))
    for t in range(T + 2):
        S = np.array(decay)[None, :, None, None] * S + k[:, t, :, :, None] * v[:, t, :, None]
        want[:, t] = (q[:, t, :, :, None] * S).sum(2).reshape(B, -1) @ Wo.T
    m = dealer.attention_material(lane, g, B, H, T, dk, dv)
    y, state = layer.prompt(lane, dev(mpc, tuple(np.ascontiguousarray(s[:, :T]) for s in xs)), m)
    lane.sync()
    # a step of 2^-16 in q, k, v and the decays (2^-17) times sums of at most 70 terms of |k v| < 16 and 16 of |q| < 5,
    # three rescales each: below 2^-16 * (70 * 16 * 5 * 2) < 0.2; typical errors add as their root, 2^-16 * 5 * sqrt(70 * 16 * 2 * 3)
    assert np.abs(real(y) - want[:, :T]).max() < 2 ** -5
    for t in (T, T + 1):
        m = dealer.attention_step_material(lane, g, B, H, dk, dv)
        y = layer.token(lane, dev(mpc, tuple(np.ascontiguousarray(s[:, t]) for s in xs)), m, state)
        lane.sync()
        assert np.abs(real(y) - want[:, t]).max() < 2 ** -5


def test_scores_form_trains(mpc, lane, attention):
    """O = (Q K^T + bias) V and all its gradients, decoded, against float64 and against differences of a float64 loss."""
    import helpers
    rng = np.random.default_rng(5)
    B, H, T, d_, n = 2, 2, 20, 8, 6
    N = B * H
    import oracle
    from paper_2209_13643_amd import synth
    deal = lambda sa, sb, turn_a=False, turn_b=False: _triple(rng, sa, sb, turn_a, turn_b)

    def _triple(rng, sa, sb, turn_a, turn_b):
        A, Bm = inputs.words(rng, *sa), inputs.words(rng, *sb)
        left, right = A.swapaxes(1, 2) if turn_a else A, Bm.swapaxes(1, 2) if turn_b else Bm
        return tuple(dev(mpc, inputs.share(rng, w)) for w in (A, Bm, left @ right))
    vals = {x: inputs.fixed(rng, 0.5, B, H, T, d_) for x in ("q", "k", "v", "go")}
    tab = inputs.fixed(rng, 0.5, n, H)
    sh = {x: dev(mpc, inputs.share(rng, w)) for x, w in vals.items()}
    m = attention.relative_buckets(T, T, n, 16, causal=True)
    o, scores = attention.scores_forward(lane, sh["q"], sh["k"], sh["v"], dev(mpc, inputs.share(rng, tab)), m.cuda(),
                                         deal((N, T, d_), (N, T, d_), turn_b=True), deal((N, T, T), (N, T, d_)))
    gq, gk, gv, gt = attention.scores_backward(lane, sh["go"], sh["q"], sh["k"], sh["v"], scores, m.cuda(), n,
                                               deal((N, T, d_), (N, T, d_), turn_b=True), deal((N, T, T), (N, T, d_), turn_a=True),
                                               deal((N, T, T), (N, T, d_)), deal((N, T, T), (N, T, d_), turn_a=True))
    lane.sync()
    real = lambda s: (mpc.to_host(s[0].contiguous()) + mpc.to_host(s[1].contiguous())).view(np.int64).astype(np.float64) / 65536
    f = {x: w.view(np.int64) / 65536.0 for x, w in vals.items()}
    f["t"] = tab.view(np.int64) / 65536.0
    at = m.numpy()[np.arange(T) - np.arange(T)[:, None] + T - 1]

    def forward(q, k, v, t):
        s = (q @ k.swapaxes(2, 3) + t[np.maximum(at, 0)].transpose(2, 0, 1)) * (at >= 0)
        return s, s @ v
    s, want = forward(f["q"], f["k"], f["v"], f["t"])
    gs = (f["go"] @ f["v"].swapaxes(2, 3)) * (at >= 0)
    grads = dict(q=gs @ f["k"], k=gs.swapaxes(2, 3) @ f["q"], v=s.swapaxes(2, 3) @ f["go"],
                 t=np.stack([(gs * (at == u)).sum((0, 2, 3)) for u in range(n)]))
    # one product's rescale is below 2 steps of 2^-16 off, and a second product sums it over at most 20 terms below 4
    near = 20 * 4 * 2 * 2.0 ** -16 + 2 * 2.0 ** -16
    assert np.abs(real(scores) - s).max() < 2 ** -15 + 1e-9 and np.abs(real(o) - want).max() < near
    for name, got in (("q", gq), ("k", gk), ("v", gv)):
        assert np.abs(real(got) - grads[name]).max() < near, name
    assert np.abs(real(gt) - grads["t"]).max() < B * T * T * 2 * 2.0 ** -16
    # the loss <go, O> is linear in every operand: its differences are exact up to rounding
    for name in ("q", "k", "v", "t"):
        moved = dict(f)
        step = rng.normal(size=f[name].shape)
        moved[name] = f[name] + step
        diff = (f["go"] * (forward(moved["q"], moved["k"], moved["v"], moved["t"])[1] - want)).sum()
        assert abs(diff - (step * grads[name]).sum()) < 1e-8 * (1 + abs(diff))


def test_wrong_tensors_are_refused(mpc, lane, attention):
    x, t = filled((1, 2, 3, 4)), filled((5, 2))
    m = torch.zeros(6, dtype=torch.int32, device="cuda:0")
    for bad in [dict(scores=(x[0], x[1].int())), dict(scores=tuple(w.transpose(2, 3) for w in x)), dict(buckets=m[:5]), dict(buckets=m.long()),
                dict(table=filled((5, 3))), dict(buckets=m.cpu()), dict(scores=(x[0],))]:
        with pytest.raises((ValueError, IndexError)):
            lane.position_bias(**{**dict(scores=x, table=t, buckets=m), **bad})
    w, s = torch.zeros(4, 32, dtype=torch.uint8, device="cuda:0"), torch.ones(4, 2, dtype=torch.int32, device="cuda:0")
    for bad in [dict(w=w[:, :16].contiguous()), dict(scales=s[:, :1].contiguous()), dict(w=w.int()), dict(group=0)]:
        with pytest.raises(ValueError):
            lane.matvec4(**{**dict(x=filled((1, 40)), w=w, scales=s, group=32), **bad})
    with pytest.raises(mpc.MpcError):
        lane.matvec4(filled((1, 40)), w, torch.ones(4, 1, dtype=torch.int32, device="cuda:0"), 48)
    q, st, d = filled((1, 2, 8)), filled((1, 2, 8, 8)), torch.zeros(2, 65, dtype=torch.int32, device="cuda:0")
    with pytest.raises(ValueError):
        lane.linear_attention_step(q, q, q, d, {}, st)
    with pytest.raises(ValueError):
        lane.linear_attention_step(q, filled((1, 3, 8)), q, d, {}, st)
