"""Attention and public-weight calls whose workgroups take several jobs each, on every share bit for bit against the plain 64-bit
forms; and calls at the ends of what they take."""
import numpy as np
import pytest
import torch

import attention_inputs as inputs
from oracle import attention as plain
from test_gpu_attention import U64, attention, dev, dev_all, equal, filled, lane, mpc  # noqa: F401

pytestmark = pytest.mark.gpu


def any_words(rng, d, shapes):
    """Shares over their whole range in place of encoded values: the ring's arithmetic alone."""
    for n, shape in shapes.items():
        d[n] = inputs.masks(rng, *shape)
    return d


@pytest.mark.parametrize("B,H,dk,dv", [(70, 16, 8, 33), (70, 16, 5, 64), (33, 16, 40, 70)])
def test_steps_of_several_jobs(mpc, lane, B, H, dk, dv):  # noqa: F811
    """More slices of 32 columns than the 1024 workgroups of a launch: k and q, partial sums and buffers are used again."""
    print(f"step {B}x{H}x{dk}x{dv}", flush=True)
    assert B * H * -(-dv // 32) > 1024
    rng = np.random.default_rng(dv)
    d = any_words(rng, inputs.one_token(rng, B, H, dk, dv), dict(q=(B, H, dk), k=(B, H, dk), v=(B, H, dv), state=(B, H, dk, dv)))
    decay = rng.integers(0, 1 << 31, (H, 65)).astype(np.int32)
    want_o, want_s = plain.step(d["q"], d["k"], d["v"], decay, d["mat"], d["state"])
    state, out = dev(mpc, d["state"]), filled((B, H, dv))
    lane.linear_attention_step(*(dev(mpc, d[n]) for n in ("q", "k", "v")), mpc.to_device(decay), dev_all(mpc, d["mat"]), state, out=out, state_out=state)
    lane.sync()
    equal(mpc, out, want_o, "o"); equal(mpc, state, want_s, "state")


# chunks x kinds of jobs beyond the 256 workgroups of a launch: kinds that take turns (2 of the first launch, 2 of the last), kinds
# that do not (3 and 5), and more state elements than the second launch has threads (524288)
MANY = [(17, 8, 70, 16, 24), (9, 16, 10, 10, 70), (9, 8, 10, 70, 72), (5, 8, 70, 128, 128)]


@pytest.mark.parametrize("B,H,T,dk,dv", MANY)
def test_prompts_of_several_jobs(mpc, lane, B, H, T, dk, dv):  # noqa: F811
    print(f"prompt {B}x{T}x{H}x{dk}x{dv}", flush=True)
    rng = np.random.default_rng(T * dk + dv)
    cells, mt, nt = B * H * -(-T // 64), -(-dk // 64), -(-dv // 64)
    assert cells * (1 + mt * nt) > 256 and (cells * nt > 256 or B * H * dk * dv > 524288 or mt > 1)
    d = any_words(rng, inputs.prompt(rng, B, H, T, dk, dv), dict(q=(B, T, H, dk), k=(B, T, H, dk), v=(B, T, H, dv), state=(B, H, dk, dv)))
    decay = rng.integers(0, 1 << 31, (H, 65)).astype(np.int32)
    want_o, want_s = plain.linear_attention(d["q"], d["k"], d["v"], decay, d["mat"], d["state"])
    out, new = filled((B, T, H, dv)), filled((B, H, dk, dv))
    lane.linear_attention(*(dev(mpc, d[n]) for n in ("q", "k", "v")), mpc.to_device(decay), dev_all(mpc, d["mat"]), dev(mpc, d["state"]), out=out, state_out=new)
    lane.sync()
    equal(mpc, out, want_o, "o"); equal(mpc, new, want_s, "state")


def test_recorded_bias_and_gradient(mpc):  # noqa: F811
    """Bias in place, a table gradient of one launch and one of two, recorded; other words for every replay, eager work between."""
    rng, ln, n = np.random.default_rng(21), mpc.Lane(0, single_queue=True), 6
    small, large = (2, 3, 2, 5), (2, 3, 130, 130)
    need = lambda s: mpc.lib().mpc_position_bias_grad_workspace_bytes(*s, n)
    assert need(large) > 2 * 3 * n * 8 * 8 >= need(small)     # the partial sums of more than eight workgroups to a head, and of one
    calls = []
    for s in (small, large):
        m = rng.integers(-1, n, s[2] + s[3] - 1).astype(np.int32)
        x, t, g = inputs.masks(rng, *s), inputs.masks(rng, n, s[1]), inputs.masks(rng, *s)
        calls.append((m, t, x, g, mpc.to_device(m), dev(mpc, t), dev(mpc, x), dev(mpc, g), filled((n, s[1])), filled(s)))

    def run():
        for *_, m, t, x, g, grad, scores in calls:
            ln.position_bias(x, t, m, out=x)
            ln.position_bias_grad(g, m, n, out=grad, scores_out=scores)
    torch.cuda.synchronize()
    run(); ln.sync()
    with ln.capture() as cap:
        run()
    want = [plain.position_bias(x, t, m) for m, t, x, *_ in calls]
    for _ in range(3):
        for *_, g, grad, scores in calls:
            for w in g:
                w.add_(w << 9)
            for w in (*grad, *scores):
                w.fill_(-1)
        torch.ones(1000, device="cuda:0").sum().item()
        torch.cuda.synchronize()
        cap.graph.launch(ln)
        ln.sync()
        want = [plain.position_bias(x, t, m) for x, (m, t, *_) in zip(want, calls)]
        for b, (m, _, _, _, _, _, x, g, grad, scores) in zip(want, calls):
            wg, ws = plain.position_bias_grad(tuple(mpc.to_host(w) for w in g), m, n)
            equal(mpc, x, b, "bias"); equal(mpc, grad, wg, "table gradient"); equal(mpc, scores, ws, "scores gradient")
    cap.graph.close()
    ln.close()


def test_temporaries_of_a_call_that_grows_the_workspace(mpc, attention):  # noqa: F811
    """Behind work that is still running, torch is given the chance to hand out the call's temporaries again."""
    rng, ln = np.random.default_rng(4), mpc.Lane(0, single_queue=True)
    B, H, T, dk, dv = 2, 2, 130, 16, 24
    d = inputs.prompt(rng, B, H, T, dk, dv)
    decay = attention.decay_powers([0.9, 0.99])
    want_o, want_s = plain.linear_attention(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], d["state"])
    big, t, m = filled((8, 12, 512, 512)), filled((32, 12)), attention.relative_buckets(512, 512, 32, 128).cuda()
    ln.reserve(4096)
    torch.cuda.synchronize()
    for _ in range(20):
        ln.position_bias(big, t, m, out=big)
    o, s = ln.linear_attention(*(dev(mpc, d[n]) for n in ("q", "k", "v")), decay.cuda(), dev_all(mpc, d["mat"]), dev(mpc, d["state"]))
    again = [filled(tuple(w[0].shape), 3) for w in (*d["mat"].values(), d["q"], d["k"], d["v"], d["state"]) for _ in range(2)]
    ln.sync()
    equal(mpc, o, want_o, "o"); equal(mpc, s, want_s, "state")
    del again
    ln.close()


def test_layer_with_more_rows_than_a_product_takes(mpc, lane, attention):  # noqa: F811
    """16 sequences of 4100 tokens against the same ones a sequence at a time."""
    from paper_2209_13643_amd import dealer
    B, T, H, d, width = 16, 4100, 1, 4, 8
    assert B * T > 65535
    g, rng = dealer.gen(5, "cuda:0"), np.random.default_rng(6)
    wq, wo = (attention.pack_weights4(torch.from_numpy(rng.integers(-8, 8, s))).cuda() for s in ((3 * H * d, width), (width, H * d)))
    sq, so = (torch.from_numpy(rng.integers(1, 1 << 18, (n, 1)).astype(np.int32)).cuda() for n in (3 * H * d, width))
    layer = attention.TokenLayer(H, d, d, wq, sq, wo, so, 32, attention.decay_powers([0.97]).cuda())
    x, m = tuple(dealer.rand_words(g, (B, T, width), "cuda:0") for _ in range(2)), dealer.attention_material(lane, g, B, H, T, d, d)
    torch.cuda.synchronize()
    y, state = layer.prompt(lane, x, m)
    lane.sync()
    for b in (0, 7, B - 1):
        z, s = layer.prompt(lane, tuple(w[b:b + 1] for w in x), {n: tuple(w[b:b + 1] for w in pair) for n, pair in m.items()})
        lane.sync()
        for p in range(2):
            assert torch.equal(y[p][b], z[p][0]) and torch.equal(state[p][b], s[p][0])


def test_dealt_material_of_more_heads_than_a_product_takes(mpc, lane):  # noqa: F811
    from paper_2209_13643_amd import dealer
    B, H, dk, dv = 2049, 16, 2, 1
    m = dealer.attention_step_material(lane, dealer.gen(2, "cuda:0"), B, H, dk, dv)
    a, v, q, s = (m[n][0] + m[n][1] for n in ("a_k", "a_v", "a_q", "a_s"))
    assert torch.equal(m["c_u"][0] + m["c_u"][1], a[..., None] * v[..., None, :] - m["a_k"][0][..., None] * m["a_v"][0][..., None, :])
    assert torch.equal(m["c_o"][0] + m["c_o"][1], (q[..., None] * s).sum(-2) - (m["a_q"][0][..., None] * m["a_s"][0]).sum(-2))


def test_strides_of_axes_of_one_entry(mpc, lane, attention):  # noqa: F811
    """One token of a long array, one batch and one head, with whatever their strides are called."""
    rng = np.random.default_rng(31)
    for B, T, H in ((2, 1, 3), (1, 66, 1)):
        d = inputs.prompt(rng, B, H, T, 12, 10)
        decay = attention.decay_powers([0.9, 0.99, 1.0][:H])
        want_o, want_s = plain.linear_attention(d["q"], d["k"], d["v"], decay.numpy(), d["mat"], d["state"])

        def odd(pair):
            a, b = dev(mpc, pair)
            return a, b.as_strided(b.shape, [1 << 40 if n == 1 else s for n, s in zip(b.shape, b.stride())])
        o, s = lane.linear_attention(*(odd(d[n]) for n in ("q", "k", "v")), decay.cuda(), dev_all(mpc, d["mat"]), dev(mpc, d["state"]))
        lane.sync()
        equal(mpc, o, want_o, "o"); equal(mpc, s, want_s, "state")


def test_matvec4_one_group_for_all_columns(mpc, lane, attention):  # noqa: F811
    """The largest group there is: the same words as with the smallest one that holds all columns."""
    rng = np.random.default_rng(1)
    M, K, N = 2, 300, 20
    x, q, s = inputs.masks(rng, M, K), rng.integers(-8, 8, (N, K)), rng.integers(-(1 << 31), 1 << 31, (N, 1)).astype(np.int32)
    z = lane.matvec4(dev(mpc, x), attention.pack_weights4(torch.from_numpy(q)).cuda(), mpc.to_device(s), (1 << 31) - 128, 20)
    lane.sync()
    equal(mpc, z, plain.matvec4(x, q, s, 384, 20))


def test_decays_that_lie_on_the_device(mpc, attention):  # noqa: F811
    d = torch.tensor([0.0, 0.97, 1 - 2.0 ** -7, 1.0], dtype=torch.float64)
    on_device = attention.decay_powers(d.cuda(), 20)
    assert on_device.is_cuda and torch.equal(on_device.cpu(), attention.decay_powers(d, 20))
