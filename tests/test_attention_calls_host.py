"""The binding of the attention and public-weight calls on a stand-in for the library: what a lane keeps, and what it hands over.
No GPU: the tensors lie in host memory, and no kernel is launched."""
import pytest
import torch

from paper_2209_13643_amd import mpc

B, T, H, DK, DV = 1, 3, 2, 4, 5


class Library:
    """Every call succeeds, other than that an entry point finds the workspace too small until one is set."""

    def __init__(self):
        self.room, self.calls = False, []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace_bytes"):
                return 4096
            if name == "mpc_ctx_set_workspace":
                self.room = True
                return 0
            if name.startswith("mpc_ctx_"):
                return 0
            self.calls.append((name, args))
            return 0 if self.room else mpc.MPC_ENOMEM
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(mpc, "lib", lambda: lib)
    return lib


def host_lane():
    lane = mpc.Lane.__new__(mpc.Lane)
    lane.device, lane._index, lane._h = torch.device("cpu"), -1, None
    lane._handed, lane._pending = set(), []
    lane._ws, lane._ws_bytes = torch.empty(8), 8              # one that has to grow
    return lane


def pair(*shape):
    return tuple(torch.zeros(shape, dtype=torch.int64) for _ in range(2))


def material(names, **sizes):
    return {n: pair(sizes[n]) for n in names}


def bias_grad(lane):
    g, m = pair(B, H, T, T), torch.zeros(2 * T - 1, dtype=torch.int32)
    out, _ = lane.position_bias_grad(g, m, 4)
    return [*g, m, *out]


def matvec4(lane):
    x, w, s = pair(2, 40), torch.zeros(3, 32, dtype=torch.uint8), torch.ones(3, 2, dtype=torch.int32)
    return [*x, w, s, *lane.matvec4(x, w, s, 32)]


def prompt(lane):
    q, k, v, d = pair(B, T, H, DK), pair(B, T, H, DK), pair(B, T, H, DV), torch.zeros(H, 65, dtype=torch.int32)
    rows, tok, cell = B * H * T, B * H * T * 64, B * H * DK * DV
    mat = material(mpc._ATTENTION_MASKS, a_q=rows * DK, a_k=rows * DK, a_qd=rows * DK, a_kd=rows * DK, a_v=rows * DV, a_w=tok, a_s=cell, c_p=tok, c_u=cell, c_o=rows * DV)
    o, s = lane.linear_attention(q, k, v, d, mat)
    return [*q, *k, *v, d, *o, *s, *(t for p in mat.values() for t in p)]


def step(lane):
    q, k, v, d, s = pair(B, H, DK), pair(B, H, DK), pair(B, H, DV), torch.zeros(H, 65, dtype=torch.int32), pair(B, H, DK, DV)
    n, cell = B * H, B * H * DK * DV
    mat = material(mpc._STEP_MASKS, a_q=n * DK, a_k=n * DK, a_v=n * DV, a_s=cell, c_u=cell, c_o=n * DV)
    o, new = lane.linear_attention_step(q, k, v, d, mat, s)
    return [*q, *k, *v, d, *s, *o, *new, *(t for p in mat.values() for t in p)]


@pytest.mark.parametrize("call", [bias_grad, matvec4, prompt, step])
def test_a_call_that_grows_the_workspace_keeps_its_tensors(library, call):
    """The growing workspace waits for the lane, which lets go of the tensors noted until then; those of the call that is enqueued
    afterwards stay with the lane until it is next waited for."""
    lane = host_lane()
    tensors = call(lane)
    assert len(library.calls) == 2                            # refused, then enqueued
    held = {id(t) for t in lane._pending}
    assert all(id(t) in held for t in tensors)
    lane.sync()
    assert not lane._pending


@pytest.mark.parametrize("B,T,H,d", [(1, 3, 2, 4), (2, 1, 2, 4), (2, 3, 1, 4), (1, 1, 1, 4), (2, 3, 2, 1)])
def test_the_stride_of_an_axis_of_one_entry_says_nothing(library, B, T, H, d):
    """Both shares of q, k, v and the output lie alike, other than in what a view of one entry calls its stride."""
    library.room = True
    lane, decay = host_lane(), torch.zeros(H, 65, dtype=torch.int32)

    def shares(*shape):
        a, b = pair(*shape)
        return a, b.as_strided(shape, [1 << 30 if n == 1 else s for n, s in zip(shape, b.stride())])
    rows, tok, cell = B * H * T, B * H * T * 64, B * H * d * d
    mat = material(mpc._ATTENTION_MASKS, a_q=rows * d, a_k=rows * d, a_qd=rows * d, a_kd=rows * d, a_v=rows * d, a_w=tok, a_s=cell, c_p=tok, c_u=cell, c_o=rows * d)
    lane.linear_attention(shares(B, T, H, d), shares(B, T, H, d), shares(B, T, H, d), decay, mat, out=shares(B, T, H, d))
    n = B * H
    mat = material(mpc._STEP_MASKS, a_q=n * d, a_k=n * d, a_v=n * d, a_s=cell, c_u=cell, c_o=n * d)
    lane.linear_attention_step(shares(B, H, d), shares(B, H, d), shares(B, H, d), decay, mat, pair(B, H, d, d), out=shares(B, H, d))
    assert [name for name, _ in library.calls] == ["mpc_linear_attention", "mpc_linear_attention_step"]


def test_shares_that_lie_differently_are_refused(library):
    lane, (a, b) = host_lane(), pair(2, 2, 4)
    n, cell = 4, 2 * 2 * 16
    mat = material(mpc._STEP_MASKS, a_q=n * 4, a_k=n * 4, a_v=n * 4, a_s=cell, c_u=cell, c_o=n * 4)
    with pytest.raises(ValueError):
        lane.linear_attention_step((a, b.transpose(0, 1)), pair(2, 2, 4), pair(2, 2, 4), torch.zeros(2, 65, dtype=torch.int32), mat, pair(2, 2, 4, 4))
    assert not library.calls
