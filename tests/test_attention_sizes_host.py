"""Sizes near the ends of their types in the attention and public-weight calls: refused or counted right, on the host (no GPU)."""
import pytest
import torch

import fake_hip
from test_attention_calls_host import host_lane, library, pair  # noqa: F401
from test_attention_host import REFUSALS

E, R = -1, -4

GROUPS = r'''
lib.mpc_ctx_set_workspace(ctx, array(big), big)
top = (1 << 31) - 128
# one group for all columns: its scales lie on the output, or apart from it
result["on the output"] = [mv(K=K, N=5, group=top, s=x.p[0], z=x) for K in (1, 128, 129, 256, 25088)]
result["apart"] = [mv(K=K, N=5, group=top) for K in (1, 128, 129, 256, 25088)]
'''


def test_a_group_of_nearly_2_to_the_31_columns(tmp_path):
    """Its number of groups is one.  (K + group - 1 is beyond an int, undefined; the compiler's unsigned division happened to give one.)"""
    r = fake_hip.run(tmp_path, REFUSALS + GROUPS)
    assert r["on the output"] == [E] * 5 and r["apart"] == [0] * 5


@pytest.mark.parametrize("group", [1 << 31, (1 << 32) + 32, (1 << 40) + 128])
def test_groups_beyond_an_int_are_refused(library, group):  # noqa: F811
    """ctypes would hand over the low 32 bits: groups of 32 with the scales of one."""
    with pytest.raises(ValueError):
        host_lane().matvec4(pair(1, 64), torch.zeros(3, 32, dtype=torch.uint8), torch.ones(3, 1, dtype=torch.int32), group)
    assert not library.calls


WRAPPED = r'''
lib.mpc_linear_attention_workspace_bytes.restype = lib.mpc_linear_attention_step_workspace_bytes.restype = c_size_t
lib.mpc_ctx_set_workspace(ctx, array(big), big)
# products of the sizes that are 2^64, so zero in 64 bits, or come out small
result["queries"] = [lib.mpc_linear_attention_workspace_bytes(1 << 30, 1 << 30, 1 << 10, 8, 8), lib.mpc_linear_attention_workspace_bytes(1 << 25, 1 << 30, 1 << 15, 8, 8),
                     lib.mpc_position_bias_grad_workspace_bytes(1 << 20, 1 << 10, 1 << 30, 1 << 30, 4)]
sizes = [dict(B=1 << 30, H=1, Tq=1 << 15, Tk=1 << 30), dict(B=1 << 20, H=1 << 10, Tq=1 << 15, Tk=1 << 30), dict(B=1, H=1, Tq=1 << 30, Tk=(1 << 30) - 4096)]
result["bias"] = [bias(**s) for s in sizes]
result["grad"] = [grad(**s) for s in sizes]
def prompts(**s):
    lib.mpc_ctx_set_workspace(ctx, array(big), 1 << 30)
    mat = Material((Share * 10)(*[share(big) for i in range(10)]))
    x = Operands(share(big), share(big), share(big), Strides(), Strides(), Strides(), array(big), none, share(big), Strides(1 << 40, 8, 8), none)
    return lib.mpc_linear_attention(ctx, ctypes.byref(x), ctypes.byref(mat), s["B"], s["T"], s["H"], 8, 8)
result["prompt"] = [prompts(B=1 << 30, T=1 << 30, H=1 << 10), prompts(B=1 << 25, T=1 << 30, H=1 << 15)]
result["launched"] = launches()
'''


def test_sizes_whose_product_wraps_are_refused(tmp_path):
    r = fake_hip.run(tmp_path, REFUSALS + WRAPPED)
    assert r["queries"] == [0, 0, 0] and r["bias"] == [R] * 3 and r["grad"] == [R] * 3 and r["prompt"] == [R] * 2
    assert r["launched"] == []


STRIDES = r'''
far = 1 << 62                                                # four batches of it are 2^64 words
o = share(big)
result["prompt"] = [prompt(B=5, sq=Strides(far, H * dk, dk)), prompt(B=5, q=o, o=o, sq=Strides(far, H * dk, dk)), prompt(B=5, so=Strides(far, 18, 6)),
                    prompt(B=2, sq=Strides((1 << 40) + 1, H * dk, dk)), prompt(T=3, so=Strides(18, 1 << 40, 6)), prompt(H=3, so=Strides(18, 6, (1 << 39) + 1))]
result["step"] = [step(B=5, so=Strides(far, 0, 6)), step(H=5, so=Strides(30, 0, far))]
result["launched by refused calls"] = launches()
# an axis of one entry has no use for its stride
result["one"] = [prompt(B=1, sq=Strides(far, H * dk, dk), so=Strides(far, 18, 6)), step(B=1, so=Strides(far, 0, 6))]
'''


def test_strides_whose_extent_wraps_are_refused(tmp_path):
    r = fake_hip.run(tmp_path, REFUSALS + "launches()\n" + STRIDES)
    assert r["prompt"] == [R] * 6 and r["step"] == [R] * 2 and r["launched by refused calls"] == []
    assert r["one"] == [0] * 2


def test_one_token_has_no_use_for_its_stride(tmp_path):
    """A view of one token of a long array may have any stride there; with two tokens the limit holds."""
    r = fake_hip.run(tmp_path, REFUSALS + "result['one'] = [prompt(T=t, sq=Strides(H * dk, 1 << 23, dk)) for t in (1, 2)]")
    assert r["one"] == [0, R]
