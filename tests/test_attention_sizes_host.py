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
