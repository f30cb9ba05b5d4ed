"""Registers of the attention and public-weight kernels, compiled here with the resource-usage remarks on (no GPU needed): which of
them spill, and how much at most, is what their comments say."""
import pytest

from test_kernel_registers import usage

SPILLED = {"k_chunk_open": 80, "k_step": 28}                  # bytes a lane, at most


@pytest.mark.parametrize("source,kernels", [("position_bias.hip", 4), ("matvec4.hip", 16), ("linear_attention.hip", 4)])
def test_attention_kernels(source, kernels):
    rows = usage(source)
    assert len(rows) == kernels, [r[0] for r in rows]
    for name, vgprs, agprs, scratch in rows:
        kernel = name.replace("void ", "").split("(")[0].split("<")[0]
        assert scratch <= SPILLED.get(kernel, 0), (name, scratch)
        assert vgprs + agprs <= 256, (name, vgprs, agprs)     # two waves to a SIMD
