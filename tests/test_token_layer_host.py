"""TokenLayer's order of calls on a stand-in for the lane, in plain whole numbers.  No GPU."""
import pytest
import torch

from paper_2209_13643_amd import attention


class Plain:
    """A lane whose products take the library's most rows, and whose attention gives back v."""

    def __init__(self):
        self.rows = []

    def matvec4(self, x, w, scales, group, scale_bits=16, out=None):
        M = x[0].shape[0]
        if M > 65535:
            raise ValueError("too many rows")
        assert all(t.is_contiguous() for t in x)
        self.rows.append(M)
        z = tuple(t @ w.T for t in x)
        if out is None:
            return z
        for o, t in zip(out, z):
            assert o.is_contiguous() and o.shape == t.shape
            o.copy_(t)
        return out

    def linear_attention(self, q, k, v, decay, mat, state=None):
        return tuple((a + b + c).contiguous() for a, b, c in zip(q, k, v)), None


@pytest.mark.parametrize("B,T", [(1, 1), (2, 16384), (1, 65537), (16, 4100)])
def test_prompts_of_any_number_of_rows(B, T):
    g = torch.Generator().manual_seed(T)
    heads, d, width = 2, 3, 5
    w_qkv, w_out = (torch.randint(-8, 8, s, generator=g) for s in ((3 * heads * d, width), (width, heads * d)))
    x = tuple(torch.randint(-1 << 40, 1 << 40, (B, T, width), generator=g) for _ in range(2))
    layer, lane = attention.TokenLayer(heads, d, d, w_qkv, None, w_out, None, 32, None), Plain()
    y, _ = layer.prompt(lane, x, None)
    for s, t in zip(x, y):
        q, k, v = (s @ w_qkv.T).split(heads * d, -1)
        assert torch.equal(t, (q + k + v) @ w_out.T)
    assert sum(lane.rows) == 2 * B * T
