"""The dealer's batched products on a stand-in for the lane.  No GPU."""
import pytest
import torch

from paper_2209_13643_amd import dealer


class Plain:
    """A lane whose ring products take the library's most matrices."""

    def wait_torch(self):
        pass

    def sync(self):
        pass

    def ring_matmul(self, left, right):
        if 2 * left.shape[0] > 65535:
            raise ValueError("too many matrices")
        return left @ right


@pytest.mark.parametrize("lead", [(1,), (3, 5), (32767,), (32768,), (2, 40000), (70000,)])
def test_ring_products_of_any_number_of_matrices(lead):
    g = torch.Generator().manual_seed(1)
    a, b = (torch.randint(-1 << 62, 1 << 62, (*lead, *s), generator=g) for s in ((2, 3), (3, 1)))
    z = dealer._ring_product(Plain(), a, b)
    assert z.shape == (*lead, 2, 1) and torch.equal(z, a @ b)


def test_copies_of_the_operands_are_waited_for():
    """Operands that are not dense are copied by torch: the lane waits for it behind that."""
    order = []

    class Watched(Plain):
        def wait_torch(self):
            order.append("wait")

    class Strided(torch.Tensor):
        @classmethod
        def __torch_function__(cls, func, types, args=(), kwargs=None):
            if func is torch.Tensor.reshape:
                order.append("copy")
            return super().__torch_function__(func, types, args, kwargs or {})
    a = torch.arange(12).view(2, 3, 2).transpose(1, 2).as_subclass(Strided)
    dealer._ring_product(Watched(), a, a.transpose(1, 2))
    assert order.index("wait") > max(i for i, o in enumerate(order) if o == "copy")
