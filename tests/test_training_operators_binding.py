"""What the binding of the training operators takes as tensors of the same order (no GPU)."""
import torch

from paper_2301_08527_b200 import binding


def test_order_of_values():
    same, a = binding._same_order, torch.empty
    strided = torch.empty_strided
    assert same(a(6, 8), a(48)) and same(a(6, 8), a(8, 6)) and same(a(0, 3), a(0))
    assert same(a(6, 8).t(), strided((8, 6), (1, 8)))
    # one value along a dimension: its stride tells nothing
    assert same(strided((5, 1, 6), (1, 777, 5)), strided((5, 1, 6), (1, 5, 5)))
    assert not same(a(6, 8).t(), a(8, 6)) and not same(a(8, 6), a(6, 8).t()) and not same(a(6, 8).t(), a(6, 8)) and not same(a(6, 8).t(), a(48))
    assert not same(strided((2, 3, 4), (1, 8, 2)), strided((2, 3, 4), (12, 4, 1)))


def test_a_list_is_refused_for_the_pair_that_differs_alone():
    # each pair by itself: a transposed gradient beside a contiguous one that goes to a flat buffer
    grads = [torch.empty(6, 8).t(), torch.empty(6, 8)]
    assert all(map(binding._same_order, grads, [torch.empty(6, 8).t(), torch.empty(48)]))
    assert not all(map(binding._same_order, grads, [torch.empty(8, 6), torch.empty(48)]))
