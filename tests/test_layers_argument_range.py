"""Sizes and positions that do not fit the 32-bit fields of adacomp_layers.h are refused, not taken for what is left of them."""
import pytest
import torch

from paper_1712_02679_amd import binding, layers

BEYOND = 2 ** 32


def test_host_calls():
    assert layers.adacomp_bias_softmax_workspace_bytes(1, 2, 3, 8, 128) > 0
    for at in range(5):
        for more in (BEYOND, -BEYOND):
            sizes = [1, 2, 3, 8, 128]
            sizes[at] += more
            assert layers.adacomp_bias_softmax_workspace_bytes(*sizes) == 0, sizes
    assert layers.adacomp_norm_workspace_bytes(-1, 8) == 0 and layers.adacomp_norm_workspace_bytes(4, 2 ** 64 + 8) == 0
    for buckets, far in ((BEYOND + 32, 128), (32, BEYOND + 128), (32 - BEYOND, 128), (32, -5)):
        with pytest.raises(binding.AdacompError):
            layers.adacomp_relative_buckets(buckets, far, False)


@pytest.mark.gpu
def test_calls():
    import paper_1712_02679_amd as A
    dev = "cuda:0"
    table, buckets = torch.zeros(8, 1, device=dev), torch.zeros(9, dtype=torch.int32, device=dev)
    bias, room = A.RelativeBias(table, buckets), torch.zeros(1 << 16, dtype=torch.uint8, device=dev)
    one = torch.zeros(1, 1, 1, 1, device=dev)
    for shape in ((BEYOND, 1, 1, 1), (1, 1, BEYOND, 1)):   # what is left of these sizes is nothing
        s = one.expand(shape)
        with pytest.raises(A.AdacompError):
            A.adacomp_bias_softmax_forward(s, bias, s, room)
        with pytest.raises(A.AdacompError):
            A.adacomp_bias_softmax_backward(s, bias, None, s, s, None, room)
    none = torch.zeros(0, 1, 1, BEYOND + 5, device=dev)
    with pytest.raises(A.AdacompError):
        A.adacomp_bias_softmax_forward(none, bias, none, room)
    for start in (2 ** 31, -2 ** 31 - 1, BEYOND):
        with pytest.raises(A.AdacompError):
            A.adacomp_bias_softmax_forward(one, bias, one.clone(), room, query_start=start)
        with pytest.raises(A.AdacompError):
            A.adacomp_bias_softmax_backward(one, bias, torch.zeros(1, 1, 1, device=dev), one, one.clone(), None, room, query_start=start)
    for start in (2 ** 31 - 1, -2 ** 31):
        A.adacomp_bias_softmax_forward(one, bias, one.clone(), room, query_start=start)
    wide, stat = torch.zeros(0, BEYOND + 8, device=dev), torch.zeros(0, device=dev)
    with pytest.raises(A.AdacompError):
        A.adacomp_norm_forward(wide, None, None, wide)
    with pytest.raises(A.AdacompError):
        A.adacomp_norm_backward(wide, wide, stat, stat, None, wide, None, None, room)
    torch.cuda.synchronize()
