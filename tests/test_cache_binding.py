"""Arguments of the rotary, cache and cache-attention calls that ctypes would cut down
to 32 bits without a word are refused by the binding."""
import pytest
import torch

import paper_2605_31057_amd as L


@pytest.mark.parametrize("heads,n", [(2 ** 32 + 2, 10), (2 ** 31, 1), (2, 2 ** 32 + 1), (1, 2 ** 31)])
def test_sizes_past_32_bits(heads, n):
    # rows of 128 elements at places of their own as far as the binding looks: on a
    # device number -1, the host's
    x = torch.zeros(128, dtype=torch.bfloat16).as_strided((heads, n, 128), (0, 0, 1))
    with pytest.raises(L.LvsaError):
        L._rows(x, -1)


def test_head_dim_past_32_bits():
    x = torch.empty(2 ** 32 + 128, dtype=torch.uint8, device="meta").view(1, 1, -1)
    with pytest.raises(L.LvsaError):
        L._rows(x, x.get_device())


@pytest.mark.parametrize("layout", [-1, 2, 2 ** 32, 2 ** 32 + 1])
def test_layouts(layout):
    with pytest.raises(L.LvsaError):
        L.Rope(3, 4, 5, layout=layout, device="cpu")
