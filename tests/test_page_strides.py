"""Strides of the pages' tensors that the paged operators take (no GPU needed)."""
import pytest
import torch

from paper_2607_21927_amd import serve


def pages(shape, strides):
    return torch.zeros(100_000, dtype=torch.bfloat16).as_strided(shape, strides)


@pytest.mark.parametrize("shape,k,v", [
    ((1, 2, 16, 64), (2048, 1024, 64, 1), (4096, 1024, 64, 1)),      # one page: no stride between pages
    ((3, 1, 16, 64), (1024, 1024, 64, 1), (1024, 7, 64, 1)),         # one KV head
    ((3, 2, 1, 64), (128, 64, 64, 1), (128, 64, 9, 1)),              # pages of one token
])
def test_dimensions_of_one_element_have_any_stride(shape, k, v):
    Kp, Vp = pages(shape, k), pages(shape, v)
    assert serve._need_pages(Kp, Vp) == shape == serve._need_pages(Vp, Kp)
    table = torch.zeros(2, 3, dtype=torch.int32)
    a, b = serve._page_map(Kp, table), serve._page_map(Vp, table)
    assert (a.page_stride, a.pages, a.page) == (b.page_stride, b.pages, b.page)


def test_other_strides_are_refused():
    Kp = pages((3, 2, 16, 64), (2048, 1024, 64, 1))
    for v in ((4096, 1024, 64, 1), (2048, 1088, 64, 1), (2048, 1024, 128, 1)):
        with pytest.raises(ValueError, match="strides"):
            serve._need_pages(Kp, pages((3, 2, 16, 64), v))
