"""The binding takes caches whatever distance stands for an axis of one element (no GPU
needed: shapes and distances are looked at before anything else)."""
import pytest

from paper_2310_07177_amd import binding


def args(k, v, layers=0):
    import torch
    i32 = dict(dtype=torch.int32)
    return binding._cache_args(k, v, torch.zeros(2, 3, **i32), torch.zeros(2, **i32), layers)


def test_one_kv_head_behind_the_page():
    """[pages, page_size, 1, D] seen as [pages, 1, page_size, D]: a page is contiguous."""
    import torch
    k, v = (torch.zeros(4, 16, 1, 64).transpose(1, 2) for _ in range(2))
    assert k.stride() == (1024, 64, 64, 1)
    assert args(k, v) == (2, 3, 1024, 4, 1, 16, 64, binding.OSD_F32)
    assert args(k, torch.zeros(4, 1, 16, 64)) == args(k, v)


def test_pages_of_one_token():
    import torch
    k, v = (torch.zeros(4, 1, 3, 64).transpose(1, 2) for _ in range(2))
    assert k.shape == (4, 3, 1, 64) and k.stride(2) == 192
    assert args(k, v) == (2, 3, 192, 4, 3, 1, 64, binding.OSD_F32)


def test_one_page():
    """The distance between pages is a page's where there is one alone."""
    import torch
    k = torch.zeros(2 * 16 * 64).as_strided((1, 2, 16, 64), (8, 1024, 64, 1))
    assert args(k, k) == (2, 3, 2048, 1, 2, 16, 64, binding.OSD_F32)
    assert args(k, torch.zeros(1, 2, 16, 64))[2] == 2048


def test_distances_that_matter_are_still_looked_at():
    import torch
    x = torch.zeros(4, 2, 16, 64)
    for k, v in ((x.transpose(1, 2).contiguous().transpose(1, 2), x), (x[..., ::2], x[..., ::2]), (x[:, :, ::2], x[:, :, ::2]),
                 (x, torch.zeros(4, 2, 2, 16, 64)[:, 0])):
        with pytest.raises(ValueError):
            args(k, v)
    layers = torch.zeros(3, 4, 2, 16, 64)
    with pytest.raises(ValueError):
        args(layers, torch.zeros(4, 3, 2, 16, 64).transpose(0, 1), 1)
    assert args(layers, layers.clone(), 1)[2] == 2048
