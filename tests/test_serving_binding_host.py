"""What the binding of the operators around a round refuses before it looks at the device."""

import pytest
import torch


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def tables():
    flat = torch.arange(12, dtype=torch.int32)
    return {"expanded": flat[:4].expand(3, -1), "overlapping": flat.as_strided((3, 4), (2, 1)), "transposed": flat.view(4, 3).T,
            "of one row apart by less": flat.as_strided((2, 4), (3, 1))}


@pytest.mark.parametrize("name", tables())
def test_tables_whose_rows_share_storage(rt, name):
    """The kernels take row b to begin max_pages entries after row b - 1 at least."""
    k = torch.zeros((12, 8, 2, 16))
    with pytest.raises(ValueError, match="page_table"):
        rt.KvCache(k, k.clone(), tables()[name])


def test_other_tables_get_as_far_as_the_device(rt):
    flat, k = torch.arange(12, dtype=torch.int32), torch.zeros((12, 8, 2, 16))
    for table in (flat.view(3, 4), flat.as_strided((2, 3), (6, 1)), flat[:4].expand(1, -1), flat.as_strided((1, 4), (0, 1)), flat.view(12, 1)[:, :0]):
        with pytest.raises(ValueError, match="CUDA"):
            rt.KvCache(k, k.clone(), table)
