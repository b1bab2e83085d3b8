"""CPU checks of the attention's Python objects: where their arrays lie and
what they refuse before a kernel is called."""
import pytest
import torch

from paper_2605_30876_amd.attention import PagedCache


def _pool(device="cpu"):
    return torch.zeros(1, 2, 32 * 64, dtype=torch.bfloat16, device=device)


@pytest.mark.parametrize("given", ["k", "v", "table", "lens", "refs"])
def test_new_arrays_lie_where_the_given_ones_do(given):
    """A cache over existing arrays of another device than the default: a kernel would follow the others' addresses."""
    array = {"k": _pool(), "v": _pool(), "table": torch.full((1, 1), -1, dtype=torch.int32), "lens": torch.zeros(1, dtype=torch.int32),
             "refs": torch.zeros(2, dtype=torch.int32)}[given]
    c = PagedCache(1, 2, 32, 1, 64, 1, 1, device="meta", **{given: array})
    assert {t.device.type for t in (c.k, c.v, c.table, c.lens, c.refs, c.status, *c._ws)} == {"cpu"} and c.device.type == "cpu"


@pytest.mark.parametrize("name", ["v", "table", "lens", "refs"])
def test_arrays_of_two_devices_are_refused(name):
    array = {"v": _pool("meta"), "table": torch.full((1, 1), -1, dtype=torch.int32, device="meta"),
             "lens": torch.zeros(1, dtype=torch.int32, device="meta"), "refs": torch.zeros(2, dtype=torch.int32, device="meta")}[name]
    with pytest.raises(ValueError):
        PagedCache(1, 2, 32, 1, 64, 1, 1, device="meta", k=_pool(), **{name: array})


def test_a_cache_remembers_refusals():
    c = PagedCache(1, 2, 32, 1, 64, 3, 1, device="cpu")
    assert c.refused.tolist() == [0, 0, 0] and c.c.refused == c.refused.data_ptr()
