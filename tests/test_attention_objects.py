"""CPU checks of the attention's Python objects: where their arrays lie and
what they refuse before a kernel is called."""
import pytest
import torch

from paper_2605_30876_amd.attention import AttentionLayer, BlockAttention, PagedCache, Rope


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


def test_gradients_are_refused():
    """Nothing is recorded: a tensor that requires a gradient is refused where one would be recorded, and only there."""
    cache = PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu")
    att = BlockAttention(cache, 1, 1, 4, 4)
    att.begin(torch.tensor([0, 4], dtype=torch.int32))
    x = torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    g = x.clone().requires_grad_(True)
    rope, pos = Rope(64, device="cpu"), torch.zeros(4, dtype=torch.int32)
    w = {n: torch.zeros(64, 64, dtype=torch.bfloat16) for n in ("wq", "wk", "wv", "wo")}
    layer, learnt = AttentionLayer(att, 0, w), AttentionLayer(att, 0, {**w, "wv": w["wv"].clone().requires_grad_(True)})
    calls = [lambda t: rope.apply(t, pos), lambda t: rope.apply(x, pos, out=t), lambda t: att.append(0, t, x), lambda t: att.append(0, x, t),
             lambda t: att.append(0, x, x, t), lambda t: att.append(0, x, x, x, t), lambda t: att.attend(0, t), lambda t: att.attend(0, x, t),
             lambda t: layer(t.view(4, 64))]
    for call in calls:
        with pytest.raises(RuntimeError, match="gradient"):
            call(g)
    with pytest.raises(RuntimeError, match="wv requires a gradient"):
        learnt(x.view(4, 64))
    with torch.no_grad():
        for call in calls[:6]:
            with pytest.raises(ValueError, match="GPU"):
                call(g)
