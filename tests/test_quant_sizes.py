"""What the size functions of the attention tell is enough for every cache and batch: drawn widely, on the CPU."""
import ctypes
import random

import pytest
import torch

from paper_2605_30876_amd import lib
from test_quant_abi import BAD, NO, batch, cache, p, status  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation tests run without a GPU")


@pytest.mark.parametrize("seed", range(4))
def test_sizes_told_are_enough(p, seed):  # noqa: F811
    L, r, wrong = lib.load(), random.Random(seed), []
    log = lambda hi: int(2 ** r.uniform(0, hi))  # noqa: E731
    for _ in range(1000):
        kv, group = r.choice([1, 1, 2, 3, 4, 8, 32, 128, 256]), r.choice([1, 1, 2, 3, 4, 8, 33, 200, 1024])
        seqs, new = log(12), log(16)
        T, heads, dim = max(1, min(seqs * new, r.choice([log(22), 1 << 24]), (1 << 30) // (group * kv))), group * kv, r.choice([8, 64, 96, 128, 192, 256])
        page, dt = r.choice([32, 64, 160, 1024]), r.choice([lib.DMOE_F32, lib.DMOE_BF16])
        b = batch(p, n_seqs=seqs, T=T, max_new=new)
        ints = L.dmoe_attention_plan_ints(seqs, T, new, heads, kv)
        ws = L.dmoe_attention_workspace_size(dt, seqs, T, new, heads, kv, dim)
        out = p + T * heads * dim * 4  # behind the queries
        pages = max(1, log(30) // page)
        for fmt in sorted(lib.KV_FORMAT.values()):
            c = cache(p, format=fmt, dt=dt, n_kv_heads=kv, head_dim=dim, n_slots=seqs, page_tokens=page, max_pages=pages)
            got = [status(L, "dmoe_attention_plan", ctypes.byref(c), b, heads, 32, p, ints, None),
                   status(L, "dmoe_attention", ctypes.byref(c), 0, b, heads, 32, p, heads * dim, 1.0, p, ints, out, heads * dim, None, p, ws, None)]
            wrong += [(fmt, seqs, T, new, group, kv, dim, page, pages, L.dmoe_last_error().decode())] if BAD in got or NO in got else []
    assert not wrong, wrong[:3]
