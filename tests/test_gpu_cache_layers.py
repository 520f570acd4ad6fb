"""The caches of a model's layers have one set of tables: fork, trim and compact move each layer's bytes from the same old
tables into arrays of their own, which come out the same every time."""
import random

import numpy as np
import pytest

import cache_pages_ref as ref
from test_gpu_cache_pages import Cache, _i32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def test_one_set_of_tables_for_all_layers(ra):
    rng = random.Random(6)
    page, blocks, pages, layers = 16, 6, 90, 3
    c = Cache(ra, rng, 12, page, blocks, pages, 2, 64, lens=[0, 40, 0, 33, 0, 96, 70, 0, 90, 15, 0, 77], window=30)
    g = np.random.default_rng(2)
    bytes_ = [g.integers(0, 256, c.bytes.shape, dtype=np.uint8) for _ in range(layers)]
    caches = [torch.from_numpy(b).cuda() for b in bytes_]
    names = ("seq_lens", "block_table", "page_refs", "free_pages", "free_count")
    old = dict(c.t)
    new = {k: torch.empty_like(v) for k, v in old.items()}
    outs = ("seq_out", "table_out", "refs_out", "free_out", "count_out")
    state = c.state
    keep = [-1, 20, 35, -1, 3, 96, 50, 0, 81, 0, -1, 66]
    for name, args, kw, step in (
            ("cache_fork", (_i32([1, 5, 5, 8]), _i32([0, 2, 4, 10])), {}, lambda s: ref.fork(s, page, blocks, [1, 5, 5, 8], [0, 2, 4, 10])),
            ("cache_trim", (), dict(keep=_i32(keep), sinks=7), lambda s: ref.trim(s, page, blocks, 30, keep, 7)),
            ("cache_compact", (), {}, lambda s: ref.compact(s, page, blocks))):
        state, status = step(state)
        assert status[0] == 0 and status[1] > 0          # bytes are to be moved in each layer
        for cache in caches:
            for v in new.values():
                v.fill_(-77)
            getattr(ra, name)(c.p, *args, *(old[k] for k in names), cache, c.ws, c.status, **kw,
                              **{o: new[k] for o, k in zip(outs, names)})
            torch.cuda.synchronize()
            assert c.status.tolist() == status
            assert new["seq_lens"].tolist() == state["seq"] and new["block_table"].tolist() == state["table"]
            assert new["page_refs"].tolist() == state["refs"] and new["free_pages"].tolist() == state["free"]
            assert new["free_count"].item() == state["count"]
        for cache, b in zip(caches, bytes_):
            assert np.array_equal(cache.cpu().numpy(), b[state["cache"]]), name
        old, new = new, old
