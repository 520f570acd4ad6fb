"""Fork, trim and compact with some tables in place and others in arrays of their own, and with very many requests."""
import random

import numpy as np
import pytest

import cache_pages_ref as ref
from test_gpu_cache_pages import Cache, _i32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

OUTS = {"seq_lens": "seq_out", "block_table": "table_out", "page_refs": "refs_out", "free_pages": "free_out", "free_count": "count_out"}


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def _call(c, name, own, *args, **kw):
    """The tables that the call leaves; those of `own` in arrays of their own, whose inputs stay."""
    out = {k: torch.full_like(v, -77) if k in own else v for k, v in c.t.items()}
    before = {k: c.t[k].clone() for k in own}
    getattr(c.ra, name)(c.p, *args, *c.t.values(), c.cache, c.ws, c.status, **{OUTS[k]: out[k] for k in own}, **kw)
    torch.cuda.synchronize()
    for k, v in before.items():
        assert torch.equal(v, c.t[k]), f"{k} was an input"
    return out


@pytest.mark.parametrize("mask", range(1, 31))
def test_any_tables_in_place(ra, mask):
    rng = random.Random(mask)
    own = [k for i, k in enumerate(OUTS) if mask >> i & 1]
    R, page, blocks, pages = 40, 16, 6, 400
    lens = [0 if rng.random() < 0.4 else rng.randint(1, blocks * page) for _ in range(R)]
    children = [r for r in range(R) if lens[r] == 0]
    parents = [rng.randrange(R) for _ in children]
    cut = [rng.randint(0, lens[a]) for a in parents]
    c = Cache(ra, rng, R, page, blocks, pages, lens=lens, share=0.4, window=20)
    state, status = ref.fork(c.state, page, blocks, parents, children, cut)
    c.check(_call(c, "cache_fork", own, _i32(parents), _i32(children), lens=_i32(cut)), state, status)
    c.state = state
    c.upload()
    keep = [rng.choice([-1, 0, n, rng.randint(0, n)]) for n in state["seq"]]
    state, status = ref.trim(state, page, blocks, 20, keep, 5)
    c.check(_call(c, "cache_trim", own, keep=_i32(keep), sinks=5), state, status)
    c.state = state
    c.upload()
    state, status = ref.compact(state, page, blocks)
    c.check(_call(c, "cache_compact", own), state, status)
    # refused: all of it as it was, in whichever array
    c.state = dict(state, count=pages + 1)
    for name, args in (("cache_fork", (_i32([0]), _i32([0]))), ("cache_trim", ()), ("cache_compact", ())):
        c.upload()
        out = _call(c, name, own, *args)
        assert c.status[0].item() & 8
        c.check(out, c.state, c.status[0].item())


@pytest.mark.parametrize("R", [30000, 65536])
def test_very_many_requests(ra, R):
    rng = random.Random(R)
    page, blocks = 16, 3
    lens = [0 if r % 2 else rng.randint(0, 40) for r in range(R)]
    c = Cache(ra, rng, R, page, blocks, 3 * R + 100, lens=lens)
    children = list(range(1, R, 2))
    rng.shuffle(children)
    parents = [rng.randrange(0, R, 2) for _ in children]
    state, status = ref.fork(dict(c.state), page, blocks, parents[:3000], children[:3000])
    c.check(c.call("cache_fork", _i32(parents[:3000]), _i32(children[:3000])), state, status)
    c.state = state
    keep = [rng.choice([-1, 0, rng.randint(0, n)]) for n in state["seq"]]
    state, status = ref.trim(state, page, blocks, 0, keep)
    c.check(c.call("cache_trim", keep=_i32(keep)), state, status)
