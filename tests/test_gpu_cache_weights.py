"""cache_attn_sinks and cache_attn_shared with bf16 outputs: how many bf16 values hold the weights times V's scales goes by
a request's own rows (queries * Hq, up to 512: two), not by the call's room or by the other requests."""
import numpy as np
import pytest

from cache_case import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


HEADS = [(32, 8, 128, True), (32, 8, 64, False), (24, 8, 128, False), (40, 1, 128, True)]   # Hq, Hkv, D, rotated


@pytest.mark.parametrize("Hq,Hkv,D,had", HEADS)
@pytest.mark.parametrize("pad", [5, 700])
def test_room_for_more_rows_changes_no_bits(ra, Hq, Hkv, D, had, pad):
    """The same queries in a call with room for others, as a captured graph has it."""
    q = 512 // Hq - 1
    for kw in (dict(window=200, sinks=9), dict(groups=[(0, 2, 250)])):
        got = []
        for extra in (0, pad):
            c = Case(ra, Hq, Hkv, D, 32, [600, 300], [q // 2, q - q // 2], rope=True, had=had, pad=extra, seed=Hq + D, **kw)
            o, lse = c.run()
            got.append((o[:q].clone(), lse[:q].clone()))
            c.check(False)
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]), kw


@pytest.mark.parametrize("Hq,Hkv,D,had", HEADS)
def test_company_takes_no_precision(ra, Hq, Hkv, D, had):
    """Thirty requests of up to 512 rows each, and one of many more beside them, whose own rows may have one value."""
    q = 512 // Hq
    for qs in ([q] * 30, [q] * 30 + [700]):
        c = Case(ra, Hq, Hkv, D, 32, [200] * 30 + [900] * (len(qs) - 30), qs, rope=True, had=had, window=100, sinks=9, seed=Hq)
        o, lse = c.run()
        n = c.start[30]
        want = [x[:n] for x in c.want()]
        c.check(False, got=(o[:n], lse[:n]), want=want)
        c.check(len(qs) > 30)


@pytest.mark.parametrize("Hq,Hkv,D,had", HEADS)
@pytest.mark.parametrize("members,queries", [(64, 1), (17, 3), (5, 12)])
def test_prefixes_of_many_requests(ra, Hq, Hkv, D, had, members, queries):
    """A decode step, or drafts, on one prefix: its rows are those of all the requests."""
    c = Case(ra, Hq, Hkv, D, 64, [700 + 3 * i for i in range(members)], [queries] * members, groups=[(0, members, 650)],
             rope=True, had=had, seed=members)
    c.run()
    c.check(False)


def test_groups_of_small_and_of_large_requests(ra):
    """One value only where every request of the group that has queries has more than 512 rows."""
    lens, qs = [400, 500, 520, 300, 900, 800, 300, 950], [0, 100, 120, 0, 200, 1, 30, 300]
    c = Case(ra, 32, 8, 128, 64, lens, qs, groups=[(0, 3, 300), (3, 6, 250), (6, 8, 200)], rope=True, had=True, seed=3)
    o, lse = c.run()
    want = c.want()
    c.check(True)
    s = c.start
    for r in (5,):   # one query in a group with 200 others
        c.check(False, got=(o[s[r]:s[r + 1]], lse[s[r]:s[r + 1]]), want=[x[s[r]:s[r + 1]] for x in want])


def test_requests_of_many_rows_may_have_one(ra):
    """More than 512 rows: half a step of bf16 for each weight, as in cache_attn, with room for more or without."""
    got = []
    for pad in (0, 300):
        c = Case(ra, 32, 8, 128, 64, [900, 400], [300, 17], rope=True, had=True, window=300, sinks=9, seed=4, pad=pad)
        o, lse = c.run()
        c.check(True)
        got.append((o[:317].clone(), lse[:317].clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_more_groups_than_are_kept_of(ra):
    """5000 groups of two requests of few queries."""
    rng = np.random.default_rng(1)
    R, n = 10000, 40
    c = Case(ra, 8, 1, 64, 16, [n] * 8, [3] * 8, seed=1)
    from cache_case import i32
    qs = [3] * R
    c.lens, c.qs = [n] * R, qs
    c.table = np.repeat(c.table[:1], R, 0)
    c.start = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
    c.T = int(c.start[-1])
    c.q = torch.tensor(rng.standard_normal((c.T, 8, 64))).to(torch.bfloat16).cuda()
    c.positions = i32([n - m + i for m in qs for i in range(m)])
    c.fresh()
    ws = ra.cache_shared_workspace(c.p, R, R // 2, c.T)
    ra.cache_attn_shared(c.p, c.q, torch.from_numpy(c.cache).cuda(), i32(c.table), i32(c.start), i32(c.lens), c.positions,
                         i32(np.arange(0, R + 1, 2)), i32(np.full(R // 2, 33)), c.o, ws, lse=c.lse)
    torch.cuda.synchronize()
    # all have the same keys: every 500th one
    pick = np.concatenate([np.arange(c.start[r], c.start[r + 1]) for r in range(0, R, 500)])
    where = torch.from_numpy(pick).cuda()
    d = Case(ra, 8, 1, 64, 16, [n] * 8, [3] * 8, seed=1)
    d.lens, d.qs, d.table = [n] * 20, [3] * 20, c.table[:20]
    d.start, d.T, d.q = np.arange(0, 61, 3).astype(np.int32), 60, c.q[where]
    d.check(False, got=(c.o[where], c.lse[where]))
    assert torch.isfinite(c.o).all()
