"""cache_attn_shared against plain numpy in 64 bits (tests/cache_case.py)."""
import numpy as np
import pytest

from cache_case import Case, i32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def _requests(rng, groups, own, queries):
    """Lengths and queries of groups (members, prefix)."""
    lens, qs, out, at = [], [], [], 0
    for members, prefix in groups:
        out.append((at, at + members, prefix))
        for _ in range(members):
            q = int(rng.choice(queries))
            lens.append(prefix + q + int(rng.integers(0, own + 1)))
            qs.append(q)
        at += members
    return lens, qs, out


def _case(ra, groups, own=30, queries=(1,), seed=0, Hq=4, Hkv=2, D=128, page=16, **kw):
    lens, qs, gr = _requests(np.random.default_rng(seed), groups, own, queries)
    return Case(ra, Hq, Hkv, D, page, lens, qs, groups=gr, seed=seed, **kw)


@pytest.mark.parametrize("D,page", [(128, 16), (64, 64), (128, 256)])
@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 63, 64, 65, 300, 1024])
@pytest.mark.parametrize("members", [1, 2, 8, 9, 70])
def test_one_group(ra, D, page, prefix, members):
    """2 rows a request: groups of 2 to 140 rows, either kernel, tiles that are not full."""
    c = _case(ra, [(members, prefix)], D=D, page=page, seed=prefix + members, own=70 if members < 70 else 10)
    c.run()
    c.check(True)


@pytest.mark.parametrize("dt,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32"), ("fp16", "fp32"), ("fp16", "bf16")])
@pytest.mark.parametrize("Hq,Hkv", [(12, 12), (5, 1), (40, 8), (20, 1), (48, 1)])
def test_types_and_heads(ra, dt, out, Hq, Hkv):
    c = _case(ra, [(5, 300), (1, 77), (3, 0), (17, 130)], own=200, queries=(1, 1, 0, 3), Hq=Hq, Hkv=Hkv, page=32, dt=dt, out=out,
              rope=True, had=True, vhad=out == "fp32", pad=3, seed=Hq, strided=True)
    c.run()
    c.check(True)


@pytest.mark.parametrize("D,Hq,Hkv,page,dt", [(128, 4, 2, 16, "bf16"), (64, 6, 2, 64, "fp16"), (128, 8, 1, 128, "fp16"),
                                              (64, 3, 3, 32, "bf16")])
@pytest.mark.parametrize("queries", [(1, 2, 5), (40, 1), (0, 130), (0,)])
def test_drafts_and_prompts(ra, D, Hq, Hkv, page, dt, queries):
    c = _case(ra, [(4, 257), (3, 64), (1, 400)], own=150, queries=queries, D=D, Hq=Hq, Hkv=Hkv, page=page, dt=dt, rope=True,
              had=D == 128, vhad=D == 64, pad=2, seed=max(queries))
    c.run()
    c.check(True)


@pytest.mark.parametrize("groups", [[(70, 33)], [(3, 40)] * 40, [(300, 20)], [(2, 17), (1, 0)] * 100])
def test_many_requests_and_groups(ra, groups):
    """More than 64 and more than 256 prefixes and requests."""
    c = _case(ra, groups, own=40, queries=(1, 1, 1, 0, 2), D=64, Hq=4, Hkv=1, rope=True, seed=len(groups), pad=5)
    c.run()
    c.check(True)


@pytest.mark.parametrize("members,queries", [(3, (1,)), (40, (1,)), (5, (30,))])
def test_long_prefixes_are_split(ra, members, queries):
    c = _case(ra, [(members, 9001)], own=300, queries=queries, Hq=2, Hkv=1, page=64, rope=True, seed=members)
    c.run()
    c.check(True)


@pytest.mark.parametrize("cut", [[0, 0], [1, 5], [100, 1], [16, 33], [2 ** 31 - 1, -2 ** 31], [150, 150]])
def test_any_part_of_what_is_shared(ra, cut):
    """Prefixes shorter than what the requests share, none, impossible ones, and one longer than the first request is."""
    c = _case(ra, [(6, 150), (5, 90)], own=40, queries=(1, 4, 0), rope=True, seed=2)
    c.run(prefix=[min(cut[0], 150), min(cut[1], 90)] if max(cut) <= 150 else cut)
    if max(cut) <= 150:
        c.check(True)
    # (2^31 - 1: cut to what the first request holds, which the others do not share; nothing outside is touched)


def test_a_first_request_without_tokens_shares_nothing(ra):
    """The group's table is the first request's: with 0 or few tokens left there, the others read their own."""
    for first in (0, 20):
        c = _case(ra, [(6, 150)], own=40, queries=(1, 2), rope=True, seed=4)
        c.lens[0], c.qs[0] = first, 0
        first_rows = c.start[1]
        c.start = np.concatenate([[0], np.cumsum(c.qs)]).astype(np.int32)
        pos = [n - m + i for n, m in zip(c.lens, c.qs) for i in range(m)]
        c.positions = i32(pos + [-1] * first_rows)
        c.table[0, -(-first // 16):] = -1
        c.run()
        c.check(True)


def test_queries_inside_the_prefix(ra):
    """Requests whose queries begin before the shared tokens end: each sees its own past alone."""
    for q, n in ((30, 40), (100, 100), (5, 45)):
        lens = [n, n + 7, 60]
        c = Case(ra, 4, 2, 128, 16, lens, [min(q, x) for x in lens], groups=[(0, 3, min(lens))], rope=True, seed=q)
        c.run()
        c.check(True)


def test_more_queries_than_tokens(ra):
    c = Case(ra, 4, 2, 64, 16, [3, 20, 20], [7, 25, 2], groups=[(0, 1, 3), (1, 3, 18)], seed=1)
    c.run()
    c.check(True)


def test_large_scores_and_one_side_that_vanishes(ra):
    """Scores of hundreds: of prefix and own keys one side often has no weight left."""
    c = _case(ra, [(20, 300), (3, 200)], own=60, queries=(1, 9), dt="fp16", out="fp32", gain=60.0, seed=5)
    c.run()
    c.check(True)


@pytest.mark.parametrize("dt,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp16"), ("bf16", "fp32")])
@pytest.mark.parametrize("D,had", [(128, True), (64, False)])
@pytest.mark.parametrize("members,prefix,own,queries", [(3, 4, 3, (1,)), (30, 5, 3, (1, 2)), (12, 700, 200, (1, 20))])
def test_lse_is_as_exact_as_binary32_arithmetic(ra, dt, out, D, had, members, prefix, own, queries):
    """Over few keys too, whatever the outputs' type and the kernel."""
    c = _case(ra, [(members, prefix)], own=own, queries=queries, D=D, dt=dt, out=out, rope=True, had=had, seed=members, gain=4.0)
    c.run()
    c.check_lse()


def test_what_a_row_does_not_see_cannot_reach_it(ra):
    """NaN keys and values behind a row, in other requests' own tokens and in places behind the ends."""
    for members, queries in ((5, (3,)), (30, (1,))):
        c = _case(ra, [(members, 100)], own=0, queries=queries, seed=members, pad=4)
        q = queries[0]
        c.q[c.start[-1]:] = float("nan")
        x, lse = (t.clone() for t in c.run())
        r = 2                                  # the last token of one request
        c.scales()[c.table[r, (c.lens[r] - 1) // 16], :, :, (c.lens[r] - 1) % 16] = np.nan
        y, lse2 = c.run()
        sees = np.zeros(c.T, bool)
        sees[c.start[r + 1] - 1] = True
        rest = torch.from_numpy(~sees)
        assert torch.equal(x[rest], y[rest]) and torch.equal(lse[rest], lse2[rest])
        assert torch.isnan(y[~rest]).all() and (y[c.start[-1]:] == 5.0).all()
        # a V of the prefix that is not finite: all rows, not their lse
        c.scales()[c.table[0, 3], :, 1, 2] = np.nan
        z, lse3 = c.run()
        assert torch.isnan(z[:c.start[-1]]).all() and torch.equal(lse3[rest], lse2[rest])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("members,queries", [(3, (1,)), (40, (1,)), (4, (20,))])
def test_queries_that_are_not_finite(ra, D, members, queries):
    """One element of a query: its rows alone are NaN, lse too."""
    for value in (float("nan"), float("inf"), -float("inf")):
        c = _case(ra, [(members, 70)], queries=queries, D=D, seed=members)
        x, lse = (t.clone() for t in c.run())
        hit = torch.zeros(c.T, 4, dtype=torch.bool)
        for t, h, d in ((0, 1, D - 1), (c.T // 2, 3, 5), (c.T - 1, 0, 33)):
            c.q[t, h, d] = value
            hit[t, h] = True
        y, lse2 = c.run()
        assert torch.isnan(y.cpu()[hit]).all() and torch.isnan(lse2.cpu()[hit]).all()
        assert torch.equal(x.cpu()[~hit], y.cpu()[~hit]) and torch.equal(lse.cpu()[~hit], lse2.cpu()[~hit])


@pytest.mark.parametrize("power", [-60, 60])
def test_queries_far_from_one(ra, power):
    """Large queries with small keys and the other way round, rows of zeros among them."""
    for members, queries in ((3, (1,)), (40, (1, 9))):
        c = _case(ra, [(members, 70)], queries=queries, seed=members)
        c.q *= 2.0 ** power
        c.q[0, 1] = 0.0
        c.scales()[:, :, 0] *= 2.0 ** -power
        c.run()
        c.check(True)


def test_pages_that_are_none_are_masked(ra):
    for members in (3, 40):
        c = _case(ra, [(members, 100)], own=50, seed=9)
        c.table[:, 2] = -1
        c.table[:, 4] = c.p.num_pages
        c.run()
        c.check(True)


def test_lengths_that_do_not_fit_touch_nothing_outside(ra):
    """Offsets, groups and lengths of another call: neighbours of outputs and workspace are unharmed."""
    c = _case(ra, [(8, 100), (9, 60)], own=30, queries=(1, 20), seed=12, pad=5)
    p, R, T = c.p, 17, c.T
    cache = torch.from_numpy(c.cache).cuda()
    size = ra.cache_shared_workspace(p, R, 2, T).numel()
    big = torch.full((T + 64, p.Hq, p.D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + 64, p.Hq), 7.0, device="cuda")
    ws = torch.full((size + 4096,), 0x33, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(1)
    bad = np.array([-2 ** 31, -1, 0, 1, 5, 17, 18, 100, 2 ** 31 - 1], np.int64)
    for k in range(20):
        mix = lambda x: np.where(rng.random(len(x)) < 0.4, rng.choice(bad, len(x)), x).astype(np.int32)
        start, lens, gs = mix(c.start), mix(np.array(c.lens)), mix(np.array([0, 8, 17]))
        pre, pos = mix(np.array([100, 60])), mix(c.positions.cpu().numpy())
        if k == 0:
            gs, start = np.array([0, 17, 17], np.int32), c.start       # groups that overlap
            gs[1] = 0
        if k == 1:
            start = np.array([0, T] * 9, np.int32)                     # every second request has all queries
        ra.cache_attn_shared(p, c.q, cache, i32(c.table), i32(start), i32(lens), i32(pos), i32(gs), i32(pre), big[32:32 + T],
                             ws[2048:2048 + size], lse=lse[32:32 + T])
        torch.cuda.synchronize()
        for t in (big, lse):
            assert (t[:32] == 7.0).all() and (t[32 + T:] == 7.0).all(), k
        assert (ws[:2048] == 0x33).all() and (ws[2048 + size:] == 0x33).all(), k


def test_offsets_whose_rows_pass_32_bits(ra):
    """3000 requests that all have all 30 000 queries, after their offsets: 4.3e9 rows."""
    R, T = 6000, 30000
    p = ra.make_cache_params(48, 1, 64, page_size=16, num_pages=8, max_blocks=4)
    cache = torch.zeros(8, ra.cache_layout(p)["page_bytes"], dtype=torch.uint8, device="cuda")
    q = torch.zeros(T, 48, 64, dtype=torch.bfloat16, device="cuda")
    size = ra.cache_shared_workspace(p, R, 1, T, device="meta").numel()
    o = torch.full((T + 64, 48, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((size + 4096,), 0x33, dtype=torch.uint8, device="cuda")
    start = np.array([0, T] * (R // 2) + [0])
    ra.cache_attn_shared(p, q, cache, i32(np.zeros((R, 4))), i32(start), i32(np.full(R, 60)), i32(np.zeros(T)), i32([0, R]),
                         i32([20]), o[32:32 + T], ws[2048:2048 + size])
    torch.cuda.synchronize()
    assert (o[:32] == 7.0).all() and (o[32 + T:] == 7.0).all()
    assert (ws[:2048] == 0x33).all() and (ws[2048 + size:] == 0x33).all()


def test_equals_cache_attn_within_roundings(ra):
    c = _case(ra, [(12, 500)], own=100, queries=(1, 2), dt="bf16", out="fp32", rope=True, seed=6)
    x, lse = (t.clone() for t in c.run())
    groups, c.groups = c.groups, []
    y, lse2 = c.run()
    # either is within the bounds of 64-bit results; of each other within twice binary32's
    assert (x - y).abs().max() <= 2.0 ** -17 * y.abs().max() and (lse - lse2).abs().max() <= 2.0 ** -17


def test_repeats_streams_and_used_workspaces(ra):
    c = _case(ra, [(12, 500), (3, 700)], own=300, queries=(1, 2, 30), rope=True, seed=7)
    x, lse = (t.clone() for t in c.run())
    ws = ra.cache_shared_workspace(c.p, len(c.lens), 2, c.T)
    ws.fill_(0xFF)                                # NaN wherever it is read before it is written
    y, lse2 = c.run(ws=ws)
    assert torch.equal(x, y) and torch.equal(lse, lse2)
    side = torch.cuda.Stream()
    y, lse2 = c.run(ws=ws, stream=side.cuda_stream)
    assert torch.equal(x, y) and torch.equal(lse, lse2)


def test_fork_then_attend_captured(ra):
    """A prompt is cached once, forked, and the continuations decode on their own pages and the shared prefix: plan,
    append and shared attention in one graph, replayed step after step, equal the eager calls of another server."""
    p = ra.make_cache_params(6, 2, 128, page_size=16, num_pages=120, max_blocks=12, out_dtype=ra.FP32)
    R, T, D = 6, 110, 128
    import cache_ref as ref
    rope = torch.from_numpy(ref.rope_table(12 * 16, D)).cuda()
    rng = np.random.default_rng(5)

    def make():
        st = ra.alloc_cache(p, R)
        st["cache"].zero_()
        buf = {n: torch.zeros(m, dtype=torch.int32, device="cuda")
               for n, m in (("q_start", R + 1), ("positions", T), ("slots", T), ("status", 4), ("new", R), ("gs", 2), ("pre", 1))}
        x = torch.zeros(T, 10, D, dtype=torch.bfloat16, device="cuda")
        o, lse = torch.zeros(T, 6, D, device="cuda"), torch.zeros(T, 6, device="cuda")
        return st, buf, x, o, lse, ra.cache_shared_workspace(p, R, 1, T), ra.cache_pages_workspace(p, R)

    def step(s):
        st, b, x, o, lse, ws, _ = s
        ra.cache_plan(p, st["seq_lens"], b["new"], st["block_table"], st["free_pages"], st["free_count"], b["q_start"],
                      b["positions"], b["slots"], b["status"])
        ra.cache_append(p, x[:, 6:8], x[:, 8:], b["slots"], st["cache"], positions=b["positions"], rope=rope)
        ra.cache_attn_shared(p, x[:, :6], st["cache"], st["block_table"], b["q_start"], st["seq_lens"], b["positions"], b["gs"],
                             b["pre"], o, ws, lse=lse, rope=rope)

    a, b = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(a)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for k in range(7):
        new = [100, 0, 0, 0, 0, 3] if k == 0 else rng.integers(0, 3, R).tolist()
        x = torch.tensor(rng.standard_normal((T, 10, D))).to(torch.bfloat16).cuda()
        for s in (a, b):
            s[1]["new"].copy_(i32(new))
            s[1]["gs"].copy_(i32([0, 5]))
            s[1]["pre"].copy_(i32([0 if k == 0 else 100]))
            s[2].copy_(x)
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        assert torch.equal(a[3], b[3]) and torch.equal(a[4], b[4]), k
        assert torch.equal(a[0]["cache"], b[0]["cache"])
        # what cache_attn makes of the same step (binary32 outputs)
        st, buf = b[0], b[1]
        o, lse = torch.zeros_like(b[3]), torch.zeros_like(b[4])
        ra.cache_attn(p, b[2][:, :6], st["cache"], st["block_table"], buf["q_start"], st["seq_lens"], T, o,
                      ra.cache_workspace(p, R, T, T), lse=lse, rope=rope)
        n = int(buf["q_start"][-1])
        assert (o[:n] - b[3][:n]).abs().max() <= 2.0 ** -17 * max(1.0, o[:n].abs().max().item()) if n else True
        if k == 0:
            for s in (a, b):
                st = s[0]
                ra.cache_fork(p, i32([0, 0, 0, 0]), i32([1, 2, 3, 4]), st["seq_lens"], st["block_table"], st["page_refs"],
                              st["free_pages"], st["free_count"], st["cache"], s[6], s[1]["status"])
                assert s[1]["status"].tolist()[:3] == [0, 4, 24]


def _regroup(c, starts, prefix, got=None):
    """The case's call with these groups."""
    ra, R = c.ra, len(c.lens)
    c.fresh()
    ws = ra.cache_shared_workspace(c.p, R, len(prefix), c.T)
    ra.cache_attn_shared(c.p, c.q, torch.from_numpy(c.cache).cuda(), i32(c.table), i32(c.start), i32(c.lens), c.positions,
                         i32(starts), i32(prefix), c.o, ws, lse=c.lse, rope=c.rope())
    torch.cuda.synchronize()


def test_no_groups_and_empty_ones(ra):
    c = _case(ra, [(5, 70), (4, 33)], own=60, queries=(1, 3, 20), rope=True, seed=21, pad=2)
    for starts, prefix in (([0], []), ([0, 0, 5, 5, 9], [7, 70, 50, 33]), ([0, 5, 9, 9, 9], [70, 33, 1, 2]), ([2, 5], [70]),
                           ([0, 0, 0], [5, 5]), ([9, 9], [3])):
        _regroup(c, starts, prefix)
        c.check(True)


def test_rows_before_the_first_request(ra):
    """q_start need not begin at 0: rows before it are left as they were."""
    c = _case(ra, [(6, 100), (3, 40)], own=50, queries=(1, 2), rope=True, seed=22)
    want = c.want()
    shift, T = 7, c.T
    c.start = c.start + shift
    c.q = torch.cat((torch.full_like(c.q[:shift], float("nan")), c.q))
    c.positions = torch.cat((c.positions.new_full((shift,), -1), c.positions))
    c.T = T + shift
    c.run()
    assert (c.o[:shift] == 5.0).all() and (c.lse[:shift] == 5.0).all()
    c.check(True, got=(c.o[shift:], c.lse[shift:]), want=want)


@pytest.mark.parametrize("R,groups", [(700, 600), (5000, 300), (3000, 2900)])
def test_thousands_of_requests_and_groups(ra, R, groups):
    """More prefixes and requests than their lengths, or their tiles, are kept of in one place."""
    rng = np.random.default_rng(R)
    page, n = 16, 24                                   # all hold the same two pages' worth of tokens, 20 shared
    qs = [int(x) for x in rng.choice([0, 1, 1, 2], R)]
    lens = [n] * R
    cuts = np.sort(rng.choice(np.arange(1, R), groups - 1, replace=False)).tolist()
    c = Case(ra, 2, 1, 64, page, [n] * 8, [q for q in [1] * 8], seed=R)
    c.lens, c.qs = lens, qs
    c.table = np.repeat(c.table[:1], R, 0)
    c.start = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
    c.T = int(c.start[-1])
    c.q = torch.tensor(rng.standard_normal((c.T, 2, 64))).to(torch.bfloat16).cuda()
    c.positions = i32([n - m + i for m in qs for i in range(m)])
    _regroup(c, [0] + cuts + [R], rng.integers(0, 21, groups).tolist())
    # every request has the same keys
    r = [i for i in range(R) if qs[i] == 1][:40] + [i for i in range(R) if qs[i] == 2][-40:]
    o, lse = c.o, c.lse
    pick = np.concatenate([np.arange(c.start[i], c.start[i + 1]) for i in r])
    d = Case(ra, 2, 1, 64, page, [n] * 8, [1] * 8, seed=R)
    d.lens, d.qs = [n] * len(r), [qs[i] for i in r]
    d.table = c.table[:len(r)]
    d.start = np.concatenate([[0], np.cumsum(d.qs)]).astype(np.int32)
    d.T, d.q = len(pick), c.q[torch.from_numpy(pick).cuda()]
    where = torch.from_numpy(pick).cuda()
    d.check(True, got=(o[where], lse[where]))
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_more_heads_than_places(ra):
    c = _case(ra, [(3, 100), (20, 70)], own=30, queries=(1, 2), Hq=600, Hkv=600, D=64, seed=23)
    c.run()
    c.check(True)


def test_two_calls_on_two_streams(ra):
    """Calls with workspaces of their own do not meet."""
    a = _case(ra, [(12, 900), (3, 700)], own=300, queries=(1, 2, 30), rope=True, seed=7)
    b = _case(ra, [(30, 500)], own=100, queries=(1,), rope=True, seed=8)
    want = [[t.clone() for t in c.run()] for c in (a, b)]
    args = []
    for c in (a, b):
        starts = [g[0] for g in c.groups] + [c.groups[-1][1]]
        ws = ra.cache_shared_workspace(c.p, len(c.lens), len(c.groups), c.T)
        args.append((c.p, c.q, torch.from_numpy(c.cache).cuda(), i32(c.table), i32(c.start), i32(c.lens), c.positions, i32(starts),
                     i32([g[2] for g in c.groups]), c.o, ws, c.lse, c.rope()))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, x, s in zip((a, b), args, streams):
            with torch.cuda.stream(s):
                c.o.zero_()
                ra.cache_attn_shared(*x[:-2], lse=x[-2], rope=x[-1])
    torch.cuda.synchronize()
    for c, w in zip((a, b), want):
        assert torch.equal(c.o, w[0]) and torch.equal(c.lse, w[1])
