"""The 4-bit paged KV cache against plain numpy in 64 bits (tests/cache_ref.py)."""
import numpy as np
import pytest

import cache_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# half a step relative to the value
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def _kind(ra, name):
    return {"bf16": ra.BF16, "fp16": ra.FP16, "fp32": ra.FP32}[name]


def _params(ra, Hq, Hkv, D, page, pages, blocks, had=False, vhad=False, dt="bf16", out=None, **kw):
    return ra.make_cache_params(Hq, Hkv, D, page_size=page, num_pages=pages, max_blocks=blocks,
                                rotation=ra.ROT_HADAMARD if had else ra.ROT_NONE,
                                v_rotation=ra.VROT_HADAMARD if vhad else ra.VROT_NONE, in_dtype=_kind(ra, dt),
                                out_dtype=_kind(ra, out or dt), **kw)


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _f64(t):
    return t.detach().cpu().double().numpy()


# ------------------------------------------------------------------- read --

@pytest.mark.parametrize("D,page,out", [(128, 16, "fp32"), (64, 32, "fp32"), (128, 256, "bf16"), (64, 16, "fp16")])
def test_read_every_code_of_every_place(ra, D, page, out):
    """Random page bytes: every byte value comes up, and every value is the code's."""
    rng = np.random.default_rng(1)
    Hkv, pages = 3, 5
    p = _params(ra, 6, Hkv, D, page, pages, pages, out=out)
    cache = rng.integers(0, 256, (pages, ra.cache_layout(p)["page_bytes"]), dtype=np.uint8)
    view = cache.reshape(pages, Hkv, -1)
    view[:, :, page * D:] = rng.uniform(0.1, 9.0, (pages, Hkv, 2 * page)).astype(np.float32).view(np.uint8).reshape(pages, Hkv, -1)
    slots = np.concatenate([rng.permutation(pages * page), [-1, pages * page, 5, 5, -2 ** 31, 2 ** 31 - 1]]).astype(np.int32)
    k, v = (torch.full((len(slots), Hkv, D), 7.0, dtype=DT[out], device="cuda") for _ in range(2))
    ra.cache_read(p, torch.from_numpy(cache).cuda(), _i32(slots), k, v)
    ok = (slots >= 0) & (slots < pages * page)
    kc, ks, vc, vs = ref.rows(cache, np.where(ok, slots, 0), page, Hkv, D)
    for got, c, s in ((k, kc, ks), (v, vc, vs)):
        want = np.where(ok[:, None, None], ref.value(c) * s[..., None].astype(np.float64), 0.0)
        # one product in binary32, one rounding to the output type
        off = np.abs(_f64(got) - want) - np.abs(want) * (2.0 ** -24 + HALF[out]) * 1.01
        assert off.max() <= 0


@pytest.mark.parametrize("D", [64, 128])
def test_read_turns_rotated_rows_back(ra, D):
    rng = np.random.default_rng(2)
    Hkv, page, pages = 2, 64, 3
    p = _params(ra, 2, Hkv, D, page, pages, pages, had=True, vhad=True, out="fp32")
    cache = rng.integers(0, 256, (pages, ra.cache_layout(p)["page_bytes"]), dtype=np.uint8)
    cache.reshape(pages, Hkv, -1)[:, :, page * D:] = np.full((pages, Hkv, 2 * page), 0.37, np.float32).view(np.uint8).reshape(pages, Hkv, -1)
    slots = np.arange(pages * page - 7)
    k, v = (torch.empty((len(slots), Hkv, D), device="cuda") for _ in range(2))
    ra.cache_read(p, torch.from_numpy(cache).cuda(), _i32(slots), k, v)
    kc, ks, vc, vs = ref.rows(cache, slots, page, Hkv, D)
    H = ref.hadamard(D) / np.sqrt(D)
    for got, c, s in ((k, kc, ks), (v, vc, vs)):
        want = (ref.value(c) * s[..., None].astype(np.float64)) @ H
        # sums of codes are exact; the scale times 1/sqrt(D) (itself rounded) and the product round.  The 64-bit
        # sum of D terms of at most 6 * 0.37 / sqrt(D) is itself off by up to D * 2^-53 * 2.3 sqrt(D) < 2^-38.
        off = np.abs(_f64(got) - want) - np.abs(want) * 3.1 * 2.0 ** -24
        assert off.max() <= 2.0 ** -38


# ----------------------------------------------------------------- append --

def _special_rows(x, rng):
    """Rows that meet borders, zeros and what is not finite (first tokens of head 0)."""
    D = x.shape[-1]
    x[0] = 0
    x[1] = rng.integers(-24, 25, x[1].shape) * 0.25         # 6 x / a meets many borders exactly
    x[1, :, 0] = 6.0
    x[2] = rng.integers(-12, 13, x[2].shape) / 8.0
    x[2, :, 1] = 3.0
    x[3] = rng.integers(-20, 21, x[3].shape)
    x[3, :, D - 1] = -20.0
    x[4, 0, 5] = np.inf
    x[5, 0, 6] = np.nan
    x[6] = 1e-38
    return x


@pytest.mark.parametrize("D,Hkv,page,dt,rope,had,vhad,strided", [
    (128, 2, 16, "bf16", False, False, False, False),
    (128, 3, 64, "fp16", False, False, True, True),
    (128, 8, 32, "bf16", True, True, False, True),
    (64, 2, 16, "fp16", True, True, True, False),
    (64, 5, 256, "bf16", False, True, False, True),
    (64, 1, 128, "bf16", True, False, False, False),
])
def test_append_writes_the_codes_of_64_bits(ra, D, Hkv, page, dt, rope, had, vhad, strided):
    rng = np.random.default_rng(D + Hkv + page)
    T, pages = 301, 301 // page + 3
    p = _params(ra, Hkv * 2, Hkv, D, page, pages, pages, had, vhad, dt)
    x = rng.standard_normal((T, 4 * Hkv, D)) * np.exp(rng.standard_normal((T, 1, 1)))
    x[:, :, 3] *= 8.0
    x[:, 2 * Hkv:] = np.concatenate([_special_rows(x[:, 2 * Hkv:3 * Hkv].copy(), rng),
                                     _special_rows(x[:, 3 * Hkv:].copy(), rng)], 1)
    xd = torch.tensor(x).to(DT[dt]).cuda()
    k, v = xd[:, 2 * Hkv:3 * Hkv], xd[:, 3 * Hkv:]
    if not strided:
        k, v = k.contiguous(), v.contiguous()
    slots = rng.permutation(pages * page)[:T].astype(np.int32)
    slots[20], slots[21], slots[22] = -1, pages * page, -77
    ok = (slots >= 0) & (slots < pages * page)
    pos = rng.integers(0, pages * page, T).astype(np.int32)
    if rope:
        pos[30], pos[31] = -1, 2 ** 31 - 1
        ok &= (pos >= 0) & (pos < 2 ** 30)
    table = ref.rope_table(pages * page, D)
    before = rng.integers(0, 256, (pages, ra.cache_layout(p)["page_bytes"]), dtype=np.uint8)
    cache = torch.from_numpy(before.copy()).cuda()
    ra.cache_append(p, k, v, _i32(slots), cache, positions=_i32(pos) if rope else None,
                    rope=torch.from_numpy(table).cuda() if rope else None)
    after = cache.cpu().numpy()
    kc, ks, vc, vs = ref.rows(after, slots[ok], page, Hkv, D)
    H = ref.hadamard(D)
    for got, s, src, h, r in ((kc, ks, k, had, rope), (vc, vs, v, vhad, False)):
        y = _f64(src)[ok]
        if r:
            y = ref.turn(y, table[pos[ok]])
        if h:
            with np.errstate(invalid="ignore"):
                y = y @ H
        want, a = ref.codes(y)
        bad = ref.value(got) != ref.value(want)
        assert not bad.any(), f"{bad.sum()} codes differ, first at {np.argwhere(bad)[0]}"
        want_s = a / 6.0 / (np.sqrt(D) if h else 1.0)
        # sums of up to D / 2 pairs: 9 roundings in a row at most, relative to the sum of magnitudes, which is at
        # most sqrt(D) times the largest (see the kernel); the division and the factor round
        tol = (10 * np.sqrt(D) * np.sqrt(2) if h else 3 if r else 0) * 2.0 ** -24 + 3 * 2.0 ** -24
        fine = np.isfinite(want_s)
        assert (np.isnan(s) == ~fine).all()
        off = np.abs(s[fine] - want_s[fine]) - tol * want_s[fine]
        assert off.max() <= 0
    # nothing else was written
    keep = np.ones((pages, Hkv, ra.cache_layout(p)["head_bytes"]), bool)
    d = np.arange(D)
    for slot in slots[ok]:
        g, t = slot // page, slot % page
        for at in (ref.k_byte(D, t, d), ref.v_byte(D, page, t, d), page * D + 4 * t + np.arange(4),
                   page * D + 4 * page + 4 * t + np.arange(4)):
            keep[g][:, at] = False
    keep = keep.reshape(before.shape)
    assert (after[keep] == before[keep]).all()


def test_append_of_many_tokens_equals_64_bits(ra):
    """Enough rotated rows that some come within rounding of a border."""
    rng = np.random.default_rng(9)
    D, Hkv, page, T = 128, 4, 64, 6000
    pages = T // page + 1
    p = _params(ra, Hkv, Hkv, D, page, pages, pages, True, True, "bf16", out="fp32")
    k, v = (torch.tensor(rng.standard_normal((T, Hkv, D))).to(torch.bfloat16).cuda() for _ in range(2))
    pos = np.arange(T)
    table = ref.rope_table(pages * page, D)
    cache = torch.empty((pages, ra.cache_layout(p)["page_bytes"]), dtype=torch.uint8, device="cuda")
    ra.cache_append(p, k, v, _i32(pos), cache, positions=_i32(pos), rope=torch.from_numpy(table).cuda())
    kc, ks, vc, vs = ref.rows(cache.cpu().numpy(), pos, page, Hkv, D)
    H = ref.hadamard(D)
    for got, y in ((kc, ref.turn(_f64(k), table[pos])), (vc, _f64(v))):
        want, _ = ref.codes(y @ H)
        assert (ref.value(got) == ref.value(want)).all()


# ------------------------------------------------------------------- plan --

def _run_plan(ra, p, st, new, T, release=None, inplace=True):
    R = len(new)
    out = {n: torch.full((m,), 99, dtype=torch.int32, device="cuda")
           for n, m in (("q_start", R + 1), ("positions", T), ("slots", T), ("status", 4))}
    kw = {} if inplace else {"seq_out": torch.full((R,), 99, dtype=torch.int32, device="cuda"),
                             "count_out": torch.full((1,), 99, dtype=torch.int32, device="cuda")}
    ra.cache_plan(p, st["seq_lens"], _i32(new), st["block_table"], st["free_pages"], st["free_count"], out["q_start"],
                  out["positions"], out["slots"], out["status"],
                  release=None if release is None else _i32(release), **kw)
    return out, kw


def _check_plan(ra, p, st, host, new, T, release=None, inplace=True):
    want = ref.plan(p.page_size, p.max_blocks, p.num_pages, T, host["seq"], new, host["table"], host["free"],
                    host["count"], release)
    out, kw = _run_plan(ra, p, st, new, T, release, inplace)
    status, table, free, count, seq, start, pos, slot = want
    assert out["status"].tolist() == status
    assert (st["block_table"].cpu().numpy() == table).all()
    assert st["free_pages"][:max(count, 0)].tolist() == free[:max(count, 0)]
    assert (kw.get("count_out", st["free_count"])).tolist() == [count]
    assert (kw.get("seq_out", st["seq_lens"])).tolist() == seq
    assert out["q_start"].tolist() == start
    assert out["positions"].tolist() == pos
    assert out["slots"].tolist() == slot
    if not inplace:      # the table is updated in any case: go on from the new lengths
        st["seq_lens"].copy_(kw["seq_out"])
        st["free_count"].copy_(kw["count_out"])
    host.update(table=table, free=free, count=count, seq=seq)
    return status


def _plan_state(ra, p, R):
    st = ra.alloc_cache(p, R)
    del st["cache"]
    return st, {"seq": [0] * R, "table": np.full((R, p.max_blocks), -1, np.int32),
                "free": st["free_pages"].tolist(), "count": p.num_pages}


@pytest.mark.parametrize("R,page,T", [(1, 16, 1), (1, 256, 5000), (7, 16, 200), (64, 32, 4096), (65, 16, 4097),
                                      (1024, 16, 3000), (1500, 64, 9001), (2500, 16, 20000)])
def test_plan_over_several_steps(ra, R, page, T):
    rng = np.random.default_rng(R)
    blocks = 40 if R > 1 else 400
    p = _params(ra, 2, 1, 64, page, R * 12 + 400, blocks)
    st, host = _plan_state(ra, p, R)
    for step in range(4):
        new = np.zeros(R, np.int64)
        left = T
        for r in rng.permutation(R):
            n = int(rng.integers(0, 3)) if rng.random() < 0.8 else int(rng.integers(0, 90))
            new[r] = min(n, left)
            left -= new[r]
        if R == 1:
            new[0] = T if step == 0 else min(T, 37)
        rel = (rng.random(R) < 0.3).astype(np.int32) if step >= 2 else None
        assert _check_plan(ra, p, st, host, new.tolist(), T, rel, inplace=step != 1)[0] == 0


def test_plan_refuses_as_a_whole(ra):
    p = _params(ra, 2, 1, 64, 16, 10, 6)
    st, host = _plan_state(ra, p, 3)
    assert _check_plan(ra, p, st, host, [20, 1, 40], 64)[0] == 0
    assert _check_plan(ra, p, st, host, [80, 0, 0], 90)[0] == 1        # past the table
    assert _check_plan(ra, p, st, host, [-1, 0, 0], 90)[0] == 1
    assert _check_plan(ra, p, st, host, [5, 6, 7], 17)[0] == 2         # more tokens than rows
    assert _check_plan(ra, p, st, host, [40, 40, 20], 100)[0] == 4     # too few pages
    assert _check_plan(ra, p, st, host, [40, 40, 20], 99)[0] == 6
    assert _check_plan(ra, p, st, host, [2 ** 31 - 1, 1, 2 ** 31 - 1], 5)[0] == 1
    # with a request released in the same step there is room
    assert _check_plan(ra, p, st, host, [40, 40, 20], 100, [0, 0, 1])[0] == 0
    st["free_count"].fill_(11)
    host["count"] = 11
    assert _check_plan(ra, p, st, host, [0, 0, 0], 4)[0] == 8
    st["free_count"].fill_(-1)
    host["count"] = -1
    assert _check_plan(ra, p, st, host, [0, 0, 0], 4)[0] == 8


def test_plan_of_nothing(ra):
    p = _params(ra, 2, 1, 64, 16, 4, 2)
    st, host = _plan_state(ra, p, 0)
    _check_plan(ra, p, st, host, [], 5)
    st, host = _plan_state(ra, p, 2)
    _check_plan(ra, p, st, host, [0, 0], 0)
    _check_plan(ra, p, st, host, [32, 32], 64)
    _check_plan(ra, p, st, host, [0, 0], 3)


def test_plan_with_damaged_tables_gives_no_slots(ra):
    """Page numbers that are none: slots of -1, nothing outside is touched."""
    p = _params(ra, 2, 1, 64, 16, 8, 4)
    st, _ = _plan_state(ra, p, 2)
    st["seq_lens"].copy_(_i32([5, 0]))
    st["block_table"].fill_(-5)
    st["free_pages"].fill_(1 << 20)
    out, _ = _run_plan(ra, p, st, [3, 4], 7)
    assert out["slots"].tolist() == [-1] * 7 and out["positions"].tolist() == [5, 6, 7, 0, 1, 2, 3]


# -------------------------------------------------------------- attention --

def _filled(ra, p, rng, lens, poison=True):
    """Random pages in a random order; scales of places behind a request's end are NaN."""
    D, page, Hkv = p.D, p.page_size, p.Hkv
    nb = [-(-n // page) for n in lens]
    perm = rng.permutation(p.num_pages)[:sum(nb)]
    table = np.full((len(lens), p.max_blocks), -1, np.int32)
    cache = rng.integers(0, 256, (p.num_pages, ra.cache_layout(p)["page_bytes"]), dtype=np.uint8)
    view = cache.reshape(p.num_pages, Hkv, -1)
    # a code is 2.7 on average: about unit values
    sc = (0.37 * np.exp(0.3 * rng.standard_normal((p.num_pages, Hkv, 2, page)))).astype(np.float32)
    used = np.zeros((p.num_pages, page), bool)
    at = 0
    for r, n in enumerate(lens):
        table[r, :nb[r]] = perm[at:at + nb[r]]
        at += nb[r]
        for j in range(nb[r]):
            used[table[r, j], :max(0, min(page, n - j * page))] = True
    if poison:
        sc = np.where(used[:, None, None, :], sc, np.float32(np.nan))
    view[:, :, page * D:] = sc.view(np.uint8).reshape(p.num_pages, Hkv, -1)
    return cache, table


def _attn_case(ra, Hq, Hkv, D, page, lens, qs, dt="bf16", out=None, rope=False, had=False, vhad=False, causal=True,
               window=0, pad=0, seed=0, gain=1.5, max_q=None, strided=False):
    rng = np.random.default_rng(seed)
    out = out or dt
    pages = sum(-(-n // page) for n in lens) + 2
    blocks = max([-(-n // page) for n in lens] + [1]) + 1
    p = _params(ra, Hq, Hkv, D, page, pages, blocks, had, vhad, dt, out, causal=causal, window=window)
    cache, table = _filled(ra, p, rng, lens)
    start = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
    T = int(start[-1]) + pad
    q = torch.tensor(rng.standard_normal((T, Hq + (2 if strided else 0), D)) * gain).to(DT[dt]).cuda()
    q = q[:, 1:Hq + 1] if strided else q
    o = torch.full((T, Hq, D), 5.0, dtype=DT[out], device="cuda")
    lse = torch.full((T, Hq), 5.0, device="cuda")
    cs = ref.rope_table(blocks * page, D) if rope else None
    max_q = max(list(qs) + [0]) if max_q is None else max_q
    ws = ra.cache_workspace(p, len(lens), T, max_q)
    args = (p, q, torch.from_numpy(cache).cuda(), _i32(table), _i32(start), _i32(lens), max_q, o, ws)
    kw = dict(lse=lse, rope=None if cs is None else torch.from_numpy(cs).cuda())
    ra.cache_attn(*args, **kw)
    G = Hq // Hkv
    H = ref.hadamard(D) / np.sqrt(D)
    want, want_lse = np.full((T, Hq, D), 5.0), np.full((T, Hq), 5.0)
    size_v, size_s = np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for r, (n, m) in enumerate(zip(lens, qs)):
        if m == 0:
            continue
        slots = [int(table[r, t // page]) * page + t % page for t in range(n)]
        kc, ks, vc, vs = ref.rows(cache, slots, page, Hkv, D)
        k, v = ref.value(kc) * ks[..., None].astype(np.float64), ref.value(vc) * vs[..., None].astype(np.float64)
        x = _f64(q[start[r]:start[r + 1]])
        if rope:
            x = ref.turn(x, cs[np.maximum(n - m + np.arange(m), 0)])
        if had:
            x = x @ H
        for h in range(Hq):
            y, z, av, a = ref.attn(x[:, h], k[:, h // G], v[:, h // G], causal, window, D ** -0.5)
            sl = slice(start[r], start[r + 1])
            # turned back, an error of one channel reaches all: bounded by the sum over channels
            want[sl, h] = y @ H if vhad else y
            size_v[sl, h] = np.abs(av).sum(1, keepdims=True) / np.sqrt(D) if vhad else av
            want_lse[sl, h], size_s[sl, h] = z, a
    _check_attn(o, lse, want, want_lse, size_v, size_s, dt, out, max(lens + [1]), max(qs + [0]) * G, vhad)
    return args, kw


def _operand(dt, out, rows):
    """Half a step of the matrix products' operands (Q, P).  Q is two values of 8 (11) bits or more, one below the
    other: 2^-16.  P is two as well, but one for requests of many rows where the output is no finer than it."""
    one = rows > 32 and out != "fp32" and (dt, out) != ("bf16", "fp16")
    return 2.0 ** -16, HALF[dt] if one else 2.0 ** -16


def _check_attn(o, lse, want, want_lse, size_v, size_s, dt, out, n, rows, turned=True):
    """Bounds by arithmetic.  Scores: Q rounded by eq relative to each element, products exact, sums of D terms and
    the scales in binary32: |ds| <= (eq + (D + 8) 2^-24) size_s.  A weight is then off by a factor e^(2 |ds|) (its
    own and the sum's), its rounding e and the sums of n terms (n / 64 steps of blocks summed in the matrix unit,
    at most 2^-24 a step and term group): the output by size_v times all of it, and its own rounding.  Binary16
    weights (requests of many rows) below 2^-14 of the largest V scale (here at most 2) are subnormal: each rounds by
    up to 2^-25 of it, times a code of up to 6, and the sum of weights is at least 1; turned back, sqrt(D) channels'
    worth of that."""
    eq, e = _operand(dt, out, rows)
    D = want.shape[2]
    ds = (eq + (D + 8) * 2.0 ** -24) * size_s + 2.0 ** -21
    acc = (n / 16 + 64) * 2.0 ** -24
    rel = np.expm1(2 * ds) + e + 2 * acc
    got, got_lse = _f64(o), _f64(lse)
    live = np.isfinite(want_lse)
    assert (np.isneginf(got_lse) == np.isneginf(want_lse)).all()
    small = n * 2.0 ** -25 * 12 * (np.sqrt(D) if turned else 1) if dt == "fp16" and rows > 32 else 0.0
    bound = small + size_v * rel[..., None] + (np.abs(want) + size_v * rel[..., None]) * HALF[out] + 1e-30
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} outputs off, worst {np.nanmax(err / bound):.3g} of the bound at {np.argwhere(bad)[0]}"
    d = np.abs(got_lse - np.where(live, want_lse, 0))[live]
    lim = (ds + acc + 2.0 ** -22 * (1 + np.abs(np.where(live, want_lse, 0))))[live]
    assert (d <= lim).all(), f"lse off by {(d / lim).max():.3g} of the bound"
    # roundings are independent: on the whole the error stays far below the bound
    norm = np.sqrt((want ** 2).mean()) + 1e-30
    rms = np.sqrt(((got - want) ** 2).mean()) / norm
    assert rms <= e + 4 * eq + HALF[out] + 2 * acc + 2.0 ** -18, f"relative error {rms:.3g}"


@pytest.mark.parametrize("D,page", [(128, 16), (64, 16), (128, 64), (64, 256)])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 257, 1000])
def test_attn_single_token(ra, D, page, n):
    _attn_case(ra, 4, 2, D, page, [n], [1], seed=n)


@pytest.mark.parametrize("dt,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32"), ("fp16", "fp32"),
                                    ("fp16", "bf16")])
@pytest.mark.parametrize("Hq,Hkv", [(12, 12), (5, 1), (32, 2), (40, 8)])
def test_attn_decode_types_and_heads(ra, dt, out, Hq, Hkv):
    _attn_case(ra, Hq, Hkv, 128, 32, [300, 1, 0, 77, 1025, 64], [1, 1, 0, 1, 1, 0], dt, out, rope=True, had=True,
               vhad=out == "fp32", pad=3, seed=Hq, strided=True)


@pytest.mark.parametrize("Hq,Hkv,dt", [(48, 1, "bf16"), (20, 1, "fp16"), (33, 1, "fp16"), (34, 2, "bf16")])
def test_attn_decode_of_large_head_groups(ra, Hq, Hkv, dt):
    """Groups of 17 to 32 rows, and of more than a request of few rows has."""
    _attn_case(ra, Hq, Hkv, 128, 64, [1500, 40, 0, 9000], [1, 1, 0, 1], dt, rope=True, seed=Hq)


def test_attn_of_many_requests_with_few_and_many_rows(ra):
    rng = np.random.default_rng(77)
    lens = rng.integers(1, 300, 80).tolist()
    qs = [min(n, int(q)) for n, q in zip(lens, rng.choice([0, 1, 1, 1, 5, 60], 80))]
    _attn_case(ra, 4, 1, 64, 32, lens, qs, "bf16", rope=True, vhad=True, pad=1, seed=77)


@pytest.mark.parametrize("R,n", [(1, 20011), (3, 9000), (70, 400), (300, 130)])
def test_attn_decode_split_and_many(ra, R, n):
    rng = np.random.default_rng(R)
    lens = [n] + rng.integers(1, n, R - 1).tolist()
    _attn_case(ra, 2, 1, 64 if R > 100 else 128, 64, lens, [1] * R, rope=R < 10, seed=R)


@pytest.mark.parametrize("D,Hq,Hkv,page,dt", [(128, 4, 2, 16, "bf16"), (64, 6, 2, 64, "fp16"), (128, 8, 1, 128, "fp16"),
                                              (64, 3, 3, 32, "bf16")])
@pytest.mark.parametrize("lens,qs", [([40, 7, 130], [40, 7, 130]), ([300, 513], [5, 257]), ([1, 1000, 90], [1, 33, 0])])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 50), (True, 1)])
def test_attn_prompts(ra, D, Hq, Hkv, page, dt, lens, qs, causal, window):
    _attn_case(ra, Hq, Hkv, D, page, lens, qs, dt, rope=causal, had=window != 1, vhad=window == 50, causal=causal,
               window=window, pad=2, seed=len(lens) + window)


def test_attn_queries_before_the_first_key_see_nothing(ra):
    """More queries than cached tokens: the first rows have no key, nor has a request of length 0."""
    _attn_case(ra, 4, 2, 128, 16, [3, 0, 20], [7, 2, 50], seed=3)
    _attn_case(ra, 4, 2, 64, 16, [0], [1], seed=4, causal=False)


def test_attn_large_scores(ra):
    """Scores of hundreds: the maximum moves, sums neither overflow nor vanish."""
    _attn_case(ra, 4, 4, 128, 64, [700, 300], [1, 20], "fp16", "fp32", seed=5, gain=60.0)


def test_attn_longer_max_q_and_bounded_queries(ra):
    """max_q above what there is changes nothing; below it, later queries are left as they were."""
    (p, q, cache, table, start, lens, _, o, ws), kw = _attn_case(ra, 4, 2, 128, 16, [200, 90], [70, 20], seed=6, max_q=90)
    base, base_lse = o.clone(), kw["lse"].clone()
    o.fill_(5.0)
    kw["lse"].fill_(5.0)
    ra.cache_attn(p, q, cache, table, start, lens, 30, o, ra.cache_workspace(p, 2, 90, 30), **kw)
    assert (o[30:70] == 5.0).all() and (kw["lse"][30:70] == 5.0).all()
    for s in (slice(0, 30), slice(70, 90)):
        # another split of the rows rounds elsewhere: half a step each of Q, P and the output, on values of order 1
        assert (o[s] - base[s]).abs().max() < 8 * HALF["bf16"] * base[s].abs().max()


def test_attn_what_a_row_does_not_see_cannot_reach_it(ra):
    """NaN scales of later keys (causal), earlier keys (window), pages that are none, padding rows of q."""
    rng = np.random.default_rng(8)
    for q_len in (6, 40):
        p = _params(ra, 4, 2, 128, 16, 12, 10, causal=True, window=30)
        cache, table = _filled(ra, p, rng, [100])
        q = torch.tensor(rng.standard_normal((q_len + 3, 4, 128))).to(torch.bfloat16).cuda()
        q[q_len:] = float("nan")
        outs = []
        for bad in (False, True):
            c = cache.copy()
            if bad:
                view = c.reshape(12, 2, -1)[:, :, 16 * 128:]
                nan = np.frombuffer(np.float32(np.nan).tobytes(), np.uint8)
                for t in list(range(0, 100 - q_len - 29)) + [98, 99]:
                    for which in (0, 1):
                        at = 64 * which + 4 * (t % 16)
                        view[table[0, t // 16], :, at:at + 4] = nan
            o = torch.zeros_like(q)
            lse = torch.zeros(q.shape[:2], device="cuda")
            ra.cache_attn(p, q, torch.from_numpy(c).cuda(), _i32(table), _i32([0, q_len]), _i32([100]), q_len, o,
                          ra.cache_workspace(p, 1, q_len + 3, q_len), lse=lse)
            outs.append((o, lse))
        assert torch.equal(outs[0][0][:q_len - 2], outs[1][0][:q_len - 2])
        assert torch.equal(outs[0][1][:q_len - 2], outs[1][1][:q_len - 2])
        assert torch.isnan(outs[1][0][q_len - 2:q_len]).all()
        assert (outs[1][0][q_len:] == 0).all()


def test_attn_pages_that_are_none_are_masked(ra):
    rng = np.random.default_rng(11)
    for q_len in (1, 20):
        p = _params(ra, 2, 1, 64, 16, 8, 6, causal=False)
        cache, table = _filled(ra, p, rng, [70], poison=False)
        q = torch.tensor(rng.standard_normal((q_len, 2, 64))).to(torch.bfloat16).cuda()
        short = table.copy()
        short[0, 1], short[0, 3] = -1, 8
        res = []
        for tb, n in ((short, [70]), (None, [38])):
            if tb is None:   # the same keys, without the holes
                tb = table.copy()
                tb[0, :3] = table[0, [0, 2, 4]]
            o, lse = torch.zeros_like(q), torch.zeros(q_len, 2, device="cuda")
            ra.cache_attn(p, q, torch.from_numpy(cache).cuda(), _i32(tb), _i32([0, q_len]), _i32(n), q_len, o,
                          ra.cache_workspace(p, 1, q_len, q_len), lse=lse)
            res.append((o.float(), lse))
        # the same keys in another place of the block: sums in another order and P rounded at another maximum
        assert (res[0][0] - res[1][0]).abs().max() <= 4 * HALF["bf16"] * res[1][0].abs().max()
        assert (res[0][1] - res[1][1]).abs().max() <= 2.0 ** -8


def test_attn_offsets_past_32_bits(ra):
    """A cache of more than 4 GiB: the last pages are read where they are."""
    D, Hkv, page = 128, 8, 256
    pages = (5 << 30) // (Hkv * page * (D + 8))
    p = _params(ra, 8, Hkv, D, page, pages, 2, out="fp32")
    cache = torch.zeros((pages, ra.cache_layout(p)["page_bytes"]), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(300, Hkv, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(300, device="cuda")
    outs = []
    for a, b in ((pages - 1, pages - 2), (0, 1)):
        slots = torch.where(pos < page, a * page + pos, b * page + pos - page).int()
        ra.cache_append(p, k, v, slots, cache)
        kd, vd = torch.empty(300, Hkv, D, device="cuda"), torch.empty(300, Hkv, D, device="cuda")
        ra.cache_read(p, cache, slots, kd, vd)
        o = torch.zeros(1, 8, D, device="cuda")
        ra.cache_attn(p, k[:1].contiguous(), cache, _i32([[a, b]]), _i32([0, 1]), _i32([300]), 1, o,
                      ra.cache_workspace(p, 1, 1, 1))
        outs.append((kd, vd, o))
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    assert (outs[0][0] - k.float()).abs().max() < 0.2 * k.float().abs().max()


# -------------------------------------------------------------- all of them --

def _serve(ra, p, steps, R, T, max_q, rng, st, rope, stream=None, release_at=None):
    """Steps as a server makes them; returns per step (new, o, lse, inputs)."""
    H, D = p.Hq + 2 * p.Hkv, p.D
    ws = ra.cache_workspace(p, R, T, max_q)
    buf = {n: torch.zeros(m, dtype=torch.int32, device="cuda")
           for n, m in (("q_start", R + 1), ("positions", T), ("slots", T), ("status", 4), ("new", R), ("rel", R))}
    out = []
    for step in range(steps):
        new = rng.integers(0, max_q + 1, R) if step == 0 else rng.integers(0, 2, R)
        rel = np.zeros(R, np.int64)
        if release_at == step:
            rel[0], new[0] = 1, 5
        x = torch.tensor(rng.standard_normal((T, H, D))).to(torch.bfloat16).cuda()
        buf["new"].copy_(_i32(new))
        buf["rel"].copy_(_i32(rel))
        o = torch.full((T, p.Hq, D), 3.0, device="cuda")
        lse = torch.full((T, p.Hq), 3.0, device="cuda")
        out.append((new, rel, x, o, lse))
        yield_args = (buf, x, o, lse, ws)
        _step(ra, p, st, rope, max_q, *yield_args)
    return out


def _step(ra, p, st, rope, max_q, buf, x, o, lse, ws):
    ra.cache_plan(p, st["seq_lens"], buf["new"], st["block_table"], st["free_pages"], st["free_count"],
                  buf["q_start"], buf["positions"], buf["slots"], buf["status"], release=buf["rel"])
    ra.cache_append(p, x[:, p.Hq:p.Hq + p.Hkv], x[:, p.Hq + p.Hkv:], buf["slots"], st["cache"],
                    positions=buf["positions"], rope=rope)
    ra.cache_attn(p, x[:, :p.Hq], st["cache"], st["block_table"], buf["q_start"], st["seq_lens"], max_q, o, ws,
                  lse=lse, rope=rope)


def _server_params(ra):
    return _params(ra, 6, 2, 128, 16, 60, 12, True, True, "bf16", "fp32")


def test_a_run_of_steps_as_a_server_makes_them(ra):
    """Prompts, then tokens, with a request replaced: every step's outputs against 64-bit attention over codes made
    in 64 bits from everything given so far."""
    rng = np.random.default_rng(21)
    p = _server_params(ra)
    R, T, max_q, D, G = 5, 160, 30, 128, 3
    st = ra.alloc_cache(p, R)
    cs = ref.rope_table(p.max_blocks * p.page_size, D)
    steps = _serve(ra, p, 7, R, T, max_q, rng, st, torch.from_numpy(cs).cuda(), release_at=4)
    H = ref.hadamard(D)
    ks, vs = [[] for _ in range(R)], [[] for _ in range(R)]
    for new, rel, x, o, lse in steps:
        t = 0
        want, want_lse = np.full((T, 6, D), 3.0), np.full((T, 6), 3.0)
        size_v, size_s = np.zeros((T, 6, D)), np.zeros((T, 6))
        for r in range(R):
            if rel[r]:
                ks[r], vs[r] = [], []
            m = int(new[r])
            pos = len(ks[r]) + np.arange(m)
            xr = _f64(x[t:t + m])
            kk = ref.turn(xr[:, 6:8], cs[pos]) @ H
            vv = xr[:, 8:] @ H
            for y, dst in ((kk, ks[r]), (vv, vs[r])):
                c, a = ref.codes(y)
                dst.extend(ref.value(c) * (a / 6.0 / np.sqrt(D))[..., None])
            if m:
                qr = ref.turn(xr[:, :6], cs[pos]) @ H / np.sqrt(D)
                k, v = np.array(ks[r]), np.array(vs[r])
                for h in range(6):
                    y, z, av, a = ref.attn(qr[:, h], k[:, h // G], v[:, h // G], True, 0, D ** -0.5)
                    want[t:t + m, h], want_lse[t:t + m, h] = y @ H / np.sqrt(D), z
                    size_v[t:t + m, h], size_s[t:t + m, h] = np.abs(av).sum(1, keepdims=True) / np.sqrt(D), a
            t += m
        # the scales of the cache round too (2^-19, the append's bound): less than what is allowed for Q
        _check_attn(o, lse, want, want_lse, size_v, size_s, "bf16", "fp32", 200, max_q * G)


def test_a_captured_step_follows_its_lengths(ra):
    """One graph of plan, append and attention, replayed with other lengths and inputs, equals eager calls; eager
    work goes on between the replays, on the same state of another server."""
    p = _server_params(ra)
    R, T, max_q = 4, 120, 30
    rope = torch.from_numpy(ref.rope_table(p.max_blocks * p.page_size, 128)).cuda()
    H = p.Hq + 2 * p.Hkv

    def make():
        st = ra.alloc_cache(p, R)
        st["cache"].zero_()
        buf = {n: torch.zeros(m, dtype=torch.int32, device="cuda")
               for n, m in (("q_start", R + 1), ("positions", T), ("slots", T), ("status", 4), ("new", R), ("rel", R))}
        x = torch.zeros(T, H, 128, dtype=torch.bfloat16, device="cuda")
        o, lse = torch.zeros(T, p.Hq, 128, device="cuda"), torch.zeros(T, p.Hq, device="cuda")
        return st, buf, x, o, lse, ra.cache_workspace(p, R, T, max_q)

    a, b = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            _step(ra, p, a[0], rope, max_q, *a[1:])
    torch.cuda.current_stream().wait_stream(side)
    rng = np.random.default_rng(5)
    for step in range(6):
        new = rng.integers(0, max_q + 1, R) if step == 0 else rng.integers(0, 3, R)
        if step == 3:
            new[1] = -1          # refused: nothing happens
        x = torch.tensor(rng.standard_normal((T, H, 128))).to(torch.bfloat16).cuda()
        for s in (a, b):
            s[1]["new"].copy_(_i32(new))
            s[1]["rel"].copy_(_i32([0, 0, int(step == 4), 0]))
            s[2].copy_(x)
        graph.replay()
        _step(ra, p, b[0], rope, max_q, *b[1:])
        torch.cuda.synchronize()
        for n in a[1]:
            assert torch.equal(a[1][n], b[1][n]), (step, n)
        for n in a[0]:
            assert torch.equal(a[0][n], b[0][n]), (step, n)
        assert torch.equal(a[3], b[3]) and torch.equal(a[4], b[4])
        assert int(a[1]["status"][0]) == (1 if step == 3 else 0)


def test_results_repeat_and_streams_do_not_matter(ra):
    args, kw = _attn_case(ra, 8, 2, 128, 32, [5000, 300, 4000], [1, 40, 2], rope=True, had=True, seed=30)
    o = args[7].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    args[7].zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ra.cache_attn(*args, **kw)
    s.synchronize()
    assert torch.equal(o, args[7])
    args[7].zero_()
    torch.cuda.synchronize()
    ra.cache_attn(*args, stream=s.cuda_stream, **kw)
    s.synchronize()
    assert torch.equal(o, args[7])
