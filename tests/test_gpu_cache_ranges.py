"""The 4-bit paged KV cache where magnitudes lie far apart, against plain numpy in 64 bits (tests/cache_ref.py)."""
import numpy as np
import pytest

import cache_ref as ref
import test_gpu_cache as base
from test_gpu_cache import DT, HALF, _f64, _filled, _i32, _params, ra  # noqa: F401  (ra: the fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

PAIR = 2.0 ** -17    # of a value held as two bf16 values: half a step of the second, which is at most half a step of the first


def _scales(cache, p):
    """K and V scales [pages, Hkv, 2, page] of page bytes, as a view."""
    at = p.page_size * p.D
    return cache.reshape(p.num_pages, p.Hkv, -1)[:, :, at:].view(np.float32).reshape(p.num_pages, p.Hkv, 2, p.page_size)


def _dense(cache, table, p, n):
    slots = [int(table[0, t // p.page_size]) * p.page_size + t % p.page_size for t in range(n)]
    kc, ks, vc, vs = ref.rows(cache, slots, p.page_size, p.Hkv, p.D)
    return ref.value(kc) * ks[..., None].astype(np.float64), ref.value(vc) * vs[..., None].astype(np.float64)


def _run(ra, p, q, cache, table, n, out):
    m = q.shape[0]
    o, lse = torch.full(q.shape, 5.0, dtype=DT[out], device="cuda"), torch.full(q.shape[:2], 5.0, device="cuda")
    ra.cache_attn(p, q, torch.from_numpy(cache).cuda(), _i32(table), _i32([0, m]), _i32([n]), m, o,
                  ra.cache_workspace(p, 1, m, m), lse=lse)
    return o, lse


def _want(p, q, cache, table, n, rows=slice(None)):
    """Outputs, lse and what the bound takes of one request's queries."""
    k, v = _dense(cache, table, p, n)
    G, H = p.Hq // p.Hkv, ref.hadamard(p.D) / np.sqrt(p.D)
    x = _f64(q)
    scale = p.sm_scale or p.D ** -0.5
    want, lse = np.zeros(x.shape), np.zeros(x.shape[:2])
    size_v, size_s = np.zeros(x.shape), np.zeros(x.shape[:2])
    for h in range(p.Hq):
        y = x[:, h] @ H if p.rotation else x[:, h]
        y, z, av, a = ref.attn(y, k[:, h // G], v[:, h // G], bool(p.causal), p.window, scale)
        want[:, h] = y @ H if p.v_rotation else y
        size_v[:, h] = np.abs(av).sum(1, keepdims=True) / np.sqrt(p.D) if p.v_rotation else av
        lse[:, h], size_s[:, h] = z, a
    return [x[rows] for x in (want, lse, size_v, size_s)]


def _check(o, lse, want, out, n, many):
    """test_gpu_cache's bounds with two values of bf16 for Q and, but for bf16 outputs of many rows, for P; nothing
    else for small weights or values.  Binary16 outputs below 2^-14 round by up to 2^-25."""
    want, want_lse, size_v, size_s = want
    e = HALF["bf16"] if many and out == "bf16" else PAIR
    ds = (PAIR + (want.shape[2] + 8) * 2.0 ** -24) * size_s + 2.0 ** -21
    acc = (n / 16 + 64) * 2.0 ** -24
    rel = np.expm1(2 * ds) + e + 2 * acc
    bound = size_v * rel[..., None] + (np.abs(want) + size_v * rel[..., None]) * HALF[out] + 1e-30
    bound += 2.0 ** -25 if out == "fp16" else 0.0
    err = np.abs(_f64(o) - want)
    assert (err <= bound).all(), f"outputs off by {np.nanmax(err / bound):.3g} of the bound"
    lim = ds + acc + 2.0 ** -22 * (1 + np.abs(want_lse))
    d = np.abs(_f64(lse) - want_lse)
    assert (d <= lim).all(), f"lse off by {np.nanmax(d / lim):.3g} of the bound"


# rows of a request that the kernel for few rows takes (24), and of one for many (80)
@pytest.mark.parametrize("q_len", [12, 40])
@pytest.mark.parametrize("dt,out", [("fp16", "fp16"), ("fp16", "fp32"), ("fp16", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("D,vhad", [(128, False), (64, True)])
def test_attn_large_values_that_a_row_does_not_see(ra, q_len, dt, out, D, vhad):
    """V of 6e4 in tokens behind a row and left of its window, beside V of 0.05: rows that do not see them are right, and
    the same bits as with ordinary tokens there."""
    rng = np.random.default_rng(q_len + D)
    n, window = 100, 30
    p = _params(ra, 4, 2, D, 16, 12, 10, vhad=vhad, dt=dt, out=out, window=window)
    cache, table = _filled(ra, p, rng, [n])
    sc = _scales(cache, p)
    sc[:, :, 1] = 0.05 / 6 * rng.uniform(0.5, 1.0, sc[:, :, 1].shape)
    first = n - q_len
    left = first - window + 4                     # the first few rows see it, as they see the tokens around it
    other = cache.copy()
    for t in (0, left, n - 2, n - 1):
        _scales(other, p)[table[0, t // 16], :, 1, t % 16] = 6e4 / 6
    q = torch.tensor(rng.standard_normal((q_len, 4, D))).to(DT[dt]).cuda()
    rows = slice(5, q_len - 2)
    ordinary, large = (_run(ra, p, q, c, table, n, out) for c in (cache, other))
    _check(large[0][rows], large[1][rows], _want(p, q, other, table, n, rows), out, n, q_len > 16)
    assert torch.equal(ordinary[0][rows], large[0][rows]) and torch.equal(ordinary[1], large[1])


@pytest.mark.parametrize("q_len", [20, 40])
@pytest.mark.parametrize("dt,out", [("fp16", "fp16"), ("fp16", "fp32"), ("bf16", "fp32")])
def test_attn_a_long_tail_of_small_weights(ra, q_len, dt, out):
    """One key takes nearly all of the softmax and has V = 0: the output is the other 20000 keys', 2^-23 to 2^-27 each."""
    rng = np.random.default_rng(q_len)
    n, D = 20000, 64
    p = _params(ra, 1, 1, D, 64, n // 64 + 2, n // 64 + 2, dt=dt, out=out, causal=False)
    cache, table = _filled(ra, p, rng, [n])
    sc = _scales(cache, p)
    sc[:, :, 0] = 0.0
    sc[table[0, 0], :, :, 0] = 1.0, 0.0
    k, _ = _dense(cache, table, p, 1)
    x = np.log(2.0) * np.linspace(23, 27, q_len)[:, None] * k[0, 0] / (k[0, 0] ** 2).sum() * np.sqrt(D)
    q = torch.tensor(x[:, None]).to(DT[dt]).cuda()
    o, lse = _run(ra, p, q, cache, table, n, out)
    _check(o, lse, _want(p, q, cache, table, n), out, n, q_len > 32)


@pytest.mark.parametrize("q_len", [12, 40])
@pytest.mark.parametrize("dt,out,D,had", [("fp16", "fp16", 128, True), ("fp16", "fp32", 64, False), ("bf16", "fp32", 128, False)])
@pytest.mark.parametrize("gain,sm_scale", [(3000.0, 64.0), (1e-4, 0.0), (1.0, 1e-5)])
def test_attn_queries_whose_scaled_values_leave_binary16(ra, q_len, dt, out, D, had, gain, sm_scale):
    """Queries times the softmax scale above 65504 against small keys, and below 2^-14 against large ones."""
    rng = np.random.default_rng(q_len + D)
    n = 300
    p = _params(ra, 4, 2, D, 32, 12, 10, had=had, dt=dt, out=out, sm_scale=sm_scale)
    cache, table = _filled(ra, p, rng, [n], poison=False)
    sc = _scales(cache, p)
    # scores of about 4
    sc[:, :, 0] *= 4 / ((sm_scale or D ** -0.5) * gain * D ** 0.5)
    q = torch.tensor(rng.standard_normal((q_len, 4, D)) * gain).to(DT[dt]).cuda()
    assert torch.isfinite(q).all()
    o, lse = _run(ra, p, q, cache, table, n, out)
    _check(o, lse, _want(p, q, cache, table, n), out, n, q_len > 16)


# ----------------------------------------------------------------- append --

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rope", [False, True])
def test_append_rows_whose_rotation_overflows_are_not_finite(ra, D, rope):
    """Finite rows whose sums leave binary32 in a stage of the rotation: infinities cancel to NaN in half of the
    channels, the others are 0.  The scale is NaN, of K and of V, and the tokens beside them are as they were."""
    T, Hkv, page = 40, 2, 16
    p = _params(ra, 2, Hkv, D, page, 4, 4, had=True, vhad=True, out="fp32")
    rng = np.random.default_rng(D)
    x = rng.standard_normal((T, 2 * Hkv, D))
    bad = np.zeros(D)
    block = np.arange(D // 8)
    bad[0::8], bad[1::8] = 3e38, -3e38
    bad *= np.repeat(np.where(block % 4 == 3, -1.0, 1.0), 8)
    rows = [3, 17, 38]
    x[rows, 0], x[rows, -1] = bad, bad            # K of head 0, V of the last head
    xd = torch.tensor(x).to(torch.bfloat16).cuda()
    assert torch.isfinite(xd).all()
    table = ref.rope_table(64, D)
    table[:] = [1.0, 0.0]                          # turned by nothing, so that the same sums come up
    cache = torch.zeros((4, ra.cache_layout(p)["page_bytes"]), dtype=torch.uint8, device="cuda")
    pos = np.arange(T)
    ra.cache_append(p, xd[:, :Hkv], xd[:, Hkv:], _i32(pos), cache, positions=_i32(pos) if rope else None,
                    rope=torch.from_numpy(table).cuda() if rope else None)
    kc, ks, vc, vs = ref.rows(cache.cpu().numpy(), pos, page, Hkv, D)
    want = np.zeros((2, T, Hkv), bool)
    want[0, rows, 0], want[1, rows, -1] = True, True
    assert (np.isnan(ks) == want[0]).all() and (np.isnan(vs) == want[1]).all()
    H = ref.hadamard(D)
    for c, src, w in ((kc, xd[:, :Hkv], want[0]), (vc, xd[:, Hkv:], want[1])):
        assert (ref.value(c) == ref.value(ref.codes(_f64(src) @ H)[0]))[~w].all()


def test_append_of_zeros_costs_what_other_values_cost(ra):
    """Heads of 96 padded to 128, RoPE without rotation: exact zeros are no border, so nothing is done again in
    binary64 for them (which takes 1.8 times as long).  Best of several runs, so that other work does not count."""
    T, Hkv, D, page = 20000, 8, 128, 64
    pages = T // page + 1
    p = _params(ra, Hkv, Hkv, D, page, pages, pages)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(T, Hkv, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rope = torch.from_numpy(ref.rope_table(pages * page, D)).cuda()
    cache = torch.empty((pages, ra.cache_layout(p)["page_bytes"]), dtype=torch.uint8, device="cuda")
    padded = k.clone()
    padded[..., 96:] = 0

    def best(x):
        times = []
        for _ in range(12):
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            for _ in range(20):
                ra.cache_append(p, x, v, pos, cache, positions=pos, rope=rope)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    best(k)
    assert best(padded) < 1.3 * best(k)
    slots = np.arange(0, T, 97)
    kc, _, _, _ = ref.rows(cache.cpu().numpy(), slots, page, Hkv, D)
    want, _ = ref.codes(ref.turn(_f64(padded)[slots], ref.rope_table(pages * page, D)[slots]))
    want_k, _ = ref.codes(ref.turn(_f64(k)[slots], ref.rope_table(pages * page, D)[slots]))
    assert (ref.value(kc) == ref.value(want_k)).all()      # k came last
    ra.cache_append(p, padded, v, pos, cache, positions=pos, rope=rope)
    kc, _, _, _ = ref.rows(cache.cpu().numpy(), slots, page, Hkv, D)
    assert (ref.value(kc) == ref.value(want)).all()


def _bf16(x):
    return torch.tensor(np.asarray(x)).to(torch.bfloat16).double().numpy()


def test_append_codes_of_rows_made_for_the_roundings_of_binary32(ra):
    """Rows whose stage roundings all push one quotient the same way.  x_0 is about 1 (chosen so that a rounded 6 / a is
    high too); x_1, x_2, x_4, .. lie just below half a step of it, so that each stage loses them, added in output 0 (the
    maximum) and subtracted in output 127; the second half makes 6 y_127 / a end up just below the border 5 and keeps
    the other outputs away from borders.  In binary32 it comes out 72 * 2^-24 above 5.  Three tokens without a slot
    between them, so that no wave has two of them."""
    rng = np.random.default_rng(0)
    T, D, page, u = 4000, 128, 64, 2.0 ** -24
    x = np.zeros((T, D))
    first = rng.choice([1.0000440, 1.0002294, 1.0002739, 1.0004641, 1.0010260, 1.0011904], T) + rng.uniform(-1e-7, 1e-7, T)
    first = first.astype(np.float32).astype(np.float64)   # the cosine of pair 0
    x[:, 0] = 1
    x[:, [2, 4, 8, 16, 32]] = 0.99609375 * u
    x[:, 1] = 0.9921875 * u
    lost = 5 * 0.99609375 * u + x[:, 1] * first
    x[:, 64 + 2 ** np.arange(6)] = _bf16(4e-4 * 2.0 ** np.arange(6))
    x[:, 71] = _bf16(rng.uniform(-3, 3, T) * u)
    turned = x[:, 65:].sum(1)                     # of opposite signs in the two outputs
    q = 5 * (1 - rng.uniform(0, 1e-8, T))
    rest = (6 * (first - lost + turned) - q * (first + lost + turned)) / (6 + q)
    for d in (64, 67, 69, 70):                    # signs alike in both outputs
        x[:, d] = _bf16(rest)
        rest = rest - x[:, d]
    table = np.zeros((T, D // 2, 2), np.float32)
    table[:, 0, 0], table[:, 1:, 0] = first, 1.0
    pages = -(-T // page)
    p = _params(ra, 1, 1, D, page, pages, 1, had=True)
    k = torch.zeros(T, 4, 1, D, dtype=torch.bfloat16, device="cuda")
    k[:, 0, 0] = torch.tensor(x).cuda()
    assert (_f64(k[:, 0, 0]) == x).all()
    pos = torch.full((T, 4), -1, dtype=torch.int32, device="cuda")
    pos[:, 0] = torch.arange(T)
    k, pos = k.flatten(0, 1), pos.flatten()
    cache = torch.zeros((pages, ra.cache_layout(p)["page_bytes"]), dtype=torch.uint8, device="cuda")
    ra.cache_append(p, k, k, pos, cache, positions=pos, rope=torch.from_numpy(table).cuda())
    kc, _, _, _ = ref.rows(cache.cpu().numpy(), np.arange(T), page, 1, D)
    want, _ = ref.codes(ref.turn(x[:, None], table) @ ref.hadamard(D))
    bad = (ref.value(kc) != ref.value(want)).any((1, 2))
    assert not bad.any(), f"{bad.sum()} rows"


@pytest.mark.parametrize("q_len,n", [(12, 150), (40, 150), (1, 9000), (70, 9000)])
@pytest.mark.parametrize("D,dt,vhad", [(128, "bf16", False), (64, "fp16", True)])
def test_attn_lse_is_of_the_keys_alone(ra, q_len, n, D, dt, vhad):
    """A token whose V alone is not finite: NaN outputs of the rows that see it, their lse as if it were finite,
    whichever kernel takes the request and however its keys are split; other rows the same bits."""
    rng = np.random.default_rng(n + q_len)
    p = _params(ra, 4, 2, D, 16, n // 16 + 3, n // 16 + 2, vhad=vhad, dt=dt, window=n - q_len // 2)
    cache, table = _filled(ra, p, rng, [n])
    q = torch.tensor(rng.standard_normal((q_len, 4, D))).to(DT[dt]).cuda()
    bad = [3, n - 1 - q_len // 3]            # out of the later rows' window, behind the earlier rows
    odd = cache.copy()
    for t, v in zip(bad, (np.nan, np.inf)):
        _scales(odd, p)[table[0, t // 16], :, 1, t % 16] = v
    plain, got = (_run(ra, p, q, c, table, n, dt) for c in (cache, odd))
    pos = n - q_len + np.arange(q_len)
    sees = np.zeros(q_len, bool)
    for t in bad:
        sees |= (t <= pos) & (t > pos - p.window)
    assert torch.isnan(got[0][sees]).all()
    assert torch.equal(got[0][~sees], plain[0][~sees])
    assert torch.isfinite(got[1]).all() and torch.equal(got[1], plain[1])


def _binary32(p, q, cache, table, n):
    """The definition in elementary binary32 operations (torch, on the host): outputs and lse."""
    f = torch.float32
    k, v = (torch.tensor(x).to(f) for x in _dense(cache, table, p, n))
    H = torch.tensor(ref.hadamard(p.D) / np.sqrt(p.D)).to(f)
    x, G, m = q.cpu().to(f), p.Hq // p.Hkv, q.shape[0]
    pos, key = n - m + torch.arange(m)[:, None], torch.arange(n)[None, :]
    out, lse = torch.empty(m, p.Hq, p.D), torch.empty(m, p.Hq)
    for h in range(p.Hq):
        y = x[:, h] @ H if p.rotation else x[:, h]
        s = (y @ k[:, h // G].T.contiguous()) * np.float32(p.D ** -0.5)
        s = torch.where(key <= pos, s, -torch.inf)
        top = s.max(1, keepdim=True).values
        w = torch.exp(s - top)
        l = w.sum(1, keepdim=True)
        y = (w @ v[:, h // G].contiguous()) / l
        out[:, h] = y @ H if p.v_rotation else y
        lse[:, h] = (top + torch.log(l))[:, 0]
    return out.double().numpy(), lse.double().numpy()


@pytest.mark.parametrize("q_len,n", [(1, 700), (6, 700), (13, 300), (40, 300), (150, 700), (1, 20000), (20, 9000)])
@pytest.mark.parametrize("D,dt,had,vhad,gain", [(128, "bf16", True, False, 1.5), (64, "fp16", False, True, 4.0),
                                                (128, "fp16", False, False, 3e-3)])
def test_attn_binary32_outputs_are_as_exact_as_binary32_arithmetic(ra, q_len, n, D, dt, had, vhad, gain):
    """Error against 64 bits at most twice that of binary32 operations throughout (there are as many roundings, in
    other places) and a rounding of the result; lse likewise.  Queries of a request differ by 2^40 in size."""
    rng = np.random.default_rng(n + q_len)
    p = _params(ra, 4, 2, D, 32, -(-n // 32) + 2, -(-n // 32) + 1, had=had, vhad=vhad, dt=dt, out="fp32")
    cache, table = _filled(ra, p, rng, [n])
    x = rng.standard_normal((q_len, 4, D)) * gain
    if dt == "bf16" and q_len > 1:
        x[0] *= 2.0 ** -40
    q = torch.tensor(x).to(DT[dt]).cuda()
    o, lse = _run(ra, p, q, cache, table, n, "fp32")
    want = _want(p, q, cache, table, n)
    _check(o, lse, want, "fp32", n, False)
    plain, plain_lse = _binary32(p, q, cache, table, n)
    rms = lambda a, b: np.sqrt(((a - b) ** 2).mean() / (b ** 2).mean())
    assert rms(_f64(o), want[0]) <= 2 * rms(plain, want[0]) + 2.0 ** -24
    # lse: in units of a rounding of scores as large as these
    unit = 2.0 ** -24 * (1 + np.abs(want[1]).max() + want[3].max())
    assert np.abs(_f64(lse) - want[1]).max() <= 2 * np.abs(plain_lse - want[1]).max() + 4 * unit
