"""The 4-bit paged KV cache: what its four operators are measured on.

The users serve a model token by token or frame by frame (causal video
generation, text): keys and values of past tokens stay in a paged cache as
4-bit floats (E2M1 codes, one binary32 scale per token and head), and every
step runs four calls:

  plan    block tables, slots and positions of the step's tokens, from lengths
  append  RoPE and rotation of the new K and V, their codes into the pages
  read    the values that cached tokens stand for, as dense K and V
  attn    attention of the new queries to everything cached

Shapes: 12, 24 and 40 heads of 128 are this library's own layers; grouped heads,
heads of 64 and the page sizes are generic.  `own` chooses between the plain
form (elementary torch operations in 32 bits or more) and the library's calls.

Page layout.  A page of `page` tokens holds, for each KV head in turn, the K
codes, the V codes, the K scales and the V scales (binary32, one per token).
  K code of (token t, channel d): byte (t/16)*8D + (d/(D/4))*2D + (t%16)*(D/8) + (d%(D/4))/2
  V code of (token t, channel d): byte (t/4)*2D + (d/(D/16))*(D/8) + (t%4)*(D/32) + (d%(D/16))/2
with channel d in the low nibble where d is even.  A code is sign (bit 3) and
one of the magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# halfway points of neighbouring magnitudes; True: the tie goes up (to the even code)
BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))

COMMON = {"Hq": 32, "Hkv": 8, "D": 128, "page": 64, "in": "bf16", "out": "bf16", "rope": True, "hadamard": True,
          "v_hadamard": False}


def _case(op, **kw):
    return dict(COMMON, op=op, **kw)


def _attn(**kw):
    base = {"R": 1, "singles": 0, "q_min": 1, "q_max": 1, "len_min": 1, "len_max": 1, "window": 0, "causal": True,
            "pad": 0, "ragged": 1}
    base.update(kw)
    return _case("attn", **base)


def listed():
    return [
        # eight running requests, one new token each: the host is idle until
        # the tables are there, only latency counts
        _case("plan", name="plan_decode", R=8, singles=8, q_max=1, len_max=4096, blocks=128, capacity=8, ragged=1),
        # a full scheduler step: a thousand requests, most of them decoding, the
        # others with prompt pieces, in a batch padded to a captured size
        _case("plan", name="plan_mixed", R=1000, singles=900, q_max=1500, len_max=7000, blocks=576, page=16,
              capacity=131072, ragged=2),
        # one decode step of 48 requests
        _case("append", name="append_decode", T=48, fused=True),
        # prompts of 21845 tokens in all, packed, out of one fused projection;
        # V rotated online, as for a model whose weights cannot be changed
        _case("append", name="append_prompt", T=21845, fused=True, v_hadamard=True, **{"in": "fp16"}),
        # a prompt of heads of 64 whose keys come in with their positions
        # applied and are kept as they are
        _case("append", name="append_plain", T=5000, fused=False, D=64, rope=False, hadamard=False, page=16),
        # cached tokens of one request handed on as dense tensors
        _case("read", name="read_request", T=1777, D=64, page=16, **{"out": "fp32"}),
        # all tokens of a batch handed on (a dense path takes over)
        _case("read", name="read_batch", T=50000, v_hadamard=True),
        # one request of a 12-head layer, one token: latency
        _attn(name="attn_single", Hq=12, Hkv=12, len_min=4097, len_max=4097),
        # a decode step of 64 requests of ragged lengths, grouped heads
        _attn(name="attn_decode", R=64, singles=64, len_min=50, len_max=16000, ragged=3),
        # two requests with long contexts on a 40-head layer, binary16
        _attn(name="attn_long", R=2, singles=2, Hq=40, Hkv=8, len_min=180001, len_max=230001, ragged=4,
              **{"in": "fp16", "out": "fp16"}),
        # prompts of ragged lengths, filled at once: bound by the matrix cores
        _attn(name="attn_prompt", R=5, q_min=1, q_max=8192, len_min=1, len_max=8192, ragged=5, whole=True),
        # a scheduler step on a 24-head layer: one prompt piece of 1000 tokens
        # over a long context, drafts of 4 tokens and plain decoding beside it,
        # rows behind the last request
        _attn(name="attn_mixed", Hq=24, Hkv=8, R=40, singles=30, q_min=4, q_max=1000, len_min=300, len_max=40000,
              pad=37, ragged=6, v_hadamard=True, page=32),
    ]


_MOST_PAIRS = 2.5e9     # query heads x visible keys of a drawn attention call, below attn_prompt's


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges."""
    D = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    Hq, Hkv = rng.choice([(12, 12), (24, 8), (40, 8), (32, 8), (32, 4), (16, 16), (8, 1), (28, 4), (20, 4), (1, 1)])
    dt = rng.choice(["bf16", "bf16", "fp16"])
    c = {"Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "in": dt, "out": rng.choice([dt, dt, "fp32"]),
         "rope": rng.random() < 0.7, "hadamard": rng.random() < 0.7, "v_hadamard": rng.random() < 0.3}
    op = rng.choice(["plan", "append", "append", "read", "attn", "attn", "attn", "attn", "attn"])
    c["ragged"] = rng.randrange(1 << 30)
    if op == "plan":
        R = _log(rng, 1, 1000)
        q_max, len_max = _log(rng, 1, 1500), _log(rng, 1, 8000)
        singles = rng.randint(0, R)
        c.update(R=R, singles=singles, q_max=q_max, len_max=len_max,
                 blocks=-(-(len_max + q_max) // page) + rng.randint(0, 20))
        c["capacity"] = min(131072, sum(_plan_lengths(c)[1]) + rng.choice([0, 0, rng.randint(1, 5000)]))
        if sum(_plan_lengths(c)[1]) > c["capacity"]:
            c.update(singles=R, q_max=1)
            c["capacity"] = sum(_plan_lengths(c)[1])
        c["capacity"] = max(1, c["capacity"])
        return dict(c, op=op)
    if op in ("append", "read"):
        most = int(21845 * 8 * 128 / (Hkv * D))
        c["T"] = _log(rng, 1, most if op == "append" else 2 * most)
        if op == "append":
            c["fused"] = rng.random() < 0.5
        return dict(c, op=op)
    c.update(causal=True, window=0, pad=rng.choice([0, 0, 0, rng.randint(1, 50)]), op=op)
    kind = rng.choice(["decode", "decode", "long", "prompt", "mixed"])
    if kind == "decode":
        c.update(R=_log(rng, 1, 100), q_min=1, q_max=rng.choice([1, 1, 1, 2, 5]), len_min=_log(rng, 1, 300),
                 len_max=_log(rng, 300, 16000))
        c["singles"] = c["R"] if c["q_max"] == 1 else rng.randint(0, c["R"])
    elif kind == "long":
        c.update(R=rng.randint(1, 3), q_min=1, q_max=1, len_min=20000, len_max=_log(rng, 20000, 230000))
        c["singles"] = c["R"]
    elif kind == "prompt":
        n = _log(rng, 2, 8000)
        c.update(R=rng.randint(1, 6), singles=0, q_min=1, q_max=n, len_min=1, len_max=n, whole=True)
        c["causal"] = rng.random() < 0.8
    else:
        c.update(R=rng.randint(2, 40), q_min=rng.randint(2, 8), q_max=_log(rng, 10, 1000), len_min=_log(rng, 20, 300),
                 len_max=_log(rng, 1000, 40000))
        c["singles"] = rng.randint(0, c["R"])
    if c["causal"] and rng.random() < 0.25:
        c["window"] = _log(rng, 10, 5000)
    # never above the largest listed calls, in pairs or in cached tokens
    while c["Hq"] * _pairs(c) > _MOST_PAIRS or sum(_lengths(c)[0]) * c["Hkv"] * c["D"] > 6e8:
        c["len_max"] = max(1, c["len_max"] * 2 // 3)
        c["len_min"] = min(c["len_min"], c["len_max"])
        c["q_max"] = min(c["q_max"], c["len_max"])
        c["q_min"] = min(c["q_min"], c["q_max"])
    return c


# ------------------------------------------------------------------ lengths --

def _plan_lengths(c):
    """Cached and new tokens of every request (from the case alone)."""
    rng = random.Random(c["ragged"])
    old, new = [], []
    for r in range(c["R"]):
        old.append(rng.randint(0, c["len_max"]))
        new.append(1 if r < c["singles"] else rng.randint(0, c["q_max"]))
    order = list(range(c["R"]))
    rng.shuffle(order)
    return [old[i] for i in order], [new[i] for i in order]


def _lengths(c):
    """Context and query length of every request (from the case alone): the
    first has the longest of both, requests below `singles` have one query."""
    rng = random.Random(c["ragged"])
    lens, qs = [], []
    for r in range(c["R"]):
        n = c["len_max"] if r == c["R"] - 1 else rng.randint(c["len_min"], c["len_max"])
        if r < c["singles"]:
            q = 1
        elif c.get("whole"):
            q = n
        else:
            q = c["q_max"] if r == c["R"] - 1 else _log(rng, c["q_min"], c["q_max"])
        lens.append(n)
        qs.append(min(q, n))
    order = list(range(c["R"]))
    rng.shuffle(order)
    return [lens[i] for i in order], [qs[i] for i in order]


def _visible(c, n, q):
    """First and last+1 visible key of the queries of one request."""
    out = []
    for i in range(q):
        pos = n - q + i
        hi = pos + 1 if c["causal"] else n
        out.append((max(0, hi - c["window"]) if c["window"] else 0, hi))
    return out


def _pairs(c):
    total = 0
    for n, q in zip(*_lengths(c)):
        if not c["causal"]:
            total += n * q
        elif c["window"]:
            total += sum(hi - lo for lo, hi in _visible(c, n, q))
        else:
            total += q * n - q * (q - 1) // 2
    return total


def work(case):
    c = case
    if c["op"] == "plan":
        new = sum(_plan_lengths(c)[1])
        # lengths in and out, offsets, the used entries of the table, positions and slots
        return {"bytes": 4 * (4 * c["R"] + 2 * c["capacity"] + new // c["page"] + c["R"]), "flops": 4 * c["capacity"]}
    D, Hkv = c["D"], c["Hkv"]
    esize = 4 if c["out"] == "fp32" else 2
    if c["op"] in ("append", "read"):
        T = c["T"]
        codes, dense = T * Hkv * (D + 8), 2 * T * Hkv * D * esize
        if c["op"] == "read":
            return {"bytes": codes + 4 * T + dense, "flops": 2 * T * Hkv * D * (9 if c["hadamard"] else 2)}
        rope = T * D * 4 if c["rope"] else 0
        # in: K and V, angles; out: the codes, and the values they stand for
        return {"bytes": 2 * T * Hkv * D * 2 + rope + 8 * T + codes + dense,
                "flops": T * Hkv * D * (3 * c["rope"] + 14 * c["hadamard"] + 14 * c["v_hadamard"] + 8)}
    lens, qs = _lengths(c)
    keys = sum(max(hi for _, hi in v) - min(lo for lo, _ in v)
               for v in (_visible(c, n, q) for n, q in zip(lens, qs)) if v)
    T = sum(qs)
    return {"bytes": keys * Hkv * (D + 8) + T * c["Hq"] * (D * (2 + esize) + 4) + (T * D * 4 if c["rope"] else 0),
            "flops": 4 * D * c["Hq"] * _pairs(c)}


# ------------------------------------------------------------------- inputs --

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rope_table(rows, D):
    """[rows, D/2, 2] cosines and sines: binary64 angles, rounded once."""
    pos = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None]
    freq = 10000.0 ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    ang = pos * freq[None, :]
    return torch.stack((torch.cos(ang), torch.sin(ang)), 2).float().contiguous()


def _page_bytes(c):
    return c["Hkv"] * c["page"] * (c["D"] + 8)


def _fill_pages(c, g, cache):
    """Pages of keys and values as a model leaves them: normal channels, token
    gains that vary, quantised and packed."""
    P, D, Hkv, page = cache.shape[0], c["D"], c["Hkv"], c["page"]
    kb = page * D // 2
    view = cache.view(P, Hkv, page * (D + 8))
    lim = torch.tensor([b for b, _ in BORDERS], device="cuda")
    step = max(1, (1 << 25) // (Hkv * page * D))
    for a in range(0, P, step):
        n = min(step, P - a)
        for which in (0, 1):
            x = _randn(g, n, Hkv, page, D) * torch.exp(0.3 * _randn(g, n, Hkv, page, 1))
            scale = x.abs().amax(3, keepdim=True) / 6
            y = x / scale
            code = torch.bucketize(y.abs(), lim).to(torch.uint8) | ((y < 0).to(torch.uint8) << 3)
            byte = code[..., 0::2] | (code[..., 1::2] << 4)
            if which == 0:
                byte = byte.view(n, Hkv, page // 16, 16, 4, D // 8).transpose(3, 4)
            else:
                byte = byte.view(n, Hkv, page // 4, 4, 16, D // 32).transpose(3, 4)
            view[a:a + n, :, which * kb:(which + 1) * kb] = byte.reshape(n, Hkv, kb)
            view[a:a + n, :, 2 * kb + 4 * page * which:2 * kb + 4 * page * (which + 1)] = \
                scale.reshape(n, Hkv, page).contiguous().view(torch.uint8)


def _inputs(c, seed):
    g = _gen(seed)
    s = {"case": c}
    D, Hkv, Hq, page = c["D"], c["Hkv"], c["Hq"], c["page"]
    dt = DTYPES[c["in"]]
    if c["op"] == "plan":
        old, new = _plan_lengths(c)
        R, W = c["R"], c["blocks"]
        held = [-(-n // page) for n in old]
        need = sum(-(-(o + n) // page) for o, n in zip(old, new)) - sum(held)
        pages = torch.randperm(sum(held) + need + 100, generator=g, device="cuda").int()
        nb = torch.tensor(held, device="cuda")
        table = torch.full((R, W), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(W, device="cuda")[None, :] < nb[:, None]] = pages[:sum(held)]
        s.update(pages=pages.numel(), seq_lens=torch.tensor(old, dtype=torch.int32, device="cuda"),
                 new_lens=torch.tensor(new, dtype=torch.int32, device="cuda"), block_table=table,
                 free_pages=torch.cat((pages[sum(held):], pages[:sum(held)])).contiguous(),
                 free_count=torch.tensor([need + 100], dtype=torch.int32, device="cuda"))
        return s
    if c["op"] in ("append", "read"):
        T = c["T"]
        P = -(-T // page) + 3
        slots = torch.randperm(P, generator=g, device="cuda")[:, None] * page + torch.arange(page, device="cuda")
        slots = slots.flatten()[:T].int().contiguous()
        cache = torch.zeros(P, _page_bytes(c), dtype=torch.uint8, device="cuda")
        s.update(pages=P, blocks=P, cache=cache, slots=slots)
        if c["op"] == "read":
            _fill_pages(c, g, cache)
            return s
        heads = c["Hq"] + 2 * Hkv if c["fused"] else 2 * Hkv
        x = _randn(g, T, heads, D) * torch.exp(0.3 * _randn(g, T, 1, 1))
        # the same few channels of K carry outliers in every token
        hot = torch.randperm(D, generator=g, device="cuda")[:4]
        x[:, -2 * Hkv:-Hkv, hot] *= 6.0
        x = x.to(dt)
        s.update(k=x[:, -2 * Hkv:-Hkv], v=x[:, -Hkv:])
        if c["rope"]:
            s.update(positions=torch.arange(T, device="cuda", dtype=torch.int32), rope=_rope_table(P * page, D))
        return s
    lens, qs = _lengths(c)
    nb = [-(-n // page) for n in lens]
    P, W = sum(nb) + 2, max(nb) + 1
    perm = torch.randperm(P, generator=g, device="cuda").int()
    table = torch.full((c["R"], W), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(W, device="cuda")[None, :] < torch.tensor(nb, device="cuda")[:, None]] = perm[:sum(nb)]
    cache = torch.empty(P, _page_bytes(c), dtype=torch.uint8, device="cuda")
    _fill_pages(c, g, cache)
    start = [0]
    for q in qs:
        start.append(start[-1] + q)
    T = start[-1] + c["pad"]
    s.update(pages=P, blocks=W, cache=cache, block_table=table, lens=lens, qs=qs, start=start, T=T,
             q=(_randn(g, T, Hq, D) * 1.5).to(dt), max_q=max(qs),
             q_start=torch.tensor(start, dtype=torch.int32, device="cuda"),
             seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if c["rope"]:
        s["rope"] = _rope_table(W * page, D)
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    od = DTYPES[c["out"]]
    if c["op"] == "plan":
        R, cap = c["R"], c["capacity"]
        for name, n in (("q_start", R + 1), ("positions", cap), ("slots", cap), ("seq_out", R), ("count_out", 1),
                        ("status", 4)):
            s[name] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif c["op"] == "attn":
        s["o"] = torch.zeros(s["T"], c["Hq"], c["D"], dtype=od, device="cuda")
        s["lse"] = torch.zeros(s["T"], c["Hq"], dtype=torch.float32, device="cuda")
    else:
        s["k_out"] = torch.zeros(c["T"], c["Hkv"], c["D"], dtype=od, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
    if own:
        from paper_2607_02584_amd import rotate_attn as ra
        dts = {"bf16": ra.BF16, "fp16": ra.FP16, "fp32": ra.FP32}
        s["p"] = ra.make_cache_params(
            c["Hq"], c["Hkv"], c["D"], page_size=c["page"], num_pages=s["pages"],
            max_blocks=c["blocks"] if c["op"] == "plan" else s["blocks"],
            rotation=ra.ROT_HADAMARD if c["hadamard"] else ra.ROT_NONE,
            v_rotation=ra.VROT_HADAMARD if c["v_hadamard"] else ra.VROT_NONE, causal=c.get("causal", True),
            window=c.get("window", 0), in_dtype=dts[c["in"]], out_dtype=dts[c["out"]])
        if c["op"] == "attn":
            s["ws"] = ra.cache_workspace(s["p"], c["R"], s["T"], s["max_q"])
    return s


# --------------------------------------------------------------- plain form --

def _butterflies(x):
    """Rows times the Sylvester-Hadamard matrix of +-1."""
    n = x.shape[-1]
    h = 1
    while h < n:
        y = x.reshape(*x.shape[:-1], n // (2 * h), 2, h)
        x = torch.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).reshape(x.shape)
        h *= 2
    return x


def _turn(x, cs):
    """Adjacent pairs of [T, H, D] turned by [T, D/2, 2] cosines and sines."""
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)


def _plain_plan(s):
    c = s["case"]
    page, cap, W = c["page"], c["capacity"], c["blocks"]
    old, new = s["seq_lens"].long(), s["new_lens"].long()
    after = old + new
    first = torch.zeros(c["R"] + 1, dtype=torch.int64, device=old.device)
    first[1:] = torch.cumsum(new, 0)
    had, has = (old + page - 1) // page, (after + page - 1) // page
    take = has - had
    base = torch.cumsum(take, 0) - take
    blk = torch.arange(W, device=old.device)[None, :]
    count = s["free_count"].long()
    at = (count - 1 - (base[:, None] + blk - had[:, None])).clamp(0, s["free_pages"].numel() - 1)
    fresh = (blk >= had[:, None]) & (blk < has[:, None])
    table = torch.where(fresh, s["free_pages"][at], s["block_table"])
    t = torch.arange(cap, device=old.device)
    r = (torch.searchsorted(first, t, right=True) - 1).clamp(0, c["R"] - 1)
    pos = old[r] + t - first[r]
    live = t < first[-1]
    slot = table[r, torch.where(live, pos, 0) // page].long() * page + pos % page
    none = torch.full_like(t, -1)
    status = torch.cat((torch.zeros_like(count), take.sum()[None], first[-1:], after.max()[None]))
    return {"block_table": table, "seq_lens": after.int(), "free_count": (count - take.sum()).int(),
            "q_start": first.int(), "positions": torch.where(live, pos, none).int(),
            "slots": torch.where(live, slot, none).int(), "status": status.int()}


def _plain_values(x, hadamard, out):
    """What [T, H, D] rows (64 bits: codes next to a border) stand for after
    the cache, in the basis they came in."""
    D = x.shape[-1]
    if hadamard:
        x = _butterflies(x)
    amax = x.abs().amax(-1, keepdim=True)
    y = torch.where(amax > 0, x * 6.0 / amax, torch.zeros_like(x))
    mag = torch.zeros_like(y)
    for (border, up), low, high in zip(BORDERS, MAGNITUDES, MAGNITUDES[1:]):
        mag += ((y.abs() >= border) if up else (y.abs() > border)).to(y.dtype) * (high - low)
    val = (torch.sign(y) * mag).float() * (amax / 6.0).float()
    if hadamard:
        val = _butterflies(val) * (1.0 / D)
    return val.to(out)


def _plain_append(s):
    c = s["case"]
    out = DTYPES[c["out"]]
    ks, vs = [], []
    for a in range(0, c["T"], 4096):
        k = s["k"][a:a + 4096].double()
        if c["rope"]:
            k = _turn(k, s["rope"][s["positions"][a:a + 4096].long()].double())
        ks.append(_plain_values(k, c["hadamard"], out))
        vs.append(_plain_values(s["v"][a:a + 4096].double(), c["v_hadamard"], out))
    return torch.cat(ks), torch.cat(vs)


def _plain_dense(c, cache, pages):
    """K and V of whole pages, as stored: [pages * page, Hkv, D] in 32 bits."""
    D, Hkv, page = c["D"], c["Hkv"], c["page"]
    n, kb = pages.numel(), page * D // 2
    raw = cache[pages].view(n, Hkv, page * (D + 8))
    lut = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=cache.device)
    out = []
    for which in (0, 1):
        byte = raw[:, :, which * kb:(which + 1) * kb]
        if which == 0:
            byte = byte.reshape(n, Hkv, page // 16, 4, 16, D // 8).transpose(3, 4)
        else:
            byte = byte.reshape(n, Hkv, page // 4, 16, 4, D // 32).transpose(3, 4)
        byte = byte.reshape(n, Hkv, page, D // 2)
        val = lut[torch.stack((byte & 15, byte >> 4), -1).flatten(-2).int()]
        at = 2 * kb + 4 * page * which
        scale = raw[:, :, at:at + 4 * page].contiguous().view(torch.float32)
        out.append((val * scale[..., None]).transpose(1, 2).reshape(n * page, Hkv, D))
    return out


def _plain_read(s):
    c = s["case"]
    out, D = DTYPES[c["out"]], c["D"]
    ks, vs = [], []
    for a in range(0, c["T"], 16384):
        slots = s["slots"][a:a + 16384].long()
        pages, where = torch.unique_consecutive(slots // c["page"], return_inverse=True)
        k, v = (x[where * c["page"] + slots % c["page"]] for x in _plain_dense(c, s["cache"], pages))
        ks.append((_butterflies(k) * D ** -0.5 if c["hadamard"] else k).to(out))
        vs.append((_butterflies(v) * D ** -0.5 if c["v_hadamard"] else v).to(out))
    return torch.cat(ks), torch.cat(vs)


def _plain_attn(s):
    c = s["case"]
    D, Hq, Hkv, page = c["D"], c["Hq"], c["Hkv"], c["page"]
    G = Hq // Hkv
    o, lse = torch.zeros_like(s["o"]), torch.zeros_like(s["lse"])
    for r, (n, q) in enumerate(zip(s["lens"], s["qs"])):
        if q == 0:
            continue
        k, v = _plain_dense(c, s["cache"], s["block_table"][r, :-(-n // page)].long())
        kt = k[:n].permute(1, 2, 0).contiguous()          # [Hkv, D, n]
        v = v[:n].transpose(0, 1).contiguous()            # [Hkv, n, D]
        rows = max(1, (1 << 28) // (Hq * n))
        for a in range(0, q, rows):
            m = min(rows, q - a)
            x = s["q"][s["start"][r] + a:s["start"][r] + a + m].float()
            pos = torch.arange(n - q + a, n - q + a + m, device=x.device)
            if c["rope"]:
                x = _turn(x, s["rope"][pos])
            if c["hadamard"]:
                x = _butterflies(x) * D ** -0.5
            x = x.view(m, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, m * G, D)
            t = torch.matmul(x, kt).mul_(D ** -0.5).view(Hkv, m, G, n)
            key = torch.arange(n, device=x.device)[None, :]
            dead = key > pos[:, None] if c["causal"] else key > n
            if c["window"]:
                dead = dead | (key <= pos[:, None] - c["window"])
            t.masked_fill_(dead[None, :, None, :], -math.inf)
            top = t.amax(3, keepdim=True)
            t.sub_(top).exp_()
            den = t.sum(3, keepdim=True)
            y = torch.matmul(t.view(Hkv, m * G, n), v).view(Hkv, m, G, D) / den
            if c["v_hadamard"]:
                y = _butterflies(y) * D ** -0.5
            at = slice(s["start"][r] + a, s["start"][r] + a + m)
            o[at] = y.permute(1, 0, 2, 3).reshape(m, Hq, D).to(o.dtype)
            lse[at] = (top + torch.log(den))[..., 0].permute(1, 0, 2).reshape(m, Hq)
    return o, lse


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"plan": _plain_plan, "append": _plain_append, "read": _plain_read, "attn": _plain_attn}[op](s)
    from paper_2607_02584_amd import rotate_attn as ra
    p = s["p"]
    if op == "plan":
        ra.cache_plan(p, s["seq_lens"], s["new_lens"], s["block_table"], s["free_pages"], s["free_count"],
                      s["q_start"], s["positions"], s["slots"], s["status"], seq_out=s["seq_out"],
                      count_out=s["count_out"])
        return {"block_table": s["block_table"], "seq_lens": s["seq_out"], "free_count": s["count_out"],
                "q_start": s["q_start"], "positions": s["positions"], "slots": s["slots"], "status": s["status"]}
    if op == "attn":
        ra.cache_attn(p, s["q"], s["cache"], s["block_table"], s["q_start"], s["seq_lens"], s["max_q"], s["o"],
                      s["ws"], lse=s["lse"], rope=s.get("rope"))
        return s["o"], s["lse"]
    if op == "append":
        ra.cache_append(p, s["k"], s["v"], s["slots"], s["cache"], positions=s.get("positions"), rope=s.get("rope"))
    ra.cache_read(p, s["cache"], s["slots"], s["k_out"], s["v_out"])
    return s["k_out"], s["v_out"]


# ------------------------------------------------------------------ 64 bits --

def _matrix(D):
    """The orthonormal Sylvester-Hadamard matrix: sign (-1)^(bits that i and j share)."""
    i = torch.arange(D, device="cuda")
    both = i[:, None] & i[None, :]
    odd = torch.zeros_like(both)
    for b in range(D.bit_length()):
        odd ^= (both >> b) & 1
    return (1.0 - 2.0 * odd.double()) / math.sqrt(D)


def _exact_codes(x):
    """Nearest E2M1 multiple of amax / 6, ties to the even code."""
    amax = x.abs().amax(-1, keepdim=True)
    y = x * 6.0 / torch.where(amax > 0, amax, torch.ones_like(amax))
    edge = torch.tensor([b for b, _ in BORDERS], dtype=torch.float64, device=x.device)
    low = torch.bucketize(y.abs().contiguous(), edge, right=False)
    high = torch.bucketize(y.abs().contiguous(), edge, right=True)
    code = torch.where((low != high) & (low % 2 == 1), high, low)
    mag = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)[code]
    return torch.where(y < 0, -mag, mag) * (amax / 6.0)


def _exact_token(c, cache, page_ids, offsets):
    """K and V [n, Hkv, D] in 64 bits of single tokens, byte by byte from the layout."""
    D, Hkv, page = c["D"], c["Hkv"], c["page"]
    d = torch.arange(D, device="cuda")
    t = offsets[:, None]
    at_k = (t // 16) * 8 * D + (d // (D // 4)) * 2 * D + (t % 16) * (D // 8) + (d % (D // 4)) // 2
    at_v = page * D // 2 + (t // 4) * 2 * D + (d // (D // 16)) * (D // 8) + (t % 4) * (D // 32) + (d % (D // 16)) // 2
    mag = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    head = torch.arange(Hkv, device="cuda")[None, :, None] * page * (D + 8)
    out = []
    for which, at in enumerate((at_k, at_v)):
        byte = cache[page_ids[:, None, None], head + at[:, None, :]].int()
        code = torch.where(d % 2 == 1, byte >> 4, byte & 15)
        val = mag[code & 7] * (1.0 - 2.0 * (code >> 3).double())
        place = page * D + which * 4 * page + 4 * offsets[:, None, None] + torch.arange(4, device="cuda")
        scale = cache[page_ids[:, None, None], head + place].contiguous().view(torch.float32).double()
        out.append(val * scale)
    return out


def exact(case, seed):
    c = case
    if c["op"] == "plan":
        return None
    if c["op"] == "attn" and work(c)["flops"] > 3e12:
        return None
    s = _inputs(c, seed)
    D, Hq, Hkv, page = c["D"], c["Hq"], c["Hkv"], c["page"]
    H = _matrix(D)
    one = torch.eye(D, dtype=torch.float64, device="cuda")
    RK, RV = H if c["hadamard"] else one, H if c["v_hadamard"] else one

    def angles(x, pos):
        if not c["rope"]:
            return x
        z = torch.view_as_complex(x.reshape(*x.shape[:-1], D // 2, 2).contiguous())
        w = torch.view_as_complex(s["rope"][pos].double().contiguous())
        return torch.view_as_real(z * w[:, None, :]).flatten(-2)

    if c["op"] != "attn":
        T = c["T"]
        k = torch.empty(T, Hkv, D, dtype=torch.float64, device="cuda")
        v = torch.empty_like(k)
        for a in range(0, T, 8192):
            b = min(T, a + 8192)
            if c["op"] == "append":
                x = angles(s["k"][a:b].double(), s["positions"][a:b].long() if c["rope"] else None)
                # codes from the sums before the orthonormal factor, so that a tie stays one
                k[a:b] = _exact_codes(x @ (RK * (math.sqrt(D) if c["hadamard"] else 1.0)).round()) @ RK
                v[a:b] = _exact_codes(s["v"][a:b].double() @ (RV * (math.sqrt(D) if c["v_hadamard"] else 1.0)).round()) @ RV
                if c["hadamard"]:
                    k[a:b] /= math.sqrt(D)
                if c["v_hadamard"]:
                    v[a:b] /= math.sqrt(D)
            else:
                slots = s["slots"][a:b].long()
                x, y = _exact_token(c, s["cache"], slots // page, slots % page)
                k[a:b], v[a:b] = x @ RK, y @ RV
        return k, v
    o = torch.zeros(s["T"], Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["T"], Hq, dtype=torch.float64, device="cuda")
    G = Hq // Hkv
    for r, (n, q) in enumerate(zip(s["lens"], s["qs"])):
        if q == 0:
            continue
        key = torch.arange(n, device="cuda")
        ids = s["block_table"][r].long()[key // page]
        k = torch.empty(n, Hkv, D, dtype=torch.float64, device="cuda")
        v = torch.empty_like(k)
        for a in range(0, n, 16384):
            k[a:a + 16384], v[a:a + 16384] = _exact_token(c, s["cache"], ids[a:a + 16384], key[a:a + 16384] % page)
        x = s["q"][s["start"][r]:s["start"][r] + q].double()
        pos = torch.arange(n - q, n, device="cuda")
        x = angles(x, pos) @ RK
        step = max(1, (1 << 26) // n)
        for h in range(Hq):
            kh, vh = k[:, h // G].t().contiguous(), v[:, h // G].contiguous()
            for a in range(0, q, step):
                t = x[a:a + step, h] @ kh / math.sqrt(D)
                p = pos[a:a + step, None]
                seen = key[None, :] <= p if c["causal"] else (key >= 0).expand(t.shape)
                if c["window"]:
                    seen = seen & (key[None, :] > p - c["window"])
                t = torch.where(seen, t, torch.full_like(t, -math.inf))
                z = torch.logsumexp(t, 1)
                at = slice(s["start"][r] + a, s["start"][r] + min(q, a + step))
                lse[at, h] = z
                o[at, h] = (torch.exp(t - z[:, None]) @ vh) @ RV
    return o, lse
