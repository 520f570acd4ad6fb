"""What serving on the 4-bit paged KV cache does with requests that begin alike,
are rolled back, or run on and on: the operators these are measured on.

Pages (tables, holders and the stack of free pages; bytes are copied, never
decoded):

  fork     requests that begin as another one does: they share its full pages
           and get a copy of the page it is filling
  trim     requests end, drop the last tokens of a rejected draft, or lose the
           pages that a sliding window has left behind; what nobody holds goes
           back on the stack
  compact  the pages in use move to the front of the cache

Attention over the cache:

  shared   queries of requests whose first tokens are the same pages; these are
           read once for all of them
  sinks    a sliding window, and a few first tokens that stay visible

A page holds, for each KV head in turn, the K codes, the V codes, the K scales
and the V scales of `page` tokens (binary32 scales, one per token):
  K code of (token t, channel d): byte (t/16)*8D + (d/(D/4))*2D + (t%16)*(D/8) + (d%(D/4))/2
  V code of (token t, channel d): byte (t/4)*2D + (d/(D/16))*(D/8) + (t%4)*(D/32) + (d%(D/16))/2
with channel d in the low nibble where d is even; a code is a sign (bit 3) and
one of the magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6.  page_refs counts the holders of
a page beyond the first.

Shapes: 12, 24 and 40 heads of 128 are this library's own layers; grouped heads,
heads of 64 and the page sizes are generic.  `own` chooses between the plain form
(elementary torch operations in 32 bits or more) and the library's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
COMMON = {"Hq": 32, "Hkv": 8, "D": 128, "page": 64, "in": "bf16", "out": "bf16", "rope": True, "hadamard": True,
          "v_hadamard": False}


def _case(op, **kw):
    return dict(COMMON, op=op, ragged=1, **kw)


def listed():
    return [
        # best of four: three more continuations of one request begin (latency)
        _case("fork", name="fork_beam", Hq=12, Hkv=12, R=8, parents=1, children=3, len_min=1000, len_max=1000),
        # a batch begins on one system prompt, heads not grouped, large pages:
        # the last pages of 255 requests, 1.4 MB each
        _case("fork", name="fork_prompt", Hq=40, Hkv=40, page=256, R=256, parents=1, children=255, len_min=24001,
              len_max=24001),
        # sixteen requests drop what was rejected of their drafts (latency)
        _case("trim", name="trim_draft", R=16, drafts=16, draft=5, done=0, groups=0, len_min=50, len_max=4000,
              window=0, sinks=0),
        # a step of a server with a thousand requests under a window: some end,
        # some drop drafts, all lose pages behind the window, prompts are shared
        _case("trim", name="trim_server", Hq=24, page=16, R=1000, drafts=300, draft=40, done=100, groups=30,
              len_min=20, len_max=3500, window=1024, sinks=16),
        # a small cache is put in order between two steps
        _case("compact", name="compact_small", Hq=12, Hkv=12, page=16, R=8, pages=500, live=0.5),
        # half of a 2.8 GB cache has become free: the rest moves together
        _case("compact", name="compact_large", R=300, pages=40000, live=0.5),
        # four continuations of one prompt on a 12-head layer (latency)
        _case("shared", name="shared_beam", Hq=12, Hkv=12, R=4, groups=1, loose=0, prefix_min=1000, prefix_max=1000,
              own_min=1, own_max=40, q_max=1, pad=0),
        # a decode step of 64 requests on one long system prompt
        _case("shared", name="shared_decode", R=64, groups=1, loose=0, prefix_min=32700, prefix_max=32700, own_min=1,
              own_max=1500, q_max=1, pad=0),
        # five documents asked about by 190 requests, ten others beside them,
        # drafts of up to 4 tokens, 40-head layer, binary16, padded batch
        _case("shared", name="shared_documents", Hq=40, R=200, groups=5, loose=10, prefix_min=3000, prefix_max=60000,
              own_min=4, own_max=1000, q_max=4, pad=11, v_hadamard=True, page=32, **{"in": "fp16", "out": "fp16"}),
        # one long-running request, one token: latency
        _case("sinks", name="sinks_single", Hq=12, Hkv=12, D=64, page=16, R=1, singles=1, q_min=1, q_max=1,
              len_min=30001, len_max=30001, window=1024, sinks=4, pad=0, **{"out": "fp32"}),
        # a decode step of 256 long-running requests; the pages between the
        # first tokens and the window are gone
        _case("sinks", name="sinks_decode", R=256, singles=256, q_min=1, q_max=1, len_min=100, len_max=60000,
              window=4000, sinks=64, pad=0),
        # prompts under a window on a 24-head layer, beside two decoding requests
        _case("sinks", name="sinks_prompt", Hq=24, R=5, singles=2, q_min=1000, q_max=8000, len_min=1500,
              len_max=12000, window=2000, sinks=100, pad=3),
    ]


# below the largest listed calls: multiply-adds of attention, bytes of a cache, page tables
_MOST_FLOPS, _MOST_CACHE, _MOST_TABLE = 5e11, 2.7e9, 1 << 19


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges."""
    c = dict(COMMON)
    c["D"] = rng.choice([128, 128, 64])
    c["page"] = rng.choice([16, 32, 64, 64, 128, 256])
    c["Hq"], c["Hkv"] = rng.choice([(12, 12), (24, 8), (40, 8), (32, 8), (32, 4), (16, 16), (8, 1), (28, 4), (40, 40)])
    c["in"] = rng.choice(["bf16", "bf16", "fp16"])
    c["out"] = rng.choice([c["in"], c["in"], "fp32"])
    c.update(rope=rng.random() < 0.7, hadamard=rng.random() < 0.7, v_hadamard=rng.random() < 0.3,
             ragged=rng.randrange(1 << 30))
    c["op"] = rng.choice(["fork", "trim", "compact", "shared", "shared", "shared", "sinks", "sinks", "sinks"])
    if c["op"] == "fork":
        R = _log(rng, 2, 300)
        children = rng.randint(1, R - 1)
        c.update(R=R, children=children, parents=rng.randint(1, min(4, R - children)), len_min=rng.choice([1, 300]))
        c["len_max"] = _log(rng, 300, 30000)
        while _cache_bytes(c) > _MOST_CACHE and c["children"] > 1:
            c["children"] //= 2
        while _cache_bytes(c) > _MOST_CACHE or c["R"] * c["len_max"] // c["page"] > _MOST_TABLE:
            c["len_max"] //= 2
        c["len_min"] = min(c["len_min"], c["len_max"])
        return c
    if c["op"] == "trim":
        R = _log(rng, 1, 1000)
        c.update(R=R, drafts=rng.randint(0, R), draft=_log(rng, 1, 50), groups=rng.choice([0, 0, rng.randint(1, 30)]),
                 len_min=1, len_max=_log(rng, 100, 4000), window=rng.choice([0, _log(rng, 20, 2000)]),
                 sinks=rng.choice([0, 4, rng.randint(1, 200)]))
        c["done"] = rng.randint(0, R - c["drafts"])
        c["groups"] = min(c["groups"], R)
        while _cache_bytes(c) > _MOST_CACHE or R * c["len_max"] // c["page"] > _MOST_TABLE:
            c["len_max"] = max(1, c["len_max"] // 2)
        return c
    if c["op"] == "compact":
        most = int(_MOST_CACHE / _page_bytes(c))
        c.update(pages=_log(rng, 20, min(most, 40000)), live=round(rng.uniform(0.05, 0.95), 2))
        c["R"] = rng.randint(1, min(300, max(1, int(c["pages"] * c["live"]))))
        return c
    if c["op"] == "shared":
        R = _log(rng, 1, 200)
        c.update(R=R, groups=rng.randint(1, max(1, min(6, R // 2))), prefix_min=_log(rng, 1, 3000), own_min=1,
                 own_max=_log(rng, 5, 1500), q_max=rng.choice([1, 1, 1, 4, 30]), pad=rng.choice([0, 0, rng.randint(1, 30)]))
        c["prefix_max"] = _log(rng, c["prefix_min"] + 1, 60000)
        c["loose"] = rng.choice([0, rng.randint(0, R - c["groups"])])
        shrink = ("prefix_max", "own_max", "prefix_min")
    else:
        R = _log(rng, 1, 256)
        kind = rng.choice(["decode", "decode", "prompt"])
        c.update(R=R, singles=R, q_min=1, q_max=rng.choice([1, 1, 3]), len_min=_log(rng, 1, 300),
                 len_max=_log(rng, 300, 60000), window=_log(rng, 1, 4000), sinks=rng.choice([1, 4, 4, _log(rng, 1, 300)]),
                 pad=rng.choice([0, 0, rng.randint(1, 30)]))
        if kind == "prompt":
            R = c["R"] = rng.randint(1, 6)
            c.update(singles=rng.randint(0, R - 1), q_min=2, q_max=_log(rng, 10, 8000))
        elif c["q_max"] > 1:
            c["singles"] = rng.randint(0, R)
        shrink = ("q_max", "len_max") if kind == "prompt" else ("window", "len_max")
    at = 0
    while work(c)["flops"] > _MOST_FLOPS or _cache_bytes(c) > _MOST_CACHE:
        c[shrink[at % len(shrink)]] = max(1, c[shrink[at % len(shrink)]] * 2 // 3)
        at += 1
    for low, high in (("prefix_min", "prefix_max"), ("len_min", "len_max"), ("q_min", "q_max"), ("own_min", "own_max")):
        if low in c:
            c[low] = min(c[low], c[high])
    return c


# ------------------------------------------------------------------ lengths --

def _up(n, page):
    return -(-n // page)


def _page_bytes(c):
    return c["Hkv"] * c["page"] * (c["D"] + 8)


def _fork_plan(c):
    """Lengths [R] and pairs (parent, child) (from the case alone)."""
    rng = random.Random(c["ragged"])
    order = list(range(c["R"]))
    rng.shuffle(order)
    parents, children = order[:c["parents"]], order[c["parents"]:c["parents"] + c["children"]]
    lens = [0] * c["R"]
    for r in parents + order[c["parents"] + c["children"]:][:4]:     # a few others run beside them
        lens[r] = rng.randint(c["len_min"], c["len_max"])
    return lens, [(parents[i % len(parents)], x) for i, x in enumerate(children)]


def _trim_plan(c):
    """Lengths, tokens kept (-1: all), prefix that a request shares with its group, and the group (from the case alone)."""
    rng = random.Random(c["ragged"])
    R, page = c["R"], c["page"]
    lens = [rng.randint(c["len_min"], c["len_max"]) for _ in range(R)]
    keep = [-1] * R
    order = list(range(R))
    rng.shuffle(order)
    for r in order[:c["drafts"]]:
        keep[r] = max(0, lens[r] - rng.randint(0, c["draft"]))
    for r in order[c["drafts"]:c["drafts"] + c["done"]]:
        keep[r] = 0
    group = [rng.randrange(2 * c["groups"]) if c["groups"] else 0 for _ in range(R)]
    shared = [0] * R
    for g in range(c["groups"]):          # the other numbers are requests that share nothing
        members = [r for r in range(R) if group[r] == g]
        if len(members) > 1:
            n = min(lens[r] for r in members) // page
            for r in members:
                shared[r] = n
    return lens, keep, shared, group


def _shared_plan(c):
    """group_start, prefix lengths, request lengths and query counts (from the case alone)."""
    rng = random.Random(c["ragged"])
    R, n = c["R"], c["R"] - c["loose"]
    cuts = sorted(rng.sample(range(1, n), c["groups"] - 1)) if c["groups"] > 1 else []
    first = rng.randint(0, c["loose"])
    start = [first + x for x in [0] + cuts + [n]]
    prefix = [c["prefix_max"] if g == 0 else rng.randint(min(c["prefix_min"], c["prefix_max"]), c["prefix_max"])
              for g in range(c["groups"])]
    lens, qs = [0] * R, [0] * R
    for r in range(R):
        own_len = rng.randint(min(c["own_min"], c["own_max"]), c["own_max"])
        qs[r] = min(own_len, rng.randint(1, c["q_max"]))
        lens[r] = own_len
    for g in range(c["groups"]):
        for r in range(start[g], start[g + 1]):
            lens[r] += prefix[g]
    return start, prefix, lens, qs


def _sinks_plan(c):
    """Context and query length of every request (from the case alone)."""
    rng = random.Random(c["ragged"])
    lens, qs = [], []
    for r in range(c["R"]):
        n = c["len_max"] if r == c["R"] - 1 else _log(rng, min(c["len_min"], c["len_max"]), c["len_max"])
        q = 1 if r < c["singles"] else c["q_max"] if r == c["R"] - 1 else _log(rng, min(c["q_min"], c["q_max"]), c["q_max"])
        lens.append(n)
        qs.append(min(q, n))
    order = list(range(c["R"]))
    rng.shuffle(order)
    return [lens[i] for i in order], [qs[i] for i in order]


def _sinks_blocks(c, n, q):
    """Blocks of a request that hold a key one of its queries sees."""
    page = c["page"]
    low = max(0, n - q - c["window"] + 1)
    return [j for j in range(_up(n, page)) if j * page < c["sinks"] or (j + 1) * page > low]


def _cache_bytes(c):
    page = c["page"]
    if c["op"] == "fork":
        lens, pairs = _fork_plan(c)
        return (sum(_up(n, page) for n in lens) + len(pairs) + 5) * _page_bytes(c)
    if c["op"] == "trim":
        return (sum(_up(n, page) for n in _trim_plan(c)[0]) + c["R"]) * _page_bytes(c)
    if c["op"] == "compact":
        return c["pages"] * _page_bytes(c)
    if c["op"] == "shared":
        start, prefix, lens, _ = _shared_plan(c)
        return (sum(_up(n, page) for n in lens) - sum(n // page * (start[g + 1] - start[g] - 1)
                                                      for g, n in enumerate(prefix)) + 2) * _page_bytes(c)
    return (sum(len(_sinks_blocks(c, n, q)) for n, q in zip(*_sinks_plan(c))) + 2) * _page_bytes(c)


def work(case):
    c = case
    D, Hkv, Hq, page, size = c["D"], c["Hkv"], c["Hq"], c["page"], _page_bytes(c)
    esize = 4 if c["out"] == "fp32" else 2
    if c["op"] == "fork":
        lens, pairs = _fork_plan(c)
        copies = sum(lens[a] % page > 0 for a, _ in pairs)
        entries = sum(_up(lens[a], page) for a, _ in pairs)
        # pages both ways; the children's entries, their parents' once; lengths and holders
        return {"bytes": 2 * copies * size + 4 * (entries + sum(_up(n, page) for n in lens) + 2 * c["R"]) + 8 * len(pairs),
                "flops": entries}
    if c["op"] == "trim":
        lens, keep, shared, _ = _trim_plan(c)
        entries = pages = copies = 0
        for n, k, sh in zip(lens, keep, shared):
            k = n if k < 0 else k
            held, left = _up(n, page), _up(k, page)
            first, last = (_up(c["sinks"], page), max(0, k - c["window"] + 1) // page) if c["window"] else (0, 0)
            entries += held - left + max(0, min(last, left) - first)
            copies += k % page > 0 and k // page < sh
            pages += held
        # tables in and out, the holders of each released entry, the stack, lengths
        return {"bytes": 2 * copies * size + 8 * pages + 12 * entries + 12 * c["R"], "flops": 4 * pages}
    if c["op"] == "compact":
        live = max(c["R"], int(c["pages"] * c["live"]))
        moves = live * (c["pages"] - live) / c["pages"]       # of a random half, say, half has to move
        return {"bytes": 2 * moves * size + 8 * c["pages"] + 8 * live, "flops": 4 * c["pages"]}
    if c["op"] == "shared":
        start, prefix, lens, qs = _shared_plan(c)
        own_keys, pairs = sum(lens), 0
        for g, n in enumerate(prefix):
            own_keys -= n * (start[g + 1] - start[g])
        keys = own_keys + sum(prefix)
        pairs = sum(q * n - q * (q - 1) // 2 for n, q in zip(lens, qs))
    else:
        lens, qs = _sinks_plan(c)
        keys = pairs = 0
        for n, q in zip(lens, qs):
            low = max(0, n - q - c["window"] + 1)
            keys += n - low + min(c["sinks"], low)
            # query at position p sees min(p + 1, window) of the window and the first tokens before it
            full = min(n, c["sinks"] + c["window"])
            edge = max(0, min(q, full - (n - q)))             # queries that see everything before them
            pairs += edge * (n - q) + edge * (edge + 1) // 2 + (q - edge) * full
    T = sum(qs)
    return {"bytes": keys * Hkv * (D + 8) + T * Hq * (D * (2 + esize) + 4) + (T * D * 4 if c["rope"] else 0),
            "flops": 4 * D * Hq * pairs}


# ------------------------------------------------------------------- inputs --

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rope_table(rows, D):
    """[rows, D/2, 2] cosines and sines: binary64 angles, rounded once."""
    pos = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None]
    freq = 10000.0 ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    ang = pos * freq[None, :]
    return torch.stack((torch.cos(ang), torch.sin(ang)), 2).float().contiguous()


def _random_cache(c, g, pages):
    """Pages of anything: their operators move bytes."""
    words = torch.empty(pages, _page_bytes(c) // 4, dtype=torch.int32, device="cuda")
    words.random_(-2 ** 31, 2 ** 31 - 1, generator=g)
    return words.view(torch.uint8)


def _fill_pages(c, g, cache):
    """Pages of keys and values as a model leaves them: normal channels, token
    gains that vary, quantised and packed."""
    P, D, Hkv, page = cache.shape[0], c["D"], c["Hkv"], c["page"]
    kb = page * D // 2
    view = cache.view(P, Hkv, page * (D + 8))
    lim = torch.tensor((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0), device="cuda")
    step = max(1, (1 << 27) // (Hkv * page * D))
    for a in range(0, P, step):
        n = min(step, P - a)
        for which in (0, 1):
            x = torch.randn(n, Hkv, page, D, generator=g, device="cuda")
            gain = torch.exp(0.3 * torch.randn(n, Hkv, page, 1, generator=g, device="cuda"))
            top = x.abs().amax(3, keepdim=True)
            code = torch.bucketize(x.abs() * (6 / top), lim, out_int32=True).to(torch.uint8) | ((x < 0).to(torch.uint8) << 3)
            byte = code[..., 0::2] | (code[..., 1::2] << 4)
            if which == 0:
                byte = byte.view(n, Hkv, page // 16, 16, 4, D // 8).transpose(3, 4)
            else:
                byte = byte.view(n, Hkv, page // 4, 4, 16, D // 32).transpose(3, 4)
            view[a:a + n, :, which * kb:(which + 1) * kb] = byte.reshape(n, Hkv, kb)
            view[a:a + n, :, 2 * kb + 4 * page * which:2 * kb + 4 * page * (which + 1)] = \
                (gain * top / 6).reshape(n, Hkv, page).contiguous().view(torch.uint8)


def _state(s, table, perm, used, lens):
    """Tables and stack: pages perm[:used] are held, the others free."""
    P = perm.numel()
    s.update(pages=P, blocks=table.shape[1], block_table=table.contiguous(), seq_lens=_i32(lens),
             free_pages=torch.cat((perm[used:], perm[:used])).contiguous(), free_count=_i32([P - used]),
             page_refs=torch.zeros(P, dtype=torch.int32, device="cuda"))


def _table(c, W, blocks, perm):
    """Block table [R, W] whose row r holds blocks[r] pages, taken from perm in order."""
    nb = torch.tensor(blocks, device="cuda")
    table = torch.full((c["R"], W), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(W, device="cuda")[None, :] < nb[:, None]] = perm[:sum(blocks)]
    return table


def _inputs(c, seed):
    g = _gen(seed)
    s = {"case": c}
    page, R = c["page"], c["R"]
    perm_of = lambda n: torch.randperm(n, generator=g, device="cuda").int()
    if c["op"] == "fork":
        lens, pairs = _fork_plan(c)
        nb = [_up(n, page) for n in lens]
        perm = perm_of(sum(nb) + len(pairs) + 5)
        _state(s, _table(c, max(nb) + 1, nb, perm), perm, sum(nb), lens)
        s.update(parents=_i32([a for a, _ in pairs]), children=_i32([b for _, b in pairs]),
                 cache=_random_cache(c, g, s["pages"]))
        return s
    if c["op"] == "trim":
        lens, keep, shared, group = _trim_plan(c)
        nb = [_up(n, page) for n in lens]
        W = max(max(nb), 1)
        perm = perm_of(sum(nb) + R + 3)
        table = _table(c, W, nb, perm).cpu()
        free, used, first = [], torch.ones(perm.numel(), dtype=torch.bool), {}
        for r in range(R):              # members of a group hold the first one's pages
            if shared[r]:
                a = first.setdefault(group[r], r)
                if a != r:
                    free += table[r, :shared[r]].tolist()
                    table[r, :shared[r]] = table[a, :shared[r]]
        _state(s, table.cuda(), perm, sum(nb), lens)
        held = torch.bincount(table[table >= 0].long(), minlength=perm.numel())
        s["page_refs"] = (held - 1).clamp(min=0).int().cuda()
        idle = perm.cpu()[held[perm.cpu().long()] == 0]
        stack = torch.zeros(perm.numel(), dtype=torch.int32)
        stack[:idle.numel()] = idle
        s.update(free_pages=stack.cuda(), free_count=_i32([idle.numel()]), cache=_random_cache(c, g, s["pages"]),
                 keep=_i32(keep))
        return s
    if c["op"] == "compact":
        live = max(R, int(c["pages"] * c["live"]))
        rng = random.Random(c["ragged"])
        nb = [live // R + (r < live % R) for r in range(R)]
        perm = perm_of(c["pages"])
        # a tenth of the requests hold another one's first page as well
        extra = [r for r in range(1, R) if rng.random() < 0.1]
        _state(s, _table(c, max(nb) + 2, nb, perm), perm, live, [(n + (r in extra)) * page for r, n in enumerate(nb)])
        s["cache"] = _random_cache(c, g, s["pages"])
        for r in extra:
            s["block_table"][r, nb[r]] = s["block_table"][0, 0]
        s["page_refs"][s["block_table"][0, 0].long()] = len(extra)
        return s
    D, Hq = c["D"], c["Hq"]
    if c["op"] == "shared":
        start, prefix, lens, qs = _shared_plan(c)
        nb = [_up(n, page) for n in lens]
        own_nb = list(nb)
        for gi, n in enumerate(prefix):
            for r in range(start[gi] + 1, start[gi + 1]):
                own_nb[r] -= n // page
        perm = perm_of(sum(own_nb) + 2)
        W = max(nb) + 1
        table = torch.full((R, W), -1, dtype=torch.int32, device="cuda")
        cache = torch.empty(perm.numel(), _page_bytes(c), dtype=torch.uint8, device="cuda")
        _fill_pages(c, g, cache)
        at = 0
        for r in range(R):
            table[r, nb[r] - own_nb[r]:nb[r]] = perm[at:at + own_nb[r]]
            at += own_nb[r]
        for gi, n in enumerate(prefix):
            a, b, full = start[gi], start[gi + 1], n // page
            if b > a + 1:
                table[a + 1:b, :full] = table[a, :full]
                if n % page:              # the page that the prefix ends in is the request's own copy
                    cache[table[a + 1:b, full].long()] = cache[table[a, full].long()].clone()
        s.update(group_start=_i32(start), prefix_lens=_i32(prefix), start_of=start, prefix=prefix)
    else:
        lens, qs = _sinks_plan(c)
        blocks = [_sinks_blocks(c, n, q) for n, q in zip(lens, qs)]
        W = max(_up(n, page) for n in lens) + 1
        perm = perm_of(sum(len(b) for b in blocks) + 2)
        table = torch.full((R, W), -1, dtype=torch.int32, device="cuda")
        rows = torch.tensor([r for r in range(R) for _ in blocks[r]], device="cuda")
        cols = torch.tensor([j for b in blocks for j in b], device="cuda")
        table[rows, cols] = perm[:rows.numel()]
        cache = torch.empty(perm.numel(), _page_bytes(c), dtype=torch.uint8, device="cuda")
        _fill_pages(c, g, cache)
        s.update(blocks_of=blocks)
    first = [0]
    for q in qs:
        first.append(first[-1] + q)
    T = first[-1] + c["pad"]
    pos = [n - q + i for n, q in zip(lens, qs) for i in range(q)]
    s.update(pages=perm.numel(), blocks=W, block_table=table, cache=cache, lens=lens, qs=qs, first=first, T=T,
             seq_lens=_i32(lens), q_start=_i32(first), positions=_i32(pos + [-1] * c["pad"]), max_q=max(qs),
             q=(torch.randn(T, Hq, D, generator=g, device="cuda") * 1.5).to(DTYPES[c["in"]]))
    if c["rope"]:
        s["rope"] = _rope_table(W * page, D)
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] in ("fork", "trim", "compact"):
        # what a step that is still running reads stays as it is: tables, holders and stack go into buffers of their own
        for name, of in (("seq_out", "seq_lens"), ("table_out", "block_table"), ("refs_out", "page_refs"),
                         ("free_out", "free_pages"), ("count_out", "free_count")):
            s[name] = torch.zeros_like(s[of])
        s["status"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    else:
        s["o"] = torch.zeros(s["T"], c["Hq"], c["D"], dtype=DTYPES[c["out"]], device="cuda")
        s["lse"] = torch.zeros(s["T"], c["Hq"], dtype=torch.float32, device="cuda")
    if own:
        from paper_2607_02584_amd import rotate_attn as ra
        dts = {"bf16": ra.BF16, "fp16": ra.FP16, "fp32": ra.FP32}
        s["p"] = ra.make_cache_params(
            c["Hq"], c["Hkv"], c["D"], page_size=c["page"], num_pages=s["pages"], max_blocks=s["blocks"],
            rotation=ra.ROT_HADAMARD if c["hadamard"] else ra.ROT_NONE,
            v_rotation=ra.VROT_HADAMARD if c["v_hadamard"] else ra.VROT_NONE, window=c.get("window", 0),
            in_dtype=dts[c["in"]], out_dtype=dts[c["out"]])
        if c["op"] == "sinks":
            s["ws"] = ra.cache_workspace(s["p"], c["R"], s["T"], s["max_q"])
        elif c["op"] == "shared":
            s["ws"] = ra.cache_shared_workspace(s["p"], c["R"], c["groups"], s["T"])
        else:
            s["ws"] = ra.cache_pages_workspace(s["p"], c["R"])
    return s


# --------------------------------------------------------------- plain form --

def _tables(s, status):
    """What an operator on pages leaves: tables, lengths, holders, stack and the pages' 32-bit words."""
    return {"seq_lens": s["seq_out"], "block_table": s["table_out"], "page_refs": s["refs_out"],
            "free_pages": s["free_out"], "free_count": s["count_out"], "status": status, "cache": s["cache"].view(torch.int32)}


def _plain_fork(s):
    page = s["case"]["page"]
    a, b = s["parents"].long(), s["children"].long()
    table, lens = s["block_table"], s["seq_lens"].long()
    n = lens[a]
    full, part = n // page, n % page > 0
    blk = torch.arange(s["blocks"], device=a.device)[None, :]
    rows = table[a]
    shares = (blk < full[:, None]) & (rows >= 0)
    took = torch.cumsum(part.long(), 0)
    fresh = s["free_pages"][(s["free_count"].long() - took).clamp(min=0)]
    last = rows.gather(1, full[:, None])[:, 0]
    copies = part.nonzero()[:, 0]
    s["cache"][fresh[copies].long()] = s["cache"][last[copies].long()]
    s["table_out"].copy_(table)
    keep = table[b]
    s["table_out"][b] = torch.where(blk < full[:, None], rows,
                                    torch.where((blk == full[:, None]) & part[:, None], fresh[:, None], keep))
    held = torch.zeros(s["pages"] + 1, dtype=torch.int64, device=a.device)
    held.scatter_add_(0, torch.where(shares, rows, s["pages"]).flatten().long(), shares.flatten().long())
    s["refs_out"].copy_(s["page_refs"] + held[:-1].int())
    s["seq_out"].copy_(s["seq_lens"])
    s["seq_out"][b] = n.int()
    s["count_out"].copy_(s["free_count"] - took[-1:].int())
    s["free_out"].copy_(s["free_pages"])
    return torch.stack((took[-1] * 0, took[-1], shares.sum(), s["seq_out"].max().long())).int()


def _plain_trim(s):
    c = s["case"]
    page, P = c["page"], s["pages"]
    table, refs = s["block_table"], s["page_refs"]
    n = s["seq_lens"].long()
    k = torch.where(s["keep"] < 0, n, s["keep"].long())
    held, left = (n + page - 1) // page, (k + page - 1) // page
    blk = torch.arange(s["blocks"], device=n.device)[None, :]
    drop = (blk >= left[:, None]) & (blk < held[:, None])
    if c["window"]:
        drop |= (blk * page >= c["sinks"]) & ((blk + 1) * page <= (k - c["window"] + 1)[:, None])
    at = (k // page).clamp(max=s["blocks"] - 1)
    last = table.gather(1, at[:, None])[:, 0].long()
    copy = (k % page > 0) & (last >= 0) & (refs[last.clamp(min=0)] > 0)
    took = torch.cumsum(copy.long(), 0)
    fresh = s["free_pages"][(s["free_count"].long() - took).clamp(0, P - 1)]
    rows = copy.nonzero()[:, 0]
    s["cache"][fresh[rows].long()] = s["cache"][last[rows]]
    lost = torch.zeros(P + 1, dtype=torch.int64, device=n.device)
    gone = drop & (table >= 0)
    lost.scatter_add_(0, torch.where(gone, table, P).flatten().long(), gone.flatten().long())
    lost.scatter_add_(0, torch.where(copy, last, P), copy.long())
    lost = lost[:-1]
    free = lost > refs
    s["refs_out"].copy_(torch.where(free, 0, refs - lost.int()))
    s["table_out"].copy_(torch.where(drop, -1, table))
    s["table_out"][rows, at[rows]] = fresh[rows]
    back = free.nonzero()[:, 0]
    s["free_out"].copy_(s["free_pages"])
    top = s["free_count"].long() - took[-1:]
    s["free_out"][top + torch.arange(back.numel(), device=n.device)] = back.int()
    s["count_out"].copy_(top + back.numel())
    s["seq_out"].copy_(k)
    return torch.stack((took[-1] * 0, took[-1], free.sum(), k.max())).int()


def _plain_compact(s):
    P = s["pages"]
    i = torch.arange(P, device="cuda")
    count = s["free_count"].long()
    free = torch.zeros(P + 1, dtype=torch.bool, device="cuda")
    free[torch.where(i < count, s["free_pages"].long(), P)] = True
    free = free[:P]
    live = P - count
    src = (~free & (i >= live)).nonzero()[:, 0]
    dst = (free & (i < live)).nonzero()[:, 0]
    s["cache"][dst] = s["cache"][src]
    to = i.clone()
    to[src] = dst
    table = s["block_table"]
    s["table_out"].copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table.long()))
    s["refs_out"].copy_(s["page_refs"])
    s["refs_out"][dst] = s["page_refs"][src]
    s["refs_out"][src] = 0
    s["free_out"].copy_(torch.where(i < count, P - 1 - i, s["free_pages"].long()))
    s["count_out"].copy_(s["free_count"])
    s["seq_out"].copy_(s["seq_lens"])
    return torch.cat((count * 0, count * 0 + src.numel(), live, count * 0)).int()


def _butterflies(x):
    """Rows times the Sylvester-Hadamard matrix of +-1."""
    n = x.shape[-1]
    h = 1
    while h < n:
        y = x.reshape(*x.shape[:-1], n // (2 * h), 2, h)
        x = torch.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).reshape(x.shape)
        h *= 2
    return x


def _plain_dense(c, cache, pages):
    """K and V of pages [B, n] (none where negative), as stored: [B, Hkv, n * page, D] in 32 bits."""
    D, Hkv, page = c["D"], c["Hkv"], c["page"]
    B, n = pages.shape
    kb = page * D // 2
    raw = cache[pages.clamp(min=0).flatten().long()].view(B * n, Hkv, page * (D + 8))
    lut = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=cache.device)
    out = []
    for which in (0, 1):
        byte = raw[:, :, which * kb:(which + 1) * kb]
        if which == 0:
            byte = byte.reshape(B * n, Hkv, page // 16, 4, 16, D // 8).transpose(3, 4)
        else:
            byte = byte.reshape(B * n, Hkv, page // 4, 16, 4, D // 32).transpose(3, 4)
        byte = byte.reshape(B * n, Hkv, page, D // 2)
        val = lut[torch.stack((byte & 15, byte >> 4), -1).flatten(-2).int()]
        at = 2 * kb + 4 * page * which
        scale = raw[:, :, at:at + 4 * page].contiguous().view(torch.float32)
        val = (val * scale[..., None]).view(B, n, Hkv, page, D)
        out.append(val.transpose(1, 2).reshape(B, Hkv, n * page, D))
    return out


def _padded(lists, fill):
    """Lists of numbers as a tensor, padded at their ends."""
    n = max(1, max(len(x) for x in lists))
    return torch.tensor([list(x) + [fill] * (n - len(x)) for x in lists], device="cuda")


def _partial(s, tokens, table_rows, blocks, lo, hi):
    """Softmax sums of padded queries (token numbers [B, M], -1: none) over the keys of the listed blocks [B, N]: those
    with lo <= key < hi ([B, 1]) that the mask leaves.  Maximum, sum and sum of p v, each [B, Hkv, M, G, ..]."""
    c = s["case"]
    D, Hkv, page = c["D"], c["Hkv"], c["page"]
    G = c["Hq"] // Hkv
    B, M = tokens.shape
    pages = s["block_table"][table_rows[:, None], blocks.clamp(min=0)]
    pages = torch.where(blocks < 0, -1, pages)
    k, v = _plain_dense(c, s["cache"], pages)
    key = (blocks[:, :, None] * page + torch.arange(page, device="cuda")).flatten(1)
    there = (pages >= 0)[:, :, None].expand(-1, -1, page).flatten(1) & (key >= lo) & (key < hi)
    at = tokens.clamp(min=0)
    pos = s["positions"][at].long()
    x = s["q"][at.flatten()].float()
    if c["rope"]:
        cs = s["rope"][pos.clamp(min=0).flatten()][:, None]
        a, b = x[..., 0::2], x[..., 1::2]
        x = torch.stack((a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]), -1).flatten(-2)
    if c["hadamard"]:
        x = _butterflies(x) * D ** -0.5
    x = x.view(B, M, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, M * G, D)
    t = torch.matmul(x, k.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(B, Hkv, M, G, -1)
    sees = key[:, None, :] <= pos[:, :, None]
    if c["op"] == "sinks":
        sees = sees & ((key[:, None, :] > pos[:, :, None] - c["window"]) | (key < c["sinks"])[:, None, :])
    sees = sees & there[:, None, :]
    t.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    top = t.amax(-1, keepdim=True)
    t.sub_(top.clamp(min=-1e30)).exp_()
    den = t.sum(-1, keepdim=True)
    y = torch.matmul(t.view(B, Hkv, M * G, -1), v).view(B, Hkv, M, G, D)
    return top, den, y


def _store(s, tokens, top, den, y):
    c = s["case"]
    y = y / den
    if c["v_hadamard"]:
        y = _butterflies(y) * c["D"] ** -0.5
    live = (tokens >= 0).flatten().nonzero()[:, 0]
    to = tokens.flatten()[live]
    s["o"][to] = y.transpose(1, 2).reshape(-1, c["Hq"], c["D"])[live].to(s["o"].dtype)
    s["lse"][to] = (top + torch.log(den)).transpose(1, 2).reshape(-1, c["Hq"])[live]


def _batches(rows, keys, c):
    """Indexes in runs that are computed together: 2^30 values of padded keys, or of their scores, at most."""
    order = sorted(range(len(rows)), key=lambda i: (keys[i], rows[i]))
    out, most_r, most_k = [], 0, 0
    for i in order:
        r, k = max(most_r, rows[i]), max(most_k, keys[i])
        n = len(out[-1]) + 1 if out else 1
        if not out or n * max(2 * k * c["Hkv"] * c["D"], r * c["Hq"] * k) > 1 << 30:
            out.append([])
            r, k = rows[i], keys[i]
        out[-1].append(i)
        most_r, most_k = r, k
    return out


def _plain_shared(s):
    c = s["case"]
    page, first, starts, prefix = c["page"], s["first"], s["start_of"], s["prefix"]
    Hkv, G, D = c["Hkv"], c["Hq"] // c["Hkv"], c["D"]
    top = torch.full((s["T"], Hkv, G, 1), -math.inf, device="cuda")
    den, y = torch.zeros_like(top), torch.zeros(s["T"], Hkv, G, D, device="cuda")

    def keep(tokens, part):
        live = (tokens >= 0).flatten().nonzero()[:, 0]
        to = tokens.flatten()[live]
        t, d, z = (x.transpose(1, 2).reshape(-1, *x.shape[1:2], *x.shape[3:])[live] for x in part)
        new = torch.maximum(top[to], t)
        a, b = (torch.exp(x - new.clamp(min=-1e30)) for x in (top[to], t))
        den[to], y[to] = den[to] * a + d * b, y[to] * a + z * b
        top[to] = new

    groups = range(c["groups"])
    rows = [first[starts[g + 1]] - first[starts[g]] for g in groups]
    for run_ in _batches(rows, prefix, c):
        tokens = _padded([range(first[starts[g]], first[starts[g + 1]]) for g in run_], -1)
        blocks = _padded([range(_up(prefix[g], page)) for g in run_], -1)
        hi = torch.tensor([[prefix[g]] for g in run_], device="cuda")
        keep(tokens, _partial(s, tokens, torch.tensor([starts[g] for g in run_], device="cuda"), blocks, 0 * hi, hi))
    behind = [0] * c["R"]
    for g in groups:
        behind[starts[g]:starts[g + 1]] = [prefix[g]] * (starts[g + 1] - starts[g])
    for run_ in _batches(s["qs"], [n - b for n, b in zip(s["lens"], behind)], c):
        tokens = _padded([range(first[r], first[r + 1]) for r in run_], -1)
        blocks = _padded([range(behind[r] // page, _up(s["lens"][r], page)) for r in run_], -1)
        lo, hi = (torch.tensor([[x[r]] for r in run_], device="cuda") for x in (behind, s["lens"]))
        keep(tokens, _partial(s, tokens, torch.tensor(run_, device="cuda"), blocks, lo, hi))
    tokens = torch.arange(first[-1], device="cuda")[None]
    _store(s, tokens, *(x[:first[-1]][None].transpose(1, 2) for x in (top, den, y)))
    return s["o"], s["lse"]


def _plain_sinks(s):
    c = s["case"]
    page, first = c["page"], s["first"]
    # long prompts in pieces of up to 1000 queries, each with the blocks that it sees
    pieces = [(r, i, min(i + 1000, s["qs"][r])) for r in range(c["R"]) for i in range(0, s["qs"][r], 1000)]

    def seen(r, i, j):
        base = s["lens"][r] - s["qs"][r]
        low = max(0, base + i - c["window"] + 1)
        return [b for b in s["blocks_of"][r] if b * page <= base + j - 1 and (b * page < c["sinks"] or (b + 1) * page > low)]

    blocks = [seen(*x) for x in pieces]
    for run_ in _batches([j - i for _, i, j in pieces], [len(b) * page for b in blocks], c):
        at = [pieces[i] for i in run_]
        tokens = _padded([range(first[r] + i, first[r] + j) for r, i, j in at], -1)
        hi = torch.tensor([[s["lens"][r]] for r, _, _ in at], device="cuda")
        part = _partial(s, tokens, torch.tensor([r for r, _, _ in at], device="cuda"), _padded([blocks[i] for i in run_], -1),
                        0 * hi, hi)
        _store(s, tokens, *part)
    return s["o"], s["lse"]


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        if op in ("shared", "sinks"):
            return _plain_shared(s) if op == "shared" else _plain_sinks(s)
        return _tables(s, {"fork": _plain_fork, "trim": _plain_trim, "compact": _plain_compact}[op](s))
    from paper_2607_02584_amd import rotate_attn as ra
    p = s["p"]
    if op == "sinks":
        ra.cache_attn_sinks(p, s["case"]["sinks"], s["q"], s["cache"], s["block_table"], s["q_start"], s["seq_lens"],
                            s["max_q"], s["o"], s["ws"], lse=s["lse"], rope=s.get("rope"))
        return s["o"], s["lse"]
    if op == "shared":
        ra.cache_attn_shared(p, s["q"], s["cache"], s["block_table"], s["q_start"], s["seq_lens"], s["positions"],
                             s["group_start"], s["prefix_lens"], s["o"], s["ws"], lse=s["lse"], rope=s.get("rope"))
        return s["o"], s["lse"]
    if op == "fork":
        ra.cache_fork(p, s["parents"], s["children"], s["seq_lens"], s["block_table"], s["page_refs"], s["free_pages"],
                      s["free_count"], s["cache"], s["ws"], s["status"], seq_out=s["seq_out"], table_out=s["table_out"],
                      refs_out=s["refs_out"], free_out=s["free_out"], count_out=s["count_out"])
    elif op == "trim":
        ra.cache_trim(p, s["seq_lens"], s["block_table"], s["page_refs"], s["free_pages"], s["free_count"], s["cache"],
                      s["ws"], s["status"], keep=s["keep"], sinks=s["case"]["sinks"] if s["case"]["window"] else -1,
                      seq_out=s["seq_out"], table_out=s["table_out"], refs_out=s["refs_out"], free_out=s["free_out"],
                      count_out=s["count_out"])
    else:
        ra.cache_compact(p, s["seq_lens"], s["block_table"], s["page_refs"], s["free_pages"], s["free_count"], s["cache"],
                         s["ws"], s["status"], seq_out=s["seq_out"], table_out=s["table_out"], refs_out=s["refs_out"],
                         free_out=s["free_out"], count_out=s["count_out"])
    return _tables(s, s["status"])


# ------------------------------------------------------------------ 64 bits --

def _matrix(D):
    """The orthonormal Sylvester-Hadamard matrix: sign (-1)^(bits that i and j share)."""
    i = torch.arange(D, device="cuda")
    both = i[:, None] & i[None, :]
    odd = torch.zeros_like(both)
    for b in range(D.bit_length()):
        odd ^= (both >> b) & 1
    return (1.0 - 2.0 * odd.double()) / math.sqrt(D)


def _exact_tokens(c, cache, page_ids, offsets):
    """K and V [Hkv, n, D] in 64 bits of single tokens, byte by byte from the layout."""
    D, Hkv, page = c["D"], c["Hkv"], c["page"]
    d = torch.arange(D, device="cuda")
    t = offsets[:, None]
    at_k = (t // 16) * 8 * D + (d // (D // 4)) * 2 * D + (t % 16) * (D // 8) + (d % (D // 4)) // 2
    at_v = page * D // 2 + (t // 4) * 2 * D + (d // (D // 16)) * (D // 8) + (t % 4) * (D // 32) + (d % (D // 16)) // 2
    value = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device="cuda")
    raw = cache.view(cache.shape[0], Hkv, -1)
    head = torch.arange(Hkv, device="cuda")[:, None, None]
    out = []
    for which, at in enumerate((at_k, at_v)):
        byte = raw[page_ids[None, :, None], head, at[None]].int()
        code = torch.where(d % 2 == 1, byte >> 4, byte & 15)
        place = page * D + which * 4 * page + 4 * offsets[None, :, None] + torch.arange(4, device="cuda")
        scale = raw[page_ids[None, :, None], head, place].contiguous().view(torch.float32).double()
        out.append(value[code] * scale)
    return out


def exact(case, seed):
    c = case
    if c["op"] in ("fork", "trim", "compact"):
        return None
    s = _inputs(c, seed)
    D, Hq, Hkv, page = c["D"], c["Hq"], c["Hkv"], c["page"]
    G = Hq // Hkv
    H = _matrix(D)
    o = torch.zeros(s["T"], Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["T"], Hq, dtype=torch.float64, device="cuda")
    for r, (n, q) in enumerate(zip(s["lens"], s["qs"])):
        base = n - q
        for i in range(0, q, 2000):
            j = min(q, i + 2000)
            pos = torch.arange(base + i, base + j, device="cuda")
            key = torch.arange(base + j, device="cuda")
            if c["op"] == "sinks":       # the others are seen by none of these queries
                key = key[(key < c["sinks"]) | (key > base + i - c["window"])]
            k = torch.empty(Hkv, key.numel(), D, dtype=torch.float64, device="cuda")
            v = torch.empty_like(k)
            for a in range(0, key.numel(), 32768):
                at = key[a:a + 32768]
                k[:, a:a + 32768], v[:, a:a + 32768] = _exact_tokens(c, s["cache"], s["block_table"][r].long()[at // page], at % page)
            x = s["q"][s["first"][r] + i:s["first"][r] + j].double()
            if c["rope"]:
                z = torch.view_as_complex(x.reshape(j - i, Hq, D // 2, 2).contiguous())
                x = torch.view_as_real(z * torch.view_as_complex(s["rope"][pos].double().contiguous())[:, None]).flatten(-2)
            if c["hadamard"]:
                x = x @ H
            sees = key[None, :] <= pos[:, None]
            if c["op"] == "sinks":
                sees = sees & ((key[None, :] > pos[:, None] - c["window"]) | (key < c["sinks"])[None, :])
            for h in range(Hkv):
                t = (x[:, h * G:(h + 1) * G].reshape(-1, D) @ k[h].t().contiguous() / math.sqrt(D)).view(j - i, G, -1)
                t = torch.where(sees[:, None, :], t, -math.inf)
                z = torch.logsumexp(t, 2)
                y = (torch.exp(t - z[..., None]).view((j - i) * G, -1) @ v[h]).view(j - i, G, D)
                rows = slice(s["first"][r] + i, s["first"][r] + j)
                lse[rows, h * G:(h + 1) * G] = z
                o[rows, h * G:(h + 1) * G] = y @ H if c["v_hadamard"] else y
    return o, lse
