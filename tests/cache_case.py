"""Calls of the cache attention with other key sets, and their results in 64 bits (for test_gpu_cache_sinks.py and
test_gpu_cache_shared.py)."""
import numpy as np
import torch

import cache_ref as ref

HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
PAIR = 2.0 ** -17       # of a value held as two bf16 values


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().cpu().double().numpy()


def up(n, page):
    return -(-n // page)


class Case:
    """Requests of lens[r] tokens and qs[r] queries.  groups: (first request, one behind the last, tokens that all of
    them begin with): full pages of those are the same, the page they end in is a copy with other tokens behind them.
    Scales of places behind a request's end are NaN."""

    def __init__(self, ra, Hq, Hkv, D, page, lens, qs, dt="bf16", out=None, rope=False, had=False, vhad=False, window=0,
                 sinks=None, groups=(), pad=0, seed=0, gain=1.5, strided=False, extra=2):
        out = out or dt
        rng = np.random.default_rng(seed)
        self.ra, self.rng, self.dt, self.out, self.groups, self.sinks = ra, rng, dt, out, list(groups), sinks
        self.lens, self.qs = list(lens), list(qs)
        nb = [up(n, page) for n in lens]
        pages, blocks = sum(nb) + extra, max(nb + [1]) + 1
        kind = {"bf16": ra.BF16, "fp16": ra.FP16, "fp32": ra.FP32}
        self.p = ra.make_cache_params(Hq, Hkv, D, page_size=page, num_pages=pages, max_blocks=blocks,
                                      rotation=ra.ROT_HADAMARD if had else ra.ROT_NONE,
                                      v_rotation=ra.VROT_HADAMARD if vhad else ra.VROT_NONE, window=window, in_dtype=kind[dt],
                                      out_dtype=kind[out])
        perm = rng.permutation(pages)
        self.table = np.full((len(lens), blocks), -1, np.int32)
        self.cache = rng.integers(0, 256, (pages, ra.cache_layout(self.p)["page_bytes"]), dtype=np.uint8)
        self.scales()[:] = 0.37 * np.exp(0.3 * rng.standard_normal((pages, Hkv, 2, page)))
        used = np.zeros((pages, page), bool)
        at = 0
        for r, n in enumerate(lens):
            self.table[r, :nb[r]] = perm[at:at + nb[r]]
            at += nb[r]
        for a, b, n in self.groups:
            for r in range(a + 1, b):
                m = min(n, lens[r], lens[a])
                self.table[r, :m // page] = self.table[a, :m // page]
                if m % page:
                    to = self.table[r, m // page]
                    own = self.scales()[to].copy()
                    self.cache[to] = self.cache[self.table[a, m // page]]
                    self.scales()[to, :, :, m % page:] = own[:, :, m % page:]
        for r, n in enumerate(lens):
            for t in range(n):
                used[self.table[r, t // page], t % page] = True
        self.scales()[~used.any(1)] = np.nan
        self.scales()[:] = np.where(used[:, None, None, :], self.scales(), np.float32(np.nan))
        self.start = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
        self.T = int(self.start[-1]) + pad
        x = torch.tensor(rng.standard_normal((self.T, Hq + (2 if strided else 0), D)) * gain).to(DT[dt]).cuda()
        self.q = x[:, 1:Hq + 1] if strided else x
        self.cs = ref.rope_table(blocks * page, D) if rope else None
        pos = [n - m + i for n, m in zip(lens, qs) for i in range(m)]
        self.positions = i32(pos + [-1] * pad)
        self.fresh()

    def scales(self):
        """[pages, Hkv, 2, page] as a view of the bytes."""
        p = self.p
        return self.cache.reshape(p.num_pages, p.Hkv, -1)[:, :, p.page_size * p.D:].view(np.float32).reshape(
            p.num_pages, p.Hkv, 2, p.page_size)

    def fresh(self):
        self.o = torch.full((self.T, self.p.Hq, self.p.D), 5.0, dtype=DT[self.out], device="cuda")
        self.lse = torch.full((self.T, self.p.Hq), 5.0, device="cuda")

    def rope(self):
        return None if self.cs is None else torch.from_numpy(self.cs).cuda()

    def run(self, ws=None, stream=None, prefix=None, cache=None):
        """The call of this case; outputs and lse."""
        ra, p, R = self.ra, self.p, len(self.lens)
        self.fresh()
        cache = torch.from_numpy(self.cache).cuda() if cache is None else cache
        tensors = (self.q, cache, i32(self.table), i32(self.start), i32(self.lens))
        max_q = max(self.qs + [0])
        kw = dict(lse=self.lse, rope=self.rope(), stream=stream)
        torch.cuda.synchronize()
        if self.sinks is not None:
            ws = ra.cache_workspace(p, R, self.T, max_q) if ws is None else ws
            ra.cache_attn_sinks(p, self.sinks, *tensors, max_q, self.o, ws, **kw)
        elif self.groups:
            G = len(self.groups)
            ws = ra.cache_shared_workspace(p, R, G, self.T) if ws is None else ws
            # requests between groups are a group that shares nothing
            starts, lens, at = [], [], None
            for a, b, n in self.groups:
                if at is not None and a > at:
                    starts.append(at)
                    lens.append(0)
                starts.append(a)
                lens.append(n)
                at = b
            starts.append(at)
            if len(lens) > G:
                ws = ra.cache_shared_workspace(p, R, len(lens), self.T)
            ra.cache_attn_shared(p, *tensors, self.positions, i32(starts), i32(lens if prefix is None else prefix), self.o,
                                 ws, **kw)
        else:
            ws = ra.cache_workspace(p, R, self.T, max_q) if ws is None else ws
            ra.cache_attn(p, *tensors, max_q, self.o, ws, **kw)
        torch.cuda.synchronize()
        return self.o, self.lse

    def want(self):
        """Outputs, lse, and what the bounds take: sum of p |v|, the largest scale * sum |q k|."""
        p = self.p
        D, G, H = p.D, p.Hq // p.Hkv, ref.hadamard(p.D) / np.sqrt(p.D)
        o, lse = np.full((self.T, p.Hq, D), 5.0), np.full((self.T, p.Hq), 5.0)
        size_v, size_s = np.zeros(o.shape), np.zeros(lse.shape)
        for r, (n, m) in enumerate(zip(self.lens, self.qs)):
            if m == 0:
                continue
            sl = slice(self.start[r], self.start[r + 1])
            pos, seen, k, v = self._seen(r)
            x = f64(self.q[sl])
            if self.cs is not None:
                x = ref.turn(x, self.cs[np.maximum(pos[:, 0], 0)])
            if p.rotation:
                x = x @ H
            for h in range(p.Hq):
                kh, vh = k[:, h // G], v[:, h // G]
                s = np.where(seen, D ** -0.5 * (x[:, h] @ kh.T), -np.inf)
                top = s.max(1, initial=-np.inf)
                w = np.where(seen, np.exp(s - np.where(np.isfinite(top), top, 0.0)[:, None]), 0.0)
                l = w.sum(1)
                with np.errstate(divide="ignore"):
                    lse[sl, h] = np.where(l > 0, top + np.log(l), -np.inf)
                w /= np.where(l > 0, l, 1.0)[:, None]
                y, av = w @ vh, w @ np.abs(vh)
                o[sl, h] = y @ H if p.v_rotation else y
                size_v[sl, h] = np.abs(av).sum(1, keepdims=True) / np.sqrt(D) if p.v_rotation else av
                size_s[sl, h] = np.where(seen, D ** -0.5 * (np.abs(x[:, h]) @ np.abs(kh).T), 0.0).max(1, initial=0.0)
        return o, lse, size_v, size_s

    def _seen(self, r):
        """Positions and mask of request r, and its keys and values in 64 bits (0 where nobody sees them)."""
        p, n, m = self.p, self.lens[r], self.qs[r]
        pos, key = n - m + np.arange(m)[:, None], np.arange(n)[None, :]
        seen = key <= pos
        if p.window:
            seen = seen & ((key > pos - p.window) | (key < (self.sinks or 0)))
        ids = self.table[r, np.arange(n) // p.page_size] if n else np.zeros(0, np.int32)
        there = (ids >= 0) & (ids < p.num_pages)
        seen = seen & there[None, :]
        slots = np.where(there, ids, 0) * p.page_size + np.arange(n) % p.page_size
        kc, ks, vc, vs = ref.rows(self.cache, slots, p.page_size, p.Hkv, p.D)
        any_sees = seen.any(0)[:, None, None]
        return pos, seen, *(np.where(any_sees, ref.value(c) * s[..., None].astype(np.float64), 0.0) for c, s in ((kc, ks), (vc, vs)))

    def lse32(self):
        """lse in elementary binary32 operations (torch, on the host)."""
        p = self.p
        G, f = p.Hq // p.Hkv, torch.float32
        H = torch.tensor(ref.hadamard(p.D) / np.sqrt(p.D)).to(f)
        lse = np.full((self.T, p.Hq), 5.0)
        for r in range(len(self.lens)):
            if self.qs[r] == 0:
                continue
            pos, seen, k, _ = self._seen(r)
            sl = slice(self.start[r], self.start[r + 1])
            k, seen = torch.tensor(k).to(f), torch.tensor(seen)
            x = self.q[sl].cpu().to(f)
            if self.cs is not None:
                cs = torch.tensor(self.cs[np.maximum(pos[:, 0], 0)])[:, None]
                a, b = x[..., 0::2], x[..., 1::2]
                x = torch.stack((a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]), -1).flatten(-2)
            for h in range(p.Hq):
                y = x[:, h] @ H if p.rotation else x[:, h]
                s = (y @ k[:, h // G].T.contiguous()) * np.float32(p.D ** -0.5)
                s = torch.where(seen, s, -torch.inf)
                top = s.max(1, keepdim=True).values
                lse[sl, h] = (top + torch.log(torch.exp(s - top).sum(1, keepdim=True)))[:, 0].double().numpy()
        return lse

    def check_lse(self):
        """Error of lse against 64 bits at most twice that of binary32 operations throughout (as many roundings, in other
        places), and four roundings of a score as large as these."""
        _, want, _, size_s = self.want()
        n = self.start[-1]
        want, size_s, got, plain = want[:n], size_s[:n], f64(self.lse)[:n], self.lse32()[:n]
        unit = 2.0 ** -24 * (1 + np.abs(want).max() + size_s.max())
        assert np.abs(got - want).max() <= 2 * np.abs(plain - want).max() + 4 * unit

    def check(self, one, n=None, got=None, want=None):
        """Bounds by arithmetic.  one: weights times V's scales may be one bf16 value (half a step, 2^-8).  Scores: Q as
        two bf16 values (2^-17 of each element), products exact, sums of D terms and the scales in binary32: |ds| <=
        (2^-17 + (D + 8) 2^-24) size_s, and 2^-21 for powers of two and logarithm.  A weight is then off by a factor e^(2 |ds|) (its own and the sum's), its
        rounding e, and sums of n terms (one rounding for 16 terms of the matrix unit, and 128 for waves, parts and joining): the output
        by size_v times all of it, and its own rounding.  Binary16 outputs below 2^-14 round by up to 2^-25."""
        o, lse = (self.o, self.lse) if got is None else got
        want, want_lse, size_v, size_s = self.want() if want is None else want
        n = max(self.lens + [1]) if n is None else n
        D = self.p.D
        e = HALF["bf16"] if one and self.out == "bf16" else PAIR
        ds = (PAIR + (D + 8) * 2.0 ** -24) * size_s + 2.0 ** -21
        acc = (n / 16 + 128) * 2.0 ** -24
        rel = np.expm1(2 * ds) + e + 2 * acc
        got_o, got_lse = f64(o), f64(lse)
        live = np.isfinite(want_lse)
        assert (np.isneginf(got_lse) == np.isneginf(want_lse)).all()
        bound = size_v * rel[..., None] + (np.abs(want) + size_v * rel[..., None]) * HALF[self.out] + 1e-30
        bound += 2.0 ** -25 if self.out == "fp16" else 0.0
        err = np.abs(got_o - want)
        bad = ~(err <= bound)
        assert not bad.any(), f"{bad.sum()} of {bad.size} outputs off, worst {np.nanmax(err / bound):.3g} of the bound at {np.argwhere(bad)[0]}"
        d = np.abs(got_lse - np.where(live, want_lse, 0))[live]
        lim = (ds + acc + 2.0 ** -22 * (1 + np.abs(np.where(live, want_lse, 0))))[live]
        assert (d <= lim).all(), f"lse off by {(d / lim).max():.3g} of the bound"
