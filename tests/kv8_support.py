"""Caches of 8 bits and shared prefixes in plain form, beside ``kv_support``."""

import types

import numpy as np
import torch

from paper_2607_16892_gb300 import kvdro
from tests.kv_support import Case

E4M3, F64 = torch.float8_e4m3fn, torch.float64


def two(e):
    """2^e in 64 bits, exactly."""
    return (e.long() + 1023 << 52).view(F64)


def nearest_code(y):
    """The e4m3 number nearest to each element of a 64-bit tensor within [-448, 448], ties to the even code."""
    step = two(torch.frexp(y)[1].clamp(min=-5) - 4)  # numbers of [2^i, 2^(i+1)) are 2^(i-3) apart, i >= -6
    return torch.round(y / step) * step


def quantise(x):
    """(values of the codes, exponents) of rows x[..., D] of a 16-bit type, in 64 bits."""
    y = x.to(F64)
    top = torch.where(torch.isfinite(y), y.abs(), 0).amax(-1)
    powers = 448 * two(torch.arange(-126, 121, device=x.device))
    e = torch.searchsorted(powers, top) - 126
    code = nearest_code(torch.where(torch.isfinite(y), y, 0) / two(e)[..., None])
    if x.dtype == torch.float16:
        code = torch.where((e == 8)[..., None], code.clamp(-240, 240), code)
    return torch.where(torch.isfinite(y), code, float("nan")), e


def arrays(n, page, heads, D, layout, fill=0x7f):
    """Codes of a cache in one of several layouts (all `fill`: NaN), keys and values."""
    if layout == "heads_first":  # [page][head][slot][d], and room between the pages
        store = torch.full((2, n, heads + 1, page, D), fill, dtype=torch.uint8, device="cuda")
        k, v = (store[i, :, :heads].transpose(1, 2) for i in range(2))
    elif layout == "packed":  # keys and values side by side in one array
        store = torch.full((n, page, heads, 2 * D), fill, dtype=torch.uint8, device="cuda")
        k, v = store[..., :D], store[..., D:]
    else:
        k, v = (torch.full((n, page, heads, D), fill, dtype=torch.uint8, device="cuda") for _ in range(2))
    return k, v


class Case8(Case):
    """A ``Case`` whose cache holds codes; ``keys`` and ``values`` become what they stand for.  Places that no token has hold NaN,
    and scale bytes of anything.

    ``Case.check``'s bounds hold as they are.  The codes are exact in the products' types.  Few rows: BF16 queries become FP16
    numbers, off by 2^-25 of the row's largest at most, which its bound on a score -- (D + 6) 2^-24 sum |q_d k_jd| -- covers
    where |k_jd| is of one size; weights are FP16 for either type, held 2^7 above the largest of w_j 2^E_j, so what is below
    2^-14 is off by 2^-32 of that: kv 448 2^-32 of a value at most, below 2^-13 of it at 20000 positions, where the bound
    has 2^-8 (BF16) or kv 2^-24 (FP16) of it."""

    def __init__(self, lens, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=0, layout="dense", scores=1.0, spread=0.0):
        super().__init__(lens, dtype, D, Hq, Hkv, page, seed, "dense" if layout == "dense" else "packed", scores)
        n = self.k.shape[0]
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.codes = arrays(n, page, Hkv, D, layout)
        self.exps = tuple(torch.randint(0, 256, (n, Hkv, page), generator=g, device="cuda", dtype=torch.uint8) for _ in "kv")
        del self.k, self.v
        for b, (_, kv) in enumerate(lens):
            k, v = self.keys[b], self.values[b]
            if spread:  # tokens of very different sizes
                v = (v.float() * torch.exp2(spread * (2 * torch.rand((kv, Hkv, 1), generator=g, device="cuda") - 1))).to(self.dt)
            self.set(b, k, v)

    def set(self, b, k, v):
        if not hasattr(self, "codes"):  # the base class fills its own arrays first
            return super().set(b, k, v)
        p, s = self.places(b, len(k))
        for x, (rows, codes, exps) in enumerate(zip((k, v), self.codes, self.exps)):
            c, e = quantise(rows)
            codes[p, s] = c.to(torch.float32).to(E4M3).view(torch.uint8)
            exps[p, :, s] = (e + 127).to(torch.uint8)
            (self.keys, self.values)[x][b] = c * two(e)[..., None]

    def open(self, ctx):
        return kvdro.kvdro_kv_open8(ctx, *(c.view(E4M3) for c in self.codes), *self.exps, self.dt)

    def run(self, ctx, lse=True, stream=None, max_q=None, **opt):
        cache = self.open(ctx)
        out = torch.full((self.T, self.Hq, self.D), 77.0, dtype=self.dt, device="cuda")
        z = torch.full((self.T, self.Hq), 77.0, dtype=torch.float32, device="cuda") if lse else None
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        kvdro.kvdro_kv_attend(cache, self.q, self.q_off, self.kv_len, self.table, out, lse=z, stream=stream,
                              max_q=max((q for q, _ in self.lens), default=0) if max_q is None else max_q, **opt)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        kvdro.kvdro_kv_close(cache)
        return out, z


class Shared:
    """Requests with prefixes: ``share`` bounds the requests of each of ``prefixes`` (lengths).  The prefixes are further rows of
    the case's table, of no new tokens; ``check`` compares with each request's own case behind its prefix.  ``wide``: the prefixes' table has
    room for so many pages that each prefix is read once for all of its requests, however few they are."""

    def __init__(self, lens, share, prefixes, bits=16, wide=False, **kw):
        self.base = (Case8 if bits == 8 else Case)(lens + [(0, n) for n in prefixes], **kw)
        c, B, G = self.base, len(lens), len(prefixes)
        self.c, self.lens, self.B, self.G, self.share = c, lens, B, G, share
        self.T = c.T
        i32 = dict(dtype=torch.int32, device="cuda")
        self.share_off, self.prefix_len = torch.tensor(share, **i32), torch.tensor(prefixes, **i32)
        self.q_off, self.kv_len = c.q_off[:B + 1].contiguous(), c.kv_len[:B].contiguous()
        self.table, self.prefix_table = c.table[:B].contiguous(), c.table[B:].contiguous()
        if wide:
            pages = (48 << 20) // (B * c.page * c.Hkv * c.D) + 1
            self.prefix_table = torch.nn.functional.pad(self.prefix_table, (0, max(0, pages - self.prefix_table.shape[1])), value=-1)

    def whole(self):
        """The requests as ``Case.check`` takes them, their prefixes in front.  A (causal) token in front of position 0 sees its prefix
        alone, all of it: a request of one token."""
        c, keys, values, lens = self.c, [], [], []
        for b, (q, kv) in enumerate(self.lens):
            k, v = c.keys[b], c.values[b]
            g = next((g for g in range(self.G) if self.share[g] <= b < self.share[g + 1]), None)
            if g is not None and kv > 0:
                for _ in range(q - kv):
                    keys.append(c.keys[self.B + g])
                    values.append(c.values[self.B + g])
                    lens.append((1, len(keys[-1])))
                q = min(q, kv)
                k, v = torch.cat([c.keys[self.B + g], k]), torch.cat([c.values[self.B + g], v])
            keys.append(k)
            values.append(v)
            lens.append((q, len(k) if kv > 0 else 0))
        off = np.concatenate([[0], np.cumsum([q for q, _ in lens])])
        return types.SimpleNamespace(dt=c.dt, D=c.D, Hq=c.Hq, Hkv=c.Hkv, lens=lens, off=off, q=c.q, keys=keys, values=values)

    def open(self, ctx):
        return self.c.open(ctx) if isinstance(self.c, Case8) else kvdro.kvdro_kv_open(ctx, self.c.k, self.c.v)

    def run(self, ctx, stream=None, work=None, max_q=None, cache=None, **opt):
        own = cache is None
        cache = self.open(ctx) if own else cache
        out = torch.full((self.T, self.c.Hq, self.c.D), 77.0, dtype=self.c.dt, device="cuda")
        z = torch.full((self.T, self.c.Hq), 77.0, dtype=torch.float32, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        kvdro.kvdro_kv_attend_shared(cache, self.c.q, self.q_off, self.kv_len, self.table, self.share_off, self.prefix_len, self.prefix_table, out,
                                     lse=z, max_q=max(q for q, _ in self.lens) if max_q is None else max_q, work=work, stream=stream, **opt)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        if own:
            kvdro.kvdro_kv_close(cache)
        return out, z

    def check(self, out, lse, **opt):
        Case.check(self.whole(), out, lse, **opt)
