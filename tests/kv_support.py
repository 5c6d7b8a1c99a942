"""The page cache's operators restated in plain form, in 64 bits, and bounds on what 32- and 16-bit kernels may differ by."""

import math

import numpy as np
import torch

from paper_2607_16892_gb300 import kvdro

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half the spacing of numbers just above a power of two


def plan(page, i):
    """One step of the page plan, request by request.  ``i``: the inputs, numpy arrays by name, and T."""
    table, ring, n = i["table"].copy(), i["ring"].copy(), len(i["ring"])
    B, mp = table.shape
    head, free = (int(x) for x in i["pool"])
    held, kv_len, q_off = i["held"].copy(), np.zeros(B, np.int64), np.zeros(B + 1, np.int64)
    slot, pos = np.full(i["T"], -1), np.full(i["T"], -1)
    taken, asked, back = 0, 0, []
    for b in range(B):
        new, have, cached = int(i["new_len"][b]), int(i["held"][b]), int(i["cached"][b])
        q_off[b + 1] = q_off[b] + max(new, 0)
        if new < 0:
            back += table[b, :have].tolist()
            held[b] = 0
            continue
        if cached + new > mp * page:
            continue
        if new > 0:
            tokens = max(cached + new, min(int(i["reserve"][b]), mp * page)) if i["reserve"] is not None else cached + new
            need = max(0, -(-tokens // page) - have)
            asked += need
            if need and asked > free:
                continue
            table[b, have:have + need] = ring[(head + taken + np.arange(need)) % n]
            taken += need
            held[b] = have + need
            p = np.arange(cached, cached + new)
            at = slice(int(q_off[b]), min(int(q_off[b + 1]), i["T"]))
            slot[at] = (table[b, p // page] * page + p % page)[:at.stop - at.start]
            pos[at] = p[:at.stop - at.start]
        kv_len[b] = cached + new
    ring[(head + free + np.arange(len(back))) % n] = back
    return {"table": table, "ring": ring, "held_out": held, "pool_out": np.array([(head + taken) % n, free - taken + len(back)]),
            "q_off": q_off, "kv_len": kv_len, "slot": slot, "pos": pos}


class Case:
    """Requests (new tokens, tokens with them) over a page cache whose unused places hold NaN."""

    def __init__(self, lens, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=0, layout="dense", scores=1.0, spare=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.page, self.Hq, self.Hkv, self.D, self.dt = lens, page, Hq, Hkv, D, DTYPES[dtype]
        pages = [-(-kv // page) for _, kv in lens]
        n = sum(pages) + spare
        ids = rng.permutation(n)[:sum(pages)]
        table = np.full((len(lens), max(max(pages), 1) + 1), -7, np.int32)
        at = 0
        for b, c in enumerate(pages):
            table[b, :c] = ids[at:at + c]
            at += c
        self.table = torch.from_numpy(table).cuda()
        self.kv_len = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
        off = np.concatenate([[0], np.cumsum([q for q, _ in lens])]).astype(np.int32)
        self.q_off, self.T = torch.from_numpy(off).cuda(), int(off[-1])
        self.off = off
        if layout == "heads_first":  # [page][head][slot][d], and room between the pages
            store = torch.full((2, n, Hkv + 1, page, D), float("nan"), dtype=self.dt, device="cuda")
            self.k, self.v = (store[i, :, :Hkv].transpose(1, 2) for i in range(2))
        elif layout == "packed":  # keys and values side by side in one array
            store = torch.full((n, page, Hkv, 2 * D), float("nan"), dtype=self.dt, device="cuda")
            self.k, self.v = store[..., :D], store[..., D:]
        else:
            self.k, self.v = (torch.full((n, page, Hkv, D), float("nan"), dtype=self.dt, device="cuda") for _ in range(2))
        self.keys, self.values = [], []
        for b, (_, kv) in enumerate(lens):
            k = (torch.randn((kv, Hkv, D), generator=g, device="cuda") * scores).to(self.dt)
            v = torch.randn((kv, Hkv, D), generator=g, device="cuda").to(self.dt)
            self.set(b, k, v)
            self.keys.append(k)
            self.values.append(v)
        qkv = torch.randn((max(self.T, 1), Hq + 2 * Hkv, D), generator=g, device="cuda").to(self.dt)
        self.q = qkv[:self.T, :Hq] if layout != "dense" else qkv[:self.T, :Hq].contiguous()

    def places(self, b, kv):
        j = torch.arange(kv, device="cuda")
        return self.table[b].long()[j // self.page], j % self.page

    def set(self, b, k, v):
        p, s = self.places(b, len(k))
        self.k[p, s], self.v[p, s] = k, v

    def run(self, ctx, lse=True, stream=None, max_q=None, **opt):
        cache = kvdro.kvdro_kv_open(ctx, self.k, self.v)
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

    def check(self, out, lse, scale=None, causal=True, window=0, softcap=0.0, only=None):
        """Every row against the definition in 64 bits.  With u the unit roundoff of the stored type, p the
        softmax weights and e_j a bound on the error of score j -- (D + 6) 2^-24 scale sum_d |q_d k_jd|, from the FP32
        product and scaling, twice that and 2^-19 cap through the cap -- the weights are off by 2 max e + 2^-18 relative (exp and its sum) and by
        u from their rounding, the result by u from its own; a weight of FP16 below 2^-14 is off by 2^-25 absolutely."""
        u, f64 = UNIT[self.dt], torch.float64
        scale = self.D ** -0.5 if scale is None else scale
        G = self.Hq // self.Hkv
        for b, (n, kv) in enumerate(self.lens):
            if n == 0 or (only is not None and b not in only):
                continue
            t0, t1 = int(self.off[b]), int(self.off[b + 1])
            got, z = out[t0:t1].to(f64), lse[t0:t1].to(f64) if lse is not None else None
            p = torch.arange(n, device="cuda") + kv - n
            j = torch.arange(kv, device="cuda")
            seen = torch.ones((n, kv), dtype=torch.bool, device="cuda")
            if causal:
                seen &= j[None] <= p[:, None]
            if window:
                seen &= j[None] > p[:, None] - window
            some = seen.any(1)
            if kv == 0 or not bool(some.any()):
                assert (got == 0).all() and (z is None or (z == -math.inf).all()), b
                continue
            for h in range(self.Hq):
                q, k, v = self.q[t0:t1, h].to(f64), self.keys[b][:, h // G].to(f64), self.values[b][:, h // G].to(f64)
                k0, v0 = (torch.where(seen.any(0)[:, None], x, 0.0) for x in (k, v))
                s = q @ k0.T * scale
                e = (self.D + 6) * 2.0 ** -24 * abs(scale) * (q.abs() @ k0.abs().T)
                if softcap:
                    s, e = softcap * torch.tanh(s / softcap), 2 * e + 2.0 ** -19 * softcap
                s = s.masked_fill(~seen, -math.inf)
                ref_z = torch.logsumexp(s, 1)
                w = torch.exp(s - torch.where(some, ref_z, 0.0)[:, None])
                ref = torch.stack([w[i] @ torch.where(seen[i][:, None], v, 0.0) for i in range(n)]) if not torch.isfinite(v0).all() else w @ v0
                absv = w @ v0.abs()
                es = torch.where(seen, e, 0.0).amax(1)
                tol = u * ref.abs() + (u + 2 * es + 2.0 ** -18)[:, None] * absv
                if self.dt == torch.float16:
                    tol = tol + kv * 2.0 ** -24 * v0.abs().max()
                tol = tol + (2.0 ** -24 if self.dt == torch.float16 else 0.0)
                bad = (got[:, h] - ref).abs() > tol
                bad &= some[:, None]
                assert torch.equal(torch.isnan(got[:, h]), torch.isnan(ref)), (b, h)
                assert not bad.any(), (b, h, int(bad.sum()), float(((got[:, h] - ref).abs() / tol).max()))
                assert (got[:, h][~some] == 0).all(), (b, h)
                if z is not None:
                    d = (z[:, h] - ref_z).abs()[some]
                    ztol = (es + 2.0 ** -20 * (1 + ref_z.abs()) + kv * 2.0 ** -24)[some]
                    assert (d <= ztol).all(), (b, h, float((d / ztol).max()))
                    assert (z[:, h][~some] == -math.inf).all(), (b, h)
