"""The page cache in 8 bits, reading it back, and prefixes that requests share: the calls of a serving step, sized over the range they use.

Four operators on one cache:
  append  new tokens' keys and values into slots, quantised as they are written: e4m3 codes, and a power of two per token and head
  read    requests' last tokens out of their pages, in 16 bits
  attend  attention of the requests' new tokens over their pages of 8 bits (one token each, or chunks of prompts)
  shared  the same where groups of requests share a prefix, held once in pages of its own (16 and 8 bits)
Plain forms are elementary torch operations in 32 bits, rounded once at the end.
"""
import math
import random
from statistics import NormalDist

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
# Most that a drawn call does: flops, (head, row, key) cells of the padded scores, and elements of the padded keys.  Each is at or
# below the largest listed case's.
MOST_FLOPS, MOST_CELLS, MOST_KEYS = 2.0e12, 4.2e9, 5.3e8


def listed():
    return [
        # The keys and values of one decoding step of 64 requests in a layer: all latency.
        {"name": "append_decode", "op": "append", "T": 64, "Hkv": 8, "D": 128, "page": 16, "n_pages": 4096, "dt": "bf16", "drop": 0.0},
        # A step of long prompts: an odd number of tokens, read out of the packed projection, some of them refused.
        {"name": "append_prompts", "op": "append", "T": 65539, "Hkv": 8, "D": 128, "page": 32, "n_pages": 4096, "dt": "fp16", "drop": 0.02},
        # One request's last 37 tokens, handed to a debugger or a drafting model.
        {"name": "read_tail", "op": "read", "B": 1, "q": 37, "kv": 1000, "mix": "even", "Hkv": 8, "D": 128, "page": 16, "dt": "bf16"},
        # 64 whole requests, of lognormal lengths, moved out of the cache.
        {"name": "read_batch", "op": "read", "B": 64, "q": 8192, "kv": 8192, "mix": "lognormal", "Hkv": 8, "D": 128, "page": 16, "dt": "bf16"},
        # One request, one token, a thousand tokens of context: the smallest attention, all latency.
        {"name": "decode_one", "op": "attend", "B": 1, "q": 1, "kv": 1000, "mix": "even", "Hq": 32, "Hkv": 8, "D": 128, "page": 16,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # The ordinary decoding step: 64 requests of lognormal lengths, grouped heads.
        {"name": "decode_batch", "op": "attend", "B": 64, "q": 1, "kv": 8192, "mix": "lognormal", "Hq": 32, "Hkv": 8, "D": 128, "page": 16,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # Four agents deep into long contexts, short heads: the cache read is split along the keys.
        {"name": "decode_long", "op": "attend", "B": 4, "q": 1, "kv": 131071, "mix": "even", "Hq": 64, "Hkv": 16, "D": 64, "page": 64,
         "dt": "fp16", "window": 0, "cap": 0.0},
        # A mixed step: chunks of some prompts beside decoding requests and a refused one (rows without keys), seven heads a group, a window.
        {"name": "chunk_mixed", "op": "attend", "B": 24, "q": 777, "kv": 6007, "mix": "mixed", "Hq": 28, "Hkv": 4, "D": 128, "page": 32,
         "dt": "fp16", "window": 4096, "cap": 0.0},
        # The last 4096 tokens of a prompt of 32768: the largest.
        {"name": "chunk_long", "op": "attend", "B": 1, "q": 4096, "kv": 32768, "mix": "even", "Hq": 32, "Hkv": 8, "D": 128, "page": 64,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # A few requests behind one instruction: the smallest shared call.
        {"name": "shared_few", "op": "shared", "B": 6, "q": 1, "kv": 203, "G": 1, "prefix": 2005, "alone": 1, "Hq": 32, "Hkv": 8, "D": 128,
         "page": 16, "dt": "bf16", "cap": 0.0, "bits": 16},
        # 64 requests that decode behind the same long document.
        {"name": "shared_document", "op": "shared", "B": 64, "q": 1, "kv": 2048, "G": 1, "prefix": 32768, "alone": 0, "Hq": 32, "Hkv": 8, "D": 128,
         "page": 16, "dt": "bf16", "cap": 0.0, "bits": 16},
        # Several instructions of odd lengths over 8 bits, drafted tokens, requests without one in between.
        {"name": "shared_groups", "op": "shared", "B": 90, "q": 3, "kv": 1501, "G": 5, "prefix": 9001, "alone": 7, "Hq": 28, "Hkv": 4, "D": 128,
         "page": 32, "dt": "fp16", "cap": 30.0, "bits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "shared", "shared"])
    if op == "append":
        T, page = _log(rng, 1, 65539), rng.choice([16, 32, 64, 128])
        return {"op": op, "T": T, "Hkv": rng.choice([1, 2, 4, 8]), "D": rng.choice([64, 128]), "page": page,
                "n_pages": T // page + _log(rng, 2, 2000), "dt": rng.choice(["bf16", "fp16"]), "drop": rng.choice([0.0, 0.02])}
    while True:
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (64, 8), (16, 16), (28, 4), (16, 8), (24, 3), (8, 1)])
        c = {"op": op, "B": _log(rng, 1, 128), "q": 0, "kv": _log(rng, 16, 131072), "mix": rng.choice(["even", "lognormal", "mixed"]), "Hq": Hq,
             "Hkv": Hkv, "D": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128]), "dt": rng.choice(["bf16", "fp16"])}
        if op == "read":
            c["q"] = rng.choice([c["kv"], _log(rng, 1, c["kv"])])
            del c["Hq"]
            if c["B"] * c["kv"] * Hkv * c["D"] <= MOST_KEYS:
                return c
            continue
        c["q"] = min(c["kv"], rng.choice([1, 1, rng.randint(2, 8), _log(rng, 16, 4096)]))
        c["cap"] = rng.choice([0.0, 0.0, 0.0, 30.0])
        long = 0
        if op == "attend":
            c["window"] = rng.choice([0, 0, 0, _log(rng, 16, 8192)])
        else:
            c |= {"G": min(c["B"], rng.choice([1, 1, 2, _log(rng, 1, 16)])), "prefix": _log(rng, 16, 65536), "alone": rng.choice([0, 0, 1, c["B"] // 4]),
                  "bits": rng.choice([16, 8])}
            c["kv"] = min(c["kv"], 16384)
            c["q"] = min(c["q"], c["kv"])
            del c["mix"]
            long = c["prefix"] * c["G"]
        cells = c["q"] * Hq * (c["B"] * c["kv"] + (c["B"] + c.get("G", 0)) * c.get("prefix", 0))
        if cells <= MOST_CELLS and (c["B"] * c["kv"] + long) * Hkv * c["D"] <= MOST_KEYS and work(c)["flops"] <= MOST_FLOPS:
            return c


def _lengths(c):
    """The (new tokens, tokens with them) of a case's requests: the same for every seed, which only orders them."""
    mix = c.get("mix", "lognormal")
    if mix == "even":
        return [(c["q"], c["kv"])] * c["B"]
    nd, out = NormalDist(), []
    for i in range(c["B"]):
        # lognormal of sigma 0.8 whose 98th percentile is the longest
        z = nd.inv_cdf((i + 0.5) / c["B"])
        kv = max(1, min(c["kv"], round(c["kv"] * math.exp(0.8 * (z - 2.05)))))
        if i == c["B"] - 1:
            kv = c["kv"]
        q = min(c["q"], kv)
        if mix == "mixed":
            if i % 6 == 2:  # refused: its tokens have no pages
                q, kv = min(c["q"], 5), 0
            elif i % 6 != 5 and i != c["B"] - 1:
                q = 1
        out.append((q, kv))
    return out


def _prefixes(c):
    """Prefix lengths, and the bounds of the requests that share each: the last `alone` requests have none."""
    n = max(1, c["B"] - c["alone"])
    off = [round(n * g / c["G"]) for g in range(c["G"] + 1)]
    return [max(1, c["prefix"] - g * (c["prefix"] // (2 * c["G"])) - g) for g in range(c["G"])], off


def _seen(c, q, kv):
    """Visible (row, key) pairs of a request, and the keys that any of its rows sees."""
    if kv < 1:
        return 0, 0
    w = c.get("window") or kv + q
    p = np.arange(kv - q, kv, dtype=np.int64)
    return int(np.minimum(p + 1, w).sum()), int(kv - max(0, kv - q - w + 1))


def work(c):
    if c["op"] == "append":
        return {"bytes": int(c["T"] * (1 - c["drop"]) * 2 * c["Hkv"] * (3 * c["D"] + 1) + 4 * c["T"]), "flops": 0}
    lens = _lengths(c)
    if c["op"] == "read":
        return {"bytes": int(sum(q * 2 * c["Hkv"] * (3 * c["D"] + 1) + 4 * q / c["page"] for q, kv in lens if kv > 0)), "flops": 0}
    T, pairs, keys = 0, 0, 0
    for q, kv in lens:
        p, k = _seen(c, q, kv)
        T, pairs, keys = T + q, pairs + p, keys + k
    if c["op"] == "shared":
        lens = _ordered(c, lens)
        plen, off = _prefixes(c)
        pairs += sum(P * sum(q for q, _ in lens[off[g]:off[g + 1]]) for g, P in enumerate(plen))
        keys += sum(plen)
    per = c["D"] + 1 if c.get("bits", 8) == 8 else 2 * c["D"]
    return {"bytes": T * c["Hq"] * (2 * c["D"] * 2 + 4) + keys * (c["Hkv"] * 2 * per + 4 / c["page"]), "flops": 4 * pairs * c["Hq"] * c["D"]}


def _ordered(c, lens):
    """A shared case's requests in an order of their own: its groups are of long and short ones."""
    return [lens[i] for i in np.random.default_rng(7).permutation(len(lens))]


_ctx = None


def _context():
    """The context that a program makes once."""
    global _ctx
    if _ctx is None:
        from paper_2607_16892_gb300 import kvdro as kv
        _ctx = kv.kvdro_create(torch.cuda.current_device())
    return _ctx


def _power(e):
    """2^e of whole numbers from -126 to 127, by its bits."""
    return (e.to(torch.int32) + 127 << 23).view(torch.float32)


def _quantise(x):
    """(codes, scale bytes) of rows x[..., D]: the least power of two 2^E, E >= -126, with max |x| <= 448 2^E; nearest codes."""
    y = x.float()
    part, e = torch.frexp(y.abs().amax(-1))  # 448 = 0.875 * 2^9
    e = torch.where(part == 0, -126, e - torch.where(part <= 0.875, 9, 8)).clamp(min=-126)
    y = y * _power(-e)[..., None]
    if x.dtype == torch.float16:  # 256 * 2^8 is no FP16 number
        y = torch.where(e[..., None] == 8, y.clamp(-240, 240), y)
    return y.to(E4M3), (e + 127).to(torch.uint8)


def _values(codes, scale):
    return codes.float().mul_(_power(scale.int() - 127)[..., None])


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    P, Hkv, D, dt = c["page"], c["Hkv"], c["D"], DT[c["dt"]]

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def keys(n, *shape):
        """Rows as a model gives them: some channels stand out, tokens differ in size."""
        k = normal(n, *shape, Hkv, D)
        k += 2 * (torch.rand(Hkv, D, generator=g, device="cuda") < 0.03).to(dt)
        return k.mul_(torch.exp2(normal(n, *shape, 1, 1)))

    def values(n, *shape):
        return normal(n, *shape, Hkv, D).add_(0.5 * normal(Hkv, D))

    def cache(n_pages, k, v, bits):
        """The cache's arrays; 8 bits: codes [page][slot][head][d] and scale bytes [page][head][slot]."""
        if bits == 16:
            return {"k": k, "v": v}
        s = {}
        for name, x in (("k", k), ("v", v)):
            s[name], e = _quantise(x)
            s[name + "_exp"] = e.transpose(1, 2).contiguous()
        return s

    if c["op"] == "append":
        N = c["n_pages"] * P
        qkv = normal(c["T"], (4 + 2) * Hkv, D)  # the packed projection: four query heads a group, keys, values
        qkv *= torch.exp2(normal(c["T"], 6 * Hkv, 1))
        slot = rng.permutation(N)[:c["T"]]
        slot[rng.random(c["T"]) < c["drop"]] = -1
        s = {"case": c, "k_new": qkv[:, 4 * Hkv:5 * Hkv], "v_new": qkv[:, 5 * Hkv:], "slot": ints(slot)}
        for x in "kv":  # what the cache held before
            s[x] = torch.randn((c["n_pages"], P, Hkv, D), generator=g, device="cuda").to(E4M3)
            s[x + "_exp"] = torch.randint(120, 130, (c["n_pages"], Hkv, P), generator=g, device="cuda", dtype=torch.uint8)
            s[x + "_scale"] = s[x + "_exp"].view(E8M0)
    else:
        B, bits = c["B"], c.get("bits", 8)
        lens = _lengths(c)
        lens = _ordered(c, lens) if c["op"] == "shared" else [lens[i] for i in rng.permutation(B)]
        q_len, kv_len = np.array([x[0] for x in lens]), np.array([x[1] for x in lens])
        plen, poff = _prefixes(c) if c["op"] == "shared" else ([], [0])
        held = np.concatenate([kv_len, plen]).astype(np.int64)  # tokens of the tables' rows, prefixes behind requests
        pages = -(-held // P)
        n_pages = int(pages.sum()) + 7
        table = np.full((len(held), max(1, int(pages.max()))), -1)
        table[np.arange(table.shape[1])[None] < pages[:, None]] = rng.permutation(n_pages)[:int(pages.sum())]
        s = {"case": c} | cache(n_pages, keys(n_pages, P), values(n_pages, P), bits)
        some = held > 0  # what nobody wrote yet after a row's last token: anything
        last = ints(table)[torch.from_numpy(np.nonzero(some)[0]).cuda(), ints(pages[some] - 1).long()].long()
        past = torch.arange(P, device="cuda")[None] > ints((held[some] - 1) % P)[:, None]
        for x in "kv":
            t = s[x].view(torch.uint8) if bits == 8 else s[x]
            t[last] = t[last].masked_fill_(past[:, :, None, None], 0x7f if bits == 8 else float("nan"))
        T = int(q_len.sum())
        own_pages = max(1, int(pages[:B].max()))
        s |= {"q_off": ints(np.concatenate([[0], np.cumsum(q_len)])), "kv_len": ints(kv_len), "table": ints(table[:B, :own_pages]),
              "max_q": int(q_len.max()), "max_kv": int(kv_len.max())}
        if c["op"] == "read":
            s |= {x + "_out": torch.empty((T, Hkv, D), dtype=dt, device="cuda") for x in "kv"}
        else:
            qkv = normal(T, c["Hq"] + 2 * Hkv, D)
            s |= {"q": qkv[:, :c["Hq"]], "out": torch.empty((T, c["Hq"], D), dtype=dt, device="cuda"),
                  "lse": torch.empty((T, c["Hq"]), dtype=torch.float32, device="cuda")}
        if c["op"] == "shared":
            first = np.concatenate([[0], np.cumsum(q_len)])[np.array(poff)]
            s |= {"share_off": ints(poff), "prefix_len": ints(plen), "prefix_table": ints(table[B:]), "max_prefix": max(plen),
                  "most": int(np.diff(first).max())}
    if own:  # the handle that a program keeps for its cache, and its workspace; the inputs are the same on both sides
        from paper_2607_16892_gb300 import kvdro as kv
        if "k_exp" in s:
            s["cache"] = kv.kvdro_kv_open8(_context(), s["k"], s["v"], s["k_exp"], s["v_exp"], dt)
        else:
            s["cache"] = kv.kvdro_kv_open(_context(), s["k"], s["v"])
        if c["op"] == "shared":
            s["work"] = torch.empty(kv.kvdro_kv_shared_bytes(s["q"].shape[0], c["Hq"], D), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    return {"append": _append, "read": _read, "attend": _attend, "shared": _shared}[s["case"]["op"]](s)


def _append(s):
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_append(s["cache"], s["k_new"], s["v_new"], s["slot"])
    else:
        keep = s["slot"] >= 0
        slot = s["slot"][keep].long()
        page, at = slot // s["case"]["page"], slot % s["case"]["page"]
        for x in "kv":
            codes, e = _quantise(s[x + "_new"][keep])
            s[x].view(torch.uint8)[page, at] = codes.view(torch.uint8)
            s[x + "_exp"][page, :, at] = e
    return {x: s[x] for x in ("k", "v", "k_scale", "v_scale")}


def _rows(s, x, table, n):
    """The first n tokens of the tables' rows, [row][n][head][d] in 32 bits."""
    pages = table.clamp(min=0).long()
    if x + "_exp" in s:
        rows = _values(s[x].view(torch.uint8)[pages].view(E4M3), s[x + "_exp"][pages].transpose(2, 3))
    else:
        rows = s[x][pages].float()
    return rows.flatten(1, 2)[:, :n]


def _requests(s):
    """Of every packed row: its request, its place in it, and its position."""
    q_off, kv_len = s["q_off"].long(), s["kv_len"].long()
    n = s["q"].shape[0] if "q" in s else s["k_out"].shape[0]
    t = torch.arange(n, device=q_off.device)
    b = torch.searchsorted(q_off[1:].contiguous(), t, right=True)
    return b, t - q_off[b], kv_len[b] - (q_off[1:] - q_off[:-1])[b] + t - q_off[b]


def _read(s):
    c = s["case"]
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_read(s["cache"], s["q_off"], s["kv_len"], s["table"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    b, _, pos = _requests(s)
    there = pos >= 0
    pos = pos.clamp(min=0)
    page = s["table"][b, pos // c["page"]].clamp(min=0).long()
    at = pos % c["page"]
    return tuple(torch.where(there[:, None, None], _values(s[x].view(torch.uint8)[page, at].view(E4M3), s[x + "_exp"][page, :, at]), 0)
                 .to(DT[c["dt"]]) for x in "kv")


def _scores(c, q, k):
    x = (q @ k).mul_(c["D"] ** -0.5)
    return x.div_(c["cap"]).tanh_().mul_(c["cap"]) if c["cap"] else x


def _own_part(s):
    """The requests padded to the longest, as one batch of products: (top, total, weighted sum) of every packed row."""
    c = s["case"]
    B, Hkv, D, dev = c["B"], c["Hkv"], c["D"], s["q"].device
    G, Q, S = c["Hq"] // Hkv, s["max_q"], s["max_kv"]
    q_off, kv_len = s["q_off"].long(), s["kv_len"].long()
    i, j = torch.arange(Q, device=dev), torch.arange(S, device=dev)
    row = (q_off[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().view(B, Q, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, D)
    there = (j < kv_len[:, None])[:, :, None, None]
    k = _rows(s, "k", s["table"], S).masked_fill_(~there, 0).permute(0, 2, 3, 1)
    v = _rows(s, "v", s["table"], S).masked_fill_(~there, 0).transpose(1, 2)
    x = _scores(c, q, k).view(B, Hkv, G, Q, S)
    p = (kv_len - (q_off[1:] - q_off[:-1]))[:, None] + i
    seen = (j <= p[:, :, None]) & (j < kv_len[:, None, None])
    if c.get("window"):
        seen &= j > p[:, :, None] - c["window"]
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == float("-inf"), 0, top)).exp_()
    total = x.sum(-1)
    out = (x.view(B, Hkv, G * Q, S) @ v).view(B, Hkv, G, Q, D)
    b, r, _ = _requests(s)
    return tuple(y[b, :, :, r].reshape(-1, c["Hq"], *y.shape[4:]) for y in (top.squeeze(-1), total, out))


def _attend(s):
    c = s["case"]
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_attend(s["cache"], s["q"], s["q_off"], s["kv_len"], s["table"], s["out"], lse=s["lse"], scale=c["D"] ** -0.5, causal=True,
                           window=c["window"], softcap=c["cap"], max_q=s["max_q"])
        return s["out"], s["lse"]
    top, total, out = _own_part(s)
    return (out / torch.where(total == 0, 1, total)[..., None]).to(s["q"].dtype), top + total.log()


def _shared(s):
    c = s["case"]
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_attend_shared(s["cache"], s["q"], s["q_off"], s["kv_len"], s["table"], s["share_off"], s["prefix_len"], s["prefix_table"],
                                  s["out"], lse=s["lse"], scale=c["D"] ** -0.5, softcap=c["cap"], max_q=s["max_q"], work=s["work"])
        return s["out"], s["lse"]
    # each prefix with the rows of all its requests, padded to the most
    N, Hkv, D, P, R = c["G"], c["Hkv"], c["D"], s["max_prefix"], s["most"]
    G, T, dev = c["Hq"] // Hkv, s["q"].shape[0], s["q"].device
    bounds = s["q_off"].long()[s["share_off"].long()]
    row = (bounds[:-1, None] + torch.arange(R, device=dev)).clamp(max=T - 1)
    q = s["q"][row].float().view(N, R, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(N, Hkv, G * R, D)
    there = (torch.arange(P, device=dev) < s["prefix_len"][:, None])
    k = _rows(s, "k", s["prefix_table"], P).masked_fill_(~there[:, :, None, None], 0).permute(0, 2, 3, 1)
    v = _rows(s, "v", s["prefix_table"], P).masked_fill_(~there[:, :, None, None], 0).transpose(1, 2)
    x = _scores(c, q, k).masked_fill_(~there[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1)
    out = x @ v
    t = torch.arange(T, device=dev)
    g = torch.searchsorted(bounds[1:].contiguous(), t, right=True)
    inside = (g < N)[:, None]
    g = g.clamp(max=N - 1)
    r = (t - bounds[g]).clamp(max=R - 1)
    top0, total0, out0 = (y.view(N, Hkv, G, R, *y.shape[3:])[g, :, :, r].reshape(T, c["Hq"], *y.shape[3:]) for y in (top.squeeze(-1), total, out))
    top0, total0 = torch.where(inside, top0, float("-inf")), torch.where(inside, total0, 0)
    # and joined with the requests' own tokens
    top1, total1, out1 = _own_part(s)
    top = torch.maximum(top0, top1)
    f0, f1 = (top0 - top).exp(), (top1 - top).exp()
    total = total0 * f0 + total1 * f1
    out = (out0 * f0[..., None] + out1 * f1[..., None]) / total[..., None]
    return out.to(s["q"].dtype), top + total.log()


def _power64(e):
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def exact(c, seed):
    global own
    was, own = own, False  # the inputs alone, without the library
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["op"] == "append":
        return _exact_append(c, s)
    P, Hkv, D, f64 = c["page"], c["Hkv"], c["D"], torch.float64
    q_off, kv_len = s["q_off"].tolist(), s["kv_len"].tolist()

    def stored(x, row, n):
        """Tokens 0 .. n-1 of a table's row, as the numbers they stand for."""
        at = row[:-(-n // P)].long()
        y = s[x].view(torch.uint8)[at].view(E4M3).to(f64) if x + "_exp" in s else s[x][at].to(f64)
        if x + "_exp" in s:
            y *= _power64(s[x + "_exp"][at].long() - 127).transpose(1, 2)[..., None]
        return y.reshape(-1, Hkv, D)[:n]

    if c["op"] == "read":
        outs = [torch.zeros((q_off[-1], Hkv, D), dtype=f64, device="cuda") for _ in "kv"]
        for b, n in enumerate(kv_len):
            new = q_off[b + 1] - q_off[b]
            if n and new:
                for out, x in zip(outs, "kv"):
                    out[q_off[b]:q_off[b + 1]] = stored(x, s["table"][b], n)[n - new:]
        return tuple(outs)
    G, T = c["Hq"] // Hkv, s["q"].shape[0]
    out, lse = torch.zeros((T, c["Hq"], D), dtype=f64, device="cuda"), torch.full((T, c["Hq"]), -math.inf, dtype=f64, device="cuda")
    groups = s["share_off"].tolist() if c["op"] == "shared" else [0]
    before, of = (None, None), -1
    for b, n in enumerate(kv_len):
        if n == 0:
            continue
        k, v = (stored(x, s["table"][b], n) for x in "kv")
        extra = 0
        if groups[0] <= b < groups[-1]:  # the prefix's tokens stand before the request's own
            g = next(i for i in range(len(groups) - 1) if b < groups[i + 1])
            if g != of:
                before, of = tuple(stored(x, s["prefix_table"][g], int(s["prefix_len"][g])) for x in "kv"), g
            extra = len(before[0])
            k, v = torch.cat([before[0], k]), torch.cat([before[1], v])
        for t0 in range(q_off[b], q_off[b + 1], 512):  # a few rows at a time
            t1 = min(t0 + 512, q_off[b + 1])
            p = torch.arange(t0, t1, device="cuda") - q_off[b + 1] + n + extra
            j = torch.arange(n + extra, device="cuda")
            hidden = j[None] > p[:, None]
            if c.get("window"):
                hidden |= j[None] <= p[:, None] - c["window"]
            for h in range(Hkv):  # the heads that share these keys, together
                x = s["q"][t0:t1, h * G:(h + 1) * G].to(f64).transpose(0, 1) @ k[:, h].T / math.sqrt(D)
                x = c["cap"] * torch.tanh(x / c["cap"]) if c["cap"] else x
                x = x.masked_fill(hidden, -math.inf)
                z = torch.logsumexp(x, 2)
                lse[t0:t1, h * G:(h + 1) * G] = z.T
                out[t0:t1, h * G:(h + 1) * G] = (torch.exp(x - torch.nan_to_num(z, neginf=0.0)[..., None]) @ v[:, h]).transpose(0, 1)
    return out, lse


def _exact_append(c, s):
    """Codes before their rounding, and the scales by comparison with every power of two."""
    P, f64, got = c["page"], torch.float64, {}
    powers = 448.0 * _power64(torch.arange(-126, 121, device="cuda"))
    for x in "kv":
        codes, scale = s[x].to(f64), _power64(s[x + "_exp"].long() - 127)
        for t in range(0, c["T"], 8192):
            slot = s["slot"][t:t + 8192].long()
            keep = torch.nonzero(slot >= 0)[:, 0]
            new, slot = s[x + "_new"][t:t + 8192].to(f64)[keep], slot[keep]
            e = torch.searchsorted(powers, new.abs().amax(-1)) - 126
            codes[slot // P, slot % P] = new / _power64(e)[..., None]
            scale[slot // P, :, slot % P] = _power64(e)
        got |= {x: codes, x + "_scale": scale}
    return got
