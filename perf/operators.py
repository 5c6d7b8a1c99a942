"""The paged-cache operators that a serving step makes of this library, sized over the range they use.

Three operators, in the order of a step:
  plan    pages for the requests' lengths and reservations: block tables, slot map, positions
  append  the new tokens' keys and values into the slots that the plan gave
  attend  attention of each request's new tokens over its pages (one token, or a chunk of a prompt)
Plain forms are elementary torch operations in 32 bits (whole numbers for the plan), rounded once at the end.
"""
import math
import random
from statistics import NormalDist

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
# Most that a drawn attention does: flops, (request, head, row, key) cells of the padded scores, and elements of the
# padded keys.  Each is at or below the largest listed case's.
MOST_FLOPS, MOST_CELLS, MOST_KEYS = 2.0e12, 4.2e9, 5.3e8


def listed():
    return [
        # A small server's step: eight requests, one token each, one of them finished, one admitted.
        {"name": "plan_small", "op": "plan", "B": 8, "page": 16, "max_pages": 512, "n_pages": 96, "new": 1, "admit": 0.125},
        # A large server's step: thousands of requests, a tenth of them admitted with prompts and their reservation.
        {"name": "plan_large", "op": "plan", "B": 4096, "page": 16, "max_pages": 1024, "n_pages": 524288, "new": 2048, "admit": 0.1},
        # The keys and values of one decoding step of 64 requests, one token each, in a layer.
        {"name": "append_decode", "op": "append", "T": 64, "Hkv": 8, "D": 128, "page": 16, "n_pages": 4096, "dt": "bf16", "drop": 0.0},
        # A step of long prompts: an odd number of tokens, read out of the packed projection, some of them refused.
        {"name": "append_prompts", "op": "append", "T": 65539, "Hkv": 8, "D": 128, "page": 32, "n_pages": 4096, "dt": "fp16", "drop": 0.02},
        # One request, one token, a thousand tokens of context: the smallest call, all latency.
        {"name": "decode_one", "op": "attend", "B": 1, "q": 1, "kv": 1000, "mix": "even", "Hq": 32, "Hkv": 8, "D": 128, "page": 16,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # The ordinary decoding step: 64 requests of lognormal lengths, grouped heads.
        {"name": "decode_batch", "op": "attend", "B": 64, "q": 1, "kv": 8192, "mix": "lognormal", "Hq": 32, "Hkv": 8, "D": 128, "page": 16,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # Four agents deep into long contexts: the cache read is split along the keys.
        {"name": "decode_long", "op": "attend", "B": 4, "q": 1, "kv": 131072, "mix": "even", "Hq": 64, "Hkv": 8, "D": 128, "page": 64,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # Every head with keys of its own, short heads, a sliding window that starts inside a page, three drafted tokens.
        {"name": "decode_window", "op": "attend", "B": 48, "q": 3, "kv": 5003, "mix": "lognormal", "Hq": 16, "Hkv": 16, "D": 64, "page": 16,
         "dt": "fp16", "window": 1023, "cap": 0.0},
        # The next 512 tokens of one prompt over 3.6 thousand cached ones.
        {"name": "chunk_one", "op": "attend", "B": 1, "q": 512, "kv": 4099, "mix": "even", "Hq": 32, "Hkv": 8, "D": 128, "page": 16,
         "dt": "bf16", "window": 0, "cap": 0.0},
        # A mixed step: chunks of some prompts beside decoding requests and a refused one (rows without keys), seven heads a group.
        {"name": "chunk_mixed", "op": "attend", "B": 24, "q": 777, "kv": 6007, "mix": "mixed", "Hq": 28, "Hkv": 4, "D": 128, "page": 32,
         "dt": "fp16", "window": 0, "cap": 0.0},
        # Whole prompts with short heads, capped scores and a window.
        {"name": "chunk_capped", "op": "attend", "B": 3, "q": 4001, "kv": 4001, "mix": "lognormal", "Hq": 16, "Hkv": 8, "D": 64, "page": 64,
         "dt": "bf16", "window": 2048, "cap": 30.0},
        # The last 4096 tokens of a prompt of 32768: the largest.
        {"name": "chunk_long", "op": "attend", "B": 1, "q": 4096, "kv": 32768, "mix": "even", "Hq": 32, "Hkv": 8, "D": 128, "page": 64,
         "dt": "bf16", "window": 0, "cap": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attend", "attend", "attend"])
    if op == "plan":
        B, page = _log(rng, 1, 4096), rng.choice([16, 32, 64, 128])
        max_pages = _log(rng, 64, 1024)
        return {"op": op, "B": B, "page": page, "max_pages": max_pages, "n_pages": max(64, B * max_pages // rng.choice([1, 2, 4, 16])),
                "new": min(_log(rng, 1, 2048), max_pages * page // 2), "admit": rng.choice([0.05, 0.1, 0.5])}
    if op == "append":
        T, page = _log(rng, 1, 65539), rng.choice([16, 32, 64, 128])
        return {"op": op, "T": T, "Hkv": rng.choice([1, 2, 4, 8]), "D": rng.choice([64, 128]), "page": page,
                "n_pages": T // page + _log(rng, 2, 2000), "dt": rng.choice(["bf16", "fp16"]), "drop": rng.choice([0.0, 0.02])}
    while True:
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (64, 8), (16, 16), (28, 4), (16, 8), (24, 3), (8, 1)])
        c = {"op": op, "B": _log(rng, 1, 128), "q": rng.choice([1, 1, rng.randint(2, 8), _log(rng, 16, 4096)]), "kv": _log(rng, 16, 131072),
             "mix": rng.choice(["even", "lognormal", "mixed"]), "Hq": Hq, "Hkv": Hkv, "D": rng.choice([64, 128, 128]),
             "page": rng.choice([16, 32, 64, 128]), "dt": rng.choice(["bf16", "fp16"]), "window": rng.choice([0, 0, 0, _log(rng, 16, 8192)]),
             "cap": rng.choice([0.0, 0.0, 0.0, 30.0])}
        c["q"] = min(c["q"], c["kv"])
        if c["B"] * c["q"] * c["Hq"] * c["kv"] <= MOST_CELLS and c["B"] * c["kv"] * c["Hkv"] * c["D"] <= MOST_KEYS and work(c)["flops"] <= MOST_FLOPS:
            return c


def _lengths(c):
    """The (new tokens, tokens with them) of a case's requests: the same for every seed, which only orders them."""
    if c["mix"] == "even":
        return [(c["q"], c["kv"])] * c["B"]
    nd, out = NormalDist(), []
    for i in range(c["B"]):
        # lognormal of sigma 0.8 whose 98th percentile is the longest
        z = nd.inv_cdf((i + 0.5) / c["B"])
        kv = max(1, min(c["kv"], round(c["kv"] * math.exp(0.8 * (z - 2.05)))))
        if i == c["B"] - 1:
            kv = c["kv"]
        q = min(c["q"], kv)
        if c["mix"] == "mixed":
            if i % 6 == 2:  # refused: its tokens have no pages
                q, kv = min(c["q"], 5), 0
            elif i % 6 != 5 and i != c["B"] - 1:
                q = 1
        out.append((q, kv))
    return out


def _seen(c, q, kv):
    """Visible (row, key) pairs of a request, and the keys that any of its rows sees."""
    if kv < 1:
        return 0, 0
    w = c["window"] or kv + q
    p = np.arange(kv - q, kv, dtype=np.int64)
    return int(np.minimum(p + 1, w).sum()), int(kv - max(0, kv - q - w + 1))


def work(c):
    if c["op"] == "plan":
        grown = c["B"] * c["admit"] * min(c["max_pages"], 1 + (c["new"] + 512) / c["page"])  # entries that move, about
        return {"bytes": int(4 * (8 * c["B"] + 2 * 2 * grown + 3 * _tokens(c))), "flops": 0}
    if c["op"] == "append":
        return {"bytes": int(c["T"] * (1 - c["drop"]) * 2 * 2 * c["Hkv"] * c["D"] * 2 + 4 * c["T"]), "flops": 0}
    T, pairs, keys = 0, 0, 0
    for q, kv in _lengths(c):
        p, k = _seen(c, q, kv)
        T, pairs, keys = T + q, pairs + p, keys + k
    return {"bytes": T * c["Hq"] * (2 * c["D"] * 2 + 4) + keys * (c["Hkv"] * c["D"] * 2 * 2 + 4 / c["page"]), "flops": 4 * pairs * c["Hq"] * c["D"]}


def _tokens(c):
    """Room for a plan's new tokens."""
    return c["B"] + int(c["B"] * c["admit"] + 1) * c["new"]


_ctx = None


def _context():
    """The context that a program makes once."""
    global _ctx
    if _ctx is None:
        from paper_2607_16892_gb300 import kvdro as kv
        _ctx = kv.kvdro_create(torch.cuda.current_device())
    return _ctx


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=DT[c["dt"]])

    if c["op"] == "plan":
        s = {k: ints(v) for k, v in _plan_inputs(c, rng).items()}  # a plan deals with page numbers alone
        B, T = c["B"], _tokens(c)
        s |= {"case": c, "held_out": ints(np.zeros(B)), "pool_out": ints(np.zeros(2)), "q_off": ints(np.zeros(B + 1)),
              "kv_len": ints(np.zeros(B)), "slot": ints(np.zeros(T)), "pos": ints(np.zeros(T))}
        return s
    elif c["op"] == "append":
        N = c["n_pages"] * c["page"]
        qkv = normal(c["T"], (4 + 2) * c["Hkv"], c["D"])  # the packed projection: four query heads a group, keys, values
        slot = rng.permutation(N)[:c["T"]]
        slot[rng.random(c["T"]) < c["drop"]] = -1
        k, v = normal(c["n_pages"], c["page"], c["Hkv"], c["D"]), normal(c["n_pages"], c["page"], c["Hkv"], c["D"])
        s = {"case": c, "k": k, "v": v, "k_new": qkv[:, 4 * c["Hkv"]:5 * c["Hkv"]], "v_new": qkv[:, 5 * c["Hkv"]:], "slot": ints(slot)}
    else:
        B, P = c["B"], c["page"]
        lens = _lengths(c)
        lens = [lens[i] for i in rng.permutation(B)]
        q_len, kv_len = np.array([x[0] for x in lens]), np.array([x[1] for x in lens])
        pages = -(-kv_len // P)
        n_pages = int(pages.sum()) + 7
        table = np.full((B, max(1, int(pages.max()))), -1)
        table[np.arange(table.shape[1])[None] < pages[:, None]] = rng.permutation(n_pages)[:int(pages.sum())]
        k, v = normal(n_pages, P, c["Hkv"], c["D"]), normal(n_pages, P, c["Hkv"], c["D"])
        # some channels stand out, as they do in keys and values of trained models
        k += 2 * (torch.rand(c["Hkv"], c["D"], generator=g, device="cuda") < 0.03).to(k.dtype)
        v += 0.5 * normal(c["Hkv"], c["D"])
        some = kv_len > 0  # what nobody wrote yet after a request's last token: anything
        last = ints(table)[torch.from_numpy(np.nonzero(some)[0]).cuda(), ints(pages[some] - 1).long()].long()
        past = torch.arange(P, device="cuda")[None] > ints((kv_len[some] - 1) % P)[:, None]
        for t in (k, v):
            t[last] = t[last].masked_fill_(past[:, :, None, None], float("nan"))
        T = int(q_len.sum())
        qkv = normal(T, c["Hq"] + 2 * c["Hkv"], c["D"])
        s = {"case": c, "k": k, "v": v, "q": qkv[:, :c["Hq"]], "q_off": ints(np.concatenate([[0], np.cumsum(q_len)])), "kv_len": ints(kv_len),
             "table": ints(table), "out": torch.empty((T, c["Hq"], c["D"]), dtype=k.dtype, device="cuda"),
             "lse": torch.empty((T, c["Hq"]), dtype=torch.float32, device="cuda"), "max_q": int(q_len.max()), "max_kv": int(kv_len.max())}
    if own:  # the handle that a program keeps for its cache; the inputs are the same on both sides
        from paper_2607_16892_gb300 import kvdro as kv
        s["cache"] = kv.kvdro_kv_open(_context(), k, v)
    return s


def _plan_inputs(c, rng):
    B, P, mp, n = c["B"], c["page"], c["max_pages"], c["n_pages"]
    cap = mp * P
    admit = np.zeros(B, bool)
    admit[rng.permutation(B)[:int(B * c["admit"] + 1)]] = True
    most = min(cap - c["new"], max(1, (n * P // 2) // B))  # running requests hold half the pages at most
    cached = np.where(admit, 0, np.minimum(1 + (most * rng.random(B) ** 2).astype(np.int64), most))
    new = np.where(admit, 1 + (c["new"] * rng.random(B)).astype(np.int64).clip(0, c["new"] - 1), 1)
    new[~admit & (rng.random(B) < 0.05)] = -1  # finished
    new[~admit & (rng.random(B) < 0.02)] = 0   # waits
    reserve = np.where(admit, new + (512 * rng.random(B)).astype(np.int64), 0)
    held = -(-cached // P)
    owner = rng.permutation(n)
    table = np.full((B, mp), -1)
    table[np.arange(mp)[None] < held[:, None]] = owner[:int(held.sum())]
    free = owner[int(held.sum()):]
    head = int(rng.integers(n))
    ring = np.full(n, -1)
    ring[(head + np.arange(len(free))) % n] = free
    return {"cached": cached, "new_len": new, "reserve": reserve, "held": held, "table": table, "ring": ring, "pool": np.array([head, len(free)])}


def run(s):
    return {"plan": _plan, "append": _append, "attend": _attend}[s["case"]["op"]](s)


def _plan(s):
    c = s["case"]
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_plan(_context(), c["page"], s["cached"], s["new_len"], s["held"], s["table"], s["ring"], s["pool"], s["held_out"], s["pool_out"],
                         s["q_off"], s["kv_len"], s["slot"], s["pos"], reserve=s["reserve"])
        return {k: s[k] for k in ("table", "ring", "held_out", "pool_out", "q_off", "kv_len", "slot", "pos")}
    P, mp, n, T = c["page"], c["max_pages"], c["n_pages"], s["slot"].numel()
    cached, new, held, table, ring = s["cached"].long(), s["new_len"].long(), s["held"].long(), s["table"], s["ring"]
    head, n_free = s["pool"].long().unbind()
    total = cached + new
    fits = total <= mp * P
    want = (torch.maximum(total, s["reserve"].long().clamp(max=mp * P)) + P - 1) // P
    need = torch.where((new > 0) & fits, (want - held).clamp(min=0), 0)
    incl = need.cumsum(0)
    ok = fits & ((need == 0) | (incl <= n_free))
    grow = torch.where(ok, need, 0)
    back = torch.where(new < 0, held, 0)
    first = head + incl - need                # of a request's new pages, in the ring
    back_first = head + n_free + back.cumsum(0) - back
    j = torch.arange(mp, device=table.device)
    mine = (j >= held[:, None]) & (j < (held + grow)[:, None])
    table = torch.where(mine, ring[(first[:, None] + j - held[:, None]) % n], table)
    at = torch.where(j < back[:, None], (back_first[:, None] + j) % n, n)  # the others to a place behind the ring
    ring = torch.cat([ring, ring[:1]]).scatter(0, at.view(-1), table.view(-1))[:n]
    q_len = new.clamp(min=0)
    q_off = torch.cat([q_len.new_zeros(1), q_len.cumsum(0)])
    t = torch.arange(T, device=table.device)
    b = torch.searchsorted(q_off[1:].contiguous(), t, right=True)
    there = b < new.numel()
    b = b.clamp(max=new.numel() - 1)
    pos = cached[b] + t - q_off[b]
    there &= ok[b]
    page = table.long()[b, (pos // P).clamp(0, mp - 1)]
    i32 = torch.int32
    pool_out = torch.stack([(head + grow.sum()) % n, n_free - grow.sum() + back.sum()])
    return {"table": table, "ring": ring, "held_out": torch.where(new < 0, 0, held + grow).to(i32), "pool_out": pool_out.to(i32), "q_off": q_off.to(i32),
            "kv_len": torch.where(ok & (new >= 0), total, 0).to(i32), "slot": torch.where(there, page * P + pos % P, -1).to(i32),
            "pos": torch.where(there, pos, -1).to(i32)}


def _append(s):
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_append(s["cache"], s["k_new"], s["v_new"], s["slot"])
    else:
        keep = s["slot"] >= 0
        slot = s["slot"][keep].long()
        for cache, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
            cache.view(-1, *cache.shape[2:])[slot] = new[keep]
    return s["k"], s["v"]


def _attend(s):
    c = s["case"]
    if own:
        from paper_2607_16892_gb300 import kvdro as kv
        kv.kvdro_kv_attend(s["cache"], s["q"], s["q_off"], s["kv_len"], s["table"], s["out"], lse=s["lse"], scale=c["D"] ** -0.5, causal=True,
                           window=c["window"], softcap=c["cap"], max_q=s["max_q"])
        return s["out"], s["lse"]
    # the requests padded to the longest: one batch of products
    B, P, Hkv, D, dev = c["B"], c["page"], c["Hkv"], c["D"], s["q"].device
    G, Q, S = c["Hq"] // Hkv, s["max_q"], s["max_kv"]
    q_off, kv_len = s["q_off"].long(), s["kv_len"].long()
    q_len = q_off[1:] - q_off[:-1]
    i, j = torch.arange(Q, device=dev), torch.arange(S, device=dev)
    row = (q_off[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().view(B, Q, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, D)
    pages = s["table"].clamp(min=0).long()
    there = (j < kv_len[:, None])[:, :, None, None]
    k = s["k"][pages].view(B, -1, Hkv, D)[:, :S].float().masked_fill_(~there, 0).permute(0, 2, 3, 1)
    v = s["v"][pages].view(B, -1, Hkv, D)[:, :S].float().masked_fill_(~there, 0).transpose(1, 2)
    x = (q @ k).mul_(D ** -0.5).view(B, Hkv, G, Q, S)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    p = (kv_len - q_len)[:, None] + i
    seen = (j <= p[:, :, None]) & (j < kv_len[:, None, None])
    if c["window"]:
        seen &= j > p[:, :, None] - c["window"]
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0, top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = x.view(B, Hkv, G * Q, S) @ v
    out = out.view(B, Hkv, G, Q, D) / torch.where(total == 0, 1, total)
    lse = (top + total.log()).squeeze(-1)
    t = torch.arange(s["q"].shape[0], device=dev)  # back to the packed rows
    b = torch.searchsorted(q_off[1:].contiguous(), t, right=True)
    r = t - q_off[b]
    return out[b, :, :, r].reshape(-1, c["Hq"], D).to(s["q"].dtype), lse[b, :, :, r].reshape(-1, c["Hq"])


def exact(c, seed):
    if c["op"] == "plan":
        return _exact_plan(c, np.random.default_rng(seed))
    global own
    was, own = own, False  # the inputs alone, without the library
    try:
        s = prepare(c, seed)
    finally:
        own = was
    P, Hkv, D, f64 = c["page"], c["Hkv"], c["D"], torch.float64
    if c["op"] == "append":
        k, v = s["k"].to(f64), s["v"].to(f64)
        for t in range(0, c["T"], 4096):  # slot by slot in the cache's own shape
            keep = torch.nonzero(s["slot"][t:t + 4096] >= 0)[:, 0]
            at = s["slot"][t:t + 4096].long()[keep]
            k[at // P, at % P], v[at // P, at % P] = s["k_new"][t + keep].to(f64), s["v_new"][t + keep].to(f64)
        return k, v
    G, T = c["Hq"] // Hkv, s["q"].shape[0]
    out, lse = torch.zeros((T, c["Hq"], D), dtype=f64, device="cuda"), torch.full((T, c["Hq"]), -math.inf, dtype=f64, device="cuda")
    q_off, kv_len = s["q_off"].tolist(), s["kv_len"].tolist()
    for b, n in enumerate(kv_len):
        if n == 0:
            continue
        rows = s["table"][b, :-(-n // P)].long()
        k, v = (s[x][rows].reshape(-1, Hkv, D)[:n].to(f64) for x in "kv")
        for t0 in range(q_off[b], q_off[b + 1], 512):  # a few rows at a time
            t1 = min(t0 + 512, q_off[b + 1])
            p = torch.arange(t0, t1, device="cuda") - q_off[b + 1] + n
            j = torch.arange(n, device="cuda")
            hidden = j[None] > p[:, None]
            if c["window"]:
                hidden |= j[None] <= p[:, None] - c["window"]
            for h in range(c["Hq"]):
                x = s["q"][t0:t1, h].to(f64) @ k[:, h // G].T / math.sqrt(D)
                x = c["cap"] * torch.tanh(x / c["cap"]) if c["cap"] else x
                x = x.masked_fill(hidden, -math.inf)
                z = torch.logsumexp(x, 1)
                lse[t0:t1, h] = z
                out[t0:t1, h] = torch.exp(x - torch.nan_to_num(z, neginf=0.0)[:, None]) @ v[:, h // G]
    return out, lse


def _exact_plan(c, rng):
    i = _plan_inputs(c, rng)
    P, mp, n = c["page"], c["max_pages"], c["n_pages"]
    table, ring, held = i["table"].copy(), i["ring"].copy(), i["held"].copy()
    head, free = (int(x) for x in i["pool"])
    start, left, tail, taken = head, free, head + free, 0
    kv_len, q_off = np.zeros(c["B"], np.int64), np.zeros(c["B"] + 1, np.int64)
    slot, pos = np.full(_tokens(c), -1), np.full(_tokens(c), -1)
    back, given = [], 0
    for b in range(c["B"]):
        new, have = int(i["new_len"][b]), int(i["held"][b])
        q_off[b + 1] = q_off[b] + max(new, 0)
        total = int(i["cached"][b]) + new
        if new < 0:
            back += [int(x) for x in table[b, :have]]
            held[b] = 0
            continue
        if total > mp * P:
            continue
        if new > 0:
            want = max(total, min(int(i["reserve"][b]), mp * P))
            need = max(0, -(-want // P) - have)
            given += need
            if need and given > left:
                continue
            for x in range(need):
                table[b, have + x] = ring[(start + taken + x) % n]
            taken += need
            held[b] = have + need
            p = np.arange(total - new, total)
            slot[q_off[b]:q_off[b + 1]] = table[b, p // P] * P + p % P
            pos[q_off[b]:q_off[b + 1]] = p
        kv_len[b] = total
    for x, page in enumerate(back):
        ring[(tail + x) % n] = page
    return {"table": table, "ring": ring, "held_out": held, "pool_out": np.array([(start + taken) % n, left - taken + len(back)]), "q_off": q_off,
            "kv_len": kv_len, "slot": slot, "pos": pos}
