"""A small server on the page cache: reservations from the cost evaluation, pages, writes and attention per step.

Requests of several classes arrive with prompts of L_in tokens and output lengths drawn from their class.  The
reservation r of a class is the one that the exact worst case over the Wasserstein ball picks (``kvdro_eval_dual``)
from the class's past output lengths, as the paper's reservation block does once per re-optimisation (Alg. 1).  Every step
then is
    kvdro_kv_plan     pages for what is admitted (its reservation) and for what grew past its own; finished
                      requests give theirs back; a request that finds no pages is refused and tries again
    kvdro_kv_append   the new tokens' keys and values, per layer
    kvdro_kv_attend   whole prompts and single tokens in one batch, per layer
There is no model here: queries, keys and values are seeded draws of a model's shapes.  The host reads back the
lengths of a step (which requests were refused) and nothing else.

    python -m paper_2607_16892_gb300.serving_loop --steps 200
"""

from __future__ import annotations

import argparse
import json
import time

import numpy as np

from . import kvdro as kv

MEDIAN_OUT, SIGMA_OUT, L_MAX = (60, 200, 500), 0.8, 4096


def reservations(ctx, rng, rho: float, eps: float, prompts, samples_per_class: int = 2000) -> np.ndarray:
    """Tokens to reserve per class, prompt included: the argmin of the exact worst-case cost over r."""
    K = len(prompts)
    draws = [np.clip(np.rint(m * np.exp(SIGMA_OUT * rng.standard_normal(samples_per_class))), 1, L_MAX) for m in MEDIAN_OUT[:K]]
    offsets = np.arange(K + 1, dtype=np.int64) * samples_per_class
    L_max, zero = np.full(K, L_MAX, np.int32), np.zeros(K, np.int32)
    kv.kvdro_load_samples(ctx, K, offsets, np.concatenate(draws).astype(np.int32), L_max, zero)
    r = np.arange(0, L_MAX + 1, 8, dtype=np.int32)
    r_idx = np.empty((1, 1, K), np.int32)
    kv.kvdro_eval_dual(ctx, len(r), r, 1, [eps], 1, [rho], [1.0], r_idx=r_idx)
    return r[r_idx[0, 0]] + np.asarray(prompts)  # the reservation of the output, behind the prompt


def run(steps: int = 200, slots: int = 32, pages: int = 1200, page_size: int = 16, layers: int = 2, heads: int = 32,
        kv_heads: int = 8, head_dim: int = 128, prompts=(37, 200, 801), rho: float = 10.0, eps: float = 20.0, arrival: float = 0.3,
        seed: int = 1, device: int = 0, watch=None) -> dict:
    """Serve ``steps`` steps; returns counts.  ``watch(step, layer, state)`` sees each layer's tensors after its attention."""
    import torch

    dev = torch.device("cuda", device)
    torch.cuda.set_device(dev)
    stream = torch.cuda.current_stream(dev)
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)
    ctx = kv.kvdro_create(device)
    i32 = dict(dtype=torch.int32, device=dev)
    try:
        reserve_of = reservations(ctx, rng, rho, eps, prompts)
        shape = (pages, page_size, kv_heads, head_dim)
        caches = [kv.kvdro_kv_open(ctx, torch.empty(shape, dtype=torch.bfloat16, device=dev),
                                   torch.empty(shape, dtype=torch.bfloat16, device=dev)) for _ in range(layers)]
        max_pages = -(-(max(prompts) + L_MAX) // page_size)
        table = torch.full((slots, max_pages), -1, **i32)
        ring = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        pool, pool_next = torch.tensor([0, pages], **i32), torch.empty(2, **i32)
        held, held_next = torch.zeros(slots, **i32), torch.empty(slots, **i32)
        q_off, kv_len = torch.empty(slots + 1, **i32), torch.empty(slots, **i32)
        cls, cached, left = np.full(slots, -1), np.zeros(slots, np.int64), np.zeros(slots, np.int64)
        reserve = np.zeros(slots, np.int64)
        stats = {"admitted": 0, "finished": 0, "refused_new": 0, "refused_running": 0, "tokens": 0, "steps": steps,
                 "reservations": [int(x) for x in reserve_of]}
        t0 = time.perf_counter()
        for step in range(steps):
            for b in np.nonzero(cls < 0)[0]:
                if rng.random() < arrival:
                    cls[b] = rng.integers(len(prompts))
                    cached[b], reserve[b] = 0, reserve_of[cls[b]]
                    left[b] = int(np.clip(np.rint(MEDIAN_OUT[cls[b]] * np.exp(SIGMA_OUT * rng.standard_normal())), 1, L_MAX))
            running = cls >= 0
            fresh = running & (cached == 0)
            done = running & (left == 0)
            new = np.where(done, -1, np.where(fresh, np.asarray(prompts)[cls], np.where(running, 1, 0)))
            T = int(np.maximum(new, 0).sum())
            d_cached, d_new, d_reserve = torch.from_numpy(np.stack([cached, new, reserve]).astype(np.int32)).to(dev).unbind()
            slot, pos = torch.empty(T, **i32), torch.empty(T, **i32)
            kv.kvdro_kv_plan(ctx, page_size, d_cached, d_new, held, table, ring, pool, held_next, pool_next, q_off, kv_len, slot, pos,
                             reserve=d_reserve, stream=stream)
            held, held_next, pool, pool_next = held_next, held, pool_next, pool
            for layer, cache in enumerate(caches):
                if T == 0:
                    break
                qkv = torch.randn((T, heads + 2 * kv_heads, head_dim), generator=gen, device=dev, dtype=torch.bfloat16)
                q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=1)
                out = torch.empty((T, heads, head_dim), dtype=torch.bfloat16, device=dev)
                kv.kvdro_kv_append(cache, k, v, slot, stream=stream)
                kv.kvdro_kv_attend(cache, q, q_off, kv_len, table, out, max_q=int(new.max()), stream=stream)
                if watch is not None:
                    watch(step, layer, {"q": q, "k": k, "v": v, "out": out, "new": new, "cls": cls.copy(), "kv_len": kv_len, "pos": pos})
            got = kv_len.cpu().numpy()  # 0: refused, done or empty
            kv.kvdro_sync(ctx)
            ok = running & ~done & (got > 0)
            stats["admitted"] += int((ok & fresh).sum())
            stats["refused_new"] += int((running & fresh & ~ok).sum())
            stats["refused_running"] += int((running & ~fresh & ~done & ~ok).sum())
            stats["finished"] += int(done.sum())
            stats["tokens"] += int(np.maximum(new, 0)[ok].sum())
            cached[ok] = got[ok]
            left[ok] -= 1
            cls[done] = -1
            cached[done] = 0
        stats["free_pages"] = int(pool[1])
        stats["held_pages"] = int(held.sum())
        stats["pages"] = pages
        stats["wall_s"] = time.perf_counter() - t0
        return stats
    finally:
        kv.kvdro_destroy(ctx)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--slots", type=int, default=32)
    p.add_argument("--pages", type=int, default=1200)
    p.add_argument("--rho", type=float, default=10.0)
    p.add_argument("--eps", type=float, default=20.0)
    p.add_argument("--device", type=int, default=0)
    a = p.parse_args()
    print(json.dumps(run(a.steps, a.slots, a.pages, rho=a.rho, eps=a.eps, device=a.device)))


if __name__ == "__main__":
    main()
